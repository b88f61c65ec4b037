"""Quantisation to 4 bits of matrices large enough to fill the GPU more than once, bit for bit: a lane has several units of a row there."""
import pytest
import torch

from test_gpu_fp4 import DT, _check_matrix, _rows

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2608_28003_gb300 import build
    build.build()
    from paper_2608_28003_gb300 import binding
    return binding


@pytest.mark.parametrize("block", [16, 32])
@pytest.mark.parametrize("dt", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows,k", [(4901, 1024), (4501, 1152), (2441, 2080), (1025, 6912), (129, 40000)])
def test_quantise(B, rows, k, dt, block):
    """Rows of 64 (a warp's, of any type), 72 (a warp's, of 16 bits), 130, 432 and 2500 units, each above 2048 units an SM."""
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    assert rows * (k // 16) >= sms * 2048
    x = _rows(rows, k, dt, rows + k, 1.0 if dt == "f16" else 3.0)
    x[5, 40] = float("nan")
    q = B.fp4_quantize(x, block)
    want = torch.from_numpy(_check_matrix(q, x, block)).cuda()
    same = lambda a, b: bool(((a == b) | (a.isnan() & b.isnan())).all())  # noqa: E731
    assert same(B.fp4_dequantize(q, torch.float32).double(), want)
    if dt != "f32":
        assert same(B.fp4_dequantize(q, DT[dt]).double(), want)
