"""Quantisation to 4 bits of matrices large enough to fill the GPU more than once, bit for bit: a lane has several units of a row there."""
import pytest
import torch

from test_gpu_fp4 import DT, _check_linear, _check_matrix, _np, _rows

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


@pytest.mark.parametrize("block", [16, 32])
def test_more_than_two_gigabytes_of_scales(B, block):
    """Rows whose scales, or codes, 32 bits do not count (all rows of the matrix are the same memory)."""
    k = 65536
    rows = (524289 if block == 16 else 1048577) + 511
    if torch.cuda.mem_get_info()[0] < 100 << 30:
        pytest.skip("needs 100 GB")
    x = torch.randn(1, k, device="cuda", generator=torch.Generator("cuda").manual_seed(1)).bfloat16()
    q, one = B.fp4_quantize(x.expand(rows, k), block), B.fp4_quantize(x, block)
    assert q.scales.numel() > 1 << 31
    for r in (0, 127, 128, 65535, 65536, rows - 129, rows - 1):
        at = B.Fp4Tensor(q.codes[r:r + 1], q.scales.view(-1, one.scales.numel())[r // 128].roll(-(r % 128 % 32 * 16 + r % 128 // 32 * 4)),
                         None if block == 32 else q.row_scale[r:r + 1], block)
        assert torch.equal(at.codes, one.codes) and torch.equal(at.block_scales(), one.block_scales())
    t = torch.randn(3, k, device="cuda", generator=torch.Generator("cuda").manual_seed(2)).bfloat16()
    got = B.fp4_linear(q, t)
    assert got.shape == (3, rows) and bool((got == got[:, :1]).all())
    tv, wv = (_np(B.fp4_dequantize(a, torch.float32)) for a in (B.fp4_quantize(t, block), one))
    _check_linear(got[:, :1], tv, wv, None, k)
