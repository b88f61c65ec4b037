"""The 4-bit linear into views of wider tensors: what lies beside a view stays as it was, whatever the rows' ends are."""
import pytest
import torch

from test_gpu_fp4 import DT, _gen

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2608_28003_gb300 import build
    build.build()
    from paper_2608_28003_gb300 import binding
    return binding


@pytest.mark.parametrize("out", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("m,k", [(1, 64), (40, 2304), (49, 64), (129, 288), (300, 4608), (2048, 64)])
@pytest.mark.parametrize("n", [1, 7, 31, 63, 127, 129, 190, 191, 193, 1150, 1156])
def test_columns_beside_a_view(B, m, k, n, out):
    g = _gen(n)
    w = B.fp4_quantize(torch.randn(n, k, device="cuda", generator=g).bfloat16())
    x = torch.randn(m, k, device="cuda", generator=g).bfloat16()
    bias = torch.randn(n, device="cuda", generator=g)
    want = B.fp4_linear(w, x, bias, dtype=DT[out], out=torch.empty(m, n, device="cuda", dtype=DT[out]))
    for pad in {-n % 8, -n % 8 + 8, -n % 4 + 4, 3, 8}:  # rows that begin on 16 bytes and others
        for off in (0, 8):
            wide = torch.full((m + 1, off + n + pad), 9.0, device="cuda", dtype=DT[out])
            got = B.fp4_linear(w, x, bias, out=wide[:m, off:off + n])
            assert torch.equal(got, want)
            wide[:m, off:off + n] = 9
            assert bool((wide == 9).all()), (pad, off, (wide != 9).nonzero()[:4].tolist())
