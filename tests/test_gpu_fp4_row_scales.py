"""Matrices in 4 bits whose rows' scales are no powers of two, read back: every value rounded once to the type."""
import numpy as np
import pytest
import torch

from oracle import fp4 as O4

pytestmark = pytest.mark.gpu

# what a 16-bit type keeps: significant bits, the exponent of its smallest normal number, its largest number
TYPES = {torch.bfloat16: (8, -126, (2 - 2.0 ** -7) * 2.0 ** 127), torch.float16: (11, -14, 65504.0)}


@pytest.fixture(scope="module")
def B():
    from paper_2608_28003_gb300 import build
    build.build()
    from paper_2608_28003_gb300 import binding
    return binding


def rounded(x, dtype):
    """x (doubles with at most 30 significant bits, so that the quotient by a power of two is exact) rounded once to the type."""
    bits, least, most = TYPES[dtype]
    e = np.frexp(np.where(np.isfinite(x), x, 0.0))[1] - 1  # of 0: -1, any will do
    step = np.ldexp(1.0, np.maximum(e, least) - bits + 1)
    y = np.rint(x / step) * step
    return np.where(np.abs(y) > most, np.copysign(np.inf, x), y)


def test_rounding_of_the_test_itself():
    x = np.random.default_rng(1).integers(0, 1 << 32, 20000, dtype=np.uint64).astype(np.uint32).view(np.float32)
    x = x[np.isfinite(x)]
    for dtype in TYPES:
        with np.errstate(over="ignore"):
            want = torch.from_numpy(x.copy()).to(dtype).double().numpy()  # from fp32: one rounding
        np.testing.assert_array_equal(rounded(x.astype(np.float64), dtype), want)


SCALES = [float.fromhex("0x1.56aaacp-2"), 0.03387920558452606, -float.fromhex("0x1.56aaacp-2"), 1.0, -0.25, 3.0, 0.0, 2.0 ** -126,
          2.0 ** -127, 2.0 ** -149, 3 * 2.0 ** -149, float.fromhex("0x1.fffffep-127"), float.fromhex("0x1.000002p-126"),
          float.fromhex("0x1.49b13ap-1"), float.fromhex("0x1.806db6p-2"), float.fromhex("0x1.56aaacp-128"), float.fromhex("0x1.fffffep+127"), float.fromhex("0x1.56aaacp+118"), 24.5, 1 / 3]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
def test_dequantised_values_are_rounded_once(B, dtype):
    """Every code under every scale byte, of rows with scales of many kinds (a code times its block's scale has six significant bits, a
    row's scale 24: the product is a double exactly)."""
    rng = np.random.default_rng(2)
    some = np.ldexp(1 + rng.integers(0, 1 << 23, 400) / (1 << 23), rng.integers(-30, 20, 400))
    row = np.concatenate([SCALES, some]).astype(np.float32)
    codes = np.tile(np.arange(16, dtype=np.uint8), (len(row), 128))
    scale = np.tile(np.arange(128, dtype=np.uint8), (len(row), 1))
    q = B.fp4_tensor(torch.from_numpy(O4.pack(codes)).cuda(), torch.from_numpy(scale).cuda(), torch.from_numpy(row).cuda())
    exact = O4.dequantise(codes, scale, row, 16)
    if dtype == torch.float32:
        with np.errstate(over="ignore"):
            want = exact.astype(np.float32).astype(np.float64)
    else:
        want = rounded(exact, dtype)
    got = B.fp4_dequantize(q, dtype).double().cpu().numpy()
    np.testing.assert_array_equal(got, want)
    assert np.isnan(got[:, -16:]).all() and not np.isnan(got[:, :-16]).any()
