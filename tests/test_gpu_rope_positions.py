"""Rotary positions near and far: a row's tolerance grows with its own position alone."""
import numpy as np
import pytest
import torch

from oracle import serving as OS
from test_gpu_serving import DT, SCALINGS, _np, _rope_tol

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2608_28003_gb300 import build
    build.build()
    from paper_2608_28003_gb300 import binding
    return binding


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("rot,inter,scaling", [(256, False, "none"), (128, True, "linear"), (64, False, "wavelength"), (48, True, "parts")])
def test_rows_of_all_positions(B, dt, rot, inter, scaling):
    """An angle of |p| f radians is off by |p| f 2^-49 in the table (a double's frequencies, 2^-52 turns) and as much in the
    oracle's, whose product is a double: 2^-48 |p| of the pair's magnitude, beside the rotation's own error."""
    pos = torch.tensor([0, 1, -1, 2, 3, 7, 63, 64, 1000, -4095, 32768, 1 << 20, -(1 << 24) - 1, (1 << 30) + 3, (1 << 31) - 1,
                        -(1 << 31)], dtype=torch.int32, device="cuda")
    x = torch.randn(len(pos), 3, rot + 16 if rot < 256 else rot, device="cuda", generator=torch.Generator("cuda").manual_seed(rot)).to(DT[dt])
    table = B.rope_table(B.RopeConfig(rot, base=5e5, interleaved=inter, scaling=scaling, **SCALINGS[scaling]))
    f, s = OS.rope_frequencies(rot, 5e5, scaling, **SCALINGS[scaling])
    want = OS.rope(_np(x), _np(pos), f, s, inter)
    slack = np.abs(_np(pos))[:, None, None] * 2.0 ** -48 * s * 2 ** 0.5 * np.abs(_np(x)).max()
    assert (np.abs(_np(B.rope(table, x, pos)) - want) <= _rope_tol(want, _np(x), DT[dt], s) + slack).all()
