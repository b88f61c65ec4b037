"""The 4-bit append under rotary tables with factors on cos and sin: codes and scales are those of exact arithmetic."""
import dataclasses

import numpy as np
import pytest
import torch

from oracle import fp4 as O4
from oracle import serving as OS
from test_gpu_serving_fp4 import _gen, _np

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2608_28003_gb300 import build
    build.build()
    from paper_2608_28003_gb300 import binding
    return binding


@pytest.mark.parametrize("dim,rot,inter,norm", [(256, 256, False, False), (128, 128, True, True), (64, 32, False, True)])
@pytest.mark.parametrize("factor,k_exp", [(1.3862944, 0), (0.01, -4), (60.0, 2), (-1.0, 0), (-60.0, 2), (-3000.0, 8)])
def test_factors(B, dim, rot, inter, norm, factor, k_exp):
    """Some million values each, so that a bound on their error that is too small shows."""
    T, n_kv, page = 2000, 8, 256
    n = -(-T // page)
    cache = B.paged_cache_fp4(n, page, n_kv, dim, k_exp=k_exp)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    batch = B.PagedBatch(i32([0, T]), i32([T]), torch.arange(n, device="cuda", dtype=torch.int32)[None], max_new=T)
    x = (torch.randn(T, 1 + 2 * n_kv, dim, device="cuda", generator=_gen(5)) * 3).bfloat16()
    w = 1 + 0.3 * torch.randn(dim, device="cuda", generator=_gen(6)) if norm else None
    table = dataclasses.replace(B.rope_table(B.RopeConfig(rot, base=1e4, interleaved=inter)), scale=factor)
    B.fp4_rope_append(table, cache, batch, x[:, :1], x[:, 1:1 + n_kv], x[:, 1 + n_kv:], k_norm=w, eps=2.0 ** -17)
    f, _ = OS.rope_frequencies(rot, 1e4)
    k = OS.rms_norm(_np(x[:, 1:1 + n_kv]), None if w is None else _np(w), 2.0 ** -17)
    y = OS.rope(k, range(T), f, float(np.float32(factor)), inter)
    c, s = O4.cache_quantise(y, k_exp)
    codes, scales = (t.transpose(1, 2).reshape(-1, page, n_kv, t.shape[-1]).reshape(n * page, n_kv, -1)[:T].cpu().numpy()
                     for t in (cache.k.transpose(1, 2), cache.k_scales.transpose(1, 2)))
    np.testing.assert_array_equal(scales, s)
    np.testing.assert_array_equal(O4.values_of(O4.unpack(codes)), O4.values_of(c))
