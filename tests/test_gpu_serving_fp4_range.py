"""Attention over a 4-bit cache whose scores are ordinary numbers, of queries, exponents and scales that are not."""
import math

import pytest
import torch

from test_gpu_serving_fp4 import DT, _gen, attn_check, fp4_batch, objects, refresh

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2608_28003_gb300 import build
    build.build()
    from paper_2608_28003_gb300 import binding
    return binding


@pytest.mark.parametrize("new,n_q,n_kv,dim", [([1, 2], 8, 2, 64), ([1, 1], 4, 1, 256), ([40, 130], 8, 2, 128), ([50, 90], 4, 1, 256),
                                              ([30, 1, 60], 6, 3, 64)])
@pytest.mark.parametrize("k_exp,up", [(-100, 118), (-60, 118), (100, -120), (90, -100)])
def test_far_exponents(B, new, n_q, n_kv, dim, k_exp, up):
    """Queries 2^up, keys 2^(k_exp + 8), and a scale that brings their products back: a query times codes alone (2^134), or the scale times
    2^k_exp alone (2^109 to 2^120, times log2 e and codes), can lie beyond fp32, a query times a key does not."""
    b = fp4_batch(new, [100, 190, 77][:len(new)], 16, n_kv, dim, 5, exps=(-8, 0))
    b["exps"] = (k_exp, 0)
    refresh(b)
    q = (torch.randn(b["n_rows"], n_q, dim, device="cuda", generator=_gen(8)) * 2.0 ** up).bfloat16()
    cache, batch = objects(B, b)
    scale = 0.1 * 2.0 ** -(up + k_exp + 8)
    assert 0 < scale < 3e38
    attn_check(B.fp4_paged_attention(cache, batch, q, scale=scale), q, b, scale, 0)


@pytest.mark.parametrize("new,n_q,n_kv,dim", [([1, 2], 8, 2, 64), ([1, 1], 4, 1, 256), ([40, 130], 8, 2, 128), ([50, 90], 4, 1, 256),
                                              ([30, 1, 60], 6, 3, 64)])
@pytest.mark.parametrize("k_exp,up", [(100, 18), (100, 14), (80, 38), (10, 108), (0, 118), (-100, 118)])
def test_products_beyond_the_type_that_the_scale_brings_back(B, new, n_q, n_kv, dim, k_exp, up):
    """Queries times keys around 2^(k_exp + up + 12), up to 2^132, and scores around 64 of which few keys of a row are near the top."""
    b = fp4_batch(new, [100, 190, 77][:len(new)], 16, n_kv, dim, 5, exps=(-8, 0))
    b["exps"] = (k_exp, 0)
    refresh(b)
    q = (torch.randn(b["n_rows"], n_q, dim, device="cuda", generator=_gen(8)) * 2.0 ** up).bfloat16()
    cache, batch = objects(B, b)
    scale = 4.0 * 2.0 ** -(up + k_exp + 8)
    assert 2.0 ** -126 <= scale
    attn_check(B.fp4_paged_attention(cache, batch, q, scale=scale), q, b, scale, 0)


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("new,n_q,n_kv,dim", [([1, 2], 8, 2, 64), ([1, 1], 4, 1, 256), ([40, 130], 8, 2, 128), ([50, 90], 4, 1, 256)])
@pytest.mark.parametrize("scale", [5 * 2.0 ** -147, 2.0 ** -149, 3 * 2.0 ** -130, 1.5 * 2.0 ** 127])
def test_scales_at_the_ends_of_the_type(B, dt, new, n_q, n_kv, dim, scale):
    """A scale below fp32's normal numbers has few bits, which log2 e must not cost it any of; one at the other end times log2 e is none."""
    b = fp4_batch(new, [100, 190], 16, n_kv, dim, 5, exps=(-8, 0))
    k_exp = 100 if scale < 1 else -100
    up = round(-math.log2(scale)) - k_exp - 8  # scores of a few units
    if dt == "f16":
        up = max(-10, min(up, 12))
    b["exps"] = (k_exp, 0)
    refresh(b)
    q = (torch.randn(b["n_rows"], n_q, dim, device="cuda", generator=_gen(8)) * 2.0 ** up).to(DT[dt])
    cache, batch = objects(B, b)
    attn_check(B.fp4_paged_attention(cache, batch, q, scale=scale), q, b, scale, 0)


@pytest.mark.parametrize("new,n_q,n_kv,dim", [([1, 2], 8, 2, 64), ([40, 130], 8, 2, 128), ([50, 90], 4, 1, 256)])
def test_a_scale_beyond_the_type_with_the_exponent(B, new, n_q, n_kv, dim):
    """scale 2^k_exp = 2^130 is no fp32 number, the scores are."""
    b = fp4_batch(new, [100, 190], 16, n_kv, dim, 5, exps=(0, 0))
    b["exps"] = (100, 0)
    refresh(b)
    q = (torch.randn(b["n_rows"], n_q, dim, device="cuda", generator=_gen(8)) * 2.0 ** -124).bfloat16()
    q = torch.where(q.abs() < 2.0 ** -126, torch.zeros_like(q), q)  # normal numbers
    cache, batch = objects(B, b)
    attn_check(B.fp4_paged_attention(cache, batch, q, scale=2.0 ** 30), q, b, 2.0 ** 30, 0)


@pytest.mark.parametrize("keys,new", [(2, 20), (3, 40), (5, 100)])
@pytest.mark.parametrize("up", [115, 116, 117])
def test_few_keys_of_which_some_lie_far_below(B, keys, new, up):
    """Rows with a handful of keys whose products with codes alone lie around fp32's end, and below it more often than above in some
    rows: a weight that is e^-2 must not vanish."""
    seqs = 24
    b = fp4_batch([new] * seqs, [new + keys] * seqs, 16, 1, 128, 9, exps=(-8, 0))
    b["exps"] = (-100, 0)
    refresh(b)
    q = (torch.randn(b["n_rows"], 4, 128, device="cuda", generator=_gen(8)) * 2.0 ** up).bfloat16()
    cache, batch = objects(B, b)
    scale = 0.1 * 2.0 ** (92 - up)
    attn_check(B.fp4_paged_attention(cache, batch, q, scale=scale, window=keys), q, b, scale, keys)
