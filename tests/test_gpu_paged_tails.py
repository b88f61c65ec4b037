"""Paged attention over one dominant key and a long tail of small weights: a weight of 2^-25 of the largest is below half of
fp16's smallest step, and tens of thousands of them make up more than a step of the output."""
import numpy as np
import pytest
import torch

from test_gpu_serving import DT, attn_check, objects

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2608_28003_gb300 import build
    build.build()
    from paper_2608_28003_gb300 import binding
    return binding


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("dim,n_q,new", [(64, 4, 1), (128, 4, 4), (256, 4, 1), (64, 8, 20), (128, 4, 70), (256, 4, 40)])
@pytest.mark.parametrize("bits,at", [(25.5, 0), (25.5, 20011), (12.0, 5)])
@pytest.mark.parametrize("first", [0.0, 0.25])
def test_a_dominant_key_and_a_long_tail(B, dt, dim, n_q, new, bits, at, first):
    """Enough sequences over the same pages that a CTA has all keys of a row, so that the tail meets the dominant key's
    reference.  The tolerance is that of every test of attention: relative to the weighted values, so that with a dominant
    value of zero it is the tail's own."""
    keys, page, seqs = 40000, 64, 170
    gen = torch.Generator("cuda").manual_seed(dim)
    pages = keys // page
    k = torch.randn(pages, page, 1, dim, device="cuda", generator=gen) * 0.02
    v = 1.0 + 0.3 * torch.randn(pages, page, 1, dim, device="cuda", generator=gen)
    k[..., 0] = 0.0
    k[at // page, at % page, 0] = 0.0
    k[at // page, at % page, 0, 0] = 8.0
    v[at // page, at % page] = first
    q = torch.randn(seqs * new, n_q, dim, device="cuda", generator=gen)
    q[..., 0] = bits * np.log(2.0) / 8.0 * dim ** 0.5  # the dominant score is bits ln 2 above the tail's
    b = dict(k=k.to(DT[dt]), v=v.to(DT[dt]), row_start=(np.arange(seqs + 1) * new).astype(np.int32),
             kv_len=np.full(seqs, keys, np.int32), pages=np.tile(np.arange(pages, dtype=np.int32), (seqs, 1)),
             n_rows=seqs * new, max_new=new)
    cache, batch = objects(B, b)
    q = q.to(DT[dt])
    attn_check(B.paged_attention(cache, batch, q), q, b, dim ** -0.5, 0, {0, seqs * new - 1})
