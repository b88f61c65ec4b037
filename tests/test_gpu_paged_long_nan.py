"""A sequence of NaN so long that computing its rows again takes longer than a wait's limit: the copies and products that wait
for them meanwhile are not taken for lost."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2608_28003_gb300 import build
    build.build()
    from paper_2608_28003_gb300 import binding
    return binding


@pytest.mark.parametrize("dim,new,keys", [(256, 32, 240000), (128, 64, 280000)])
def test_the_limit_of_a_wait_is_not_a_rows(B, dim, new, keys):
    """About 2.7 s for the rows of one sequence (11 and 9.7 us a key for the 32 rows of a warp) in the middle of the items of one
    CTA, whose limit is 2 s; every sequence has the same page, all ones, again and again."""
    seqs, n_q, page = 400, 4, 256
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    k = torch.zeros(2, page, 1, dim, device="cuda", dtype=torch.bfloat16)
    v = torch.ones_like(k)
    v[1, 3, 0, 5] = float("nan")
    pages = torch.zeros(seqs, -(-keys // page), dtype=torch.int32, device="cuda")
    bad = 201  # items of a CTA: 2.6, this one whole
    pages[bad, 0] = 1
    batch = B.PagedBatch(i32([i * new for i in range(seqs + 1)]), i32([keys] * seqs), pages, max_new=new)
    q = torch.randn(seqs * new, n_q, dim, device="cuda").bfloat16()
    B.paged_attention_check()
    out = B.paged_attention(B.PagedCache(k, v), batch, q).view(seqs, new, n_q, dim)
    B.paged_attention_check()
    assert bool(torch.isnan(out[bad, ..., 5]).all())
    out[bad, ..., 5] = 1.0
    assert bool((out == 1).all())
