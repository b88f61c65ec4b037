"""Calls at the edge of what the serving operators' documentation allows."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2608_28003_gb300 import build
    build.build()
    from paper_2608_28003_gb300 import binding
    return binding


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("dim", [64, 256])
def test_a_page_table_without_columns(B, dim, new):
    """Sequences that have no page yet: rows at negative positions see no keys and write none."""
    k = torch.full((2, 16, 1, dim), 3.0, device="cuda", dtype=torch.bfloat16)
    cache = B.PagedCache(k, k.clone())
    batch = B.PagedBatch(_i32([0, new, 2 * new]), _i32([new, 5]), torch.empty(2, 0, dtype=torch.int32, device="cuda"), max_new=new)
    x = torch.randn(2 * new, 6, dim, device="cuda").bfloat16()
    table = B.rope_table(B.RopeConfig(dim))
    q = B.rope_append(table, cache, batch, x[:, :4], x[:, 4:5], x[:, 5:])
    pos = torch.arange(new, device="cuda", dtype=torch.int32).repeat(2) - new
    assert torch.equal(q, B.rope(table, x[:, :4], pos))
    assert bool((cache.k == 3).all()) and bool((cache.v == 3).all())
    assert bool((B.paged_attention(cache, batch, q) == 0).all())
