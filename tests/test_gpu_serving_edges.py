"""Calls at the edge of what the serving operators' documentation allows."""
import pytest
import torch

import synth

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


@pytest.mark.parametrize("base", [float("inf"), 1.0, 0.5])
def test_a_decoder_whose_rope_base_the_paged_step_refuses(B, base):
    """Such a model is made, and its own cache's calls run, as they did before there was a paged step."""
    _, bf, norms = synth.decoder_weights(1, 1152, 256, 512, n_q=4, n_kv=1, seed=2)
    w = {k: [t.cuda() for t in v] if isinstance(v, list) else v.cuda() for k, v in bf.items()}
    n = {k: [torch.from_numpy(a).cuda() for a in v] if isinstance(v, list) else torch.from_numpy(v).cuda()
         for k, v in norms.items()}
    dec = B.Decoder(B.DecoderConfig(max_batch=1, max_seq=64, max_tokens=64, layers=1, inter=256, vocab=512, window=64,
                                    global_layers=(), rope_local=base), w, n)
    toks = torch.arange(12, dtype=torch.int32, device="cuda").view(1, 12)
    assert bool(torch.isfinite(dec.forward(toks, 0)[0]).all())
    k = torch.zeros(1, 1, 16, 1, 256, device="cuda", dtype=torch.bfloat16)
    with pytest.raises(B.W8A8Error) as e:
        dec.step_paged(toks[0], k, k.clone(), B.PagedBatch(_i32([0, 12]), _i32([12]), _i32([[0]]), max_new=12))
    assert e.value.status == 5


def test_numbers_beyond_32_bits_are_refused(B):
    """They were cut to their lower half: one row of 2^32 + 1 was sampled, and the other tokens left unwritten."""
    n = (1 << 32) + 1
    logits, u = torch.zeros(1, 8, device="cuda").expand(n, 8), torch.empty(n, device="cuda")
    with pytest.raises(ValueError, match="32 bits"):
        B.sample(logits, u)
    del u
    k = torch.zeros(1, 16, 1, 64, device="cuda", dtype=torch.bfloat16)
    batch = B.PagedBatch(_i32([0, 2]), _i32([2]), _i32([[0]]), max_new=n)
    q = torch.zeros(2, 4, 64, device="cuda", dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="32 bits"):
        B.paged_attention(B.PagedCache(k, k), batch, q)
    with pytest.raises(ValueError, match="32 bits"):
        batch.c(2)


@pytest.mark.parametrize("hint", [1, 40])  # either kernel
@pytest.mark.parametrize("new", [1, 3, 40])
def test_a_decoder_without_a_window_and_rows_at_negative_positions(B, new, hint):
    """A window of 2^31 - 1 is none, also for sequences that have more rows than keys."""
    _, bf, norms = synth.decoder_weights(1, 1152, 256, 512, n_q=4, n_kv=1, seed=2)
    w = {k: [t.cuda() for t in v] if isinstance(v, list) else v.cuda() for k, v in bf.items()}
    n = {k: [torch.from_numpy(a).cuda() for a in v] if isinstance(v, list) else torch.from_numpy(v).cuda()
         for k, v in norms.items()}
    toks = torch.arange(2 * new + 20, dtype=torch.int32, device="cuda")
    got = []
    for window in (64, (1 << 31) - 1, 0):
        dec = B.Decoder(B.DecoderConfig(max_batch=4, max_seq=64, max_tokens=256, layers=1, inter=256, vocab=512, window=window,
                                        global_layers=()), w, n)
        k = torch.zeros(1, 4, 16, 1, 256, device="cuda", dtype=torch.bfloat16)
        batch = B.PagedBatch(_i32([0, new, 2 * new, 2 * new + 20]), _i32([0, new // 2, 21]), _i32([[-1, -1], [2, 0], [1, 3]]),
                             max_new=hint)
        got.append(dec.step_paged(toks, k, k.clone(), batch, want_logits=True)[1])
        B.paged_attention_check()
    assert torch.equal(got[0], got[1]) and torch.equal(got[0], got[2])
