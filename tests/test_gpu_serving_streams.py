"""Calls with `stream=`: their outputs and scratch belong to that stream, whatever is still queued on the current one."""
import pytest
import torch

import synth
from test_gpu_serving import _gen, make_batch, objects

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2608_28003_gb300 import build
    build.build()
    from paper_2608_28003_gb300 import binding
    return binding


def _decoder(B):
    f32, bf, norms = synth.decoder_weights(1, 1152, 256, 512, n_q=4, n_kv=1, seed=2)
    w = {k: [t.cuda() for t in v] if isinstance(v, list) else v.cuda() for k, v in bf.items()}
    n = {k: [torch.from_numpy(a).cuda() for a in v] if isinstance(v, list) else torch.from_numpy(v).cuda()
         for k, v in norms.items()}
    return B.Decoder(B.DecoderConfig(max_batch=4, max_seq=64, max_tokens=256, layers=1, inter=256, vocab=512, window=64,
                                     global_layers=(0,), n_q=4, n_kv=1), w, n)


def _calls(B):
    b = make_batch([1] * 30, [900] * 30, 64, 1, 256, torch.bfloat16, 3)
    cache, batch = objects(B, b)
    x = torch.randn(30, 6, 256, device="cuda", generator=_gen(1)).bfloat16()
    table = B.rope_table(B.RopeConfig(256))
    pos = torch.arange(30, device="cuda", dtype=torch.int32)
    logits, u = torch.randn(30, 5000, device="cuda", generator=_gen(2)), torch.rand(30, device="cuda", generator=_gen(3))
    dec, toks = _decoder(B), torch.arange(30, device="cuda", dtype=torch.int32)
    pool, q = [t[None] for t in (cache.k, cache.v)], x[:, :4].contiguous()
    return dict(rope=lambda **kw: [B.rope(table, x, pos, **kw)],
                append=lambda **kw: [B.rope_append(table, cache, batch, x[:, :4], x[:, 4:5], x[:, 5:], **kw)],
                attention=lambda **kw: [B.paged_attention(cache, batch, q, **kw)],
                workspace=lambda **kw: [B.paged_attention(cache, batch, q, ws=B.Workspace(), **kw)],
                sample=lambda **kw: list(B.sample(logits, u, want_probs=True, **kw)),
                step=lambda **kw: list(dec.step_paged(toks, *pool, batch, u=u, want_logits=True, want_probs=True, **kw)))


@pytest.mark.parametrize("name", ["rope", "append", "attention", "sample", "step"])
def test_outputs_belong_to_the_calls_stream(B, name):
    """Blocks of the outputs' sizes are freed with a write to them still queued on the current stream."""
    call, side = _calls(B)[name], torch.cuda.Stream()
    want = call()
    torch.cuda.synchronize()
    for _ in range(2):
        junk = [torch.empty_like(t) for t in want for _ in range(3)]
        torch.cuda._sleep(200_000_000)  # about 0.1 s
        for t in junk:
            t.fill_(7)
        del junk, t
        got = call(stream=side)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_a_workspace_grown_by_a_call_is_zeroed_on_its_stream(B):
    call, side = _calls(B)["workspace"], torch.cuda.Stream()
    want = call()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):  # what the grown buffer may find
        junk = [torch.full((n << 20,), 255, dtype=torch.uint8, device="cuda") for n in (16, 64, 128)]
    torch.cuda.synchronize()
    del junk
    torch.cuda._sleep(200_000_000)
    got = call(stream=side)
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0])
