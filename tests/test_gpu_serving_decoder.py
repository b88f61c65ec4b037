"""A serving step of the decoder (ragged chunks and single tokens over a paged cache, sampled next tokens) against the
oracle decoder fed sequence by sequence, against the uniform-batch forward, captured and replayed, and its refusals."""
import numpy as np
import pytest
import torch

import synth
from oracle import decoder as OD
from oracle import masks as OM
from oracle import serving as OS

pytestmark = pytest.mark.gpu

L, H, F, V, WINDOW, SEQ, PAGE = 2, 1152, 256, 1024, 100, 320, 16


@pytest.fixture(scope="module")
def B():
    from paper_2608_28003_gb300 import build
    build.build()
    from paper_2608_28003_gb300 import binding
    return binding


def _decoders(B, n_q, n_kv, qk_norm):
    f32, bf, norms = synth.decoder_weights(L, H, F, V, n_q=n_q, n_kv=n_kv, seed=9)
    w = {k: [t.cuda() for t in v] if isinstance(v, list) else v.cuda() for k, v in bf.items()}
    n = {k: [torch.from_numpy(a).cuda() for a in v] if isinstance(v, list) else torch.from_numpy(v).cuda()
         for k, v in norms.items()}
    shape = dict(layers=L, inter=F, vocab=V, window=WINDOW, global_layers=(0,), n_q=n_q, n_kv=n_kv, qk_norm=qk_norm)
    ow = dict(f32)
    ow.update(norms)
    dec = B.Decoder(B.DecoderConfig(max_batch=4, max_seq=SEQ, max_tokens=4 * SEQ, **shape), w, n)
    return dec, lambda: OD.OracleDecoder(OD.DecoderConfig(**shape), ow, batch=1, max_len=SEQ)


class Pool:
    """Pages handed out in a scattered order; slots nobody wrote hold NaN."""

    def __init__(self, n_kv, pages=90, seqs=3):
        self.k, self.v = (torch.full((L, pages, PAGE, n_kv, 256), float("nan"), device="cuda", dtype=torch.bfloat16)
                          for _ in range(2))
        self.free = list(np.random.default_rng(3).permutation(pages))
        self.table = np.full((seqs, SEQ // PAGE), -1, np.int32)
        self.len = np.zeros(seqs, np.int32)

    def batch(self, B, new):
        for s, n in enumerate(new):
            self.len[s] += n
            for c in range(-(-int(self.len[s]) // PAGE)):
                if self.table[s, c] < 0:
                    self.table[s, c] = self.free.pop()
        dev = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()  # noqa: E731
        return B.PagedBatch(dev(np.concatenate([[0], np.cumsum(new)])), dev(self.len), dev(self.table), max_new=max([1] + list(new)))


STEPS = [[130, 7, 1], [1, 40, 1], [1, 1, 1], [0, 1, 60], [17, 1, 1]]  # new tokens of the three sequences, step by step


@pytest.mark.parametrize("n_q,n_kv,qk_norm", [(4, 1, True), (8, 2, False)])
def test_steps_match_the_oracle(B, n_q, n_kv, qk_norm):
    dec, oracle = _decoders(B, n_q, n_kv, qk_norm)
    pool, ods = Pool(n_kv), [oracle() for _ in range(3)]
    toks = synth.tokens(3 * SEQ, V, seed=4).reshape(3, SEQ)
    u = torch.rand(3, device="cuda", generator=torch.Generator("cuda").manual_seed(1))
    top_k = torch.tensor([50, 0, 5], device="cuda", dtype=torch.int32)
    last = [None] * 3
    for new in STEPS:
        at = pool.len.copy()
        batch = pool.batch(B, new)
        flat = np.concatenate([toks[s, at[s]:at[s] + n] for s, n in enumerate(new)]).astype(np.int32)
        nxt, logits, probs = dec.step_paged(torch.from_numpy(flat).cuda(), pool.k, pool.v, batch, u=u, top_k=top_k,
                                            want_logits=True, want_probs=True)
        got = logits.cpu().numpy().astype(np.float64)
        for s, n in enumerate(new):
            if n == 0:
                continue
            last[s] = ods[s].forward(toks[s:s + 1, at[s]:at[s] + n], int(at[s]), OM.make_mask())["logits"][0, -1]
            rel = np.linalg.norm(got[s] - last[s]) / np.linalg.norm(last[s])
            assert rel <= 1e-2, (new, s, rel)  # the decoder's stated tolerance, all bf16
            t, p, _ = OS.sample(got[s], float(u[s]), top_k=int(top_k[s]))
            assert int(nxt[s]) == t and abs(float(probs[s]) - p) <= 1e-6
    greedy, none, no_probs = dec.step_paged(torch.from_numpy(flat[:0]).cuda(), pool.k, pool.v, pool.batch(B, [0, 0, 0]))
    assert none is None and no_probs is None and greedy.tolist() == [-1] * 3


def test_step_agrees_with_the_uniform_forward_under_a_mask(B):
    """W8A8 layers and lm_head: two sequences of equal length, fed whole and as a chunk and single tokens; the logits agree
    to the decoder's tolerance under a mask, greedy tokens are the largest logits, and other calls of the model between
    the steps change nothing (the paged step keeps its keys in the caller's pages)."""
    dec, _ = _decoders(B, 4, 1, True)
    toks = torch.from_numpy(synth.tokens(2 * 60, V, seed=6).reshape(2, 60)).cuda()
    dec.calibrate(toks)
    dec.prepare()
    dec.set_mask(0b10, 0b01, True)
    ref, _ = dec.forward(toks, 0)
    ref = ref.view(2, 60, V)
    pool = Pool(1, seqs=2)
    for a, b in ((0, 57), (57, 58), (58, 60)):
        batch = pool.batch(B, [b - a, b - a])
        nxt, logits, _ = dec.step_paged(toks[:, a:b].reshape(-1).contiguous(), pool.k, pool.v, batch, want_logits=True)
        rel = (logits - ref[:, b - 1]).norm(dim=1) / ref[:, b - 1].norm(dim=1)
        assert rel.max() <= 2e-2, (a, b, rel)
        assert torch.equal(nxt.long(), logits.argmax(1))
        dec.forward(toks.flip(0).contiguous(), 0)


def test_step_captured(B):
    """A step captured in a graph and replayed with other tokens, lengths and pages gives what the eager step gives; rows
    behind the last sequence are padding."""
    dec, _ = _decoders(B, 4, 1, True)
    pool = Pool(1)
    toks = torch.from_numpy(synth.tokens(64, V, seed=8)).cuda()
    dec.step_paged(toks[:30].contiguous(), pool.k, pool.v, pool.batch(B, [10, 12, 8]))
    batch = pool.batch(B, [1, 1, 1])
    one = torch.cat([toks[30:33], toks[40:45]]).contiguous()  # three tokens and five rows of padding
    u = torch.tensor([0.1, 0.5, 0.9], device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    k0, v0 = pool.k.clone(), pool.v.clone()
    want = dec.step_paged(one, pool.k, pool.v, batch, u=u, want_logits=True)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        got = dec.step_paged(one, pool.k, pool.v, batch, u=u, want_logits=True)
    pool.k.copy_(k0)
    pool.v.copy_(v0)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    for step in range(2):
        nxt = pool.batch(B, [1, 1, 1])
        batch.kv_len.copy_(nxt.kv_len)
        batch.pages.copy_(nxt.pages)
        one[:3] = got[0]
        k0, v0 = pool.k.clone(), pool.v.clone()
        g.replay()
        torch.cuda.synchronize()
        kept = got[0].clone(), got[1].clone()
        pool.k.copy_(k0)
        pool.v.copy_(v0)
        want = dec.step_paged(one, pool.k, pool.v, batch, u=u, want_logits=True)
        assert torch.equal(kept[0], want[0]) and torch.equal(kept[1], want[1]), step


def test_step_refusals(B):
    dec, _ = _decoders(B, 4, 1, True)
    pool = Pool(1)
    batch = pool.batch(B, [2, 1, 1])
    toks = torch.zeros(4, device="cuda", dtype=torch.int32)
    with pytest.raises(ValueError):
        dec.step_paged(toks, pool.k[:1], pool.v[:1], batch)
    with pytest.raises(ValueError):
        dec.step_paged(toks.long(), pool.k, pool.v, batch)
    with pytest.raises(ValueError):
        dec.step_paged(toks, pool.k, pool.v, batch, top_k=toks[:3])  # parameters without u
    with pytest.raises(B.W8A8Error) as e:
        dec.step_paged(toks, pool.k.half(), pool.v.half(), batch)
    assert e.value.status == 2
    with pytest.raises(B.W8A8Error) as e:
        dec.step_paged(torch.zeros(4 * SEQ + 1, device="cuda", dtype=torch.int32), pool.k, pool.v, batch)
    assert e.value.status == 2
