"""What the serving and 4-bit calls take and give as tensors: subclasses, parameters, tensors they refuse; and captured calls whose
scratch held something else before."""
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


class Mine(torch.Tensor):
    pass


KINDS = {"subclass": lambda t: t.as_subclass(Mine),
         "parameter": lambda t: torch.nn.Parameter(t, requires_grad=False),
         "inference": lambda t: t}


def _serving(B):
    """name -> (call of a list of tensors, the tensors)"""
    b = make_batch([1, 30, 2], [40, 30, 333], 16, 1, 64, torch.bfloat16, 3)
    cache, batch = objects(B, b)
    x = torch.randn(33, 6, 64, device="cuda", generator=_gen(1)).bfloat16()
    table, pos = B.rope_table(B.RopeConfig(64)), torch.arange(33, device="cuda", dtype=torch.int32)
    logits, u = torch.randn(33, 500, device="cuda", generator=_gen(2)), torch.rand(33, device="cuda", generator=_gen(3))
    w4 = B.fp4_quantize(torch.randn(96, 384, device="cuda", generator=_gen(4)).bfloat16())
    norm = torch.rand(64, device="cuda", generator=_gen(5))
    c4 = B.paged_cache_fp4(cache.k.shape[0], 16, 1, 64)
    B.fp4_rope_append(table, c4, batch, x[:, :4], x[:, 4:5], x[:, 5:])
    paged = [cache.k, cache.v, batch.row_start, batch.kv_len, batch.pages]

    def attend(k, v, r, n, p, q):
        return [B.paged_attention(B.PagedCache(k, v), B.PagedBatch(r, n, p, batch.max_new), q)]

    def append(k, v, r, n, p, q, kk, vv, w):
        return [B.rope_append(table, B.PagedCache(k, v), B.PagedBatch(r, n, p, batch.max_new), q, kk, vv, w, w), k, v]

    def attend4(k, v, ks, vs, r, n, p, q):
        return [B.fp4_paged_attention(B.PagedCacheFp4(k, v, ks, vs), B.PagedBatch(r, n, p, batch.max_new), q)]

    def append4(k, v, ks, vs, r, n, p, q, kk, vv, w):
        c = B.PagedCacheFp4(k, v, ks, vs)
        return [B.fp4_rope_append(table, c, B.PagedBatch(r, n, p, batch.max_new), q, kk, vv, w, w), k, v, ks, vs,
                *B.fp4_paged_values(c)]

    def quantise(t):
        q = B.fp4_quantize(t)
        return [q.codes, q.scales, q.row_scale, B.fp4_dequantize(q)]

    def linear(codes, scales, rows, t):
        return [B.fp4_linear(B.Fp4Tensor(codes, scales, rows, 16), t)]
    four = [c4.k, c4.v, c4.k_scales, c4.v_scales, batch.row_start, batch.kv_len, batch.pages]
    return dict(attend=(attend, paged + [x[:, :4]]), append=(append, paged + [x[:, :4], x[:, 4:5], x[:, 5:], norm]),
                attend4=(attend4, four + [x[:, :4]]), append4=(append4, four + [x[:, :4], x[:, 4:5], x[:, 5:], norm]),
                quantise=(quantise, [x.view(33, 384)]), linear=(linear, [w4.codes, w4.scales, w4.row_scale, x.view(33, 384)]),
                rope=(lambda t, p: [B.rope(table, t, p)], [x, pos]),
                sample=(lambda t, v: list(B.sample(t, v, want_probs=True)), [logits, u]))


NAMES = ["attend", "append", "attend4", "append4", "quantise", "linear", "rope", "sample"]


def _bits(t):
    return t.as_subclass(torch.Tensor).detach().contiguous().view(torch.uint8)


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("name", NAMES)
def test_kinds_of_tensors(B, name, kind):
    """Each of a call's tensors in turn, and all of them, of another kind: the same bits, outputs plain tensors."""
    call, given = _serving(B)[name]
    want = [t.clone() for t in call(*given)]

    def same(tensors):
        with torch.inference_mode(kind == "inference"):
            got = call(*tensors)
        assert len(got) == len(want)
        for a, w, made in zip(got, want, [not any(a is t for t in tensors) for a in got]):
            assert a.shape == w.shape and a.dtype == w.dtype and a.device == w.device
            assert not made or (type(a) is torch.Tensor and a.is_contiguous() and not a.requires_grad)
            assert torch.equal(_bits(a), _bits(w))
    for i in range(len(given)):
        same(given[:i] + [KINDS[kind](given[i])] + given[i + 1:])
    same([KINDS[kind](t) for t in given])


@pytest.mark.parametrize("name", NAMES)
def test_tensors_that_are_refused(B, name):
    """On the host, on no device, sparse, of too many dimensions, of another type: an error, whichever tensor it is."""
    call, given = _serving(B)[name]
    others = [lambda t: t.cpu(), lambda t: t.to("meta"), lambda t: t[(None,) * (7 - t.dim())], lambda t: t.double(),
              lambda t: t.reshape(-1, t.shape[-1]).to_sparse(), lambda t: None, lambda t: "no tensor"]
    for i in range(len(given)):
        for other in others:
            if name in ("append", "append4") and i == len(given) - 1 and other is others[5]:
                continue  # no norm is fine
            with pytest.raises((AssertionError, ValueError, TypeError, AttributeError, RuntimeError)):
                call(*given[:i], other(given[i]), *given[i + 1:])
    torch.cuda.synchronize()


def _captured_calls(B):
    calls = {}
    for name, new in (("tokens", [1] * 20), ("chunks", [40, 1, 150])):
        b = make_batch(new, [900] * len(new), 64, 2, 128, torch.bfloat16, 3)
        cache, batch = objects(B, b)
        q = torch.randn(b["n_rows"], 8, 128, device="cuda", generator=_gen(1)).bfloat16()
        calls["attend " + name] = lambda ws, a=(cache, batch, q): B.paged_attention(*a, ws=ws)
        c4 = B.paged_cache_fp4(cache.k.shape[0], 64, 2, 128)
        for t in (c4.k, c4.v, c4.k_scales, c4.v_scales):
            t.copy_(torch.randint(0, 120, t.shape, device="cuda", generator=_gen(2)))
        calls["attend4 " + name] = lambda ws, a=(c4, batch, q): B.fp4_paged_attention(*a, ws=ws)
    for m in (1, 17, 200):
        x = synth.activations(m, 1152, 8, seed=3)[1].cuda()
        w = synth.weight(2304, 1152, seed=3)[1].cuda()
        q, w4 = B.prepare_weights(w, B.act_absmax(x)), B.fp4_quantize(w)
        calls[f"linear {m}"] = lambda ws, a=(q, x): B.linear(*a, ws=ws)
        calls[f"bf16 {m}"] = lambda ws, a=(w, x): B.linear_bf16(*a, ws=ws)
        calls[f"fp4 {m}"] = lambda ws, a=(w4, x): B.fp4_linear(*a, ws=ws)
    return calls


CAPTURED = ["attend tokens", "attend4 tokens", "attend chunks", "attend4 chunks"] + [f"{n} {m}" for m in (1, 17, 200)
                                                                                    for n in ("linear", "bf16", "fp4")]


@pytest.mark.parametrize("own", [False, True])
@pytest.mark.parametrize("name", CAPTURED)
def test_captured_scratch_may_hold_anything_but_its_counters(B, monkeypatch, name, own):
    """A captured call's scratch, all ones (NaN of every type) behind the counters ahead of every replay."""
    call, made = _captured_calls(B)[name], []
    want = call(B.Workspace())

    def scratch(nbytes, device):
        buf = torch.full((nbytes,), 255, dtype=torch.uint8, device=device)
        buf[:B.WS_RESERVED].zero_()
        made.append(nbytes)
        return buf
    monkeypatch.setattr(B, "_graph_scratch", scratch)
    g = torch.cuda.CUDAGraph()
    ws = B.Workspace() if own or name[:6] in ("linear", "bf16 1", "bf16 2") else None  # (the others take the stream's)
    with torch.cuda.graph(g):
        y = call(ws)
    for _ in range(3):
        y.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want)
    assert made or "linear" in name or "bf16" in name
