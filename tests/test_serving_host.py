"""CPU checks of a serving step's operators: the oracle against closed forms and brute force, the host function
of the rotary frequencies against it, and every refusal of the entry points (nothing reaches a GPU)."""
import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import serving as OS


@pytest.fixture(scope="module")
def B():
    from paper_2608_28003_gb300 import build
    build.build()
    from paper_2608_28003_gb300 import binding
    return binding


# ------------------------------------------------------------------------------------- the oracle
def test_rope_oracle_is_a_rotation():
    rng = np.random.default_rng(1)
    f, s = OS.rope_frequencies(32, 1e4)
    assert s == 1.0 and f[0] == 1.0 and abs(f[8] - 0.01) < 1e-15
    x = rng.standard_normal((4, 2, 64))
    for inter in (False, True):
        y = OS.rope(x, [0, 1, 5, 100000], f, s, inter)
        np.testing.assert_array_equal(y[0], x[0])
        np.testing.assert_array_equal(y[..., 32:], x[..., 32:])
        np.testing.assert_allclose(np.linalg.norm(y, axis=-1), np.linalg.norm(x, axis=-1), rtol=1e-13)
        # scores depend on the distance alone
        a = (OS.rope(x[:1], [7], f, s, inter) * OS.rope(x[1:2], [3], f, s, inter)).sum()
        b = (OS.rope(x[:1], [1007], f, s, inter) * OS.rope(x[1:2], [1003], f, s, inter)).sum()
        assert abs(a - b) < 1e-10


def test_attention_oracle_against_plain_softmax():
    rng = np.random.default_rng(2)
    k, v = rng.standard_normal((2, 6, 4, 2, 8))
    batch = dict(row_start=np.array([0, 1, 4]), kv_len=np.array([7, 3]), pages=np.array([[4, 0], [2, 9]]), n_rows=5)
    q = rng.standard_normal((5, 4, 8))
    o, _, _ = OS.attention(q, k, v, batch, 0.3)
    keys = np.concatenate([k[4], k[0]])[:7, 1]
    w = np.exp(0.3 * keys @ q[0, 3])
    np.testing.assert_allclose(o[0, 3], w @ np.concatenate([v[4], v[0]])[:7, 1] / w.sum(), rtol=1e-12)
    np.testing.assert_allclose(o[1, 0], v[2, 0, 0])  # the first of three rows sees one key
    assert np.isnan(o[4]).all()                      # a row of no sequence
    o, _, _ = OS.attention(q, k, v, batch, 0.3, window=1)
    np.testing.assert_allclose(o[3, 2], v[2, 2, 1])
    batch["pages"][1, 0] = 6                         # outside the cache: no keys
    assert (OS.attention(q, k, v, batch, 0.3)[0][1:4] == 0).all()


def test_sample_oracle():
    row = np.log([0.5, 0.125, 0.25, 0.125])
    assert OS.sample(row, 0.49)[0] == 0 and OS.sample(row, 0.51)[0] == 1 and OS.sample(row, 0.99)[0] == 3
    assert OS.sample(row, 0.9, top_k=2)[0] == 2 and OS.sample(row, 0.9, top_k=3)[0] == 2  # the tie: the lower index
    assert OS.sample(row, 0.72, top_k=3) == (2, pytest.approx(0.25 / 0.875), 3)
    assert OS.sample(row, 0.99, top_p=0.7)[0] == 2 and OS.sample(row, 0.99, top_p=0.4)[0] == 0
    assert OS.sample(row, 0.99, min_p=0.4)[0] == 2 and OS.sample([1.0, 3.0, 3.0], 0.9, temperature=0)[0] == 1
    assert OS.sample([-np.inf, np.nan], 0.5)[0] == -1 and OS.sample([0, np.inf, np.inf], 0.6)[0] == 2


# -------------------------------------------------------------------------------- frequencies
@pytest.mark.parametrize("rot,base,scaling,kw", [
    (16, 1e4, "none", {}), (64, 5e5, "linear", dict(factor=4.0)), (256, 1e6, "none", {}),
    (128, 5e5, "wavelength", dict(factor=8.0, low=1.0, high=4.0, original_len=8192)),
    (128, 1e4, "parts", dict(factor=16.0, low=1.0, high=32.0, original_len=4096)),
    (64, 1e4, "parts", dict(factor=4.0, low=1.0, high=32.0, original_len=2048, attn_factor=1.25)),
    (32, 1.5, "none", {}), (16, 1e4, "linear", dict(factor=0.01))])
def test_rope_frequencies(B, rot, base, scaling, kw):
    turns, scale = B.rope_frequencies(B.RopeConfig(rot, base=base, scaling=scaling, **kw))
    f, s = OS.rope_frequencies(rot, base, scaling, **kw)
    got = np.array([int(t) % (1 << 64) for t in turns], dtype=np.float64) / 2.0 ** 64
    want = f / (2 * math.pi) % 1.0
    assert len(turns) == rot // 2 and abs(scale - s) <= 2 ** -23 * s
    assert (np.abs(got - want) <= 2.0 ** -48 * np.maximum(1, f)).all()


def test_rope_frequencies_refusals(B):
    def status(**kw):
        try:
            B.rope_frequencies(B.RopeConfig(**{**dict(rotary_dim=64), **kw}))
        except B.W8A8Error as e:
            return e.status
        return 0
    assert status() == 0
    for r in (0, -16, 8, 24, 272):
        assert status(rotary_dim=r) == 2
    for bad in (dict(base=1.0), dict(base=float("nan")), dict(base=float("inf")), dict(scaling="linear", factor=0.0),
                dict(scaling="parts", factor=2.0, low=1.0, high=1.0, original_len=10),
                dict(scaling="wavelength", factor=2.0, low=1.0, high=4.0), dict(attn_factor=-1.0),
                dict(scaling="linear", factor=float("inf"))):
        assert status(**bad) == 1, bad
    with pytest.raises(ValueError):
        B.rope_frequencies(B.RopeConfig(64, scaling="other"))


# ----------------------------------------------------------------------------------- refusals
P = 0x10000  # an aligned address nothing reads


def _cache(B, **kw):
    d = dict(dtype=0, n_pages=4, page_size=16, n_kv=2, head_dim=128, page_stride=4096, slot_stride=256, head_stride=128, k=P, v=P)
    d.update(kw)
    return B.PagedCacheC(*d.values())


def _batch(B, **kw):
    d = dict(n_seqs=2, n_rows=3, max_new=2, max_pages=4, row_start=P, kv_len=P, pages=P)
    d.update(kw)
    return B.PagedBatchC(*d.values())


BAD_CACHES = [(dict(dtype=2), 1), (dict(dtype=-1), 1), (dict(n_pages=0), 1), (dict(n_kv=0), 1), (dict(head_dim=96), 2),
              (dict(head_dim=512), 2), (dict(page_size=24), 2), (dict(page_size=8), 2), (dict(page_size=512), 2),
              (dict(page_stride=4100), 2), (dict(slot_stride=64), 2), (dict(head_stride=0), 2), (dict(page_stride=-4096), 2),
              (dict(k=None), 1), (dict(v=None), 1), (dict(k=P + 2), 3), (dict(n_kv=1024), 2)]
BAD_BATCHES = [(dict(n_seqs=-1), 1), (dict(n_rows=-1), 1), (dict(max_new=0), 1), (dict(max_pages=-1), 1),
               (dict(max_pages=1 << 28), 2), (dict(row_start=None), 1), (dict(kv_len=None), 1), (dict(pages=None), 1),
               (dict(pages=P + 2), 3)]


def test_paged_refusals(B):
    L = B.lib()
    rt = B.RopeTableC(64, 0, 1.0, P)

    def attn(c, b, q=P, q_row=1024, q_head=128, n_q=8, scale=0.1, window=0, o=P, o_row=1024, o_head=128, ws=P, n=0):
        return L.w8a8_paged_attention(ctypes.byref(c), ctypes.byref(b), q, q_row, q_head, n_q, scale, window, o, o_row, o_head,
                                      ws, n, None)

    def append(c, b, t=rt, q=P, q_row=1536, n_q=8, k=P, k_row=1536, v=P, qo=P, qo_row=1536, eps=1e-6, qn=None):
        return L.w8a8_rope_append(ctypes.byref(t), ctypes.byref(c), ctypes.byref(b), q, q_row, n_q, k, k_row, v, k_row, qn,
                                  None, eps, qo, qo_row, None)
    for kw, want in BAD_CACHES:
        assert attn(_cache(B, **kw), _batch(B)) == want, kw
        assert append(_cache(B, **kw), _batch(B)) == want, kw
    for kw, want in BAD_BATCHES:
        assert attn(_cache(B), _batch(B, **kw)) == want, kw
        assert append(_cache(B), _batch(B, **kw)) == want, kw
    c, b = _cache(B), _batch(B)
    for kw, want in [(dict(n_q=7), 2), (dict(n_q=0), 2), (dict(n_q=512), 2), (dict(scale=0.0), 1), (dict(scale=float("nan")), 1),
                     (dict(window=-1), 1), (dict(q=None), 1), (dict(o=None), 1), (dict(q=P + 8), 3), (dict(q_row=1020), 2),
                     (dict(o_head=64), 2), (dict(o_row=512), 2), (dict(q_head=-128), 2)]:
        assert attn(c, b, **kw) == want, kw
    for kw, want in [(dict(n_q=0), 2), (dict(q=None), 1), (dict(qo=None), 1), (dict(q_row=1001), 2), (dict(k_row=-8), 2),
                     (dict(q=P + 2), 3), (dict(qo_row=512), 2), (dict(qo_row=2048), 2), (dict(eps=-1.0, qn=P), 1),
                     (dict(eps=float("nan"), qn=P), 1), (dict(t=B.RopeTableC(60, 0, 1.0, P)), 2), (dict(t=B.RopeTableC(256, 0, 1.0, P)), 2),
                     (dict(t=B.RopeTableC(64, 0, 1.0, None)), 1), (dict(t=B.RopeTableC(64, 0, 1.0, P + 8)), 3)]:
        assert append(c, b, **kw) == want, kw
    # nothing to do succeeds without a device
    for kw in (dict(n_rows=0), dict(n_seqs=0)):
        assert attn(c, _batch(B, **kw)) == 0 and append(c, _batch(B, **kw)) == 0
    n = ctypes.c_size_t()
    assert L.w8a8_paged_attention_workspace_size(ctypes.byref(c), 8, ctypes.byref(n)) == 0 and n.value >= 65536
    assert L.w8a8_paged_attention_workspace_size(ctypes.byref(c), 9, ctypes.byref(n)) == 2
    assert L.w8a8_paged_attention_workspace_size(None, 8, ctypes.byref(n)) == 1


def test_rope_refusals(B):
    L = B.lib()

    def rope(t=(64, 0, 1.0, P), dtype=0, x=P, x_row=512, x_head=128, T=3, heads=4, dim=128, pos=P, y=2 * P, y_row=512, y_head=128):
        return L.w8a8_rope(ctypes.byref(B.RopeTableC(*t)), dtype, x, x_row, x_head, T, heads, dim, pos, y, y_row, y_head, None)
    for kw, want in [(dict(T=-1), 1), (dict(heads=-1), 1), (dict(dtype=2), 1), (dict(dim=120), 2), (dict(dim=272), 2),
                     (dict(t=(0, 0, 1.0, P)), 2), (dict(t=(144, 0, 1.0, P)), 2), (dict(t=(64, 0, 1.0, None)), 1), (dict(x=None), 1),
                     (dict(y=None), 1), (dict(pos=None), 1), (dict(x=P + 8), 3), (dict(pos=P + 1), 3), (dict(x_row=500), 2),
                     (dict(x_head=-128), 2), (dict(y_head=0), 2), (dict(y_row=256), 2), (dict(y=P, y_row=1024), 2)]:
        assert rope(**kw) == want, kw
    assert rope(T=0, x=None, y=None, pos=None) == 0 and rope(heads=0, x=None, y=None, pos=None) == 0
    assert L.w8a8_rope(None, 0, P, 0, 0, 1, 1, 64, P, P, 0, 0, None) == 1


def test_sample_refusals(B):
    L = B.lib()

    def sample(dtype=2, x=P, row=1024, M=2, V=1000, sp=(None, None, None, None), u=P, tok=P, prob=None):
        return L.w8a8_sample(dtype, x, row, M, V, ctypes.byref(B.SamplingC(*sp)) if sp else None, u, tok, prob, None)
    for kw, want in [(dict(dtype=3), 1), (dict(dtype=-1), 1), (dict(M=-1), 1), (dict(V=0), 1), (dict(V=1 << 21), 2),
                     (dict(sp=None), 1), (dict(x=None), 1), (dict(u=None), 1), (dict(tok=None), 1), (dict(x=P + 2), 3),
                     (dict(V=1 << 20, row=(1 << 20) + 2), 2), (dict(V=1 << 20, x=P + 4, M=1), 2), (dict(row=-4), 2), (dict(u=P + 2), 3), (dict(sp=(None, P + 1, None, None)), 3)]:
        assert sample(**kw) == want, kw
    assert sample(M=0, x=None, u=None, tok=None) == 0


def test_binding_refuses(B):
    """The binding's own checks, on host tensors: each raises before the library is asked."""
    x = torch.zeros(2, 4, 64, dtype=torch.bfloat16)
    k = torch.zeros(3, 16, 2, 64, dtype=torch.bfloat16)
    t = B.RopeTable(64, False, 1.0, torch.zeros(32, dtype=torch.int64))
    batch = B.PagedBatch(torch.zeros(2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32), torch.zeros(1, 1, dtype=torch.int32))
    for call in (lambda: B.rope(t, x, torch.zeros(2, dtype=torch.int32)), lambda: B.paged_attention(B.PagedCache(k, k), batch, x),
                 lambda: B.rope_append(t, B.PagedCache(k, k), batch, x, x[:, :2], x[:, :2]),
                 lambda: B.sample(torch.zeros(2, 8), torch.zeros(2))):
        with pytest.raises(AssertionError, match="CUDA"):
            call()
    with pytest.raises(ValueError):
        B.PagedCache(k, k[:2]).c()
    with pytest.raises(ValueError):
        B.PagedCache(k, k.transpose(1, 2).contiguous().transpose(1, 2)).c()
    with pytest.raises(ValueError):
        B.PagedBatch(torch.zeros(3, dtype=torch.int32), batch.kv_len, batch.pages).c(2)
    with pytest.raises(ValueError):
        B.PagedBatch(torch.zeros(2, dtype=torch.int64), batch.kv_len, batch.pages).c(2)
    assert B.PagedCache(k, k).c().slot_stride == 128 and batch.c(2).max_pages == 1
