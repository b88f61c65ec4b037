"""A serving step's operators on the GPU against the 64-bit oracle: rotary positions, the append to a paged
cache, attention of a ragged batch over it, and sampling, at the sizes, layouts and masks where they can go
wrong; the operators run together; and calls on other streams, captured and replayed."""
import random

import numpy as np
import pytest
import torch

from oracle import serving as OS

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module")
def B():
    from paper_2608_28003_gb300 import build
    build.build()
    from paper_2608_28003_gb300 import binding
    return binding


def _gen(seed):
    return torch.Generator("cuda").manual_seed(seed)


def _np(t):
    return t.detach().double().cpu().numpy()


SCALINGS = {"none": {}, "linear": dict(factor=4.0), "wavelength": dict(factor=8.0, low=1.0, high=4.0, original_len=8192),
            "parts": dict(factor=16.0, low=1.0, high=32.0, original_len=4096)}


# ---------------------------------------------------------------------------------------- rope
def _rope_tol(y, x, dt, scale):
    """Half a step of the result; cos and sin off by 2^-22 (half-turns rounded to 24 bits: 9e-8 rad, the functions and
    the factor an ulp each), two products and a sum of 24 bits: 2^-21 of the pair's magnitude in all."""
    return torch.finfo(dt).eps / 2 * np.abs(y) + 2.0 ** -21 * scale * np.abs(x).max() + (2.0 ** -25 if dt == torch.float16 else 0)


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("T,heads,dim,rot,inter,scaling", [
    (1, 1, 16, 16, False, "none"), (5, 3, 64, 64, True, "linear"), (33, 5, 256, 256, False, "wavelength"),
    (7, 2, 96, 48, False, "parts"), (130, 32, 128, 64, True, "parts"), (2, 1, 256, 16, True, "none")])
def test_rope(B, dt, T, heads, dim, rot, inter, scaling):
    x = torch.randn(T, heads, dim, device="cuda", generator=_gen(T + dim)).to(DT[dt])
    pos = torch.randint(0, 1 << 20, (T,), device="cuda", generator=_gen(3), dtype=torch.int32)
    pos[0], pos[-1] = 0, -(1 << 31) if T > 1 else 1000003  # the first position, and one as far as they go
    table = B.rope_table(B.RopeConfig(rot, base=5e5, interleaved=inter, scaling=scaling, **SCALINGS[scaling]))
    y = B.rope(table, x, pos)
    f, s = OS.rope_frequencies(rot, 5e5, scaling, **SCALINGS[scaling])
    want = OS.rope(_np(x), _np(pos), f, s, inter)
    # an angle of |p| f radians is itself known to 2^-53 of it in the oracle and in the frequencies
    assert (np.abs(_np(y) - want) <= _rope_tol(want, _np(x), DT[dt], s) + 2.0 ** -50 * 2.0 ** 31).all()
    assert torch.equal(y[..., rot:], x[..., rot:])
    z = x.clone()
    assert B.rope(table, z, pos, out=z) is z and torch.equal(z, y)  # in place


def test_rope_strides(B):
    """Head-major and padded inputs and outputs, a broadcast input, and nothing written between them."""
    T, H, D = 6, 4, 64
    big = torch.randn(H, T + 2, D + 16, device="cuda", generator=_gen(1)).bfloat16()
    x = big[:, 1:T + 1, :D].transpose(0, 1)
    pos = torch.arange(T, device="cuda", dtype=torch.int32) * 1000
    table = B.rope_table(B.RopeConfig(32, interleaved=True))
    want = B.rope(table, x.contiguous(), pos)
    out = torch.full((H, T, D + 8), 7.0, device="cuda", dtype=torch.bfloat16)
    B.rope(table, x, pos, out=out[..., :D].transpose(0, 1))
    assert torch.equal(out[..., :D].transpose(0, 1), want) and (out[..., D:] == 7).all()
    one = x[:, :1].expand(T, H, D)
    assert torch.equal(B.rope(table, one, pos), B.rope(table, one.contiguous(), pos))
    assert B.rope(table, x[:0], pos[:0]).shape == (0, H, D)


def test_rope_turns_as_positions_add(B):
    """Far positions: p + 2^20 turns a pair as p and then 2^20 do (to the rounding of two bf16 results)."""
    x = torch.randn(64, 2, 128, device="cuda", generator=_gen(2)).half()
    table = B.rope_table(B.RopeConfig(128))
    p = torch.randint(0, 1 << 19, (64,), device="cuda", generator=_gen(4), dtype=torch.int32)
    far = torch.full_like(p, 1 << 20)
    a, b = B.rope(table, x, p + far), B.rope(table, B.rope(table, x, p), far)
    # two roundings of the middle result and one of each end, on a pair of magnitude up to max|x| sqrt(2)
    assert (a.float() - b.float()).abs().max().item() <= 5 * 2.0 ** -11 * float(x.abs().max()) * 1.5


# ------------------------------------------------------------------------------------ paged batches
def make_batch(new, keys, page, n_kv, dim, dt, seed, head_major=False, together=False, spare=2, rows_after=0,
               fill=None):
    """A ragged batch over scattered pages; fill: what slots that hold no key of the batch contain."""
    rng = random.Random(seed)
    wide = max(1, max(-(-k // page) for k in keys)) if keys else 1
    used = [-(-k // page) for k in keys]
    n_pages = max(1, sum(used)) + spare
    ids = list(range(n_pages))
    rng.shuffle(ids)
    table = np.full((len(keys), wide), -1, np.int32)
    for s, u in enumerate(used):
        table[s, :u] = [ids.pop() for _ in range(u)]
    shape = (n_pages, n_kv, page, dim) if head_major else (n_pages, page, n_kv, dim)
    if together:  # keys and values side by side in one tensor
        both = torch.randn(n_pages, 2, *shape[1:], device="cuda", generator=_gen(seed)).to(dt)
        k, v = both[:, 0], both[:, 1]
    else:
        k, v = (torch.randn(shape, device="cuda", generator=_gen(seed + i)).to(dt) for i in (0, 1))
    if head_major:
        k, v = k.transpose(1, 2), v.transpose(1, 2)
    if fill is not None:
        live = torch.zeros(n_pages, page, dtype=torch.bool)
        for s, n in enumerate(keys):
            for p in range(n):
                live[table[s, p // page], p % page] = True
        for t in (k, v):
            t[~live.cuda()] = fill
    starts = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    rows = int(starts[-1]) + rows_after
    return dict(k=k, v=v, row_start=starts, kv_len=np.array(keys, np.int32), pages=table, n_rows=rows,
                max_new=max(list(new) + [1]))


def objects(B, b):
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    return (B.PagedCache(b["k"], b["v"]),
            B.PagedBatch(dev(b["row_start"]), dev(b["kv_len"]), dev(b["pages"]), max_new=b["max_new"]))


# -------------------------------------------------------------------------------------- append
@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("new,keys,page,n_q,n_kv,dim,rot,inter,norm,layout", [
    ([1], [1], 16, 4, 1, 256, 256, False, True, ""),
    ([1, 1, 1, 1, 1], [17, 1, 16, 64, 33], 16, 4, 1, 256, 256, False, True, ""),
    ([5, 0, 40, 1], [5, 9, 100, 64], 32, 8, 2, 128, 64, True, True, "heads"),
    ([3, 20], [130, 20], 64, 5, 5, 64, 64, True, False, "both"),
    ([300], [311], 256, 28, 4, 128, 128, False, False, "both heads")])
def test_rope_append(B, dt, new, keys, page, n_q, n_kv, dim, rot, inter, norm, layout):
    b = make_batch(new, keys, page, n_kv, dim, DT[dt], 11, "heads" in layout, "both" in layout, rows_after=2)
    cache, batch = objects(B, b)
    T = b["n_rows"]
    qkv = (torch.randn(T, n_q + 2 * n_kv, dim, device="cuda", generator=_gen(5)) * 3).to(DT[dt])
    q, k, v = qkv[:, :n_q], qkv[:, n_q:n_q + n_kv], qkv[:, n_q + n_kv:]
    qn, kn = ((1 + 0.3 * torch.randn(dim, device="cuda", generator=_gen(6 + i))) if norm else None for i in (0, 1))
    table = B.rope_table(B.RopeConfig(rot, base=1e4, interleaved=inter, scaling="linear", factor=4.0))
    k0, v0 = _np(b["k"]), _np(b["v"])
    out = torch.full((T, n_q, dim), 9.0, device="cuda", dtype=DT[dt])
    got = B.rope_append(table, cache, batch, q, k, v, q_norm=qn, k_norm=kn, eps=1e-5, q_out=out)
    assert got is out and (out[T - 2:] == 9).all()  # rows of no sequence
    f, s = OS.rope_frequencies(rot, 1e4, "linear", factor=4.0)
    nq, nk = OS.rms_norm(_np(q), None if qn is None else _np(qn), 1e-5), OS.rms_norm(_np(k), None if kn is None else _np(kn), 1e-5)
    eps = torch.finfo(DT[dt]).eps / 2

    def check(y, x, want):  # rotation as above; the norm: a sum of dim squares, a root and a quotient, two products
        tol = eps * np.abs(want) + (2.0 ** -21 + (dim / 16 + 8) * 2.0 ** -24) * np.abs(x).max() + 2.0 ** -25
        assert (np.abs(y - want) <= tol).all(), float((np.abs(y - want) - tol).max())
    for r, seq, pos, _ in OS.rows_of(b, page):
        check(_np(out[r:r + 1]), nq[r], OS.rope(nq[r:r + 1], [pos], f, s, inter))
        page_id, slot = OS.place(b, b["k"].shape[0], page, seq, pos)
        k0[page_id, slot] = OS.rope(nk[r:r + 1], [pos], f, s, inter)[0]
        v0[page_id, slot] = _np(v[r])
    check(_np(b["k"]), nk, k0)          # and every other slot as it was
    np.testing.assert_array_equal(_np(b["v"]), v0)


def test_rope_append_leaves_bad_pages_alone(B):
    """Pages outside the cache and rows at negative positions: nothing is written, q is rotated all the same."""
    b = make_batch([2, 3, 1], [40, 2, 9], 16, 2, 64, torch.bfloat16, 3)
    b["pages"][0, 2] = b["k"].shape[0]
    b["pages"][2, 0] = -7
    cache, batch = objects(B, b)
    k0, v0 = b["k"].clone(), b["v"].clone()
    x = torch.randn(6, 8, 64, device="cuda", generator=_gen(1)).bfloat16()
    table = B.rope_table(B.RopeConfig(64))
    q = B.rope_append(table, cache, batch, x[:, :4], x[:, 4:6], x[:, 6:])
    pos = torch.tensor([38, 39, -1, 0, 1, 8], device="cuda", dtype=torch.int32)
    assert torch.equal(q, B.rope(table, x[:, :4], pos))
    changed = {(int(i), int(j)) for i, j in torch.nonzero((b["v"] != v0).flatten(2).any(2)).cpu()}
    assert changed == {(int(b["pages"][1, 0]), 0), (int(b["pages"][1, 0]), 1)}
    assert {(int(i), int(j)) for i, j in torch.nonzero((b["k"] != k0).flatten(2).any(2)).cpu()} <= changed


# ----------------------------------------------------------------------------------- attention
def attn_check(got, q, b, scale, window, rows=None):
    """Per output: half a step of the result; weights rounded to the type and their sum (2 half-steps of the weighted
    |v|); scores summed in fp32 (dim 2^-24 of the largest sum of |q k|, twice: numerator and sum) and exponentials and
    sums of 2^-20; fp16 also half its smallest step."""
    want, mass, mag = OS.attention(_np(q), _np(b["k"]), _np(b["v"]), b, scale, window, rows)
    dt = q.dtype
    eps, dim = torch.finfo(dt).eps / 2, q.shape[2]
    delta = scale * dim * 2.0 ** -24 * mag
    tol = eps * np.abs(want) + (2 * eps + 2 * delta[..., None] + 2.0 ** -20) * mass + (2.0 ** -25 if dt == torch.float16 else 1e-38)
    got, some = _np(got), ~np.isnan(want).all(axis=(1, 2))
    err = np.abs(got - want)[some] - tol[some]
    assert err.max() <= 0, (float(err.max()), np.argwhere(err > 0)[:4].tolist())
    return want


ATTN = [  # new, keys, page, n_q, n_kv, dim, window
    ([1], [1], 16, 4, 1, 256, 0),
    ([1], [700], 16, 4, 1, 256, 0),
    ([1, 1, 1, 1], [15, 16, 17, 300], 16, 4, 1, 256, 0),
    ([1, 1, 1], [500, 40, 64], 32, 4, 1, 256, 64),
    ([1] * 9, [3, 1000, 129, 128, 127, 64, 65, 513, 2], 64, 8, 4, 256, 0),
    ([4, 4, 4], [4, 200, 77], 16, 24, 8, 64, 0),
    ([5, 1, 3], [90, 1, 333], 128, 5, 5, 64, 50),
    ([1, 2], [1500, 900], 256, 16, 2, 128, 0),
    ([37], [37], 16, 4, 1, 256, 0),
    ([128, 1, 0, 50], [128, 60, 5, 250], 16, 4, 1, 256, 0),
    ([200], [333], 64, 4, 1, 256, 100),
    ([33, 65], [400, 65], 32, 16, 4, 128, 0),
    ([130], [1000], 64, 28, 4, 128, 0),
    ([70, 9], [70, 640], 128, 6, 6, 64, 128),
    ([129], [129], 16, 12, 4, 64, 1),
    ([21], [300], 16, 80, 1, 64, 0),
    ([3], [50], 16, 128, 1, 64, 0),
]


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("new,keys,page,n_q,n_kv,dim,window", ATTN)
def test_attention(B, dt, new, keys, page, n_q, n_kv, dim, window):
    b = make_batch(new, keys, page, n_kv, dim, DT[dt], len(keys) + dim)
    cache, batch = objects(B, b)
    q = (torch.randn(b["n_rows"], n_q, dim, device="cuda", generator=_gen(8)) * 1.5).to(DT[dt])
    attn_check(B.paged_attention(cache, batch, q, window=window), q, b, dim ** -0.5, window)


@pytest.mark.parametrize("dim,n_q,n_kv", [(256, 4, 1), (128, 8, 2), (64, 6, 3)])
@pytest.mark.parametrize("new,keys", [([1, 1, 1], [37, 700, 16]), ([40, 1, 150], [60, 33, 420])])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -3e38])
def test_attention_never_reads_what_is_masked(B, dim, n_q, n_kv, new, keys, bad):
    """Slots behind a sequence's end, before its window and in pages of nobody hold NaN, infinities or huge
    values; rows of no sequence stay as they were; strides of both kinds."""
    window = 150
    b = make_batch(new, keys, 16, n_kv, dim, torch.bfloat16, 5, head_major=dim == 128, together=dim == 64, rows_after=3, fill=bad)
    for s, (n, kk) in enumerate(zip(new, keys)):  # evicted: what no row of the sequence sees
        for p in range(0, max(0, kk - n - window + 1)):
            for t in (b["k"], b["v"]):
                t[int(b["pages"][s, p // 16]), p % 16] = bad
    cache, batch = objects(B, b)
    wide = torch.randn(b["n_rows"], n_q + 2, dim + 8, device="cuda", generator=_gen(8)).bfloat16()
    q = wide[:, 1:n_q + 1, :dim]
    out = torch.full((n_q, b["n_rows"], dim), 5.0, device="cuda", dtype=torch.bfloat16).transpose(0, 1)
    got = B.paged_attention(cache, batch, q, scale=0.11, window=window, out=out)
    assert (got[-3:] == 5).all()
    clean = dict(b, k=torch.nan_to_num(b["k"], 0, 0, 0), v=torch.nan_to_num(b["v"], 0, 0, 0))
    attn_check(got[:-3], q[:-3], dict(clean, n_rows=b["n_rows"] - 3), 0.11, window)


@pytest.mark.parametrize("dim,n_q,n_kv,new,keys", [(256, 4, 1, 3, 90), (128, 4, 2, 60, 200), (64, 3, 1, 150, 150),
                                                   (256, 4, 1, 40, 300)])
def test_attention_nan_reaches_only_rows_that_see_it(B, dim, n_q, n_kv, new, keys):
    """A key with NaN, and one whose value is infinite in a single dim, among the new tokens: earlier rows are exact,
    later ones get what the formula gives (NaN everywhere; an infinity in that dim)."""
    b = make_batch([new], [keys], 16, n_kv, dim, torch.bfloat16, 2)
    at = lambda p: (int(b["pages"][0, p // 16]), p % 16)  # noqa: E731
    p_inf, p_nan = keys - new + 1, keys - 1
    b["v"][at(p_inf)][0, 5] = float("inf")
    b["k"][at(p_nan)][0, 3] = float("nan")
    cache, batch = objects(B, b)
    q = torch.randn(new, n_q, dim, device="cuda", generator=_gen(8)).bfloat16()
    got = _np(B.paged_attention(cache, batch, q))
    want, _, _ = OS.attention(_np(q), _np(b["k"]), _np(b["v"]), b, dim ** -0.5)
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(np.isinf(got), np.isinf(want))
    assert np.isnan(got[-1, 0]).all() and np.isinf(got[1, 0, 5]) and np.isfinite(got[0]).all()
    fine = np.isfinite(want)
    assert np.abs(got - np.where(fine, want, got))[fine].max() <= 2.0 ** -6


def test_attention_bad_pages_and_empty_rows(B):
    """Page ids outside the cache hold no keys; rows at negative positions, sequences without keys and sequences
    all of whose pages are bad give zeros."""
    for new, keys in (([2, 3, 1, 1], [70, 2, 40, 90]), ([30, 40, 50, 1], [70, 25, 64, 90])):
        b = make_batch(new, keys, 16, 1, 256, torch.bfloat16, 4)
        b["pages"][0, 1], b["pages"][0, 3], b["pages"][2, :] = -1, b["k"].shape[0] + 5, 1 << 30
        b["kv_len"][3] = 0
        cache, batch = objects(B, b)
        q = torch.randn(b["n_rows"], 4, 256, device="cuda", generator=_gen(8)).bfloat16()
        got = B.paged_attention(cache, batch, q)
        want = attn_check(got, q, b, 1 / 16, 0)
        first = int(b["row_start"][2])
        assert (got[first:] == 0).all() and (got[int(b["row_start"][1])] == 0).all() and np.isfinite(want).all()


def test_attention_rows_outside_the_batch(B):
    """row_start that begins after row 0, ends before the last, or points outside the call."""
    b = make_batch([3, 4], [50, 20], 16, 2, 128, torch.float16, 4)
    b["row_start"] = np.array([2, 5, 9], np.int32)
    b["n_rows"] = 12
    cache, batch = objects(B, b)
    q = torch.randn(12, 4, 128, device="cuda", generator=_gen(8)).half()
    out = torch.full_like(q, 3.0)
    B.paged_attention(cache, batch, q, out=out)
    assert (out[:2] == 3).all() and (out[9:] == 3).all()
    attn_check(out, q, b, 128 ** -0.5, 0)
    b["row_start"] = np.array([-4, 5, 400], np.int32)  # held within the call's rows
    cache, batch = objects(B, b)
    attn_check(B.paged_attention(cache, batch, q), q, b, 128 ** -0.5, 0)


@pytest.mark.parametrize("n_q,n_kv,dim,seqs,new,ctx,window", [(4, 1, 256, 40, 1, 3000, 0), (4, 1, 256, 300, 1, 90, 0),
                                                              (8, 8, 64, 3, 400, 900, 0), (4, 1, 256, 2, 700, 2000, 512),
                                                              (16, 2, 128, 5, 7, 4000, 1000), (28, 4, 128, 1, 512, 3000, 0)])
def test_attention_split_over_the_gpu(B, n_q, n_kv, dim, seqs, new, ctx, window):
    """Enough keys that rows are divided between CTAs and joined again; the same bits every time, and the row that a
    batch of one gives within the tolerance of either."""
    rng = random.Random(seqs)
    keys = [rng.randint(new, ctx) for _ in range(seqs)]
    b = make_batch([new] * seqs, keys, 64, n_kv, dim, torch.bfloat16, 6)
    cache, batch = objects(B, b)
    q = (torch.randn(b["n_rows"], n_q, dim, device="cuda", generator=_gen(8)) * 1.5).bfloat16()
    got = B.paged_attention(cache, batch, q, window=window)
    rows = set(rng.sample(range(b["n_rows"]), min(60, b["n_rows"]))) | {0, b["n_rows"] - 1}
    attn_check(got, q, b, dim ** -0.5, window, rows)
    for _ in range(3):
        assert torch.equal(B.paged_attention(cache, batch, q, window=window), got)


def test_attention_large_strides(B):
    """A pool whose last page begins beyond 2^31 elements."""
    n_pages, page, dim = 8200, 256, 256
    pool = torch.empty(n_pages, 4, page, 1, dim, dtype=torch.bfloat16, device="cuda")  # 2.15e9 elements
    b = make_batch([1, 30], [300, 500], page, 1, dim, torch.bfloat16, 1, spare=0)
    ids = np.array([n_pages - 1 - i for i in range(b["k"].shape[0])])
    k, v = pool[:, 1], pool[:, 3]
    for i, p in enumerate(ids):
        k[p], v[p] = b["k"][i], b["v"][i]
    pages = np.where(b["pages"] >= 0, ids[np.maximum(b["pages"], 0)], -1).astype(np.int32)
    q = torch.randn(31, 4, dim, device="cuda", generator=_gen(8)).bfloat16()
    cache, batch = objects(B, dict(b, k=k, v=v, pages=pages))
    attn_check(B.paged_attention(cache, batch, q), q, b, 1 / 16, 0)
    table = B.rope_table(B.RopeConfig(dim))
    x = torch.randn(31, 1, dim, device="cuda", generator=_gen(9)).bfloat16()
    B.rope_append(table, cache, batch, q, x, x)
    last = int(pages[1, 1])
    assert torch.equal(v[last, 499 - 256, 0], x[30, 0])


# ------------------------------------------------------------------------------------ sampling
def _params(M, temperature=None, top_k=None, top_p=None, min_p=None):
    f = lambda v, t: None if v is None else torch.tensor([v[i % len(v)] for i in range(M)], dtype=t, device="cuda")  # noqa: E731
    return dict(temperature=f(temperature, torch.float32), top_k=f(top_k, torch.int32), top_p=f(top_p, torch.float32),
                min_p=f(min_p, torch.float32))


def sample_check(B, x, u, **kw):
    p = _params(x.shape[0], **kw)
    tok, prob = B.sample(x, u, want_probs=True, **p)
    tok, prob = tok.cpu().numpy(), prob.cpu().numpy()
    for r in range(x.shape[0]):
        one = {n: float(t[r]) for n, t in p.items() if t is not None}
        one["top_k"] = int(one.get("top_k", 0))
        t, pr, _ = OS.sample(_np(x[r]), float(u[r]), **one)
        assert tok[r] == t, (r, one, tok[r], t, float(u[r]))
        assert abs(prob[r] - pr) <= 2.0 ** -22 * pr + 1e-12  # one rounding to fp32, weights to 2^-31
    return tok


FILTERS = [dict(), dict(top_k=[1]), dict(top_k=[40]), dict(top_p=[0.9]), dict(top_p=[0.0]), dict(min_p=[0.1]),
           dict(temperature=[0.7], top_k=[50], top_p=[0.95], min_p=[0.02]), dict(temperature=[0.0, 1.0, -1.0, 100.0]),
           dict(top_p=[1e-6, 0.5, 0.999, 1.0]), dict(top_k=[3, 0, -5, 1000000]), dict(min_p=[1.0, 0.0, 2.0, 1e-9])]


@pytest.mark.parametrize("kw", FILTERS)
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("M,V", [(1, 1), (4, 7), (5, 1000), (3, 5003)])
def test_sample(B, dt, M, V, kw):
    x = (torch.randn(M, V, device="cuda", generator=_gen(V)) * 3).to(dt)
    unit = 4 if dt == torch.float32 else 8
    pad = torch.zeros(M, -(-V // unit) * unit, device="cuda", dtype=dt)
    pad[:, :V] = x
    sample_check(B, pad[:, :V], torch.rand(M, device="cuda", generator=_gen(2)), **kw)


@pytest.mark.parametrize("kw", [dict(), dict(top_k=[300]), dict(top_p=[0.7]), dict(top_k=[900], top_p=[0.5], min_p=[0.3])])
def test_sample_ties(B, kw):
    """Few distinct logits: the border falls among equals, and the lower indices win."""
    x = torch.randint(0, 4, (6, 2049), device="cuda", generator=_gen(3)).float()
    pad = torch.zeros(6, 2052, device="cuda")
    pad[:, :2049] = x
    sample_check(B, pad[:, :2049], torch.rand(6, device="cuda", generator=_gen(4)), **kw)
    sample_check(B, torch.zeros(3, 4096, device="cuda"), torch.tensor([0.0, 0.5, 0.999999], device="cuda"), **kw)


def test_sample_masked_and_odd_rows(B):
    """Rows with -inf, NaN, +inf, the type's lowest value, one token, none; u at and beyond its ends."""
    inf, nan, low = float("inf"), float("nan"), torch.finfo(torch.float32).min
    rows = [[-inf] * 8, [nan] * 8, [nan, -inf, 1.0, -inf, nan, 0.5, -inf, 1.0], [inf, 0, inf, nan, 3, -inf, inf, 1],
            [low] * 8, [low, low, 0.0, low, low, 0.0, low, low], [-inf, -inf, -5e37, -inf, -inf, -inf, -inf, -inf],
            [0.0, -0.0, 0.0, -0.0, -1.0, -0.0, 0.0, -0.0]]
    x = torch.tensor(rows, device="cuda")
    for u in (0.0, 0.4, 0.75, 0.99999994, 1.0, 7.0, -1.0, nan, inf):
        for kw in (dict(), dict(top_k=[2]), dict(top_p=[0.6]), dict(min_p=[0.5]), dict(temperature=[0.0]),
                   dict(temperature=[1e-38]), dict(temperature=[inf]), dict(temperature=[nan], top_p=[nan], min_p=[nan])):
            if kw.get("temperature") == [inf]:  # equal weights of what is finite
                tok = B.sample(x, torch.full((8,), u, device="cuda"), **_params(8, **kw)).cpu().tolist()
                assert tok[0] == tok[1] == -1 and tok[2] in (2, 5, 7) and tok[6] == 2
                continue
            sample_check(B, x, torch.full((8,), u, device="cuda"), **kw)


@pytest.mark.parametrize("V", [32000, 50257, 262144])
def test_sample_large(B, V):
    """A vocabulary's worth of logits, smooth and flat; every filter; the fp32 logits of a decode batch."""
    pad = -(-V // 4) * 4
    x = torch.randn(8, pad, device="cuda", generator=_gen(V)) * torch.tensor([3, 0.01, 1, 6, 3, 0, 1, 2.0], device="cuda")[:, None]
    x[4, 100:120] += 15
    x = x[:, :V]
    u = torch.rand(8, device="cuda", generator=_gen(7))
    got = {}
    for name, kw in (("all", dict(temperature=[0.8], top_k=[64], top_p=[0.95], min_p=[0.02])), ("p", dict(top_p=[0.9])),
                     ("k", dict(top_k=[1000])), ("m", dict(min_p=[0.01])), ("none", dict())):
        p = _params(8, **kw)
        got[name] = B.sample(x, u, want_probs=True, **p)
        for r in range(8):
            row = _np(x[r])
            t, pr = _fast_oracle(row, float(u[r]), **{n: float(v[r]) for n, v in p.items() if v is not None})
            assert int(got[name][0][r]) == t, (name, r)
            assert abs(float(got[name][1][r]) - pr) <= 2.0 ** -20 * pr + 1e-12


def _fast_oracle(row, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """The oracle's rule on a long row by sorting (long double sums)."""
    w = np.exp((row - row.max()) / temperature)
    order = np.lexsort((np.arange(len(row)), -row))
    if top_k > 0:
        order = order[:int(top_k)]
    if top_p < 1:
        c = np.cumsum(w[order], dtype=np.longdouble)
        order = order[:1 + int(np.searchsorted(c[:-1], np.longdouble(top_p) * c[-1], side="left"))]
    order = np.sort(order[w[order] >= min_p])
    c = np.cumsum(w[order], dtype=np.longdouble)
    i = min(int(np.searchsorted(c, np.longdouble(u) * c[-1], side="right")), len(order) - 1)
    return int(order[i]), float(w[order[i]] / c[-1])


def test_sample_follows_the_distribution(B):
    """Equally spaced u: the counts are the probabilities' to a step at either border."""
    x = torch.tensor([[0.3, -1.0, 2.0, 0.0, 1.9, -3.0, 0.5, 0.1]], device="cuda")
    n = 4096
    u = (torch.arange(n, device="cuda") + 0.5) / n
    tok = B.sample(x.expand(n, 8), u)
    p = torch.softmax(x.double(), 1)[0] * n
    assert (torch.bincount(tok.long(), minlength=8) - p).abs().max() <= 1 and (tok[1:] >= tok[:-1]).all()


# ------------------------------------------------------------------ together; streams and graphs
def _step(B, table, cache, batch, qkv, n_q, n_kv, wo, head, u, ws=None):
    q, k, v = qkv[:, :n_q], qkv[:, n_q:n_q + n_kv], qkv[:, n_q + n_kv:]
    q = B.rope_append(table, cache, batch, q, k, v)
    o = B.paged_attention(cache, batch, q, ws=ws)
    x = B.linear_bf16(wo, o.view(o.shape[0], -1), ws=ws)
    logits, _ = B.lm_head(head, B.W8A8_PREC_BF16, x, ws=ws)
    return B.sample(logits, u), o, logits


@pytest.mark.parametrize("new,keys", [([1, 1, 1, 1], [3, 100, 33, 64]), ([30, 1, 17], [30, 200, 90])])
def test_operators_together(B, new, keys):
    """Append, attention, projection, lm_head and sampling in one stream, as a serving step strings them; and
    captured, with lengths and pages changed between replays."""
    n_q, n_kv, dim, V = 4, 1, 256, 2048
    b = make_batch(new, keys, 16, n_kv, dim, torch.bfloat16, 5, spare=6)
    cache, batch = objects(B, b)
    T = b["n_rows"]
    qkv = torch.randn(T, n_q + 2 * n_kv, dim, device="cuda", generator=_gen(1)).bfloat16()
    wo = (torch.randn(256, n_q * dim, device="cuda", generator=_gen(2)) * 0.05).bfloat16()
    head = B.HeadWeights(V, 256, bf16=(torch.randn(V, 256, device="cuda", generator=_gen(3)) * 0.2).bfloat16())
    u = torch.rand(T, device="cuda", generator=_gen(4))
    table = B.rope_table(B.RopeConfig(dim))
    ws = B.Workspace(torch.device("cuda", 0))
    ws.get(64 << 20)
    tok, o, logits = _step(B, table, cache, batch, qkv, n_q, n_kv, wo, head, u, ws)
    attn_check(o, B.rope_append(table, cache, batch, qkv[:, :n_q], qkv[:, n_q:n_q + n_kv], qkv[:, n_q + n_kv:]), b, 1 / 16, 0)
    for r in range(T):
        assert int(tok[r]) == OS.sample(_np(logits[r]), float(u[r]))[0]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        gt, go, gl = _step(B, table, cache, batch, qkv, n_q, n_kv, wo, head, u, ws)
    for change in (0, 1):
        if change:  # one position back for every sequence but the first, other pages for it
            b["kv_len"][1:] -= 1
            b["pages"][0, 0] = b["k"].shape[0] - 1 if (b["pages"] != b["k"].shape[0] - 1).all() else b["pages"][0, 0]
            batch.kv_len.copy_(torch.from_numpy(b["kv_len"]))
            batch.pages.copy_(torch.from_numpy(b["pages"]))
        g.replay()
        torch.cuda.synchronize()
        kept = [t.clone() for t in (gt, go, gl)]
        want = _step(B, table, cache, batch, qkv, n_q, n_kv, wo, head, u, ws)
        for a, w in zip(kept, want):
            assert torch.equal(a, w)


def test_two_streams_and_two_graphs(B):
    """Calls without a workspace on two streams at once, and two captured graphs replayed side by side: each has
    scratch of its own."""
    shapes = [([1] * 24, [1500] * 24), ([90, 200], [900, 1200])]
    work = []
    for i, (new, keys) in enumerate(shapes):
        b = make_batch(new, keys, 64, 1, 256, torch.bfloat16, i)
        cache, batch = objects(B, b)
        q = torch.randn(b["n_rows"], 4, 256, device="cuda", generator=_gen(i)).bfloat16()
        work.append((cache, batch, q, B.paged_attention(cache, batch, q)))
    streams = [torch.cuda.Stream() for _ in work]
    torch.cuda.synchronize()
    outs = [[], []]
    for _ in range(6):
        for i, (cache, batch, q, _) in enumerate(work):
            outs[i].append(B.paged_attention(cache, batch, q, stream=streams[i]))
    torch.cuda.synchronize()
    graphs = []
    for i, (cache, batch, q, _) in enumerate(work):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            y = B.paged_attention(cache, batch, q)
        graphs.append((g, y))
    for _ in range(4):
        for i, (g, _) in enumerate(graphs):
            with torch.cuda.stream(streams[i]):
                g.replay()
    torch.cuda.synchronize()
    for i, (_, _, _, want) in enumerate(work):
        assert all(torch.equal(y, want) for y in outs[i]) and torch.equal(graphs[i][1], want)


def test_calls_of_nothing(B):
    b = make_batch([0, 0], [5, 0], 16, 1, 256, torch.bfloat16, 1)
    cache, batch = objects(B, b)
    q = torch.empty(0, 4, 256, device="cuda", dtype=torch.bfloat16)
    assert B.paged_attention(cache, batch, q).shape == q.shape
    assert B.rope_append(B.rope_table(B.RopeConfig(256)), cache, batch, q, q[:, :1], q[:, :1]).shape == q.shape
    none = B.PagedBatch(torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros(0, dtype=torch.int32, device="cuda"),
                        torch.zeros(0, 4, dtype=torch.int32, device="cuda"))
    q = torch.ones(3, 4, 256, device="cuda", dtype=torch.bfloat16)
    assert torch.equal(B.paged_attention(cache, none, q, out=q.clone()), q)
    assert B.sample(torch.empty(0, 8, device="cuda"), torch.empty(0, device="cuda")).shape == (0,)


# ------------------------------------------------------------------- calls at the edge of what is allowed
@pytest.mark.parametrize("new,n_q,n_kv,dim", [([1, 2, 1], 8, 2, 64), ([1, 1, 1], 4, 1, 256), ([40, 3, 130], 8, 2, 128),
                                              ([20, 90, 1], 4, 1, 256)])
def test_attention_pages_in_common(B, new, n_q, n_kv, dim):
    """Sequences that share their first pages, and one that holds the same page twice."""
    keys = [n + 150 for n in new]
    b = make_batch(new, keys, 32, n_kv, dim, torch.bfloat16, 12)
    b["pages"][1, :3] = b["pages"][0, :3]
    b["pages"][2, 1] = b["pages"][2, 0]
    cache, batch = objects(B, b)
    q = (torch.randn(b["n_rows"], n_q, dim, device="cuda", generator=_gen(8)) * 1.5).bfloat16()
    attn_check(B.paged_attention(cache, batch, q), q, b, dim ** -0.5, 0)


@pytest.mark.parametrize("new,n_q,n_kv,dim", [([1, 2], 8, 2, 64), ([1, 1], 4, 1, 256), ([40, 130], 8, 2, 128), ([50, 90], 4, 1, 256)])
def test_attention_values_near_the_types_end(B, new, n_q, n_kv, dim):
    """Values of 2^126 meet weights of up to 2^8: sums on the way overflow fp32, the result does not."""
    b = make_batch(new, [n + 200 for n in new], 16, n_kv, dim, torch.bfloat16, 13)
    b["v"].copy_(torch.where(b["v"] > 0, 2.0 ** 126, 2.0 ** 125))
    b["k"].copy_(b["k"] * torch.linspace(0.1, 3, b["k"].shape[1], device="cuda")[None, :, None, None])  # the maximum grows on the way
    cache, batch = objects(B, b)
    q = (torch.randn(b["n_rows"], n_q, dim, device="cuda", generator=_gen(8)) * 1.5).bfloat16()
    got = B.paged_attention(cache, batch, q)
    assert torch.isfinite(got).all()
    attn_check(got, q, b, dim ** -0.5, 0)


@pytest.mark.parametrize("new,n_q,dim", [([1, 1, 2, 1], 4, 256), ([30, 1, 50, 2], 4, 128)])
def test_lengths_beyond_the_pages(B, new, n_q, dim):
    """kv_len past the page table's columns counts as all of them; a negative one as none."""
    b = make_batch(new, [60, 64, 64, 30], 16, 1, dim, torch.bfloat16, 14)
    b["kv_len"] = np.array([60, 2 ** 31 - 1, 65, -2 ** 31], np.int32)
    cache, batch = objects(B, b)
    q = torch.randn(b["n_rows"], n_q, dim, device="cuda", generator=_gen(8)).bfloat16()
    got = B.paged_attention(cache, batch, q)
    attn_check(got, q, b, dim ** -0.5, 0)
    assert (got[int(b["row_start"][3]):] == 0).all()
    x = torch.randn(b["n_rows"], 1, dim, device="cuda", generator=_gen(9)).bfloat16()
    B.rope_append(B.rope_table(B.RopeConfig(dim)), cache, batch, q, x, x)
    assert torch.equal(b["v"][int(b["pages"][1, 3]), 15, 0], x[int(b["row_start"][2]) - 1, 0])


@pytest.mark.parametrize("n_q,n_kv,dim,most", [(4, 2, 64, 1), (4, 1, 256, 40), (8, 2, 128, 20)])
def test_attention_many_sequences(B, n_q, n_kv, dim, most):
    """More sequences than a block has threads, most of them without rows."""
    rng = random.Random(3)
    new = [rng.choice([0, 0, 0, 1, 1, most]) if i else 1 for i in range(1500)]
    keys = [n + rng.randint(0, 40) for n in new]
    b = make_batch(new, keys, 16, n_kv, dim, torch.float16, 15)
    cache, batch = objects(B, b)
    q = (torch.randn(b["n_rows"], n_q, dim, device="cuda", generator=_gen(8)) * 1.5).half()
    rows = set(rng.sample(range(b["n_rows"]), 200)) | {0, b["n_rows"] - 1}
    got = B.paged_attention(cache, batch, q)
    attn_check(got, q, b, dim ** -0.5, 0, rows)
    low = dict(b, max_new=1)  # the hint too small: slower, the same
    cache, batch = objects(B, low)
    attn_check(B.paged_attention(cache, batch, q), q, b, dim ** -0.5, 0, rows)


def test_sample_widest(B):
    """The largest vocabulary, rows of the type's smallest alignment."""
    V = 1048576
    for dt, unit in ((torch.float32, 4), (torch.bfloat16, 8)):
        x = torch.empty(2, V + unit, device="cuda", dtype=dt)
        x.copy_((torch.randn(2, V + unit, device="cuda", generator=_gen(7)) * 2).to(dt))
        sample_check(B, x[:, :V], torch.tensor([0.3, 0.999], device="cuda"), temperature=[0.8], top_k=[200, 3], top_p=[0.9])


@pytest.mark.parametrize("n_q,n_kv,dim,seqs,new,ctx,window", [
    (4, 1, 256, 32, 8, 4000, 1024), (4, 1, 256, 64, 8, 4000, 0), (16, 1, 256, 20, 2, 3000, 0), (8, 2, 256, 30, 25, 2500, 700),
    (28, 4, 128, 30, 3, 4000, 0), (24, 8, 64, 20, 10, 4000, 0), (4, 1, 256, 3, 70, 30000, 0)])
def test_attention_few_rows_over_many_keys(B, n_q, n_kv, dim, seqs, new, ctx, window):
    """Chunks that leave most of a row tile empty, or one of an item's two: its warps do nothing and are far ahead."""
    rng = random.Random(seqs + dim)
    b = make_batch([new] * seqs, [rng.randint(ctx // 2, ctx) for _ in range(seqs)], 64, n_kv, dim, torch.bfloat16, 16)
    cache, batch = objects(B, b)
    q = (torch.randn(b["n_rows"], n_q, dim, device="cuda", generator=_gen(8)) * 1.5).bfloat16()
    got = B.paged_attention(cache, batch, q, window=window)
    rows = set(rng.sample(range(b["n_rows"]), 24)) | {0, b["n_rows"] - 1}
    attn_check(got, q, b, dim ** -0.5, window, rows)
    for _ in range(10):
        assert torch.equal(B.paged_attention(cache, batch, q, window=window), got)


@pytest.mark.parametrize("kw", [dict(), dict(temperature=[0.7, 0.0], top_k=[50, 3], top_p=[0.95], min_p=[0.02])])
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("M,V,first", [(5, 1, 1), (6, 3, 0), (5, 1001, 0), (4, 5002, 3), (3, 33001, 2), (70, 8207, 1)])
def test_sample_rows_that_begin_anywhere(B, dt, M, V, first, kw):
    """Contiguous rows of an odd length, at any offset; what lies before the first and behind the last is larger than any
    logit of theirs, and so is each row's neighbour."""
    x = torch.full((M * V + 16,), float("inf"), device="cuda", dtype=dt)
    rows = x[first:first + M * V].view(M, V)
    rows.copy_(((torch.randn(M, V, device="cuda", generator=_gen(V)) * 3) + 8 * torch.arange(M, device="cuda")[:, None]).to(dt))
    sample_check(B, rows, torch.rand(M, device="cuda", generator=_gen(2)), **kw)
    if M > 2:  # infinities within a row of the same kind
        rows[1, V // 2] = float("inf")
        rows[2].fill_(float("-inf"))
        sample_check(B, rows, torch.rand(M, device="cuda", generator=_gen(5)), **kw)
