"""A paged cache in 4 bits on the GPU against the 64-bit oracle: the append, its codes bit for bit, attention over it, its
pages' values, and a layer of 4-bit operators together."""
import random

import numpy as np
import pytest
import torch

from oracle import fp4 as O4
from oracle import serving as OS
from test_gpu_serving import ATTN, make_batch

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


def fp4_batch(new, keys, page, n_kv, dim, seed, heads_first=False, exps=(1, -2), fill=None, tight=False, **kw):
    """make_batch with its cache in 4 bits: codes and scales as views of one pool (with room between heads, or tight), and what
    they stand for as k and v.  fill: scale bytes of the slots that hold no key of the batch."""
    b = make_batch(new, keys, page, n_kv, dim, torch.float32, seed, **kw)
    n = b["k"].shape[0]
    live = torch.zeros(n, page, dtype=torch.bool, device="cuda")
    for s, m in enumerate(keys):
        for p in range(m):
            live[int(b["pages"][s, p // page]), p % page] = True
    for name, exp in (("k", exps[0]), ("v", exps[1])):
        x = b[name]
        m = x.abs().unflatten(-1, (-1, 16)).amax(-1) * 2.0 ** -exp
        scale = (m / 6).clamp_max(448).to(torch.float8_e4m3fn)
        unit = scale.float()[..., None] * 2.0 ** exp
        a = x.unflatten(-1, (-1, 16)).abs() / torch.where(unit > 0, unit, torch.ones_like(unit))
        c = torch.zeros_like(a, dtype=torch.uint8)
        for mid in (0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0):  # (any codes will do)
            c += a > mid
        c = (c + 8 * (x.unflatten(-1, (-1, 16)) < 0).to(torch.uint8)).flatten(-2)
        bits = scale.view(torch.uint8)
        if fill is not None:
            bits[~live] = fill
        shape = (n, n_kv, page) if heads_first else (n, page, n_kv)
        pool = torch.randint(0, 256, (*shape, dim // 2 + 32), device="cuda", generator=_gen(seed + 7), dtype=torch.int32).to(torch.uint8)
        spool = torch.full((*shape, dim // 8), 127, device="cuda", dtype=torch.uint8)
        codes, scales = pool[..., :dim // 2], spool[..., dim // 16:]
        if tight:
            codes, scales = pool[..., :dim // 2].contiguous(), spool[..., :dim // 16].contiguous()
        elif dim == 64:
            codes, scales = pool[..., 16:dim // 2 + 16], spool[..., :dim // 16]
        if heads_first:
            codes, scales = codes.transpose(1, 2), scales.transpose(1, 2)
        codes.copy_(c[..., 0::2] | (c[..., 1::2] << 4))
        scales.copy_(bits)
        if spool.data_ptr() % 16 or scales.data_ptr() % 16:  # an aligned first byte
            scales = scales.contiguous()
        b[name + "4"], b[name + "s"] = codes, scales
    b["exps"] = exps
    return refresh(b)


def refresh(b):
    for name, exp in zip(("k", "v"), b["exps"]):
        b[name] = torch.from_numpy(O4.cache_values(O4.unpack(b[name + "4"].cpu().numpy()), b[name + "s"].cpu().numpy(), exp)).cuda()
    return b


def objects(B, b):
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    return (B.PagedCacheFp4(b["k4"], b["v4"], b["ks"], b["vs"], *b["exps"]),
            B.PagedBatch(dev(b["row_start"]), dev(b["kv_len"]), dev(b["pages"]), max_new=b["max_new"]))


def attn_check(got, q, b, scale, window, rows=None):
    """Per output: half a step of the result; weights rounded to the type and their sum (2 half-steps of the weighted |v|);
    scores summed in fp32 (dim 2^-24 of the largest sum of |q k|, twice: numerator and sum) and exponentials and sums of 2^-20;
    fp16 also half its smallest step.  Where weights are fp16, lifted by 2^12 against a reference that is at most the row's
    largest, one below 2^-14 is off by up to 2^-25, 2^-37 of the largest, and vanishes below that: n 2^-37 of the largest |v|
    over n keys (every weight's part of the sum is at most its share of the largest weight, which the sum holds)."""
    want, mass, mag = OS.attention(_np(q), _np(b["k"]), _np(b["v"]), b, scale, window, rows)
    dt = q.dtype
    eps, dim = torch.finfo(dt).eps / 2, q.shape[2]
    delta = scale * dim * 2.0 ** -24 * mag
    vanish = float(np.max(b["kv_len"], initial=1)) if window == 0 else float(window)
    vanish = min(vanish, b["pages"].shape[1] * b["k"].shape[1]) * 2.0 ** -37 * float(torch.nan_to_num(b["v"], 0, 0, 0).abs().max())
    tol = eps * np.abs(want) + (2 * eps + 2 * delta[..., None] + 2.0 ** -20) * mass + (2.0 ** -25 if dt == torch.float16 else 1e-38)
    got, some = _np(got), ~np.isnan(want).all(axis=(1, 2))
    err = np.abs(got - want)[some] - tol[some] - vanish
    assert err.max() <= 0, (float(err.max()), np.argwhere(err > 0)[:4].tolist())
    return want


# -------------------------------------------------------------------------------------- append
@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("new,keys,page,n_q,n_kv,dim,rot,inter,norm,heads_first", [
    ([1], [1], 16, 4, 1, 256, 256, False, True, False),
    ([1, 1, 1, 1, 1], [17, 1, 16, 64, 33], 16, 4, 1, 256, 256, False, True, True),
    ([5, 0, 40, 1], [5, 9, 100, 64], 32, 8, 2, 128, 64, True, True, True),
    ([3, 20], [130, 20], 64, 5, 5, 64, 64, True, False, False),
    ([7, 30], [40, 30], 16, 2, 2, 64, 16, False, True, True), ([9], [9], 16, 2, 1, 256, 48, False, True, False),
    ([300], [311], 256, 28, 4, 128, 128, False, False, True), ([200, 90], [500, 90], 64, 4, 1, 256, 256, False, True, False)])
def test_append(B, dt, new, keys, page, n_q, n_kv, dim, rot, inter, norm, heads_first):
    """Codes and scales of keys and values equal the oracle's from the 64-bit keys: none is left to the rounding of fp32."""
    b = fp4_batch(new, keys, page, n_kv, dim, 11, heads_first, rows_after=2)
    cache, batch = objects(B, b)
    T = b["n_rows"]
    qkv = (torch.randn(T, n_q + 2 * n_kv, dim, device="cuda", generator=_gen(5)) * 3).to(DT[dt])
    q, k, v = qkv[:, :n_q], qkv[:, n_q:n_q + n_kv], qkv[:, n_q + n_kv:]
    qn, kn = ((1 + 0.3 * torch.randn(dim, device="cuda", generator=_gen(6 + i))) if norm else None for i in (0, 1))
    table = B.rope_table(B.RopeConfig(rot, base=1e4, interleaved=inter, scaling="linear", factor=4.0))
    before = {n: b[n].clone() for n in ("k4", "v4", "ks", "vs")}
    out = torch.full((T, n_q, dim), 9.0, device="cuda", dtype=DT[dt])
    eps = float(np.float32(1e-5))
    got = B.fp4_rope_append(table, cache, batch, q, k, v, q_norm=qn, k_norm=kn, eps=eps, q_out=out)
    assert got is out and (out[T - 2:] == 9).all()  # rows of no sequence
    f, s = OS.rope_frequencies(rot, 1e4, "linear", factor=4.0)
    nq, nk = (OS.rms_norm(_np(t), None if w is None else _np(w), eps) for t, w in ((q, qn), (k, kn)))
    want = {n: t.cpu().numpy().copy() for n, t in before.items()}
    for r, seq, pos, _ in OS.rows_of(b, page):
        y = OS.rope(nq[r:r + 1], [pos], f, s, inter)[0]
        tol = torch.finfo(DT[dt]).eps / 2 * np.abs(y) + (2.0 ** -21 + (dim / 16 + 8) * 2.0 ** -24) * np.abs(nq[r]).max() + 2.0 ** -25
        assert (np.abs(_np(out[r]) - y) <= tol).all()
        at = OS.place(b, b["k"].shape[0], page, seq, pos)
        for name, x, e in (("k", OS.rope(nk[r:r + 1], [pos], f, s, inter)[0], b["exps"][0]), ("v", _np(v[r]), b["exps"][1])):
            c, sc = O4.cache_quantise(x, e)
            want[name + "4"][at], want[name + "s"][at] = O4.pack(c), sc
    for n in ("ks", "vs"):
        np.testing.assert_array_equal(b[n].cpu().numpy(), want[n])
    for n in ("k4", "v4"):  # (a zero's sign is not a value)
        np.testing.assert_array_equal(O4.values_of(O4.unpack(b[n].cpu().numpy())), O4.values_of(O4.unpack(want[n])))


def test_append_borders(B):
    """Values on the borders between codes and between scales, NaN and infinities, and values beyond the largest scale."""
    b = fp4_batch([8], [8], 16, 1, 64, 3, exps=(0, 3))
    cache, batch = objects(B, b)
    x = torch.randint(-24, 25, (8, 3, 64), device="cuda", generator=_gen(1)).float() * 0.25
    x[0, 2] *= 4096
    x[1, 1:, 5], x[2, 1:, 20], x[3, 1:, 63] = float("nan"), float("inf"), -60000.0
    x[4] = 0
    x[5, :, :16] = 2.0 ** -9 * 6
    x[5, :, 1:16] *= 0.25
    x = x.bfloat16()
    table = B.rope_table(B.RopeConfig(16))
    x[:, :, :16][1:4] = 0  # what turns: exact only at zero, and at position 0
    B.fp4_rope_append(table, cache, batch, x[:, :1], x[:, 1:2], x[:, 2:])
    page = int(b["pages"][0, 0])
    f, s = OS.rope_frequencies(16, 1e4)
    k = OS.rope(_np(x[:, 1:2]), range(8), f, s, False)[:, 0]
    for name, y, e in (("k", k, 0), ("v", _np(x[:, 2]), 3)):
        c, sc = O4.cache_quantise(y, e)
        np.testing.assert_array_equal(b[name + "s"][page, :8, 0].cpu().numpy(), sc)
        got = O4.unpack(b[name + "4"][page, :8, 0].cpu().numpy())
        np.testing.assert_array_equal(O4.values_of(got), O4.values_of(c))


@pytest.mark.parametrize("dim,rot,inter", [(256, 256, False), (128, 64, True), (64, 32, False)])
def test_append_beyond_the_range_of_fp32(B, dim, rot, inter):
    """Norms whose sum of squares fp32 does not hold (above it, and below it without an eps), and rotations that leave it."""
    table = B.rope_table(B.RopeConfig(rot, interleaved=inter))
    f, s = OS.rope_frequencies(rot, 1e4)
    qn = (1 + 0.3 * torch.randn(dim, device="cuda", generator=_gen(1)))
    for scale, norm, eps, exps in ((1e30, qn, 1e-5, (0, 0)), (1e-30, qn, 0.0, (-1, 0)), (0.8e38, None, 1e-5, (100, 99)),
                                   (0.8e38, None, 1e-5, (-100, -90)), (1e-30, qn, 1e-5, (-80, -90))):
        b = fp4_batch([7, 1], [90, 60], 16, 2, dim, 5, exps=exps)
        cache, batch = objects(B, b)
        x = (torch.randn(8, 5, dim, device="cuda", generator=_gen(2)).clamp(-4, 4) * scale).bfloat16()
        x[3, 1, 5], x[4, 2, 7], x[5, 2] = float("inf"), float("nan"), 0.0
        want = {n: b[n].cpu().numpy().copy() for n in ("k4", "v4", "ks", "vs")}
        B.fp4_rope_append(table, cache, batch, x[:, :1], x[:, 1:3], x[:, 3:], k_norm=norm, eps=eps)
        eps = float(np.float32(eps))
        for r, seq, pos, _ in OS.rows_of(b, 16):
            at = OS.place(b, b["k"].shape[0], 16, seq, pos)
            with np.errstate(all="ignore"):
                k = _np(x[r:r + 1, 1:3])
                k = OS.rope(k if norm is None else OS.rms_norm(k, _np(norm), eps), [pos], f, s, inter)[0]
                for name, y, e in (("k", k, exps[0]), ("v", _np(x[r, 3:]), exps[1])):
                    c, sc = O4.cache_quantise(y, e)
                    want[name + "4"][at], want[name + "s"][at] = O4.pack(c), sc
        for n in ("ks", "vs"):
            np.testing.assert_array_equal(b[n].cpu().numpy(), want[n])
        for n in ("k4", "v4"):
            np.testing.assert_array_equal(O4.values_of(O4.unpack(b[n].cpu().numpy())), O4.values_of(O4.unpack(want[n])))


def test_append_leaves_bad_pages_alone(B):
    b = fp4_batch([2, 3, 1], [40, 2, 9], 16, 2, 64, 3)
    b["pages"][0, 2] = b["k"].shape[0]
    b["pages"][2, 0] = -7
    cache, batch = objects(B, b)
    before = {n: b[n].clone() for n in ("k4", "v4", "ks", "vs")}
    x = torch.randn(6, 8, 64, device="cuda", generator=_gen(1)).bfloat16()
    table = B.rope_table(B.RopeConfig(64))
    q = x[:, :4].clone()
    assert B.fp4_rope_append(table, cache, batch, q, x[:, 4:6], x[:, 6:], q_out=q) is q  # in place
    pos = torch.tensor([38, 39, -1, 0, 1, 8], device="cuda", dtype=torch.int32)
    assert (q.float() - B.rope(table, x[:, :4], pos).float()).abs().max() <= 2.0 ** -6
    page = int(b["pages"][1, 0])
    for n, t in before.items():
        changed = {(int(i), int(j)) for i, j in torch.nonzero((b[n] != t).flatten(2).any(2)).cpu()}
        assert changed <= {(page, 0), (page, 1)} and (n[1] != "4" or len(changed) == 2)


def test_values_of_pages(B):
    b = fp4_batch([1, 1], [40, 33], 32, 3, 128, 4, True, exps=(-3, 5))
    cache, _ = objects(B, b)
    for dt in (torch.bfloat16, torch.float16, torch.float32):
        k, v = B.fp4_paged_values(cache, dt)
        assert k.dtype == dt and torch.equal(k, b["k"].to(dt)) and torch.equal(v, b["v"].to(dt))
    ids = torch.tensor([2, 0, -1, 2, b["k"].shape[0], 1], device="cuda", dtype=torch.int32)
    k, v = B.fp4_paged_values(cache, torch.float32, pages=ids)
    for i, p in enumerate(ids.tolist()):
        for got, all_ in ((k, b["k"]), (v, b["v"])):
            assert torch.equal(got[i], all_[p].float() if 0 <= p < all_.shape[0] else torch.zeros_like(got[i]))
    assert B.fp4_paged_values(cache, pages=ids[:0])[0].shape == (0, 32, 3, 128)
    with pytest.raises(ValueError):
        B.fp4_paged_values(cache, pages=ids.long())


# ----------------------------------------------------------------------------------- attention
@pytest.mark.parametrize("tight", [False, True])
@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("new,keys,page,n_q,n_kv,dim,window", ATTN)
def test_attention(B, dt, new, keys, page, n_q, n_kv, dim, window, tight):
    """Pools with room between the heads and without (where a page's scales are one piece if its slots follow one another)."""
    b = fp4_batch(new, keys, page, n_kv, dim, len(keys) + dim, heads_first=page != 16, tight=tight)
    cache, batch = objects(B, b)
    q = (torch.randn(b["n_rows"], n_q, dim, device="cuda", generator=_gen(8)) * 1.5).to(DT[dt])
    attn_check(B.fp4_paged_attention(cache, batch, q, window=window), q, b, dim ** -0.5, window)


@pytest.mark.parametrize("dim,n_q,n_kv", [(256, 4, 1), (128, 8, 2), (64, 6, 3), (128, 16, 1)])
@pytest.mark.parametrize("new,keys", [([1, 1, 1], [37, 700, 16]), ([40, 1, 150], [60, 33, 420])])
@pytest.mark.parametrize("bad", [127, 255, 126])
def test_attention_never_reads_what_is_masked(B, dim, n_q, n_kv, new, keys, bad):
    """Slots behind a sequence's end, before its window and in pages of nobody hold NaN or the largest scales; rows of no
    sequence stay as they were; strides of both kinds."""
    window = 150
    b = fp4_batch(new, keys, 32, n_kv, dim, 5, heads_first=dim == 128, rows_after=3, fill=bad, tight=n_q == 4 or n_q == 8)
    for s, (n, kk) in enumerate(zip(new, keys)):  # evicted: what no row of the sequence sees
        for p in range(0, max(0, kk - n - window + 1)):
            for t in (b["ks"], b["vs"]):
                t[int(b["pages"][s, p // 32]), p % 32] = bad
    refresh(b)
    cache, batch = objects(B, b)
    wide = torch.randn(b["n_rows"], n_q + 2, dim + 8, device="cuda", generator=_gen(8)).bfloat16()
    q = wide[:, 1:n_q + 1, :dim]
    out = torch.full((n_q, b["n_rows"], dim), 5.0, device="cuda", dtype=torch.bfloat16).transpose(0, 1)
    got = B.fp4_paged_attention(cache, batch, q, scale=0.11, window=window, out=out)
    assert (got[-3:] == 5).all()
    clean = dict(b, k=torch.nan_to_num(b["k"], 0, 0, 0), v=torch.nan_to_num(b["v"], 0, 0, 0))
    attn_check(got[:-3], q[:-3], dict(clean, n_rows=b["n_rows"] - 3), 0.11, window)


@pytest.mark.parametrize("dim,n_q,n_kv,new,keys", [(256, 4, 1, 3, 90), (128, 4, 2, 60, 200), (64, 3, 1, 150, 150),
                                                   (256, 4, 1, 40, 300), (64, 4, 1, 3, 500)])
def test_attention_nan_reaches_only_rows_that_see_it(B, dim, n_q, n_kv, new, keys):
    """A key with a NaN block and one whose values have one, among the new tokens: earlier rows are exact, later ones get what
    the formula gives."""
    b = fp4_batch([new], [keys], 16, n_kv, dim, 2)
    at = lambda p: (int(b["pages"][0, p // 16]), p % 16)  # noqa: E731
    p_val, p_key = keys - new + 1, keys - 1
    b["vs"][at(p_val)][0, 1] = 127
    b["ks"][at(p_key)][0, 0] = 127
    refresh(b)
    cache, batch = objects(B, b)
    q = torch.randn(new, n_q, dim, device="cuda", generator=_gen(8)).bfloat16()
    got = _np(B.fp4_paged_attention(cache, batch, q))
    want, _, _ = OS.attention(_np(q), _np(b["k"]), _np(b["v"]), b, dim ** -0.5)
    assert np.array_equal(np.isnan(got), np.isnan(want))
    assert np.isnan(got[-1, 0]).all() and np.isnan(got[1, 0, 16:32]).all() and np.isfinite(got[0]).all()
    fine = np.isfinite(want)
    assert np.abs(got - np.where(fine, want, got))[fine].max() <= 2.0 ** -6


@pytest.mark.parametrize("new", [1, 3, 30])
def test_attention_queries_that_are_not_finite(B, new):
    """A row whose query holds a NaN or an infinity is NaN; rows without keys give zeros all the same; the others are exact."""
    b = fp4_batch([new, new], [200, 90], 16, 1, 128, 2)
    cache, batch = objects(B, b)
    q = torch.randn(2 * new, 4, 128, device="cuda", generator=_gen(8)).bfloat16()
    q[0, 1, 7], q[new, 2, 100], q[new, 3] = float("nan"), float("inf"), 3e38
    got = B.fp4_paged_attention(cache, batch, q)
    assert got[0, 1].isnan().all() and got[new, 2].isnan().all()
    q[0, 1], q[new, 2] = 0, 0
    keep = torch.ones(2 * new, 4, dtype=torch.bool, device="cuda")
    keep[0, 1] = keep[new, 2] = keep[new, 3] = False
    want = B.fp4_paged_attention(cache, batch, q)
    assert torch.equal(got[keep], want[keep])
    b["kv_len"][:] = 0
    _, batch = objects(B, b)
    assert (B.fp4_paged_attention(cache, batch, torch.full_like(q, float("nan"))) == 0).all()


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("new,n_q,dim", [(1, 4, 256), (2, 4, 64), (40, 4, 128)])
def test_attention_queries_of_many_sizes(B, dt, new, n_q, dim):
    """Rows of queries from the smallest numbers to large ones, and dims of one query many binades apart."""
    b = fp4_batch([new, new], [300, 77], 16, 1, dim, 5, exps=(0, 0))
    cache, batch = objects(B, b)
    q = torch.randn(2 * new, n_q, dim, device="cuda", generator=_gen(8))
    q[:, 0] *= 2.0 ** -30 if dt == "bf16" else 2.0 ** -14
    q[:, 1] *= torch.exp2(-torch.arange(dim, device="cuda") % 12.0)
    q[:, 2] *= 2.0 ** -120 if dt == "bf16" else 2.0 ** -20
    q = q.to(DT[dt])
    attn_check(B.fp4_paged_attention(cache, batch, q), q, b, dim ** -0.5, 0)


def test_attention_bad_pages_and_empty_rows(B):
    for new, keys in (([2, 3, 1, 1], [70, 2, 40, 90]), ([30, 40, 50, 1], [70, 25, 64, 90])):
        b = fp4_batch(new, keys, 16, 1, 256, 4, fill=127)
        b["pages"][0, 1], b["pages"][0, 3], b["pages"][2, :] = -1, b["k"].shape[0] + 5, 1 << 30
        b["kv_len"][3] = 0
        cache, batch = objects(B, b)
        q = torch.randn(b["n_rows"], 4, 256, device="cuda", generator=_gen(8)).bfloat16()
        got = B.fp4_paged_attention(cache, batch, q)
        want = attn_check(got, q, b, 1 / 16, 0)
        first = int(b["row_start"][2])
        assert (got[first:] == 0).all() and (got[int(b["row_start"][1])] == 0).all() and np.isfinite(want).all()
        none = B.PagedBatch(batch.row_start, batch.kv_len, batch.pages[:, :0], max_new=b["max_new"])
        assert (B.fp4_paged_attention(cache, none, q) == 0).all()


def test_attention_rows_outside_the_batch(B):
    b = fp4_batch([3, 4], [50, 20], 16, 2, 128, 4)
    b["row_start"] = np.array([2, 5, 9], np.int32)
    b["n_rows"] = 12
    cache, batch = objects(B, b)
    q = torch.randn(12, 4, 128, device="cuda", generator=_gen(8)).half()
    out = torch.full_like(q, 3.0)
    B.fp4_paged_attention(cache, batch, q, out=out)
    assert (out[:2] == 3).all() and (out[9:] == 3).all()
    attn_check(out, q, b, 128 ** -0.5, 0)
    b["row_start"] = np.array([-4, 5, 400], np.int32)  # held within the call's rows
    cache, batch = objects(B, b)
    attn_check(B.fp4_paged_attention(cache, batch, q), q, b, 128 ** -0.5, 0)


@pytest.mark.parametrize("n_q,n_kv,dim,seqs,new,ctx,window", [(4, 1, 256, 40, 1, 3000, 0), (4, 1, 256, 300, 1, 90, 0),
                                                              (8, 8, 64, 3, 400, 900, 0), (4, 1, 256, 2, 700, 2000, 512),
                                                              (16, 2, 128, 5, 7, 4000, 1000), (28, 4, 128, 1, 512, 3000, 0),
                                                              (16, 2, 128, 12, 2, 3000, 0), (12, 4, 64, 20, 4, 2500, 0),
                                                              (4, 1, 256, 1, 64, 8000, 0), (16, 2, 128, 1, 32, 9000, 0),
                                                              (5, 5, 64, 2, 40, 6000, 0), (4, 1, 256, 40, 20, 1500, 600)])
def test_attention_split_over_the_gpu(B, n_q, n_kv, dim, seqs, new, ctx, window):
    """Enough keys that rows are divided between CTAs and joined again; the same bits every time."""
    rng = random.Random(seqs)
    keys = [rng.randint(new, ctx) for _ in range(seqs)]
    b = fp4_batch([new] * seqs, keys, 64, n_kv, dim, 6, heads_first=True, tight=True)
    cache, batch = objects(B, b)
    q = (torch.randn(b["n_rows"], n_q, dim, device="cuda", generator=_gen(8)) * 1.5).bfloat16()
    got = B.fp4_paged_attention(cache, batch, q, window=window)
    rows = set(rng.sample(range(b["n_rows"]), min(60, b["n_rows"]))) | {0, b["n_rows"] - 1}
    attn_check(got, q, b, dim ** -0.5, window, rows)
    for _ in range(3):
        assert torch.equal(B.fp4_paged_attention(cache, batch, q, window=window), got)


@pytest.mark.parametrize("new,keys", [([1, 1], [300, 77]), ([20, 40], [300, 77])])
def test_attention_large_strides(B, new, keys):
    """A pool whose last page begins beyond 2^32 bytes, in codes and scales."""
    n_pages, page, dim = 8300, 256, 128
    b = fp4_batch(new, keys, page, 1, dim, 1, spare=0)
    ids = np.array([n_pages - 1 - i for i in range(b["k"].shape[0])])
    pool = torch.zeros(n_pages, 2, page, 1, 16 * dim // 2, dtype=torch.uint8, device="cuda")  # 4.35e9 bytes
    for i, name in enumerate(("k", "v")):
        codes, scales = pool[:, i, :, :, :dim // 2], pool[:, i, :, :, dim:dim + dim // 16]
        for j, p in enumerate(ids):
            codes[p], scales[p] = b[name + "4"][j], b[name + "s"][j]
        b[name + "4"], b[name + "s"] = codes, scales
    b["k_pages"] = b["pages"]
    cache, batch = objects(B, dict(b, pages=np.where(b["pages"] >= 0, ids[np.maximum(b["pages"], 0)], -1).astype(np.int32)))
    q = torch.randn(b["n_rows"], 4, dim, device="cuda", generator=_gen(8)).bfloat16()
    attn_check(B.fp4_paged_attention(cache, batch, q), q, b, dim ** -0.5, 0)


@pytest.mark.parametrize("new,n_q,n_kv,dim", [([1, 2, 1], 8, 2, 64), ([1, 1, 1], 4, 1, 256), ([40, 3, 130], 8, 2, 128)])
def test_attention_pages_in_common(B, new, n_q, n_kv, dim):
    """Sequences that share pages, as forks of one prompt do, and a page twice in one sequence."""
    b = fp4_batch(new, [200, 190, 180], 16, n_kv, dim, 5)
    b["pages"][1, :9], b["pages"][2, :9] = b["pages"][0, :9], b["pages"][0, :9]
    b["pages"][2, 3] = b["pages"][2, 2]
    cache, batch = objects(B, b)
    q = torch.randn(b["n_rows"], n_q, dim, device="cuda", generator=_gen(8)).bfloat16()
    attn_check(B.fp4_paged_attention(cache, batch, q), q, b, dim ** -0.5, 0)


@pytest.mark.parametrize("new,n_q,n_kv,dim", [([1, 2], 8, 2, 64), ([1, 1], 4, 1, 256), ([40, 130], 8, 2, 128), ([50, 90], 4, 1, 256)])
@pytest.mark.parametrize("exps", [(-90, 100), (5, 90), (-20, -100)])
def test_attention_exponents(B, new, n_q, n_kv, dim, exps):
    """A cache's exponents far from 0: the same attention, scaled."""
    b = fp4_batch(new, [100, 190], 16, n_kv, dim, 5, exps=(0, 0))
    q = torch.randn(b["n_rows"], n_q, dim, device="cuda", generator=_gen(8)).bfloat16()
    cache, batch = objects(B, b)
    want = B.fp4_paged_attention(cache, batch, q, scale=0.1)
    cache, batch = objects(B, dict(b, exps=exps))
    got = B.fp4_paged_attention(cache, batch, q, scale=0.1 * 2.0 ** -exps[0])
    assert torch.equal(got.float() * 2.0 ** -exps[1], want.float())


@pytest.mark.parametrize("new,n_q,dim", [([1, 1, 2, 1], 4, 256), ([30, 1, 50, 2], 4, 128)])
def test_lengths_beyond_the_pages(B, new, n_q, dim):
    b = fp4_batch(new, [40, 64, 80, 33], 16, 1, dim, 5)
    b["kv_len"] = np.array([1 << 30, 64, 2147483647, 33], np.int32)
    b["kv_len"][3] = -5
    cache, batch = objects(B, b)
    q = torch.randn(b["n_rows"], n_q, dim, device="cuda", generator=_gen(8)).bfloat16()
    attn_check(B.fp4_paged_attention(cache, batch, q), q, b, dim ** -0.5, 0)


def test_attention_many_sequences(B):
    keys = [1 + (7 * i) % 50 for i in range(1500)]
    b = fp4_batch([1] * 1500, keys, 16, 1, 64, 5)
    cache, batch = objects(B, b)
    q = torch.randn(1500, 4, 64, device="cuda", generator=_gen(8)).bfloat16()
    attn_check(B.fp4_paged_attention(cache, batch, q), q, b, 0.125, 0, set(range(0, 1500, 31)))


# ------------------------------------------------------------------------------------ together
def _layer(B, w, table, cache, batch, x, n_q, n_kv, dim):
    """Projection, append, attention and output projection, all in 4 bits."""
    qkv = B.fp4_linear(w[0], x).view(-1, n_q + 2 * n_kv, dim)
    q = B.fp4_rope_append(table, cache, batch, qkv[:, :n_q], qkv[:, n_q:n_q + n_kv], qkv[:, n_q + n_kv:])
    o = B.fp4_paged_attention(cache, batch, q)
    return qkv, q, o, B.fp4_linear(w[1], o.view(len(x), -1), dtype=torch.float32)


@pytest.mark.parametrize("block", [16, 32])
@pytest.mark.parametrize("new,keys", [([1, 1, 1, 1], [3, 100, 33, 64]), ([30, 1, 17], [30, 200, 90])])
def test_operators_together(B, new, keys, block):
    """A layer's attention in 4 bits, step by step: each operator against the oracle on its own inputs; then captured, and replayed
    for the next token of every sequence with lengths that the graph reads on the device."""
    n_q, n_kv, dim, hidden = 4, 1, 256, 512
    b = fp4_batch(new, [k + 1 for k in keys], 16, n_kv, dim, 9, heads_first=True, exps=(0, 0))
    b["kv_len"] = np.array(keys, np.int32)
    cache, batch = objects(B, b)
    w = [B.fp4_quantize(torch.randn(n, k, device="cuda", generator=_gen(n)).bfloat16() * 0.05, block)
         for n, k in (((n_q + 2 * n_kv) * dim, hidden), (hidden, n_q * dim))]
    table = B.rope_table(B.RopeConfig(dim))
    x = torch.randn(b["n_rows"], hidden, device="cuda", generator=_gen(3)).bfloat16()
    qkv, q, o, y = _layer(B, w, table, cache, batch, x, n_q, n_kv, dim)
    values = lambda t, blk: _np(B.fp4_dequantize(t if not torch.is_tensor(t) else B.fp4_quantize(t, blk), torch.float32))  # noqa: E731
    want, mass = O4.linear(values(x, block), values(w[0], block))
    assert (np.abs(_np(qkv.flatten(1)) - want) <= 2.0 ** -8 * np.abs(want) + hidden * 2.0 ** -22 * mass).all()
    refresh(b)
    attn_check(o, q, b, dim ** -0.5, 0)
    f, s = OS.rope_frequencies(dim, 1e4)
    for r, seq, pos, _ in OS.rows_of(b, 16):
        at = OS.place(b, b["k"].shape[0], 16, seq, pos)
        np.testing.assert_array_equal(_np(b["k"][at]), O4.cache_values(*O4.cache_quantise(OS.rope(_np(qkv[r:r + 1, n_q:n_q + 1]), [pos], f, s, False)[0], 0), 0))
    want, mass = O4.linear(values(o.view(b["n_rows"], -1), block), values(w[1], block))
    assert (np.abs(_np(y) - want) <= 2.0 ** -20 * np.abs(want) + n_q * dim * 2.0 ** -22 * mass).all()

    # the next token of every sequence, captured once
    n = len(keys)
    one = B.PagedBatch(torch.arange(n + 1, dtype=torch.int32, device="cuda"), batch.kv_len.clone(), batch.pages, max_new=1)
    static = torch.zeros(n, hidden, device="cuda", dtype=torch.bfloat16)
    _layer(B, w, table, cache, one, static, n_q, n_kv, dim)  # (writes the last slots, again below)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = _layer(B, w, table, cache, one, static, n_q, n_kv, dim)
    one.kv_len += 1
    static.copy_(torch.randn(n, hidden, device="cuda", generator=_gen(4)).bfloat16())
    g.replay()
    torch.cuda.synchronize()
    again = _layer(B, w, table, cache, one, static, n_q, n_kv, dim)
    for a, c in zip(out, again):
        assert torch.equal(a, c)
    refresh(b)
    attn_check(out[2], out[1], dict(b, row_start=np.arange(n + 1), kv_len=np.array(keys) + 1, n_rows=n, max_new=1), dim ** -0.5, 0)


def test_two_streams_at_once(B):
    """Calls on two streams, each with scratch of its own, while the other's runs."""
    works = []
    for i, (new, keys, n_q, dim) in enumerate((([1] * 8, [1500 + 300 * j for j in range(8)], 4, 256), ([90, 40], [3000, 500], 8, 128))):
        b = fp4_batch(new, keys, 16, 1, dim, 20 + i)
        cache, batch = objects(B, b)
        q = torch.randn(b["n_rows"], n_q, dim, device="cuda", generator=_gen(8)).bfloat16()
        works.append((cache, batch, q, B.fp4_paged_attention(cache, batch, q)))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in works]
    outs = [[], []]
    for _ in range(25):
        for i, ((cache, batch, q, _), s) in enumerate(zip(works, streams)):
            outs[i].append(B.fp4_paged_attention(cache, batch, q, stream=s))
    torch.cuda.synchronize()
    for i, w in enumerate(works):
        assert all(torch.equal(o, w[3]) for o in outs[i])


def test_cache_views_are_checked(B):
    b = fp4_batch([1], [20], 16, 2, 64, 4)
    cache, batch = objects(B, b)
    q = torch.randn(1, 4, 64, device="cuda").bfloat16()
    good = dict(k=cache.k, v=cache.v, k_scales=cache.k_scales, v_scales=cache.v_scales)
    for bad in (dict(k=cache.k.int()), dict(v=cache.v[:-1]), dict(k_scales=cache.k_scales[..., :3]), dict(v=cache.v.contiguous()),
                dict(v_scales=cache.v_scales.transpose(1, 2).contiguous().transpose(1, 2))):
        with pytest.raises(ValueError):
            B.fp4_paged_attention(B.PagedCacheFp4(**{**good, **bad}), batch, q)
    with pytest.raises(ValueError):
        B.fp4_paged_attention(cache, batch, q.float())
    with pytest.raises(ValueError):
        B.fp4_paged_attention(cache, batch, torch.randn(1, 4, 128, device="cuda").bfloat16())
    e = B.paged_cache_fp4(5, 32, 2, 128)
    assert e.k.shape == (5, 32, 2, 64) and e.k_scales.shape == (5, 32, 2, 8)
    assert (B.fp4_paged_values(e)[0] == 0).all()
