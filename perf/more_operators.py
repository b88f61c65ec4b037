"""What the 4-bit operators are measured on: floating point of 4 bits (e2m1: 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their
negatives) with a scale for every block of 16 or 32 values, as weights and activations of a linear and as the
keys and values of a paged cache.

A case is a dict of plain values; ``op`` names the operator.  Head counts, head dim, window, RoPE bases, hidden and
intermediate widths and vocabulary are those of the decoder this library runs (hidden 1152, intermediate 6912, 4 query
heads on 1 key/value head of 256, window 1024, vocabulary 262144), beside generic ones.  ``block`` 32 has scales that
are powers of two, ``block`` 16 has e4m3 scales under a power of two a row (or, in a cache, one for all keys and one for
all values).  A ragged batch is given by ``seqs``, ``new`` (new tokens a sequence), ``ctx`` (longest context) and
``lens``, the seed of its lengths, so that the work of a case does not depend on the data's seed.  Where ``own`` is false
the operators run in their plain form: elementary torch operations in 32 bits, in 64 where a value's nearness to a
rounding border decides its code, rounded once at the end.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

HIDDEN, INTER, N_Q, N_KV, HEAD, WINDOW, VOCAB, EPS = 1152, 6912, 4, 1, 256, 1024, 262144, 1e-6
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
MAX_ROWS = 8192 * INTER          # values of the largest quantisation
MAX_PRODUCT = 2048 * HIDDEN * 2 * INTER   # multiply-adds of the largest linear
MAX_WEIGHT = VOCAB * HIDDEN
MAX_APPEND = 4096                # new tokens of the largest append
MAX_KEYS = 64 * 16384 * 256      # key elements a pass of single tokens reads at most
MAX_CHUNK = 30 << 30             # (row, key, head, dim) products of the largest chunks


def listed():
    return [
        # the input of one sublayer for 16 tokens, there and back: launches and latency only
        {"name": "quantise_t16", "op": "quantise", "rows": 16, "k": HIDDEN, "block": 16, "type": "bf16"},
        # a long prompt's GeGLU output, an odd number of rows, there and back as in a check of a layer's quality
        {"name": "quantise_t8191", "op": "quantise", "rows": 8191, "k": INTER, "block": 32, "type": "bf16"},
        # the gate of one token: latency
        {"name": "linear_m1", "op": "linear", "m": 1, "n": INTER, "k": HIDDEN, "block": 16, "bias": False, "type": "bf16",
         "out": "bf16"},
        # the down projection of a few tokens, a long row of weights a channel, with a bias
        {"name": "linear_m37_down", "op": "linear", "m": 37, "n": HIDDEN, "k": INTER, "block": 32, "bias": True,
         "type": "f16", "out": "f16"},
        # the lm_head of a decode batch: the whole table once, fp32 logits
        {"name": "linear_m16_head", "op": "linear", "m": 16, "n": VOCAB, "k": HIDDEN, "block": 16, "bias": False,
         "type": "bf16", "out": "f32"},
        # gate and up of a prompt
        {"name": "linear_m2048", "op": "linear", "m": 2048, "n": 2 * INTER, "k": HIDDEN, "block": 16, "bias": False,
         "type": "bf16", "out": "bf16"},
        # one decode step of 48 sequences: QK-norm, rotation, one slot a sequence
        {"name": "append_b48", "op": "append", "seqs": 48, "new": 1, "ctx": 150, "lens": 1, "n_q": N_Q, "n_kv": N_KV,
         "dim": HEAD, "rot": HEAD, "inter": False, "base": 1e6, "norm": True, "page": 16, "heads_first": False,
         "type": "bf16"},
        # chunks of five prompts in one call, an odd number of rows, grouped heads of 128, no norm
        {"name": "append_chunks", "op": "append", "seqs": 5, "new": 811, "ctx": 900, "lens": 2, "n_q": 16, "n_kv": 4,
         "dim": 128, "rot": 128, "inter": False, "base": 5e5, "norm": False, "page": 64, "heads_first": True,
         "type": "bf16"},
        # the next token of one short conversation on a global layer: latency
        {"name": "attn_b1_ctx700", "op": "attention", "seqs": 1, "new": 1, "ctx": 700, "lens": 0, "n_q": N_Q, "n_kv": N_KV,
         "dim": HEAD, "window": 0, "page": 16, "heads_first": False, "type": "bf16"},
        # a decode batch with long ragged contexts on a global layer: memory bound
        {"name": "attn_b64_long", "op": "attention", "seqs": 64, "new": 1, "ctx": 30000, "lens": 4, "n_q": N_Q,
         "n_kv": N_KV, "dim": HEAD, "window": 0, "page": 64, "heads_first": False, "type": "bf16"},
        # four drafted tokens a sequence to be checked, grouped heads of 64
        {"name": "attn_draft_f16", "op": "attention", "seqs": 20, "new": 4, "ctx": 5000, "lens": 5, "n_q": 24, "n_kv": 8,
         "dim": 64, "window": 0, "page": 16, "heads_first": True, "type": "f16"},
        # chunks of four prompts behind long contexts, grouped heads of 128: tensor bound
        {"name": "attn_chunks_ctx9000", "op": "attention", "seqs": 4, "new": 1001, "ctx": 9000, "lens": 6, "n_q": 28,
         "n_kv": 4, "dim": 128, "window": 0, "page": 64, "heads_first": True, "type": "bf16"},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    op = rng.choice(["quantise", "linear", "linear", "append", "attention", "attention"])
    block, typ = rng.choice([16, 32]), rng.choice(["bf16", "bf16", "f16"])
    if op == "quantise":
        k = rng.choice([HIDDEN, INTER, 32 * _log_int(rng, 1, 256)])
        return {"op": op, "rows": _log_int(rng, 1, min(8192, MAX_ROWS // k)), "k": k, "block": block,
                "type": rng.choice(["bf16", "f16", "f32"])}
    if op == "linear":
        k = rng.choice([HIDDEN, INTER, 32 * _log_int(rng, 1, 256)])
        n = rng.choice([HIDDEN, 2 * INTER, _log_int(rng, 1, min(VOCAB, MAX_WEIGHT // k))])
        n = min(n, MAX_WEIGHT // k)
        return {"op": op, "m": _log_int(rng, 1, max(1, min(8192, MAX_PRODUCT // (n * k)))), "n": n, "k": k, "block": block,
                "bias": rng.random() < 0.5, "type": typ, "out": rng.choice([typ, typ, "f32"])}
    n_q, n_kv, dim = rng.choice([(4, 1, 256), (4, 1, 256), (8, 4, 256), (16, 2, 128), (28, 4, 128), (5, 5, 64), (24, 8, 64)])
    page, heads_first = rng.choice([16, 32, 64, 128]), rng.random() < 0.5
    if op == "append":
        seqs = _log_int(rng, 1, 96)
        new = 1 if rng.random() < 0.4 else _log_int(rng, 1, max(1, MAX_APPEND // seqs))
        return {"op": op, "seqs": seqs, "new": new, "ctx": max(new, _log_int(rng, 16, 1000)), "lens": rng.randrange(1 << 20),
                "n_q": n_q, "n_kv": n_kv, "dim": dim, "rot": dim if rng.random() < 0.6 else dim // 2,
                "inter": rng.random() < 0.5, "base": rng.choice([1e4, 5e5, 1e6]), "norm": rng.random() < 0.5, "page": page,
                "heads_first": heads_first, "type": typ}
    window = WINDOW if rng.random() < 0.3 else 0
    if rng.random() < 0.5:  # single tokens or a few drafted ones
        seqs, new = _log_int(rng, 1, 64), rng.choice([1, 1, 1, 2, 5])
        ctx = _log_int(rng, 16, min(30000, MAX_KEYS // (seqs * n_kv * dim)))
    else:  # chunks
        new = _log_int(rng, 6, 2048)
        seqs = _log_int(rng, 1, max(1, min(8, 4096 // new)))
        ctx = _log_int(rng, new, max(new, min(16000, MAX_CHUNK // (seqs * new * n_q * dim))))
    return {"op": op, "seqs": seqs, "new": new, "ctx": max(new, ctx), "lens": rng.randrange(1 << 20), "n_q": n_q,
            "n_kv": n_kv, "dim": dim, "window": window, "page": page, "heads_first": heads_first, "type": typ}


# ------------------------------------------------------------------------------------- 4-bit values
def _e4m3(x):
    """The nearest e4m3 value of x >= 0, 448 above it."""
    return x.clamp_max(448.0).float().to(torch.float8_e4m3fn)


def _codes(x, unit):
    """Codes (sign in bit 3) of x in units of `unit` (> 0 or 0, where every code is 0): nearest, ties to the even code."""
    a = x.abs()
    c = torch.zeros_like(a, dtype=torch.uint8)
    for mid, tie_up in ((0.25, False), (0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False)):
        c += (a >= mid * unit) if tie_up else (a > mid * unit)
    c = torch.where(unit > 0, c, torch.zeros_like(c))
    return c + 8 * (x < 0).to(torch.uint8)


def _values(codes):
    """fp32 values of codes, one a byte."""
    grid = torch.tensor(GRID + tuple(-g for g in GRID), device=codes.device)
    return grid[codes.long()]


def _two_to(e):
    """2^e in 64 bits, exactly."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _over(x, by):
    """x / by, rounded correctly (a division by a plain number becomes a product with its reciprocal on the GPU)."""
    return x / torch.full((), by, dtype=x.dtype, device=x.device)


def _rounded(x, block):
    """x [rows, K] as what its 4-bit form stands for, fp32."""
    rows, k = x.shape
    b = x.double().view(rows, k // block, block)
    top = b.abs().amax(-1, keepdim=True)
    if block == 32:  # 2^(floor(log2 top) - 2)
        unit = _two_to((torch.frexp(top)[1] - 3).clamp(-127, 127))
        unit = torch.where(top > 0, unit, torch.zeros_like(unit))
    else:  # the smallest power of two that keeps every block's scale within e4m3, then e4m3
        m, e = torch.frexp(_over(x.double().abs().amax(-1), 2688.0))
        row = _two_to(torch.where(m == 0.5, e - 1, e).clamp_min(-126))[:, None, None]
        unit = _e4m3(_over(top / row, 6.0)).double() * row
    return (_values(_codes(b, unit)) * unit.float()).view(rows, k)


def _pack(x, exponent):
    """x [..., dim] as a cache holds it: codes [..., dim / 2], two a byte, the lower dim in the low half, and e4m3 scales
    [..., dim / 16]; a value is code x scale x 2^exponent."""
    b = (x * 2.0 ** -exponent).unflatten(-1, (-1, 16))
    scale = _e4m3(_over(b.abs().amax(-1), 6.0))
    c = _codes(b, scale.to(x.dtype).unsqueeze(-1)).flatten(-2)
    return c[..., 0::2] | (c[..., 1::2] << 4), scale.view(torch.uint8)


def _unpack(codes, scales, exponent):
    """fp32 values [..., dim] of codes [..., dim / 2] and scales [..., dim / 16]."""
    v = _values(torch.stack([codes & 15, codes >> 4], -1).flatten(-2))
    s = scales.contiguous().view(torch.float8_e4m3fn).float() * 2.0 ** exponent
    return (v.unflatten(-1, (-1, 16)) * s.unsqueeze(-1)).flatten(-2)


# ------------------------------------------------------------------------------------------- inputs
def _lengths(case):
    """New tokens and keys (new ones included) of every sequence of a ragged batch."""
    rng = random.Random(case["lens"])
    if case["seqs"] == 1:
        return [case["new"]], [case["ctx"]]
    new = [case["new"] if case["new"] <= 8 else rng.randint(max(1, case["new"] // 2), case["new"]) for _ in range(case["seqs"])]
    return new, [rng.randint(n, max(n, case["ctx"])) for n in new]


K_EXP, V_EXP = 1, -2  # the cache's powers of two: keys after a norm reach a few times the values


def _paged(case, gen, dev):
    """A ragged batch over a 4-bit cache whose pages are scattered; every page holds values."""
    new, keys = _lengths(case)
    page, wide = case["page"], -(-max(keys) // case["page"])
    used = [-(-k // page) for k in keys]
    n_pages = sum(used) + 3
    order = torch.randperm(n_pages, generator=gen, device=dev).to(torch.int32)
    table = torch.full((len(keys), wide), -1, dtype=torch.int32)
    at, host = 0, order.cpu()
    for s, u in enumerate(used):
        table[s, :u] = host[at:at + u]
        at += u
    n_kv, dim = case["n_kv"], case["dim"]
    shape = (n_pages, n_kv, page) if case["heads_first"] else (n_pages, page, n_kv)
    pools = {}
    for name, exp in (("k", K_EXP), ("v", V_EXP)):
        codes = torch.empty(*shape, dim // 2, dtype=torch.uint8, device=dev)
        scales = torch.empty(*shape, dim // 16, dtype=torch.uint8, device=dev)
        step = max(1, (1 << 26) // (page * n_kv * dim))
        for a in range(0, n_pages, step):
            b = min(n_pages, a + step)
            codes[a:b], scales[a:b] = _pack(torch.randn(b - a, *shape[1:], dim, generator=gen, device=dev), exp)
        if case["heads_first"]:
            codes, scales = codes.transpose(1, 2), scales.transpose(1, 2)
        pools[name], pools[name + "_scales"] = codes, scales
    return {"new": new, "keys": keys, **pools, "pages": table.to(dev),
            "row_start": torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32, device=dev),
            "kv_len": torch.tensor(keys, dtype=torch.int32, device=dev), "rows": sum(new), "max_new": max(new)}


def _activations(rows, k, gen, dev):
    """A linear's input: a few channels are much larger than the others, and rows differ in size."""
    x = torch.randn(rows, k, generator=gen, device=dev)
    x *= torch.exp(0.5 * torch.randn(rows, 1, generator=gen, device=dev))
    wide = torch.randint(0, k, (max(1, k // 100),), generator=gen, device=dev)
    x[:, wide] *= 20.0
    return x


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(dev).manual_seed(seed)
    dt = TYPES[case["type"]]
    s = {"case": case}
    if own:
        from paper_2608_28003_gb300 import binding as B
    if case["op"] == "quantise":
        s["x"] = _activations(case["rows"], case["k"], gen, dev).to(dt)
        return s
    if case["op"] == "linear":
        n, k = case["n"], case["k"]
        s["x"] = _activations(case["m"], k, gen, dev).to(dt)
        w = (0.02 * torch.randn(n, k, generator=gen, device=dev)).to(dt)
        s["bias"] = torch.randn(n, generator=gen, device=dev) if case["bias"] else None
        if own:  # a program quantises its weights once
            s["w"] = B.fp4_quantize(w, block=case["block"])
        else:
            step = max(1, (1 << 26) // k)
            s["w"] = torch.cat([_rounded(w[a:a + step], case["block"]) for a in range(0, n, step)])
        return s
    s.update(_paged(case, gen, dev))
    n_q, n_kv, dim = case["n_q"], case["n_kv"], case["dim"]
    if case["op"] == "append":
        qkv = 2.0 * torch.randn(s["rows"], n_q + 2 * n_kv, dim, generator=gen, device=dev)
        qkv = qkv.to(dt)
        s["q"], s["k_new"], s["v_new"] = qkv[:, :n_q], qkv[:, n_q:n_q + n_kv], qkv[:, n_q + n_kv:]
        s["qn"], s["kn"] = ((1.0 + 0.2 * torch.randn(dim, generator=gen, device=dev)) if case["norm"] else None
                            for _ in range(2))
    else:
        s["q"] = (1.5 * torch.randn(s["rows"], n_q, dim, generator=gen, device=dev)).to(dt)
    if own:
        s["cache"] = B.PagedCacheFp4(s["k"], s["v"], s["k_scales"], s["v_scales"], k_exp=K_EXP, v_exp=V_EXP)
        s["batch"] = B.PagedBatch(s["row_start"], s["kv_len"], s["pages"], max_new=s["max_new"])
        if case["op"] == "append":
            s["table"] = B.rope_table(B.RopeConfig(case["rot"], base=case["base"], interleaved=case["inter"]), dev)
    return s


# ---------------------------------------------------------------------------------------------- runs
def _rotate(x, pos, case):
    """x [T, H, D] rotated at positions [T]: angles in 64 bits, the rotation in x's type."""
    rot = case["rot"]
    f = torch.tensor([case["base"] ** (-2.0 * i / rot) for i in range(rot // 2)], dtype=torch.float64, device=x.device)
    a = pos.double()[:, None] * f[None, :]
    cos, sin = torch.cos(a).to(x.dtype)[:, None, :], torch.sin(a).to(x.dtype)[:, None, :]
    y = x.clone()
    first = slice(0, rot, 2) if case["inter"] else slice(0, rot // 2)
    second = slice(1, rot, 2) if case["inter"] else slice(rot // 2, rot)
    y[..., first] = x[..., first] * cos - x[..., second] * sin
    y[..., second] = x[..., second] * cos + x[..., first] * sin
    return y


def _norm(x, w):
    return x if w is None else x / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS) * w


def _positions(s):
    return torch.cat([torch.arange(k - n, k, device=s["q"].device) for n, k in zip(s["new"], s["keys"])])


def _plain_append(s):
    case, dt = s["case"], s["q"].dtype
    pos, page = _positions(s), case["page"]
    seq = torch.repeat_interleave(torch.arange(len(s["new"]), device=pos.device), torch.tensor(s["new"], device=pos.device))
    at, slot = s["pages"][seq, pos // page].long(), pos % page
    q = _rotate(_norm(s["q"].float(), s["qn"]), pos, case).to(dt)
    k = _rotate(_norm(s["k_new"].double(), s["kn"]), pos, case)  # 64 bits: codes are decided at their borders
    for name, x, exp in (("k", k, K_EXP), ("v", s["v_new"].double(), V_EXP)):
        s[name][at, slot], s[name + "_scales"][at, slot] = _pack(x, exp)
    return q, _unpack(s["k"], s["k_scales"], K_EXP).to(dt), _unpack(s["v"], s["v_scales"], V_EXP).to(dt)


def _plain_attention(s):
    case, q = s["case"], s["q"]
    n_kv, dim, page, w = case["n_kv"], case["dim"], case["page"], case["window"]
    group, out, row = case["n_q"] // n_kv, torch.empty_like(q), 0
    for i, (n, keys) in enumerate(zip(s["new"], s["keys"])):
        lo = max(0, keys - n - w + 1) // page * page if w else 0
        pages = s["pages"][i, lo // page:-(-keys // page)].long()
        k, v = (_unpack(s[c][pages], s[c + "_scales"][pages], e).reshape(-1, n_kv, dim)[:keys - lo]
                for c, e in (("k", K_EXP), ("v", V_EXP)))
        pos, j = torch.arange(keys - n, keys, device=q.device), torch.arange(lo, keys, device=q.device)
        hide = j[None, :] > pos[:, None]
        if w:
            hide |= j[None, :] <= pos[:, None] - w
        for h in range(n_kv):
            qh = q[row:row + n, h * group:(h + 1) * group].float().transpose(0, 1)
            x = torch.matmul(qh, k[:, h].t()) / math.sqrt(dim)
            x.masked_fill_(hide, -math.inf)
            x = torch.exp(x - x.amax(-1, keepdim=True))
            x = torch.matmul(x, v[:, h]) / x.sum(-1, keepdim=True)
            out[row:row + n, h * group:(h + 1) * group] = x.transpose(0, 1).to(q.dtype)
        row += n
    return out


def run(s):
    case = s["case"]
    if own:
        from paper_2608_28003_gb300 import binding as B
        if case["op"] == "quantise":
            return B.fp4_dequantize(B.fp4_quantize(s["x"], block=case["block"]), s["x"].dtype)
        if case["op"] == "linear":
            return B.fp4_linear(s["w"], s["x"], bias=s["bias"], dtype=TYPES[case["out"]])
        if case["op"] == "append":
            q = B.fp4_rope_append(s["table"], s["cache"], s["batch"], s["q"], s["k_new"], s["v_new"], q_norm=s["qn"],
                                  k_norm=s["kn"], eps=EPS)
            return (q, *B.fp4_paged_values(s["cache"], s["q"].dtype))
        return B.fp4_paged_attention(s["cache"], s["batch"], s["q"], window=case["window"])
    if case["op"] == "quantise":
        return _rounded(s["x"], case["block"]).to(s["x"].dtype)
    if case["op"] == "linear":
        y = torch.matmul(_rounded(s["x"], case["block"]), s["w"].t())
        return (y if s["bias"] is None else y + s["bias"]).to(TYPES[case["out"]])
    return _plain_append(s) if case["op"] == "append" else _plain_attention(s)


def _held(values, block):
    """Bytes of so many values in 4 bits with their scales."""
    return values // 2 + values // block


def work(case):
    """Each input read once and each output written once; the operations of the formulas."""
    e = 4 if case["type"] == "f32" else 2
    if case["op"] == "quantise":  # there, and the values back: the 4-bit form is an output and an input
        n = case["rows"] * case["k"]
        return {"bytes": 2 * n * e + 2 * _held(n, case["block"]), "flops": 4 * n}
    if case["op"] == "linear":
        m, n, k = case["m"], case["n"], case["k"]
        out = 4 if case["out"] == "f32" else 2
        return {"bytes": m * k * e + _held(n * k, case["block"]) + m * n * out + 4 * n * case["bias"], "flops": 2 * m * n * k}
    new, keys = _lengths(case)
    rows, n_q, n_kv, dim = sum(new), case["n_q"], case["n_kv"], case["dim"]
    if case["op"] == "append":
        heads = n_q + 2 * n_kv
        slots = (sum(-(-k // case["page"]) for k in keys) + 3) * case["page"]  # the cache is read back whole
        return {"bytes": rows * heads * dim * e + rows * n_q * dim * e + 2 * _held(rows * n_kv * dim, 16)
                + 2 * slots * n_kv * (_held(dim, 16) + dim * e),
                "flops": rows * (n_q + n_kv) * (3 * case["rot"] + 4 * dim * case["norm"]) + 2 * slots * n_kv * dim}
    w = case["window"]
    visible = sum(k - (max(0, k - n - w + 1) if w else 0) for n, k in zip(new, keys))
    pairs = 0  # visible (row, key) pairs
    for n, k in zip(new, keys):
        for p in range(k - n, k):
            pairs += min(p + 1, w) if w else p + 1
    return {"bytes": 2 * rows * n_q * dim * e + 2 * _held(visible * n_kv * dim, 16), "flops": 4 * pairs * n_q * dim}


# ---------------------------------------------------------------------------------------- 64 bits
def _nearest(r):
    """r >= 0 rounded to 0, 0.5, .. 2 by halves, to 4 by ones, to 6 by twos: an even multiple at a tie, as the even code is."""
    y = torch.where(r < 2, torch.round(r * 2) / 2, torch.where(r < 4, torch.round(r), torch.round(r / 2) * 2))
    return y.clamp_max(6.0)


def _nearest_e4m3(x):
    """x in [0, 448] rounded to 4 significant bits, or to a multiple of 2^-9 where that is coarser."""
    step = _power(x.clamp_min(2.0 ** -6)) / 8
    return torch.round(x / step) * step


def _power(x):
    """The largest power of two that is at most x > 0 (a normal number): x without its fraction."""
    return (x.view(torch.int64) & (0x7FF << 52)).view(torch.float64)


def _stands_for(x, block, exponent=None):
    """x [..., K] in 64 bits as its 4-bit form has it; with an exponent, as a cache has it."""
    b = x.double().unflatten(-1, (-1, block))
    top = b.abs().amax(-1, keepdim=True)
    six = torch.full_like(top, 6.0)
    if block == 32:
        unit = _power(top.clamp_min(2.0 ** -125)) * 0.25
    else:
        if exponent is None:  # 21 2^7 = 6 448
            least = x.double().abs().amax(-1, keepdim=True).clamp_min(2.0 ** -115) / torch.full_like(top[..., 0, :], 21.0)
            row = _power(least) / 128
            row = torch.where(row * 2688 < x.double().abs().amax(-1, keepdim=True), row * 2, row)
            row = row.clamp_min(2.0 ** -126).unsqueeze(-1)
        else:
            row = 2.0 ** exponent
        unit = _nearest_e4m3((top / row / six).clamp_max(448.0)) * row
    r = torch.where(unit > 0, b.abs() / unit, torch.zeros_like(b))
    return (_nearest(r) * unit * torch.sign(b)).flatten(-2)


def _held_values(codes, scales, exponent):
    """64-bit values of what a cache holds."""
    c = torch.stack((codes.bitwise_and(15), codes.bitwise_right_shift(4)), dim=-1).flatten(-2).to(torch.int64)
    m = c & 7
    mag = torch.where(m < 2, m * 0.5, (1.0 + 0.5 * (m & 1)) * (1 << (m >> 1)) * 0.5).double()
    b = scales.long()
    exp, man = (b >> 3) & 15, b & 7
    sc = torch.where(exp > 0, (8 + man) * (1 << exp), man * 2) * 2.0 ** -10
    return torch.where(c > 7, -mag, mag).double() * sc.double().repeat_interleave(16, -1) * 2.0 ** exponent


def _turned(x, pos, case):
    """x [T, H, D] in 64 bits, its pairs as complex numbers times exp(i p f)."""
    rot, t, h = case["rot"], x.shape[0], x.shape[1]
    f = torch.tensor([case["base"] ** (-2.0 * i / rot) for i in range(rot // 2)], dtype=torch.float64, device=x.device)
    unit = torch.polar(torch.ones(t, rot // 2, dtype=torch.float64, device=x.device), torch.outer(pos.double(), f))
    part = x[..., :rot].reshape(t, h, rot // 2, 2) if case["inter"] else x[..., :rot].reshape(t, h, 2, rot // 2).transpose(2, 3)
    z = torch.view_as_real(torch.view_as_complex(part.contiguous()) * unit[:, None, :])
    z = z.reshape(t, h, rot) if case["inter"] else z.transpose(2, 3).reshape(t, h, rot)
    return torch.cat([z, x[..., rot:]], -1)


def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed) if case["op"] != "linear" else None
    finally:
        own = was
    if case["op"] == "quantise":
        return _stands_for(s["x"], case["block"])
    if case["op"] == "linear":
        return _exact_linear(case, seed)
    if case["op"] == "attention":
        return _exact_attention(case, s)

    def unit(x, w):
        if w is None:
            return x.double()
        x = x.double()
        return x * torch.rsqrt(x.pow(2).sum(-1, keepdim=True) / case["dim"] + EPS) * w.double()
    page = case["page"]
    place = [(i, p) for i, (n, k) in enumerate(zip(s["new"], s["keys"])) for p in range(k - n, k)]
    pos = torch.tensor([p for _, p in place], device=s["q"].device)
    table = s["pages"].cpu()
    at = torch.tensor([int(table[i, p // page]) for i, p in place], device=pos.device)
    k, v = (_held_values(s[c], s[c + "_scales"], e) for c, e in (("k", K_EXP), ("v", V_EXP)))
    k[at, pos % page] = _stands_for(_turned(unit(s["k_new"], s["kn"]), pos, case), 16, K_EXP)
    v[at, pos % page] = _stands_for(s["v_new"], 16, V_EXP)
    return _turned(unit(s["q"], s["qn"]), pos, case), k, v


def _exact_linear(case, seed):
    """The inputs of `prepare`, drawn again in its order."""
    dev = torch.device("cuda")
    gen = torch.Generator(dev).manual_seed(seed)
    dt, n, k = TYPES[case["type"]], case["n"], case["k"]
    x = _stands_for(_activations(case["m"], k, gen, dev).to(dt), case["block"])
    w = (0.02 * torch.randn(n, k, generator=gen, device=dev)).to(dt)
    bias = torch.randn(n, generator=gen, device=dev) if case["bias"] else None
    y = torch.empty(case["m"], n, dtype=torch.float64, device=dev)
    step = max(1, (1 << 26) // k)
    for a in range(0, n, step):
        y[:, a:a + step] = torch.einsum("mk,nk->mn", x, _stands_for(w[a:a + step], case["block"]))
    return y if bias is None else y + bias.double()


def _exact_attention(case, s):
    n_kv, dim = case["n_kv"], case["dim"]
    group, parts, first = case["n_q"] // n_kv, [], 0
    for i, (n, keys) in enumerate(zip(s["new"], s["keys"])):
        rows = s["q"][first:first + n].double().view(n, n_kv, group, dim)
        first += n
        pages = s["pages"][i, :-(-keys // case["page"])].long()
        k, v = (_held_values(s[c].index_select(0, pages), s[c + "_scales"].index_select(0, pages), e)
                .flatten(0, 1)[:keys].transpose(0, 1) for c, e in (("k", K_EXP), ("v", V_EXP)))  # [n_kv, keys, D]
        age = torch.arange(keys - n, keys, device=k.device)[:, None] - torch.arange(keys, device=k.device)[None, :]
        ok = (age >= 0) & (age < (case["window"] or keys + 1))
        out = torch.empty_like(rows)
        step = max(1, (1 << 27) // (keys * group * n_kv))  # rows at a time
        for a in range(0, n, step):
            b = min(n, a + step)
            x = torch.einsum("nhgd,hkd->hgnk", rows[a:b], k) * dim ** -0.5
            x = torch.where(ok[a:b], x, torch.full((), -math.inf, dtype=x.dtype, device=x.device))
            x = torch.exp(x - torch.logsumexp(x, -1, keepdim=True))
            out[a:b] = torch.einsum("hgnk,hkd->nhgd", x, v)
        parts.append(out.reshape(n, case["n_q"], dim))
    return torch.cat(parts)
