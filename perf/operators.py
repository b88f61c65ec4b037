"""What the operators of a serving step are measured on: rotary positions, the append of rotated keys and of
values to a paged cache, attention of a ragged batch over that cache, and sampling of the next token.

A case is a dict of plain values; ``op`` names the operator.  Head counts, head dim, window, RoPE bases and
vocabulary are those of the decoder this library runs (4 query heads on 1 key/value head of 256, window
1024, vocabulary 262144), beside generic grouped layouts of head dims 64 and 128.  A ragged batch is given by
``seqs``, ``new`` (new tokens a sequence), ``ctx`` (longest context) and ``lens``, the seed of its lengths, so
that the work of a case does not depend on the data's seed.  Where ``own`` is false the operators run in their
plain form: elementary torch operations in 32 bits (angles, long sums and whatever decides a token in 64),
rounded once at the end.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

N_Q, N_KV, HEAD, WINDOW, VOCAB, EPS = 4, 1, 256, 1024, 262144, 1e-6
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
MAX_ROPE = 8192 * 32 * 128     # elements of the largest rotation
MAX_APPEND = 4096              # new tokens of the largest append
MAX_KEYS = 64 * 16384 * 256    # key elements a pass of single tokens reads at most
MAX_CHUNK = 30 << 30           # (row, key, head, dim) products of the largest chunks


def listed():
    return [
        # q and the key of 16 single tokens of the decoder, plain frequencies: launch and latency only
        {"name": "rope_t16", "op": "rope", "t": 16, "heads": N_Q + N_KV, "dim": HEAD, "rot": HEAD, "inter": False,
         "scaling": "none", "base": 1e6, "maxpos": 32768, "type": "bf16"},
        # a long document's rows: pairs side by side, half of the head, frequencies scaled by parts, far positions
        {"name": "rope_t8192_part", "op": "rope", "t": 8192, "heads": 32, "dim": 128, "rot": 64, "inter": True,
         "scaling": "parts", "base": 1e4, "maxpos": 1 << 20, "type": "f16"},
        # one decode step of 48 sequences: QK-norm, rotation, one slot a sequence
        {"name": "append_b48", "op": "append", "seqs": 48, "new": 1, "ctx": 2000, "lens": 1, "n_q": N_Q, "n_kv": N_KV,
         "dim": HEAD, "rot": HEAD, "inter": False, "scaling": "none", "base": 1e6, "norm": True, "page": 16,
         "type": "bf16"},
        # chunks of five prompts in one call, an odd number of rows, grouped heads of 128, no norm
        {"name": "append_chunks", "op": "append", "seqs": 5, "new": 811, "ctx": 4000, "lens": 2, "n_q": 16, "n_kv": 4,
         "dim": 128, "rot": 128, "inter": False, "scaling": "wavelength", "base": 5e5, "norm": False, "page": 64,
         "type": "bf16"},
        # the next token of one short conversation on a global layer: latency
        {"name": "attn_b1_ctx700", "op": "attention", "seqs": 1, "new": 1, "ctx": 700, "lens": 0, "n_q": N_Q, "n_kv": N_KV,
         "dim": HEAD, "window": 0, "page": 16, "type": "bf16"},
        # a decode batch on a layer with the sliding window: contexts beyond and below it
        {"name": "attn_b32_window", "op": "attention", "seqs": 32, "new": 1, "ctx": 6000, "lens": 3, "n_q": N_Q,
         "n_kv": N_KV, "dim": HEAD, "window": WINDOW, "page": 32, "type": "bf16"},
        # a decode batch with long ragged contexts on a global layer: memory bound
        {"name": "attn_b64_long", "op": "attention", "seqs": 64, "new": 1, "ctx": 30000, "lens": 4, "n_q": N_Q,
         "n_kv": N_KV, "dim": HEAD, "window": 0, "page": 64, "type": "bf16"},
        # four drafted tokens a sequence to be checked, grouped heads of 64
        {"name": "attn_draft_f16", "op": "attention", "seqs": 20, "new": 4, "ctx": 5000, "lens": 5, "n_q": 24, "n_kv": 8,
         "dim": 64, "window": 0, "page": 16, "type": "f16"},
        # a whole prompt of the decoder on a global layer: tensor bound
        {"name": "attn_prompt_2048", "op": "attention", "seqs": 1, "new": 2048, "ctx": 2048, "lens": 0, "n_q": N_Q,
         "n_kv": N_KV, "dim": HEAD, "window": 0, "page": 64, "type": "bf16"},
        # chunks of four prompts behind long contexts, grouped heads of 128
        {"name": "attn_chunks_ctx9000", "op": "attention", "seqs": 4, "new": 1001, "ctx": 9000, "lens": 6, "n_q": 28,
         "n_kv": 4, "dim": 128, "window": 0, "page": 64, "type": "bf16"},
        # the next token of one conversation, every filter: latency
        {"name": "sample_m1", "op": "sample", "m": 1, "vocab": VOCAB, "top_k": 64, "top_p": 0.95, "min_p": 0.02,
         "temp": 1.0, "type": "f32"},
        # the next tokens of a large decode batch, nucleus only, the lm_head's fp32 logits
        {"name": "sample_m64", "op": "sample", "m": 64, "vocab": VOCAB, "top_k": 0, "top_p": 0.9, "min_p": 0.0,
         "temp": 0.8, "type": "f32"},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    op = rng.choice(["rope", "append", "attention", "attention", "attention", "sample"])
    scaling, inter = rng.choice(["none", "linear", "wavelength", "parts"]), rng.random() < 0.5
    base = rng.choice([1e4, 5e5, 1e6])
    if op == "rope":
        dim, heads = rng.choice([64, 96, 128, 256]), _log_int(rng, 1, 64)
        rot = 16 * rng.randint(1, dim // 16) if rng.random() < 0.5 else dim
        return {"op": op, "t": _log_int(rng, 1, min(16384, MAX_ROPE // (heads * dim))), "heads": heads, "dim": dim, "rot": rot,
                "inter": inter, "scaling": scaling, "base": base, "maxpos": _log_int(rng, 1 << 12, 1 << 20),
                "type": rng.choice(["bf16", "f16"])}
    n_q, n_kv, dim = rng.choice([(4, 1, 256), (4, 1, 256), (8, 4, 256), (16, 2, 128), (28, 4, 128), (5, 5, 64), (24, 8, 64)])
    page = rng.choice([16, 32, 64, 128])
    if op == "append":
        seqs = _log_int(rng, 1, 96)
        new = 1 if rng.random() < 0.4 else _log_int(rng, 1, max(1, MAX_APPEND // seqs))
        rot = dim if rng.random() < 0.6 else dim // 2
        return {"op": op, "seqs": seqs, "new": new, "ctx": max(new, _log_int(rng, 64, 4000)), "lens": rng.randrange(1 << 20),
                "n_q": n_q, "n_kv": n_kv, "dim": dim, "rot": rot, "inter": inter, "scaling": scaling, "base": base,
                "norm": rng.random() < 0.5, "page": page, "type": rng.choice(["bf16", "bf16", "f16"])}
    if op == "attention":
        window = WINDOW if rng.random() < 0.3 else 0
        typ = rng.choice(["bf16", "bf16", "f16"])
        if rng.random() < 0.5:  # single tokens or a few drafted ones
            seqs, new = _log_int(rng, 1, 64), rng.choice([1, 1, 1, 2, 5])
            ctx = _log_int(rng, 16, min(30000, MAX_KEYS // (seqs * n_kv * dim)))
        else:  # chunks
            new = _log_int(rng, 6, 2048)
            seqs = _log_int(rng, 1, max(1, min(8, 4096 // new)))
            ctx = _log_int(rng, new, max(new, min(16000, MAX_CHUNK // (seqs * new * n_q * dim))))
        return {"op": op, "seqs": seqs, "new": new, "ctx": max(new, ctx), "lens": rng.randrange(1 << 20), "n_q": n_q,
                "n_kv": n_kv, "dim": dim, "window": window, "page": page, "type": typ}
    return {"op": op, "m": _log_int(rng, 1, 64), "vocab": rng.choice([VOCAB, VOCAB, _log_int(rng, 1000, 200000)]),
            "top_k": rng.choice([0, 0, 1, _log_int(rng, 2, 500)]), "top_p": rng.choice([1.0, 0.95, rng.uniform(0.2, 0.99)]),
            "min_p": rng.choice([0.0, 0.05, rng.uniform(0.0, 0.3)]), "temp": rng.choice([1.0, rng.uniform(0.4, 1.6)]),
            "type": rng.choice(["f32", "f32", "bf16"])}


# ------------------------------------------------------------------------------------------- inputs
def _lengths(case):
    """New tokens and keys (new ones included) of every sequence of a ragged batch."""
    rng = random.Random(case["lens"])
    if case["seqs"] == 1:
        return [case["new"]], [case["ctx"]]
    new = [case["new"] if case["new"] <= 8 else rng.randint(max(1, case["new"] // 2), case["new"]) for _ in range(case["seqs"])]
    return new, [rng.randint(n, max(n, case["ctx"])) for n in new]


def _seen(case):
    """(first visible key of any row, keys) of every sequence."""
    new, keys = _lengths(case)
    w = case["window"]
    return [(max(0, k - n - w + 1) if w else 0, k) for n, k in zip(new, keys)]


def _frequencies(case):
    """Angles a position turns the pairs by (radians, 64 bits), and the factor on cos and sin."""
    rot, base = case["rot"], case["base"]
    f = torch.tensor([base ** (-2.0 * i / rot) for i in range(rot // 2)], dtype=torch.float64)
    s = SCALING[case["scaling"]]
    if case["scaling"] == "linear":
        return f / s["factor"], 1.0
    if case["scaling"] == "wavelength":
        turns = s["original"] * f / (2 * math.pi)
        mix = ((turns - s["low"]) / (s["high"] - s["low"])).clamp(0.0, 1.0)
        return f * ((1 - mix) / s["factor"] + mix), 1.0
    if case["scaling"] == "parts":
        at = [rot * math.log(s["original"] / (2 * math.pi * b)) / (2 * math.log(base)) for b in (s["high"], s["low"])]
        lo, hi = max(0, math.floor(at[0])), min(rot - 1, math.ceil(at[1]))
        ramp = ((torch.arange(rot // 2, dtype=torch.float64) - lo) / max(hi - lo, 0.001)).clamp(0.0, 1.0)
        return f * (ramp / s["factor"] + (1 - ramp)), 0.1 * math.log(s["factor"]) + 1.0
    return f, 1.0


SCALING = {"none": {}, "linear": {"factor": 4.0}, "wavelength": {"factor": 8.0, "low": 1.0, "high": 4.0, "original": 8192},
           "parts": {"factor": 16.0, "low": 1.0, "high": 32.0, "original": 4096}}


def _table(case, dev):
    """The rotation as the library keeps it: built once by a program."""
    if not own:
        return None
    from paper_2608_28003_gb300 import binding as B
    s = SCALING[case["scaling"]]
    return B.rope_table(B.RopeConfig(case["rot"], base=case["base"], interleaved=case["inter"], scaling=case["scaling"],
                                     factor=s.get("factor", 1.0), low=s.get("low", 1.0), high=s.get("high", 4.0),
                                     original_len=s.get("original", 0)), dev)


def _paged(case, gen, dev, dt):
    """A ragged batch over a cache whose pages are scattered; every page holds values."""
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
    k, v = (torch.empty(n_pages, page, case["n_kv"], case["dim"], dtype=dt, device=dev).normal_(generator=gen)
            for _ in range(2))
    return {"new": new, "keys": keys, "k": k, "v": v, "pages": table.to(dev),
            "row_start": torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32, device=dev),
            "kv_len": torch.tensor(keys, dtype=torch.int32, device=dev), "rows": sum(new), "max_new": max(new)}


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(dev).manual_seed(seed)
    dt = TYPES[case["type"]]
    s = {"case": case}

    def normal(*shape, scale=1.0):
        return (torch.randn(*shape, generator=gen, device=dev) * scale).to(dt)
    if case["op"] == "rope":
        s["x"] = normal(case["t"], case["heads"], case["dim"])
        s["pos"] = torch.randint(0, case["maxpos"], (case["t"],), generator=gen, device=dev).to(torch.int32)
        s["table"] = _table(case, dev)
    elif case["op"] == "sample":
        m, n = case["m"], case["vocab"]
        x = torch.randn(m, n, generator=gen, device=dev) * 2.0
        peaks = torch.randint(0, n, (m, 24), generator=gen, device=dev)  # the tokens a model thinks of
        x.scatter_add_(1, peaks, torch.rand(m, 24, generator=gen, device=dev) * 9.0)
        s["logits"] = x.to(dt)
        s["u"] = torch.rand(m, generator=gen, device=dev)
        for name, value, kind in (("temp", case["temp"], torch.float32), ("top_k", case["top_k"], torch.int32),
                                  ("top_p", case["top_p"], torch.float32), ("min_p", case["min_p"], torch.float32)):
            s[name] = torch.full((m,), value, dtype=kind, device=dev)
    else:
        s.update(_paged(case, gen, dev, dt))
        n_q, n_kv, dim = case["n_q"], case["n_kv"], case["dim"]
        if case["op"] == "append":
            qkv = normal(s["rows"], (n_q + 2 * n_kv) * dim, scale=2.0).view(s["rows"], n_q + 2 * n_kv, dim)
            s["q"], s["k_new"], s["v_new"] = qkv[:, :n_q], qkv[:, n_q:n_q + n_kv], qkv[:, n_q + n_kv:]
            s["qn"], s["kn"] = ((1.0 + 0.2 * torch.randn(dim, generator=gen, device=dev)) if case["norm"] else None
                                for _ in range(2))
            s["table"] = _table(case, dev)
        else:
            s["q"] = normal(s["rows"], n_q, dim, scale=1.5)
        if own:
            from paper_2608_28003_gb300 import binding as B
            s["cache"] = B.PagedCache(s["k"], s["v"])
            s["batch"] = B.PagedBatch(s["row_start"], s["kv_len"], s["pages"], max_new=s["max_new"])
    return s


# ---------------------------------------------------------------------------------------------- runs
def _rotate(x, pos, case):
    """x [T, H, D] fp32 rotated at positions [T]: angles in 64 bits, the rotation in 32."""
    f, scale = _frequencies(case)
    a = torch.remainder(pos.double()[:, None] * f.to(x.device)[None, :], 2 * math.pi)
    cos, sin = (torch.cos(a) * scale).float()[:, None, :], (torch.sin(a) * scale).float()[:, None, :]
    rot = case["rot"]
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


def _slots(s):
    """Cache slot of every new row."""
    seq = torch.repeat_interleave(torch.arange(len(s["new"]), device=s["q"].device),
                                  torch.tensor(s["new"], device=s["q"].device))
    pos, page = _positions(s), s["case"]["page"]
    return s["pages"][seq, pos // page].long() * page + pos % page


def _plain_append(s):
    case, dt = s["case"], s["q"].dtype
    pos, slots = _positions(s), _slots(s)
    q = _rotate(_norm(s["q"].float(), s["qn"]), pos, case).to(dt)
    k = _rotate(_norm(s["k_new"].float(), s["kn"]), pos, case).to(dt)
    s["k"].view(-1, case["n_kv"], case["dim"])[slots] = k
    s["v"].view(-1, case["n_kv"], case["dim"])[slots] = s["v_new"]
    return q, s["k"], s["v"]


def _plain_attention(s):
    case, q = s["case"], s["q"]
    n_kv, dim, page, w = case["n_kv"], case["dim"], case["page"], case["window"]
    group, out, row = case["n_q"] // n_kv, torch.empty_like(q), 0
    for i, (n, keys) in enumerate(zip(s["new"], s["keys"])):
        lo = max(0, keys - n - w + 1) // page * page if w else 0
        pages = s["pages"][i, lo // page:-(-keys // page)].long()
        k = s["k"][pages].reshape(-1, n_kv, dim)[:keys - lo].float()
        v = s["v"][pages].reshape(-1, n_kv, dim)[:keys - lo].float()
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


def _plain_sample(s):
    x = s["logits"].double() / s["temp"].double()[:, None]
    w = torch.exp(x - x.amax(1, keepdim=True))
    x, order = torch.sort(w, dim=1, descending=True, stable=True)
    k = s["top_k"].long()[:, None]
    x[(torch.arange(x.shape[1], device=x.device)[None, :] >= k) & (k > 0)] = 0.0
    before = torch.cumsum(x, 1) - x
    p = s["top_p"].double()[:, None]
    x[(before >= p * x.sum(1, keepdim=True)) & (p < 1)] = 0.0
    x[x < s["min_p"].double()[:, None]] = 0.0
    kept = torch.zeros_like(x).scatter_(1, order, x)
    total = torch.cumsum(kept, 1)
    target = s["u"].double()[:, None] * total[:, -1:]
    token = torch.searchsorted(total, target, right=True).clamp_max(x.shape[1] - 1)
    prob = torch.gather(kept, 1, token) / total[:, -1:]
    return token[:, 0].int(), prob[:, 0].float()


def run(s):
    case = s["case"]
    if own:
        from paper_2608_28003_gb300 import binding as B
        if case["op"] == "rope":
            return B.rope(s["table"], s["x"], s["pos"])
        if case["op"] == "append":
            q = B.rope_append(s["table"], s["cache"], s["batch"], s["q"], s["k_new"], s["v_new"], q_norm=s["qn"],
                              k_norm=s["kn"], eps=EPS)
            return q, s["k"], s["v"]
        if case["op"] == "attention":
            return B.paged_attention(s["cache"], s["batch"], s["q"], window=case["window"])
        return B.sample(s["logits"], s["u"], temperature=s["temp"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"],
                        want_probs=True)
    if case["op"] == "rope":
        return _rotate(s["x"].float(), s["pos"], case).to(s["x"].dtype)
    if case["op"] == "append":
        return _plain_append(s)
    if case["op"] == "attention":
        return _plain_attention(s)
    return _plain_sample(s)


def work(case):
    """Each input read once and each output written once; the operations of the formulas."""
    e = 4 if case["type"] == "f32" else 2
    if case["op"] == "rope":
        n = case["t"] * case["heads"] * case["dim"]
        return {"bytes": 2 * n * e + 4 * case["t"], "flops": 3 * case["t"] * case["heads"] * case["rot"]}
    if case["op"] == "sample":
        return {"bytes": case["m"] * (case["vocab"] * e + 28), "flops": 4 * case["m"] * case["vocab"]}
    new, keys = _lengths(case)
    rows, n_q, n_kv, dim = sum(new), case["n_q"], case["n_kv"], case["dim"]
    if case["op"] == "append":
        heads = n_q + 2 * n_kv
        return {"bytes": 2 * rows * heads * dim * e, "flops": rows * (n_q + n_kv) * (3 * case["rot"] + 4 * dim * case["norm"])}
    visible = sum(k - lo for lo, k in _seen(case))
    pairs = 0  # visible (row, key) pairs
    for n, k in zip(new, keys):
        for p in range(k - n, k):
            pairs += min(p + 1, case["window"]) if case["window"] else p + 1
    return {"bytes": 2 * rows * n_q * dim * e + 2 * visible * n_kv * dim * e, "flops": 4 * pairs * n_q * dim}


# ---------------------------------------------------------------------------------------- 64 bits
def _turned(x, pos, case):
    """x [T, H, D] in 64 bits, its pairs as complex numbers times exp(i p f)."""
    rot, t, h = case["rot"], x.shape[0], x.shape[1]
    f, scale = _frequencies(case)
    unit = torch.polar(torch.full((t, rot // 2), scale, dtype=torch.float64, device=x.device),
                       torch.outer(pos.double(), f.to(x.device)))
    part = x[..., :rot].reshape(t, h, rot // 2, 2) if case["inter"] else x[..., :rot].reshape(t, h, 2, rot // 2).transpose(2, 3)
    z = torch.view_as_real(torch.view_as_complex(part.contiguous()) * unit[:, None, :])
    z = z.reshape(t, h, rot) if case["inter"] else z.transpose(2, 3).reshape(t, h, rot)
    return torch.cat([z, x[..., rot:]], -1)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "rope":
        return _turned(s["x"].double(), s["pos"], case)
    if case["op"] == "sample":
        return _exact_sample(case, s)
    dim, page = case["dim"], case["page"]
    if case["op"] == "append":
        def unit(x, w):
            if w is None:
                return x.double()
            x = x.double()
            return x * torch.rsqrt(x.pow(2).sum(-1, keepdim=True) / dim + EPS) * w.double()
        caches = [s["k"].double(), s["v"].double()]
        place = [(i, p) for i, (n, k) in enumerate(zip(s["new"], s["keys"])) for p in range(k - n, k)]
        pos = torch.tensor([p for _, p in place], device=caches[0].device)
        table = s["pages"].cpu()
        at = torch.tensor([int(table[i, p // page]) for i, p in place], device=pos.device)
        caches[0][at, pos % page] = _turned(unit(s["k_new"], s["kn"]), pos, case)
        caches[1][at, pos % page] = s["v_new"].double()
        return _turned(unit(s["q"], s["qn"]), pos, case), caches[0], caches[1]
    return _exact_attention(case, s)


def _exact_attention(case, s):
    n_kv, dim = case["n_kv"], case["dim"]
    group, parts, first = case["n_q"] // n_kv, [], 0
    for i, (n, keys) in enumerate(zip(s["new"], s["keys"])):
        rows = s["q"][first:first + n].double().view(n, n_kv, group, dim)
        first += n
        pages = s["pages"][i, :-(-keys // case["page"])].long()
        k, v = (s[c].index_select(0, pages).flatten(0, 1)[:keys].double().transpose(0, 1) for c in ("k", "v"))  # [n_kv, keys, D]
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


def _exact_sample(case, s):
    tokens, probs = [], []
    logits, u = s["logits"].double().cpu().numpy(), s["u"].double().cpu().numpy()
    temp, top_p, min_p = (float(s[k][0].double()) for k in ("temp", "top_p", "min_p"))
    for row, r in zip(logits, u):
        order = np.lexsort((np.arange(row.size), -row))  # the largest first, the lower index at a tie
        if case["top_k"] > 0:
            order = order[:case["top_k"]]
        w = np.exp((row[order] - row[order[0]]) / temp)
        if top_p < 1.0:
            order = order[:1 + int(np.searchsorted(np.cumsum(w)[:-1], top_p * w.sum(), side="left"))]
            w = w[:order.size]
        keep = w >= min_p
        order, w = order[keep], w[keep]
        by_index = np.argsort(order)
        order, w = order[by_index], w[by_index]
        c = np.cumsum(w)
        i = min(int(np.searchsorted(c, r * c[-1], side="right")), order.size - 1)
        tokens.append(order[i])
        probs.append(w[i] / c[-1])
    return (torch.tensor(np.array(tokens), dtype=torch.int32, device=s["u"].device),
            torch.tensor(np.array(probs), dtype=torch.float64, device=s["u"].device))
