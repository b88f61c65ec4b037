"""A serving step's operators in numpy, 64 bits, row by row from their definitions: rotary positions, the append
of keys and values to a paged cache, attention of a ragged batch over it, and sampling."""
from __future__ import annotations

import math

import numpy as np


def rope_frequencies(rot, base, scaling="none", factor=1.0, low=1.0, high=4.0, original_len=0, attn_factor=0.0):
    """Radians a position of the rot / 2 pairs, and the factor on cos and sin."""
    out = []
    at = lambda x: rot * math.log(original_len / (2 * math.pi * x)) / (2 * math.log(base))  # noqa: E731
    for i in range(rot // 2):
        f = base ** (-2.0 * i / rot)
        if scaling == "linear":
            f /= factor
        elif scaling == "wavelength":
            wave = 2 * math.pi / f
            if wave > original_len / low:
                f /= factor
            elif wave >= original_len / high:
                m = (original_len / wave - low) / (high - low)
                f = (1 - m) * f / factor + m * f
        elif scaling == "parts":
            a, b = max(0, math.floor(at(high))), min(rot - 1, math.ceil(at(low)))
            r = min(1.0, max(0.0, (i - a) / max(b - a, 0.001)))
            f = f * (1 - r) + f / factor * r
        out.append(f)
    s = attn_factor if attn_factor > 0 else (0.1 * math.log(factor) + 1.0 if scaling == "parts" and factor > 1 else 1.0)
    return np.array(out), s


def rope(x, positions, freqs, scale, interleaved):
    """x [T, heads, dim] rotated at positions [T]."""
    x = np.asarray(x, np.float64)
    y = x.copy()
    n = len(freqs)
    for i in range(n):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + n)
        angle = np.asarray(positions, np.float64) * freqs[i]
        c, s = (np.cos(angle) * scale)[:, None], (np.sin(angle) * scale)[:, None]
        y[..., a] = x[..., a] * c - x[..., b] * s
        y[..., b] = x[..., b] * c + x[..., a] * s
    return y


def rms_norm(x, w, eps):
    x = np.asarray(x, np.float64)
    return x if w is None else x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * np.asarray(w, np.float64)


def rows_of(batch, page_size):
    """(row, sequence, position, keys) of every row of a sequence; batch: dict of row_start, kv_len, pages [n, wide],
    n_rows."""
    wide = batch["pages"].shape[1]
    for s in range(len(batch["kv_len"])):
        r0, r1 = (min(max(int(batch["row_start"][s + i]), 0), batch["n_rows"]) for i in (0, 1))
        keys = min(max(int(batch["kv_len"][s]), 0), wide * page_size)
        for r in range(r0, r1):
            yield r, s, keys - (r1 - r0) + r - r0, keys


def place(batch, n_pages, page_size, s, p):
    """(page, slot) of position p of sequence s; None where no page holds it."""
    col = p // page_size
    if p < 0 or col >= batch["pages"].shape[1]:
        return None
    page = int(batch["pages"][s, col])
    return (page, p % page_size) if 0 <= page < n_pages else None


def attention(q, k, v, batch, scale, window=0, rows=None):
    """q [T, n_q, D], k and v [pages, page_size, n_kv, D] -> (o, sum of weight * |v| per output, the largest
    sum |q_d k_d| per row and head); rows of no sequence are NaN."""
    q, k, v = (np.asarray(t, np.float64) for t in (q, k, v))
    T, n_q, dim = q.shape
    n_pages, page, n_kv, _ = k.shape
    o, mass, mag = np.full(q.shape, np.nan), np.zeros(q.shape), np.zeros(q.shape[:2])
    for r, s, pos, _ in rows_of(batch, page):
        if rows is not None and r not in rows:
            continue
        lo = max(0, pos - window + 1) if window else 0
        at = [place(batch, n_pages, page, s, p) for p in range(lo, pos + 1)]
        at = [a for a in at if a is not None]
        o[r] = 0.0
        if not at:
            continue
        pg, sl = np.array(at).T
        for h in range(n_q):
            kk, vv = k[pg, sl, h // (n_q // n_kv)], v[pg, sl, h // (n_q // n_kv)]
            with np.errstate(all="ignore"):
                x = kk @ q[r, h] * scale
                w = np.exp(x - (x.max() if not np.isnan(x).any() else np.nan))
                w /= w.sum()
                o[r, h] = (w[:, None] * vv).sum(0)
                mass[r, h] = (w[:, None] * np.abs(vv)).sum(0)
                mag[r, h] = (np.abs(kk) @ np.abs(q[r, h])).max()
    return o, mass, mag


def sample(row, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, its share of the kept weight, kept tokens) of one row of logits."""
    row = np.asarray(row, np.float64)
    row = np.where(np.isnan(row), -np.inf, row)
    top = row.max()
    if top == -np.inf:
        return -1, 0.0, 0
    if not temperature > 0:
        return int(np.argmax(row)), 1.0, 1
    if top == np.inf:
        w = (row == np.inf).astype(np.float64)
    else:
        w = np.exp((row - top) / np.float64(np.float32(temperature)))
        w[w < 2.0 ** -43] = 0.0
    order = sorted(range(len(row)), key=lambda i: (-row[i], i))
    if top_k > 0:
        order = order[:top_k]
    if top_p < 1:
        goal, have, cut = float(np.float32(top_p)) * math.fsum(w[order]), [], []
        for i in order:
            if cut and math.fsum(have) >= goal:
                break
            cut.append(i)
            have.append(w[i])
        order = cut
    order = order[:1] + [i for i in order[1:] if not min_p > 0 or w[i] >= float(np.float32(min_p)) or w[i] == 1.0]
    kept = sorted(order)
    total, run = math.fsum(w[kept]), 0.0
    u = 0.0 if not u >= 0 else min(float(u), 1 - 2.0 ** -24)
    for i in kept:
        run += w[i]
        if run > u * total:
            return i, w[i] / total, int((w[kept] > 0).sum())
    return kept[-1], w[kept[-1]] / total, int((w[kept] > 0).sum())
