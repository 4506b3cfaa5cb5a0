"""Plain implementations of the sequence operators (include/rh_seq.h) in 64 bits, for tests only:
loops over streams and tokens, one step of the definition at a time."""
from __future__ import annotations

import numpy as np

AMAX_MIN = 2.0 ** -100
E4M3_MAX = 448.0                      # scales are amax / 448; the kernels' product with 1/448 is within an ulp of fp32
FP4 = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6])


def plan(n_new, lengths, table, free, count, page, n_slots):
    """-> (slots, new_off, new_lengths, new_count, table, free), the last two as they are afterwards."""
    table, free = np.array(table), np.array(free)
    n, width = table.shape
    lengths = [max(0, int(v)) for v in lengths]
    height = min(max(0, int(count)), len(free))
    for b in range(n):
        if n_new[b] < 0:
            for j in range(min(-(-lengths[b] // page), width)):
                if height < len(free):
                    free[height] = table[b, j]
                height += 1
    asked_pages = asked_tokens = taken = 0
    slots, off, after = [], [0], []
    for b in range(n):
        if n_new[b] < 0:
            off.append(off[-1]); after.append(0)
            continue
        have = -(-lengths[b] // page)
        need = -(-(lengths[b] + int(n_new[b])) // page) - have
        ok = have + need <= width
        if ok:
            asked_pages += need
            asked_tokens += int(n_new[b])
            ok = (need == 0 or asked_pages <= height) and asked_tokens <= n_slots
        got = int(n_new[b]) if ok else 0
        if ok:
            for j in range(need):
                table[b, have + j] = free[height - 1 - taken]
                taken += 1
            for i in range(got):
                pos = lengths[b] + i
                slots.append(int(table[b, pos // page]) * page + pos % page)
        off.append(off[-1] + got)
        after.append(lengths[b] + got)
    slots += [-1] * (n_slots - len(slots))
    return np.array(slots), np.array(off), np.array(after), height - taken, table, free


def e4m3_values():
    """The 256 values of e4m3 (codes 0x7F and 0xFF are NaN)."""
    out = np.empty(256)
    for c in range(256):
        s, e, m = c >> 7, c >> 3 & 15, c & 7
        v = m / 8 * 2.0 ** -6 if e == 0 else np.nan if e == 15 and m == 7 else (1 + m / 8) * 2.0 ** (e - 7)
        out[c] = -v if s else v
    return out


def attend(q, k, v, table, lengths, page, scale, window=0):
    """q [n, q_heads, dim]; k, v [n_pages, page, heads, dim] as values in 64 bits -> (out, lse)."""
    n, q_heads, dim = q.shape
    n_pages, _, heads, _ = k.shape
    out, lse = np.zeros((n, q_heads, dim)), np.full((n, q_heads), -np.inf)
    for b in range(n):
        length = min(max(0, int(lengths[b])), table.shape[1] * page)
        pos = np.arange(max(0, length - window) if window else 0, length)
        p = table[b][pos // page] if len(pos) else np.zeros(0, int)
        keep = (p >= 0) & (p < n_pages)
        p, line = p[keep], (pos % page)[keep]
        if len(p) == 0:
            continue
        for h in range(q_heads):
            c = h // (q_heads // heads)
            s = k[p, line, c] @ q[b, h] * scale
            e = np.exp(s - s.max())
            out[b, h] = e @ v[p, line, c] / e.sum()
            lse[b, h] = s.max() + np.log(e.sum())
    return out, lse


def norm(x, weight, residual, eps):
    """-> (sum, y, scale of the 8-bit form)."""
    s = x if residual is None else x + residual
    y = s / np.sqrt((s * s).mean(-1, keepdims=True) + eps) * weight
    return s, y, np.maximum(np.abs(y).max(-1), AMAX_MIN) / E4M3_MAX


def unpack_weights(w, w_scale, n_in):
    n, blocks = w_scale.shape
    code = np.empty((n, 32 * blocks), int)
    code[:, 0::2], code[:, 1::2] = w & 15, w >> 4
    factor = np.where(w_scale == 255, np.nan, np.exp2(w_scale.astype(np.float64) - 127))
    return (FP4[code].reshape(n, blocks, 32) * factor[..., None]).reshape(n, -1)[:, :n_in]


def matvec(x, w, w_scale, x_scale=None, relu=False):
    y = x @ unpack_weights(w, w_scale, x.shape[1]).T
    if x_scale is not None:
        y = y * x_scale[:, None]
    return np.maximum(y, 0) if relu else y
