"""Plain implementations of the operators that keep a state of fixed size for a stream (include/rh_seq.h) in 64 bits, for tests only: loops over streams and
tokens, one step of the definition at a time."""
from __future__ import annotations

import numpy as np


def silu(v):
    with np.errstate(over="ignore"):
        return v / (1 + np.exp(-v))


def softplus(v):
    return np.logaddexp(0.0, v)


def _streams(offsets, slots, past, into, n_slots, rows):
    """Of every stream with rows: its rows, the slot that it reads (None: zeros) and the one that it writes (None: none)."""
    offsets = np.arange(rows + 1) if offsets is None else np.clip(offsets, 0, rows)
    into = slots if into is None else into
    for b in range(len(slots)):
        begin, end = int(offsets[b]), int(offsets[b + 1])
        if begin < end:
            keep = 0 <= slots[b] < n_slots and (past is None or past[b] > 0)
            yield begin, end, int(slots[b]) if keep else None, int(into[b]) if 0 <= into[b] < n_slots else None


def conv(x, weight, state, slots, bias=None, offsets=None, past=None, into=None, act=True):
    """x [rows, channels], weight [width, channels], state [n_slots, width - 1, channels] -> (y, state afterwards); NaN in rows of no stream."""
    wide = weight.shape[0]
    y, new = np.full(x.shape, np.nan), np.array(state)
    for begin, end, old, to in _streams(offsets, slots, past, into, state.shape[0], x.shape[0]):
        line = np.concatenate((np.zeros((wide - 1, x.shape[1])) if old is None else state[old], x[begin:end]))
        for t in range(begin, end):
            s = (weight * line[t - begin:t - begin + wide]).sum(0) + (0 if bias is None else bias)
            y[t] = silu(s) if act else s
        if to is not None:
            new[to] = line[end - begin:]
    return y, new


def scan(x, dt, a, b, c, state, slots, skip=None, gate=None, dt_bias=None, soft=True, offsets=None, past=None, into=None):
    """x, dt, gate [rows, channels], a [channels, n], b, c [rows, groups, n], state [n_slots, channels, n] -> (y, state afterwards, sum |c h| of every y);
    NaN in rows of no stream."""
    y, most, new = np.full(x.shape, np.nan), np.zeros(x.shape), np.array(state)
    per = x.shape[1] // b.shape[1]
    for begin, end, old, to in _streams(offsets, slots, past, into, state.shape[0], x.shape[0]):
        h = np.zeros(state.shape[1:]) if old is None else np.array(state[old])
        for t in range(begin, end):
            d = dt[t] + (0 if dt_bias is None else dt_bias)
            d = softplus(d) if soft else d
            h = np.exp(d[:, None] * a) * h + (d * x[t])[:, None] * np.repeat(b[t], per, 0)
            terms = np.repeat(c[t], per, 0) * h
            y[t] = terms.sum(1) + (0 if skip is None else skip * x[t])
            most[t] = np.abs(terms).sum(1)
            if gate is not None:
                y[t] *= silu(gate[t])
        if to is not None:
            new[to] = h
    return y, new, most


def gated_norm(x, gate, weight, groups, eps):
    """-> y; the scale of its 8-bit form is that of oracle.sequence.norm."""
    s = (x * silu(gate)).reshape(x.shape[0], groups, -1)
    return (s / np.sqrt((s * s).mean(-1, keepdims=True) + eps)).reshape(x.shape) * weight
