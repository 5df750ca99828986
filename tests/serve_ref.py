"""Plain float64 definitions of normalised heads and of the verification of drafted tokens, for the tests: one row, one
token at a time, on the host. Shares no code with the library. (Attention over shared prefixes is the attention of
draft_ref.)"""
from __future__ import annotations

import math

import numpy as np

import draft_ref as D


def deal(sections, order):
    """Axis of every pair."""
    if order == "blocks":
        return [a for a, n in enumerate(sections) for _ in range(n)]
    left, out = list(sections), []
    while sum(left):
        for a in range(len(left)):
            if left[a] > 0:
                out.append(a)
                left[a] -= 1
    return out


def section_freqs(sections, order, theta, rdim, own):
    """(axis, frequency) of every pair."""
    axis, seen, f = deal(sections, order), [0] * len(sections), []
    for i, a in enumerate(axis):
        f.append(theta ** (-2.0 * seen[a] / (2 * sections[a])) if own else theta ** (-2.0 * i / rdim))
        seen[a] += 1
    return np.array(axis), np.array(f)


def heads(x, pos, axis, f, rdim, interleaved, gain_q=None, gain_k=None, n_q=0, eps=0.0, amp=1.0):
    """x [rows, heads, D] float64; pos [rows, axes]. Returns (y, bound per element)."""
    x = np.array(x, np.float64)
    if gain_q is not None or gain_k is not None:
        rms = np.sqrt((x * x).mean(-1, keepdims=True) + eps)
        x = x / rms
        for h in range(x.shape[1]):
            x[:, h] *= gain_q if h < n_q else gain_k
    y = x.copy()
    ang = np.asarray(pos, np.float64)[:, axis] * f
    i = np.arange(rdim // 2)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rdim // 2)
    c, s = amp * np.cos(ang)[:, None, :], amp * np.sin(ang)[:, None, :]
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
    # Half a bf16 step of the result; the rotation in fp32 as in draft_ref.rotate_bound (2^-20 of |a| + |b|); the norm in
    # fp32: squares and sums of at most 16 values of a lane and 5 sums of lanes, each rounding 2^-24 of a positive sum,
    # under 2^-19 of it, half of that in its root; root, mean and two products add 2^-21: 2^-19 of a value in all.
    t = D.U_BF16 * np.abs(y) + 2.0 ** -19 * np.abs(y)
    part = (2.0 ** -20 + 2.0 ** -19) * abs(amp) * (np.abs(x[..., a]) + np.abs(x[..., b]))
    t[..., a] += part
    t[..., b] += part
    return y, t


def positive(v):
    """Probabilities as the verification takes them: negative or not finite ones are 0."""
    v = np.asarray(v, np.float64)
    return np.where((v > 0) & np.isfinite(v), v, 0.0)


def draw(w, u):
    """The first token whose running sum exceeds u of the whole, the last one of some probability, or -1."""
    total, run, last = math.fsum(w), 0.0, -1
    for t in np.flatnonzero(w > 0):
        run += w[t]
        last = int(t)
        if run > u * total:
            return last
    return last


def verify(row_off, rows, max_rows, tokens, parent, target, proposal, accept_u, next_u, path_cols, vocab):
    """(path [B, path_cols], path_len [B], next [B])."""
    B = len(row_off) - 1
    path, lens, nxt = np.full((B, path_cols), -1, np.int32), np.zeros(B, np.int32), np.full(B, -1, np.int32)
    for b in range(B):
        r0, e = int(row_off[b]), min(int(row_off[b + 1]), rows)
        n = min(e - r0, max_rows) if 0 <= r0 < rows and e > r0 else 0
        if n == 0:
            continue
        kids = {}
        for j in range(1, n):
            if 0 <= parent[r0 + j] < j and 0 <= tokens[r0 + j] < vocab:
                kids.setdefault(int(parent[r0 + j]), []).append(j)
        cur, keep = 0, [0]
        while True:
            w, z, went = positive(target[r0 + cur]), 1.0, None
            if len(keep) < path_cols:
                q = None if proposal is None else positive(proposal[r0 + cur])
                for c in kids.get(cur, []):
                    x, u = int(tokens[r0 + c]), float(accept_u[r0 + c])
                    if w[x] > 0 and u * z * (1.0 if q is None else q[x]) < w[x]:
                        went = c
                        break
                    if q is None:
                        z -= w[x]
                        w[x] = 0.0
                    else:
                        w = np.maximum(w - z * q, 0.0)
                        z = math.fsum(w)
            if went is None:
                break
            cur = went
            keep.append(cur)
        nxt[b] = draw(w, float(next_u[b]))
        if nxt[b] < 0:
            nxt[b] = draw(positive(target[r0 + cur]), float(next_u[b]))
        path[b, :len(keep)] = keep
        lens[b] = len(keep)
    return path, lens, nxt
