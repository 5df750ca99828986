"""Plain float64 definitions of the drafted-row operators, rotary positions and page moves, for the tests: one
sequence, one row, one head at a time, on the host. Shares no code with the library."""
from __future__ import annotations

import math

import numpy as np
import torch

PAGE = 16
U_BF16 = 2.0 ** -8  # half a step of bf16, relative


def freqs(rdim, theta, scaling="plain", factor=1.0, orig=8192.0, hi=None, lo=None):
    out = []
    for i in range(rdim // 2):
        f = theta ** (-2.0 * i / rdim)
        if scaling == "linear":
            f /= factor
        elif scaling == "base" and rdim > 2:
            f *= factor ** (-2.0 * i / (rdim - 2))
        elif scaling == "rotations":
            w = min(1.0, max(0.0, (orig * f / (2 * math.pi) - lo) / (hi - lo)))
            f = w * f + (1 - w) * f / factor
        elif scaling == "index":
            a, b = (rdim * math.log(orig / (2 * math.pi * n)) / (2 * math.log(theta)) for n in (hi, lo))
            a, b = max(0, math.floor(a)), min(rdim - 1, math.ceil(b))
            w = min(1.0, max(0.0, (i - a) / max(b - a, 0.001)))
            f = (1 - w) * f + w * f / factor
        out.append(f)
    return np.array(out)


def rotate(x, pos, f, rdim, interleaved, amp=1.0):
    """x [..., heads, D] float64 at positions pos [...]."""
    y = np.array(x, dtype=np.float64)
    ang = np.asarray(pos, np.float64)[..., None, None] * f
    c, s = amp * np.cos(ang), amp * np.sin(ang)
    i = np.arange(rdim // 2)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rdim // 2)
    u, v = x[..., a], x[..., b]
    y[..., a], y[..., b] = u * c - v * s, v * c + u * s
    return y


def rotate_bound(x, y, rdim, interleaved, amp=1.0):
    """Per element: half a bf16 step of the result, and fp32's part. The reduced angle (below pi) is rounded to fp32
    (2^-24 of it), sin and cos are good to 2 fp32 steps, two products and a sum round once each: under 2^-20 of
    amp (|a| + |b|) together."""
    i = np.arange(rdim // 2)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rdim // 2)
    t = U_BF16 * np.abs(y)
    part = 2.0 ** -20 * abs(amp) * (np.abs(x[..., a]) + np.abs(x[..., b]))
    t[..., a] += part
    t[..., b] += part
    t[..., rdim:] = 0.0
    return t


def forest(n, rng, spread=4):
    """A random forest of n drafted tokens: (depth, ancestor sets with the token itself, paths root..j)."""
    depth, anc = [], []
    for j in range(n):
        p = j - 1 - int(rng.integers(0, spread))
        if p < 0:
            depth.append(0)
            anc.append([j])
        else:
            depth.append(depth[p] + 1)
            anc.append(anc[p] + [j])
    return depth, anc


def mask_words(sets, max_rows):
    """[n, words] int64 bit patterns of sets of drafted indices."""
    words = -(-max_rows // 64)
    out = np.zeros((len(sets), words), np.uint64)
    for r, s in enumerate(sets):
        for j in s:
            out[r, j // 64] |= np.uint64(1) << np.uint64(j % 64)
    return out.view(np.int64)


def slot(pool, table_row, t, ring, n_kv, D):
    """(k, v) [n_kv, D] of token position t, or None without a page."""
    lp = t // PAGE
    if ring:
        lp %= ring
    elif lp >= len(table_row):
        return None
    page = int(table_row[lp])
    if not 0 <= page < pool.shape[0]:
        return None
    blk = pool[page].reshape(2, n_kv, PAGE * D)
    k = blk[0].reshape(n_kv, PAGE, D)[:, t % PAGE]
    v = blk[1].reshape(n_kv, D, PAGE)[:, :, t % PAGE]
    return k, v


def tree_attention(q, pool, table, ctx, row_off, depth, sets, n_kv, window=0, ring=0, max_rows=256):
    """q [rows, n_q, D] float64; pool [P, 2, n_kv, 16 D] float64; sets[r]: drafted indices row r sees. Returns (o,
    weight of |v| under the same softmax), NaN rows where the definition is NaN; rows outside every sequence None."""
    R, n_q, D = q.shape
    o, mag = np.full((R, n_q, D), np.nan), np.full((R, n_q, D), np.nan)
    touched = np.zeros(R, bool)
    group = n_q // n_kv
    for b in range(len(ctx)):
        r0, n = int(row_off[b]), min(int(row_off[b + 1]) - int(row_off[b]), max_rows)   # rows past max_rows are padding
        for j in range(n):
            r = r0 + j
            touched[r] = True
            o[r] = mag[r] = 0.0
            if ctx[b] < 0:
                continue
            p = int(ctx[b]) + int(depth[r])
            seen = [t for t in range(max(0, p - window + 1) if window else 0, int(ctx[b]))]
            seen += [int(ctx[b]) + i for i in sorted(sets[r]) if i < n and (not window or depth[r0 + i] > depth[r] - window)]
            kv = [slot(pool, table[b], t, ring, n_kv, D) for t in seen]
            kv = [x for x in kv if x is not None]
            if not kv:
                continue
            K, V = np.stack([x[0] for x in kv]), np.stack([x[1] for x in kv])
            for h in range(n_q):
                s = K[:, h // group] @ q[r, h] / math.sqrt(D)
                w = np.exp(s - s.max())
                w /= w.sum()
                o[r, h] = w @ V[:, h // group]
                mag[r, h] = w @ np.abs(V[:, h // group])
    return o, mag, touched


def tree_bound(o, mag):
    """Per element: half a bf16 step of the result, half a step of every probability before the product (their sum in
    the denominator is not rounded), and 2 % more of the latter for fp32's part: scores of at most 2^4 with sums of
    128 products, off by less than 2^-24 * 128 * 2^4 = 2^-13 of a probability, a 32nd of its bf16 half step."""
    return U_BF16 * np.abs(o) + U_BF16 * (1 + 1 / 32) * mag


def accept(pools, tables, rings, ctx, row_off, path, path_len, n_kvs, Ds):
    """Moves the slots of each path in every pool [P, 2, n_kv, 16 D] (any dtype, in place); returns new contexts."""
    out = np.array(ctx).copy()
    for b in range(len(ctx)):
        n = int(row_off[b + 1]) - int(row_off[b])
        if ctx[b] < 0:
            continue
        last, keep = -1, []
        for k in range(min(max(int(path_len[b]), 0), path.shape[1])):
            if not last < path[b, k] < n:
                break
            last = int(path[b, k])
            keep.append(last)
        out[b] = ctx[b] + len(keep)
        for pool, table, ring, n_kv, D in zip(pools, tables, rings, n_kvs, Ds):
            for k, i in enumerate(keep):
                a = slot(pool, table[b], int(ctx[b]) + i, ring, n_kv, D)
                z = slot(pool, table[b], int(ctx[b]) + k, ring, n_kv, D)
                if a is None or z is None:
                    continue
                z[0][...] = np.array(a[0])
                z[1][...] = np.array(a[1])
    return out


def bits(t: torch.Tensor) -> np.ndarray:
    """bf16 tensor as its int16 bit patterns on the host."""
    return t.contiguous().view(torch.int16).cpu().numpy()
