"""Operators for several tokens per sequence on the paged KV cache, as timed and compared cases.

Three kinds of operator, each with its plain form (elementary torch operations
in 32 bits, rounded once at the end) and the package's own call:

  rope    rotary positions of the q and k heads of qkv rows: interleaved and
          half layouts, part of the head, frequencies scaled for long contexts
  tree    attention of a tree of drafted tokens per sequence over the paged
          cache: every row sees the cached tokens in its window and the drafted
          rows its mask names
  accept  the accepted path of each tree kept: its slots of the cache move to
          the front of the drafted ones, in every layer
  copy    pages copied inside the pools of every layer (forks, compaction)

A KV page holds 16 tokens, [2][n_kv][16 * D]: keys row-major, then values
dim-major. Head layouts are those of the repository's workloads (8B-shaped
layer, MoE layer, tensor-parallel share, tiny layer, narrow 64-wide heads).
"""
import math

import numpy as np
import torch

own = False

PAGE = 16


# ---------------------------------------------------------------- cases

def _rope(rows, heads, D, rdim, layout, scaling, pos_hi, **kw):
    """x is the first `heads` heads of rows of heads + extra heads (a qkv row's v heads follow)."""
    return dict(op="rope", rows=rows, heads=heads, extra=kw.pop("extra", 0), D=D, rdim=rdim, layout=layout,
                scaling=scaling, factor=kw.pop("factor", 8.0), orig=kw.pop("orig", 8192), theta=kw.pop("theta", 10000.0),
                amp=kw.pop("amp", 1.0), pos_hi=pos_hi, **kw)


def _tree(batch, rows_lo, rows_hi, n_q, n_kv, D, ctx_lo, ctx_hi, window=0, **kw):
    return dict(op="tree", batch=batch, rows_lo=rows_lo, rows_hi=rows_hi, n_q=n_q, n_kv=n_kv, D=D, ctx_lo=ctx_lo,
                ctx_hi=ctx_hi, window=window, **kw)


def _accept(batch, rows, n_kv, D, ctx_lo, ctx_hi, layers, **kw):
    return dict(op="accept", batch=batch, rows=rows, n_kv=n_kv, D=D, ctx_lo=ctx_lo, ctx_hi=ctx_hi, layers=layers, **kw)


def _copy(pairs, pages, n_kv, D, layers, **kw):
    return dict(op="copy", pairs=pairs, pages=pages, n_kv=n_kv, D=D, layers=layers, **kw)


def listed():
    return [
        # The tiny layer's decode step: 4 q and 2 k heads of 64, all latency.
        _rope(4, 6, 64, 64, "half", "plain", 128, extra=2, name="rope_tiny"),
        # A decode step of 64 long-context requests on the 8B-shaped layer: scaled frequencies, far positions.
        _rope(64, 40, 128, 128, "half", "index", 131072, extra=8, factor=16.0, theta=500000.0, amp=1.25,
              name="rope_b64_scaled"),
        # A prompt's worth of rows, half of each head rotated in the interleaved layout.
        _rope(8192, 40, 128, 64, "interleaved", "base", 32768, extra=8, name="rope_8192_part"),
        # The tiny layer with 8 drafted tokens for each of 4 sequences.
        _tree(4, 8, 8, 4, 2, 64, 128, 128, name="tree_tiny"),
        # One interactive request on the 8B-shaped layer, 16 drafted tokens.
        _tree(1, 16, 16, 32, 8, 128, 3000, 3000, name="tree_b1"),
        # Ordinary serving load: ragged contexts and ragged trees of up to 24 tokens.
        _tree(64, 1, 24, 32, 8, 128, 512, 4096, name="tree_b64_ragged"),
        # A sliding-window layer of the hybrid block, 32 tokens a tree.
        _tree(32, 32, 32, 32, 8, 128, 1024, 16384, 1024, name="tree_b32_window"),
        # High load: 64 sequences of 8192 tokens, the widest one-word trees.
        _tree(64, 64, 64, 32, 8, 128, 8192, 8192, name="tree_b64_r64"),
        # The accepted paths of 64 trees of 16, one layer: a short list of slots.
        _accept(64, 16, 8, 128, 64, 256, 1, name="accept_b64"),
        # 256 trees of 64 over a 4-layer block.
        _accept(256, 64, 8, 128, 64, 256, 4, name="accept_b256_l4"),
        # 64 forked sequences take copies of their last pages in a 4-layer block.
        _copy(64, 1024, 8, 128, 4, name="copy_fork"),
        # A pool's upper pages compacted into its free lower ones, two layers.
        _copy(4001, 10000, 8, 128, 2, name="copy_compact"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _fits(c):
    """Within the listed cases' cost: the plain form's gathered keys and scores, the pools, the work."""
    w = work(c)
    if c["op"] == "tree":
        t = c["ctx_hi"] + c["rows_hi"] + PAGE
        if c["batch"] * t * c["n_kv"] * c["D"] > 5.5e8 or c["batch"] * c["rows_hi"] * c["n_q"] * t > 1.1e9:
            return False
    if c["op"] == "accept" and c["batch"] * (c["ctx_hi"] + c["rows"] + PAGE) * 4 * c["n_kv"] * c["D"] * c["layers"] > 1.5e9:
        return False
    return w["bytes"] <= 2.2e9 and w["flops"] <= 5.5e11


def draw(rng):
    while True:
        op = rng.choice(["rope", "rope", "tree", "tree", "tree", "accept", "copy"])
        if op == "rope":
            D = rng.choice([64, 64, 96, 128, 128, 256])
            rdim = rng.choice([D, D, D // 2, D // 4, 2 * rng.randint(2, D // 2)])
            c = _rope(_log_int(rng, 1, 8192), rng.randint(1, 40), D, rdim, rng.choice(["half", "interleaved"]),
                      rng.choice(["plain", "linear", "base", "rotations", "index"]), _log_int(rng, 16, 1 << 20),
                      extra=rng.choice([0, 1, 8]), factor=rng.choice([2.0, 4.0, 8.0, 32.0]),
                      theta=rng.choice([10000.0, 500000.0, 1000000.0]), amp=rng.choice([1.0, 1.25]))
        elif op == "tree":
            hi = _log_int(rng, 16, 32768)
            rows = _log_int(rng, 1, 128)
            n_kv = rng.choice([1, 2, 4, 8])
            c = _tree(_log_int(rng, 1, 256), max(1, int(rows * rng.uniform(0.1, 1.0))), rows,
                      n_kv * rng.choice([1, 2, 4, 8, 16] if n_kv < 8 else [1, 4]), n_kv, rng.choice([64, 128]),
                      max(1, int(hi * rng.uniform(0.05, 1.0))), hi, rng.choice([0, 0, 0, 100, 1024, 4096]))
        elif op == "accept":
            hi = _log_int(rng, 8, 2000)
            c = _accept(_log_int(rng, 1, 256), _log_int(rng, 1, 128), rng.choice([1, 2, 4, 8]), rng.choice([64, 128]),
                        max(1, hi // 3), hi, rng.choice([1, 2, 4]))
        else:
            pairs = _log_int(rng, 1, 5000)
            c = _copy(pairs, 2 * pairs + rng.randint(1, 2000), rng.choice([1, 2, 4, 8]), rng.choice([64, 128]),
                      rng.choice([1, 2, 4]))
            if work(c)["bytes"] * (c["pages"] / (2 * pairs)) > 1.6e9:
                continue
        if _fits(c):
            return c


# ---------------------------------------------------------------- sizes and work, from the case alone

def _tree_rows(c):
    """Drafted rows of each sequence; the first has the most."""
    rows = np.random.default_rng(13).integers(c["rows_lo"], c["rows_hi"] + 1, c["batch"]).astype(np.int64)
    rows[0] = c["rows_hi"]
    return rows


def work(case):
    c = case
    if c["op"] == "rope":
        n = c["rows"] * c["heads"] * c["D"]
        return {"bytes": 4 * n + 4 * c["rows"], "flops": 3 * c["rows"] * c["heads"] * c["rdim"]}
    if c["op"] == "tree":
        rows = float(_tree_rows(c).sum())
        mean_ctx = (c["ctx_lo"] + c["ctx_hi"]) / 2
        seen = min(mean_ctx, c["window"]) if c["window"] else mean_ctx
        mean_rows = rows / c["batch"]
        return {"bytes": (c["batch"] * seen + rows) * c["n_kv"] * c["D"] * 4 + 2 * rows * c["n_q"] * c["D"] * 2,
                "flops": 4 * rows * (seen + mean_rows) * c["n_q"] * c["D"]}
    if c["op"] == "accept":
        moved = c["batch"] * min(c["rows"], 12) / 2  # the mean accepted length; what stays in its place still counts as kept
        return {"bytes": c["layers"] * moved * c["n_kv"] * c["D"] * 4 * 2 + 8 * c["batch"], "flops": 0}
    return {"bytes": c["layers"] * c["pairs"] * PAGE * c["n_kv"] * c["D"] * 4 * 2, "flops": 0}


# ---------------------------------------------------------------- inputs

def _g(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(shape, g):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(torch.bfloat16)


def _forest(rows, n, r):
    """Trees of rows[b] <= n drafted tokens: each token's parent is a recent earlier one, or the last cached token.
    Depths [B, n] and ancestor masks [B, n, words] with each token's own bit."""
    B, words = len(rows), -(-n // 64)
    depth = np.zeros((B, n), np.int32)
    mask = np.zeros((B, n, words), np.uint64)
    at = np.arange(B)
    for j in range(n):
        parent = j - 1 - r.integers(0, 4, B)
        has = parent >= 0
        p = np.maximum(parent, 0)
        depth[:, j] = np.where(has, depth[at, p] + 1, 0)
        mask[:, j] = np.where(has[:, None], mask[at, p], 0)
        mask[:, j, j // 64] |= np.uint64(1) << np.uint64(j % 64)
    return depth, mask


def _paths(rows, lens, r):
    """Increasing draft indices, `lens` of them at most, of trees of rows[b] tokens."""
    width = max(1, int(max(lens)))
    step = r.integers(1, 5, (len(rows), width))
    idx = np.cumsum(step, axis=1) - 1
    n = np.minimum(lens, (idx < rows[:, None]).sum(axis=1))
    return idx.astype(np.int32), n.astype(np.int32)


def _pages(ctx, extra, r):
    """A shuffled page table that covers ctx + extra tokens of each sequence, and the pool's page count."""
    need = -(-(ctx + extra) // PAGE)
    P = int(need.sum()) + 8
    ids = r.permutation(P).astype(np.int32)
    table = np.full((len(ctx), int(need.max())), -1, np.int32)
    off = 0
    for b, n in enumerate(need):
        table[b, :n] = ids[off:off + n]
        off += n
    return table, P


def _cuda(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def prepare(case, seed):
    c, g, r = case, _g(seed), np.random.default_rng(seed)
    s = {"case": c}
    if c["op"] == "rope":
        D = c["D"]
        rows = _normal((c["rows"], c["heads"] + c["extra"], D), g)
        s["x"] = rows[:, :c["heads"]]
        s["y"] = torch.empty((c["rows"], c["heads"], D), dtype=torch.bfloat16, device="cuda")
        s["pos"] = _cuda(r.integers(0, c["pos_hi"], c["rows"]).astype(np.int32))
        s["freqs"] = _cuda(_freqs(c))
    elif c["op"] == "tree":
        rows, n = _tree_rows(c), c["rows_hi"]
        ctx = r.integers(c["ctx_lo"], c["ctx_hi"] + 1, c["batch"]).astype(np.int64)
        depth, mask = _forest(rows, n, r)
        table, P = _pages(ctx, rows, r)
        off = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
        live = np.arange(n)[None, :] < rows[:, None]
        s["ctx"], s["table"], s["off"] = _cuda(ctx.astype(np.int32)), _cuda(table), _cuda(off)
        s["depth"], s["mask"] = _cuda(depth[live]), _cuda(mask[live].view(np.int64))
        s["total"], s["tokens"] = int(off[-1]), int((ctx + rows).max())
        s["pool"] = _normal((P, 2, c["n_kv"], PAGE * c["D"]), g)
        s["qkv"] = _normal((s["total"], (c["n_q"] + 2 * c["n_kv"]) * c["D"]), g)
    elif c["op"] == "accept":
        B = c["batch"]
        ctx = r.integers(c["ctx_lo"], c["ctx_hi"] + 1, B).astype(np.int64)
        rows = np.full(B, c["rows"], np.int64)
        depth, mask = _forest(rows, c["rows"], r)
        table, _ = _pages(ctx, rows, r)
        P = B * -(-(c["ctx_hi"] + c["rows"]) // PAGE) + 8
        idx, n = _paths(rows, r.integers(0, min(c["rows"], 12) + 1, B), r)
        s["ctx"], s["table"] = _cuda(ctx.astype(np.int32)), _cuda(table)
        s["off"] = _cuda((np.arange(B + 1) * c["rows"]).astype(np.int32))
        s["depth"], s["mask"] = _cuda(depth.reshape(-1)), _cuda(mask.reshape(B * c["rows"], -1).view(np.int64))
        s["idx"], s["n"], s["total"] = _cuda(idx), _cuda(n), B * c["rows"]
        s["pools"] = _normal((c["layers"], P, 2, c["n_kv"], PAGE * c["D"]), g)
        s["ctx_out"] = torch.empty_like(s["ctx"])
    else:
        ids = r.permutation(c["pages"])[:2 * c["pairs"]].astype(np.int32)
        s["pairs"] = _cuda(ids.reshape(2, -1).T)
        s["pools"] = _normal((c["layers"], c["pages"], 2, c["n_kv"], PAGE * c["D"]), g)
    if own:
        _handles(s)
    return s


class _Cfg:
    """One layer's shape, as the package's DeviceBlock reads it."""

    def __init__(self, n_q, n_kv, D, window=0):
        self.hidden, self.ffn, self.n_experts, self.top_k, self.moe_ffn = 256, 256, 0, 0, 0
        self.n_q, self.n_kv, self.head_dim, self.window = n_q, n_kv, D, window
        self.rope_theta, self.rms_eps = 10000.0, 1e-6


def _handles(s):
    """The objects a serving program keeps across steps: the block, the batch, the draft, the live buffers."""
    from paper_2609_14237_amd import runtime as R
    c = s["case"]
    if c["op"] == "rope":
        s["rope"] = R.Rope(c["D"], theta=c["theta"], rotary_dim=c["rdim"], interleaved=c["layout"] == "interleaved",
                           scaling=c["scaling"], factor=c["factor"], orig_ctx=c["orig"], amplitude=c["amp"])
        return
    if c["op"] == "tree":
        s["block"] = R.DeviceBlock([_Cfg(c["n_q"], c["n_kv"], c["D"], c["window"])], [{}], [s["pool"]], s["pool"].shape[0])
        s["batch"] = R.DeviceBatch(s["ctx"], s["table"])
        s["draft"] = R.DeviceDraft(s["off"], s["depth"], s["mask"], max_rows=c["rows_hi"])
        s["state"] = R.DeviceState(s["block"], s["batch"], draft=s["draft"])
        s["state"].view("qkv", *s["qkv"].shape).copy_(s["qkv"])
        return
    L, P = s["pools"].shape[:2]
    cfgs = [_Cfg(c["n_kv"], c["n_kv"], c["D"])] * L
    s["block"] = R.DeviceBlock(cfgs, [{}] * L, list(s["pools"].unbind(0)), P)
    if c["op"] == "accept":
        s["batch"] = R.DeviceBatch(s["ctx"], s["table"])
        s["draft"] = R.DeviceDraft(s["off"], s["depth"], s["mask"], max_rows=c["rows"])


# ---------------------------------------------------------------- plain forms

def _freqs(c):
    """Angle per position of each rotated pair, float64 [rdim / 2]."""
    i = np.arange(c["rdim"] // 2, dtype=np.float64)
    theta, f, d = c["theta"], c["factor"], c["rdim"]
    if c["scaling"] == "base" and d > 2:
        theta = theta * f ** (d / (d - 2))
    inv = theta ** (-2.0 * i / d)
    if c["scaling"] == "linear":
        inv = inv / f
    if c["scaling"] == "rotations":  # kept from 4 turns over the first context up, divided from 1 turn down
        keep = np.clip((c["orig"] * inv / (2 * np.pi) - 1.0) / 3.0, 0.0, 1.0)
        inv = inv * keep + inv / f * (1.0 - keep)
    if c["scaling"] == "index":  # the same between the pairs that turn 32 times and once, linear in the pair's index
        at = lambda turns: d * np.log(c["orig"] / (turns * 2 * np.pi)) / (2 * np.log(c["theta"]))  # noqa: E731
        lo, hi = max(np.floor(at(32.0)), 0.0), min(np.ceil(at(1.0)), d - 1.0)
        ramp = np.clip((i - lo) / max(hi - lo, 0.001), 0.0, 1.0)
        inv = inv / f * ramp + inv * (1.0 - ramp)
    return inv


def _plain_rope(s):
    c, x = s["case"], s["x"].float()
    r = c["rdim"]
    ang = torch.remainder(s["pos"].double()[:, None] * s["freqs"], 2 * math.pi).float()
    cos, sin = (torch.cos(ang) * c["amp"])[:, None, :], (torch.sin(ang) * c["amp"])[:, None, :]
    y = x.clone()
    if c["layout"] == "half":
        a, b = x[..., :r // 2], x[..., r // 2:r]
        y[..., :r // 2], y[..., r // 2:r] = a * cos - b * sin, b * cos + a * sin
    else:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        y[..., 0:r:2], y[..., 1:r:2] = a * cos - b * sin, b * cos + a * sin
    return y.to(torch.bfloat16)


def _plain_tree(s):
    """All sequences at once, padded to the longest context and the most rows."""
    c = s["case"]
    B, N, G, D, g = c["batch"], c["rows_hi"], c["n_kv"], c["D"], c["n_q"] // c["n_kv"]
    dev = s["ctx"].device
    off, ctx = s["off"].long(), s["ctx"].long()
    P = -(-s["tokens"] // PAGE)
    T = P * PAGE
    pages = s["table"][:, :P].long().clamp(min=0)
    kv = s["pool"][pages]                                                  # [B, P, 2, G, 16 D]
    K = kv[:, :, 0].reshape(B, P, G, PAGE, D).permute(0, 2, 1, 3, 4).reshape(B, G, T, D).float()
    V = kv[:, :, 1].reshape(B, P, G, D, PAGE).permute(0, 2, 1, 4, 3).reshape(B, G, T, D).float()
    j = torch.arange(N, device=dev)
    live = j[None, :] < (off[1:] - off[:-1])[:, None]                      # [B, N]
    at = (off[:-1, None] + j[None, :]).clamp(max=s["total"] - 1)
    depth = s["depth"].long()[at]                                          # [B, N]
    bits = ((s["mask"][at][:, :, j // 64] >> (j % 64)) & 1).bool() & live[:, None, :]   # row, drafted token
    if c["window"]:
        bits = bits & (depth[:, None, :] > depth[:, :, None] - c["window"])
    t = torch.arange(T, device=dev)
    seen = t[None, None, :] < ctx[:, None, None]
    if c["window"]:
        seen = seen & (t[None, None, :] > ctx[:, None, None] + depth[:, :, None] - c["window"])
    drafted = t[None, :] - ctx[:, None]                                    # [B, T]
    here = (drafted >= 0) & (drafted < N)
    seen = seen.expand(B, N, T) | (here[:, None, :] & torch.gather(bits, 2, drafted.clamp(0, N - 1)[:, None, :].expand(B, N, T)))
    q = s["qkv"][:, :c["n_q"] * D].reshape(-1, G, g, D)[at].float()        # [B, N, G, g, D]
    q = q.permute(0, 2, 1, 3, 4).reshape(B, G, N * g, D)
    sc = torch.matmul(q, K.transpose(2, 3)).reshape(B, G, N, g, T) / math.sqrt(D)
    sc = sc.masked_fill(~seen[:, None, :, None, :], -math.inf)
    top = sc.amax(dim=4, keepdim=True)
    p = torch.exp(sc - torch.where(torch.isinf(top), 0.0, top))
    den = p.sum(dim=4, keepdim=True)
    o = torch.matmul(p.reshape(B, G, N * g, T), V).reshape(B, G, N, g, D) / torch.where(den == 0, 1.0, den)
    o = o.permute(0, 2, 1, 3, 4).reshape(B, N, c["n_q"] * D)
    return o[live].to(torch.bfloat16)


def _plain_accept(s):
    c = s["case"]
    L, P = s["pools"].shape[:2]
    G, D = c["n_kv"], c["D"]
    ctx = s["ctx"].long()
    k = torch.arange(s["idx"].shape[1], device=ctx.device)
    kept = k[None, :] < s["n"][:, None]
    to = ctx[:, None] + k
    at = torch.where(kept, ctx[:, None] + s["idx"], ctx[:, None])
    to = torch.where(kept, to, ctx[:, None])[kept]
    at = at[kept]
    b = torch.arange(len(ctx), device=ctx.device)[:, None].expand_as(kept)[kept]
    page = lambda pos: s["table"][b, pos // PAGE].long()  # noqa: E731
    K, V = s["pools"][:, :, 0].view(L, P, G, PAGE, D), s["pools"][:, :, 1].view(L, P, G, D, PAGE)
    pa, pt = page(at), page(to)
    k_new, v_new = K[:, pa, :, at % PAGE].clone(), V[:, pa, :, :, at % PAGE].clone()
    K[:, pt, :, to % PAGE] = k_new
    V[:, pt, :, :, to % PAGE] = v_new
    return {"pools": s["pools"], "ctx": (s["ctx"] + s["n"])}


def _plain_copy(s):
    src, dst = s["pairs"][:, 0].long(), s["pairs"][:, 1].long()
    s["pools"][:, dst] = s["pools"][:, src]
    return s["pools"]


# ---------------------------------------------------------------- one pass

def _own_run(s):
    from paper_2609_14237_amd import runtime as R
    c = s["case"]
    if c["op"] == "rope":
        return R.rope(s["rope"], s["x"], s["pos"], out=s["y"])
    if c["op"] == "tree":
        R.run_draft(s["block"], 4, 5, s["batch"], s["draft"], s["state"])
        return s["state"].view("o", s["total"], c["n_q"] * c["D"])
    if c["op"] == "accept":
        R.kv_accept(s["block"], s["batch"], s["draft"], s["idx"], s["n"], ctx_out=s["ctx_out"])
        return {"pools": s["pools"], "ctx": s["ctx_out"]}
    R.kv_copy_pages(s["block"], s["pairs"])
    return s["pools"]


def run(state):
    if own:
        return _own_run(state)
    return {"rope": _plain_rope, "tree": _plain_tree, "accept": _plain_accept, "copy": _plain_copy}[state["case"]["op"]](state)


# ---------------------------------------------------------------- the definition in 64 bits

def exact(case, seed):
    """Rotary positions as products of complex numbers; attention sequence by sequence. Copies compute nothing."""
    if case["op"] not in ("rope", "tree"):
        return None
    s = prepare(case, seed)
    c = case
    if c["op"] == "rope":
        f = []
        for i in range(c["rdim"] // 2):
            inv = c["theta"] ** (-2.0 * i / c["rdim"])
            turns = c["orig"] * inv / (2 * math.pi)
            if c["scaling"] == "linear":
                inv /= c["factor"]
            elif c["scaling"] == "base" and c["rdim"] > 2:
                inv *= c["factor"] ** (-2.0 * i / (c["rdim"] - 2))
            elif c["scaling"] == "rotations":
                keep = min(1.0, max(0.0, (turns - 1.0) / 3.0))
                inv = inv / c["factor"] + keep * (inv - inv / c["factor"])
            elif c["scaling"] == "index":
                pair = [c["rdim"] / 2 * math.log(c["orig"] / (2 * math.pi * n)) / math.log(c["theta"]) for n in (32, 1)]
                lo, hi = max(0, math.floor(pair[0])), min(c["rdim"] - 1, math.ceil(pair[1]))
                w = min(1.0, max(0.0, (i - lo) / max(hi - lo, 0.001)))
                inv = inv * (1 - w + w / c["factor"])
            f.append(inv)
        ang = s["pos"].double()[:, None, None] * torch.tensor(f, dtype=torch.float64, device="cuda")
        turn = torch.polar(torch.full_like(ang, c["amp"]), ang)
        x, y = s["x"].double(), s["x"].double()
        r = c["rdim"]
        if c["layout"] == "half":
            z = torch.complex(x[..., :r // 2], x[..., r // 2:r]) * turn
            y = torch.cat([z.real, z.imag, x[..., r:]], dim=-1)
        else:
            z = torch.complex(x[..., 0:r:2], x[..., 1:r:2]) * turn
            y = torch.cat([torch.view_as_real(z).flatten(-2), x[..., r:]], dim=-1)
        return y
    off, ctxs = s["off"].tolist(), s["ctx"].tolist()
    G, D, g = c["n_kv"], c["D"], c["n_q"] // c["n_kv"]
    out = torch.zeros(s["total"], c["n_q"] * D, dtype=torch.float64, device="cuda")
    words = s["mask"].cpu().numpy().view(np.uint64)
    depths = s["depth"].cpu().numpy()
    for b, ctx in enumerate(ctxs):
        a, e = off[b], off[b + 1]
        n = e - a
        pages = s["table"][b, :-(-(ctx + n) // PAGE)].long()
        blk = s["pool"][pages].double().view(len(pages), 2, G, PAGE * D)
        K = blk[:, 0].reshape(-1, G, PAGE, D).transpose(1, 2).reshape(-1, G, D)[:ctx + n]
        V = blk[:, 1].reshape(-1, G, D, PAGE).permute(0, 3, 1, 2).reshape(-1, G, D)[:ctx + n]
        pos = np.concatenate([np.arange(ctx), ctx + depths[a:e]])
        see = np.zeros((n, ctx + n), bool)
        see[:, :ctx] = True
        for i in range(n):
            see[:, ctx + i] = (words[a:e, i // 64] >> np.uint64(i % 64)) & np.uint64(1)
        if c["window"]:
            see &= pos[None, :] > ctx + depths[a:e, None] - c["window"]
        bias = torch.from_numpy(np.where(see, 0.0, -np.inf)).cuda().repeat_interleave(g, dim=0)
        for h in range(G):
            q = s["qkv"][a:e, h * g * D:(h + 1) * g * D].double().reshape(n * g, D)
            p = torch.softmax(q @ K[:, h].T / math.sqrt(D) + bias, dim=1).nan_to_num(0.0)
            out[a:e, h * g * D:(h + 1) * g * D] = (p @ V[:, h]).reshape(n, g * D)
    return out
