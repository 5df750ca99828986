"""Operators of a serving step on drafted and forked sequences, as timed and compared cases.

Three kinds of operator, each with its plain form (elementary torch operations
in 32 bits, sums over a vocabulary in 64, rounded once at the end) and the
package's own call:

  heads   the q and k heads of qkv rows, each head normalised (root mean square
          and a gain) and turned to its row's position in the same pass; a
          position has one axis, or several (time, height, width)
  shared  attention of drafted rows (a single new token included) of sequences
          in groups that share the pages of a long prefix, over the paged cache
  verify  drafted tokens tested against the target's probabilities with given
          random numbers: the accepted path of each tree and the token after it

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

def _heads(rows, n_q, n_k, D, pos_hi, **kw):
    """x is the first n_q + n_k heads of rows of n_q + n_k + extra heads. sections: pairs of each axis ("": one axis),
    dealt in blocks or cyclically; own_freqs: every axis starts its own series of frequencies."""
    return dict(op="heads", rows=rows, n_q=n_q, n_k=n_k, extra=kw.pop("extra", 0), D=D, rdim=kw.pop("rdim", D),
                layout=kw.pop("layout", "half"), sections=kw.pop("sections", ""), order=kw.pop("order", "blocks"),
                own_freqs=kw.pop("own_freqs", False), norm=kw.pop("norm", True), theta=kw.pop("theta", 10000.0),
                pos_hi=pos_hi, **kw)


def _shared(batch, groups, prefix_lo, prefix_hi, tail_lo, tail_hi, rows_lo, rows_hi, n_q, n_kv, D, **kw):
    return dict(op="shared", batch=batch, groups=groups, prefix_lo=prefix_lo, prefix_hi=prefix_hi, tail_lo=tail_lo,
                tail_hi=tail_hi, rows_lo=rows_lo, rows_hi=rows_hi, n_q=n_q, n_kv=n_kv, D=D, **kw)


def _verify(batch, rows_lo, rows_hi, vocab, shape, proposal, **kw):
    """shape "chain" or "tree"; proposal: the draft's probabilities are given (else its tokens are plain guesses)."""
    return dict(op="verify", batch=batch, rows_lo=rows_lo, rows_hi=rows_hi, vocab=vocab, pad=kw.pop("pad", 0), shape=shape,
                proposal=proposal, dtype=kw.pop("dtype", "float32"), **kw)


def listed():
    return [
        # The tiny layer's decode step with normalised heads: all latency.
        _heads(4, 4, 2, 64, 128, extra=2, name="heads_tiny"),
        # A prompt's worth of rows on the 8B-shaped layer.
        _heads(8192, 32, 8, 128, 32768, extra=8, theta=500000.0, name="heads_8192"),
        # Rows of a prompt with images: three axes, half of each head turned, an odd number of rows.
        _heads(4097, 32, 4, 128, 2048, extra=4, rdim=64, sections="8,12,12", order="cyclic", theta=1000000.0,
               name="heads_4097_axes"),
        # Four continuations of one short prompt on the tiny layer.
        _shared(4, 1, 96, 96, 32, 32, 1, 1, 4, 2, 64, name="shared_tiny"),
        # Eight samples of one prompt, one token each per step.
        _shared(8, 1, 2000, 2000, 50, 500, 1, 1, 32, 8, 128, name="shared_b8"),
        # Ordinary load: users of seven system prompts of different lengths, ragged trees of up to 8 drafted tokens.
        _shared(64, 7, 500, 6000, 100, 2000, 1, 8, 32, 8, 128, name="shared_b64_ragged"),
        # One long document, 64 questions about it, a token of each.
        _shared(64, 1, 8192, 8192, 64, 512, 1, 1, 32, 8, 128, name="shared_b64_decode"),
        # High load: 128 sequences over one 32768-token prefix, four drafted tokens each, MoE layer's heads.
        _shared(128, 1, 32768, 32768, 256, 1024, 4, 4, 32, 4, 128, name="shared_b128_long"),
        # One interactive request, a chain of 7 drafted tokens behind the last one.
        _verify(1, 8, 8, 32000, "chain", True, name="verify_b1"),
        # A batch of chains with a large vocabulary.
        _verify(64, 8, 8, 128000, "chain", True, name="verify_b64_chain"),
        # Trees of guesses (no probabilities of the draft), ragged.
        _verify(64, 4, 16, 128000, "tree", False, name="verify_b64_tree"),
        # Trees whose siblings were drawn from the draft's probabilities; odd vocabulary.
        _verify(200, 2, 10, 50257, "tree", True, pad=47, name="verify_b200_drawn"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _fits(c):
    """Within the listed cases' cost: the plain form's gathered keys and scores, the tables, the work."""
    w = work(c)
    if c["op"] == "shared":
        B, rows, tail = c["batch"], c["batch"] * c["rows_hi"], c["tail_hi"] + c["rows_hi"] + PAGE
        pages = c["groups"] * c["prefix_hi"] + B * tail
        if pages * c["n_kv"] * c["D"] > 5e8 or B * tail * c["n_kv"] * c["D"] > 3e8:
            return False
        if rows * c["n_q"] * (c["prefix_hi"] + tail) > 6e8:
            return False
    if c["op"] == "verify" and c["batch"] * c["rows_hi"] * (c["vocab"] + c["pad"]) > 1.35e8:
        return False
    return w["bytes"] <= 8.5e8 and w["flops"] <= 2.9e11


def draw(rng):
    while True:
        op = rng.choice(["heads", "shared", "shared", "verify"])
        if op == "heads":
            D = rng.choice([64, 64, 80, 96, 128, 128, 256])
            rdim = rng.choice([D, D, D // 2, 2 * rng.randint(2, D // 2)])
            sections = ""
            if rng.random() < 0.5:
                n = rng.choice([2, 3])
                cuts = sorted(rng.randint(0, rdim // 2) for _ in range(n - 1))
                sections = ",".join(str(b - a) for a, b in zip([0] + cuts, cuts + [rdim // 2]))
            n_q = rng.randint(1, 32)
            c = _heads(_log_int(rng, 1, 8192), n_q, rng.choice([0, 1, 2, 4, 8]), D, _log_int(rng, 16, 1 << 20),
                       extra=rng.choice([0, 1, 8]), rdim=rdim, layout=rng.choice(["half", "half", "interleaved"]),
                       sections=sections, order=rng.choice(["blocks", "cyclic"]), own_freqs=rng.random() < 0.3,
                       norm=rng.random() < 0.8, theta=rng.choice([10000.0, 500000.0, 1000000.0]))
        elif op == "shared":
            B = _log_int(rng, 1, 256)
            hi, tail, rows = _log_int(rng, 16, 32768), _log_int(rng, 1, 4096), _log_int(rng, 1, 16)
            n_kv = rng.choice([1, 2, 4, 8])
            c = _shared(B, _log_int(rng, 1, max(1, min(B, 12))), max(1, int(hi * rng.uniform(0.1, 1.0))), hi,
                        max(1, int(tail * rng.uniform(0.1, 1.0))), tail, max(1, int(rows * rng.uniform(0.1, 1.0))), rows,
                        n_kv * rng.choice([1, 2, 4, 8] if n_kv < 8 else [1, 4]), n_kv, rng.choice([64, 128]))
        else:
            rows = _log_int(rng, 1, 32)
            c = _verify(_log_int(rng, 1, 256), max(1, int(rows * rng.uniform(0.2, 1.0))), rows,
                        _log_int(rng, 500, 160000), rng.choice(["chain", "tree"]), rng.random() < 0.6,
                        pad=rng.choice([0, 0, 1, 63]), dtype=rng.choice(["float32", "float32", "bfloat16"]))
        if _fits(c):
            return c


# ---------------------------------------------------------------- sizes and work, from the case alone

def _rows_of(c):
    """Drafted rows of each sequence; the first has the most."""
    rows = np.random.default_rng(17).integers(c["rows_lo"], c["rows_hi"] + 1, c["batch"]).astype(np.int64)
    rows[0] = c["rows_hi"]
    return rows


def _groups_of(c):
    """Bounds of the groups, each group's shared tokens, each sequence's cached tokens."""
    r = np.random.default_rng(19)
    B, n = c["batch"], c["groups"]
    cuts = np.sort(r.permutation(np.arange(1, B))[:n - 1])
    bounds = np.concatenate([[0], cuts, [B]]).astype(np.int64)
    prefix = r.integers(c["prefix_lo"], c["prefix_hi"] + 1, n).astype(np.int64)
    prefix[0] = c["prefix_hi"]
    tail = r.integers(c["tail_lo"], c["tail_hi"] + 1, B).astype(np.int64)
    return bounds, prefix, np.repeat(prefix, np.diff(bounds)) + tail


def work(case):
    c = case
    if c["op"] == "heads":
        n = c["rows"] * (c["n_q"] + c["n_k"]) * c["D"]
        axes = len(c["sections"].split(","))
        return {"bytes": 4 * n + 4 * c["rows"] * axes, "flops": (4 * n if c["norm"] else 0) + 3 * n * c["rdim"] // c["D"]}
    if c["op"] == "shared":
        bounds, prefix, ctx = _groups_of(c)
        rows = _rows_of(c)
        whole = prefix // PAGE * PAGE  # what lies on shared pages
        tokens = float(whole.sum() + (ctx - np.repeat(whole, np.diff(bounds))).sum())
        R = float(rows.sum())
        return {"bytes": (tokens + R) * c["n_kv"] * c["D"] * 4 + 2 * R * c["n_q"] * c["D"] * 2,
                "flops": 4 * float((rows * (ctx + rows / 2)).sum()) * c["n_q"] * c["D"]}
    size = 4 if c["dtype"] == "float32" else 2
    return {"bytes": c["batch"] * c["vocab"] * size * (2 if c["proposal"] else 1) + 12 * int(_rows_of(c).sum()),
            "flops": c["batch"] * c["vocab"] * 3}


# ---------------------------------------------------------------- inputs

def _g(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(shape, g):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(torch.bfloat16)


def _cuda(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def _trees(rows, n, spread, r):
    """Trees of rows[b] <= n tokens: token 0 is the last one kept, each other's parent one of the `spread` before it.
    Parents [B, n] (-1 for token 0), depths [B, n], ancestor masks [B, n, words] with each token's own bit."""
    B, words = len(rows), -(-n // 64)
    parent, depth = np.full((B, n), -1, np.int32), np.zeros((B, n), np.int32)
    mask = np.zeros((B, n, words), np.uint64)
    at = np.arange(B)
    for j in range(n):
        if j:
            p = np.maximum(j - 1 - r.integers(0, spread, B), 0)
            parent[:, j], depth[:, j], mask[:, j] = p, depth[at, p] + 1, mask[at, p]
        mask[:, j, j // 64] |= np.uint64(1) << np.uint64(j % 64)
    return parent, depth, mask


def _axis_of(c):
    """Axis of each rotated pair, and its place among that axis's pairs."""
    left = [int(n) for n in c["sections"].split(",")] if c["sections"] else [c["rdim"] // 2]
    axis, place, used, a = [], [], [0] * len(left), 0
    for _ in range(c["rdim"] // 2):
        while used[a] == left[a]:
            a = (a + 1) % len(left)
        axis.append(a)
        place.append(used[a])
        used[a] += 1
        if c["order"] == "cyclic":
            a = (a + 1) % len(left)
    return np.array(axis, np.int64), np.array(place, np.float64), left


def _freqs(c):
    """Angle per position of each rotated pair, float64 [rdim / 2]."""
    axis, place, sizes = _axis_of(c)
    if c["own_freqs"] and c["sections"]:
        return c["theta"] ** (-place / np.array(sizes, np.float64)[axis])
    return c["theta"] ** (-2.0 * np.arange(c["rdim"] // 2) / c["rdim"])


def _prepare_heads(s, g, r):
    c, D = s["case"], s["case"]["D"]
    heads = c["n_q"] + c["n_k"]
    rows = _normal((c["rows"], heads + c["extra"], D), g)
    s["x"] = rows[:, :heads]
    s["y"] = torch.empty((c["rows"], heads, D), dtype=torch.bfloat16, device="cuda")
    s["gain_q"], s["gain_k"] = ((1 + 0.2 * torch.randn(D, generator=g, device="cuda")).to(torch.bfloat16) for _ in range(2))
    axis, _, sizes = _axis_of(c)
    shape = (c["rows"], len(sizes)) if c["sections"] else c["rows"]
    s["pos"] = _cuda(r.integers(0, c["pos_hi"], shape).astype(np.int32))
    s["axis"], s["freqs"] = _cuda(axis), _cuda(_freqs(c))


def _prepare_shared(s, g, r):
    c = s["case"]
    rows, n = _rows_of(c), c["rows_hi"]
    bounds, prefix, ctx = _groups_of(c)
    _, depth, mask = _trees(rows, n, 4, r)
    common, need = prefix // PAGE, -(-(ctx + rows) // PAGE)
    group = np.repeat(np.arange(len(prefix)), np.diff(bounds))
    P = int(common.sum() + (need - common[group]).sum()) + 8
    ids = r.permutation(P).astype(np.int32)
    table, off = np.full((c["batch"], int(need.max())), -1, np.int32), 0
    for i, k in enumerate(common):
        table[bounds[i]:bounds[i + 1], :k] = ids[off:off + k]
        off += k
    for b, k in enumerate(need):
        first = common[group[b]]
        table[b, first:k] = ids[off:off + k - first]
        off += k - first
    live = np.arange(n)[None, :] < rows[:, None]
    at = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
    s["ctx"], s["table"], s["off"] = _cuda(ctx.astype(np.int32)), _cuda(table), _cuda(at)
    s["depth"], s["mask"] = _cuda(depth[live]), _cuda(mask[live].view(np.int64))
    s["bounds"], s["prefix"] = _cuda(bounds.astype(np.int32)), _cuda((common * PAGE).astype(np.int32))
    s["total"], s["group"] = int(at[-1]), _cuda(group)
    s["split"] = [(int(bounds[i]), int(bounds[i + 1]), int(at[bounds[i]]), int(at[bounds[i + 1]]), int(k) * PAGE)
                  for i, k in enumerate(common)]  # a group's sequences, rows and tokens, as a scheduler knows them
    s["tail"] = int((ctx + rows - common[group] * PAGE).max())
    s["pool"] = _normal((P, 2, c["n_kv"], PAGE * c["D"]), g)
    s["qkv"] = _normal((s["total"], (c["n_q"] + 2 * c["n_kv"]) * c["D"]), g)


def _prepare_verify(s, g, r):
    """Target and draft that mostly agree: logits of one source, the draft's blurred. Tokens are drawn from the draft's
    probabilities after their parent, or, as guesses, the likeliest of them in turn."""
    c = s["case"]
    rows, n, V = _rows_of(c), c["rows_hi"], c["vocab"]
    parent, _, mask = _trees(rows, n, 1 if c["shape"] == "chain" else 3, r)
    live = np.arange(n)[None, :] < rows[:, None]
    at = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
    R = int(at[-1])
    row_parent = parent[live]
    above = np.maximum(np.repeat(at[:-1], rows) + row_parent, 0)  # row of the parent
    nth = np.zeros(R, np.int64)                                   # place among its siblings
    seen = {}
    for i, (a, p) in enumerate(zip(above.tolist(), row_parent.tolist())):
        if p >= 0:
            nth[i] = seen.get(a, 0)
            seen[a] = nth[i] + 1
    dt = getattr(torch, c["dtype"])
    target = torch.zeros((R, V + c["pad"]), dtype=dt, device="cuda")
    proposal = torch.zeros_like(target) if c["proposal"] else None
    tokens = torch.zeros(R, dtype=torch.int32, device="cuda")
    drawn = torch.empty((R, int(nth.max()) + 1), dtype=torch.int64, device="cuda")  # a row's children in turn
    for a in range(0, R, 128):
        b = min(a + 128, R)
        logits = 2.5 * torch.randn((b - a, V), generator=g, device="cuda")
        target[a:b, :V] = torch.softmax(logits, 1).to(dt)
        blurred = torch.softmax(0.9 * logits + 0.5 * torch.randn((b - a, V), generator=g, device="cuda"), 1).to(dt)
        if c["proposal"]:
            proposal[a:b, :V] = blurred
            for k in range(drawn.shape[1]):
                race = torch.empty((b - a, V), device="cuda").exponential_(generator=g)
                drawn[a:b, k] = (blurred.float() / race).argmax(1)
        else:
            drawn[a:b] = blurred.float().topk(min(drawn.shape[1], V), dim=1).indices
    up = torch.from_numpy(above).cuda()
    tokens.copy_(drawn[up, torch.from_numpy(nth).cuda()].to(torch.int32))
    s["target"], s["proposal"], s["tokens"] = target, proposal, tokens
    s["off"], s["parent"], s["total"] = _cuda(at), _cuda(row_parent), R
    s["depth"], s["mask"] = torch.zeros(R, dtype=torch.int32, device="cuda"), _cuda(mask[live].view(np.int64))
    s["u"] = torch.rand(R, generator=g, device="cuda")
    s["u_next"] = torch.rand(c["batch"], generator=g, device="cuda")


def prepare(case, seed):
    s = {"case": case}
    {"heads": _prepare_heads, "shared": _prepare_shared, "verify": _prepare_verify}[case["op"]](s, _g(seed), np.random.default_rng(seed))
    if own:
        _handles(s)
    return s


class _Cfg:
    """One layer's shape, as the package's DeviceBlock reads it."""

    def __init__(self, n_q, n_kv, D):
        self.hidden, self.ffn, self.n_experts, self.top_k, self.moe_ffn = 256, 256, 0, 0, 0
        self.n_q, self.n_kv, self.head_dim, self.window = n_q, n_kv, D, 0
        self.rope_theta, self.rms_eps = 10000.0, 1e-6


def _handles(s):
    """The objects a serving program keeps across steps: the rotary table, the block, the batch, the live buffers."""
    from paper_2609_14237_amd import runtime as R
    c = s["case"]
    if c["op"] == "heads":
        sections = tuple(int(n) for n in c["sections"].split(",")) if c["sections"] else None
        s["rope"] = R.Rope(c["D"], theta=c["theta"], rotary_dim=c["rdim"], interleaved=c["layout"] == "interleaved",
                           sections=sections, order=c["order"], own_freqs=c["own_freqs"])
        s["norm"] = R.HeadNorm(s["gain_q"], s["gain_k"], n_q=c["n_q"], eps=1e-6) if c["norm"] else None
    elif c["op"] == "shared":
        s["block"] = R.DeviceBlock([_Cfg(c["n_q"], c["n_kv"], c["D"])], [{}], [s["pool"]], s["pool"].shape[0])
        s["batch"] = R.DeviceBatch(s["ctx"], s["table"])
        s["draft"] = R.DeviceDraft(s["off"], s["depth"], s["mask"], max_rows=c["rows_hi"],
                                   shared=R.SharedPrefix(s["bounds"], s["prefix"]))
        s["state"] = R.DeviceState(s["block"], s["batch"], draft=s["draft"])
        s["state"].view("qkv", *s["qkv"].shape).copy_(s["qkv"])
    else:
        s["draft"] = R.DeviceDraft(s["off"], s["depth"], s["mask"], max_rows=c["rows_hi"])
        s["verifier"] = R.DraftVerifier(c["batch"], c["rows_hi"], c["vocab"])


# ---------------------------------------------------------------- plain forms

def _plain_heads(s):
    c, x = s["case"], s["x"].float()
    r, n_q = c["rdim"], c["n_q"]
    if c["norm"]:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6)
        x = torch.cat([x[:, :n_q] * s["gain_q"].float(), x[:, n_q:] * s["gain_k"].float()], dim=1)
    pos = s["pos"].double()
    pos = pos[:, s["axis"]] if c["sections"] else pos[:, None]
    ang = torch.remainder(pos * s["freqs"], 2 * math.pi).float()
    cos, sin = torch.cos(ang)[:, None, :], torch.sin(ang)[:, None, :]
    y = x.clone()
    if c["layout"] == "half":
        a, b = x[..., :r // 2], x[..., r // 2:r]
        y[..., :r // 2], y[..., r // 2:r] = a * cos - b * sin, b * cos + a * sin
    else:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        y[..., 0:r:2], y[..., 1:r:2] = a * cos - b * sin, b * cos + a * sin
    return y.to(torch.bfloat16)


def _kv(s, pages):
    """Keys and values [..., G, tokens, D] in 32 bits of page ids [..., n]."""
    c = s["case"]
    G, D, lead, n = c["n_kv"], c["D"], pages.shape[:-1], pages.shape[-1]
    kv = s["pool"][pages]                                                        # [..., n, 2, G, 16 D]
    K = kv[..., 0, :, :].reshape(*lead, n, G, PAGE, D).transpose(-4, -3).reshape(*lead, G, n * PAGE, D).float()
    V = kv[..., 1, :, :].reshape(*lead, n, G, D, PAGE).transpose(-4, -3).transpose(-2, -1).reshape(*lead, G, n * PAGE, D).float()
    return K, V


def _partial(q, K, V, seen):
    """Maximum, denominator and sums of softmax(q K^T) V over the seen tokens (None: all of them)."""
    sc = torch.matmul(q, K.transpose(-2, -1)) / math.sqrt(q.shape[-1])
    if seen is not None:
        sc = sc.masked_fill(~seen, -math.inf)
    top = sc.amax(dim=-1, keepdim=True)
    p = torch.exp(sc - torch.where(torch.isinf(top), 0.0, top))
    return top, p.sum(dim=-1, keepdim=True), torch.matmul(p, V)


def _plain_shared(s):
    """Each group's prefix once for all its rows, the tails of all sequences at once, the two joined."""
    c = s["case"]
    B, N, G, D, g = c["batch"], c["rows_hi"], c["n_kv"], c["D"], c["n_q"] // c["n_kv"]
    dev = s["ctx"].device
    off, ctx = s["off"].long(), s["ctx"].long()
    q = s["qkv"][:, :c["n_q"] * D].reshape(-1, G, g, D).float()                  # [rows, G, g, D]
    top = torch.full((s["total"], G, g, 1), -math.inf, device=dev)
    den, acc = torch.zeros_like(top), torch.zeros((s["total"], G, g, D), device=dev)
    for b0, _, r0, r1, tokens in s["split"]:
        if tokens == 0:
            continue
        K, V = _kv(s, s["table"][b0, :tokens // PAGE].long())
        part = _partial(q[r0:r1].transpose(0, 1).reshape(G, (r1 - r0) * g, D), K, V, None)
        for whole, x in zip((top, den, acc), part):
            whole[r0:r1] = x.reshape(G, r1 - r0, g, -1).transpose(0, 1)
    first = s["prefix"].long()[s["group"]]                                       # [B]
    n_pages = -(-s["tail"] // PAGE)
    lp = first[:, None] // PAGE + torch.arange(n_pages, device=dev)
    K, V = _kv(s, torch.gather(s["table"], 1, lp.clamp(max=s["table"].shape[1] - 1)).long().clamp(min=0))
    T = n_pages * PAGE
    t = first[:, None] + torch.arange(T, device=dev)                             # [B, T]
    j = torch.arange(N, device=dev)
    live = j[None, :] < (off[1:] - off[:-1])[:, None]                            # [B, N]
    at = (off[:-1, None] + j[None, :]).clamp(max=s["total"] - 1)
    bits = ((s["mask"][at][:, :, j // 64] >> (j % 64)) & 1).bool() & live[:, None, :]
    drafted = t - ctx[:, None]
    here = (drafted >= 0) & (drafted < N)
    seen = (drafted < 0)[:, None, :].expand(B, N, T) | (
        here[:, None, :] & torch.gather(bits, 2, drafted.clamp(0, N - 1)[:, None, :].expand(B, N, T)))
    seen = seen[:, None, :, None, :].expand(B, G, N, g, T).reshape(B, G, N * g, T)
    part = _partial(q[at].permute(0, 2, 1, 3, 4).reshape(B, G, N * g, D), K, V, seen)
    top2, den2, acc2 = (x.reshape(B, G, N, g, -1).permute(0, 2, 1, 3, 4)[live] for x in part)
    most = torch.maximum(top, top2)
    a, b = torch.exp(top - most), torch.exp(top2 - most)
    return ((acc * a + acc2 * b) / (den * a + den2 * b)).reshape(s["total"], c["n_q"] * D).to(torch.bfloat16)


def _plain_verify(s):
    """All sequences at once, token by token. W: what is left of the target's probabilities at a sequence's present token
    (not normalised), Z its sum as tests see it."""
    c = s["case"]
    B, N, V = c["batch"], c["rows_hi"], c["vocab"]
    off = s["off"].long()
    r0, rows = off[:-1], off[1:] - off[:-1]
    dev, each = off.device, torch.arange(B, device=off.device)
    positive = lambda x: torch.where((x > 0) & (x < math.inf), x, 0.0)  # noqa: E731
    W = positive(s["target"][r0, :V].double())
    Z = torch.ones(B, dtype=torch.float64, device=dev)
    cur = torch.zeros(B, dtype=torch.int64, device=dev)
    path = torch.full((B, N), -1, dtype=torch.int32, device=dev)
    path[:, 0] = 0
    n = torch.ones(B, dtype=torch.int64, device=dev)
    for j in range(1, N):
        row = (r0 + j).clamp(max=s["total"] - 1)
        tested = (j < rows) & (s["parent"][row] == cur)
        x = s["tokens"][row].long()
        w = W[each, x]
        left = Z * s["u"][row].double()
        if c["proposal"]:
            Q = positive(s["proposal"][r0 + cur, :V].double())
            left = left * Q[each, x]
            rest = (W - Z[:, None] * Q).clamp(min=0.0)
            rest_sum = rest.sum(1)
        else:
            rest = W.clone()
            rest[each, x] = 0.0
            rest_sum = Z - w
        kept = tested & (w > 0) & (left < w)
        lost = tested & ~kept
        cur = torch.where(kept, j, cur)
        path[each, torch.where(kept, n, 0)] = torch.where(kept, j, 0).to(torch.int32)
        n = n + kept
        W = torch.where(kept[:, None], positive(s["target"][r0 + cur, :V].double()), torch.where(lost[:, None], rest, W))
        Z = torch.where(kept, 1.0, torch.where(lost, rest_sum, Z))
    empty = (W > 0).sum(1) == 0
    W = torch.where(empty[:, None], positive(s["target"][r0 + cur, :V].double()), W)
    sums = torch.cumsum(W, dim=1)
    above = sums > (s["u_next"].double() * sums[:, -1])[:, None]
    index = torch.arange(V, device=dev)
    last = torch.where(W > 0, index, -1).amax(1)
    first = torch.where(above & (W > 0), index, V).amin(1)
    nxt = torch.where(first < V, first, last)
    return {"path": path, "path_len": n.to(torch.int32), "next": nxt.to(torch.int32)}


# ---------------------------------------------------------------- one pass

def _own_run(s):
    from paper_2609_14237_amd import runtime as R
    c = s["case"]
    if c["op"] == "heads":
        return R.rope(s["rope"], s["x"], s["pos"], out=s["y"], norm=s["norm"])
    if c["op"] == "shared":
        R.run_draft(s["block"], 4, 5, s["batch"], s["draft"], s["state"])
        return s["state"].view("o", s["total"], c["n_q"] * c["D"])
    v = s["verifier"]
    v.run(s["draft"], s["tokens"], s["parent"], s["target"][:, :c["vocab"]], s["u"], s["u_next"],
          proposal=None if s["proposal"] is None else s["proposal"][:, :c["vocab"]])
    return {"path": v.path, "path_len": v.path_len, "next": v.next}


def run(state):
    if own:
        return _own_run(state)
    return {"heads": _plain_heads, "shared": _plain_shared, "verify": _plain_verify}[state["case"]["op"]](state)


# ---------------------------------------------------------------- the definition in 64 bits

def exact(case, seed):
    """Heads as vectors of length sqrt(D) turned by complex numbers; attention sequence by sequence over its own table.
    What verify returns are whole numbers."""
    if case["op"] == "verify":
        return None
    s, c = prepare(case, seed), case
    if c["op"] == "heads":
        x, r = s["x"].double(), c["rdim"]
        if c["norm"]:
            x = x / torch.sqrt(torch.linalg.vector_norm(x, dim=-1, keepdim=True) ** 2 / c["D"] + 1e-6)
            gains = torch.stack([s["gain_q"]] * c["n_q"] + [s["gain_k"]] * c["n_k"]).double()
            x = x * gains
        axis, place, sizes = _axis_of(c)
        f = [c["theta"] ** (-(place[i] / sizes[axis[i]] if c["own_freqs"] and c["sections"] else 2.0 * i / r))
             for i in range(r // 2)]
        pos = s["pos"].double().reshape(c["rows"], -1)[:, axis]
        ang = (pos * torch.tensor(f, dtype=torch.float64, device="cuda"))[:, None, :]
        turn = torch.polar(torch.ones_like(ang), ang)
        if c["layout"] == "half":
            z = torch.complex(x[..., :r // 2], x[..., r // 2:r]) * turn
            return torch.cat([z.real, z.imag, x[..., r:]], dim=-1)
        z = torch.complex(x[..., 0:r:2], x[..., 1:r:2]) * turn
        return torch.cat([torch.view_as_real(z).flatten(-2), x[..., r:]], dim=-1)
    off, ctxs = s["off"].tolist(), s["ctx"].tolist()
    G, D, g = c["n_kv"], c["D"], c["n_q"] // c["n_kv"]
    out = torch.zeros(s["total"], c["n_q"] * D, dtype=torch.float64, device="cuda")
    words = s["mask"].cpu().numpy().view(np.uint64)
    for b, ctx in enumerate(ctxs):
        a, e = off[b], off[b + 1]
        n = e - a
        blk = s["pool"][s["table"][b, :-(-(ctx + n) // PAGE)].long()].double().view(-1, 2, G, PAGE * D)
        K = blk[:, 0].reshape(-1, G, PAGE, D).transpose(1, 2).reshape(-1, G, D)[:ctx + n]
        V = blk[:, 1].reshape(-1, G, D, PAGE).permute(0, 3, 1, 2).reshape(-1, G, D)[:ctx + n]
        see = np.ones((n, ctx + n), bool)
        for i in range(n):
            see[:, ctx + i] = (words[a:e, i // 64] >> np.uint64(i % 64)) & np.uint64(1)
        bias = torch.from_numpy(np.where(see, 0.0, -np.inf)).cuda().repeat_interleave(g, dim=0)
        for h in range(G):
            q = s["qkv"][a:e, h * g * D:(h + 1) * g * D].double().reshape(n * g, D)
            p = torch.softmax(q @ K[:, h].T / math.sqrt(D) + bias, dim=1)
            out[a:e, h * g * D:(h + 1) * g * D] = (p @ V[:, h]).reshape(n, g * D)
    return out
