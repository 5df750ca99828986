"""PyTorch-side marshalling around the C ABI: packs device tensors into the
ods_* structs and allocates the live buffers and workspace the library sizes.
No operator of the decode step is computed here."""
from __future__ import annotations

import ctypes as C

import numpy as np
import torch

from . import binding as _b
from .binding import (ods_batch, ods_block, ods_draft, ods_head_norm, ods_layer, ods_layer_cfg, ods_pages, ods_rope,
                      ods_shared, ods_state, ods_verify)


def layer_cfg(cfg) -> ods_layer_cfg:
    """ods_layer_cfg from any object with the layer-shape attributes."""
    return ods_layer_cfg(cfg.hidden, cfg.n_q, cfg.n_kv, cfg.head_dim, cfg.ffn, cfg.n_experts, cfg.top_k,
                         cfg.moe_ffn, cfg.window, cfg.rope_theta, cfg.rms_eps)


def _ptr(t):
    if t is None:
        return None
    return t.data_ptr()


def _devices(*tensors) -> tuple:
    """Indices of the devices that the tensors are on (-1: the host); None and what is no tensor has none."""
    return tuple({t.get_device() for t in tensors if isinstance(t, torch.Tensor)})


def _tile_shapes(cfg):
    """(out, in, gated, groups) of each projection weight, as ods_tile_weight takes them."""
    qkv = (cfg.n_q + 2 * cfg.n_kv) * cfg.head_dim
    H, E = cfg.hidden, cfg.n_experts
    shapes = {"w_qkv": (qkv, H, 0, 1), "w_o": (H, cfg.n_q * cfg.head_dim, 0, 1)}
    if E:
        shapes.update(w_gate_up=(cfg.moe_ffn, H, 1, E), w_down=(H, cfg.moe_ffn, 0, E))
    else:
        shapes.update(w_gate_up=(cfg.ffn, H, 1, 1), w_down=(H, cfg.ffn, 0, 1))
    return shapes


def tile_weights(cfg, w: dict, stream=None) -> dict:
    """Tiled copies (ODS_WEIGHTS_TILED) of a layer's projection weights, converted
    by ods_tile_weight on the device; the other entries of w are passed through."""
    stream = stream if stream is not None else torch.cuda.current_stream()
    out = dict(w)
    for name, (o, i, gated, groups) in _tile_shapes(cfg).items():
        src = w[name]
        n = _b.ods_tiled_weight_bytes(o, i, gated, groups)
        if n == 0:
            raise ValueError(f"{name}: no tiled layout for out={o}, in={i} (in must be a multiple of 64)")
        dst = torch.empty(n // 2, dtype=torch.bfloat16, device=src.device)
        _b._check(_b.ods_tile_weight(src.data_ptr(), dst.data_ptr(), o, i, gated, groups, stream.cuda_stream),
                  f"ods_tile_weight({name})")
        out[name] = dst
    return out


class DeviceBlock:
    """ods_block over per-layer weight dicts and KV pools (tensors stay referenced).
    pool_pages is one count for every layer or a list with one per layer. With
    tiled=True the projection weights are converted once into the tiled layout
    (ODS_WEIGHTS_TILED) the weight-streaming GEMM reads fastest, and the block
    references those copies; pretiled=True takes weights tile_weights() already
    converted."""

    WEIGHTS = ("g_attn", "w_qkv", "w_o", "g_ffn", "w_gate_up", "w_down", "w_router")

    def __init__(self, cfgs, weights, pools, pool_pages, tiled: bool = False, pretiled: bool = False):
        self.cfgs = list(cfgs)
        self.tiled = tiled or pretiled
        self.weights = [tile_weights(c, w) if tiled and not pretiled else w for c, w in zip(self.cfgs, weights)]
        self.pools = list(pools)
        n = len(self.cfgs)
        pages = list(pool_pages) if isinstance(pool_pages, (list, tuple)) else [pool_pages] * n
        self._layers = (ods_layer * n)()
        for i, (cfg, w, pool) in enumerate(zip(self.cfgs, self.weights, self.pools)):
            L = self._layers[i]
            L.cfg = layer_cfg(cfg)
            for name in self.WEIGHTS:
                setattr(L, name, _ptr(w.get(name)))
            L.kv_pool = _ptr(pool)
            L.pool_pages = pages[i] if pool is not None else 0
            L.weight_layout = _b.ODS_WEIGHTS_TILED if self.tiled else _b.ODS_WEIGHTS_ROWS
        self.c = ods_block(n, C.cast(self._layers, C.POINTER(ods_layer)))
        self._pool_devices = [_devices(pool) for pool in self.pools]
        self._op_devices = [_devices(pool, *map(w.get, self.WEIGHTS)) for w, pool in zip(self.weights, self.pools)]
        self._devices = {d for on in self._op_devices for d in on}

    def pool_devices(self, layer_begin: int, layer_end: int) -> set:
        """Devices of the pools of layers [layer_begin, layer_end)."""
        if len(self._devices) <= 1:  # the whole block's
            return self._devices
        return {d for on in self._pool_devices[max(layer_begin, 0):max(layer_end, 0)] for d in on}

    def op_devices(self, op_begin: int, op_end: int) -> set:
        """Devices of the layers that operators [op_begin, op_end) belong to."""
        if len(self._devices) <= 1:
            return self._devices
        on, at = set(), 0
        for cfg, devices in zip(self.cfgs, self._op_devices):
            end = at + (14 if cfg.n_experts else 10)
            if op_begin < end and at < op_end:
                on.update(devices)
            at = end
        return on

    def num_ops(self) -> int:
        return _b.ods_block_num_ops(self.c)

    def op_name(self, op: int):
        return _b.ods_op_name(self.c, op)

    def layer_offset(self, layer: int) -> int:
        return sum(14 if c.n_experts else 10 for c in self.cfgs[:layer])


class DeviceBatch:
    """ods_batch over device int32 ctx_lens [B] and page_table [B, max_pages], and
    optionally a window-only page ring [B, ring_pages] for sliding-window layers."""

    def __init__(self, ctx_lens: torch.Tensor, page_table: torch.Tensor, split_pages: int = 0,
                 ring_table: torch.Tensor | None = None):
        assert ctx_lens.dtype == torch.int32 and page_table.dtype == torch.int32
        self.ctx_lens = ctx_lens.contiguous()
        self.page_table = page_table.contiguous()
        self.ring_table = None if ring_table is None else ring_table.contiguous()
        B, max_pages = self.page_table.shape
        ring_pages = 0
        if self.ring_table is not None:
            assert self.ring_table.dtype == torch.int32 and self.ring_table.shape[0] == B
            ring_pages = self.ring_table.shape[1]
        self.c = ods_batch(B, max_pages, _ptr(self.ctx_lens), _ptr(self.page_table), split_pages, ring_pages,
                           _ptr(self.ring_table))
        self.devices = _devices(self.ctx_lens, self.page_table, self.ring_table)

    @property
    def batch(self) -> int:
        return self.c.batch


_BUF_DTYPE = {"logits": torch.float32, "topk_w": torch.float32, "topk_ids": torch.int32,
              "perm": torch.int32, "slot_pos": torch.int32, "expert_off": torch.int32}


def _stream_of(who: str, stream: int | None, *devices: int) -> int:
    """`stream`, or the current one. What the call names is on one device: the current one, or, with a stream that the
    caller names, the device of that stream, which is not looked at."""
    if stream is None:
        device = torch.cuda.current_device()
        for d in devices:
            if d != device:
                raise ValueError(f"{who}: a tensor is on {_name(d)}, the current device is cuda:{device}")
        return torch._C._cuda_getCurrentRawStream(device)
    for d in devices:
        if d != devices[0]:
            raise ValueError(f"{who}: tensors are on {_name(devices[0])} and on {_name(d)}, a call takes one device")
    return stream


def _name(device: int) -> str:
    return "the host" if device < 0 else f"cuda:{device}"


class Rope:
    """Rotary positions with their device table of frequencies (ods_rope): theta, the rotated part of the head
    (rotary_dim, default all), pair layout, and scaling for long contexts: "plain", "linear", "base", "rotations" or
    "index" (include/ods.h has the formulas). `turns` is (turns_hi, turns_lo) of the last two, by default (4, 1) and
    (32, 1).

    Positions of several axes (time, height, width): `sections` has the pairs of each axis, rotary_dim / 2 in all, dealt
    out in `order` "blocks" (the first pairs are the first axis's) or "cyclic" (one pair each in turn, while an axis has
    some left). A pair keeps the frequency of its place in the head, or, with own_freqs, every axis has the frequencies
    of a rotary part of its own size."""

    SCALINGS = {"plain": _b.ODS_ROPE_PLAIN, "linear": _b.ODS_ROPE_LINEAR, "base": _b.ODS_ROPE_BASE,
                "rotations": _b.ODS_ROPE_ROTATIONS, "index": _b.ODS_ROPE_INDEX}

    def __init__(self, head_dim: int, theta: float = 10000.0, rotary_dim: int | None = None, interleaved: bool = False,
                 scaling: str = "plain", factor: float = 1.0, orig_ctx: float = 8192.0, turns=None,
                 amplitude: float = 1.0, device="cuda", sections=None, order: str = "blocks", own_freqs: bool = False):
        if scaling not in self.SCALINGS:
            raise ValueError(f"scaling {scaling!r}: one of {', '.join(self.SCALINGS)}")
        hi, lo = turns if turns is not None else ((32.0, 1.0) if scaling == "index" else (4.0, 1.0))
        rdim = head_dim if rotary_dim is None else rotary_dim
        self.c = ods_rope(head_dim, rdim, int(interleaved), self.SCALINGS[scaling], theta, factor, orig_ctx, hi, lo,
                          amplitude, None)
        host = np.zeros(max(rdim // 2, 1), np.float64)
        _b._check(_b.ods_rope_freqs(self.c, host), "ods_rope_freqs")
        self.axes, self.axis = 1, None
        if sections is not None:
            sections = [int(n) for n in sections]
            if order not in ("blocks", "cyclic"):
                raise ValueError(f"Rope: order {order!r}: blocks or cyclic")
            if min(sections, default=-1) < 0 or sum(sections) != rdim // 2 or len(sections) > _b.ROPE_AXES:
                raise ValueError(f"Rope: sections {sections} of {rdim // 2} pairs (at most {_b.ROPE_AXES} axes)")
            self.axes = len(sections)
            axis = _deal(sections, order)
            if own_freqs:
                part = ods_rope.from_buffer_copy(self.c)
                for a, n in enumerate(sections):
                    own = np.zeros(max(n, 1), np.float64)
                    part.rotary_dim = 2 * n
                    if n:
                        _b._check(_b.ods_rope_freqs(part, own), "ods_rope_freqs")
                        host[:rdim // 2][axis == a] = own
            self.axis = torch.from_numpy(axis).to(device)
        self.freqs = torch.from_numpy(host).to(device)
        self.c.freqs = self.freqs.data_ptr()


def _deal(sections, order: str) -> np.ndarray:
    """Axis of every pair, int32."""
    if order == "blocks":
        return np.repeat(np.arange(len(sections), dtype=np.int32), sections)
    left, axis = list(sections), []
    while any(left):
        for a, n in enumerate(left):
            if n:
                axis.append(a)
                left[a] = n - 1
    return np.array(axis, np.int32)


class HeadNorm:
    """Heads normalised before they turn (ods_head_norm): x / rms(x) * gain over a head. gain_q, gain_k: bf16 [head_dim]
    for the query heads, the first n_q of a row (default: all of them), and for the key heads behind them."""

    def __init__(self, gain_q: torch.Tensor, gain_k: torch.Tensor | None = None, n_q: int | None = None, eps: float = 1e-6):
        for name, g in (("gain_q", gain_q), ("gain_k", gain_k)):
            if g is not None and (g.dtype != torch.bfloat16 or g.dim() != 1 or g.shape != gain_q.shape):
                raise ValueError(f"HeadNorm: {name} is bf16 [head_dim], got {g.dtype} {tuple(g.shape)}")
        self.gain_q = gain_q.contiguous()
        self.gain_k = None if gain_k is None else gain_k.contiguous()
        self.n_q = n_q
        self.head_dim = gain_q.shape[0]
        self.c = ods_head_norm(_ptr(self.gain_q), _ptr(self.gain_k), eps)
        self.devices = _devices(self.gain_q, self.gain_k)


def rope(r: Rope, x: torch.Tensor, pos: torch.Tensor, out: torch.Tensor | None = None, stream: int | None = None,
         norm: HeadNorm | None = None):
    """Rotate x [rows, heads, head_dim] (bf16; the last two dims contiguous, rows at any stride of 8) to positions
    pos [rows] (int32; rows with a negative one are left alone) into out (default x, in place); returns out. With `norm`
    the heads are normalised first, in the same pass. A Rope with sections takes pos [rows, axes]."""
    y = x if out is None else out
    for t in (x, y):
        if t.dtype != torch.bfloat16 or t.dim() != 3 or t.shape[2] != r.c.head_dim:
            raise ValueError(f"rope takes bf16 [rows, heads, {r.c.head_dim}], got {t.dtype} {tuple(t.shape)}")
        if t.numel() and (t.stride(2) != 1 or (t.shape[1] > 1 and t.stride(1) != r.c.head_dim)):
            raise ValueError("rope: the heads of a row must be contiguous")
    places = x.shape[:1] if r.axis is None else (x.shape[0], r.axes)
    if x.shape != y.shape or pos.dtype != torch.int32 or pos.shape != places or not pos.is_contiguous():
        raise ValueError(f"rope: x {tuple(x.shape)}, out {tuple(y.shape)}, pos {pos.dtype} {tuple(pos.shape)}")
    rows, heads = x.shape[:2]
    width = heads * r.c.head_dim  # the stride of a single row means nothing
    xs, ys = (t.stride(0) if rows > 1 else width for t in (x, y))
    if norm is not None or r.axis is not None:
        n_q = heads if norm is None or norm.n_q is None else norm.n_q
        if norm is not None and (norm.head_dim != r.c.head_dim or not 0 <= n_q <= heads or (n_q < heads and norm.gain_k is None)):
            raise ValueError(f"rope: a norm of heads of {norm.head_dim}, {n_q} with gain_q, for {heads} of {r.c.head_dim}")
        on = (x.get_device(), y.get_device(), pos.get_device(), r.freqs.get_device(), *(norm.devices if norm is not None else ()))
        _b._check(_b.ods_head_rows(r.c, None if norm is None else norm.c, _ptr(r.axis), r.axes, x.data_ptr(), xs, y.data_ptr(),
                                   ys, rows, n_q, heads - n_q, pos.data_ptr(), _stream_of("rope", stream, *on)),
                  "ods_head_rows")
        return y
    _b._check(_b.ods_rope_rows(r.c, x.data_ptr(), xs, y.data_ptr(), ys, rows, heads, pos.data_ptr(),
                               _stream_of("rope", stream, x.get_device(), y.get_device(), pos.get_device(),
                                          r.freqs.get_device())), "ods_rope_rows")
    return y


class SharedPrefix:
    """Groups of a batch's sequences that share the pages of a prefix (ods_shared): group g is sequences
    group_off[g] .. group_off[g + 1] - 1, whose tables name the same pages for their first tokens[g] tokens. Device int32
    [groups + 1] and [groups]; KvPages.shared() finds them. Both may be rewritten between calls, as this object's `group_off`
    and `tokens` (copies of what was given, where that is not contiguous); their lengths stay."""

    def __init__(self, group_off: torch.Tensor, tokens: torch.Tensor):
        if group_off.dtype != torch.int32 or tokens.dtype != torch.int32 or tokens.dim() != 1 or group_off.shape != (len(tokens) + 1,):
            raise ValueError(f"SharedPrefix: int32 group_off [groups + 1] and tokens [groups], got {group_off.dtype} "
                             f"{tuple(group_off.shape)} and {tokens.dtype} {tuple(tokens.shape)}")
        self.group_off, self.tokens = group_off.contiguous(), tokens.contiguous()
        self.c = ods_shared(len(tokens), _ptr(self.group_off), _ptr(self.tokens))
        self.devices = _devices(self.group_off, self.tokens)


class DeviceDraft:
    """ods_draft: drafted rows of a batch. row_off [B + 1] and depth [rows] int32, mask [rows, ceil(max_rows / 64)]
    int64 (bit patterns; a 1-D tensor is one word per row). `rope`: None for the layers' own, or one Rope per layer
    (of one with sections every axis is at the row's position, as in text). `norm`: None, or one HeadNorm per layer, of
    whose gains the layer's q and k heads take one each. `shared`: None, or the prefixes that groups of the batch's
    sequences share, read once where the tables are large and the trees narrow enough for that to pay (ods_shared)."""

    def __init__(self, row_off: torch.Tensor, depth: torch.Tensor, mask: torch.Tensor, max_rows: int, rope=None, norm=None,
                 shared: SharedPrefix | None = None):
        words = (max_rows + 63) // 64
        mask = mask if mask.dim() == 2 else mask.reshape(-1, words)
        if row_off.dtype != torch.int32 or depth.dtype != torch.int32 or mask.dtype != torch.int64:
            raise ValueError("DeviceDraft: row_off and depth are int32, mask is int64")
        if depth.dim() != 1 or tuple(mask.shape) != (depth.shape[0], words):
            raise ValueError(f"DeviceDraft: depth {tuple(depth.shape)} and mask {tuple(mask.shape)} for max_rows {max_rows}")
        self.row_off, self.depth, self.mask = row_off.contiguous(), depth.contiguous(), mask.contiguous()
        self.rope = None if rope is None else list(rope)
        table = None
        if self.rope is not None:
            table = (ods_rope * len(self.rope))(*(r.c for r in self.rope))
        self._table = table
        self.norm, self.shared = None if norm is None else list(norm), shared
        gains = None
        if self.norm is not None:
            gains = (ods_head_norm * len(self.norm))(*(n.c for n in self.norm))
        self._gains = gains
        self.c = ods_draft(depth.shape[0], max_rows, _ptr(self.row_off), _ptr(self.depth), _ptr(self.mask),
                           None if table is None else C.cast(table, C.POINTER(ods_rope)),
                           None if gains is None else C.cast(gains, C.POINTER(ods_head_norm)),
                           None if shared is None else C.pointer(shared.c))
        self.devices = _devices(self.row_off, self.depth, self.mask, *(r.freqs for r in self.rope or ()),
                                *(g for n in self.norm or () for g in (n.gain_q, n.gain_k)),
                                *((shared.group_off, shared.tokens) if shared is not None else ()))

    @property
    def rows(self) -> int:
        return self.c.rows

    def check(self, block: DeviceBlock, batch: DeviceBatch) -> None:
        """The host-visible sizes fit the block and the batch."""
        if self.row_off.shape != (batch.batch + 1,):
            raise ValueError(f"DeviceDraft: row_off {tuple(self.row_off.shape)} for a batch of {batch.batch}")
        if batch.ctx_lens.numel() < batch.batch:
            raise ValueError(f"DeviceDraft: ctx_lens {tuple(batch.ctx_lens.shape)} for a batch of {batch.batch}")
        if self.rope is not None and len(self.rope) != len(block.cfgs):
            raise ValueError(f"DeviceDraft: {len(self.rope)} ropes for {len(block.cfgs)} layers")
        if self.norm is not None and len(self.norm) != len(block.cfgs):
            raise ValueError(f"DeviceDraft: {len(self.norm)} norms for {len(block.cfgs)} layers")
        for n, cfg in zip(self.norm or (), block.cfgs):
            if n.head_dim != cfg.head_dim:
                raise ValueError(f"DeviceDraft: a norm of heads of {n.head_dim} for a layer's of {cfg.head_dim}")


class DeviceState:
    """Live buffers sized by ods_live_bytes and a workspace of ods_workspace_bytes; with `draft`, for its rows
    (ods_draft_workspace_bytes). `rows`: what the buffers hold; a call on more is refused, since the library sees
    addresses only."""

    def __init__(self, block: DeviceBlock, batch: DeviceBatch, device="cuda", fill=None,
                 draft: DeviceDraft | None = None):
        self.buffers = {}
        self.rows = batch.batch if draft is None else draft.rows
        for i, name in enumerate(_b.BUFFERS):
            nbytes = _b.ods_live_bytes(block.c, self.rows, i)
            if nbytes == 0:
                continue
            dt = _BUF_DTYPE.get(name, torch.bfloat16)
            n = nbytes // torch.tensor([], dtype=dt).element_size()
            t = torch.empty(n, dtype=dt, device=device)
            if fill is not None:
                t.fill_(fill if dt != torch.int32 else -7)
            self.buffers[name] = t
        self.ws_bytes = (_b.ods_workspace_bytes(block.c, batch.c) if draft is None
                         else _b.ods_draft_workspace_bytes(block.c, batch.c, draft.c))
        self.ws = torch.empty(self.ws_bytes, dtype=torch.uint8, device=device)
        self.devices = _devices(self.ws)
        self.c = ods_state()
        for name, t in self.buffers.items():
            setattr(self.c, name, t.data_ptr())
        self.c.ws = self.ws.data_ptr()
        self.c.ws_bytes = self.ws_bytes

    def view(self, name: str, *shape):
        t = self.buffers[name]
        n = 1
        for s in shape:
            n *= s
        return t[:n].view(*shape)

    def check(self, who: str, rows: int) -> None:
        """The live buffers hold `rows` rows."""
        if rows > self.rows:
            raise ValueError(f"{who}: {rows} rows, the state's buffers hold {self.rows}")


def current_stream() -> int:
    # the handle alone: torch.cuda.current_stream() makes a Stream object first, 2.9 us
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


def run_partition(block: DeviceBlock, op_begin: int, op_end: int, batch: DeviceBatch, state: DeviceState,
                  stream: int | None = None) -> None:
    state.check("run_partition", batch.batch)
    st = _b.ods_run_partition(block.c, op_begin, op_end, batch.c, state.c,
                              current_stream() if stream is None else stream)
    _b._check(st, f"ods_run_partition[{op_begin},{op_end})")


def run_partition_scratch(block: DeviceBlock, op_begin: int, op_end: int, batch: DeviceBatch, state: DeviceState,
                          stream: int | None = None) -> None:
    """ods_run_partition_scratch: the same range on the library's own workspace (state.ws is not used)."""
    state.check("run_partition_scratch", batch.batch)
    st = _b.ods_run_partition_scratch(block.c, op_begin, op_end, batch.c, state.c,
                                      current_stream() if stream is None else stream)
    _b._check(st, f"ods_run_partition_scratch[{op_begin},{op_end})")


def attn_stage(block, layer, batch, state, stream=None) -> None:
    state.check("attn_stage", batch.batch)
    st = _b.ods_attn_stage(block.c, layer, batch.c, state.c, current_stream() if stream is None else stream)
    _b._check(st, f"ods_attn_stage({layer})")


def ffn_stage(block, layer, batch, state, stream=None) -> None:
    state.check("ffn_stage", batch.batch)
    st = _b.ods_ffn_stage(block.c, layer, batch.c, state.c, current_stream() if stream is None else stream)
    _b._check(st, f"ods_ffn_stage({layer})")


class PartitionGraph:
    """Operators [op_begin, op_end) captured once as a HIP graph; launch()
    replays them on a stream with the buffers bound at capture. Rewrite the
    device contents (resid, ctx_lens, page_table) between launches; keep the
    block, batch and state objects (and their buffers) alive while the graph is."""

    def __init__(self, block: DeviceBlock, op_begin: int, op_end: int, batch: DeviceBatch, state: DeviceState):
        self.handle = None
        state.check("PartitionGraph", batch.batch)
        st, h = _b.ods_partition_graph(block.c, op_begin, op_end, batch.c, state.c)
        _b._check(st, f"ods_partition_graph[{op_begin},{op_end})")
        self.handle = h
        self._keep = (block, batch, state)

    def launch(self, stream: int | None = None) -> None:
        _b._check(_b.ods_graph_launch(self.handle, current_stream() if stream is None else stream), "ods_graph_launch")

    def close(self) -> None:
        if self.handle:
            _b.ods_graph_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


# ---------------------------------------------------------------- drafted rows and pages

def run_draft(block: DeviceBlock, op_begin: int, op_end: int, batch: DeviceBatch, draft: DeviceDraft,
              state: DeviceState, stream: int | None = None) -> None:
    """Operators [op_begin, op_end) for the drafted rows of a batch (ods_run_draft): ctx_lens counts the cached
    tokens, the drafted ones not among them."""
    draft.check(block, batch)
    state.check("run_draft", draft.rows)
    st = _b.ods_run_draft(block.c, op_begin, op_end, batch.c, draft.c, state.c,
                          _stream_of("run_draft", stream, *block.op_devices(op_begin, op_end), *batch.devices, *draft.devices,
                                     *state.devices))
    _b._check(st, f"ods_run_draft[{op_begin},{op_end})")


class DraftGraph(PartitionGraph):
    """PartitionGraph for drafted rows: rewrite row_off, depth, mask and ctx_lens between launches."""

    def __init__(self, block: DeviceBlock, op_begin: int, op_end: int, batch: DeviceBatch, draft: DeviceDraft,
                 state: DeviceState):
        self.handle = None
        draft.check(block, batch)
        state.check("DraftGraph", draft.rows)
        _stream_of("DraftGraph", None, *block.op_devices(op_begin, op_end), *batch.devices, *draft.devices, *state.devices)
        st, h = _b.ods_draft_graph(block.c, op_begin, op_end, batch.c, draft.c, state.c)
        _b._check(st, f"ods_draft_graph[{op_begin},{op_end})")
        self.handle = h
        self._keep = (block, batch, draft, state)


def _layers(block: DeviceBlock, layers):
    return (0, len(block.cfgs)) if layers is None else layers


def kv_accept(block: DeviceBlock, batch: DeviceBatch, draft: DeviceDraft, path: torch.Tensor, path_len: torch.Tensor,
              ctx_out: torch.Tensor | None = None, layers=None, stream: int | None = None) -> None:
    """Keep drafted tokens path[b, :path_len[b]] (int32, ascending) of every sequence: their cache slots move to
    positions ctx, ctx + 1, ... in every layer (or layers = (begin, end)); ctx_out (may be batch.ctx_lens) gets the
    new contexts."""
    draft.check(block, batch)
    B = batch.batch
    for name, t, shape in (("path", path, (B, path.shape[-1])), ("path_len", path_len, (B,)), ("ctx_out", ctx_out, (B,))):
        if t is not None and (t.dtype != torch.int32 or tuple(t.shape) != shape or not t.is_contiguous()):
            raise ValueError(f"kv_accept: {name} must be contiguous int32 {shape}, got {t.dtype} {tuple(t.shape)}")
    a, b = _layers(block, layers)
    st = _b.ods_kv_accept(block.c, a, b, batch.c, draft.c, path.data_ptr(), path.shape[1], path_len.data_ptr(),
                          _ptr(ctx_out), _stream_of("kv_accept", stream, *block.pool_devices(a, b), *batch.devices, *draft.devices,
                                                    *_devices(path, path_len, ctx_out)))
    _b._check(st, "ods_kv_accept")


def kv_copy_pages(block: DeviceBlock, pairs: torch.Tensor, layers=None, stream: int | None = None) -> None:
    """Copy pages pairs[i, 0] -> pairs[i, 1] (device int32 [n, 2]) in the pools of every layer (or layers = (begin,
    end)). No page may be a dst twice, or both a src and a dst."""
    if pairs.dtype != torch.int32 or pairs.dim() != 2 or pairs.shape[1] != 2 or not pairs.is_contiguous():
        raise ValueError(f"kv_copy_pages: pairs must be contiguous int32 [n, 2], got {pairs.dtype} {tuple(pairs.shape)}")
    a, b = _layers(block, layers)
    st = _b.ods_kv_copy_pages(block.c, a, b, pairs.data_ptr(), pairs.shape[0],
                              _stream_of("kv_copy_pages", stream, *block.pool_devices(a, b), pairs.get_device()))
    _b._check(st, "ods_kv_copy_pages")


class KvPages:
    """Page table of up to `rows` sequences that may share pages (ods_pages_*), on the host: `table` int32 numpy
    [rows, max_pages] and `tokens` [rows]. Growing a sequence whose last page is shared gives it a page of its own;
    the copies that takes collect until take_copies(). Upload `table` after changes, and run the copies before the
    next step writes the cache."""

    def __init__(self, pool_pages: int, rows: int, max_pages: int, table=None, tokens=None):
        self.table = np.full((rows, max_pages), -1, np.int32)
        self.tokens = np.zeros(rows, np.int32)
        if table is not None:
            self.table[:] = table
            self.tokens[:] = tokens
        self._refs, self._free = np.zeros(pool_pages, np.int32), np.zeros(pool_pages, np.int32)
        self.c = ods_pages(pool_pages, _b._np(self._refs), _b._np(self._free), 0)
        _b._check(_b.ods_pages_init(self.c, None if table is None else self.table), "ods_pages_init")
        self._copies: list[list[tuple[int, int]]] = []
        self._read: set[int] = set()     # pages of the last list of copies
        self._written: set[int] = set()

    @property
    def free(self) -> int:
        return self.c.n_free

    def _add(self, pairs) -> None:
        """Copies in the order they must happen. A list's copies run in any order, so a page that one of them writes
        may be in it once only (a page they only read, more often): the next copy of it starts a new list."""
        for src, dst in np.asarray(pairs).tolist():
            if not self._copies or src in self._written or dst in self._written or dst in self._read:
                self._copies.append([])
                self._read, self._written = set(), set()
            self._copies[-1].append((src, dst))
            self._read.add(src)
            self._written.add(dst)

    def resize(self, row: int, tokens: int) -> None:
        """Sequence `row` grows or shrinks to `tokens` tokens."""
        if not 0 <= tokens < 1 << 31:  # the library would see its low 32 bits
            raise ValueError(f"KvPages.resize: {tokens} tokens")
        pair = np.zeros(2, np.int32)
        st, n = _b.ods_pages_resize(self.c, self.table[row], int(self.tokens[row]), tokens, pair)
        _b._check(st, "ods_pages_resize")
        self.tokens[row] = tokens
        if n:
            self._add([pair])

    def fork(self, src: int, dst: int) -> None:
        """Empty sequence `dst` shares every page of `src`."""
        if self.tokens[dst]:
            raise ValueError(f"KvPages.fork: row {dst} holds {self.tokens[dst]} tokens")
        _b._check(_b.ods_pages_fork(self.c, self.table[src], self.table[dst], int(self.tokens[src])), "ods_pages_fork")
        self.tokens[dst] = self.tokens[src]

    def release(self, row: int) -> None:
        """Sequence `row` gives back its pages."""
        _b._check(_b.ods_pages_release(self.c, self.table[row]), "ods_pages_release")
        self.tokens[row] = 0

    def shared(self) -> tuple:
        """Groups of adjacent rows that share leading pages: (group_off [groups + 1], tokens [groups]) int32 numpy, for
        SharedPrefix (ods_pages_shared). No groups where none shares two pages, the least that attention reads once: each
        sequence is then read by itself at its full speed."""
        rows = len(self.tokens)
        off, tokens = np.zeros(rows + 1, np.int32), np.zeros(max(rows, 1), np.int32)
        st, n = _b.ods_pages_shared(self.table, self.tokens, off, tokens)
        _b._check(st, "ods_pages_shared")
        if n and tokens[:n].max() < 2 * _b.PAGE_TOKENS:
            n = 0
        return off[:n + 1].copy(), tokens[:n].copy()

    def compact(self, max_pairs: int | None = None) -> int:
        """Move the highest held pages into the lowest free ones; returns how many."""
        n = int(self.c.pool_pages) if max_pairs is None else max_pairs
        pairs = np.zeros((max(n, 1), 2), np.int32)
        st, got = _b.ods_pages_compact(self.c, self.table, pairs[:n])
        _b._check(st, "ods_pages_compact")
        self._add(pairs[:got])
        return got

    def take_copies(self) -> list:
        """The copies since the last call: int32 numpy [n, 2] arrays for kv_copy_pages, to be run in this order."""
        out = [np.array(c, np.int32).reshape(-1, 2) for c in self._copies]
        self._copies = []
        return out


# ---------------------------------------------------------------- verification of drafted tokens

class DraftVerifier:
    """Accepted paths of drafted tokens and the tokens after them (ods_draft_verify), for batches of up to `batch`
    sequences over up to `vocab` tokens: `path` [batch, path_cols], `path_len` [batch] (what kv_accept takes) and `next`
    [batch], int32, with a workspace. A run writes the rows of its batch; runs on one verifier are ordered by the caller."""

    DTYPES = {torch.float32: _b.ODS_PROBS_F32, torch.bfloat16: _b.ODS_PROBS_BF16}

    def __init__(self, batch: int, path_cols: int, vocab: int, device="cuda"):
        nbytes = _b.ods_verify_workspace_bytes(batch, vocab)
        if nbytes == 0 or not 1 <= path_cols <= _b.DRAFT_MAX_ROWS:
            raise ValueError(f"DraftVerifier: batch {batch}, path_cols {path_cols}, vocab {vocab}")
        self.batch, self.path_cols, self.vocab = batch, path_cols, vocab
        self.path = torch.full((batch, path_cols), -1, dtype=torch.int32, device=device)
        self.path_len = torch.zeros(batch, dtype=torch.int32, device=device)
        self.next = torch.full((batch,), -1, dtype=torch.int32, device=device)
        self.ws = torch.empty(nbytes, dtype=torch.uint8, device=device)
        self._device = self.ws.get_device()
        self.c = ods_verify()
        self.c.path_cols, self.c.path, self.c.path_len = path_cols, _ptr(self.path), _ptr(self.path_len)
        self.c.next_token, self.c.ws, self.c.ws_bytes = _ptr(self.next), _ptr(self.ws), nbytes

    def run(self, draft: DeviceDraft, tokens: torch.Tensor, parent: torch.Tensor, target: torch.Tensor,
            accept_u: torch.Tensor, next_u: torch.Tensor, proposal: torch.Tensor | None = None,
            stream: int | None = None) -> None:
        """tokens, parent int32 [rows]; target and proposal [rows, vocab] probabilities, fp32 or bf16, rows at any stride
        (proposal None: the tokens are guesses); accept_u [rows] and next_u [batch of this call] fp32 in [0, 1)."""
        c, B, rows = self.c, draft.row_off.shape[0] - 1, draft.c.rows
        vocab = target.shape[1] if target.dim() == 2 else 0
        # one condition for what is right, reasons afterwards: a call of a few microseconds is host work first
        if not (B <= self.batch and 1 <= vocab <= self.vocab and target.dtype in self.DTYPES
                and tokens.shape == parent.shape == accept_u.shape == (rows,) and next_u.shape == (B,)
                and tokens.dtype == parent.dtype == torch.int32 and accept_u.dtype == next_u.dtype == torch.float32
                and tokens.is_contiguous() and parent.is_contiguous() and accept_u.is_contiguous() and next_u.is_contiguous()
                and target.shape == (rows, vocab) and (target.stride(1) == 1 or vocab == 1 or rows == 0)
                and (proposal is None or (proposal.shape == target.shape and proposal.dtype == target.dtype
                                          and (proposal.stride(1) == 1 or vocab == 1 or rows == 0)))):
            self._refuse(rows, B, tokens, parent, target, accept_u, next_u, proposal)
        # the stride of a single row means nothing
        c.vocab, c.dtype, c.target = vocab, self.DTYPES[target.dtype], target.data_ptr()
        c.target_stride = target.stride(0) if rows > 1 else vocab
        if proposal is None:
            c.proposal, c.proposal_stride = None, 0
        else:
            c.proposal, c.proposal_stride = proposal.data_ptr(), proposal.stride(0) if rows > 1 else vocab
        c.tokens, c.parent = tokens.data_ptr(), parent.data_ptr()
        c.accept_u, c.next_u = accept_u.data_ptr(), next_u.data_ptr()
        stream = _stream_of("DraftVerifier", stream, self._device, draft.row_off.get_device(), tokens.get_device(), parent.get_device(),
                            target.get_device(), accept_u.get_device(), next_u.get_device(),
                            self._device if proposal is None else proposal.get_device())
        _b._check(_b.ods_draft_verify(B, draft.c, c, stream), "ods_draft_verify")

    def _refuse(self, rows, B, tokens, parent, target, accept_u, next_u, proposal):
        if B > self.batch:
            raise ValueError(f"DraftVerifier: {B} sequences, made for {self.batch}")
        for name, t, dtype, shape in (("tokens", tokens, torch.int32, (rows,)), ("parent", parent, torch.int32, (rows,)),
                                      ("accept_u", accept_u, torch.float32, (rows,)), ("next_u", next_u, torch.float32, (B,))):
            if t.dtype != dtype or tuple(t.shape) != shape or not t.is_contiguous():
                raise ValueError(f"DraftVerifier: {name} must be contiguous {dtype} {shape}, got {t.dtype} {tuple(t.shape)}")
        for name, t in (("target", target), ("proposal", proposal)):
            if t is None:
                continue
            if t.dtype not in self.DTYPES or t.dtype != target.dtype or t.dim() != 2 or t.shape != target.shape or t.shape[0] != rows:
                raise ValueError(f"DraftVerifier: {name} is fp32 or bf16 [{rows}, vocab], target and proposal alike, got "
                                 f"{t.dtype} {tuple(t.shape)}")
            if t.stride(1) != 1 and t.numel() > t.shape[0]:
                raise ValueError(f"DraftVerifier: the values of a row of {name} must be contiguous")
        raise ValueError(f"DraftVerifier: {target.shape[1]} tokens, made for {self.vocab}")
