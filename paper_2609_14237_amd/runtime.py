"""PyTorch-side marshalling around the C ABI: packs device tensors into the
ods_* structs and allocates the live buffers and workspace the library sizes.
No operator of the decode step is computed here."""
from __future__ import annotations

import ctypes as C

import numpy as np
import torch

from . import binding as _b
from .binding import ods_batch, ods_block, ods_draft, ods_layer, ods_layer_cfg, ods_pages, ods_rope, ods_state


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
    (32, 1)."""

    SCALINGS = {"plain": _b.ODS_ROPE_PLAIN, "linear": _b.ODS_ROPE_LINEAR, "base": _b.ODS_ROPE_BASE,
                "rotations": _b.ODS_ROPE_ROTATIONS, "index": _b.ODS_ROPE_INDEX}

    def __init__(self, head_dim: int, theta: float = 10000.0, rotary_dim: int | None = None, interleaved: bool = False,
                 scaling: str = "plain", factor: float = 1.0, orig_ctx: float = 8192.0, turns=None,
                 amplitude: float = 1.0, device="cuda"):
        if scaling not in self.SCALINGS:
            raise ValueError(f"scaling {scaling!r}: one of {', '.join(self.SCALINGS)}")
        hi, lo = turns if turns is not None else ((32.0, 1.0) if scaling == "index" else (4.0, 1.0))
        rdim = head_dim if rotary_dim is None else rotary_dim
        self.c = ods_rope(head_dim, rdim, int(interleaved), self.SCALINGS[scaling], theta, factor, orig_ctx, hi, lo,
                          amplitude, None)
        host = np.zeros(max(rdim // 2, 1), np.float64)
        _b._check(_b.ods_rope_freqs(self.c, host), "ods_rope_freqs")
        self.freqs = torch.from_numpy(host).to(device)
        self.c.freqs = self.freqs.data_ptr()


def rope(r: Rope, x: torch.Tensor, pos: torch.Tensor, out: torch.Tensor | None = None, stream: int | None = None):
    """Rotate x [rows, heads, head_dim] (bf16; the last two dims contiguous, rows at any stride of 8) to positions
    pos [rows] (int32; rows with a negative one are left alone) into out (default x, in place); returns out."""
    y = x if out is None else out
    for t in (x, y):
        if t.dtype != torch.bfloat16 or t.dim() != 3 or t.shape[2] != r.c.head_dim:
            raise ValueError(f"rope takes bf16 [rows, heads, {r.c.head_dim}], got {t.dtype} {tuple(t.shape)}")
        if t.numel() and (t.stride(2) != 1 or (t.shape[1] > 1 and t.stride(1) != r.c.head_dim)):
            raise ValueError("rope: the heads of a row must be contiguous")
    if x.shape != y.shape or pos.dtype != torch.int32 or pos.shape != x.shape[:1] or not pos.is_contiguous():
        raise ValueError(f"rope: x {tuple(x.shape)}, out {tuple(y.shape)}, pos {pos.dtype} {tuple(pos.shape)}")
    rows, heads = x.shape[:2]
    width = heads * r.c.head_dim  # the stride of a single row means nothing
    xs, ys = (t.stride(0) if rows > 1 else width for t in (x, y))
    _b._check(_b.ods_rope_rows(r.c, x.data_ptr(), xs, y.data_ptr(), ys, rows, heads, pos.data_ptr(),
                               _stream_of("rope", stream, x.get_device(), y.get_device(), pos.get_device(),
                                          r.freqs.get_device())), "ods_rope_rows")
    return y


class DeviceDraft:
    """ods_draft: drafted rows of a batch. row_off [B + 1] and depth [rows] int32, mask [rows, ceil(max_rows / 64)]
    int64 (bit patterns; a 1-D tensor is one word per row). `rope`: None for the layers' own, or one Rope per layer."""

    def __init__(self, row_off: torch.Tensor, depth: torch.Tensor, mask: torch.Tensor, max_rows: int, rope=None):
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
        self.c = ods_draft(depth.shape[0], max_rows, _ptr(self.row_off), _ptr(self.depth), _ptr(self.mask),
                           None if table is None else C.cast(table, C.POINTER(ods_rope)))
        self.devices = _devices(self.row_off, self.depth, self.mask, *(r.freqs for r in self.rope or ()))

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
