"""Without a GPU: calls whose tensors lie on different devices are refused, whichever of them it is, with a stream named or
not. The stand-ins for tensors of another device have no memory, and no call here could reach a launch."""
import pytest
import torch

import workloads as W

B = pytest.importorskip("paper_2609_14237_amd.binding")
from paper_2609_14237_amd import runtime as R  # noqa: E402

CFG = W.LayerCfg(hidden=256, n_q=4, n_kv=2, head_dim=64, ffn=512)


def z(*shape, dt=torch.int32):
    return torch.zeros(*shape, dtype=dt)


class Far(torch.Tensor):
    """A host tensor that says it is on device 3."""

    def get_device(self):
        return 3


def far(t):
    return t.as_subclass(Far)


WEIGHTS = ("g_attn", "w_qkv", "w_o", "g_ffn", "w_gate_up", "w_down", "w_router")


def block_of(n=1, far_pool=(), far_weight=()):
    t = z(64, dt=torch.bfloat16)
    ws = [{k: far(t) if (l, k) in far_weight else None for k in WEIGHTS} for l in range(n)]
    return R.DeviceBlock([CFG] * n, ws, [far(t) if l in far_pool else t for l in range(n)], 0)


def batch_of(name=None):
    ts = {"ctx_lens": z(2), "page_table": z(2, 4), "ring_table": z(2, 4)}
    if name:
        ts[name] = far(ts[name])
    return R.DeviceBatch(ts["ctx_lens"], ts["page_table"], ring_table=ts["ring_table"])


def draft_of(name=None, rope=None):
    ts = {"row_off": z(3), "depth": z(8), "mask": z(8, 1, dt=torch.int64)}
    if name:
        ts[name] = far(ts[name])
    return R.DeviceDraft(ts["row_off"], ts["depth"], ts["mask"], 64, rope=rope)


def run(block=None, batch=None, draft=None, state=None, ops=(2, 5)):
    block, batch, draft = block or block_of(), batch or batch_of(), draft or draft_of()
    state = state or R.DeviceState(block, batch, device="cpu", draft=draft)
    R.run_draft(block, *ops, batch, draft, state, stream=0)


def test_drafted_rows_of_two_devices():
    with pytest.raises(B.OdsError):  # one device: the library's own checks, pool_pages is 0
        run()
    for kw in ([dict(batch=batch_of(n)) for n in ("ctx_lens", "page_table", "ring_table")] +
               [dict(draft=draft_of(n)) for n in ("row_off", "depth", "mask")] +
               [dict(block=block_of(far_pool=(0,))), dict(block=block_of(far_weight=((0, "w_o"),)))]):
        with pytest.raises(ValueError, match="device"):
            run(**kw)
    r = R.Rope(64, device="cpu")
    r.freqs = far(r.freqs)
    with pytest.raises(ValueError, match="device"):
        run(draft=draft_of(rope=[r]))
    t = z(64, dt=torch.bfloat16)  # what a weight dictionary holds beside the weights is not looked at
    with pytest.raises(B.OdsError):
        run(block=R.DeviceBlock([CFG], [{"w_o": None, "lm_head": far(t)}], [t], 0))
    block, batch, draft = block_of(), batch_of(), draft_of()
    state = R.DeviceState(block, batch, device="cpu", draft=draft)
    state.devices = (3,)  # as made with device="cuda:3"
    with pytest.raises(ValueError, match="device"):
        run(block, batch, draft, state)


def test_layers_of_two_devices():
    """A block whose layers lie on two devices runs on either's layers; a call over both is refused."""
    block = block_of(3, far_pool=(2,))
    for ops in ((0, 10), (2, 15), (12, 20)):
        with pytest.raises(B.OdsError):
            run(block, ops=ops)
    for ops in ((0, 30), (19, 21), (22, 25)):
        with pytest.raises(ValueError, match="device"):
            run(block, ops=ops)
    for ops in ((-1, 3), (5, 5), (0, 31)):  # not a range: the library says so
        with pytest.raises((B.OdsError, ValueError)):
            run(block, ops=ops)
    pairs, path, n = z(0, 2), z(2, 4), z(2)
    for layers in (None, (0, 3), (2, 3)):
        with pytest.raises(ValueError, match="device"):
            R.kv_copy_pages(block, pairs, layers=layers, stream=0)
        with pytest.raises(ValueError, match="device"):
            R.kv_accept(block, batch_of(), draft_of(), path, n, layers=layers, stream=0)
    for layers in ((0, 2), (1, 2)):
        with pytest.raises(B.OdsError):
            R.kv_copy_pages(block, pairs, layers=layers, stream=0)
        with pytest.raises(B.OdsError):
            R.kv_accept(block, batch_of(), draft_of(), path, n, layers=layers, stream=0)


def test_cache_and_rotary_tensors_of_two_devices():
    block, path, n = block_of(), z(2, 4), z(2)
    for args in ((batch_of("page_table"), draft_of(), path, n, None), (batch_of(), draft_of("row_off"), path, n, None),
                 (batch_of(), draft_of(), far(path), n, None), (batch_of(), draft_of(), path, far(n), None),
                 (batch_of(), draft_of(), path, n, far(z(2)))):
        with pytest.raises(ValueError, match="device"):
            R.kv_accept(block, *args, stream=0)
    with pytest.raises(ValueError, match="device"):
        R.kv_copy_pages(block, far(z(4, 2)), stream=0)
    with pytest.raises(B.OdsError):  # page operators read no weights
        R.kv_copy_pages(block_of(far_weight=((0, "w_o"),)), z(4, 2), stream=0)
    r, x, pos = R.Rope(64, device="cpu"), z(0, 2, 64, dt=torch.bfloat16), z(0)
    assert R.rope(r, x, pos, stream=0) is x
    for kw in (dict(x=far(x), pos=pos), dict(x=x, pos=far(pos)), dict(x=x, pos=pos, out=far(x))):
        with pytest.raises(ValueError, match="device"):
            R.rope(r, **kw, stream=0)
