"""What rdkv_slots_tree_attn and rdkv_slots_accept refuse, without a GPU: nothing is launched for a bad argument."""
import ctypes

import pytest
import torch

from paper_2605_08317_amd import binding as b
from tests.test_slots_host import INVALID, SHAPE, struct


def attn(c, n=4, q=16, k=16, v=16, parent=4, counts=None, out=16, stats=None, ws=16, ws_bytes=1 << 40):
    return b.lib.rdkv_slots_tree_attn(ctypes.byref(c), n, q, k, v, parent, counts, out, stats, ws, ws_bytes, None)


def accept(c, n=4, m=3, q=16, k=16, v=16, path=4, stats=8, slot=None, ws=16, ws_bytes=1 << 40):
    return b.lib.rdkv_slots_accept(ctypes.byref(c), n, m, q, k, v, path, stats, slot, ws, ws_bytes, None)


@pytest.mark.parametrize("kw, status", [
    (dict(batch=-1), INVALID), (dict(head_dim=64), SHAPE), (dict(hq=7), SHAPE), (dict(capacity=0), SHAPE), (dict(bits=8), SHAPE), (dict(sinks=100), SHAPE),
    (dict(score_cap=-1.0), INVALID), (dict(decay=1.5), INVALID), (dict(k=None), INVALID), (dict(v=17), INVALID), (dict(len=None), INVALID)])
def test_a_bad_struct_is_refused(kw, status):
    assert attn(struct(**kw)) == status and accept(struct(**kw)) == status
    assert b.lib.rdkv_slots_tree_attn(None, 4, 16, 16, 16, 4, None, 16, None, 16, 0, None) == INVALID
    assert b.lib.rdkv_slots_accept(None, 4, 3, 16, 16, 16, 4, 8, None, 16, 1 << 40, None) == INVALID


def test_bad_arguments_are_refused():
    c = struct(weight=16)
    for n in (0, -1, 65, 2 ** 31 - 1):
        assert attn(c, n=n) == SHAPE and accept(c, n=n) == SHAPE and accept(c, m=n) == SHAPE
        assert b.lib.rdkv_slots_tree_workspace_bytes(ctypes.byref(c), n) == 0
    for kw in (dict(q=None), dict(k=None), dict(v=None), dict(parent=None), dict(out=None), dict(q=8), dict(k=24), dict(v=2), dict(out=17), dict(stats=12)):
        assert attn(c, **kw) == INVALID, kw
    for kw in (dict(q=None), dict(k=None), dict(v=None), dict(path=None), dict(stats=None), dict(q=8), dict(k=24), dict(v=2), dict(stats=12)):
        assert accept(c, **kw) == INVALID, kw
    assert accept(struct(), k=None, q=None, stats=None) == INVALID


def test_workspaces():
    r = ctypes.byref
    large = struct(batch=1, capacity=100000)
    need = b.lib.rdkv_slots_tree_workspace_bytes(r(large), 8)
    assert need > 0 and need % 16 == 0
    assert attn(large, n=8, ws=16, ws_bytes=need - 1) == INVALID and attn(large, n=8, ws=None) == INVALID and attn(large, n=8, ws=24, ws_bytes=need) == INVALID
    need = b.lib.rdkv_slots_accept_workspace_bytes(r(large))
    assert need > 0 and need % 16 == 0 and b.lib.rdkv_slots_accept_workspace_bytes(r(struct(hq=7))) == 0
    for ws, n in ((16, need - 1), (None, need), (24, need)):
        assert accept(large, ws=ws, ws_bytes=n) == INVALID
    assert b.lib.rdkv_slots_tree_workspace_bytes(r(struct(hq=7)), 8) == 0 and b.lib.rdkv_slots_tree_workspace_bytes(None, 8) == 0


def test_nothing_to_do_is_no_error():
    c = struct(batch=0, k=None, v=None, pos=None, len=None, next=None)
    assert attn(c, q=None, k=None, v=None, parent=None, out=None, ws=None, ws_bytes=0) == 0
    assert accept(c, q=None, k=None, v=None, path=None, stats=None) == 0
    assert b.lib.rdkv_slots_tree_workspace_bytes(ctypes.byref(c), 4) == 0


def test_the_binding_refuses_tensors_the_library_would_misread():
    bf, i32 = torch.bfloat16, torch.int32
    s = b.Slots(2, 8, 2, 100, device="cpu")
    q, k = torch.zeros(2, 5, 8, 128, dtype=bf), torch.zeros(2, 5, 2, 128, dtype=bf)
    parent, path, stats = torch.zeros(2, 5, dtype=i32), torch.zeros(2, 3, dtype=i32), torch.zeros(2, 5, 8, 2)
    good = dict(q=q, k_draft=k, v_draft=k, parent=parent)
    for bad in (dict(q=q.float()), dict(q=q[:, :4]), dict(q=q.transpose(1, 2)), dict(k_draft=k[:, :, :1]), dict(k_draft=k[0]), dict(v_draft=k.transpose(0, 1)), dict(parent=parent.long()),
                dict(parent=parent[:, :4]), dict(counts=torch.zeros(2)), dict(counts=torch.zeros(3, dtype=i32)), dict(out=q.float()), dict(stats=stats[..., 0]),
                dict(workspace=torch.zeros(64)), dict(workspace=torch.zeros(128, dtype=torch.uint8)[::2])):
        with pytest.raises(ValueError):
            b.rdkv_slots_tree_attn(s, **dict(good, **bad))
    good = dict(q=q, k_draft=k, v_draft=k, path=path, stats=stats)
    for bad in (dict(q=q.float()), dict(k_draft=k[0]), dict(v_draft=k[:, :4]), dict(path=path.long()), dict(path=path[0]), dict(path=path[:1]), dict(stats=stats[:, :4]),
                dict(stats=stats.double()), dict(slot=torch.zeros(2, 2, 4, dtype=i32)), dict(slot=torch.zeros(2, 2, 3)), dict(workspace=torch.zeros(4096))):
        with pytest.raises(ValueError):
            b.rdkv_slots_accept(s, **dict(good, **bad))
    for call in (lambda: b.rdkv_slots_tree_attn(s, q, k, k, parent), lambda: b.rdkv_slots_accept(s, q, k, k, path, stats)):
        with pytest.raises(ValueError, match="cpu"):
            call()
    with pytest.raises(ValueError, match="32-bit"):
        s.tree_workspace(2.5)
    assert s.tree_workspace(65).numel() == 16
