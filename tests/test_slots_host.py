"""What the slot caches' entry points refuse, without a GPU: nothing is launched for a bad argument."""
import copy
import ctypes
import os
import subprocess

import pytest
import torch

from paper_2605_08317_amd import binding as b

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INVALID, SHAPE = 1, 2


def struct(**kw):
    c = b.rdkv_slots()
    assert b.lib.rdkv_slots_default(ctypes.byref(c)) == 0
    for name, x in dict(dict(batch=2, hq=8, hkv=2, capacity=100, k=16, v=16, pos=16, len=16, next=16), **kw).items():
        setattr(c, name, x)
    return c


def calls(c, seq=(5, 5), first=0, w=16, ws=None, ws_bytes=0):
    """Every entry point's status for the struct, with pointers that no call may look at."""
    r = ctypes.byref(c)
    lens = (ctypes.c_int32 * len(seq))(*seq)
    return {"fill": lambda: b.lib.rdkv_slots_fill(r, first, len(seq), lens, 16, 16, w, ws, ws_bytes, None),
            "append": lambda: b.lib.rdkv_slots_append(r, 16, 16, None, None),
            "decode": lambda: b.lib.rdkv_slots_decode_attn(r, 16, 16, None, 16, 1 << 40, None),
            "read": lambda: b.lib.rdkv_slots_read(r, None, 4, 16, 16, None)}


@pytest.mark.parametrize("kw, status", [
    (dict(batch=-1), INVALID), (dict(hq=0), INVALID), (dict(hkv=0), INVALID), (dict(head_dim=64), SHAPE), (dict(hq=7), SHAPE),
    (dict(hq=6), SHAPE), (dict(hq=32), SHAPE), (dict(capacity=0), SHAPE), (dict(capacity=-5), SHAPE), (dict(bits=8), SHAPE), (dict(bits=2), SHAPE),
    (dict(sinks=-1), INVALID), (dict(recent=-1), INVALID), (dict(window=-1), INVALID), (dict(sinks=100), SHAPE), (dict(sinks=60, recent=41), SHAPE),
    (dict(sinks=2 ** 31 - 1, recent=2 ** 31 - 1), SHAPE), (dict(score_cap=-1.0), INVALID), (dict(score_cap=float("nan")), INVALID),
    (dict(score_cap=float("inf")), INVALID), (dict(score_cap=1e-40), INVALID), (dict(decay=-0.1), INVALID), (dict(decay=1.5), INVALID), (dict(decay=float("nan")), INVALID),
    (dict(batch=2 ** 20, capacity=2 ** 12), SHAPE), (dict(batch=2 ** 19, capacity=1), SHAPE), (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(pos=None), INVALID), (dict(len=None), INVALID),
    (dict(next=None), INVALID), (dict(k=24), INVALID), (dict(v=17), INVALID)])
def test_a_bad_struct_is_refused_by_every_call(kw, status):
    for name, call in calls(struct(**kw)).items():
        assert call() == status, name
        assert b.lib.rdkv_last_error()
    assert b.lib.rdkv_slots_append(None, 16, 16, None, None) == INVALID


def test_bad_arguments_are_refused():
    lib, r = b.lib, ctypes.byref(struct())
    assert lib.rdkv_slots_append(r, None, 16, None, None) == INVALID
    assert lib.rdkv_slots_append(r, 16, 24, None, None) == INVALID
    need = lib.rdkv_slots_decode_workspace_bytes(r)
    assert need > 0
    for q, out, ws, n in ((None, 16, 16, need), (16, None, 16, need), (16, 16, None, need), (16, 16, 16, need - 1), (8, 16, 16, need), (16, 16, 24, need)):
        assert lib.rdkv_slots_decode_attn(r, q, out, None, ws, n, None) == INVALID
    assert lib.rdkv_slots_read(r, None, -1, 16, 16, None) == INVALID
    assert lib.rdkv_slots_read(r, None, 4, None, 16, None) == INVALID
    assert lib.rdkv_slots_read(r, None, 2 ** 30, 16, 16, None) == SHAPE
    assert lib.rdkv_slots_read(r, None, 2 ** 26 - 64, 16, 16, None) == SHAPE                       # a launch's threads: 2^28 rows
    for bits in (16, 4):
        assert calls(struct(batch=1, hq=1, hkv=1, capacity=2 ** 29, bits=bits), seq=(2 ** 28,))["fill"]() == SHAPE
    c = struct()
    assert calls(c, seq=(5, -1))["fill"]() == SHAPE
    assert calls(c, seq=(5, 5), first=1)["fill"]() == INVALID and calls(c, seq=(5,), first=-1)["fill"]() == INVALID
    assert calls(c, seq=(5,), first=2 ** 31 - 1)["fill"]() == INVALID
    assert calls(c, seq=(101,), w=None)["fill"]() == INVALID          # too long to keep whole, and no weights to choose by
    assert calls(c, seq=(2 ** 30, 2 ** 30))["fill"]() == SHAPE
    assert lib.rdkv_slots_fill(r, 0, 1, None, 16, 16, 16, None, 0, None) == INVALID
    assert lib.rdkv_slots_fill(r, 0, -1, None, 16, 16, 16, None, 0, None) == INVALID


def test_nothing_to_do_is_no_error():
    c = struct(batch=0, k=None, v=None, pos=None, len=None, next=None)
    r = ctypes.byref(c)
    assert b.lib.rdkv_slots_append(r, None, None, None, None) == 0
    assert b.lib.rdkv_slots_decode_attn(r, None, None, None, None, 0, None) == 0
    assert b.lib.rdkv_slots_read(r, None, 4, None, None, None) == 0
    assert b.lib.rdkv_slots_fill(r, 0, 0, None, None, None, None, None, 0, None) == 0
    assert b.lib.rdkv_slots_read(ctypes.byref(struct()), None, 0, None, None, None) == 0


def test_sizes():
    r = ctypes.byref
    assert b.lib.rdkv_slots_side_bytes(r(struct())) == 2 * 2 * 100 * 256
    assert b.lib.rdkv_slots_side_bytes(r(struct(bits=4))) == 2 * 2 * 2 * 5120
    assert b.lib.rdkv_slots_side_bytes(r(struct(bits=4, capacity=64))) == 2 * 2 * 5120
    assert b.lib.rdkv_slots_side_bytes(r(struct(batch=1, hkv=1, hq=1, capacity=2 ** 30))) == 2 ** 38       # past 32 bits
    assert b.lib.rdkv_slots_side_bytes(r(struct(hq=7))) == 0 and b.lib.rdkv_slots_side_bytes(None) == 0
    assert b.lib.rdkv_slots_decode_workspace_bytes(r(struct(hq=7))) == 0


def test_the_binding_refuses_tensors_the_library_would_misread():
    s = b.Slots(2, 8, 2, 100, device="cpu")
    assert s.k.shape == (2, 2, 100, 128) and s.weight.shape == s.pos.shape == (2, 2, 100) and s.lens.shape == (2, 2)
    assert b.Slots(2, 8, 2, 100, bits=4, device="cpu").v.shape == (2, 2, 2, 5120)
    assert b.Slots(2, 8, 2, 100, track=False, device="cpu").weight is None
    bf = torch.bfloat16
    good = {"k": torch.zeros(2, 2, 100, 128, dtype=bf), "pos": torch.zeros(2, 2, 100, dtype=torch.int32)}
    s = b.Slots(2, 8, 2, 100, **good)
    assert s.c.k == good["k"].data_ptr() and s.pos is good["pos"]
    for bad in ({"k": good["k"].float()}, {"k": good["k"][:, :, :99]}, {"k": torch.zeros(2, 2, 128, 100, dtype=bf).transpose(2, 3)},
                {"pos": good["pos"].long()}, {"lens": torch.zeros(2, dtype=torch.int32)}, {"slopes": torch.zeros(2)}):
        with pytest.raises(ValueError):
            b.Slots(2, 8, 2, 100, device="cpu", **bad)
    for bad in (dict(hq=7), dict(capacity=0), dict(bits=5), dict(sinks=100), dict(decay=2.0), dict(score_cap=-1.0)):
        with pytest.raises(b.RdkvError):
            b.Slots(**dict(dict(batch=2, hq=8, hkv=2, capacity=100, device="cpu"), **bad))
    with pytest.raises(ValueError):
        b.Slots(2, 8, 2, 2 ** 33, device="cpu")
    new = torch.zeros(2, 2, 128, dtype=bf)
    for k in (new.float(), new[:1], new.transpose(0, 1).contiguous().transpose(0, 1)[:, :, ::2]):
        with pytest.raises(ValueError):
            b.rdkv_slots_append(s, k, new)
    q = torch.zeros(2, 8, 128, dtype=bf)
    for call in (lambda: b.rdkv_slots_decode_attn(s, q.float()), lambda: b.rdkv_slots_decode_attn(s, q[:, :4]),
                 lambda: b.rdkv_slots_decode_attn(s, q, out=torch.zeros(2, 8, 64)),
                 lambda: b.rdkv_slots_decode_attn(s, q, workspace=torch.zeros(64)),
                 lambda: b.rdkv_slots_read(s, torch.zeros(2, 2, 3, dtype=torch.int64)), lambda: b.rdkv_slots_read(s, torch.zeros(2, 2, dtype=torch.int32)),
                 lambda: b.rdkv_slots_fill(s, new, new, [5, 5])):
        with pytest.raises(ValueError):
            call()


def test_the_binding_refuses_what_would_be_cut_to_32_bits_and_host_memory():
    s = b.Slots(2, 8, 2, 100, device="cpu")
    new, q = torch.zeros(2, 2, 128, dtype=torch.bfloat16), torch.zeros(2, 8, 128, dtype=torch.bfloat16)
    rows = torch.zeros(2 * 2 * 5, 128, dtype=torch.bfloat16)
    for call in (lambda: b.rdkv_slots_fill(s, rows, rows, [5, 5], first=2 ** 32), lambda: b.rdkv_slots_fill(s, rows, rows, [2 ** 32 + 5, 5]),
                 lambda: b.rdkv_slots_read(s, n=2 ** 32)):
        with pytest.raises(ValueError, match="32-bit"):
            call()
    for call in (lambda: b.rdkv_slots_fill(s, rows, rows, [5, 5]), lambda: b.rdkv_slots_append(s, new, new), lambda: b.rdkv_slots_decode_attn(s, q),
                 lambda: b.rdkv_slots_read(s, n=3)):
        with pytest.raises(ValueError, match="cpu"):
            call()


def test_the_ctypes_struct_matches_the_c_header(tmp_path):
    fields = [f[0] for f in b.rdkv_slots._fields_]
    src = tmp_path / "layout.c"
    src.write_text("\n".join(['#include <stdio.h>', '#include <stddef.h>', '#include "rdkv.h"', 'int main(void) {',
                              '  printf("%zu\\n", sizeof(rdkv_slots));'] +
                             [f'  printf("%zu\\n", offsetof(rdkv_slots, {f}));' for f in fields] + ['  return 0;', '}']))
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    out = [int(x) for x in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    assert out == [ctypes.sizeof(b.rdkv_slots)] + [getattr(b.rdkv_slots, f).offset for f in fields]


@pytest.mark.parametrize("bits", [16, 4])
def test_the_most_rows_that_a_fill_puts_into_an_item(bits):
    """2^28 - 16: with one more, the launch that copies rows has 2^32 threads.  (Pointers that are not aligned: nothing is launched either way.)"""
    s = struct(batch=1, hq=1, hkv=1, capacity=2 ** 29, bits=bits)
    for n, status in ((2 ** 28 - 16, INVALID), (2 ** 28 - 15, SHAPE), (2 ** 28 - 1, SHAPE), (2 ** 28, SHAPE)):
        lens = (ctypes.c_int32 * 1)(n)
        assert b.lib.rdkv_slots_fill(ctypes.byref(s), 0, 1, lens, 24, 24, 16, None, 0, None) == status, n


def test_a_tensor_assigned_to_a_cache_is_the_one_its_calls_use():
    s = b.Slots(2, 8, 2, 9000, slopes=torch.zeros(8), device="cpu")
    assert (s.c.k, s.c.weight, s.c.slopes, s.c.len) == (s.k.data_ptr(), s.weight.data_ptr(), s.slopes.data_ptr(), s.lens.data_ptr())
    fields = {"k": "k", "v": "v", "pos": "pos", "weight": "weight", "lens": "len", "next_pos": "next", "slopes": "slopes"}
    for name, field in fields.items():
        new = torch.zeros_like(getattr(s, name))
        setattr(s, name, new)
        assert getattr(s, name) is new and getattr(s.c, field) == new.data_ptr(), name
        for bad in (new[:1], new.double(), new.unsqueeze(0), new.transpose(0, -1) if new.dim() > 1 else new[::2]):
            with pytest.raises(ValueError):
                setattr(s, name, bad)
            assert getattr(s, name) is new and getattr(s.c, field) == new.data_ptr(), name
        with pytest.raises(AttributeError):
            delattr(s, name)
        if name not in ("weight", "slopes"):
            with pytest.raises(ValueError):
                setattr(s, name, None)
    for name in ("c", "device", "batch", "hq", "hkv", "capacity", "bits", "d", "workspace_bytes", "address"):
        with pytest.raises(AttributeError):
            setattr(s, name, getattr(s, name))
    kept = s.workspace_bytes
    s.weight = s.slopes = None
    assert s.c.weight is None and s.c.slopes is None and s.workspace_bytes < kept
    s.weight = torch.zeros(2, 2, 9000)
    assert s.workspace_bytes == kept == s.workspace().numel()


def test_a_copy_of_a_cache_has_its_tensors_and_a_struct_of_its_own():
    s = b.Slots(2, 8, 2, 100, bits=4, sinks=3, recent=5, window=50, score_cap=20.0, decay=0.5, slopes=torch.zeros(8), device="cpu")
    t = copy.copy(s)
    assert t.address != s.address and all(getattr(t.c, f[0]) == getattr(s.c, f[0]) for f in b.rdkv_slots._fields_)
    t.k, old = torch.zeros_like(s.k), s.k
    assert s.k is old and s.c.k == old.data_ptr() and t.c.k == t.k.data_ptr()
    s.weight = None
    assert copy.copy(s).weight is None


def test_numbers_that_the_struct_cannot_hold_are_refused():
    """A cap that 32 bits make 0 would be no cap; half a slot is none."""
    for cap in (1e-50, -1e-50, 1e-46):
        with pytest.raises(ValueError, match="score_cap"):
            b.Slots(2, 8, 2, 100, score_cap=cap, device="cpu")
    for bad in (dict(capacity=100.5), dict(sinks=0.5), dict(window=1e3 + 0.25), dict(recent=float("nan"))):
        with pytest.raises(ValueError):
            b.Slots(**dict(dict(batch=2, hq=8, hkv=2, capacity=100, device="cpu"), **bad))
    s, rows = b.Slots(2, 8, 2, 100.0, device="cpu"), torch.zeros(2 * 2 * 5, 128, dtype=torch.bfloat16)
    assert s.capacity == 100
    for call in (lambda: b.rdkv_slots_fill(s, rows, rows, [5.5, 4.5]), lambda: b.rdkv_slots_fill(s, rows, rows, [5, 5], first=0.5), lambda: b.rdkv_slots_read(s, n=2.5)):
        with pytest.raises(ValueError, match="32-bit"):
            call()
