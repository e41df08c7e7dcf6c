"""What rdkv_prompt_attn_bf16 refuses, without a GPU: nothing is launched for a bad argument."""
import ctypes
import os
import subprocess

import pytest
import torch

from paper_2605_08317_amd import binding as b

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INVALID, SHAPE = 1, 2


def struct(lens=(5, 7), **kw):
    c = b.rdkv_prompt()
    assert b.lib.rdkv_prompt_default(ctypes.byref(c)) == 0
    c.held = (ctypes.c_int32 * len(lens))(*lens) if lens is not None else None
    c.seq_lens = ctypes.cast(c.held, ctypes.POINTER(ctypes.c_int32)) if lens is not None else None
    for name, x in dict(dict(batch=len(lens or ()), hq=8, hkv=2), **kw).items():
        setattr(c, name, x)
    return c


def call(c, Q=16, K=16, V=16, out=16):
    return b.lib.rdkv_prompt_attn_bf16(ctypes.byref(c), Q, K, V, out, None, None)


@pytest.mark.parametrize("kw, status", [
    (dict(batch=-1), INVALID), (dict(hq=0), INVALID), (dict(hkv=0), INVALID), (dict(head_dim=64), SHAPE), (dict(hq=7), SHAPE), (dict(hq=6), SHAPE), (dict(hq=32), SHAPE),
    (dict(hq=65536, hkv=8192), SHAPE), (dict(window=-1), INVALID), (dict(sinks=-1), INVALID), (dict(score_cap=-1.0), INVALID), (dict(score_cap=float("nan")), INVALID),
    (dict(score_cap=float("inf")), INVALID), (dict(score_cap=1e-40), INVALID), (dict(lens=(5, -1)), SHAPE), (dict(lens=None, batch=1), INVALID),
    (dict(lens=(2 ** 28,)), SHAPE), (dict(lens=(2 ** 31 - 1,) * 64, hq=1, hkv=1), SHAPE), (dict(lens=(1023,) * 64, hq=32768, hkv=4096), SHAPE),
    (dict(q_stride=1000), SHAPE), (dict(q_stride=1028), SHAPE), (dict(k_stride=128), SHAPE), (dict(v_stride=2 ** 23 + 8), SHAPE), (dict(out_stride=-1024), SHAPE),
    (dict(k_stride=2 ** 40), SHAPE)])
def test_a_bad_struct_is_refused(kw, status):
    assert call(struct(**kw)) == status
    assert b.lib.rdkv_last_error()


def test_bad_pointers_are_refused():
    for kw in (dict(Q=None), dict(K=None), dict(V=None), dict(out=None), dict(Q=24), dict(K=8), dict(V=18), dict(out=17)):
        assert call(struct(), **kw) == INVALID
    assert b.lib.rdkv_prompt_attn_bf16(None, 16, 16, 16, 16, None, None) == INVALID
    assert b.lib.rdkv_prompt_default(None) == INVALID


def test_nothing_to_do_is_no_error():
    assert call(struct(lens=()), Q=None, K=None, V=None, out=None) == 0
    assert call(struct(lens=(0, 0, 0)), Q=None, K=None, V=None, out=None) == 0


def test_the_binding_refuses_tensors_the_library_would_misread():
    bf = torch.bfloat16
    q, k = torch.zeros(12, 8, 128, dtype=bf), torch.zeros(12, 2, 128, dtype=bf)
    lens = [5, 7]
    for bad in (dict(Q=q.float()), dict(Q=q[:11]), dict(Q=q.transpose(0, 1)), dict(Q=q.reshape(12, 1024)), dict(Q=q.view(-1)[:-1]), dict(K=k.repeat(1, 2, 1)[:, ::2]),
                dict(K=torch.zeros(12, 2, 256, dtype=bf)[..., ::2]), dict(V=k.view(-1)[::2]), dict(V=k.unsqueeze(0)), dict(out=q[:, :4]), dict(out=q.float()),
                dict(lse=torch.zeros(95)), dict(lse=torch.zeros(96, dtype=torch.float64)), dict(slopes=torch.zeros(2)), dict(score_cap=1e-50),
                dict(seq_lens=[5, 7.5]), dict(seq_lens=[5, 2 ** 32 + 7]), dict(window=2 ** 32), dict(hq=8.5)):
        with pytest.raises(ValueError):
            b.rdkv_prompt_attn_bf16(**dict(dict(Q=q, K=k, V=k, seq_lens=lens, hq=8, hkv=2), **bad))
    with pytest.raises(ValueError, match="cpu"):
        b.rdkv_prompt_attn_bf16(q, k, k, lens, 8, 2)


@pytest.mark.parametrize("side, heads", [("Q", 8), ("K", 2), ("V", 2), ("out", 8)])
def test_the_binding_refuses_rows_that_overlap(side, heads):
    """A view that is expanded over tokens has a row stride of 0, which the library takes for flat blocks: rows behind the view's memory.  So do rows that
    begin inside the one before, which are no layout of their own either; of one token the stride means nothing."""
    bf = torch.bfloat16
    q, k = torch.zeros(12, 8, 128, dtype=bf), torch.zeros(12, 2, 128, dtype=bf)
    good = dict(Q=q, K=k, V=k, seq_lens=[5, 7], hq=8, hkv=2)
    row = torch.zeros(heads * 128 + 12 * 8, dtype=bf)
    for bad in (row[:heads * 128].view(1, heads, 128).expand(12, heads, 128), row.as_strided((12, heads, 128), (8, 128, 1))):
        with pytest.raises(ValueError, match=side):
            b.rdkv_prompt_attn_bf16(**dict(good, **{side: bad}))
    one = dict(Q=q[:1], K=k[:1], V=k[:1], seq_lens=[1], hq=8, hkv=2)
    with pytest.raises(ValueError, match="cpu"):           # (it is where the tensors lie that is wrong)
        b.rdkv_prompt_attn_bf16(**dict(one, **{side: row.as_strided((1, heads, 128), (0, 128, 1))}))


def test_the_ctypes_struct_matches_the_c_header(tmp_path):
    fields = [f[0] for f in b.rdkv_prompt._fields_]
    src = tmp_path / "layout.c"
    src.write_text("\n".join(['#include <stdio.h>', '#include <stddef.h>', '#include "rdkv.h"', 'int main(void) {',
                              '  printf("%zu\\n", sizeof(rdkv_prompt));'] +
                             [f'  printf("%zu\\n", offsetof(rdkv_prompt, {f}));' for f in fields] + ['  return 0;', '}']))
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    out = [int(x) for x in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    assert out == [ctypes.sizeof(b.rdkv_prompt)] + [getattr(b.rdkv_prompt, f).offset for f in fields]
