"""Slot caches on the GPU against tests/slots_plain.py, in 64 bits: filling, appending, the decode step, reading back, and all of
them together as a generation uses them."""
import math

import numpy as np
import pytest
import torch

from oracle import rdkv_oracle as O
from paper_2605_08317_amd import binding as b
from tests import slots_plain as P

pytestmark = pytest.mark.gpu
D = 128
BF, F32, I32 = torch.bfloat16, torch.float32, torch.int32


def cuda(x, dtype=None):
    return torch.as_tensor(x).to(device="cuda", dtype=dtype).contiguous()


def host(t):
    return t.detach().cpu().to(torch.float64 if t.is_floating_point() else t.dtype).numpy()


def rows_of(rng, n, big=False):
    x = rng.standard_normal((n, D))
    if big:
        x[:, rng.integers(0, D, 3)] *= 10
    return P.bf16(x)


def tiles_of(rows, side):
    """The bytes of 4-bit tiles [tiles, 5120] that hold float32 rows [n, 128]."""
    c, s, m = O.quantize_rows(np.asarray(rows, np.float32), 4)
    data, meta = O.pack_tiles64(c, s.view(np.uint16), m.view(np.uint16), 4, side)
    nt = (len(rows) + 63) // 64
    return np.concatenate([data.reshape(nt, 4096), meta.reshape(nt, 1024)], axis=1)


def loaded(rng, lens, hq, hkv, capacity, bits, garbage=True, gap=3, **kw):
    """A cache with lens[s] slots in use and its plain items.  garbage: what no token lies in holds NaN."""
    batch = len(lens)
    items = [P.Item(capacity, bits, kw.get("sinks", 0), kw.get("recent", 0)) for _ in range(batch * hkv)]
    if bits == 16:
        k = np.full((batch * hkv, capacity, D), np.nan if garbage else 0.0, np.float32)
    else:
        k = np.full((batch * hkv, (capacity + 63) // 64, 5120), 0xFF if garbage else 0, np.uint8)      # NaN scales
    v = k.copy()
    pos = np.full((batch * hkv, capacity), 12345, np.int32)
    weight = np.full((batch * hkv, capacity), np.nan if garbage else 0.0, np.float32)
    for i, it in enumerate(items):
        n = lens[i // hkv]
        it.n = n
        kr, vr = rows_of(rng, n, True), rows_of(rng, n)
        at = np.sort(rng.choice(max(1, gap * n), n, replace=False))
        it.next = int(at[-1]) + 1 if n else 0
        it.pos[:n] = at = rng.permutation(at)
        it.weight[:n] = rng.exponential(2.0, n).astype(np.float32)
        it.put(slice(0, n), kr, vr)
        pos[i, :n], weight[i, :n] = at, it.weight[:n]
        if n == 0:
            continue
        if bits == 16:
            k[i, :n], v[i, :n] = kr, vr
        else:
            for x, rows, side in ((k, kr, "k"), (v, vr, "v")):
                nt, fill = (n + 63) // 64, -n % 64
                x[i, :nt] = tiles_of(rows, side)
                if fill and garbage:              # the rows behind the last one: codes and scales that no call may let through
                    sc, of = O.tile64_meta_positions(side)
                    meta = x[i, nt - 1, 4096:].view(np.uint16)
                    meta[sc[64 - fill:].ravel()] = meta[of[64 - fill:].ravel()] = 0x7E00
    kind = BF if bits == 16 else torch.uint8
    shape = (batch, hkv) + k.shape[1:]
    lens_t = np.repeat(np.asarray(lens, np.int32), hkv).reshape(batch, hkv)
    nxt = np.array([it.next for it in items], np.int32).reshape(batch, hkv)
    s = b.Slots(batch, hq, hkv, capacity, bits=bits, k=cuda(k, kind).view(shape), v=cuda(v, kind).view(shape), pos=cuda(pos).view(batch, hkv, capacity),
                weight=cuda(weight).view(batch, hkv, capacity), lens=cuda(lens_t), next_pos=cuda(nxt), **kw)
    return s, items


def check_step(s, items, q, out, lse, weight, before, **kw):
    """One step's outputs against the plain items, which take it too."""
    g = s.hq // s.hkv
    qs, out, lse, weight = P.bf16(host(q)).astype(np.float64), host(out), host(lse), host(weight).reshape(-1, s.capacity)
    slopes = kw.pop("slopes", None)
    for i, it in enumerate(items):
        sl, h0 = i // s.hkv, (i % s.hkv) * g
        n = it.n
        o, l, p, off = it.decode(qs[sl, h0:h0 + g], slopes=None if slopes is None else slopes[h0:h0 + g], **kw)
        rel = (2 * off + P.sums_off(n) + 2.0 ** -20)[:, None]           # of a probability (exponentials and the quotient: 2^-21)
        assert np.all(np.abs(out[sl, h0:h0 + g] - o) <= rel * (p @ it.V_size[:n]) + 1e-30), (i, np.abs(out[sl, h0:h0 + g] - o).max())
        seen = np.isfinite(l)
        assert np.array_equal(np.isneginf(lse[sl, h0:h0 + g]), ~seen)
        assert np.all(np.abs(lse[sl, h0:h0 + g][seen] - l[seen]) <= off[seen] + P.sums_off(n) + 2.0 ** -22 * (1 + np.abs(l[seen])))
        assert np.all(np.abs(weight[i, :n] - it.weight[:n]) <= (rel * p).sum(0) + 2.0 ** -22 * np.abs(it.weight[:n]) + 1e-37), i
        assert np.array_equal(weight[i, n:], before.reshape(-1, s.capacity)[i, n:], equal_nan=True)     # slots without a token: as they were


CASES = [
    # lens, hq, hkv, capacity
    ([1], 1, 1, 1), ([0, 1, 2], 2, 2, 2), ([63, 64, 65], 4, 1, 65), ([0, 64, 7], 8, 2, 130), ([128, 100, 1], 8, 1, 128),
    ([1000, 17], 16, 4, 1000), ([300, 513, 1200], 8, 8, 1201), ([5000], 8, 1, 5000), ([4100, 1], 16, 8, 4200),
]


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("lens, hq, hkv, capacity", CASES)
def test_decode(lens, hq, hkv, capacity, bits):
    rng = np.random.default_rng(hash((tuple(lens), hq, hkv, capacity)) % 2 ** 32)
    s, items = loaded(rng, lens, hq, hkv, capacity, bits)
    q = cuda(rng.standard_normal((len(lens), hq, D)), BF)
    before = host(s.weight)
    out, lse = b.rdkv_slots_decode_attn(s, q)
    check_step(s, items, q, out, lse, s.weight, before)


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("cap, bias, window, sinks, decay", [
    (20.0, False, 0, 0, 1.0), (0.5, False, 0, 0, 0.5), (0.0, True, 0, 0, 1.0), (0.0, False, 50, 3, 1.0), (30.0, True, 200, 4, 0.9),
    (0.0, False, 1, 0, 0.0), (1e4, False, 0, 0, 1.0), (0.0, False, 10 ** 9, 0, 1.0)])
@pytest.mark.parametrize("lens, hq, hkv, capacity", [([700, 1, 0, 65], 8, 2, 700), ([1500], 8, 1, 1600), ([200, 130], 2, 2, 200)])
def test_decode_capped_biased_and_windowed(lens, hq, hkv, capacity, bits, cap, bias, window, sinks, decay):
    rng = np.random.default_rng(hash((tuple(lens), hq, int(cap), bias, window)) % 2 ** 32)
    slopes = 2.0 ** (-8.0 * (np.arange(hq) + 1) / hq) if bias else None
    s, items = loaded(rng, lens, hq, hkv, capacity, bits, sinks=sinks, window=window, score_cap=cap, decay=decay,
                      slopes=None if slopes is None else cuda(slopes, F32))
    q = cuda(2 * rng.standard_normal((len(lens), hq, D)), BF)
    before = host(s.weight)
    out, lse = b.rdkv_slots_decode_attn(s, q)
    # decay 0 of a NaN weight stays out of this test: slots in use hold numbers
    check_step(s, items, q, out, lse, s.weight, before, cap=cap, slopes=None if slopes is None else slopes.astype(np.float32).astype(np.float64),
               window=window, decay=float(np.float32(decay)))


@pytest.mark.parametrize("bits", [16, 4])
def test_a_step_that_sees_nothing(bits):
    """Every token is behind the window: zeros, -inf, and only the decay of the weights."""
    rng = np.random.default_rng(5)
    s, items = loaded(rng, [150, 64], 4, 2, 150, bits, window=7, decay=0.5)
    s.next_pos += 1000
    for it in items:
        it.next += 1000
    before = host(s.weight)
    q = cuda(rng.standard_normal((2, 4, D)), BF)
    out, lse = b.rdkv_slots_decode_attn(s, q)
    assert not out.any() and torch.isneginf(lse).all()
    check_step(s, items, q, out, lse, s.weight, before, window=7, decay=0.5)


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), 3.38e38])
def test_what_a_window_hides_has_no_say(bits, bad):
    """Rows that the window hides hold values that no sum survives."""
    rng = np.random.default_rng(6)
    s, items = loaded(rng, [333], 8, 2, 400, bits, window=60, sinks=2)
    out0, lse0 = b.rdkv_slots_decode_attn(s, q := cuda(rng.standard_normal((1, 8, D)), BF))
    away = s.next_pos.unsqueeze(-1) - 1 - s.pos
    hidden = (away >= 60) & (s.pos >= 2) & (torch.arange(400, device="cuda") < s.lens.unsqueeze(-1))
    assert hidden.any()
    if bits == 16:
        s.k[hidden] = bad
        s.v[hidden] = bad
    else:
        half = torch.tensor([bad if bad != 3.38e38 else 65504.0], dtype=torch.float16).view(torch.int16).item()
        for side, t in (("k", s.k), ("v", s.v)):
            sc, of = (torch.as_tensor(x) for x in O.tile64_meta_positions(side))
            meta = t.view(torch.int16)
            for _, h, i in hidden.nonzero().tolist():
                meta[0, h, i // 64, 2048 + torch.cat([sc[i % 64], of[i % 64]])] = half
    out, lse = b.rdkv_slots_decode_attn(s, q)
    assert torch.equal(out, out0) and torch.equal(lse, lse0)


def test_scores_that_are_no_numbers_stay_with_their_head():
    rng = np.random.default_rng(7)
    for bits in (16, 4):
        s, _ = loaded(rng, [200, 200], 8, 2, 200, bits)
        q = cuda(rng.standard_normal((2, 8, D)), BF)
        good, lse = b.rdkv_slots_decode_attn(s, q)
        q[0, 1, 5] = float("nan")
        out, lse1 = b.rdkv_slots_decode_attn(s, q)
        assert out[0, 1].isnan().all() and lse1[0, 1].isnan()
        keep = torch.ones(2, 8, dtype=torch.bool)
        keep[0, 1] = False
        assert torch.equal(out[keep], good[keep]) and torch.equal(lse1[keep], lse[keep])
        assert s.weight[0, 0].isnan().all() and not s.weight[0, 1].isnan().any() and not s.weight[1].isnan().any()


@pytest.mark.parametrize("scale_q, scale_k, scale_v", [(1e-3, 1.0, 1e-3), (8.0, 4.0, 900.0), (1.0, 1e-4, 1e-6), (1e-20, 1e18, 1e5), (100.0, 1e-2, 2e4), (1.0, 1.0, 8e3)])
@pytest.mark.parametrize("bits", [16, 4])
def test_magnitudes(bits, scale_q, scale_k, scale_v):
    """Values far from one keep their precision.  (4 bits hold what fp16 scales and offsets do: the plain items quantize the same.)"""
    if bits == 4 and scale_v > 1e4:
        pytest.skip("normal numbers times this are past fp16's largest, which 4-bit rows do not hold")
    if bits == 4:
        scale_k, scale_q = min(scale_k, 1e3), max(scale_q, 1e-6)
    rng = np.random.default_rng(8)
    s, items = loaded(rng, [130, 64], 8, 2, 192, bits, garbage=False)
    for i, it in enumerate(items):
        n, sl, h = it.n, i // 2, i % 2
        kr, vr = P.bf16(rows_of(rng, n, True) * scale_k), P.bf16(rows_of(rng, n) * scale_v)
        it.put(slice(0, n), kr, vr)
        for t, rows, side in ((s.k, kr, "k"), (s.v, vr, "v")):
            if bits == 16:
                t[sl, h, :n] = cuda(rows, BF)
            else:
                t[sl, h, :(n + 63) // 64] = cuda(tiles_of(rows, side))
    q = cuda(rng.standard_normal((2, 8, D)) * scale_q, BF)
    before = host(s.weight)
    out, lse = b.rdkv_slots_decode_attn(s, q)
    check_step(s, items, q, out, lse, s.weight, before)


def test_no_weights_kept():
    rng = np.random.default_rng(9)
    s, items = loaded(rng, [700, 64], 8, 2, 700, 16)
    t = b.Slots(2, 8, 2, 700, k=s.k, v=s.v, pos=s.pos, lens=s.lens, next_pos=s.next_pos, track=False)
    q = cuda(rng.standard_normal((2, 8, D)), BF)
    out, lse = b.rdkv_slots_decode_attn(s, q)
    out1, lse1 = b.rdkv_slots_decode_attn(t, q)
    assert torch.equal(out, out1) and torch.equal(lse, lse1)
    # a full item without weights gives up its oldest token
    slot = host(b.rdkv_slots_append(t, cuda(rng.standard_normal((2, 2, D)), BF), cuda(rng.standard_normal((2, 2, D)), BF)))
    for h in range(2):
        assert slot[0, h] == items[h].pos.argmin() and slot[1, h] == 64


def test_lengths_out_of_range_are_taken_for_the_nearest():
    rng = np.random.default_rng(10)
    for bits in (16, 4):
        s, _ = loaded(rng, [200, 200], 4, 1, 200, bits, garbage=False)
        q = cuda(rng.standard_normal((2, 4, D)), BF)
        want, _ = b.rdkv_slots_decode_attn(s, q)
        s.lens[0], s.lens[1] = 1 << 30, -7
        out, lse = b.rdkv_slots_decode_attn(s, q)
        assert torch.equal(out[0], want[0]) and not out[1].any() and torch.isneginf(lse[1]).all()


# ---- filling -----------------------------------------------------------------------------------------------------------------------

def ragged(rng, lens, hkv):
    K = [rows_of(rng, T, True) for T in lens for _ in range(hkv)]
    V = [rows_of(rng, T) for T in lens for _ in range(hkv)]
    return K, V


def cat(xs):
    return cuda(np.concatenate([x.reshape(-1) for x in xs]) if xs else np.zeros(0), BF)


def check_filled(s, items, first=0):
    n_of, nxt, pos, weight = host(s.lens).reshape(-1), host(s.next_pos).reshape(-1), host(s.pos).reshape(-1, s.capacity), host(s.weight).reshape(-1, s.capacity)
    K, V = (host(t).reshape(-1, s.capacity, D) for t in b.rdkv_slots_read(s))
    for i, it in enumerate(items):
        i += first * s.hkv
        n = it.n
        assert (n_of[i], nxt[i]) == (n, it.next), i
        assert np.array_equal(pos[i, :n], it.pos[:n]), i
        assert np.array_equal(weight[i, :n], it.weight[:n], equal_nan=True)
        for got, want in ((K, it.K), (V, it.V)):
            want = want[:n] if s.bits == 16 else P.bf16((want[:n]).astype(np.float32)).astype(np.float64)
            # 4 bits: scale x code rounded to fp32, the sum again, then bf16 once: 2^-8 of the value, and an fp32 step of the terms
            off = 0.0 if s.bits == 16 else 2.0 ** -8 * np.abs(want) + 2.0 ** -22 * np.abs(want).max(initial=0)
            assert np.all(np.abs(got[i, :n] - want) <= off), i
            assert not got[i, n:].any()


FILLS = [
    # prompts, hkv, capacity, sinks, recent, weights
    ([0, 1, 5], 2, 5, 1, 2, "any"), ([6, 5, 4], 1, 5, 1, 2, "any"), ([1, 2], 1, 1, 0, 0, "any"), ([100], 1, 64, 4, 60, "any"), ([300, 64, 65, 200], 3, 65, 4, 20, "any"),
    ([3000, 1023], 2, 1024, 0, 0, "any"), ([5000, 4097, 1], 2, 700, 4, 32, "ties"), ([2500], 2, 500, 0, 17, "equal"), ([2500], 2, 500, 3, 0, "nan"),
    ([2500, 900], 1, 500, 3, 9, "infinite"), ([20000], 1, 3000, 4, 100, "any"), ([70001], 1, 9999, 0, 0, "ties"), ([1500], 1, 200, 0, 200, "any"),
]


def weights_of(rng, n, how):
    w = np.exp(2 * rng.standard_normal(n)).astype(np.float32)
    if how == "ties":
        w = P.bf16(np.round(w, 1))
    if how == "equal":
        w[:] = 0.25
    if how == "nan":
        w = np.where(rng.random(n) < 0.9, np.nan, rng.standard_normal(n)).astype(np.float32)
    if how == "infinite":
        w = rng.choice(np.array([np.inf, -np.inf, 0.0, -0.0, 1.0, -1e-45, 1e-45, 3e38], np.float32), n)
    return w


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("prompts, hkv, capacity, sinks, recent, how", FILLS)
def test_fill(prompts, hkv, capacity, sinks, recent, how, bits):
    rng = np.random.default_rng(hash((tuple(prompts), hkv, capacity)) % 2 ** 32)
    K, V = ragged(rng, prompts, hkv)
    W = [weights_of(rng, len(k), how) for k in K]
    s = b.Slots(len(prompts), 2 * hkv, hkv, capacity, bits=bits, sinks=sinks, recent=recent)
    for t in (s.pos, s.lens, s.next_pos):
        t.fill_(77)
    s.weight.fill_(-5.0)
    s.k.fill_(3)
    items = [P.Item(capacity, bits, sinks, recent) for _ in K]
    for it, k, v, w in zip(items, K, V, W):
        it.fill(k, v, w)
    w_tok = cuda(np.concatenate(W), F32)
    b.rdkv_slots_fill(s, cat(K), cat(V), prompts, w_tok)
    check_filled(s, items)
    # what no token took is as it was
    free = torch.arange(capacity, device="cuda") >= s.lens.unsqueeze(-1)
    assert (s.pos[free] == 77).all() and (s.weight[free] == -5.0).all()
    if bits == 16:
        assert (s.k[free] == 3).all()
    else:                                   # codes, scales and offsets bit for bit
        for i, (it, k) in enumerate(zip(items, K)):
            nt = (it.n + 63) // 64
            got = s.k.view(-1, (capacity + 63) // 64, 5120)[i]
            if nt:
                assert np.array_equal(host(got[:nt]), tiles_of(k[it.pos[:it.n]], "k"))
                assert np.array_equal(host(s.v.view(-1, (capacity + 63) // 64, 5120)[i, :nt]), tiles_of(V[i][it.pos[:it.n]], "v"))
            assert (got[nt:] == 3).all()


@pytest.mark.parametrize("bits", [16, 4])
def test_fill_of_some_sequences_and_without_weights(bits):
    rng = np.random.default_rng(11)
    s = b.Slots(5, 4, 2, 100, bits=bits)
    K, V = ragged(rng, [50, 100, 100, 7, 99], 2)
    items = [P.Item(100, bits, 0, 0) for _ in K]
    for it, k, v in zip(items, K, V):
        it.fill(k, v, None)
    b.rdkv_slots_fill(s, cat(K), cat(V), [50, 100, 100, 7, 99])
    check_filled(s, items)
    K2, V2 = ragged(rng, [100, 3], 2)
    for it, k, v in zip(items[4:8], K2, V2):
        it.__init__(100, bits, 0, 0)
        it.fill(k, v, None)
    b.rdkv_slots_fill(s, cat(K2), cat(V2), [100, 3], first=2)
    check_filled(s, items)


def test_fill_of_many_sequences():
    """More of them than go with a launch."""
    rng = np.random.default_rng(12)
    prompts = [int(x) for x in rng.integers(0, 90, 150)]
    K, V = ragged(rng, prompts, 1)
    W = [weights_of(rng, len(k), "any") for k in K]
    s = b.Slots(150, 1, 1, 40, sinks=2, recent=5)
    items = [P.Item(40, 16, 2, 5) for _ in K]
    for it, k, v, w in zip(items, K, V, W):
        it.fill(k, v, w)
    b.rdkv_slots_fill(s, cat(K), cat(V), prompts, cuda(np.concatenate(W), F32))
    check_filled(s, items)


def test_fill_takes_values_that_four_bits_cannot_hold():
    """Rows beyond fp16's range: scales and offsets that are not finite, as rdkv_pack stores them."""
    rng = np.random.default_rng(13)
    K, V = ragged(rng, [70], 1)
    K[0][5, 3], V[0][66, 100], V[0][2, 7] = P.bf16(1e30), P.bf16(-7e4), np.inf
    s = b.Slots(1, 1, 1, 70, bits=4)
    b.rdkv_slots_fill(s, cat(K), cat(V), [70])
    with np.errstate(all="ignore"):
        want = tiles_of(K[0], "k"), tiles_of(V[0], "v")
    for t, w in ((s.k, want[0]), (s.v, want[1])):
        got = host(t)[0, 0]
        meta = got[:, 4096:].copy().view(np.float16)
        assert np.array_equal(meta, w[:, 4096:].copy().view(np.float16), equal_nan=True)


# ---- appending and reading -----------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("lens, hkv, capacity, sinks, recent, steps", [
    ([0, 1], 1, 2, 0, 0, 7), ([0, 60], 2, 66, 3, 10, 90), ([300, 300, 5], 1, 300, 0, 299, 12), ([130], 2, 130, 129, 1, 5), ([1000, 999], 2, 1000, 4, 32, 20), ([5000], 1, 5000, 0, 0, 9)])
def test_append(lens, hkv, capacity, sinks, recent, steps, bits):
    rng = np.random.default_rng(hash((tuple(lens), capacity)) % 2 ** 32)
    s, items = loaded(rng, lens, 2 * hkv, hkv, capacity, bits, garbage=False, sinks=sinks, recent=recent)
    for it in items:                                           # ties and NaN among the weights
        it.weight[:it.n:3] = 0.5
        it.weight[1:it.n:7] = np.nan if capacity == 1000 else 0.0
    s.weight.copy_(cuda(np.stack([it.weight for it in items]), F32).view_as(s.weight))
    for _ in range(steps):
        k, v = rows_of(rng, len(items)), rows_of(rng, len(items), True)
        want = [it.append(k[i], v[i]) for i, it in enumerate(items)]
        got = b.rdkv_slots_append(s, cuda(k, BF).view(len(lens), hkv, D), cuda(v, BF).view(len(lens), hkv, D))
        assert host(got).reshape(-1).tolist() == want
    check_filled(s, items)


@pytest.mark.parametrize("bits", [16, 4])
def test_read(bits):
    rng = np.random.default_rng(15)
    s, items = loaded(rng, [200, 63, 0], 2, 2, 200, bits)
    K, V = b.rdkv_slots_read(s)
    assert K.shape == (3, 2, 200, D)
    index = cuda(rng.integers(-3, 210, (3, 2, 77)), I32)
    index[0, 0, :4] = torch.tensor([5, 5, -1, 2 ** 31 - 1], device="cuda", dtype=I32)
    Ki, Vi = b.rdkv_slots_read(s, index)
    for got, whole in ((Ki, K), (Vi, V)):
        ok = (index >= 0) & (index < s.lens.unsqueeze(-1))
        want = whole.gather(2, index.clamp(0, 199).long().unsqueeze(-1).expand(-1, -1, -1, D))
        assert torch.equal(got, torch.where(ok.unsqueeze(-1), want, 0))
    K5, _ = b.rdkv_slots_read(s, n=5)
    assert torch.equal(K5, K[:, :, :5])
    K250, _ = b.rdkv_slots_read(s, n=250)                       # beyond the capacity: zeros
    assert torch.equal(K250[:, :, :200], K) and not K250[:, :, 200:].any()
    check_filled(s, items)


# ---- together -------------------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("bits", [16, 4])
def test_a_generation(bits):
    """Weights of the prompt, the slots filled by them, then tokens appended and attended to, the least attended evicted."""
    rng = np.random.default_rng(16)
    prompts, hq, hkv, capacity, sinks, recent = [900, 333, 2000], 8, 2, 400, 4, 16
    K, V = ragged(rng, prompts, hkv)
    q_obs = cuda(rng.standard_normal((3, hq, 32, D)), BF)
    cfg = b.Config(prompts, hq, hkv, **b.torch_allocator_hooks())
    w_tok, _ = b.rdkv_weights(cfg, cat(K), q_obs)
    s = b.Slots(3, hq, hkv, capacity, bits=bits, sinks=sinks, recent=recent, decay=0.97, score_cap=25.0)
    b.rdkv_slots_fill(s, cat(K), cat(V), prompts, w_tok)
    W = np.split(host(w_tok).astype(np.float32), np.cumsum([T for T in prompts for _ in range(hkv)])[:-1])
    items = [P.Item(capacity, bits, sinks, recent) for _ in K]
    for it, k, v, w in zip(items, K, V, W):
        it.fill(k, v, w)
    check_filled(s, items)
    for _ in range(100):
        k, v = rows_of(rng, len(items), True), rows_of(rng, len(items))
        slot = host(b.rdkv_slots_append(s, cuda(k, BF).view(3, hkv, D), cuda(v, BF).view(3, hkv, D))).reshape(-1)
        for i, it in enumerate(items):
            if it.n == it.capacity:        # the library's weights are fp32: its choice is one of the least, as far as they go
                may = (it.pos >= sinks) & (it.pos <= it.next - recent)
                assert may[slot[i]] and it.weight[slot[i]] <= it.weight[may].min() * (1 + 1e-4)
            else:
                assert slot[i] == it.n
            it.append(k[i], v[i], slot[i])
        q = cuda(rng.standard_normal((3, hq, D)), BF)
        before = host(s.weight)
        out, lse = b.rdkv_slots_decode_attn(s, q)
        check_step(s, items, q, out, lse, s.weight, before, cap=25.0, decay=float(np.float32(0.97)))
        for it, w in zip(items, host(s.weight).reshape(-1, capacity)):     # (the steps' roundings are not to add up)
            it.weight[:it.n] = w[:it.n]
    assert host(s.next_pos)[:, 0].tolist() == [T + 100 for T in prompts]


def clone(s, **kw):
    return b.Slots(s.batch, s.hq, s.hkv, s.capacity, bits=s.bits, sinks=s.c.sinks, recent=s.c.recent, k=s.k.clone(), v=s.v.clone(), pos=s.pos.clone(),
                   weight=s.weight.clone(), lens=s.lens.clone(), next_pos=s.next_pos.clone(), **kw)


@pytest.mark.parametrize("bits", [16, 4])
def test_captured_and_replayed(bits):
    """A recorded append and step go on from token to token, as eager calls do, with other work between the replays; two graphs of
    two caches, replayed in turn on two streams."""
    rng = np.random.default_rng(17)
    pairs = [loaded(rng, lens, 8, 2, cap, bits, garbage=False, sinks=2, recent=8)[0] for lens, cap in (([500, 90], 500), ([70, 2500], 2500))]
    runs = []
    for s in pairs:
        twin = clone(s)
        k, v, q = (torch.zeros((2, n, D), device="cuda", dtype=BF) for n in (2, 2, 8))
        out, lse, ws = torch.zeros((2, 8, D), device="cuda"), torch.zeros((2, 8), device="cuda"), s.workspace()
        slot = torch.zeros((2, 2), device="cuda", dtype=I32)
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            b.rdkv_slots_append(s, k, v, slot)
            b.rdkv_slots_decode_attn(s, q, out, lse, ws)
        runs.append((s, twin, k, v, q, out, lse, slot, (graph, ws), torch.cuda.Stream()))      # (a graph owns no workspace)
    for step in range(12):
        new = [[cuda(rng.standard_normal((2, n, D)), BF) for n in (2, 2, 8)] for _ in runs]
        torch.cuda.synchronize()
        for (s, twin, k, v, q, out, lse, slot, graph, stream), (k1, v1, q1) in zip(runs, new):
            with torch.cuda.stream(stream):
                k.copy_(k1), v.copy_(v1), q.copy_(q1)
                graph[0].replay()
        if step % 3 == 2:
            torch.cuda.synchronize()
        for (s, twin, k, v, q, out, lse, slot, graph, stream), (k1, v1, q1) in zip(runs, new):
            slot1 = b.rdkv_slots_append(twin, k1, v1)
            out1, lse1 = b.rdkv_slots_decode_attn(twin, q1)
            torch.cuda.synchronize()
            assert torch.equal(slot, slot1) and torch.equal(out, out1) and torch.equal(lse, lse1)
            assert torch.equal(s.weight, twin.weight) and torch.equal(s.pos, twin.pos) and torch.equal(s.next_pos, twin.next_pos)
            assert torch.equal(s.k.view(torch.uint8), twin.k.view(torch.uint8)) and torch.equal(s.v.view(torch.uint8), twin.v.view(torch.uint8))


@pytest.mark.parametrize("bits", [16, 4])
def test_a_captured_fill(bits):
    rng = np.random.default_rng(18)
    prompts = [900, 20]
    K, V = ragged(rng, prompts, 2)
    w = [weights_of(rng, len(k), "any") for k in K]
    Kd, Vd, wd = cat(K), cat(V), cuda(np.concatenate(w), F32)
    s = b.Slots(2, 2, 2, 300, bits=bits, sinks=4, recent=30)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        b.rdkv_slots_fill(s, Kd, Vd, prompts, wd)
    for seed in range(4):
        w = [weights_of(rng, len(k), "any") for k in K]
        wd.copy_(cuda(np.concatenate(w), F32))
        graph.replay()
        torch.cuda.synchronize()
        items = [P.Item(300, bits, 4, 30) for _ in K]
        for it, k, v, x in zip(items, K, V, w):
            it.fill(k, v, x)
        check_filled(s, items)


def test_steps_on_two_streams():
    """Two caches' steps side by side, each with a workspace of its own."""
    rng = np.random.default_rng(19)
    sides = []
    for bits in (16, 4):
        s, _ = loaded(rng, [3000, 2000], 8, 2, 3000, bits, garbage=False)
        q = cuda(rng.standard_normal((2, 8, D)), BF)
        twin = clone(s)
        want = [b.rdkv_slots_decode_attn(twin, q) for _ in range(30)][-1]
        sides.append((s, q, twin, want, torch.cuda.Stream()))
    torch.cuda.synchronize()
    got = [None, None]
    for _ in range(30):
        for i, (s, q, twin, want, stream) in enumerate(sides):
            with torch.cuda.stream(stream):
                got[i] = b.rdkv_slots_decode_attn(s, q)
    torch.cuda.synchronize()
    for (s, q, twin, want, stream), (out, lse) in zip(sides, got):
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1]) and torch.equal(s.weight, twin.weight)


def test_views_that_share_memory_with_others():
    """Tensors that are parts of larger ones, at offsets that are no multiple of a cache line: nothing beside them changes."""
    rng = np.random.default_rng(20)
    cap = 77
    lens = torch.zeros((3, 3), device="cuda", dtype=I32)
    whole = {"pos": torch.full((4, 2, cap), 9, device="cuda", dtype=I32), "weight": torch.full((4, 2, cap), 9.0, device="cuda"),
             "k": torch.full((4, 2, cap, D), 9.0, device="cuda", dtype=BF), "v": torch.full((4, 2, cap, D), 9.0, device="cuda", dtype=BF)}
    s = b.Slots(2, 4, 2, cap, sinks=1, recent=4, **{k: t[1:3] for k, t in whole.items()})
    K, V = ragged(rng, [100, 60], 2)
    w = [weights_of(rng, len(k), "any") for k in K]
    b.rdkv_slots_fill(s, cat(K), cat(V), [100, 60], cuda(np.concatenate(w), F32))
    k, v = cuda(rng.standard_normal((2, 2, D)), BF), cuda(rng.standard_normal((2, 2, D)), BF)
    for _ in range(20):
        b.rdkv_slots_append(s, k, v)
        b.rdkv_slots_decode_attn(s, cuda(rng.standard_normal((2, 4, D)), BF))
    for t in whole.values():
        assert (t[0] == 9).all() and (t[3] == 9).all()


# ---- many items, long items, few tokens in large caches --------------------------------------------------------------------------------
# What shape of launch a step takes follows from the cache's sizes, not from the tokens in it: large caches with few tokens go the ways of
# large ones.  Items shared out among workgroups, with empty ones between; items one each to a workgroup, in several turns; rows read past
# the caches (64 MiB on) or through them.

def some_lens(rng, batch, most):
    lens = rng.integers(0, 130, batch)
    lens[rng.integers(0, batch, batch // 4)] = 0
    lens[batch // 2], lens[-1] = most, most - 70
    lens[0] = 0
    return [int(x) for x in lens]


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("g, batch, hkv, capacity", [
    (1, 40, 2, 6000), (2, 85, 1, 5950), (4, 40, 2, 6000), (8, 80, 1, 6001), (1, 4, 1, 4000), (4, 4, 2, 3500), (2, 2, 1, 9000),       # shared out
    (1, 130, 2, 600), (4, 300, 1, 500), (8, 65, 4, 513), (2, 260, 1, 1700), (4, 260, 1, 1700)])                                     # one each
def test_decode_in_large_caches(g, batch, hkv, capacity, bits):
    rng = np.random.default_rng(21 + g + batch + capacity)
    lens = some_lens(rng, batch, capacity)
    s, items = loaded(rng, lens, g * hkv, hkv, capacity, bits, gap=2, window=3000, sinks=2, score_cap=40.0, decay=0.75)
    q = cuda(rng.standard_normal((batch, g * hkv, D)), BF)
    before = host(s.weight)
    out, lse = b.rdkv_slots_decode_attn(s, q)
    check_step(s, items, q, out, lse, s.weight, before, window=3000, cap=40.0, decay=0.75)
    t = b.Slots(batch, g * hkv, hkv, capacity, bits=bits, k=s.k, v=s.v, pos=s.pos, lens=s.lens, next_pos=s.next_pos, track=False, window=3000, sinks=2, score_cap=40.0)
    out1, lse1 = b.rdkv_slots_decode_attn(t, q)
    for it in items:
        it.weight[:] = 0
    zeros = np.zeros((batch * hkv, capacity))
    w = [it.decode(P.bf16(host(q)).astype(np.float64)[i // hkv, (i % hkv) * g:(i % hkv + 1) * g], window=3000, cap=40.0)[2].sum(0) for i, it in enumerate(items)]
    for i, p in enumerate(w):
        zeros[i, :len(p)] = p
        items[i].weight[:] = 0
    check_step(t, items, q, out1, lse1, torch.as_tensor(zeros), zeros, window=3000, cap=40.0)       # (the outputs; no weights are there)


@pytest.mark.parametrize("batch, bits, capacity", [(135, 4, 3600), (280, 4, 3600), (75, 16, 2600)])
def test_decode_of_items_that_share_workgroups(batch, bits, capacity):
    """More items than workgroups, and as many as leave some workgroups the end of one and the begin of the next."""
    rng = np.random.default_rng(batch)
    lens = [int(x) for x in np.where(rng.random(batch) < 0.3, 0, rng.integers(1, 260, batch))] if bits == 4 else [1500] * batch
    lens[0], lens[batch // 3], lens[-1] = 0, capacity, 0
    s, items = loaded(rng, lens, 32, 4, capacity, bits)
    q = cuda(rng.standard_normal((batch, 32, D)), BF)
    before = host(s.weight)
    out, lse = b.rdkv_slots_decode_attn(s, q)
    check_step(s, items, q, out, lse, s.weight, before)


def test_decode_of_thousands_of_items():
    """One step of 8240 items against steps of 412 of them.  Both add up the same fp32 scores' exponentials in another order: each is off by
    (2 x the scores' error + sums + 2^-20) of the largest value, as in check_step."""
    g = torch.Generator(device="cuda").manual_seed(26)
    batch, capacity, some = 2060, 2600, 150
    rand = lambda *shape: torch.randn(shape, device="cuda", generator=g)
    s = b.Slots(batch, 32, 4, capacity)
    s.k[:, :, :some], s.v[:, :, :some] = rand(batch, 4, some, D).to(BF), rand(batch, 4, some, D).to(BF)
    s.lens.copy_(torch.randint(0, some + 1, (batch, 4), device="cuda", generator=g, dtype=I32))
    s.lens[7, 2] = s.lens[2000, 3] = capacity
    s.lens[-1] = 0
    q = rand(batch, 32, D).to(BF)
    out, lse = b.rdkv_slots_decode_attn(s, q)
    weight = s.weight.clone()
    s.weight.zero_()
    # a score: 130 roundings of the sum of its terms' sizes, at most |q| |k| / sqrt d < 30
    off = 2.0 ** -24 * 138 * 30
    rel = 2 * (2 * off + P.sums_off(capacity) + 2.0 ** -20)
    for i in range(0, batch, 103):
        part = slice(i, i + 103)
        t = b.Slots(103, 32, 4, capacity, k=s.k[part], v=s.v[part], pos=s.pos[part], weight=s.weight[part], lens=s.lens[part], next_pos=s.next_pos[part])
        out1, lse1 = b.rdkv_slots_decode_attn(t, q[part])
        assert (out[part] - out1).abs().max() <= rel * s.v.abs().max()
        assert torch.equal(lse[part].isneginf(), lse1.isneginf())
        assert (lse[part] - lse1).nan_to_num().abs().max() <= rel
        assert ((weight[part] - s.weight[part]).abs() <= rel * s.weight[part] + 1e-30).all()


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("hq, batch, capacity", [(2, 1, 300), (8, 3, 9000), (16, 140, 3600)])
def test_empty_caches(hq, batch, capacity, bits):
    s = b.Slots(batch, hq, 2, capacity, bits=bits)
    s.weight.fill_(3.0)
    for _ in range(2):
        out, lse = torch.full((batch, hq, D), 7.0, device="cuda"), torch.zeros((batch, hq), device="cuda")
        b.rdkv_slots_decode_attn(s, torch.ones((batch, hq, D), device="cuda", dtype=BF), out, lse)
        assert not out.any() and torch.isneginf(lse).all() and (s.weight == 3).all()


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("capacity", [100, 9000])
def test_scores_near_the_lowest_number(capacity, bits):
    """A bias of -2.2e38 a position: alone it takes the probability, beside another token none; -3e38, past what a score holds, is not seen."""
    rng = np.random.default_rng(27)
    for slope, seen in ((2.2e38, True), (3.0e38, False)):
        s, items = loaded(rng, [1, 2], 4, 1, capacity, bits, slopes=torch.full((4,), slope, device="cuda"))
        s.pos[0, 0, 0] = 10
        s.next_pos[0] = 12                              # the token is one position back
        s.pos[1, 0, :2] = torch.tensor([11, 10], device="cuda", dtype=I32)
        s.next_pos[1] = 12
        before = s.weight.clone()
        out, lse = b.rdkv_slots_decode_attn(s, cuda(rng.standard_normal((2, 4, D)), BF))
        if seen:
            assert np.abs(host(out)[0] - items[0].V[0]).max() <= 2.0 ** -20 * items[0].V_size[0].max()
            assert ((lse[0] + 2.2e38).abs() <= 2.2e38 * 2.0 ** -22).all() and abs((s.weight - before)[0, 0, 0].item() - 4) <= 2.0 ** -20 * (4 + before[0, 0, 0].item())
        else:
            assert not out[0].any() and torch.isneginf(lse[0]).all()
        assert np.abs(host(out)[1] - items[1].V[0]).max() <= 2.0 ** -20 * items[1].V_size[0].max()
        assert torch.isfinite(lse[1]).all() and s.weight[1, 0, 1] == before[1, 0, 1]


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("hq, capacity", [(8, 300), (8, 4000), (2, 5000), (16, 4000)])
def test_scores_that_are_no_numbers_whichever_way_items_are_taken(hq, capacity, bits):
    rng = np.random.default_rng(22)
    s, _ = loaded(rng, [capacity, capacity - 50], hq, 2, capacity, bits)
    q = cuda(rng.standard_normal((2, hq, D)), BF)
    good, lse = b.rdkv_slots_decode_attn(s, q)
    for bad, head in ((float("nan"), 0), (float("inf"), hq // 2 - 1)):
        t = clone(s)
        qb = q.clone()
        qb[1, head, 77] = bad
        out, lse1 = b.rdkv_slots_decode_attn(t, qb)
        assert out[1, head].isnan().all() and lse1[1, head].isnan()
        keep = torch.ones(2, hq, dtype=torch.bool)
        keep[1, head] = False
        assert torch.equal(out[keep], good[keep]) and torch.equal(lse1[keep], lse[keep])
        n = capacity - 50
        assert t.weight[1, 0, :n].isnan().all() and not t.weight[1, 1, :n].isnan().any() and not t.weight[0].isnan().any()


LONG_FILLS = [
    # prompts, hkv, capacity, sinks, recent, weights
    ([8192], 1, 8191, 0, 0, "any"), ([8193], 2, 8192, 1, 1, "any"), ([12289, 300, 0, 9000], 2, 9500, 4, 64, "any"), ([20000, 15000], 1, 20000, 3, 5, "any"),
    ([300000], 1, 1000, 4, 32, "any"), ([270001, 4096, 1001], 1, 1000, 0, 900, "ties"), ([280000], 1, 5, 0, 0, "equal"), ([9000, 10000], 2, 500, 3, 9, "infinite"),
    ([30000], 1, 2000, 0, 17, "nan"), ([16384], 1, 4096, 4096 - 17, 17, "any"), ([33333], 1, 1, 0, 1, "any"), ([40000], 1, 39999, 10, 10, "ties"),
]


@pytest.mark.parametrize("prompts, hkv, capacity, sinks, recent, how", LONG_FILLS)
def test_fill_of_long_prompts(prompts, hkv, capacity, sinks, recent, how):
    rng = np.random.default_rng(hash((tuple(prompts), hkv, capacity)) % 2 ** 32)
    K, V = ragged(rng, prompts, hkv)
    W = [weights_of(rng, len(k), how) for k in K]
    for track in (True, False):
        s = b.Slots(len(prompts), hkv, hkv, capacity, sinks=sinks, recent=recent, track=track)
        items = [P.Item(capacity, 16, sinks, recent) for _ in K]
        for it, k, v, w in zip(items, K, V, W):
            it.fill(k, v, w)
        b.rdkv_slots_fill(s, cat(K), cat(V), prompts, cuda(np.concatenate(W), F32))
        if not track:
            s.weight = cuda(np.stack([it.weight for it in items]), F32).view(len(prompts), hkv, capacity)
        check_filled(s, items)


def test_fill_of_many_sequences_some_of_them_long():
    """Several launches' worth, the tables of each in the same workspace."""
    rng = np.random.default_rng(23)
    prompts = [int(x) for x in rng.integers(0, 400, 140)]
    prompts[3], prompts[70], prompts[100], prompts[139] = 9001, 30011, 8500, 13000
    K, V = ragged(rng, prompts, 1)
    W = [weights_of(rng, len(k), "any") for k in K]
    s = b.Slots(140, 1, 1, 120, bits=4, sinks=2, recent=5)
    items = [P.Item(120, 4, 2, 5) for _ in K]
    for it, k, v, w in zip(items, K, V, W):
        it.fill(k, v, w)
    b.rdkv_slots_fill(s, cat(K), cat(V), prompts, cuda(np.concatenate(W), F32))
    check_filled(s, items)


def test_a_captured_fill_of_a_long_prompt():
    rng = np.random.default_rng(24)
    prompts = [300, 21000]
    K, V = ragged(rng, prompts, 2)
    Kd, Vd, wd = cat(K), cat(V), cuda(np.zeros(2 * sum(prompts)), F32)
    s = b.Slots(2, 2, 2, 500, sinks=4, recent=30)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        b.rdkv_slots_fill(s, Kd, Vd, prompts, wd)
    for how in ("any", "ties", "nan", "any"):
        w = [weights_of(rng, len(k), how) for k in K]
        wd.copy_(cuda(np.concatenate(w), F32))
        graph.replay()
        torch.cuda.synchronize()
        items = [P.Item(500, 16, 4, 30) for _ in K]
        for it, k, v, x in zip(items, K, V, w):
            it.fill(k, v, x)
        check_filled(s, items)
        b.rdkv_slots_fill(s, Kd[:0], Vd[:0], [0, 0])            # between replays: an empty cache, by an eager call
        assert not s.lens.any()


@pytest.mark.parametrize("bits", [16, 4])
def test_past_four_gigabytes(bits):
    """Items whose rows lie further than 32 bits reach: appended to, attended to, read, and filled."""
    n = 17_000_003 if bits == 16 else 54_000_005
    s = b.Slots(1, 1, 1, n, bits=bits, sinks=3, recent=8)
    s.lens.fill_(n)
    s.next_pos.fill_(n)
    s.pos.view(-1).copy_(torch.arange(n, dtype=I32, device="cuda"))
    s.weight.fill_(1.0)
    gone = n - 1000
    s.weight[0, 0, gone] = 0.5
    rng = np.random.default_rng(25)
    k, v, q = (P.bf16(rng.standard_normal((1, 1, D))) for _ in range(3))
    k = P.bf16(q * 0.5)
    slot = b.rdkv_slots_append(s, cuda(k, BF), cuda(v, BF))
    assert slot.item() == gone and s.next_pos.item() == n + 1 and s.pos[0, 0, gone].item() == n
    out, lse = b.rdkv_slots_decode_attn(s, cuda(q, BF))
    # every other row is zeros: their scores are 0, their values nothing
    kh, vh, kt, vt = P.held(k[0], bits), P.held(v[0], bits), P.terms(k[0], bits), P.terms(v[0], bits, 8)
    x = (q[0].astype(np.float64) @ kh[0]).item() / math.sqrt(D)
    off = 2.0 ** -24 * 138 * (np.abs(q[0]).astype(np.float64) @ kt[0]).item() / math.sqrt(D)
    total = math.exp(x) + n - 1
    p = math.exp(x) / total
    # sums: shares of tiles in steps of four, each wavefront's at most n / 2000 slots of 64 lanes, then parts in turn
    rel = 2 * off + P.sums_off(n // 2000 + 2048) + 2.0 ** -20
    assert np.all(np.abs(host(out)[0, 0] - p * vh[0]) <= rel * p * vt[0] + 1e-30)
    assert abs(lse.item() - math.log(total)) <= rel + 2.0 ** -22 * math.log(total)
    w = s.weight[0, 0]
    assert abs(w[gone].item() - p) <= rel * p
    for at in (0, 1, n // 3, n - 1):
        assert abs(w[at].item() - (1 + 1 / total)) <= 2.0 ** -22
    K, V = b.rdkv_slots_read(s, torch.tensor([[[gone, 5, n - 1, n]]], device="cuda", dtype=I32))
    for got, want in ((K, kh), (V, vh)):
        assert np.all(np.abs(host(got)[0, 0, 0] - want[0]) <= 2.0 ** -8 * np.abs(want[0]) + 2.0 ** -22 * np.abs(want).max())
        assert not got[0, 0, 1:].any()
    if bits == 4:
        return
    rows = torch.zeros((n + 7, D), device="cuda", dtype=BF)
    mark = torch.arange(n + 7, device="cuda", dtype=torch.int64)
    for c in range(4):                                         # a row's number in its channels, 6 bits in each
        rows[:, c] = ((mark >> (6 * c)) & 63).to(BF)
    w_tok = torch.ones(n + 7, device="cuda")
    lost = torch.tensor([3, 4, 1000, n // 2, n - 900, n - 5, n - 2], device="cuda")
    w_tok[lost] = 0.25
    b.rdkv_slots_fill(s, rows, rows, [n + 7], w_tok)
    kept = torch.ones(n + 7, dtype=torch.bool, device="cuda")
    kept[lost] = False
    assert torch.equal(s.pos[0, 0].long(), mark[kept]) and s.lens.item() == n
    for c in range(4):
        assert torch.equal(s.k[0, 0, :, c], rows[:, c][kept]) and torch.equal(s.v[0, 0, :, c], rows[:, c][kept])


# ---- the calls from Python: native code and ctypes --------------------------------------------------------------------------------------

def test_native_code_and_ctypes_make_the_same_calls(monkeypatch):
    rng = np.random.default_rng(28)
    s, _ = loaded(rng, [300, 120], 8, 2, 300, 4, garbage=False)
    k, v, q = (cuda(rng.standard_normal((2, n, D)), BF) for n in (2, 2, 8))
    index = cuda(rng.integers(-2, 310, (2, 2, 9)), I32)

    prompts = [310, 9000]
    K, V, w = (cuda(rng.standard_normal(n), t) for n, t in ((2 * sum(prompts) * D, BF), (2 * sum(prompts) * D, BF), (2 * sum(prompts), F32)))

    def every(s):
        t = clone(s)
        assert b.rdkv_slots_fill(t, K, V.view(-1, D), prompts, w.view(2, -1)) is None
        b.rdkv_slots_fill(t, K[:2 * 310 * D], V[:2 * 310 * D], (310,), w[:620], first=1)
        b.rdkv_slots_fill(t, K[:0], V[:0], [0])
        filled = [t.k.clone(), t.v.clone(), t.pos.clone(), t.weight.clone(), t.lens.clone(), t.next_pos.clone()]
        made = [b.rdkv_slots_append(s, k, v), *b.rdkv_slots_decode_attn(s, q), *b.rdkv_slots_read(s, index), *b.rdkv_slots_read(s), *b.rdkv_slots_read(s, n=7)]
        given = [torch.zeros_like(t) for t in made[:5]]
        r = [b.rdkv_slots_append(s, k, v, given[0]), *b.rdkv_slots_decode_attn(s, q, given[1], given[2], s.workspace()), *b.rdkv_slots_read(s, index, 9, given[3], given[4])]
        assert all(x is y for x, y in zip(r, given))
        one = b.rdkv_slots_decode_attn(s, q, lse=given[2])
        assert isinstance(one, tuple) and one[1] is given[2]
        return filled + [t.clone() for t in made + given] + [one[0], s.weight.clone(), s.k.clone(), s.lens.clone(), s.next_pos.clone()]
    assert b._call is not None
    a = every(clone(s))
    monkeypatch.setattr(b, "_call", None)
    for x, y in zip(a, every(clone(s))):
        assert x.dtype == y.dtype and x.shape == y.shape and x.device == y.device and x.is_contiguous() and torch.equal(x, y)


@pytest.mark.parametrize("native", [True, False])
def test_the_binding_refuses_on_the_gpu_what_it_refuses_elsewhere(native, monkeypatch):
    if not native:
        monkeypatch.setattr(b, "_call", None)
    s = b.Slots(2, 8, 2, 100)
    new, q = torch.zeros((2, 2, D), device="cuda", dtype=BF), torch.zeros((2, 8, D), device="cuda", dtype=BF)
    wide = torch.zeros((2, 8, 2 * D), device="cuda", dtype=BF)[:, :, ::2]
    index = torch.zeros((2, 2, 3), device="cuda", dtype=I32)
    for call in (lambda: b.rdkv_slots_append(s, new.float(), new), lambda: b.rdkv_slots_append(s, new, new[:1]), lambda: b.rdkv_slots_append(s, new, new.cpu()),
                 lambda: b.rdkv_slots_append(s, new, new, torch.zeros((2, 2), device="cuda")), lambda: b.rdkv_slots_append(s, new, new, index),
                 lambda: b.rdkv_slots_decode_attn(s, wide), lambda: b.rdkv_slots_decode_attn(s, q.cpu()), lambda: b.rdkv_slots_decode_attn(s, q, q),
                 lambda: b.rdkv_slots_decode_attn(s, q, lse=torch.zeros((2, 7), device="cuda")), lambda: b.rdkv_slots_decode_attn(s, q, workspace=s.workspace().cpu()),
                 lambda: b.rdkv_slots_decode_attn(s, q, workspace=torch.zeros(4096, device="cuda")), lambda: b.rdkv_slots_read(s, index.long()),
                 lambda: b.rdkv_slots_read(s, index, 4), lambda: b.rdkv_slots_read(s, index[0]), lambda: b.rdkv_slots_read(s, n=2 ** 32),
                 lambda: b.rdkv_slots_read(s, index, K=new), lambda: b.rdkv_slots_fill(s, new, new, [3]), lambda: b.rdkv_slots_fill(s, q, q, [4, 4], new),
                 lambda: b.rdkv_slots_fill(s, q.cpu(), q, [4, 4]), lambda: b.rdkv_slots_fill(s, wide[:, :, :D], q, [4, 4]),
                 lambda: b.rdkv_slots_fill(s, q, q, [4, 2 ** 32 + 4]), lambda: b.rdkv_slots_fill(s, q, q, [4, 4], first=2 ** 32)):
        with pytest.raises((ValueError, RuntimeError)) as e:
            call()
        assert not isinstance(e.value, b.RdkvError)
    for call in (lambda: b.rdkv_slots_read(s, n=-1), lambda: b.rdkv_slots_fill(s, q, q, [4, 4], first=1), lambda: b.rdkv_slots_fill(s, q, q, [4, 4], first=-1),
                 lambda: b.rdkv_slots_fill(s, q, q, [8, -1]), lambda: b.rdkv_slots_fill(b.Slots(1, 8, 2, 7), q, q, [8]),
                 lambda: b.rdkv_slots_decode_attn(b.Slots(2, 8, 2, 9000), q, workspace=torch.zeros(64, device="cuda", dtype=torch.uint8))):
        with pytest.raises(b.RdkvError):
            call()
    assert not s.lens.any() and not s.next_pos.any()


def test_subclasses_take_the_way_that_asks_them():
    class Own(torch.Tensor):
        pass
    s = b.Slots(2, 8, 2, 100)
    new, q = torch.ones((2, 2, D), device="cuda", dtype=BF), torch.ones((2, 8, D), device="cuda", dtype=BF)
    slot = b.rdkv_slots_append(s, new.as_subclass(Own), new)
    assert not slot.any() and (s.lens == 1).all()
    out, lse = b.rdkv_slots_decode_attn(s, q.as_subclass(Own))
    assert torch.equal(out, torch.ones_like(out))
