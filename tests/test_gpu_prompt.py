"""Attention of whole prompts on the GPU against tests/prompt_plain.py, in 64 bits."""
import math

import numpy as np
import pytest
import torch

from paper_2605_08317_amd import binding as b
from tests import prompt_plain as P

pytestmark = pytest.mark.gpu
D = 128
BF, F32 = torch.bfloat16, torch.float32


def inputs(seed, lens, hq, hkv):
    """q, k, v bf16 on the host, [tokens, heads, 128]; K has channels that are larger."""
    gen = torch.Generator().manual_seed(seed)
    n = sum(lens)
    q, k, v = (torch.randn((n, h, D), generator=gen).to(BF) for h in (hq, hkv, hkv))
    k[..., torch.randperm(D, generator=gen)[:3]] *= 10
    return q, k, v


def laid(x, lens, heads, tokens):
    """On the GPU as a part of wider rows, or as flat blocks."""
    if not tokens:
        return P.rows_to(x, lens, heads).cuda()
    wide = torch.full((x.shape[0], heads + 3, D), math.nan, dtype=BF, device="cuda")
    wide[:, 1:1 + heads] = x.cuda()
    return wide[:, 1:1 + heads]


def check(out, lse, q, k, v, lens, hq, hkv, tokens, **kw):
    out, lse = out.float().cpu(), lse.cpu().double().numpy()
    slopes = kw.pop("slopes", None)
    g, at = hq // hkv, 0
    f64 = lambda t: t.double().numpy()
    for s, T in enumerate(lens):
        if T == 0:
            continue
        t0 = sum(lens[:s])
        for h in range(hkv):
            qs = f64(q[t0:t0 + T, h * g:h * g + g]).transpose(1, 0, 2)
            o, l, o_off, l_off = P.attend(qs, f64(k[t0:t0 + T, h]), f64(v[t0:t0 + T, h]), slopes=None if slopes is None else slopes[h * g:h * g + g], **kw)
            for i in range(g):
                got = f64(P.heads_of(out if tokens else out.view(-1, D), lens, hq, s, h * g + i, tokens))
                assert np.all(np.abs(got - o[i]) <= o_off[i]), (s, h, i, np.nanmax(np.abs(got - o[i]) / o_off[i]))
                row = lse[at + (h * g + i) * T:at + (h * g + i + 1) * T]
                assert np.all(np.abs(row - l[i]) <= l_off[i]), (s, h, i, np.abs(row - l[i]).max())
        at += hq * T


def run(seed, lens, hq, hkv, tokens=False, **kw):
    q, k, v = inputs(seed, lens, hq, hkv)
    slopes = kw.pop("slopes", None)
    out, lse = b.rdkv_prompt_attn_bf16(laid(q, lens, hq, tokens), laid(k, lens, hkv, tokens), laid(v, lens, hkv, tokens), lens, hq, hkv,
                                       window=kw.get("window", 0), sinks=kw.get("sinks", 0), score_cap=kw.get("cap", 0.0),
                                       slopes=None if slopes is None else torch.as_tensor(slopes, dtype=F32).cuda())
    assert out.shape == ((sum(lens), hq, D) if tokens else (sum(lens) * hq * D,)) and lse.shape == (sum(lens) * hq,)
    check(out, lse, q, k, v, lens, hq, hkv, tokens, slopes=slopes, **kw)


@pytest.mark.parametrize("lens, hq, hkv", [
    ([1], 1, 1), ([2], 8, 1), ([0, 1, 0, 3], 2, 2), ([31, 32, 33], 4, 1), ([63, 64, 65], 4, 2), ([127, 128, 129], 2, 1), ([255, 256, 257], 2, 2),
    ([300], 8, 2), ([513, 1, 100], 16, 2), ([1100], 8, 8)])
@pytest.mark.parametrize("tokens", [False, True])
def test_prompts(lens, hq, hkv, tokens):
    run(sum(lens) + hq, lens, hq, hkv, tokens)


@pytest.mark.parametrize("kw", [
    dict(window=1), dict(window=1, sinks=1), dict(window=5, sinks=3), dict(window=64), dict(window=65, sinks=64), dict(window=200, sinks=70), dict(window=10 ** 9),
    dict(cap=20.0), dict(cap=0.5), dict(cap=1e4), dict(slopes=True), dict(slopes=True, cap=30.0, window=100, sinks=4)], ids=str)
@pytest.mark.parametrize("lens, hq, hkv", [([700, 33], 8, 2), ([129, 1, 64], 8, 1)])
def test_windows_caps_and_biases(lens, hq, hkv, kw):
    kw = dict(kw)
    if kw.get("slopes"):
        kw["slopes"] = (2.0 ** (-8.0 * (np.arange(hq) + 1) / hq)).astype(np.float32).astype(np.float64)
    for tokens in (False, True):
        run(7, lens, hq, hkv, tokens, **kw)


@pytest.mark.parametrize("kw", [dict(cap=30.0, window=64), dict(cap=30.0, window=100, sinks=2), dict(cap=1.5, window=40), dict(cap=0.25, window=33, sinks=1),
                                dict(cap=50.0, window=400), dict(cap=1e30, window=100)], ids=str)
@pytest.mark.parametrize("lens, hq, hkv", [([700, 33], 8, 2), ([300] * 12, 8, 2), ([1500], 2, 1)])         # with shared tiles, without, and with
def test_caps_with_windows(lens, hq, hkv, kw):
    """Rows whose first tile is hidden from them as a whole, while scores are kept over the cap."""
    run(31, lens, hq, hkv, True, **kw)


@pytest.mark.parametrize("cap", [1e37, 9.9e37, 1.01e38, 2.3e38, 2.4e38, 3.4e38])
@pytest.mark.parametrize("kw", [dict(), dict(window=50), dict(window=50, sinks=2)], ids=str)
def test_caps_up_to_the_largest_number(cap, kw):
    """A cap far above the scores changes nothing.  Over the cap a product's factor is a number below fp32's normal ones, of 18 bits at least, and what it makes may
    be off by 2^-150, times the cap 2^-22: scores are off by 2^-17 of themselves and 2^-20 at most."""
    lens, hq, hkv = [300, 1, 70], 4, 2
    q, k, v = inputs(37, lens, hq, hkv)
    out, lse = b.rdkv_prompt_attn_bf16(q.cuda(), k.cuda(), v.cuda(), lens, hq, hkv, score_cap=cap, **kw)
    out, lse, at = out.double().cpu().numpy(), lse.double().cpu().numpy(), 0
    q, k, v = (x.double().numpy() for x in (q, k, v))
    for s, T in enumerate(lens):
        seq = slice(sum(lens[:s]), sum(lens[:s + 1]))
        for h in range(hq):
            o, l, o_off, l_off = P.attend(q[seq, h][None], k[seq, h // 2], v[seq, h // 2], **kw)
            most = 2.0 ** -17 * np.abs(q[seq, h] @ k[seq, h // 2].T).max() / math.sqrt(D) + 2.0 ** -20
            assert np.all(np.abs(out[seq, h] - o[0]) <= o_off[0] + 2 * most * np.abs(v[seq, h // 2]).max(0))
            assert np.all(np.abs(lse[at:at + T] - l[0]) <= l_off[0] + most)
            at += T


SLOPES = (2.0 ** (-8.0 * (np.arange(8) + 1) / 8)).astype(np.float32).astype(np.float64)


@pytest.mark.parametrize("kw", [{}, dict(window=150, sinks=2), dict(window=64), dict(cap=25.0), dict(slopes=SLOPES, cap=30.0, window=100, sinks=70)], ids=str)
def test_more_workgroups_than_compute_units(kw):
    """Fewer than that share their rows' tiles between wavefronts; here each has its rows to itself.  More than 64 sequences are several launches."""
    rng = np.random.default_rng(3)
    run(9, [int(x) for x in rng.integers(0, 400, 70)], 8, 2, True, **kw)


@pytest.mark.parametrize("kw", [{}, dict(window=700, sinks=100), dict(cap=25.0)], ids=str)
@pytest.mark.parametrize("hq, hkv", [(4, 2), (32, 4)])         # with shared tiles, and without
def test_longer_prompts(hq, hkv, kw):
    run(10, [1500, 33, 900], hq, hkv, False, **kw)


@pytest.mark.parametrize("hq, n", [(4, 1), (8, 70)])           # with shared tiles, and without
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_what_hidden_rows_hold_does_not_matter(hq, n, bad):
    """Rows of K and V that a token does not see may hold anything; a token that does see such a row has no finite outputs."""
    lens, hkv = [300] * n, 2
    q, k, v = inputs(11, lens, hq, hkv)
    at, head, kw = 130, 1, dict(window=40, sinks=3)
    clean = b.rdkv_prompt_attn_bf16(*(laid(x, lens, h, True) for x, h in ((q, hq), (k, hkv), (v, hkv))), lens, hq, hkv, **kw)
    for side in ("k", "v"):
        k2, v2 = k.clone(), v.clone()
        (k2 if side == "k" else v2)[at, head, 17] = bad
        out, lse = b.rdkv_prompt_attn_bf16(*(laid(x, lens, h, True) for x, h in ((q, hq), (k2, hkv), (v2, hkv))), lens, hq, hkv, **kw)
        g = hq // hkv
        sees = torch.zeros(sum(lens), hq, dtype=torch.bool)
        sees[at:at + 40, head * g:(head + 1) * g] = True
        # (numbers of a workgroup with such a row may be added up in another order)
        got, want = out.float().cpu(), clean[0].float().cpu()
        hidden = ~sees
        assert torch.all((got - want)[hidden].abs() <= 2 * P.HALF_BF16 * want[hidden].abs() + 2 * P.HALF_BF16 * 4)
        assert torch.isfinite(got[hidden]).all()
        if side == "v":
            assert not torch.isfinite(got[sees][:, 17]).any() and torch.isfinite(got[sees][:, :17]).all()
            if math.isnan(bad):
                assert torch.isnan(got[sees][:, 17]).all()
            else:
                assert torch.all(got[sees][:, 17] == bad)
        elif math.isnan(bad):
            assert torch.isnan(got[sees]).all()


def test_scores_that_are_not_numbers():
    """q k of +inf or NaN: the row is NaN; of -inf: the key takes no part; of -inf for all keys: zeros and -inf."""
    T = 70
    q, k, v = (torch.ones((T, 1, D), dtype=BF) for _ in range(3))
    k[5, 0, 0] = -math.inf
    v[5] = 100.0
    out, lse = b.rdkv_prompt_attn_bf16(q.cuda(), k.cuda(), v.cuda(), [T], 1, 1)
    assert torch.all((out[5:].float() - 1).abs() <= P.HALF_BF16) and torch.isfinite(lse).all()
    k[:] = -math.inf
    out, lse = b.rdkv_prompt_attn_bf16(q.cuda(), k.cuda(), v.cuda(), [T], 1, 1)
    assert torch.all(out == 0) and torch.all(lse == -math.inf)
    k[:] = 1.0
    k[40, 0, 3] = math.inf
    out, lse = b.rdkv_prompt_attn_bf16(q.cuda(), k.cuda(), v.cuda(), [T], 1, 1)
    assert torch.isnan(out[40:].float()).all() and torch.isnan(lse[40:]).all() and torch.isfinite(out[:40].float()).all() and torch.isfinite(lse[:40]).all()


@pytest.mark.parametrize("size", [1.0, 2.0 ** 12, 2.0 ** 22])
def test_a_large_number_common_to_all_scores_costs_nothing(size):
    """One channel gives every key the same large score; the others are small and exact beside it (multiples of the sum's last place), so that fp32
    sums are exact: what is left is the rounding of probabilities and outputs."""
    T, gen = 200, torch.Generator().manual_seed(5)
    q, k = torch.zeros((T, 2, D)), torch.zeros((T, 1, D))
    unit = max(size * size * 2.0 ** -20, 1.0)
    q[..., 0], k[..., 0] = size, size
    q[..., 1] = 1.0
    k[:, 0, 1] = torch.randint(0, 8, (T,), generator=gen).float() * unit
    v = torch.randn((T, 1, D), generator=gen).to(BF)
    out, lse = b.rdkv_prompt_attn_bf16(q.to(BF).cuda(), k.to(BF).cuda(), v.cuda(), [T], 2, 1)
    small = k[:, 0, 1].double() / math.sqrt(D)
    x = torch.where(torch.ones(T, T).tril() > 0, small, -math.inf)
    p = torch.softmax(x, -1)
    want, size_of = p @ v[:, 0].double(), p @ v[:, 0].double().abs()
    for h in range(2):
        got = out[:, h].double().cpu()
        # exponents of 2 are differences of exact products times a factor, rounded once: 2^-23 of up to 7 units x 0.1275
        assert torch.all((got - want).abs() <= (2 * P.HALF_BF16 + 2.0 ** -18 + 2.0 ** -22 * unit) * size_of + P.HALF_BF16 * want.abs())


@pytest.mark.parametrize("n", [1, 40])                         # with shared tiles, and without
@pytest.mark.parametrize("most", [0, 3, 4, 5, 6, 7])
@pytest.mark.parametrize("size", [2.0 ** 12, 2.0 ** 16, 2.0 ** 19, 2.0 ** 22, 2.0 ** 40, 2.0 ** 60])
def test_scores_of_any_size(size, most, n):
    """A number common to all scores, up to 2^120, and up to `most` units of its 20th bit for each key, so that fp32 products and sums are exact.  Exponents are
    the difference of a product times a factor and a number that the row's keys share, rounded once: off by 2^-24 of their own size, which with a reference
    that is rounded itself stays below 2^7 where it is not done again.  lse has a few roundings of its size."""
    T, hq, gen = 200, 2, torch.Generator().manual_seed(most)
    lens = [T] * n
    unit = size * size * 2.0 ** -20
    q, k = torch.zeros((n * T, hq, D)), torch.zeros((n * T, 1, D))
    q[..., 0], k[..., 0], q[..., 1] = size, size, 1.0
    k[:, 0, 1] = torch.randint(0, most + 1, (n * T,), generator=gen).float() * unit
    v = torch.randn((n * T, 1, D), generator=gen).to(BF)
    out, lse = b.rdkv_prompt_attn_bf16(q.to(BF).cuda(), k.to(BF).cuda(), v.cuda(), lens, hq, 1)
    out, lse = out.double().cpu(), lse.view(n, hq, T).double().cpu()
    for s in range(n):
        seq = slice(s * T, s * T + T)
        x = torch.where(torch.ones(T, T).tril() > 0, k[seq, 0, 1].double() / math.sqrt(D), -math.inf)
        p, rows = torch.softmax(x, -1), v[seq, 0].double()
        want, want_lse = p @ rows, torch.logsumexp(x, -1) + size * size / math.sqrt(D)
        for h in range(hq):
            assert torch.all((out[seq, h] - want).abs() <= (P.HALF_BF16 + 2.0 ** -16) * (p @ rows.abs()) + P.HALF_BF16 * want.abs() + 2.0 ** -16 * rows.abs().max()), (s, h)
            assert torch.all((lse[s, h] - want_lse).abs() <= 2.0 ** -22 * want_lse.abs() + 2.0 ** -16), (s, h)


def test_strides_past_32_bits():
    """Rows of 2^21 elements: bytes past 2^31 and, in K, past 2^32."""
    lens, hq, hkv = [1100, 30], 2, 1
    q, k, v = inputs(13, lens, hq, hkv)
    def wide(x, heads, row):
        t = torch.empty_strided((sum(lens), heads, D), (row, D, 1), dtype=BF, device="cuda")
        t.copy_(x.cuda())
        return t
    out = wide(torch.zeros((sum(lens), hq, D), dtype=BF), hq, 2 ** 20)
    got, lse = b.rdkv_prompt_attn_bf16(wide(q, hq, 2 ** 20), wide(k, hkv, 2 ** 21), wide(v, hkv, 2 ** 20 + 8), lens, hq, hkv, out=out)
    assert got is out
    check(out.contiguous(), lse, q, k, v, lens, hq, hkv, True)


def test_mixed_layouts_and_results_that_are_given():
    """Each tensor has a layout of its own; what lies around a strided result stays as it was."""
    lens, hq, hkv = [65, 3, 130], 8, 4
    q, k, v = inputs(17, lens, hq, hkv)
    wide = torch.full((sum(lens), hq + 2, D), 7.0, dtype=BF, device="cuda")
    lse = torch.zeros(sum(lens) * hq, device="cuda")
    out, got_lse = b.rdkv_prompt_attn_bf16(laid(q, lens, hq, False), laid(k, lens, hkv, True), laid(v, lens, hkv, False).view(-1, D), lens, hq, hkv, out=wide[:, 1:-1], lse=lse)
    assert got_lse is lse and torch.all(wide[:, 0] == 7) and torch.all(wide[:, -1] == 7)
    check(out, lse, q, k, v, lens, hq, hkv, True)


def test_in_a_graph_and_on_another_stream():
    lens, hq, hkv = [200, 64], 8, 2
    q, k, v = inputs(19, lens, hq, hkv)
    Q, K, V = (laid(x, lens, h, True) for x, h in ((q, hq), (k, hkv), (v, hkv)))
    want = b.rdkv_prompt_attn_bf16(Q, K, V, lens, hq, hkv)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        other = b.rdkv_prompt_attn_bf16(Q, K, V, lens, hq, hkv)
    torch.cuda.current_stream().wait_stream(stream)
    assert torch.equal(other[0], want[0]) and torch.equal(other[1], want[1])
    out, lse = torch.empty_like(want[0]), torch.empty_like(want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.rdkv_prompt_attn_bf16(Q, K, V, lens, hq, hkv, out=out, lse=lse)
    for step in range(3):
        Q.mul_(0.5)
        eager = b.rdkv_prompt_attn_bf16(Q, K, V, lens, hq, hkv)
        torch.cuda.synchronize()
        out.zero_()
        graph.replay()
        assert torch.equal(out, eager[0]) and torch.equal(lse, eager[1]), step


def test_the_same_twice():
    lens, hq, hkv = [900, 17], 16, 2
    x = [laid(t, lens, h, False) for t, h in zip(inputs(23, lens, hq, hkv), (hq, hkv, hkv))]
    first, again = (b.rdkv_prompt_attn_bf16(*x, lens, hq, hkv) for _ in range(2))
    assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


@pytest.mark.parametrize("native", [True, False])
def test_rows_that_overlap_are_refused(native, monkeypatch):
    """A view that is expanded over tokens has the row stride that names flat blocks; nothing is launched."""
    if not native:
        monkeypatch.setattr(b, "_call", None)
    lens, hq, hkv = [40, 24], 4, 2
    q, k, v = (x.cuda() for x in inputs(67, lens, hq, hkv))
    good = dict(Q=q, K=k, V=v, seq_lens=lens, hq=hq, hkv=hkv)
    for side, heads in (("Q", hq), ("K", hkv), ("V", hkv), ("out", hq)):
        row = torch.full((heads * D + 64 * 8,), 7.0, dtype=BF, device="cuda")
        for bad in (row[:heads * D].view(1, heads, D).expand(64, heads, D), row.as_strided((64, heads, D), (8, D, 1))):
            with pytest.raises(ValueError, match=side):
                b.rdkv_prompt_attn_bf16(**dict(good, **{side: bad}))
        assert torch.all(row == 7)
    one = [x[:1] for x in (q, k, v)]
    want = b.rdkv_prompt_attn_bf16(*one, [1], hq, hkv)
    got = b.rdkv_prompt_attn_bf16(*(x.as_strided(x.shape, (0, D, 1)) for x in one), [1], hq, hkv)      # (of one token the stride means nothing)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_native_calls_do_as_the_others(monkeypatch):
    """Layouts, results made and given, and refusals, through the native code and without it."""
    lens, hq, hkv = [70, 0, 33], 8, 2
    q, k, v = inputs(61, lens, hq, hkv)
    slopes, tokens = torch.rand(hq, device="cuda"), sum(lens)
    rows = [laid(x, lens, h, True) for x, h in ((q, hq), (k, hkv), (v, hkv))]
    flat = [laid(x, lens, h, False) for x, h in ((q, hq), (k, hkv), (v, hkv))]

    def every():
        made = [*b.rdkv_prompt_attn_bf16(*rows, lens, hq, hkv), *b.rdkv_prompt_attn_bf16(*flat, lens, hq, hkv, window=20, sinks=2, score_cap=9, slopes=slopes),
                *b.rdkv_prompt_attn_bf16(flat[0].view(-1, D), rows[1], flat[2], lens, hq, hkv, 128, score_cap=9.5)]
        assert [x.shape for x in made[::2]] == [(tokens, hq, D), (tokens * hq * D,), (tokens * hq, D)]
        out, lse = torch.full((tokens, hq + 1, D), 7.0, dtype=BF, device="cuda"), torch.zeros((hq, tokens), device="cuda")
        r = b.rdkv_prompt_attn_bf16(flat[0], rows[1], rows[2], tuple(lens), hq, hkv, out=out[:, 1:], lse=lse)
        assert r[1] is lse and torch.all(out[:, 0] == 7)
        empty = b.rdkv_prompt_attn_bf16(*(x[:0] for x in rows), [0, 0], hq, hkv)
        assert empty[0].shape == (0, hq, D) and empty[1].shape == (0,)
        for bad in (lambda: b.rdkv_prompt_attn_bf16(rows[0].float(), *rows[1:], lens, hq, hkv), lambda: b.rdkv_prompt_attn_bf16(*rows, lens, hq, hq),
                    lambda: b.rdkv_prompt_attn_bf16(*rows, [70, 33, 1], hq, hkv), lambda: b.rdkv_prompt_attn_bf16(rows[0], flat[1].cpu(), rows[2], lens, hq, hkv),
                    lambda: b.rdkv_prompt_attn_bf16(*rows, lens, hq, hkv, score_cap=1e-60), lambda: b.rdkv_prompt_attn_bf16(*rows, lens, hq, hkv, window=2.5),
                    lambda: b.rdkv_prompt_attn_bf16(*rows, lens, hq, hkv, slopes=slopes[:4]), lambda: b.rdkv_prompt_attn_bf16(*rows, lens, hq, hkv, out=rows[1]),
                    lambda: b.rdkv_prompt_attn_bf16(*rows, lens, hq, hkv, lse=lse.double()), lambda: b.rdkv_prompt_attn_bf16(*(x[:, ::2] for x in rows), lens, hq // 2, hkv // 2),
                    lambda: b.rdkv_prompt_attn_bf16(*rows, [70, 2 ** 32, 33], hq, hkv)):
            with pytest.raises(ValueError):
                bad()
        for bad in (lambda: b.rdkv_prompt_attn_bf16(*rows, lens, hq, hkv, window=-1), lambda: b.rdkv_prompt_attn_bf16(*rows, lens, hq, hkv, score_cap=-1.0),
                    lambda: b.rdkv_prompt_attn_bf16(*rows, lens, hq, hkv, score_cap=math.nan), lambda: b.rdkv_prompt_attn_bf16(*rows, [70, -1, 33], hq, hkv)):
            with pytest.raises(b.RdkvError):
                bad()
        return made + [out, lse]
    assert b._call is not None
    native = every()
    monkeypatch.setattr(b, "_call", None)
    for x, y in zip(native, every()):
        assert x.dtype == y.dtype and x.shape == y.shape
        same = torch.equal(x.view(torch.uint8), y.view(torch.uint8))
        assert same
