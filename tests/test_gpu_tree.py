"""Drafted trees over slot caches on the GPU against tests/tree_plain.py, in 64 bits: the attention of a tree, accepting a path of it, and both
with what comes before and after as a generation uses them."""
import math

import numpy as np
import pytest
import torch

from oracle import rdkv_oracle as O
from paper_2605_08317_amd import binding as b
from tests import prompt_plain, slots_plain as P, tree_plain as T
from tests.test_gpu_slots import cuda, host, loaded, rows_of

pytestmark = pytest.mark.gpu
D = 128
BF, F32, I32 = torch.bfloat16, torch.float32, torch.int32


def cached(rng, lens, hq, hkv, capacity, bits, **kw):
    s, items = loaded(rng, lens, hq, hkv, capacity, bits, **kw)
    for it in items:
        it.K_size4 = None
        if bits == 4:              # scale x (code + 16), 16 x scale and the offset: no smaller than these
            it.K_size4 = np.zeros((capacity, D))
    if bits == 4:
        tiles = s.k.cpu().numpy().reshape(len(items), -1, 5120)
        sc, of = O.tile64_meta_positions("k")
        for it, t in zip(items, tiles):
            meta = t[:, 4096:].copy().view(np.float16).astype(np.float64)
            scale = np.repeat(meta[:, sc].reshape(-1, 4), 32, axis=1)[:it.n]
            it.K_size4[:it.n] = np.abs(it.K[:it.n]) + 64 * np.abs(scale)
    return s, items


def tree(rng, n, kind="random"):
    if kind == "chain":
        return np.arange(n) - 1
    if kind == "star":
        return np.full(n, -1)
    return np.array([rng.integers(max(-1, i - 5), i) if i else -1 for i in range(n)])


def drafted(rng, batch, n, hq, hkv, big=1.0):
    q = cuda(big * rng.standard_normal((batch, n, hq, D)), BF)
    k, v = (cuda(np.stack([[rows_of(rng, hkv, side) for _ in range(n)] for _ in range(batch)]), BF) for side in (True, False))
    return q, k, v


def f64(t):
    return t.detach().cpu().double().numpy()


def check_tree(s, items, q, k, v, parent, counts, out, stats, **kw):
    g = s.hq // s.hkv
    q, k, v, out, stats = f64(q), f64(k), f64(v), f64(out), f64(stats)
    slopes = kw.pop("slopes", None)
    for i, it in enumerate(items):
        sq, h = i // s.hkv, i % s.hkv
        c = min(max(int(counts[sq]), 0), parent.shape[1])
        if c == 0:
            continue
        way, heads = T.ways(parent[sq], c), slice(h * g, h * g + g)
        o, M, S, o_off, M_off, S_off = T.attend(it, q[sq, :c, heads], k[sq, :c, h], v[sq, :c, h], way, sinks=s.c.sinks,
                                                slopes=None if slopes is None else slopes[heads], **kw)
        got, m, sm = out[sq, :c, heads], stats[sq, :c, heads, 0], stats[sq, :c, heads, 1]
        assert np.all(np.abs(got - o) <= o_off), (i, (np.abs(got - o) / o_off).max())
        seen = np.isfinite(M)
        assert np.array_equal(np.isneginf(m), ~seen) and np.all(sm[~seen] == 0)
        assert np.all(np.abs(m - M)[seen] <= M_off[seen]), (i, np.abs(m - M)[seen].max())
        assert np.all(np.abs(sm - S)[seen] <= ((S_off + M_off) * S)[seen]), (i, (np.abs(sm - S) / S)[seen].max())


def run(rng, lens, hq, hkv, capacity, bits, n, kind="random", counts=None, big=1.0, **kw):
    slopes = kw.pop("slopes", None)
    s, items = cached(rng, lens, hq, hkv, capacity, bits, sinks=kw.get("sinks", 0), window=kw.get("window", 0), score_cap=kw.get("cap", 0.0),
                      slopes=None if slopes is None else cuda(slopes, F32))
    kw.pop("sinks", None)
    batch = len(lens)
    q, k, v = drafted(rng, batch, n, hq, hkv, big)
    parent = np.stack([tree(rng, n, kind) for _ in range(batch)])
    counts_t = None if counts is None else cuda(np.asarray(counts), I32)
    before = [t.clone() for t in (s.k, s.v, s.pos, s.weight, s.lens, s.next_pos)]
    out, stats = torch.full_like(q, 7.0), torch.full((batch, n, hq, 2), 7.0, device="cuda")
    got = b.rdkv_slots_tree_attn(s, q, k, v, cuda(parent, I32), counts=counts_t, out=out, stats=stats)
    assert got[0] is out and got[1] is stats
    for x, y in zip(before, (s.k, s.v, s.pos, s.weight, s.lens, s.next_pos)):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
    counts = [n] * batch if counts is None else counts
    check_tree(s, items, q, k, v, parent, counts, out, stats, slopes=slopes, **kw)
    for sq, c in enumerate(counts):                        # rows behind the last: as they were
        assert torch.all(out[sq, max(c, 0):] == 7) and torch.all(stats[sq, max(c, 0):] == 7)
    return s, items


CASES = [
    # lens, hq, hkv, capacity, n
    ([0], 1, 1, 1, 1), ([1], 8, 1, 1, 1), ([0, 1, 2], 2, 2, 2, 3), ([63, 64, 65], 4, 1, 65, 8), ([0, 64, 7], 8, 2, 130, 9), ([128, 100, 1], 8, 1, 128, 5),
    ([1000, 17], 16, 4, 1000, 17), ([300, 513, 1200], 8, 8, 1201, 64), ([700], 8, 1, 720, 64), ([700, 30], 8, 2, 700, 33), ([4100, 1], 16, 8, 4200, 7),
    ([9000], 2, 1, 9000, 2)]


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("lens, hq, hkv, capacity, n", CASES)
def test_trees(lens, hq, hkv, capacity, n, bits):
    run(np.random.default_rng(sum(lens) + n), lens, hq, hkv, capacity, bits, n)


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("kind", ["chain", "star"])
def test_chains_and_stars(bits, kind):
    run(np.random.default_rng(2), [200, 70], 8, 2, 200, bits, 16, kind)
    run(np.random.default_rng(3), [130], 4, 1, 130, bits, 64, kind)


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("kw", [
    dict(cap=20.0), dict(cap=0.5), dict(slopes=True), dict(window=50, sinks=3), dict(window=1), dict(window=3, sinks=1), dict(window=10 ** 9),
    dict(cap=30.0, slopes=True, window=200, sinks=4)], ids=str)
@pytest.mark.parametrize("lens, hq, hkv, capacity, n", [([700, 1, 0, 65], 8, 2, 700, 12), ([1500], 8, 1, 1600, 3), ([200, 130], 2, 2, 200, 64)])
def test_caps_biases_and_windows(lens, hq, hkv, capacity, n, bits, kw):
    kw = dict(kw)
    if kw.get("slopes"):
        kw["slopes"] = (2.0 ** (-8.0 * (np.arange(hq) + 1) / hq)).astype(np.float32).astype(np.float64)
    for kind in ("random", "chain"):
        run(np.random.default_rng(5), lens, hq, hkv, capacity, bits, n, kind, big=2.0, **kw)


@pytest.mark.parametrize("bits", [16, 4])
def test_fewer_drafted_tokens_and_parents_that_are_none(bits):
    rng = np.random.default_rng(7)
    run(rng, [200, 64, 5, 100], 8, 2, 200, bits, 20, counts=[20, 1, 0, 13])
    lens, hq, hkv, n = [100, 40], 4, 2, 6
    s, items = cached(rng, lens, hq, hkv, 100, bits)
    q, k, v = drafted(rng, 2, n, hq, hkv)
    counts = np.array([99, -4])
    parent = np.array([[0, 5, -7, 2 ** 31 - 1, 1, -2 ** 31], [0, 0, 0, 0, 0, 0]])           # all but the fifth: the last cached token
    out, stats = torch.full_like(q, 7.0), torch.full((2, n, hq, 2), 7.0, device="cuda")
    b.rdkv_slots_tree_attn(s, q, k, v, cuda(parent, I32), counts=cuda(counts, I32), out=out, stats=stats)
    check_tree(s, items, q, k, v, parent, counts, out, stats)
    assert torch.all(out[1] == 7) and torch.all(stats[1] == 7)


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("n, hq", [(8, 4), (33, 8)])
def test_drafted_rows_that_are_hidden_may_hold_anything(bits, bad, n, hq):
    rng = np.random.default_rng(11)
    hkv = 2
    s, items = cached(rng, [90, 90], hq, hkv, 100, bits)
    q, k, v = drafted(rng, 2, n, hq, hkv)
    parent = np.stack([tree(rng, n), tree(rng, n)])
    counts = np.array([n, n - 3])
    who = 2
    k2, v2, q2 = k.clone(), v.clone(), q.clone()
    v2[0, who, :, 5] = bad
    for t in (k2, v2, q2):
        t[1, n - 3:] = bad                             # behind the last drafted token
    out, stats = torch.zeros_like(q), torch.zeros((2, n, hq, 2), device="cuda")
    b.rdkv_slots_tree_attn(s, q2, k2, v2, cuda(parent, I32), counts=cuda(counts, I32), out=out, stats=stats)
    assert torch.all(out[1, n - 3:] == 0)
    assert torch.isfinite(stats).all()
    sees = torch.tensor([who in w for w in T.ways(parent[0], n)])
    got = out[0].float().cpu()
    assert torch.isfinite(got[~sees]).all() and torch.isfinite(got[sees][:, :, :5]).all() and not torch.isfinite(got[sees][:, :, 5]).any()
    v2[0, who], out[0, sees.cuda()] = v[0, who], b.rdkv_slots_tree_attn(s, q, k, v, cuda(parent, I32))[0][0, sees.cuda()]
    check_tree(s, items, q, k, v, parent, counts, out, stats)


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("kw", [dict(), dict(score_cap=20.0, window=100, sinks=2)], ids=str)
@pytest.mark.parametrize("n, hq, counts", [(8, 8, [5, 8, 1]), (20, 8, [13, 1, 0]), (40, 8, [33, 17, 40]), (64, 8, [1, 50, 64])])
def test_what_is_behind_the_last_drafted_token_changes_no_bits(bits, kw, n, hq, counts):
    """Whatever rows from counts on hold, the others' numbers are the same to the bit: what is not finite there sends no one over the slots again, and no
    row's reference moves for a large score of theirs."""
    rng = np.random.default_rng(79)
    s, _ = cached(rng, [700, 130, 65], hq, 1, 720, bits, **kw)
    q, k, v = drafted(rng, 3, n, hq, 1)
    parent = cuda(np.stack([tree(rng, n) for _ in range(3)]), I32)
    got = []
    for fill in (0.0, math.nan, math.inf, -math.inf, 1e4, 3e38):
        q2, k2, v2 = q.clone(), k.clone(), v.clone()
        for t in (q2, k2, v2):
            for sq, c in enumerate(counts):
                t[sq, c:] = fill * t[sq, c:].sign() if math.isfinite(fill) else fill
        out, stats = torch.full_like(q, 7.0), torch.full((3, n, hq, 2), 7.0, device="cuda")
        b.rdkv_slots_tree_attn(s, q2, k2, v2, parent, counts=cuda(counts, I32), out=out, stats=stats)
        got.append((out, stats))
    assert torch.isfinite(got[0][0].float()).all()
    for out, stats in got[1:]:
        assert torch.equal(out, got[0][0]) and torch.equal(stats, got[0][1])


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("n, hq", [(6, 4), (40, 8)])
def test_slots_behind_a_window_may_hold_anything(bits, n, hq):
    """Some tokens of the tree see a slot, and those further along do not."""
    rng = np.random.default_rng(13)
    s, items = cached(rng, [150], hq, 2, 160, bits, window=60, sinks=2, gap=1)
    q, k, v = drafted(rng, 1, n, hq, 2)
    parent = tree(rng, n, "chain")[None]
    want = b.rdkv_slots_tree_attn(s, q, k, v, cuda(parent, I32))
    nxt = items[0].next
    edge = nxt + 2 - 60                                # seen by tokens 0, 1 and 2 (positions next .. next + 2), but for the first
    for it in range(2):
        slot = int(np.nonzero(items[it].pos[:150] == edge + 1)[0][0])
        if bits == 16:
            s.v[0, it, slot, 9] = math.inf
            s.k[0, it, int(np.nonzero(items[it].pos[:150] == 20)[0][0])] = math.nan          # seen by none
            s.v[0, it, int(np.nonzero(items[it].pos[:150] == 20)[0][0])] = math.nan
        else:
            sc, of = O.tile64_meta_positions("v")
            s.v[0, it].view(-1, 5120)[slot // 64, 4096:].view(torch.float16)[int(of[slot % 64].ravel()[0])] = math.inf
    out, stats = b.rdkv_slots_tree_attn(s, q, k, v, cuda(parent, I32))
    assert torch.equal(stats, want[1])
    depth = np.arange(n)
    sees = torch.tensor(nxt + depth - (edge + 1) < 60)
    assert 0 < int(sees.sum()) < n
    got, ref = out[0].float().cpu(), want[0][0].float().cpu()
    assert torch.isfinite(got[~sees]).all() and (got[~sees] - ref[~sees]).abs().max() <= 2 * T.HALF_BF16 * 8
    assert torch.all(got[sees][:, :, 9] == math.inf) and torch.isfinite(got[sees][:, :, 64:]).all()


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("n, hq", [(6, 4), (20, 8), (40, 8)])
def test_an_infinite_value_that_is_seen(bits, n, hq):
    """The last slot's, in a tile that ends there: infinite in its channel, and nothing else changes."""
    rng = np.random.default_rng(14)
    s, items = cached(rng, [150], hq, 2, 160, bits)
    q, k, v = drafted(rng, 1, n, hq, 2)
    parent = cuda(tree(rng, n)[None], I32)
    want, stats = b.rdkv_slots_tree_attn(s, q, k, v, parent)
    for it in range(2):
        if bits == 16:
            s.v[0, it, 149, 9] = math.inf
        else:
            sc, of = O.tile64_meta_positions("v")
            s.v[0, it].view(-1, 5120)[149 // 64, 4096:].view(torch.float16)[int(of[149 % 64].ravel()[0])] = math.inf
    got, same = b.rdkv_slots_tree_attn(s, q, k, v, parent)
    assert torch.equal(same, stats)
    at = torch.zeros(D, dtype=torch.bool, device="cuda")
    at[9 if bits == 16 else slice(0, 32)] = True           # (a group of 32 channels has one offset)
    assert torch.all(got[..., at] == math.inf)
    assert (got[..., ~at].float() - want[..., ~at].float()).abs().max() <= 2 * T.HALF_BF16 * 8


@pytest.mark.parametrize("bits", [16, 4])
def test_a_tree_that_sees_nothing(bits):
    """No slot, and scores of -inf for the token itself."""
    s, _ = cached(np.random.default_rng(17), [0], 4, 2, 10, bits)
    q, k, v = drafted(np.random.default_rng(1), 1, 3, 4, 2)
    q[:] = 1.0
    k[:] = 1.0
    k[..., 0] = -math.inf
    out, stats = b.rdkv_slots_tree_attn(s, q, k, v, cuda([[-1, 0, 1]], I32))
    assert torch.all(out == 0) and torch.all(stats[..., 0] == -math.inf) and torch.all(stats[..., 1] == 0)


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("size", [2.0 ** -40, 2.0 ** -6, 2.0 ** 6, 2.0 ** 12])
def test_queries_of_any_size(bits, size):
    run(np.random.default_rng(19), [130, 70], 4, 1, 130, bits, 5, big=size)


def tiny(rng, shape, size):
    """Queries of a few sizes beside each other and zeros, all of them exact and no value between 0 and 2^-126."""
    return cuda(size * rng.choice([-2.0, -1.5, -1.0, 0.0, 0.0, 1.0, 1.5, 2.0], shape), BF)


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("size", [2.0 ** -112, 2.0 ** -119, 2.0 ** -121, 2.0 ** -126])
@pytest.mark.parametrize("kw", [dict(), dict(cap=20.0, window=100, sinks=2)], ids=str)
def test_queries_of_the_smallest_sizes(bits, size, kw):
    """Down to the smallest normal number, with zeros among them, beside a row of zeros and rows of ordinary size: scores are 0 or next to it, and a tree
    and what is accepted of it are an even share."""
    rng, lens, hq, hkv, n = np.random.default_rng(71), [130, 70], 4, 1, 5
    s, items = cached(rng, lens, hq, hkv, 140, bits, window=kw.get("window", 0), sinks=kw.get("sinks", 0), score_cap=kw.get("cap", 0.0))
    q, k, v = drafted(rng, 2, n, hq, hkv)
    q[:, :3] = tiny(rng, (2, 3, hq, D), size)
    q[0, 0, 1] = 0
    parent = np.stack([tree(rng, n, "chain")] * 2)
    out, stats = b.rdkv_slots_tree_attn(s, q, k, v, cuda(parent, I32))
    assert torch.isfinite(out.float()).all() and torch.isfinite(stats).all()
    plain = {x: kw[x] for x in ("window", "cap") if x in kw}
    for i, it in enumerate(items):
        o, M, S, o_off, M_off, S_off = T.attend(it, f64(q)[i], f64(k)[i, :, 0], f64(v)[i, :, 0], T.ways(parent[i], n), sinks=s.c.sinks, **plain)
        assert np.all(np.abs(f64(out)[i] - o) <= o_off)
        # products, their sums and scores below 2^-126 may be taken for 0: less than 300 of them
        assert np.all(np.abs(f64(stats)[i, ..., 0] - M) <= M_off + 300 * 2.0 ** -126)
        assert np.all(np.abs(f64(stats)[i, ..., 1] - S) <= (S_off + M_off) * S)
    paths = [[0, 1, 2, 3, 4], [0, 1, -1, -1, -1]]
    slot = b.rdkv_slots_accept(s, q, k, v, cuda(paths, I32), stats)
    check_accept(s, items, q, k, v, paths, stats, slot, **plain)


@pytest.mark.parametrize("bits", [16, 4])
def test_queries_of_the_largest_size_against_keys_of_zero(bits):
    """Scores of 0 whatever the queries are: the mean of the values that are seen."""
    rng = np.random.default_rng(73)
    s, items = cached(rng, [130], 4, 1, 140, bits)
    q, k, v = drafted(rng, 1, 5, 4, 1)
    s.k.zero_(), k.zero_()
    for it in items:
        it.K[:] = 0
        it.K_size4 = np.zeros((140, D))
    q[0, 1:3] = tiny(rng, (2, 4, D), 2.0 ** 126)
    q[0, 3] = 0
    parent = tree(rng, 5, "chain")[None]
    out, stats = b.rdkv_slots_tree_attn(s, q, k, v, cuda(parent, I32))
    check_tree(s, items, q, k, v, parent, [5], out, stats)


def test_the_size_of_queries_against_keys_is_nothing():
    """Queries times a power of two, keys over it: the same bits."""
    rng = np.random.default_rng(20)
    s, items = cached(rng, [130], 4, 1, 130, 16)
    q, k, v = drafted(rng, 1, 5, 4, 1)
    parent = cuda(tree(rng, 5)[None], I32)
    want = b.rdkv_slots_tree_attn(s, q, k, v, parent)
    held = s.k.clone()
    for size in (2.0 ** -20, 2.0 ** 40):
        s.k.copy_((held.double() / size).to(BF))
        got = b.rdkv_slots_tree_attn(s, q * size, (k.double() / size).to(BF), v, parent)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


# ---- accepting ---------------------------------------------------------------------------------------------------------------------

def check_accept(s, items, q, k, v, paths, stats, slot, tracked=True, decay=1.0, slopes=None, **kw):
    """The plain items take the tokens as well; the library's slots are followed where they are least by its weights."""
    g, n = s.hq // s.hkv, q.shape[1]
    q, k, v, stats, slot = f64(q), f64(k), f64(v), f64(stats), slot.cpu().numpy()
    decay = float(np.float32(decay))
    pos, weight = s.pos.cpu().numpy().reshape(len(items), -1), f64(s.weight).reshape(len(items), -1) if tracked else None
    for i, it in enumerate(items):
        sq, h = i // s.hkv, i % s.hkv
        path = []
        for t in paths[sq]:
            if not 0 <= t < n:
                break
            path.append(int(t))
        c, used = len(path), it.n
        off = np.zeros(it.capacity)
        if tracked and c:
            p, p_off = T.given(it, q[sq, path, h * g:h * g + g], k[sq, path, h], stats[sq, path, h * g:h * g + g], decay, sinks=s.c.sinks,
                               slopes=None if slopes is None else slopes[h * g:h * g + g], **kw)
            it.weight[:used] = decay ** c * it.weight[:used] + p[:used]
            off[:used] = p_off[:used] + 2.0 ** -22 * c * np.abs(it.weight[:used])
        for j, t in enumerate(path):
            want = it.n
            if it.n == it.capacity:
                may = np.nonzero((it.pos >= s.c.sinks) & (it.pos <= it.next - s.c.recent))[0]
                if tracked:
                    assert slot[sq, h, j] in may
                    mine = slot[sq, h, j]
                    assert it.weight[mine] - off[mine] <= (it.weight[may] + off[may]).min()
                    want = mine
                else:
                    want = may[np.argmin(it.pos[may])]
            assert slot[sq, h, j] == want
            it.append(k[sq, t, h].astype(np.float32), v[sq, t, h].astype(np.float32), slot=want)
            if tracked:
                it.weight[want], off[want] = p[used + j], p_off[used + j] + 1e-37
        assert np.all(slot[sq, h, c:] == -1)
        assert np.array_equal(pos[i, :it.n], it.pos[:it.n])
        if tracked:
            assert np.all(np.abs(weight[i, :it.n] - it.weight[:it.n]) <= off[:it.n] + 1e-37), (i, np.abs(weight[i, :it.n] - it.weight[:it.n]).max())
    lens, nxt = s.lens.cpu().numpy().ravel(), s.next_pos.cpu().numpy().ravel()
    assert np.array_equal(lens, [it.n for it in items]) and np.array_equal(nxt, [it.next for it in items])
    K, V = b.rdkv_slots_read(s)
    K, V = f64(K).reshape(len(items), -1, D), f64(V).reshape(len(items), -1, D)
    for i, it in enumerate(items):
        for got, want in ((K, it.K), (V, it.V)):
            assert np.all(np.abs(got[i, :it.n] - want[:it.n]) <= T.HALF_BF16 * np.abs(want[:it.n]))


def accept(rng, lens, hq, hkv, capacity, bits, n, paths, kind="chain", tracked=True, decay=1.0, sinks=0, recent=0, **kw):
    slopes = kw.pop("slopes", None)
    s, items = cached(rng, lens, hq, hkv, capacity, bits, sinks=sinks, recent=recent, window=kw.get("window", 0), score_cap=kw.get("cap", 0.0), decay=decay,
                      slopes=None if slopes is None else cuda(slopes, F32))
    if not tracked:
        s.weight = None
    batch = len(lens)
    q, k, v = drafted(rng, batch, n, hq, hkv)
    parent = np.stack([tree(rng, n, kind) for _ in range(batch)])
    _, stats = b.rdkv_slots_tree_attn(s, q, k, v, cuda(parent, I32))
    paths = [(list(p) + [-1] * max(map(len, paths)))[:max(map(len, paths))] for p in paths]
    slot = b.rdkv_slots_accept(s, q if tracked else None, k, v, cuda(paths, I32), stats if tracked else None)
    check_accept(s, items, q, k, v, paths, stats, slot, tracked, decay, slopes, **kw)
    return s, items


PATHS = [
    # lens, hq, hkv, capacity, n, paths
    ([0], 1, 1, 1, 1, [[0]]), ([1], 8, 1, 1, 1, [[0]]), ([0, 1, 2], 2, 2, 2, 3, [[0, 1, 2], [0], []]), ([63, 64, 65], 4, 1, 66, 8, [range(8), range(3), [0]]),
    ([128, 100, 1], 8, 1, 128, 64, [range(64), range(40), range(64)]), ([1000, 17], 16, 4, 1000, 17, [range(5), range(17)]),
    ([4100, 1], 16, 8, 4200, 7, [range(7), [0, 1]]), ([4200, 4199], 8, 2, 4200, 9, [range(9), range(9)])]


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("tracked", [True, False])
@pytest.mark.parametrize("lens, hq, hkv, capacity, n, paths", PATHS)
def test_accepting(lens, hq, hkv, capacity, n, paths, bits, tracked):
    accept(np.random.default_rng(sum(lens) + n), lens, hq, hkv, capacity, bits, n, paths, tracked=tracked)


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("kw", [
    dict(decay=0.9), dict(decay=0.0), dict(cap=20.0), dict(slopes=True, decay=0.5), dict(window=50, sinks=3), dict(window=2), dict(sinks=4, recent=60), dict(recent=2),
    dict(cap=30.0, slopes=True, window=100, sinks=4, recent=3, decay=0.97)], ids=str)
def test_accepting_with_all_that_a_cache_has(bits, kw):
    kw = dict(kw)
    hq, hkv = 8, 2
    if kw.get("slopes"):
        kw["slopes"] = (2.0 ** (-8.0 * (np.arange(hq) + 1) / hq)).astype(np.float32).astype(np.float64)
    accept(np.random.default_rng(23), [200, 190, 65], hq, hkv, 200, bits, 16, [range(16), range(12), range(1)], **kw)


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("kw", [dict(), dict(recent=200, sinks=4, decay=0.99), dict(recent=100, tracked=False)], ids=str)
def test_long_paths_into_long_caches(bits, kw):
    """More segments than a workgroup has threads, and tokens that become old enough on the way in many of them."""
    accept(np.random.default_rng(33), [33100, 500], 1, 1, 33100, bits, 64, [range(64), range(30)], **kw)


@pytest.mark.parametrize("bits", [16, 4])
def test_paths_that_end_and_paths_that_repeat(bits):
    """A path ends at the first index that is none; one that names a token twice takes it in twice."""
    rng = np.random.default_rng(29)
    accept(rng, [40, 40, 38, 40], 4, 2, 40, bits, 6, [[0, -1, 2], [6, 1, 2], [5, 2 ** 31 - 1, 0], [3, 3, 3]], kind="star")


@pytest.mark.parametrize("bits", [16, 4])
def test_tokens_given_up_for_the_ones_after_them(bits):
    """A cache so small that accepted tokens go again: their slots hold the last one's rows."""
    accept(np.random.default_rng(31), [3, 2], 2, 1, 3, bits, 12, [range(12), range(12)], recent=1)
    accept(np.random.default_rng(32), [5], 2, 1, 5, bits, 12, [range(12)], recent=0, sinks=2, tracked=False)


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("kw", [dict(), dict(decay=0.9), dict(score_cap=20.0, window=60, sinks=2)], ids=str)
def test_an_accepted_chain_is_as_many_steps(bits, kw):
    """While slots are free: the same cache as appends, each followed by its step.  (In 4 bits the steps see rows that have been quantized, a tree does
    not: what is compared there is where tokens are, and their rows.)"""
    rng = np.random.default_rng(37)
    lens, hq, hkv, n = [100, 30], 8, 2, 7
    s, _ = cached(rng, lens, hq, hkv, 120, bits, **kw)
    q, k, v = drafted(rng, 2, n, hq, hkv)
    steps = b.Slots(2, hq, hkv, 120, bits=bits, k=s.k.clone(), v=s.v.clone(), pos=s.pos.clone(), weight=s.weight.clone(), lens=s.lens.clone(),
                    next_pos=s.next_pos.clone(), **kw)
    parent = cuda(np.tile(np.arange(n) - 1, (2, 1)), I32)
    out, stats = b.rdkv_slots_tree_attn(s, q, k, v, parent)
    b.rdkv_slots_accept(s, q, k, v, cuda(np.tile(np.arange(n), (2, 1)), I32), stats)
    for j in range(n):
        b.rdkv_slots_append(steps, k[:, j].contiguous(), v[:, j].contiguous())
        o, lse = b.rdkv_slots_decode_attn(steps, q[:, j].contiguous())
        if bits == 16:                                 # roundings of probabilities and outputs
            assert torch.all((o - out[:, j].float()).abs() <= 2 * T.HALF_BF16 * (o.abs() + 1))
            assert torch.all((lse - stats[:, j, :, 0] - stats[:, j, :, 1].log()).abs() <= 1e-4)
    assert torch.equal(s.lens, steps.lens) and torch.equal(s.next_pos, steps.next_pos)
    for i in range(4):
        m = int(s.lens.view(-1)[i])
        assert torch.equal(s.pos.view(4, -1)[i, :m], steps.pos.view(4, -1)[i, :m])
        if bits == 16:
            x, y = s.weight.view(4, -1)[i, :m], steps.weight.view(4, -1)[i, :m]
            assert torch.all((x - y).abs() <= 1e-5 * (x + 1))
    rows = [b.rdkv_slots_read(t, torch.arange(100, 107, dtype=I32, device="cuda").expand(2, hkv, 7).contiguous()) for t in (s, steps)]
    assert torch.equal(rows[0][0], rows[1][0]) and torch.equal(rows[0][1], rows[1][1])


def test_nan_weights_go_first():
    rng = np.random.default_rng(41)
    s, items = cached(rng, [50], 2, 1, 50, 16, recent=2)
    s.weight[0, 0, 33] = math.nan
    q, k, v = drafted(rng, 1, 2, 2, 1)
    _, stats = b.rdkv_slots_tree_attn(s, q, k, v, cuda([[-1, 0]], I32))
    slot = b.rdkv_slots_accept(s, q, k, v, cuda([[0, 1]], I32), stats)
    assert slot[0, 0, 0] == (33 if items[0].pos[33] <= items[0].next - 2 else slot[0, 0, 0])


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("m", [1, 2])
def test_a_nan_weight_goes_before_all_others(bits, m):
    """Of two slots that may go and have none for a weight the older one first, whatever the others have gathered."""
    rng = np.random.default_rng(83)
    s, items = cached(rng, [150], 2, 1, 150, bits, sinks=2, recent=2)
    it = items[0]
    may = np.nonzero((it.pos >= 2) & (it.pos <= it.next - 40))[0]
    old, young = sorted((int(x) for x in (may[3], may[-5])), key=lambda x: it.pos[x])
    s.weight[0, 0, old] = s.weight[0, 0, young] = math.nan
    s.weight[0, 0, int(may[0])] = -1e30                     # (less than any that is gathered, and still a number)
    q, k, v = drafted(rng, 1, 2, 2, 1)
    _, stats = b.rdkv_slots_tree_attn(s, q, k, v, cuda([[-1, 0]], I32))
    slot = b.rdkv_slots_accept(s, q, k, v, cuda([[0, 1][:m]], I32), stats)
    assert slot.flatten().tolist() == [old, young][:m]


# ---- together ------------------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("bits", [16, 4])
def test_a_generation(bits):
    """Prompts attended to, cut to a cache by their weights, then trees and accepted paths, eager and as a graph: the same."""
    lens, hq, hkv, capacity, n = [300, 90], 8, 2, 128, 10
    rng = np.random.default_rng(43)
    gen = torch.Generator().manual_seed(3)
    Q, K, V = (torch.randn((sum(lens), h, D), generator=gen).to(BF).cuda() for h in (hq, hkv, hkv))
    out, lse = b.rdkv_prompt_attn_bf16(Q, K, V, lens, hq, hkv)
    flat = [prompt_plain.rows_to(t.cpu(), lens, h).cuda() for t, h in ((K, hkv), (V, hkv))]
    same, _ = b.rdkv_prompt_attn_bf16(Q, *flat, lens, hq, hkv)
    assert torch.equal(out, same)
    obs = torch.stack([Q[sum(lens[:s + 1]) - 32:sum(lens[:s + 1])].transpose(0, 1) for s in range(2)]).contiguous()
    w, _ = b.rdkv_weights(b.Config(lens, hq, hkv, s_obs=32), flat[0], obs)
    s = b.Slots(2, hq, hkv, capacity, bits=bits, sinks=2, recent=16, decay=0.99)
    b.rdkv_slots_fill(s, *flat, lens, w)
    twin = b.Slots(2, hq, hkv, capacity, bits=bits, sinks=2, recent=16, decay=0.99, k=s.k.clone(), v=s.v.clone(), pos=s.pos.clone(), weight=s.weight.clone(),
                   lens=s.lens.clone(), next_pos=s.next_pos.clone())
    q, k, v = drafted(rng, 2, n, hq, hkv)
    parent, path = cuda(np.stack([tree(rng, n, "chain")] * 2), I32), cuda([[0, 1, 2, -1], [0, -1, -1, -1]], I32)
    ws = s.tree_workspace(n)
    o, st, slot = torch.zeros_like(q), torch.zeros((2, n, hq, 2), device="cuda"), torch.zeros((2, hkv, 4), dtype=I32, device="cuda")

    def step(c):
        b.rdkv_slots_tree_attn(c, q, k, v, parent, out=o, stats=st, workspace=ws)
        b.rdkv_slots_accept(c, q, k, v, path, st, slot=slot)

    saved = [t.clone() for t in (twin.k, twin.v, twin.pos, twin.weight, twin.lens, twin.next_pos)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(twin)
    for x, y in zip((twin.k, twin.v, twin.pos, twin.weight, twin.lens, twin.next_pos), saved):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))                       # (recorded, not run)
    for it in range(5):
        q.copy_(cuda(rng.standard_normal(tuple(q.shape)), BF))
        k.copy_(cuda(rng.standard_normal(tuple(k.shape)), BF))
        step(s)
        eager = [o.clone(), st.clone(), slot.clone()]
        torch.cuda.synchronize()
        o.zero_(), st.zero_(), slot.zero_()
        graph.replay()
        for x, y in zip(eager, (o, st, slot)):
            assert torch.equal(x, y), it
        for x, y in zip((s.k, s.v, s.pos, s.weight, s.lens, s.next_pos), (twin.k, twin.v, twin.pos, twin.weight, twin.lens, twin.next_pos)):
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8)), it
    assert s.next_pos.cpu().tolist() == [[315, 315], [95, 95]]
    b.rdkv_slots_append(s, k[:, 0].contiguous(), v[:, 0].contiguous())
    d, _ = b.rdkv_slots_decode_attn(s, q[:, 0].contiguous())
    assert torch.isfinite(d).all()


@pytest.mark.parametrize("bits", [16, 4])
def test_on_another_stream_and_twice_the_same(bits):
    rng = np.random.default_rng(47)
    s, _ = cached(rng, [3000, 100], 8, 2, 3000, bits)
    q, k, v = drafted(rng, 2, 9, 8, 2)
    parent = cuda(np.stack([tree(rng, 9)] * 2), I32)
    want = b.rdkv_slots_tree_attn(s, q, k, v, parent)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        got = b.rdkv_slots_tree_attn(s, q, k, v, parent)
    torch.cuda.current_stream().wait_stream(stream)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("bits", [16, 4])
def test_graphs_that_share_a_workspace_and_streams_that_do_not(bits):
    """Two graphs of steps on two caches, replayed in turn over one workspace; the same calls at once on two streams with a workspace each."""
    rng = np.random.default_rng(59)
    made = []
    for lens, n in (([900, 40], 9), ([300, 900], 33)):
        s, _ = cached(rng, lens, 8, 2, 900, bits)
        q, k, v = drafted(rng, 2, n, 8, 2)
        made.append((s, q, k, v, cuda(np.stack([tree(rng, n)] * 2), I32), cuda([[0, -1], [0, 1]], I32)))
    kept = [[t.clone() for t in (m[0].k, m[0].v, m[0].pos, m[0].weight, m[0].lens, m[0].next_pos)] for m in made]

    def back():
        for m, ts in zip(made, kept):
            for t, name in zip(ts, ("k", "v", "pos", "weight", "lens", "next_pos")):
                getattr(m[0], name).copy_(t)

    def step(m, ws):
        s, q, k, v, parent, path = m
        out, stats = b.rdkv_slots_tree_attn(s, q, k, v, parent, workspace=ws)
        return [out, stats, b.rdkv_slots_accept(s, q, k, v, path, stats, workspace=ws)]

    def state(m):
        return [t.clone() for t in (m[0].k, m[0].v, m[0].pos, m[0].weight, m[0].lens, m[0].next_pos)]

    def same(a, c):
        return all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(a, c))
    size = max(max(m[0].tree_workspace(m[1].shape[1]).numel(), m[0].accept_workspace().numel()) for m in made)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    want = [[x.clone() for x in step(m, ws)] + state(m) for m in made]
    twice = [[x.clone() for x in step(m, ws)] + state(m) for m in made]
    back()
    graphs, results = [], []
    for m in made:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            results.append(step(m, ws))
        graphs.append(g)
    back()
    for expected in (want, twice):
        for g, r, m, w in zip(graphs, results, made, expected):
            g.replay()
            assert same([x.clone() for x in r] + state(m), w)
    back()
    streams, others = [torch.cuda.Stream() for _ in made], [torch.empty_like(ws) for _ in made]
    torch.cuda.synchronize()
    got = []
    for m, st, w in zip(made, streams, others):
        with torch.cuda.stream(st):
            got.append(step(m, w))
    torch.cuda.synchronize()
    for m, r, w in zip(made, got, want):
        assert same(r + state(m), w)


def test_native_calls_do_as_the_others(monkeypatch):
    """Results made and given, with and without counts and a workspace, through the native code and without it."""
    rng = np.random.default_rng(53)
    s, _ = cached(rng, [300, 290], 8, 2, 300, 16)
    q, k, v = drafted(rng, 2, 9, 8, 2)
    parent, path, counts = cuda(np.stack([tree(rng, 9)] * 2), I32), cuda([[0, 1, 2], [3, -1, 0]], I32), cuda([9, 4], I32)

    def every():
        t = s.__copy__()
        for name in ("k", "v", "pos", "weight", "lens", "next_pos"):
            setattr(t, name, getattr(s, name).clone())
        made = [*b.rdkv_slots_tree_attn(t, q, k, v, parent)]
        given = [torch.zeros_like(x) for x in made]
        r = b.rdkv_slots_tree_attn(t, q, k, v, parent, counts, given[0], given[1], t.tree_workspace(9))
        assert r[0] is given[0] and r[1] is given[1]
        one = b.rdkv_slots_tree_attn(t, q, k, v, parent, stats=given[1].clone())
        a = b.rdkv_slots_accept(t, q, k, v, path, made[1])
        slot = torch.zeros_like(a)
        assert b.rdkv_slots_accept(t, q, k, v, path, made[1], slot, t.accept_workspace()) is slot
        assert torch.equal(a[1, :, 1:], torch.full_like(a[1, :, 1:], -1))
        return made + given + [one[0], a, slot, t.k, t.v, t.pos, t.weight, t.lens, t.next_pos]
    assert b._call is not None
    native = every()
    monkeypatch.setattr(b, "_call", None)
    for x, y in zip(native, every()):
        assert x.dtype == y.dtype and x.shape == y.shape
        same = torch.equal(x.view(torch.uint8), y.view(torch.uint8))
        assert same


@pytest.mark.parametrize("native", [True, False])
def test_the_binding_refuses(native, monkeypatch):
    if not native:
        monkeypatch.setattr(b, "_call", None)
    s, q = b.Slots(2, 8, 2, 100), torch.zeros((2, 3, 8, D), device="cuda", dtype=BF)
    k, wide = torch.zeros((2, 3, 2, D), device="cuda", dtype=BF), torch.zeros((2, 3, 8, 2 * D), device="cuda", dtype=BF)[..., ::2]
    parent, path, stats = torch.zeros((2, 3), device="cuda", dtype=I32), torch.zeros((2, 2), device="cuda", dtype=I32), torch.zeros((2, 3, 8, 2), device="cuda")
    small = torch.zeros(64, device="cuda", dtype=torch.uint8)
    for call in (lambda: b.rdkv_slots_tree_attn(s, q.float(), k, k, parent), lambda: b.rdkv_slots_tree_attn(s, q, k, k[:, :2], parent), lambda: b.rdkv_slots_tree_attn(s, wide, k, k, parent),
                 lambda: b.rdkv_slots_tree_attn(s, q, k.cpu(), k, parent), lambda: b.rdkv_slots_tree_attn(s, q, k[0], k, parent), lambda: b.rdkv_slots_tree_attn(s, q, k, k, parent.long()),
                 lambda: b.rdkv_slots_tree_attn(s, q, k, k, parent, counts=parent), lambda: b.rdkv_slots_tree_attn(s, q, k, k, parent, out=stats),
                 lambda: b.rdkv_slots_tree_attn(s, q, k, k, parent, stats=stats[..., 0]), lambda: b.rdkv_slots_tree_attn(s, q, k, k, parent, workspace=stats),
                 lambda: b.rdkv_slots_accept(s, q, k, k, path[0], stats), lambda: b.rdkv_slots_accept(s, q, k, k, path.float(), stats), lambda: b.rdkv_slots_accept(s, q, k, k, path, stats[:1]),
                 lambda: b.rdkv_slots_accept(s, q[:, :2], k, k, path, stats), lambda: b.rdkv_slots_accept(s, q, k, k, path, stats, slot=path), lambda: b.rdkv_slots_accept(s, q, k, k, path, stats, workspace=small.cpu())):
        with pytest.raises(ValueError):
            call()
    many = torch.zeros((2, 65, 2, D), device="cuda", dtype=BF)
    for call in (lambda: b.rdkv_slots_accept(s, None, k, k, path, stats), lambda: b.rdkv_slots_accept(s, q, k, k, path, None),
                 lambda: b.rdkv_slots_accept(s, torch.zeros((2, 65, 8, D), device="cuda", dtype=BF), many, many, path, torch.zeros((2, 65, 8, 2), device="cuda")),
                 lambda: b.rdkv_slots_accept(s, q, k, k, torch.zeros((2, 65), device="cuda", dtype=I32), stats),
                 lambda: b.rdkv_slots_accept(s, q, k, k, path, stats, workspace=small), lambda: b.rdkv_slots_tree_attn(b.Slots(2, 8, 2, 9000), q, k, k, parent, workspace=small)):
        with pytest.raises(b.RdkvError):
            call()
    assert not s.lens.any() and not s.next_pos.any()


@pytest.mark.parametrize("bits", [16, 4])
def test_caches_past_4_gib(bits):
    """The last item's slots lie past 2^32 bytes of a side."""
    capacity, hkv = (4200000, 5) if bits == 16 else (11000000, 6)
    s = b.Slots(1, hkv, hkv, capacity, bits=bits)
    rng, m = np.random.default_rng(53), 70
    rows = torch.tensor(np.concatenate([rows_of(rng, m) for _ in range(hkv)])).to(BF).cuda()
    small = b.Slots(1, hkv, hkv, 100, bits=bits)
    for c in (s, small):
        b.rdkv_slots_fill(c, rows, rows, [m])
    assert s.k.numel() * s.k.element_size() > 2 ** 32
    q, k, v = drafted(rng, 1, 3, hkv, hkv)
    parent, path = cuda([[-1, 0, 1]], I32), cuda([[0, 1, 2]], I32)
    got, want = (b.rdkv_slots_tree_attn(c, q, k, v, parent) for c in (s, small))
    assert (got[0].float() - want[0].float()).abs().max() <= 2 * T.HALF_BF16 * 4
    slots = [b.rdkv_slots_accept(c, q, k, v, path, want[1]) for c in (s, small)]
    assert torch.equal(slots[0], slots[1])
    rows = [b.rdkv_slots_read(c, n=m + 3) for c in (s, small)]
    assert torch.equal(rows[0][0], rows[1][0]) and torch.equal(rows[0][1], rows[1][1])
    assert torch.allclose(s.weight[..., :m + 3], small.weight[..., :m + 3], rtol=1e-6)
