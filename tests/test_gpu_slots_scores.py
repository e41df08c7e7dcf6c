"""Slot caches on the GPU: steps whose scores are far from 0, far from their head's maximum, or far from the neighbouring head's."""
import math

import numpy as np
import pytest
import torch

from paper_2605_08317_amd import binding as b
from tests import slots_plain as P
from tests.test_gpu_slots import BF, D, I32, check_step, cuda, host, loaded, tiles_of

pytestmark = pytest.mark.gpu


def codes(rng, n):
    """V rows [n, 128] that bf16 and 4 bits hold exactly, and whose sums fp32 does: whole numbers 0 .. 15, both in every group."""
    v = rng.integers(0, 16, (n, 4, 32))
    v[:, :, 0], v[:, :, 1] = 0, 15
    return v.reshape(n, D).astype(np.float32)


def cache(K, V, lens, hq, capacity, bits, **kw):
    """Rows [batch][hkv] of [len, 128] as a cache.  Every row is held exactly."""
    batch, hkv = len(lens), len(K[0])
    s = b.Slots(batch, hq, hkv, capacity, bits=bits, **kw)
    for t, rows, side in ((s.k, K, "k"), (s.v, V, "v")):
        for i in range(batch):
            for h in range(hkv):
                r = rows[i][h]
                assert np.array_equal(P.held(r, bits), r)
                if bits == 16:
                    t[i, h, :lens[i]] = cuda(r, BF)
                else:
                    t[i, h, :(lens[i] + 63) // 64] = cuda(tiles_of(r, side))
    s.pos.copy_(torch.arange(capacity, dtype=I32, device="cuda").expand_as(s.pos))
    s.lens.copy_(torch.tensor(lens, dtype=I32, device="cuda")[:, None].expand_as(s.lens))
    s.next_pos.copy_(s.lens)
    return s


def off(got, want):
    """The largest difference, relative to the value; where that is 0 nothing else will do."""
    got, want = np.broadcast_arrays(got, want)
    assert not got[want == 0].any() and np.isfinite(got).all()
    return np.max(np.abs(got - want)[want != 0] / np.abs(want[want != 0]))


LENS = {300: [300, 219], 5000: [5000, 4321]}      # capacities: an item to a workgroup, and cut into pieces


# ---- scores far from 0 -------------------------------------------------------------------------------------------------------------

def equal_scores(rng, bits, g, capacity, e, biased):
    """Every K row is 64 and the query 2^e: all scores are 2^(13 + e) / sqrt(128), and their products and sums exact."""
    lens = LENS[capacity]
    K = [[np.full((n, D), 64.0, np.float32)] * 2 for n in lens]
    V = [[codes(rng, n) for _ in range(2)] for n in lens]
    s = cache(K, V, lens, 2 * g, capacity, bits, slopes=torch.zeros(2 * g, device="cuda") if biased else None)
    return s, V, lens, torch.full((2, 2 * g, D), 2.0 ** e, device="cuda", dtype=BF)


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("g", [1, 4, 8])
@pytest.mark.parametrize("capacity", sorted(LENS))
@pytest.mark.parametrize("e, biased", [(1, False), (1, True), (7, False), (17, False), (17, True)])      # scores 1.4e3, 9.3e4, 9.5e7
def test_outputs_of_equal_scores(bits, g, capacity, e, biased):
    """The mean of V.  Exponentials are of 0, sums whole numbers below 2^24; there remain the quotient, a product, and factors near 1 of
    the wavefronts' and the pieces' sums: 8 wavefronts or 20 pieces of 4, each two roundings of a sum that is a part of the whole."""
    rng = np.random.default_rng(30)
    s, V, lens, q = equal_scores(rng, bits, g, capacity, e, biased)
    out, lse = b.rdkv_slots_decode_attn(s, q)
    score = 2.0 ** (13 + e) / math.sqrt(D)
    for i, n in enumerate(lens):
        for h in range(2):
            mean = V[i][h].astype(np.float64).mean(0)
            got = host(out)[i, h * g:(h + 1) * g]
            assert off(got, mean) <= 2.0 ** -20
            assert off(host(lse)[i, h * g:(h + 1) * g], score + math.log(n)) <= 2.0 ** -22


# ---- maxima far from 0, and others near them ----------------------------------------------------------------------------------------

def two_scores(rng, bits, g, capacity, e, biased):
    """Products with the query are 2^e, and 8 more in an item's first half: exact in fp32, as is their difference."""
    lens = LENS[capacity]
    K = [[np.zeros((n, D), np.float32) for _ in range(2)] for n in lens]
    for n, two in zip(lens, K):
        for k in two:
            k[:, :32] = 2.0 ** (e // 2)
            k[:n // 2, 32:64] = 8.0
    V = [[codes(rng, n) for _ in range(2)] for n in lens]
    s = cache(K, V, lens, 2 * g, capacity, bits, slopes=torch.zeros(2 * g, device="cuda") if biased else None)
    q = torch.zeros((2, 2 * g, D), device="cuda", dtype=BF)
    q[:, :, 0], q[:, :, 32] = 2.0 ** (e - e // 2), 1.0
    return s, V, lens, q


def two_probabilities(n):
    p = np.where(np.arange(n) < n // 2, 1.0, math.exp(-8 / math.sqrt(D)))
    return p / p.sum()


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("g", [1, 4, 8])
@pytest.mark.parametrize("capacity", sorted(LENS))
@pytest.mark.parametrize("e, biased", [(10, False), (20, False), (23, False), (23, True)])
def test_outputs_of_two_scores(bits, g, capacity, e, biased):
    """Wavefronts and pieces have maxima that differ by 8 / sqrt(128), 1.02 in the exponent.  With biases the scores are products over
    sqrt(128), rounded: 2^-24 of them each; else they are exact.  A probability is off by that, 1.02 x 2^-24 x ln 2 and an exponential's
    2^-23; the sums as everywhere, relative to their terms (of 4-bit rows scale x (code - 8) and offset + 8 scale)."""
    rng = np.random.default_rng(31)
    s, V, lens, q = two_scores(rng, bits, g, capacity, e, biased)
    out, _ = b.rdkv_slots_decode_attn(s, q)
    rel = 2 * (2 * 2.0 ** (e - 24) / math.sqrt(D) if biased else 0.0) + P.sums_off(lens[0]) + 2.0 ** -20
    for i, n in enumerate(lens):
        for h in range(2):
            p = two_probabilities(n)
            worst = np.abs(host(out)[i, h * g:(h + 1) * g] - p @ V[i][h].astype(np.float64)) / (p @ P.terms(V[i][h], bits, 8) + 1e-30)
            assert worst.max() <= rel


# ---- the weights -----------------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("g", [1, 2, 4, 8])
@pytest.mark.parametrize("capacity", sorted(LENS))
@pytest.mark.parametrize("e, biased", [(1, False), (1, True), (7, False), (17, False), (17, True)])
def test_weights_of_equal_scores(bits, g, capacity, e, biased):
    """Every token's grows by g / n: a quotient and g - 1 additions, then one to what there was."""
    rng = np.random.default_rng(32)
    s, V, lens, q = equal_scores(rng, bits, g, capacity, e, biased)
    s.weight.fill_(0.0)
    for before in (0.0, g / 8192):
        s.weight.fill_(before)
        b.rdkv_slots_decode_attn(s, q)
        for i, n in enumerate(lens):
            assert off(host(s.weight)[i, :, :n], before + g / n) <= 2.0 ** -24 * (g + 2)
            assert (s.weight[i, :, n:] == before).all()


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("g", [1, 2, 4, 8])
@pytest.mark.parametrize("capacity", sorted(LENS))
@pytest.mark.parametrize("e, biased", [(10, False), (16, False), (23, False), (10, True)])
def test_weights_of_two_scores(bits, g, capacity, e, biased):
    """As the outputs: a probability's rounding, and the sum's."""
    rng = np.random.default_rng(33)
    s, V, lens, q = two_scores(rng, bits, g, capacity, e, biased)
    b.rdkv_slots_decode_attn(s, q)
    # the sum, of 64 slots a wavefront: four additions a tile and lane, and 4 + 3 + 20 of lanes, wavefronts and pieces
    rel = 2 * (2 * 2.0 ** (e - 24) / math.sqrt(D) if biased else 0.0) + 2.0 ** -24 * (8 + 27 + g + 8)
    for i, n in enumerate(lens):
        assert off(host(s.weight)[i, :, :n], g * two_probabilities(n)) <= rel


# ---- heads of one group far from each other ----------------------------------------------------------------------------------------------

@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("e", [[30, 0], [25, 0, -8, 12], [0, 40, -3, -20, 60, 1, -60, 18]])
@pytest.mark.parametrize("lens, capacity", [([300, 77], 300), ([5000, 64], 5000)])
@pytest.mark.parametrize("kw", [{}, {"score_cap": 30.0}])
def test_heads_of_different_magnitudes(bits, e, lens, capacity, kw):
    """Queries 2^e times normal numbers: each head's scores keep their own digits."""
    rng = np.random.default_rng(34)
    g = len(e)
    s, items = loaded(rng, lens, 2 * g, 2, capacity, bits, **kw)
    q = rng.standard_normal((2, 2 * g, D)) * 2.0 ** np.array(e * 2)[None, :, None]
    before = host(s.weight)
    out, lse = b.rdkv_slots_decode_attn(s, cuda(q, BF))
    check_step(s, items, cuda(q, BF), out, lse, s.weight, before, **({"cap": 30.0} if kw else {}))


# ---- how many digits a probability has -----------------------------------------------------------------------------------------------------

def a_term_less(p, bits):
    """Probabilities as they would meet the rows with one term less: two bf16 terms, cut off, or one of fp16."""
    p = p.astype(np.float32)
    if bits == 4:
        return (p * np.float32(2 ** 14)).astype(np.float16).astype(np.float64) / 2 ** 14
    hi = (p.view(np.uint32) & np.uint32(0xFFFF0000)).view(np.float32)
    lo = ((p - hi).view(np.uint32) & np.uint32(0xFFFF0000)).view(np.float32)
    return hi.astype(np.float64) + lo


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("g", [1, 4, 8])
@pytest.mark.parametrize("capacity", [300, 5000])
def test_probabilities_keep_their_digits(bits, g, capacity):
    """One token, and others whose products with the query are 29 less, exp(-29 / sqrt(128)) of its probability, a number that loses much
    with a term less.  Values are not negative, so that nothing cancels.  In units of 2^-24: the exponent 3.7 is rounded by 2 and its factor
    by 1.9, times ln 2; the exponential by 2: 5 of a probability, twice.  A wavefront's tile: 4 + 4 additions to its sum; 16 steps of three
    terms to the outputs, each off by 2 at most; the merge 8 and 8, the quotient 2."""
    rng = np.random.default_rng(35)
    bound = 2.0 ** -24 * (2 * 5 + 8 + 2 * 48 + 16 + 2)
    lens = [200, 77]
    K = [[np.zeros((n, D), np.float32)] * 2 for n in lens]
    for two in K:
        two[0][0, :32] = 29.0
    V = [[codes(rng, n) for _ in range(2)] for n in lens]
    s = cache(K, V, lens, 2 * g, capacity, bits)
    q = torch.zeros((2, 2 * g, D), device="cuda", dtype=BF)
    q[:, :, 0] = 1.0
    out, _ = b.rdkv_slots_decode_attn(s, q)
    for i, n in enumerate(lens):
        e = np.where(np.arange(n) == 0, 1.0, math.exp(-29 / math.sqrt(D)))
        p = e / e.sum()
        for h in range(2):
            v, size = V[i][h].astype(np.float64), p @ P.terms(V[i][h], bits, 8) + 1e-30
            assert np.max(np.abs(host(out)[i, h * g:(h + 1) * g] - p @ v) / size) <= bound
            # (the bound would see it)
            assert np.max(np.abs(a_term_less(e, bits) @ v / e.sum() - p @ v) / size) > 2 * bound
