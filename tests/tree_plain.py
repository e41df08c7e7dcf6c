"""Drafted trees over slot caches in plain numpy, 64 bits, one item at a time: what the tests of rdkv_slots_tree_attn and rdkv_slots_accept
compare with.  Items are those of tests/slots_plain.py."""
import math

import numpy as np

from tests import slots_plain as P

D = 128
HALF_BF16, HALF_FP16 = 2.0 ** -8, 2.0 ** -11      # a rounding to bf16 and to fp16, relative to the value


def ways(parent, count):
    """Of each token those that it descends from, itself the last."""
    way = []
    for i in range(count):
        p = int(parent[i])
        way.append((way[p] if 0 <= p < i else []) + [i])
    return way


def scores(item, q, k_draft, way, sinks=0, window=0, cap=0.0, slopes=None):
    """q [t, g, 128], k_draft [t, 128] of tokens with these ways -> float64 scores [t, g, slots + t], -inf where hidden, and what fp32 scores can
    be off [t, g].

    As in slots_plain.attend; of 4-bit rows the terms that are added up are scale x (code + 16), 16 x scale and the offset, each with the query's
    values (the query's sums in 22 bits: 2 units more)."""
    n, t = item.n, len(way)
    K = np.concatenate([item.K[:n], k_draft])
    if item.bits == 4:
        size = np.concatenate([np.abs(item.K_size4[:n]), np.abs(k_draft)])
    else:
        size = np.abs(K)
    depth = np.array([len(w) - 1 for w in way])
    place = np.concatenate([item.pos[:n], item.next + depth]).astype(np.float64)
    away = (item.next + depth)[:, None] - place[None]
    seen = np.zeros((t, n + t), bool)
    seen[:, :n] = True
    for i, w in enumerate(way):
        seen[i, n + np.array(w)] = True
    if window:
        seen &= (away < window) | (place[None] < sinks)
    x = q @ K.T / math.sqrt(D)
    sizes = np.where(seen[:, None], np.abs(q) @ size.T / math.sqrt(D), 0.0).max(-1)
    most = np.where(seen[:, None], np.abs(x), 0.0).max(-1)
    if cap:
        x = cap * np.tanh(x / cap)
        most = most + cap
    if slopes is not None:
        bias = slopes[None, :, None] * away[:, None]
        x = x - bias
        most = most + np.where(seen[:, None], np.abs(bias), 0.0).max(-1)
    return np.where(seen[:, None], x, -np.inf), 2.0 ** -24 * (134 * sizes + 8 * most)


def attend(item, q, k_draft, v_draft, way, **kw):
    """-> out [t, g, 128], M [t, g], S [t, g] and bounds of out, M and the relative error of S."""
    n = item.n
    x, off = scores(item, q, k_draft, way, **kw)
    top = x.max(-1)
    e = np.exp(x - np.where(np.isfinite(top), top, 0.0)[..., None])
    total = e.sum(-1)
    p = e / np.where(total == 0, 1.0, total)[..., None]
    out = p[..., :n] @ item.V[:n] + p[..., n:] @ v_draft
    fp32 = (2 * off + P.sums_off(n + 64) + 2.0 ** -20)[..., None]
    # values: bf16 rows as they are, codes scaled to fp16 (the value and the offset plus 8 scales are rounded); probabilities to bf16 or fp16, there over 2^-11
    # and a slack of 2^-4: below 2^-25 x 2^-11 x 2^4 they lose bits
    rel, least = (HALF_BF16, 0.0) if item.bits == 16 else (3 * HALF_FP16, 2.0 ** -32)
    bound = (rel + fp32) * (p[..., :n] @ item.V_size[:n]) * (1 + rel) + (HALF_BF16 + fp32) * (p[..., n:] @ np.abs(v_draft)) * (1 + HALF_BF16)
    if n:
        bound = bound + least * np.abs(item.V_size[:n]).sum(0)
    return out, top, total, bound + HALF_BF16 * np.abs(out) + 1e-30, off + 2.0 ** -22 * np.abs(np.where(np.isfinite(top), top, 0.0)), fp32[..., 0] + 2.0 ** -22


def given(item, q, k_draft, stats, decay, **kw):
    """What a path's tokens [c, g, 128] give the slots and the path's tokens, float64 [slots + c], and its bound, with the stats [c, g, 2] as they are."""
    c = q.shape[0]
    x, off = scores(item, q, k_draft, [list(range(i + 1)) for i in range(c)], **kw)
    M, S = stats[..., 0].astype(np.float64), stats[..., 1].astype(np.float64)
    p = np.exp(x - np.where(np.isfinite(M), M, 0.0)[..., None]) / np.where(S == 0, 1.0, S)[..., None]
    p = p * (float(np.float32(decay)) ** (c - 1 - np.arange(c)))[:, None, None]
    rel = (off + 2.0 ** -22 * (1 + np.abs(np.where(np.isfinite(M), M, 0.0))) + 2.0 ** -20 + 2.0 ** -24 * c * q.shape[1])[..., None]
    return p.sum((0, 1)), (p * rel).sum((0, 1))
