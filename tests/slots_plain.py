"""A slot cache in plain numpy, 64 bits, one item at a time: what the tests of rdkv_slots_* compare with."""
import math

import numpy as np
import torch

from oracle import rdkv_oracle as O

D = 128


def bf16(x):
    """float -> the nearest bf16, as float32."""
    return torch.as_tensor(np.asarray(x)).to(torch.float32).to(torch.bfloat16).float().numpy()


def held(rows, bits):
    """float64 values that `bits` hold of float32 rows [n, 128]."""
    rows = np.asarray(rows, np.float32)
    if bits == 16:
        return rows.astype(np.float64)
    c, s, m = O.quantize_rows(rows, 4)
    n = rows.shape[0]
    return O.dequantize_groups(c.reshape(n, 4, 32), s, m).reshape(n, D)


def terms(rows, bits, centre=0):
    """Sizes of the terms that a kernel adds up for these rows' values.  Of 4-bit rows those are scale x (code - centre) and
    offset + centre x scale (centre 0 in K rows, 8 in V rows), each multiplied and summed by itself and rounded relative to itself,
    wherever they nearly cancel: off by 2^-24 of their sizes per operation, not of the value's."""
    rows = np.asarray(rows, np.float32)
    if bits == 16:
        return np.abs(rows).astype(np.float64)
    c, s, m = O.quantize_rows(rows, 4)
    n = rows.shape[0]
    s, m = s.astype(np.float64), m.astype(np.float64)
    return (np.abs(s[..., None] * (c.reshape(n, 4, 32).astype(np.float64) - centre)) + np.abs(m + centre * s)[..., None]).reshape(n, D)


def choose(T, capacity, sinks, recent, w):
    """Positions a filled item keeps, ascending."""
    if T <= capacity:
        return np.arange(T)
    at = np.arange(T)
    always = (at < sinks) | (at >= T - recent)
    others = at[~always]
    v = np.asarray(w, np.float64)[others]
    # NaN behind every number; stable: lower positions first among equal ones
    order = np.lexsort((others, -np.where(np.isnan(v), 0.0, v), np.isnan(v)))
    return np.sort(np.concatenate([at[always], others[order[:capacity - always.sum()]]]))


def evict(pos, weight, nxt, sinks, recent):
    """Slot that a full item gives up (weight None: all equal)."""
    may = np.nonzero((pos >= sinks) & (pos <= nxt - recent))[0]
    v = np.zeros(len(may)) if weight is None else np.asarray(weight, np.float64)[may]
    return int(may[np.lexsort((pos[may], np.where(np.isnan(v), 0.0, v), ~np.isnan(v)))[0]])


def attend(q, K, V, pos, nxt, K_size, sinks=0, window=0, cap=0.0, slopes=None):
    """q [g, 128], K, V [n, 128] float64 values, K_size = terms() -> out [g, 128], lse [g], p [g, n], and the bound of what fp32 scores
    can be off.

    A score is a sum of 128 products (exact in fp32: 8 bits by 8, or 8 by 4 and a scale): in any order it is off by at most
    130 x 2^-24 times the sum of their sizes; the cap, the bias and their rounding add a few units in the last place of the
    largest term."""
    n = K.shape[0]
    g = q.shape[0]
    away = (nxt - 1) - pos.astype(np.float64)
    seen = np.ones(n, bool) if window == 0 else (away < window) | (pos < sinks)
    out, lse, p = np.zeros((g, D)), np.full(g, -np.inf), np.zeros((g, n))
    if not seen.any():
        return out, lse, p, np.zeros(g)
    x = q @ K[seen].T / math.sqrt(D)
    size = (np.abs(q) @ K_size[seen].T / math.sqrt(D)).max(axis=1)
    most = np.abs(x).max(axis=1)
    if cap:
        x = cap * np.tanh(x / cap)
        most = most + cap
    if slopes is not None:
        bias = slopes[:, None] * away[seen][None]
        x = x - bias
        most = most + np.abs(bias).max(axis=1)
    off = 2.0 ** -24 * (130 * size + 8 * most)
    top = x.max(axis=1)
    e = np.exp(x - top[:, None])
    lse = top + np.log(e.sum(axis=1))
    p[:, seen] = e / e.sum(axis=1, keepdims=True)
    out = p[:, seen] @ V[seen]
    return out, lse, p, off


def sums_off(n):
    """What n fp32 additions in steps of four, and the merge of parts, are off by, relative to the sum of the terms' sizes."""
    return 2.0 ** -24 * (n / 2 + 64)


class Item:
    """One (sequence, KV head)."""

    def __init__(self, capacity, bits, sinks, recent):
        self.capacity, self.bits, self.sinks, self.recent = capacity, bits, sinks, recent
        self.K, self.V, self.K_size, self.V_size = (np.zeros((capacity, D)) for _ in range(4))
        self.pos, self.weight = np.zeros(capacity, np.int64), np.zeros(capacity)
        self.n = self.next = 0

    def put(self, at, k, v):
        """float32 rows into slots `at`."""
        self.K[at], self.V[at] = held(k, self.bits), held(v, self.bits)
        self.K_size[at], self.V_size[at] = terms(k, self.bits), terms(v, self.bits, 8)

    def fill(self, K, V, w):
        T = K.shape[0]
        at = choose(T, self.capacity, self.sinks, self.recent, w)
        self.n, self.next = len(at), T
        self.put(slice(0, self.n), K[at], V[at])
        self.pos[:self.n] = at
        self.weight[:self.n] = 0.0 if w is None else w[at]

    def append(self, k, v, slot=None, tracked=True):
        """slot: where the library put it (None: found here)."""
        if self.n < self.capacity:
            slot = self.n
            self.n += 1
        elif slot is None:
            slot = evict(self.pos, self.weight if tracked else None, self.next, self.sinks, self.recent)
        self.put(slice(slot, slot + 1), k[None], v[None])
        self.pos[slot], self.weight[slot] = self.next, 0.0
        self.next += 1
        return slot

    def decode(self, q, decay=1.0, **kw):
        n = self.n
        out, lse, p, off = attend(q, self.K[:n], self.V[:n], self.pos[:n], self.next, self.K_size[:n], sinks=self.sinks, **kw)
        self.weight[:n] = decay * self.weight[:n] + p.sum(axis=0)
        return out, lse, p, off
