"""Causal attention of prompts in plain numpy, 64 bits, one sequence and KV head at a time: what the tests of rdkv_prompt_attn_bf16
compare with."""
import math

import numpy as np
import torch

D = 128
HALF_BF16 = 2.0 ** -8             # a rounding to bf16, relative to the value


def attend(q, k, v, window=0, sinks=0, cap=0.0, slopes=None):
    """q [g, T, 128], k, v [T, 128] float64 -> out [g, T, 128], lse [g, T], and bounds of what they can be off.

    A score is a sum of 128 products, exact in fp32 (8 bits by 8): in any order it is off by at most 130 x 2^-24 times the sum of their
    sizes; the cap, the bias and the last factor add a few units in the last place of the largest term.  A probability is off by twice that
    (its own score's and the row's largest), by 2^-20 (exponential, quotient), by what fp32 sums of up to T terms are off, and by its
    rounding to bf16; the output is rounded once more."""
    T = k.shape[0]
    away = np.arange(T)[:, None] - np.arange(T)[None]
    seen = away >= 0
    if window:
        seen &= (away < window) | (np.arange(T)[None] < sinks)
    x = q @ k.T / math.sqrt(D)
    size = np.where(seen, np.abs(q) @ np.abs(k).T / math.sqrt(D), 0.0).max(-1)
    most = np.where(seen, np.abs(x), 0.0).max(-1)
    if cap:
        x = cap * np.tanh(x / cap)
        most = most + cap
    if slopes is not None:
        bias = slopes[:, None, None] * away
        x = x - bias
        most = most + np.where(seen, np.abs(bias), 0.0).max(-1)
    off = 2.0 ** -24 * (130 * size + 8 * most)
    x = np.where(seen, x, -np.inf)
    top = x.max(-1, keepdims=True)
    e = np.exp(x - top)
    total = e.sum(-1, keepdims=True)
    p = e / total
    lse = (top + np.log(total))[..., 0]
    out = p @ v
    sums = 2.0 ** -24 * (T / 2 + 64)
    out_off = (HALF_BF16 + 2 * off + sums + 2.0 ** -20)[..., None] * (p @ np.abs(v)) * (1 + HALF_BF16) + HALF_BF16 * np.abs(out) + 1e-38
    return out, lse, out_off, off + sums + 2.0 ** -22 * (1 + np.abs(lse))


def heads_of(x, lens, heads, s, h, tokens):
    """[T, 128] of head h of sequence s out of [rows, 128] ragged blocks, or [tokens, heads, 128]."""
    t0, T = sum(lens[:s]), lens[s]
    return x[t0:t0 + T, h] if tokens else x.reshape(-1, D)[t0 * heads + h * T:t0 * heads + (h + 1) * T]


def rows_to(x, lens, heads):
    """[tokens, heads, 128] -> flat ragged [heads][T][128] blocks."""
    t0, parts = 0, []
    for T in lens:
        parts.append(x[t0:t0 + T].transpose(0, 1).reshape(-1))
        t0 += T
    return torch.cat(parts)
