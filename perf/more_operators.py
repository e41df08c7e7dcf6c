"""Attention of whole prompts, and of trees of drafted tokens over slot caches, as cases that a timing program can prepare and run, and
their plain forms.  A case names what is called ("op"):

  prompt   a ragged batch of prompts, every token attending to itself and the tokens before it (scores capped, biased by distance or
           limited to a window where the case says so); q, k and v as ragged [heads][T][128] blocks or as parts of a projection's rows
  tree     `drafted` tokens per sequence, each the child of an earlier one or of the last cached token: a token attends to the slots of
           the cache, to the drafted tokens that it descends from, and to itself
  accept   the first tokens of a path through such a tree become part of the cache: every slot gathers the attention weight that they gave
           it, and each token takes a free slot, or that of the token of least weight

`own` False: plain torch operations.  `own` True: the library's calls.  Rows that come back from 4-bit caches are the values the codes stand for.
"""
import math
import random

import torch

own = False

D = 128
GROUP = 32                       # channels that share a scale and an offset in 4 bits
TILE = 64                        # rows of a 4-bit tile: 4096 bytes of codes, 1024 of scales and offsets
TILE_BYTES = 5120
BLOCK = 1 << 29                  # scores that the plain form of a prompt holds at once


def _case(op, name=None, *, batch=1, hq=32, hkv=8, capacity=0, lo=None, bits=16, sinks=0, recent=32, window=0, cap=0.0, bias=False, decay=1.0,
          tokens=False, drafted=0, padded=False, accepted=0):
    """capacity: of a prompt the tokens of the longest; lo: of the shortest, or the fewest slots in use (the first sequence has them all);
    tokens: a prompt's q, k and v lie token by token; padded: sequences with fewer drafted tokens than `drafted`; accepted: of the longest path."""
    c = {"op": op, "batch": batch, "hq": hq, "hkv": hkv, "capacity": capacity, "lo": capacity if lo is None else lo, "bits": bits, "sinks": sinks,
         "recent": recent, "window": window, "cap": cap, "bias": bias, "decay": decay, "tokens": tokens, "drafted": drafted, "padded": padded,
         "accepted": accepted}
    return dict(c, name=name) if name else c


def listed():
    return [
        # A short question to a tensor-parallel shard with two KV heads: latency.
        _case("prompt", "prompt_tiny", hq=8, hkv=2, capacity=300),
        # Requests that arrive together at an 8B-shaped layer, q, k and v from one projection.
        _case("prompt", "prompt_batch", batch=16, capacity=4096, lo=17, tokens=True),
        # One long document.
        _case("prompt", "prompt_long", capacity=32768),
        # A 70B-shaped layer with capped scores that sees a window and the first tokens.
        _case("prompt", "prompt_window_capped", batch=2, hq=64, capacity=16384, lo=9001, window=4096, sinks=4, cap=30.0, tokens=True),
        # The smallest check of drafted tokens: two KV heads, a thousand slots.
        _case("tree", "tree_tiny_bf16", hq=8, hkv=2, capacity=1000, drafted=8),
        # Batched serving of a 70B-shaped layer, ragged, capped scores, some sequences with fewer drafted tokens.
        _case("tree", "tree_batch_capped_bf16", batch=16, hq=64, capacity=4096, lo=1500, cap=30.0, drafted=16, padded=True),
        # Long contexts and the widest tree: the largest cache in bf16.
        _case("tree", "tree_long_bf16", batch=4, capacity=131072, drafted=64),
        # Linear position biases, 4-bit rows, many sequences.
        _case("tree", "tree_batch_biased_4bit", batch=32, capacity=8192, lo=5000, bits=4, bias=True, drafted=32),
        # Long contexts in 4 bits, a few drafted tokens.
        _case("tree", "tree_long_4bit", batch=4, capacity=131072, lo=90001, bits=4, drafted=8),
        # Accepted tokens into the smallest cache.
        _case("accept", "accept_tiny_bf16", hq=8, hkv=2, capacity=1000, drafted=8, accepted=4),
        # Accepted tokens of many sequences in 4 bits, some with free slots, weights that age.
        _case("accept", "accept_batch_4bit", batch=32, capacity=8192, lo=5000, bits=4, bias=True, decay=0.98, drafted=32, accepted=8),
        # Accepted tokens into long caches.
        _case("accept", "accept_long_bf16", batch=4, capacity=131072, drafted=16, accepted=6),
    ]


def _log(rng, lo, hi):
    return lo if hi <= lo else int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["prompt", "prompt", "tree", "tree", "accept"])
    hkv = rng.choice([1, 2, 4, 8, 8])
    kw = {"hkv": hkv, "hq": hkv * rng.choice([1, 2, 4, 4, 8]), "batch": _log(rng, 1, 48), "sinks": rng.randint(0, 16),
          "cap": rng.choice([0.0, 0.0, 20.0, 50.0]), "bias": rng.random() < 0.25}
    if op == "prompt":
        most = int(math.sqrt((1 << 35) / (kw["batch"] * kw["hq"])))         # scores: what the longest listed prompt has
        kw["capacity"] = _log(rng, 1, min(32768, most))
        kw["tokens"] = rng.random() < 0.5
    else:
        kw["bits"] = rng.choice([4, 16])
        kw["drafted"] = _log(rng, 1, 64)
        rows = kw["batch"] * kw["hq"] * kw["drafted"]
        longest = min(131072, (1 << 22) // (kw["batch"] * hkv), (1 << 30) // rows)
        if op == "accept":
            longest = min(longest, (1 << 20) // (kw["batch"] * hkv))
            kw["accepted"] = rng.randint(1, min(16, kw["drafted"]))
            kw["decay"] = rng.choice([1.0, 1.0, 0.9])
        kw["capacity"] = max(100, _log(rng, 100, longest))
        kw["recent"] = rng.randint(0, 48)
        kw["padded"] = rng.random() < 0.4
    kw["lo"] = rng.choice([kw["capacity"], rng.randint(1, kw["capacity"])])
    if rng.random() < 0.3:
        kw["window"] = rng.randint(1, 2 * kw["capacity"])
    return _case(op, **kw)


def _rng(case, what):
    """What is part of the case, the same for every seed."""
    return random.Random("%s %d %d %d %d" % (what, case["batch"], case["lo"], case["capacity"], case["drafted"]))


def _lens(case):
    rng = _rng(case, "lengths")
    return [case["capacity"]] + [rng.randint(case["lo"], case["capacity"]) for _ in range(case["batch"] - 1)]


def _trees(case):
    """parent [batch][drafted], the tokens that each sequence drafted, and the paths [batch][accepted] that are taken of them, ended by -1."""
    rng, n, m = _rng(case, "trees"), case["drafted"], case["accepted"]
    parents, counts, paths = [], [], []
    for s in range(case["batch"]):
        count = rng.randint(1, n) if case["padded"] and s > 0 else n
        parent = [max(-1, i - 1 - int(rng.expovariate(0.7))) for i in range(n)]
        leaf, path = max(range(count), key=lambda i: len(_up(parent, i))), []
        path = _up(parent, leaf)[::-1][:m]
        path = path[:rng.randint(0, len(path))] if s > 0 else path
        parents.append(parent)
        counts.append(count)
        paths.append(path + [-1] * (m - len(path)))
    return parents, counts, paths


def _up(parent, i):
    way = []
    while i >= 0:
        way.append(i)
        i = parent[i]
    return way


# ---- 4 bits: the library's tiles of 64 rows -----------------------------------------------------------------------------------
# A lane (K: a row of the tile; V: 32 (row // 32) + channel % 32) has 16 words, word W at byte 1024 (W // 4) + 16 lane + 4 (W % 4); four
# words hold 32 codes (K: the channels of group W // 4; V: the 32 rows of the lane's half, of channel 32 (W // 4) + lane % 32), code
# 16 p + 4 f + 2 w + h of them in word 2 p + w, bits 16 h + 4 f.  Behind the codes fp16 scales and offsets: K per row 4 scales, then 4
# offsets; V per four rows and group 4 scales, then 4 offsets.

def _quantize(x):
    """float32 [..., 128] -> codes int32 [..., 128], scales and offsets float16 [..., 4]."""
    x = x.unflatten(-1, (4, GROUP))
    mn, mx = x.amin(-1) + 0.0, x.amax(-1)
    s, m = ((mx - mn) / 15.0).half(), mn.half()
    sf, mf = s.float().unsqueeze(-1), m.float().unsqueeze(-1)
    c = torch.where(sf == 0, torch.zeros_like(x), ((x - mf) / sf).round().clamp(0.0, 15.0))
    return c.to(torch.int32).flatten(-2), s, m


def _values(codes, s, m):
    return (codes.unflatten(-1, (4, GROUP)).float() * s.float().unsqueeze(-1) + m.float().unsqueeze(-1)).flatten(-2)


def _word_shifts(device):
    f, h = torch.arange(4, device=device), torch.arange(2, device=device)
    return (4 * f).view(4, 1, 1) + (16 * h).view(1, 1, 2)             # [f, w, h]


def _to_words(codes):
    """codes [..., 32] -> int32 words [..., 4]."""
    c = codes.long().unflatten(-1, (2, 4, 2, 2))                      # [p, f, w, h]
    v = (c << _word_shifts(c.device)).sum(dim=(-3, -1)).flatten(-2)   # [p, w]
    return (v - ((v >> 31) << 32)).to(torch.int32)


def _from_words(words):
    """int32 words [..., 4] -> codes [..., 32]."""
    w = words.unflatten(-1, (2, 2))[..., :, None, :, None]            # [p, ., w, .]
    return ((w >> _word_shifts(words.device)) & 15).flatten(-4)


def _pack(rows, side):
    """float32 rows [items, slots, 128], slots a multiple of 64 -> tiles uint8 [items, tiles, TILE_BYTES]."""
    codes, s, m = _quantize(rows.unflatten(1, (-1, TILE)))
    if side == "k":
        words = _to_words(codes.unflatten(-1, (4, GROUP)))                                    # [items, tiles, 64 lanes, 4, 4]
        meta = torch.cat([s, m], -1)
    else:
        lanes = codes.unflatten(2, (2, 32)).unflatten(-1, (4, GROUP)).permute(0, 1, 2, 5, 4, 3)
        words = _to_words(lanes.flatten(2, 3))
        meta = torch.cat([t.unflatten(2, (16, 4)).transpose(-1, -2) for t in (s, m)], -1)     # [items, tiles, 16, 4 groups, 8]
    words = words.transpose(2, 3).contiguous().view(torch.uint8).flatten(2)
    return torch.cat([words, meta.contiguous().view(torch.uint8).flatten(2)], -1)


def _unpack(tiles, side):
    """tiles uint8 [items, tiles, TILE_BYTES] -> float32 rows [items, slots, 128]."""
    words = tiles[..., :4096].contiguous().view(torch.int32).unflatten(-1, (4, TILE, 4)).transpose(2, 3)      # [items, tiles, 64, 4, 4]
    meta = tiles[..., 4096:].contiguous().view(torch.float16)
    codes = _from_words(words)                                                                # [items, tiles, 64, 4, 32]
    if side == "k":
        codes, meta = codes.flatten(-2), meta.unflatten(-1, (TILE, 8))
        s, m = meta[..., :4], meta[..., 4:]
    else:
        codes = codes.unflatten(2, (2, 32)).permute(0, 1, 2, 5, 4, 3).flatten(-2).flatten(2, 3)
        meta = meta.unflatten(-1, (16, 4, 8)).transpose(-1, -2)                               # [items, tiles, 16, 8, 4 groups]
        s, m = meta[..., :4, :].flatten(2, 3), meta[..., 4:, :].flatten(2, 3)
    return _values(codes, s, m).flatten(1, 2)


# ---- inputs ----------------------------------------------------------------------------------------------------------------------

def _rows(n, T, gen, outliers):
    """bf16 [n, T, 128]: normal; K has three channels per item ten times larger."""
    x = torch.randn((n, T, D), generator=gen, device="cuda", dtype=torch.bfloat16)
    if outliers:
        ch = torch.rand((n, D), generator=gen, device="cuda").topk(3, dim=-1).indices
        x *= torch.ones((n, 1, D), device="cuda", dtype=torch.bfloat16).scatter_(2, ch[:, None], 10.0)
    return x


def _held(case, gen, outliers):
    """One side of a cache that has been filled: bf16 [batch, hkv, capacity, 128], or 4-bit tiles [batch, hkv, tiles, TILE_BYTES]."""
    hkv, cap = case["hkv"], case["capacity"]
    parts = []
    for _ in range(case["batch"]):
        x = _rows(hkv, cap, gen, outliers)
        if case["bits"] == 4:
            x = _pack(torch.nn.functional.pad(x.float(), (0, 0, 0, -cap % TILE)), "k" if outliers else "v")
        parts.append(x)
    return torch.stack(parts)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    batch, hq, hkv, cap, op, n = case["batch"], case["hq"], case["hkv"], case["capacity"], case["op"], case["drafted"]
    items = batch * hkv
    st = {"case": case}
    slopes = [2.0 ** (-8.0 * (h + 1) / hq) for h in range(hq)] if case["bias"] else None
    st["slopes"] = torch.tensor(slopes, device="cuda", dtype=torch.float32) if slopes else None
    if op == "prompt":
        st["seq_lens"] = lens = _lens(case)
        total = sum(lens)
        if case["tokens"]:
            qkv = _rows(total, hq + 2 * hkv, gen, False)
            ch = torch.rand((hkv, D), generator=gen, device="cuda").topk(3, dim=-1).indices
            qkv[:, hq:hq + hkv] *= torch.ones((hkv, D), device="cuda", dtype=torch.bfloat16).scatter_(1, ch, 10.0)
            st["Q"], st["K"], st["V"] = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
        else:
            st["Q"], st["K"], st["V"] = (_rows(1, total * h, gen, out).view(-1) for h, out in ((hq, False), (hkv, True), (hkv, False)))
        torch.cuda.synchronize()
        return st
    st["k"], st["v"] = _held(case, gen, True), _held(case, gen, False)
    lens = torch.tensor(_lens(case), device="cuda", dtype=torch.int32).view(batch, 1).expand(batch, hkv).contiguous()
    st["lens"] = lens
    # positions: every third token or so was kept, the newest ones are together, and slots were used again in no order
    at = torch.arange(cap, device="cuda", dtype=torch.int32)
    kept = torch.where(at < case["sinks"], at, at * 3 + torch.randint(0, 3, (items, cap), generator=gen, device="cuda", dtype=torch.int32))
    flat = lens.view(items, 1)
    newest = kept.gather(1, (flat - 1).long())
    kept = torch.where(at >= flat - case["recent"], newest - (flat - 1 - at), kept)
    order = torch.rand((items, cap), generator=gen, device="cuda").masked_fill_(at >= flat, 2.0).argsort(1)
    st["pos"] = kept.gather(1, order).to(torch.int32).view(batch, hkv, cap)
    # (one next position for the items of a sequence, as where all of them have seen the same tokens)
    st["next"] = (newest + 1).view(batch, hkv).amax(1, keepdim=True).expand(batch, hkv).to(torch.int32).contiguous()
    st["weight"] = torch.randn((batch, hkv, cap), generator=gen, device="cuda").mul_(2.0).exp_()
    st["q"] = torch.randn((batch, n, hq, D), generator=gen, device="cuda", dtype=torch.bfloat16)
    st["k_draft"] = _rows(items, n, gen, True).view(batch, hkv, n, D).transpose(1, 2).contiguous()
    st["v_draft"] = _rows(items, n, gen, False).view(batch, hkv, n, D).transpose(1, 2).contiguous()
    parents, counts, paths = _trees(case)
    st["parent"] = torch.tensor(parents, device="cuda", dtype=torch.int32)
    st["counts"] = torch.tensor(counts, device="cuda", dtype=torch.int32) if case["padded"] else None
    sees = torch.zeros((batch, n, n), dtype=torch.bool)          # [token, drafted token that it sees]
    for s in range(batch):
        for i in range(n):
            sees[s, i, _up(parents[s], i)] = True
    st["sees"] = sees.cuda()
    st["live"] = (torch.arange(n).view(1, n) < torch.tensor(counts).view(batch, 1)).cuda()
    st["out"] = torch.zeros((batch, n, hq, D), device="cuda", dtype=torch.bfloat16)
    st["stats"] = torch.zeros((batch, n, hq, 2), device="cuda")
    if op == "accept":
        st["path"] = torch.tensor(paths, device="cuda", dtype=torch.int32)
        st["stats"] = _stats(*_scores(st))[0]
    torch.cuda.synchronize()
    return st


# ---- the plain forms ---------------------------------------------------------------------------------------------------------------

def _capped(case, x):
    return case["cap"] * torch.tanh(x / case["cap"]) if case["cap"] > 0 else x


def _softmax(x):
    """Largest, sum of exponentials of what is left, and those: of nothing 0."""
    top = x.amax(-1, keepdim=True)
    p = torch.exp(x - torch.where(top == -math.inf, torch.zeros_like(top), top))
    return top, p.sum(-1, keepdim=True), p


def _plain_prompt(st):
    case = st["case"]
    batch, hq, hkv, lens = case["batch"], case["hq"], case["hkv"], st["seq_lens"]
    g, longest, total = hq // hkv, max(lens), sum(lens)
    T = torch.tensor(lens, device="cuda")
    first = (torch.cumsum(T, 0) - T).view(batch, 1, 1)
    at = torch.arange(longest, device="cuda").view(1, 1, longest)
    inside = at < T.view(batch, 1, 1)

    def rows(heads):                                                  # [batch, heads, longest]: where a row is, of ragged blocks or of tokens
        h, t = torch.arange(heads, device="cuda").view(1, heads, 1), torch.where(inside, at, 0)
        return first * heads + h * T.view(batch, 1, 1) + t, (first + t).expand(batch, heads, longest), h.expand(batch, heads, longest)

    def padded(x, heads):
        ragged, token, head = rows(heads)
        return (x[token, head] if case["tokens"] else x.view(-1, D)[ragged]).float()

    q, k, v = padded(st["Q"], hq).unflatten(1, (hkv, g)), padded(st["K"], hkv).transpose(2, 3).contiguous(), padded(st["V"], hkv)
    out, lse = torch.empty_like(q), torch.empty(q.shape[:-1], device="cuda")
    step = max(16, min(longest, BLOCK // (batch * hq * longest)))
    for t0 in range(0, longest, step):                                # (all scores at once do not fit the card)
        t1 = min(t0 + step, longest)
        away = torch.arange(t0, t1, device="cuda").view(-1, 1) - torch.arange(t1, device="cuda")
        seen = away >= 0
        if case["window"] > 0:
            seen &= (away < case["window"]) | (torch.arange(t1, device="cuda") < case["sinks"])
        x = torch.matmul(q[:, :, :, t0:t1].reshape(batch, hkv, -1, D), k[..., :t1]).div_(math.sqrt(D)).view(batch, hkv, g, t1 - t0, t1)
        x = _capped(case, x)
        if st["slopes"] is not None:
            x = x - st["slopes"].view(hkv, g, 1, 1) * away.float()
        top, sums, p = _softmax(x.masked_fill_(~seen, -math.inf))
        out[:, :, :, t0:t1] = torch.matmul(p.div_(sums).view(batch, hkv, -1, t1), v[:, :, :t1]).view(batch, hkv, g, t1 - t0, D)
        lse[:, :, :, t0:t1] = (top + torch.log(sums)).squeeze(-1)
    ragged, token, head = rows(hq)
    keep = inside.expand(batch, hq, longest)
    out, lse = out.flatten(1, 2)[keep].to(torch.bfloat16), lse.flatten(1, 2)[keep]
    flat_lse = torch.empty(total * hq, device="cuda")
    flat_lse[ragged[keep]] = lse
    if case["tokens"]:
        laid = torch.empty((total, hq, D), device="cuda", dtype=torch.bfloat16)
        laid[token[keep], head[keep]] = out
        return [laid, flat_lse]
    laid = torch.empty((total * hq, D), device="cuda", dtype=torch.bfloat16)
    laid[ragged[keep]] = out
    return [laid.view(-1), flat_lse]


def _values_of(st, side):
    """float32 [items, capacity, 128]."""
    case = st["case"]
    held = st[side].flatten(0, 1)
    return held.float() if case["bits"] == 16 else _unpack(held, side)[:, :case["capacity"]]


def _scores(st):
    """Of every drafted token and head with the slots [items, n, g, capacity] and with the drafted tokens [items, n, g, n], -inf where hidden."""
    case = st["case"]
    batch, hq, hkv, cap, n = case["batch"], case["hq"], case["hkv"], case["capacity"], case["drafted"]
    g, items = hq // hkv, batch * hkv
    lens, pos, nxt = st["lens"].view(items, 1, 1), st["pos"].view(items, 1, cap), st["next"].view(items, 1, 1)
    q = st["q"].float().view(batch, n, hkv, g, D).transpose(1, 2).reshape(items, n * g, D)
    depth = st["sees"].sum(-1).sub(1).repeat_interleave(hkv, 0)                              # [items, n]
    at_q = nxt + depth.unsqueeze(-1)                                                         # [items, n, 1]
    slots = torch.arange(cap, device="cuda").view(1, 1, cap)
    drafted = st["k_draft"].float().transpose(1, 2).reshape(items, n, D)
    got = []
    for keys, where, seen in ((_values_of(st, "k"), pos, (slots < lens).expand(items, n, cap)),
                              (drafted, (nxt.squeeze(-1) + depth).unsqueeze(1), st["sees"].repeat_interleave(hkv, 0))):
        x = torch.matmul(q, keys.transpose(1, 2).contiguous()).div_(math.sqrt(D)).view(items, n, g, -1)
        x = _capped(case, x)
        away = at_q - where
        if st["slopes"] is not None:
            x = x - st["slopes"].view(1, hkv, 1, g, 1).expand(batch, hkv, 1, g, 1).reshape(items, 1, g, 1) * away.float().unsqueeze(2)
        if case["window"] > 0:
            seen = seen & ((away < case["window"]) | (where < case["sinks"]))
        got.append(x.masked_fill_(~seen.unsqueeze(2), -math.inf))
    return st, got[0], got[1]


def _tokenwise(st, x):
    """[items, n, g, ...] -> [batch, n, hq, ...]."""
    case = st["case"]
    return x.unflatten(0, (case["batch"], case["hkv"])).transpose(1, 2).flatten(2, 3)


def _stats(st, x, y):
    """(largest score, sum of exponentials of what is left) float32 [batch, n, hq, 2], and the exponentials."""
    top = torch.maximum(x.amax(-1, keepdim=True), y.amax(-1, keepdim=True))
    ref = torch.where(top == -math.inf, torch.zeros_like(top), top)
    px, py = torch.exp(x - ref), torch.exp(y - ref)
    total = px.sum(-1, keepdim=True) + py.sum(-1, keepdim=True)
    return _tokenwise(st, torch.cat([top, total], -1)), px, py, total


def _plain_tree(st):
    case = st["case"]
    stats, px, py, total = _stats(*_scores(st))
    items, n, g, cap = px.shape
    v_draft = st["v_draft"].float().transpose(1, 2).reshape(items, n, D)
    out = torch.matmul(px.view(items, n * g, cap), _values_of(st, "v")) + torch.matmul(py.view(items, n * g, n), v_draft)
    out = out.view(items, n, g, D) / torch.where(total == 0, torch.ones_like(total), total)
    live = st["live"].view(case["batch"], n, 1, 1)
    st["out"].copy_(torch.where(live, _tokenwise(st, out).to(torch.bfloat16), st["out"]))
    st["stats"].copy_(torch.where(live, stats, st["stats"]))
    return [st["out"], st["stats"]]


def _on_path(st):
    """The state with the path's tokens in the place of all, and which of them there are [batch, accepted]."""
    case = st["case"]
    m = case["accepted"]
    path = st["path"].long()
    there = torch.cumprod((path >= 0).int(), 1).bool()
    at = torch.where(there, path, 0)
    batch = torch.arange(case["batch"], device="cuda").view(-1, 1)
    sees = torch.ones((m, m), device="cuda", dtype=torch.bool).tril().expand(case["batch"], m, m)
    short = dict(st, case=dict(case, drafted=m), sees=sees, **{x: st[x][batch, at] for x in ("q", "k_draft", "v_draft", "stats")})
    return short, there


def _plain_accept(st):
    case = st["case"]
    batch, hq, hkv, cap, m = case["batch"], case["hq"], case["hkv"], case["capacity"], case["accepted"]
    items, g = batch * hkv, hq // hkv
    short, there = _on_path(st)
    _, x, y = _scores(short)
    top, total = (t.unsqueeze(-1) for t in short["stats"].view(batch, m, hkv, g, 2).transpose(1, 2).reshape(items, m, g, 2).unbind(-1))
    top, total = torch.where(top == -math.inf, 0.0, top), torch.where(total == 0, 1.0, total)
    count = there.sum(1).repeat_interleave(hkv).view(items, 1)                               # tokens that come
    j = torch.arange(m, device="cuda")
    factor = torch.where(j < count, float(case["decay"]) ** (count - 1 - j).clamp(min=0).double(), 0.0).float().view(items, m, 1, 1)
    given = (torch.exp(x - top) / total * factor).sum((1, 2))                                # [items, capacity]
    own_weight = (torch.exp(y - top) / total * factor).sum((1, 2))                           # [items, accepted]
    lens, nxt, pos, weight = st["lens"].view(items, 1), st["next"].view(items, 1), st["pos"].view(items, cap), st["weight"].view(items, cap)
    live = torch.arange(cap, device="cuda") < lens
    weight.copy_(torch.where(live, (float(case["decay"]) ** count.double()).float() * weight + given, weight))
    item = torch.arange(items, device="cuda")
    slots = torch.full((items, m), -1, device="cuda", dtype=torch.int64)
    for t in range(m):                                                                       # (each append sees what the one before left)
        comes = t < count
        may = (pos >= case["sinks"]) & (pos <= nxt - case["recent"])
        w = torch.where(may, weight, math.inf)
        lowest = (w == w.amin(1, keepdim=True)) & may
        gone = torch.where(lowest, pos, 2 ** 31 - 1).argmin(1, keepdim=True)
        slot = torch.where(lens < cap, lens.long(), gone)
        slots[:, t:t + 1] = torch.where(comes, slot, -1)
        pos.scatter_(1, slot, torch.where(comes, nxt, pos.gather(1, slot)))
        weight.scatter_(1, slot, torch.where(comes, own_weight[:, t:t + 1], weight.gather(1, slot)))
        _put(st, item, slot.view(-1), comes.view(-1), *(short[x + "_draft"][:, t].reshape(items, D) for x in ("k", "v")))
        lens.copy_(torch.where(comes, (lens + 1).clamp(max=cap), lens))
        nxt.copy_(torch.where(comes, nxt + 1, nxt))
    slots = slots.to(torch.int32).view(batch, hkv, m)
    return _accepted(st, slots, _plain_read(st, slots) if case["bits"] == 4 else [st["k"], st["v"]])


def _put(st, item, slot, comes, k_new, v_new):
    """Rows [items, 128] into a slot of each item, where one comes."""
    item, slot, k_new, v_new = item[comes], slot[comes], k_new[comes], v_new[comes]
    if st["case"]["bits"] == 16:
        st["k"].flatten(0, 1)[item, slot] = k_new
        st["v"].flatten(0, 1)[item, slot] = v_new
        return
    tile, r = slot // TILE, slot % TILE
    lane, group = torch.arange(32, device=slot.device), torch.arange(4, device=slot.device)
    for side, new in (("k", k_new), ("v", v_new)):
        held = st[side].flatten(0, 1)
        words, halves = held.view(torch.int32), held.view(torch.float16)
        codes, sc, of = _quantize(new.float())
        if side == "k":
            at = (256 * group).view(1, 4, 1) + 4 * r.view(-1, 1, 1) + group.view(1, 1, 4)
            words[item.view(-1, 1, 1), tile.view(-1, 1, 1), at] = _to_words(codes.unflatten(-1, (4, GROUP)))
            at = 2048 + 8 * r.view(-1, 1) + group
        else:
            c = r % 32                       # code 16 p + 4 f + 2 w + h of the lane's 32
            at = (256 * group).view(1, 4, 1) + 4 * (32 * (r // 32)).view(-1, 1, 1) + 4 * lane + (2 * (c // 16) + c // 2 % 2).view(-1, 1, 1)
            shift = (16 * (c % 2) + 4 * (c // 4 % 4)).view(-1, 1, 1)
            i, t = item.view(-1, 1, 1), tile.view(-1, 1, 1)
            old = words[i, t, at].long() & 0xFFFFFFFF
            new = (old & ~(15 << shift)) | (codes.unflatten(-1, (4, GROUP)).long() << shift)
            words[i, t, at] = (new - ((new >> 31) << 32)).to(torch.int32)
            at = 2048 + (32 * (r // 4) + r % 4).view(-1, 1) + 8 * group
        halves[item.view(-1, 1), tile.view(-1, 1), at] = sc
        halves[item.view(-1, 1), tile.view(-1, 1), at + 4] = of


def _plain_read(st, index):
    """bf16 rows of slots index [batch, hkv, m]; zeros where an index is negative."""
    batch, hkv = st["case"]["batch"], st["case"]["hkv"]
    at = index.clamp(min=0).long().flatten(0, 1).unsqueeze(-1)
    got = []
    for side in ("k", "v"):
        held = st[side].flatten(0, 1).gather(1, (at // TILE).expand(-1, -1, TILE_BYTES))
        rows = _unpack(held, side).unflatten(1, (-1, TILE)).gather(2, (at % TILE).unsqueeze(-1).expand(-1, -1, 1, D)).squeeze(2)
        got.append(torch.where((index >= 0).unsqueeze(-1), rows.to(torch.bfloat16).unflatten(0, (batch, hkv)), 0))
    return got


def _accepted(st, slot, rows):
    return [slot, *rows, st["pos"], st["weight"], st["lens"], st["next"]]


# ---- the library's calls -------------------------------------------------------------------------------------------------------------

def _slots(st):
    """The handle over the state's tensors, and the workspace of its steps, made once as a program makes them."""
    if "slots" not in st:
        from paper_2605_08317_amd import binding as b
        case = st["case"]
        st["b"] = b
        st["slots"] = b.Slots(case["batch"], case["hq"], case["hkv"], case["capacity"], bits=case["bits"], sinks=case["sinks"],
                              recent=case["recent"], window=case["window"], score_cap=case["cap"], decay=case["decay"],
                              slopes=st["slopes"], k=st["k"], v=st["v"], pos=st["pos"], weight=st["weight"], lens=st["lens"],
                              next_pos=st["next"])
        st["workspace"] = st["slots"].tree_workspace(case["drafted"]) if case["op"] == "tree" else None
    return st["b"], st["slots"]


def run(st):
    case = st["case"]
    op = case["op"]
    if not own:
        return _plain_prompt(st) if op == "prompt" else _plain_tree(st) if op == "tree" else _plain_accept(st)
    if op == "prompt":
        from paper_2605_08317_amd import binding as b
        return list(b.rdkv_prompt_attn_bf16(st["Q"], st["K"], st["V"], st["seq_lens"], case["hq"], case["hkv"], window=case["window"],
                                            sinks=case["sinks"], score_cap=case["cap"], slopes=st["slopes"]))
    b, slots = _slots(st)
    if op == "tree":
        return list(b.rdkv_slots_tree_attn(slots, st["q"], st["k_draft"], st["v_draft"], st["parent"], counts=st["counts"], out=st["out"],
                                           stats=st["stats"], workspace=st["workspace"]))
    # (the statistics of one head a KV head come from the plain form in another order)
    slot = b.rdkv_slots_accept(slots, st["q"], st["k_draft"], st["v_draft"], st["path"], st["stats"].contiguous())
    return _accepted(st, slot, b.rdkv_slots_read(slots, slot) if case["bits"] == 4 else [st["k"], st["v"]])


def work(case):
    """Bytes: every input once, every output once; what a window hides is not counted.  Flops: of pairs that are seen."""
    hkv, hq, batch, bits, n = case["hkv"], case["hq"], case["batch"], case["bits"], case["drafted"]
    window = case["window"]
    if case["op"] == "prompt":
        pairs = 0
        for T in _lens(case):
            pairs += T * (T + 1) // 2
            if 0 < window < T:
                pairs -= (T - window) * (T - window + 1) // 2
        total = sum(_lens(case))
        return {"bytes": total * (4 * hq * D + 4 * hkv * D + 4 * hq), "flops": 4 * D * hq * pairs}
    side = 2 * D if bits == 16 else D // 2 + 16                       # K, or V, of a slot
    _, counts, paths = _trees(case)
    lens, where = _lens(case), 4 if window or case["bias"] else 0
    seen = [min(T, window // 3 + 1) if window else T for T in lens]
    if case["op"] == "tree":
        rows = sum(counts) * hq
        return {"bytes": sum(seen) * hkv * (2 * side + where) + rows * (4 * D + 8) + sum(counts) * hkv * 4 * D,
                "flops": 4 * D * hq * sum(c * s for c, s in zip(counts, seen))}
    m = [sum(i >= 0 for i in p) for p in paths]
    touched = sum(s for s, c in zip(seen, m) if c) * hkv
    full = sum(T for T, c in zip(lens, m) if c and T + c > case["capacity"]) * hkv           # positions that decide who goes
    back = sum(m) * hkv * (2 * side + 4 * D) if bits == 4 else 0
    return {"bytes": touched * (side + 8 + where) + (0 if where else full * 4) + sum(m) * (hq * (2 * D + 8) + hkv * (4 * D + 2 * side)) + back,
            "flops": 2 * D * hq * sum(c * s for c, s in zip(m, seen))}


# ---- 64 bits --------------------------------------------------------------------------------------------------------------------------

def _exact_rows(st, side, item, slots):
    """float64 [slots, 128] of one item's slots, code by code from the bytes."""
    case = st["case"]
    held = st[side].flatten(0, 1)[item]
    if case["bits"] == 16:
        return held[slots].double()
    t, r = (slots // TILE).unsqueeze(1), (slots % TILE).unsqueeze(1)
    c = torch.arange(D, device=held.device).unsqueeze(0)
    lane, k = (r, c % 32) if side == "k" else (32 * (r // 32) + c % 32, r % 32)
    word = 4 * (c // 32) + 2 * (k // 16) + (k // 2) % 2
    bit = 16 * (k % 2) + 4 * ((k // 4) % 4)
    byte = held[t, 1024 * (word // 4) + 16 * lane + 4 * (word % 4) + bit // 8].to(torch.int32)
    code = ((byte >> (bit % 8)) & 15).double()
    at = 8 * r + c // 32 if side == "k" else 32 * (r // 4) + 8 * (c // 32) + r % 4
    meta = held[:, 4096:].contiguous().view(torch.float16)
    return code * meta[t, at].double() + meta[t, at + 4].double()


def _exact_scores(case, q, k, slopes, away, sees, place):
    """float64 [g, queries, keys] of one item: q [g, queries, 128], k [keys, 128]; away, sees [queries, keys], place [keys]: positions."""
    x = q @ k.t() / math.sqrt(D)
    if case["cap"]:
        x = case["cap"] * torch.tanh(x / case["cap"])
    if slopes is not None:
        x = x - slopes.view(-1, 1, 1) * away
    if case["window"]:
        sees = sees & ((away < case["window"]) | (place < case["sinks"]))
    return torch.where(sees, x, -math.inf)


def _exact_prompt(case, st):
    hq, hkv, lens = case["hq"], case["hkv"], st["seq_lens"]
    g, total = hq // hkv, sum(lens)
    outs, lses, token0 = [], [], 0
    for T in lens:
        def of(x, heads, h):
            return (x[token0:token0 + T, h] if case["tokens"] else x.view(-1, D)[(token0 * heads + h * T):(token0 * heads + h * T) + T]).double()
        out = torch.empty((hq, T, D), device="cuda", dtype=torch.float64)
        lse = torch.empty((hq, T), device="cuda", dtype=torch.float64)
        for h in range(hkv):
            q = torch.stack([of(st["Q"], hq, h * g + i) for i in range(g)])
            k, v = of(st["K"], hkv, h), of(st["V"], hkv, h)
            step = max(1, (1 << 27) // (g * T))
            for t0 in range(0, T, step):
                t1 = min(T, t0 + step)
                lo = max(0, t0 - case["window"] + 1) if case["window"] else 0
                keys = torch.cat([torch.arange(min(lo, case["sinks"])), torch.arange(lo, t1)]).cuda()
                away = torch.arange(t0, t1, device="cuda").unsqueeze(1) - keys
                x = _exact_scores(case, q[:, t0:t1], k[keys], None if st["slopes"] is None else st["slopes"][h * g:h * g + g].double(), away, away >= 0, keys)
                lse[h * g:h * g + g, t0:t1] = torch.logsumexp(x, -1)
                out[h * g:h * g + g, t0:t1] = torch.softmax(x, -1) @ v[keys]
        outs.append(out.transpose(0, 1) if case["tokens"] else out.reshape(-1))
        lses.append(lse.reshape(-1))
        token0 += T
    return [torch.cat(outs), torch.cat(lses)]


def _exact_item(case, st, i, tokens, depth, sees):
    """float64 scores [g, tokens, slots in use + tokens] of one item for `tokens` of its sequence, at positions next + depth."""
    hq, hkv, cap = case["hq"], case["hkv"], case["capacity"]
    g, s, h = hq // hkv, i // hkv, i % hkv
    slots = torch.arange(int(st["lens"].view(-1)[i]), device="cuda")
    k = torch.cat([_exact_rows(st, "k", i, slots), st["k_draft"][s, tokens, h].double()])
    nxt = st["next"].view(-1)[i].long()
    place = torch.cat([st["pos"].view(-1, cap)[i, slots].long(), nxt + depth])
    away = (nxt + depth).unsqueeze(1) - place
    sees = torch.cat([torch.ones((len(tokens), len(slots)), device="cuda", dtype=torch.bool), sees], 1)
    slopes = None if st["slopes"] is None else st["slopes"][h * g:h * g + g].double()
    return slots, _exact_scores(case, st["q"][s, tokens][:, h * g:h * g + g].double().transpose(0, 1), k, slopes, away, sees, place)


def _exact_tree(case, st):
    hkv, g, n = case["hkv"], case["hq"] // case["hkv"], case["drafted"]
    out = torch.zeros(st["out"].shape, device="cuda", dtype=torch.float64)
    stats = torch.zeros(st["stats"].shape, device="cuda", dtype=torch.float64)
    parents, counts, _ = _trees(case)
    for s in range(case["batch"]):
        tokens = torch.arange(counts[s], device="cuda")
        ways = [_up(parents[s], t) for t in range(counts[s])]
        depth = torch.tensor([len(w) - 1 for w in ways], device="cuda")
        sees = torch.tensor([[u in w for u in range(counts[s])] for w in ways], device="cuda")
        for h in range(hkv):
            slots, x = _exact_item(case, st, s * hkv + h, tokens, depth, sees)
            top = x.amax(-1)
            e = torch.exp(x - torch.where(top == -math.inf, 0.0, top).unsqueeze(-1))
            total = e.sum(-1)
            v = torch.cat([_exact_rows(st, "v", s * hkv + h, slots), st["v_draft"][s, tokens, h].double()])
            got = (e / torch.where(total == 0, 1.0, total).unsqueeze(-1)) @ v
            out[s, :counts[s], h * g:h * g + g] = got.transpose(0, 1)
            stats[s, :counts[s], h * g:h * g + g] = torch.stack([top, total], -1).transpose(0, 1)
    return [out, stats]


def _exact_accept(case, st):
    batch, hkv, cap, m, g = case["batch"], case["hkv"], case["capacity"], case["accepted"], case["hq"] // case["hkv"]
    paths = [[i for i in p if i >= 0] for p in _trees(case)[2]]
    weight = st["weight"].view(-1, cap).double()
    held = None if case["bits"] == 4 else [st[x].flatten(0, 1).double() for x in ("k", "v")]
    rows = [torch.zeros((batch * hkv, m, D), device="cuda", dtype=torch.float64) for _ in range(2)]
    for i in range(batch * hkv):
        s, h = i // hkv, i % hkv
        c = len(paths[s])
        if c == 0:
            continue
        tokens, depth = torch.tensor(paths[s], device="cuda"), torch.arange(c, device="cuda")
        slots, x = _exact_item(case, st, i, tokens, depth, depth.unsqueeze(1) >= depth)
        top, total = st["stats"][s, tokens][:, h * g:h * g + g].double().transpose(0, 1).unbind(-1)
        p = torch.exp(x - torch.where(top == -math.inf, 0.0, top).unsqueeze(-1)) / torch.where(total == 0, 1.0, total).unsqueeze(-1)
        p = (p.sum(0) * (float(case["decay"]) ** (c - 1 - depth).double()).unsqueeze(1)).sum(0)
        used = len(slots)
        weight[i, :used] = float(case["decay"]) ** c * weight[i, :used] + p[:used]
        pos, nxt = st["pos"].view(-1, cap)[i].long().clone(), int(st["next"].view(-1)[i])
        new = [st[x + "_draft"][s, tokens, h].double() for x in ("k", "v")]
        for t in range(c):
            slot = used + t
            if slot >= cap:
                may = ((pos >= case["sinks"]) & (pos <= nxt + t - case["recent"])).nonzero().view(-1)
                may = may[weight[i, may] == weight[i, may].min()]
                slot = int(may[pos[may].argmin()])
            pos[slot], weight[i, slot] = nxt + t, p[used + t]
            for side in range(2):
                x = new[side][t]
                if held is not None:
                    held[side][i, slot] = x
                    continue
                x = x.unflatten(0, (4, GROUP))
                low, high = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
                sc, of = ((high - low) / 15).float().half().double(), low.half().double()
                rows[side][i, t] = (torch.where(sc > 0, torch.round((x - of) / torch.where(sc > 0, sc, 1.0)).clamp(0, 15), 0.0) * sc + of).flatten()
    sides = [x.view(batch, hkv, m, D) for x in rows] if held is None else [x.view(batch, hkv, cap, D) for x in held]
    return [None, *sides, None, weight.view(batch, hkv, cap), None, None]


def exact(case, seed):
    st = prepare(case, seed)
    return _exact_prompt(case, st) if case["op"] == "prompt" else _exact_tree(case, st) if case["op"] == "tree" else _exact_accept(case, st)
