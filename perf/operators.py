"""The operators of a slot cache as cases that a timing program can prepare and run, and their plain forms.

A slot cache holds `capacity` tokens per (sequence, KV head), an item, however long the generation gets: rows of K and V as bf16 or in
4 bits, and per slot the token's position and the attention weight it has gathered.  A case names what is called ("op"):

  fill     a ragged batch of prompts into the slots; where a prompt is longer than the capacity, the first `sinks` and the last
           `recent` tokens stay, and of the others those of largest weight
  append   one generated token per sequence: into a free slot, or in the place of the token of least weight
  decode   one decode step over the slots (scores capped, biased by distance or masked by a window where the case says so), which adds
           every token's attention weight to its slot
  read     the slots' rows as bf16, all of them or those of an index

`own` False: plain torch operations.  `own` True: the library's calls.  Outputs of 4-bit caches are the values the codes stand for.
"""
import math
import random

import torch

own = False

D = 128
GROUP = 32                       # channels that share a scale and an offset in 4 bits
TILE = 64                        # rows of a 4-bit tile: 4096 bytes of codes, 1024 of scales and offsets
TILE_BYTES = 5120


def _case(op, name=None, *, batch=1, hq=32, hkv=8, capacity, lo=None, bits=16, sinks=4, recent=32, window=0, cap=0.0, bias=False,
          decay=1.0, prompt=0, prompt_lo=None, ties=False, rows=0):
    """lo: the shortest sequence's filled slots (the first sequence has them all); prompt, prompt_lo: tokens of a filled prompt;
    rows: of a read by index."""
    c = {"op": op, "batch": batch, "hq": hq, "hkv": hkv, "capacity": capacity, "lo": capacity if lo is None else lo, "bits": bits,
         "sinks": sinks, "recent": recent, "window": window, "cap": cap, "bias": bias, "decay": decay, "prompt": prompt,
         "prompt_lo": prompt_lo or prompt, "ties": ties, "rows": rows}
    return dict(c, name=name) if name else c


def listed():
    return [
        # The smallest step in earnest: two KV heads of a tensor-parallel shard, a thousand tokens.  Launch latency, host side.
        _case("decode", "decode_tiny_bf16", hq=8, hkv=2, capacity=1000),
        # Batched serving of a 70B-shaped layer, ragged, 8 query heads per KV head, capped scores.
        _case("decode", "decode_batch_capped_bf16", batch=16, hq=64, capacity=4096, lo=1500, cap=30.0),
        # Long contexts kept whole in bf16: the largest cache.
        _case("decode", "decode_long_bf16", batch=4, capacity=131072),
        # A model with linear position biases, 4-bit rows, many sequences, weights that age.
        _case("decode", "decode_batch_biased_4bit", batch=32, capacity=8192, lo=5000, bits=4, bias=True, decay=0.98),
        # Long contexts in 4 bits.
        _case("decode", "decode_long_4bit", batch=4, capacity=131072, lo=90001, bits=4),
        # A prompt of a layer of an 8B-shaped model cut to 4K tokens.
        _case("fill", "fill_prompt_bf16", capacity=4096, prompt=32768),
        # A ragged batch of prompts cut to 4K tokens in 4 bits.
        _case("fill", "fill_batch_4bit", batch=16, capacity=4096, prompt=32768, prompt_lo=2000, bits=4),
        # One long prompt, weights with many ties, a quarter of it kept.
        _case("fill", "fill_long_ties_4bit", capacity=32768, prompt=131072, bits=4, ties=True),
        # A generated token in the smallest cache.
        _case("append", "append_tiny_bf16", hq=8, hkv=2, capacity=1000),
        # A generated token for each of many sequences, some with free slots.
        _case("append", "append_batch_4bit", batch=32, capacity=8192, lo=5000, bits=4),
        # The rows of a 4-bit cache as bf16, for a pass over them that wants rows.
        _case("read", "read_batch_4bit", batch=4, capacity=32768, lo=20001, bits=4),
        # A few rows by index.
        _case("read", "read_rows_bf16", batch=8, capacity=4096, lo=100, rows=65),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["decode", "decode", "decode", "fill", "fill", "append", "read"])
    hkv = rng.choice([1, 2, 4, 8, 8])
    kw = {"hkv": hkv, "hq": hkv * rng.choice([1, 2, 4, 4, 8]), "batch": _log(rng, 1, 48), "bits": rng.choice([4, 16])}
    longest = min(131072, (1 << 22) // (kw["batch"] * hkv))       # slots in all: what the largest listed cache has
    if op in ("fill", "append"):
        longest = min(longest, 32768, (1 << 19) // (kw["batch"] * hkv))
    if op == "read":
        longest = min(longest, 32768, (1 << 20) // (kw["batch"] * hkv))
    kw["capacity"] = max(70, _log(rng, 70, longest) if longest > 70 else 70)
    kw["lo"] = rng.choice([kw["capacity"], rng.randint(1, kw["capacity"])])
    kw["sinks"], kw["recent"] = rng.randint(0, 16), rng.randint(0, 48)
    if op == "decode":
        kw["cap"] = rng.choice([0.0, 0.0, 20.0, 50.0])
        kw["bias"] = rng.random() < 0.3
        kw["decay"] = rng.choice([1.0, 1.0, 0.9])
        if rng.random() < 0.3:
            kw["window"] = rng.randint(1, 2 * kw["capacity"])
    if op == "fill":
        kw["prompt"] = _log(rng, 70, min(131072, (1 << 22) // (kw["batch"] * hkv)))
        kw["prompt_lo"] = rng.choice([kw["prompt"], rng.randint(1, kw["prompt"])])
        kw["ties"] = rng.random() < 0.3
    if op == "read" and rng.random() < 0.5:
        kw["rows"] = _log(rng, 1, kw["capacity"])
    return _case(op, **kw)


def _ragged(case, lo, hi):
    """A length of every sequence: part of the case, the same for every seed."""
    rng = random.Random("%d %d %d" % (case["batch"], lo, hi))
    return [hi] + [rng.randint(lo, hi) for _ in range(case["batch"] - 1)]


def _lens(case):
    return _ragged(case, case["lo"], case["capacity"])


def _prompts(case):
    return _ragged(case, case["prompt_lo"], case["prompt"])


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


def _lanes_k(x):         # [..., 64 rows, 128] -> [..., 64 lanes, 4, 32]
    return x.unflatten(-1, (4, GROUP))


def _lanes_v(x):         # the same of V, and back: it is its own inverse on the last three of five axes
    return x.unflatten(-2, (2, 32)).unflatten(-1, (4, GROUP)).permute(*range(x.dim() - 2), -4, -1, -2, -3).flatten(-4, -3)


def _pack(rows, side):
    """float32 rows [items, slots, 128], slots a multiple of 64 -> tiles uint8 [items, tiles, TILE_BYTES]."""
    codes, s, m = _quantize(rows.unflatten(1, (-1, TILE)))
    words = _to_words((_lanes_k if side == "k" else _lanes_v)(codes))                         # [items, tiles, 64, 4, 4]
    if side == "k":
        meta = torch.cat([s, m], -1)
    else:
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
    batch, hq, hkv, cap, op = case["batch"], case["hq"], case["hkv"], case["capacity"], case["op"]
    items = batch * hkv
    st = {"case": case}
    slopes = [2.0 ** (-8.0 * (h + 1) / hq) for h in range(hq)] if case["bias"] else None
    st["slopes"] = torch.tensor(slopes, device="cuda", dtype=torch.float32) if slopes else None
    if op == "fill":
        T = _prompts(case)
        st["seq_lens"] = T
        st["T"] = torch.tensor([t for t in T for _ in range(hkv)], device="cuda")
        st["row0"] = torch.cumsum(st["T"], 0) - st["T"]
        total = sum(T) * hkv
        st["K"], st["V"] = _rows(1, total, gen, True).view(-1), _rows(1, total, gen, False).view(-1)
        w = torch.randn(total, generator=gen, device="cuda").mul_(2.0).exp_()          # attention weights: a long tail
        st["w_tok"] = w.to(torch.bfloat16).float() if case["ties"] else w
        side = (batch, hkv, cap, D) if case["bits"] == 16 else (batch, hkv, -(-cap // TILE), TILE_BYTES)
        kind = torch.bfloat16 if case["bits"] == 16 else torch.uint8
        st["k"], st["v"] = torch.zeros(side, device="cuda", dtype=kind), torch.zeros(side, device="cuda", dtype=kind)
        st["pos"] = torch.full((batch, hkv, cap), -1, device="cuda", dtype=torch.int32)
        st["weight"] = torch.zeros((batch, hkv, cap), device="cuda")
        st["lens"] = torch.zeros((batch, hkv), device="cuda", dtype=torch.int32)
        st["next"] = torch.zeros((batch, hkv), device="cuda", dtype=torch.int32)
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
    st["next"] = (newest + 1).to(torch.int32).view(batch, hkv).contiguous()
    st["weight"] = torch.randn((batch, hkv, cap), generator=gen, device="cuda").mul_(2.0).exp_()
    if op == "decode":
        st["q"] = torch.randn((batch, hq, D), generator=gen, device="cuda", dtype=torch.bfloat16)
    if op == "append":
        st["k_new"] = _rows(items, 1, gen, True).view(batch, hkv, D)
        st["v_new"] = _rows(items, 1, gen, False).view(batch, hkv, D)
    if op == "read" and case["rows"]:
        st["index"] = torch.randint(0, cap, (batch, hkv, case["rows"]), generator=gen, device="cuda", dtype=torch.int32)
    torch.cuda.synchronize()
    return st


# ---- the plain forms ---------------------------------------------------------------------------------------------------------------

def _values_of(st, side):
    """float32 [items, capacity, 128]."""
    case = st["case"]
    held = st[side].flatten(0, 1)
    return held.float() if case["bits"] == 16 else _unpack(held, side)[:, :case["capacity"]]


def _plain_decode(st):
    case = st["case"]
    batch, hq, hkv, cap = case["batch"], case["hq"], case["hkv"], case["capacity"]
    g, items = hq // hkv, batch * hkv
    lens, pos, at_q = st["lens"].view(items, 1), st["pos"].view(items, cap), st["next"].view(items, 1) - 1
    x = torch.matmul(st["q"].float().view(items, g, D), _values_of(st, "k").transpose(1, 2).contiguous()) / math.sqrt(D)
    if case["cap"] > 0:
        x = case["cap"] * torch.tanh(x / case["cap"])
    away = at_q - pos
    if st["slopes"] is not None:
        x = x - st["slopes"].view(1, hkv, g).expand(batch, hkv, g).reshape(items, g, 1) * away.float().unsqueeze(1)
    live = torch.arange(cap, device=pos.device) < lens
    seen = live
    if case["window"] > 0:
        seen = live & ((away < case["window"]) | (pos < case["sinks"]))
    x = x.masked_fill(~seen.unsqueeze(1), -math.inf)
    top = x.amax(-1, keepdim=True)
    p = torch.exp(x - torch.where(top == -math.inf, torch.zeros_like(top), top))
    total = p.sum(-1, keepdim=True)
    lse = (top + torch.log(total)).view(batch, hq)
    p = p / torch.where(total == 0, torch.ones_like(total), total)
    out = torch.matmul(p, _values_of(st, "v")).view(batch, hq, D)
    weight = st["weight"].view(items, cap)
    weight.copy_(torch.where(live, case["decay"] * weight + p.sum(1), weight))
    return [out, lse, st["weight"]]


def _plain_fill(st):
    case = st["case"]
    batch, hkv, cap = case["batch"], case["hkv"], case["capacity"]
    items, T, longest = batch * hkv, st["T"].unsqueeze(1), max(st["seq_lens"])
    at = torch.arange(longest, device=T.device).expand(items, longest)
    w = st["w_tok"][(st["row0"].unsqueeze(1) + at).clamp_(max=st["w_tok"].numel() - 1)]
    always = (at < case["sinks"]) | (at >= T - case["recent"])
    key = torch.where(at < T, torch.where(always, math.inf, w), -math.inf)
    if longest < cap:
        key = torch.nn.functional.pad(key, (0, cap - longest), value=-math.inf)
    order = torch.sort(key, dim=1, descending=True, stable=True).indices[:, :cap]
    n = T.clamp(max=cap)
    rank = torch.arange(cap, device=T.device)
    far = 1 << 30
    pos = torch.where(rank < n, order, far).sort(1).values
    live = rank < n
    at = st["row0"].unsqueeze(1) + torch.where(live, pos, 0)
    sides = [torch.where(live.unsqueeze(-1), st[x].view(-1, D)[at], 0) for x in ("K", "V")]
    for x, rows in zip(("k", "v"), sides):
        held = st[x].flatten(0, 1)
        if case["bits"] == 16:
            held.copy_(torch.where(live.unsqueeze(-1), rows, held))
        else:
            held.copy_(_pack(torch.nn.functional.pad(rows.float(), (0, 0, 0, -cap % TILE)), x))
    st["pos"].copy_(torch.where(live, pos, st["pos"].view(items, cap).long()).view(batch, hkv, cap))
    st["weight"].copy_(torch.where(live, st["w_tok"][at], st["weight"].view(items, cap)).view(batch, hkv, cap))
    st["lens"].copy_(n.view(batch, hkv))
    st["next"].copy_(T.view(batch, hkv))
    return _filled(st, _plain_read(st) if case["bits"] == 4 else [st["k"], st["v"]])


def _filled(st, rows):
    return [*rows, st["pos"], st["weight"], st["lens"], st["next"]]


def _plain_append(st):
    case = st["case"]
    batch, hkv, cap = case["batch"], case["hkv"], case["capacity"]
    items = batch * hkv
    lens, nxt, pos = st["lens"].view(items, 1), st["next"].view(items, 1), st["pos"].view(items, cap)
    weight = st["weight"].view(items, cap)
    may = (pos >= case["sinks"]) & (pos <= nxt - case["recent"])
    w = torch.where(may, weight, math.inf)
    lowest = w == w.amin(1, keepdim=True)
    gone = torch.where(lowest & may, pos, 2 ** 31 - 1).argmin(1, keepdim=True)
    slot = torch.where(lens < cap, lens.long(), gone)
    pos.scatter_(1, slot, nxt)
    weight.scatter_(1, slot, torch.zeros_like(slot, dtype=torch.float32))
    item, s = torch.arange(items, device=slot.device), slot.view(-1)
    if case["bits"] == 16:
        st["k"].flatten(0, 1)[item, s] = st["k_new"].view(items, D)
        st["v"].flatten(0, 1)[item, s] = st["v_new"].view(items, D)
    else:
        tile, r = s // TILE, s % TILE
        lane = torch.arange(32, device=s.device)
        for side in ("k", "v"):
            held = st[side].flatten(0, 1)
            words, halves = held.view(torch.int32), held.view(torch.float16)
            codes, sc, of = _quantize(st[side + "_new"].view(items, D).float())
            group = torch.arange(4, device=s.device)
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
    lens.copy_((lens + 1).clamp(max=cap))
    nxt.add_(1)
    slot = slot.to(torch.int32).view(batch, hkv)
    return _appended(st, slot, _plain_read(st, slot.unsqueeze(-1)) if case["bits"] == 4 else [st["k"], st["v"]])


def _appended(st, slot, rows):
    return [slot, *rows, st["pos"], st["weight"], st["lens"], st["next"]]


def _plain_read(st, index=None):
    case = st["case"]
    batch, hkv, cap = case["batch"], case["hkv"], case["capacity"]
    if index is None:
        index = torch.arange(cap, device="cuda").expand(batch, hkv, cap)
    live = (index >= 0) & (index < st["lens"].unsqueeze(-1))
    at = torch.where(live, index, 0).long().flatten(0, 1).unsqueeze(-1)
    got = []
    for side in ("k", "v"):
        if case["bits"] == 16:
            rows = st[side].flatten(0, 1).gather(1, at.expand(-1, -1, D))
        else:
            # only the tiles that hold a row that is asked for
            few = at.shape[1] * TILE <= cap
            held = st[side].flatten(0, 1)
            if few:
                held = held.gather(1, (at // TILE).expand(-1, -1, TILE_BYTES))
                rows = _unpack(held, side).unflatten(1, (-1, TILE)).gather(2, (at % TILE).unsqueeze(-1).expand(-1, -1, 1, D)).squeeze(2)
            else:
                rows = _unpack(held, side).gather(1, at.expand(-1, -1, D))
            rows = rows.to(torch.bfloat16)
        got.append(torch.where(live.unsqueeze(-1), rows.unflatten(0, (batch, hkv)), 0))
    return got


# ---- the library's calls -------------------------------------------------------------------------------------------------------------

def _slots(st):
    """The handle over the state's tensors, and the workspace of its decode steps, made once as a program makes them."""
    if "slots" not in st:
        from paper_2605_08317_amd import binding as b
        case = st["case"]
        st["b"] = b
        st["slots"] = b.Slots(case["batch"], case["hq"], case["hkv"], case["capacity"], bits=case["bits"], sinks=case["sinks"],
                              recent=case["recent"], window=case["window"], score_cap=case["cap"], decay=case["decay"],
                              slopes=st["slopes"], k=st["k"], v=st["v"], pos=st["pos"], weight=st["weight"], lens=st["lens"],
                              next_pos=st["next"])
        st["workspace"] = st["slots"].workspace() if case["op"] == "decode" else None
    return st["b"], st["slots"]


def run(st):
    op, bits = st["case"]["op"], st["case"]["bits"]
    if not own:
        if op == "decode":
            return _plain_decode(st)
        if op == "fill":
            return _plain_fill(st)
        if op == "append":
            return _plain_append(st)
        return _plain_read(st, st.get("index"))
    b, slots = _slots(st)
    if op == "decode":
        out, lse = b.rdkv_slots_decode_attn(slots, st["q"], workspace=st["workspace"])
        return [out, lse, st["weight"]]
    if op == "fill":
        b.rdkv_slots_fill(slots, st["K"], st["V"], st["seq_lens"], st["w_tok"])
        return _filled(st, b.rdkv_slots_read(slots) if bits == 4 else [st["k"], st["v"]])
    if op == "append":
        slot = b.rdkv_slots_append(slots, st["k_new"], st["v_new"])
        return _appended(st, slot, b.rdkv_slots_read(slots, slot.unsqueeze(-1)) if bits == 4 else [st["k"], st["v"]])
    return list(b.rdkv_slots_read(slots, st.get("index")))


def work(case):
    """Bytes: every input once, every output once; rows that a window hides are not counted."""
    hkv, hq, batch, bits = case["hkv"], case["hq"], case["batch"], case["bits"]
    pair = 4 * D if bits == 16 else 2 * (D // 2 + 16)                 # K and V of a slot
    tokens = sum(_lens(case)) * hkv
    if case["op"] == "decode":
        seen = sum(min(n, case["window"] // 3 + 1) if case["window"] else n for n in _lens(case)) * hkv
        where = 4 if case["window"] or case["bias"] else 0
        return {"bytes": seen * pair + tokens * (8 + where) + batch * hq * (D * (2 + 4) + 4), "flops": seen * 4 * (hq // hkv) * D}
    if case["op"] == "fill":
        prompt, n = sum(_prompts(case)) * hkv, sum(min(t, case["capacity"]) for t in _prompts(case)) * hkv
        back = n * (pair + 4 * D) if bits == 4 else 0                 # the rows read back as bf16
        return {"bytes": prompt * 4 + n * (4 * D + pair + 8) + back, "flops": 0}
    if case["op"] == "append":
        return {"bytes": tokens * 8 + batch * hkv * (4 * D + pair + (4 * D + pair if bits == 4 else 0)), "flops": 0}
    n = case["rows"] * batch * hkv or tokens
    return {"bytes": n * (pair + 4 * D), "flops": 0}


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


def exact(case, seed):
    st = prepare(case, seed)
    batch, hq, hkv, cap, op = case["batch"], case["hq"], case["hkv"], case["capacity"], case["op"]
    g, items = hq // hkv, batch * hkv
    if op == "decode":
        lens = st["lens"].view(-1).tolist()
        out = torch.zeros((items, g, D), device="cuda", dtype=torch.float64)
        lse = torch.full((items, g), -math.inf, device="cuda", dtype=torch.float64)
        weight = st["weight"].view(items, cap).double()
        for i, n in enumerate(lens):
            sl = torch.arange(n, device="cuda")
            x = _exact_rows(st, "k", i, sl) @ st["q"].view(items, g, D)[i].double().t() / math.sqrt(D)       # [n, g]
            if case["cap"]:
                x = case["cap"] * torch.tanh(x / case["cap"])
            dist = st["next"].view(-1)[i].double() - 1 - st["pos"].view(items, cap)[i, :n].double()
            if case["bias"]:
                x -= dist.unsqueeze(1) * st["slopes"].view(hkv, g)[i % hkv].double()
            if case["window"]:
                x[(dist >= case["window"]) & (st["pos"].view(items, cap)[i, :n] >= case["sinks"])] = -math.inf
            lse[i] = torch.logsumexp(x, 0)
            p = torch.exp(x - torch.where(torch.isfinite(lse[i]), lse[i], 0.0))
            out[i] = p.t() @ _exact_rows(st, "v", i, sl)
            weight[i, :n] = case["decay"] * weight[i, :n] + p.sum(1)
        return [out.view(batch, hq, D), lse.view(batch, hq), weight.view(batch, hkv, cap)]
    if op == "read":
        index = st.get("index")
        got = []
        for side in ("k", "v"):
            rows = torch.zeros((items, case["rows"] or cap, D), device="cuda", dtype=torch.float64)
            for i, n in enumerate(st["lens"].view(-1).tolist()):
                sl = index.view(items, -1)[i].long() if index is not None else torch.arange(cap, device="cuda")
                at = (sl < n).nonzero().view(-1)
                rows[i, at] = _exact_rows(st, side, i, sl[at])
            got.append(rows.view(batch, hkv, -1, D))
        return got

    def nearest(x):                    # what 4 bits hold of float64 rows, or the rows
        if case["bits"] == 16:
            return x
        x = x.unflatten(-1, (4, GROUP))
        low, high = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
        s, m = ((high - low) / 15).float().half().double(), low.half().double()
        return (torch.where(s > 0, torch.round((x - m) / torch.where(s > 0, s, 1.0)).clamp(0, 15), 0.0) * s + m).flatten(-2)

    if op == "append":
        new = [nearest(st[x].view(items, D).double()) for x in ("k_new", "v_new")]
        weight = st["weight"].view(items, cap).double()
        held = [None if case["bits"] == 4 else st[x].flatten(0, 1).double() for x in ("k", "v")]
        for i in range(items):
            n, nxt, pos = int(st["lens"].view(-1)[i]), int(st["next"].view(-1)[i]), st["pos"].view(items, cap)[i].long()
            slot = n
            if n == cap:
                may = ((pos >= case["sinks"]) & (pos <= nxt - case["recent"])).nonzero().view(-1)
                may = may[weight[i, may] == weight[i, may].min()]
                slot = int(may[pos[may].argmin()])
            weight[i, slot] = 0.0
            if case["bits"] == 16:
                held[0][i, slot], held[1][i, slot] = new[0][i], new[1][i]
        rows = [x.view(batch, hkv, 1, D) for x in new] if case["bits"] == 4 else [x.view(batch, hkv, cap, D) for x in held]
        return [None, *rows, None, weight.view(batch, hkv, cap), None, None]
    sides = [torch.zeros((items, cap, D), device="cuda", dtype=torch.float64) for _ in range(2)]
    weight = torch.zeros((items, cap), device="cuda", dtype=torch.float64)
    for i in range(items):
        T, row0 = int(st["T"][i]), int(st["row0"][i])
        w = st["w_tok"][row0:row0 + T].double()
        at = torch.arange(T, device="cuda")
        if T > cap:
            always = (at < case["sinks"]) | (at >= T - case["recent"])
            others = (~always).nonzero().view(-1)
            best = others[torch.argsort(-w[others], stable=True)[:cap - int(always.sum())]]
            at = torch.cat([at[always], best]).sort().values
        weight[i, :len(at)] = w[at]
        for x, rows in zip(("K", "V"), sides):
            rows[i, :len(at)] = nearest(st[x].view(-1, D)[row0 + at].double())
    return [*(x.view(batch, hkv, cap, D) for x in sides), None, weight.view(batch, hkv, cap), None, None]
