"""Timed cases of the calls that keep a coded cache bounded: attention through a sliding window with sinks,
attention weights added up per cached token, and the eviction that goes by them.

A case is a dict of plain values.  ``op`` names the call:

  window         cq_decode_attention_window[_paged]: one query token per sequence over the last `window` tokens and
                 the first `n_sink`
  chunk_window   cq_chunk_attention_window[_paged]: the last m tokens of a sequence, each through its own window
  weights        cq_decode_attention_weights[_paged]: decode attention that also adds each cached token's weight to
                 its accumulator
  chunk_weights  cq_chunk_weights[_paged]: the same accumulators from the last m tokens of a prompt, keys only
  evict          cq_select_tokens, then cq_compact_cache[_paged]: the tokens to keep per KV head, and the caches and
                 accumulators moved together, in place or into smaller caches

Formats are CQ-8c8b, 4c8b, 2c8b and 8c10b, 32 query heads x 128 channels over 32 or 8 KV heads.  Codes are skewed
towards low numbers as nearest-centroid codes of real codebooks are, the first four tokens of every
sequence draw weight as the first tokens of a prompt do, and the scores of the others have a standard deviation of 2.
"""
from __future__ import annotations

import math

import torch

own = False

HEAD = 128
Q_HEADS = 32
SCALE = 1.0 / math.sqrt(HEAD)
TILE = 64
DECAY = 0.75


def listed():
    return [
        # one user, one layer's step, a short window: latency
        dict(name="window_8c8b_b1_w512", op="window", c=8, b=8, hkv=32, batch=1, t=1500, window=512, sink=4, paged=False, ragged=False),
        # a serving engine's step: paged pools, grouped queries, ragged lengths, sinks that end inside a tile
        dict(name="window_paged_4c8b_gqa_b24_w2048", op="window", c=4, b=8, hkv=8, batch=24, t=6007, window=2048, sink=70, paged=True, ragged=True),
        # long contexts of which a step sees a few thousand tokens, 4 bits per channel
        dict(name="window_2c8b_b32_w4095", op="window", c=2, b=8, hkv=32, batch=32, t=16384, window=4095, sink=4, paged=False, ragged=False),
        # verification of five speculated tokens per sequence through a window
        dict(name="chunk_window_4c8b_b16_m5_w1024", op="chunk_window", c=4, b=8, hkv=32, batch=16, m=5, t=4096, window=1024, sink=4, paged=False, ragged=False),
        # a later prefill chunk of long prompts through a window
        dict(name="chunk_window_8c8b_b4_m512_w4096", op="chunk_window", c=8, b=8, hkv=32, batch=4, m=512, t=65536, window=4096, sink=4, paged=False, ragged=False),
        # one user's step with its weights: latency
        dict(name="weights_8c8b_b1_ctx2000", op="weights", c=8, b=8, hkv=32, batch=1, t=2000, paged=False, ragged=False),
        # the serving step on paged pools, grouped queries, 10-bit codes and ragged lengths
        dict(name="weights_paged_8c10b_gqa_b24_ctx6007", op="weights", c=8, b=10, hkv=8, batch=24, t=6007, paged=True, ragged=True),
        # long contexts at 1 bit per channel
        dict(name="weights_8c8b_b4_ctx131072", op="weights", c=8, b=8, hkv=32, batch=4, t=131072, paged=False, ragged=False),
        # the last 32 tokens of prompts look back, before the first eviction; grouped queries, ragged
        dict(name="chunk_weights_8c8b_gqa_b2_m32_ctx9001", op="chunk_weights", c=8, b=8, hkv=8, batch=2, m=32, t=9001, paged=False, ragged=True),
        # a chunk of 500 tokens of long prompts adds its weights
        dict(name="chunk_weights_4c8b_gqa_b4_m500_ctx32768", op="chunk_weights", c=4, b=8, hkv=8, batch=4, m=500, t=32768, paged=False, ragged=False),
        # the steady state of a bounded cache: 64 tokens over budget, in place
        dict(name="evict_4c8b_b16_4160_to_4096", op="evict", c=4, b=8, hkv=32, batch=16, t=4160, keep=4096, sink=4, recent=512, paged=False, ragged=False, inplace=True),
        # long prompts leave for small caches after their prefill
        dict(name="evict_8c8b_gqa_b4_131072_to_2047", op="evict", c=8, b=8, hkv=8, batch=4, t=131072, keep=2047, sink=4, recent=32, paged=False, ragged=False, inplace=False),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("window", "chunk_window", "weights", "chunk_weights", "evict"))
    hkv = rng.choice((8, 32))
    c, b = rng.choice(((8, 8), (4, 8), (2, 8), (8, 10)))
    case = dict(op=op, c=c, b=b, hkv=hkv, paged=rng.random() < 0.4, ragged=rng.random() < 0.5)
    t = _log_int(rng, 1, 65536)
    cap = 400_000_000 // (2 * 16 * b * HEAD // (c * HEAD) * hkv * t)        # at most 400 MB of codes
    most = max(1, min(64, cap))
    if op in ("chunk_window", "chunk_weights"):
        m = min(t, _log_int(rng, 1, 600))
        window = _log_int(rng, 1, 8192)
        seen = t if op == "chunk_weights" else min(t, window + m + 128)
        most = max(1, min(most, int(6e9 // (m * seen * Q_HEADS))))           # (query token, cached token, head) triples
        case.update(m=m)
        if op == "chunk_window":
            case.update(window=window, sink=rng.choice((0, 4, rng.randint(0, 200))))
    elif op == "window":
        case.update(window=_log_int(rng, 1, 8192), sink=rng.choice((0, 4, rng.randint(0, 200))))
    elif op == "evict":
        sink, recent = rng.choice((0, 4)), rng.randint(0, 64)
        case.update(keep=max(1, sink + recent, _log_int(rng, 1, t)), sink=sink, recent=recent, inplace=rng.random() < 0.5)
    case.update(batch=_log_int(rng, 1, most), t=t)
    return case


# ---------------------------------------------------------------- inputs

def _gen(seed, salt):
    g = torch.Generator(device="cuda")
    g.manual_seed((int(seed) * 1000003 + salt) % (2 ** 62))
    return g


def _tile_bytes(case):
    return TILE * (HEAD // case["c"]) * case["b"] // 8


def _codes(case, tiles, streams, g):
    """`streams` x `tiles` tiles of random codes as a cache holds them; every byte pattern is a valid tile."""
    shape = (streams, tiles, _tile_bytes(case))
    a = torch.randint(0, 256, shape, generator=g, device="cuda", dtype=torch.uint8)
    r = torch.randint(0, 256, shape, generator=g, device="cuda", dtype=torch.uint8)
    return torch.minimum(a, r)


def _first_tokens(case, tile0):
    """Tokens 0 .. 3 of a stream's first tile get code 0 in every group: the centroid near the queries' common part."""
    low = HEAD // case["c"] * TILE
    tile0[:, :low].view(tile0.shape[0], -1, TILE, 16)[:, :, :4] = 0
    if case["b"] == 10:
        tile0[:, low:].view(tile0.shape[0], TILE, 4)[:, :4] = 0


def _lengths(case, rng):
    low = max(case.get("m", 1), case["t"] // 8)
    lens = [rng.randint(low, case["t"]) if case["ragged"] else case["t"] for _ in range(case["batch"])]
    lens[0] = case["t"]
    return lens


def _cache(case, g, rng, t_cap, batch, zeros=False):
    """A key and a value cache (contiguous, or pools and a block table) of capacity t_cap."""
    tiles, hkv = t_cap // TILE, case["hkv"]
    make = (lambda n, s: torch.zeros(s, n, _tile_bytes(case), dtype=torch.uint8, device="cuda")) if zeros else (lambda n, s: _codes(case, n, s, g))
    if not case["paged"]:
        kv = [make(tiles, batch * hkv) for _ in range(2)]
        if not zeros:
            _first_tokens(case, kv[0][:, 0])
        return kv + [None, 0]
    n_pages = batch * tiles + 3
    table = list(range(n_pages))
    rng.shuffle(table)
    table = torch.tensor(table[:batch * tiles], dtype=torch.int32, device="cuda").view(batch, tiles)
    kv = [make(hkv, n_pages) for _ in range(2)]
    if not zeros:
        first = table[:, 0].long()
        low = kv[0][first].reshape(batch * hkv, -1)
        _first_tokens(case, low)
        kv[0][first] = low.view(batch, hkv, -1)
    return kv + [table, n_pages]


def prepare(case, seed):
    import random
    rng = random.Random(int(seed) * 7919 + 13)
    g = _gen(seed, 1)
    c, b, hkv, batch, t = case["c"], case["b"], case["hkv"], case["batch"], case["t"]
    gh, k = HEAD // c, 1 << b
    normal = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    st = dict(case=case, t_cap=-(-t // TILE) * TILE)
    st["k"], st["v"], st["table"], st["n_pages"] = _cache(case, g, rng, st["t_cap"], batch)
    lens = _lengths(case, rng)
    st["lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda") if case["ragged"] else None
    if case["op"] in ("weights", "chunk_weights", "evict"):
        # accumulators as earlier steps leave them: heavy tails, tokens that never drew any weight, and the sum that
        # decay and the weights of a call balance at
        w = torch.exp(2 * normal(batch, hkv, st["t_cap"])) * (normal(batch, hkv, st["t_cap"]) > -0.6)
        w = w * (torch.arange(st["t_cap"], device="cuda") < torch.tensor(lens, device="cuda")[:, None, None])
        st["w"] = w * (case.get("m", 1) * (Q_HEADS // hkv) / (1 - DECAY)) / w.sum(-1, keepdim=True).clamp(min=1e-3)
    if case["op"] == "evict":
        if case["inplace"]:
            st.update(k2=st["k"], v2=st["v"], table2=st["table"], n_pages2=st["n_pages"], w2=st["w"], t_cap2=st["t_cap"])
        else:
            st["t_cap2"] = -(-(case["keep"] + 200) // TILE) * TILE
            st["k2"], st["v2"], st["table2"], st["n_pages2"] = _cache(case, g, rng, st["t_cap2"], batch, zeros=True)
            st["w2"] = torch.zeros(batch, hkv, st["t_cap2"], device="cuda")
        return st
    # scores: standard deviation 2, and 4 more for the first tokens
    common = normal(hkv, HEAD)
    ck = 1.4 * normal(hkv, gh, k, c)
    ck[:, :, 0] = 0.6 * common.view(hkv, gh, c)
    m = case.get("m", 1)
    q = (0.6 * common.view(1, 1, hkv, 1, HEAD) + 1.3 * normal(batch, m, hkv, Q_HEADS // hkv, HEAD)).view(batch, m, Q_HEADS, HEAD)
    st["ck"] = ck.half().view(hkv * gh, k, c)
    st["cv"] = (normal(hkv, gh, k, c) + 0.5 * normal(hkv, gh, 1, c)).half().view(hkv * gh, k, c)
    st["q"] = q.half() if "m" in case else q[:, 0].half()
    return st


# ---------------------------------------------------------------- the calls

def _call(st):
    """The call (or calls) of a case with the arguments laid out once, as a serving loop keeps them, and what they write."""
    import paper_2405_03917_amd as cq
    case = st["case"]
    op, t, t_cap = case["op"], case["t"], st["t_cap"]
    fmt = cq.CQFormat(case["c"], case["b"], HEAD, case["hkv"])
    k, v = st["k"].view(-1), st["v"].view(-1)
    pages = cq.PageTable(st["table"], st["n_pages"]) if case["paged"] else None
    if op == "window":
        call, out = cq.prepare_decode_attention_window(st["q"], k, v, st["ck"], st["cv"], SCALE, fmt, t, t_cap, case["window"], case["sink"],
                                                       pages=pages, seq_lens=st["lens"])
        return [call], {"out": out}
    if op == "chunk_window":
        call, out = cq.prepare_chunk_attention_window(st["q"], k, v, st["ck"], st["cv"], SCALE, fmt, t, t_cap, case["window"], case["sink"],
                                                      pages=pages, seq_lens=st["lens"])
        return [call], {"out": out}
    if op == "weights":
        call, out = cq.prepare_decode_attention_weights(st["q"], k, v, st["ck"], st["cv"], SCALE, fmt, t, t_cap, st["w"], DECAY,
                                                        pages=pages, seq_lens=st["lens"])
        return [call], {"out": out, "weights": st["w"]}
    if op == "chunk_weights":
        call = cq.prepare_chunk_weights(st["q"], k, st["ck"], SCALE, fmt, t, t_cap, st["w"], DECAY, pages=pages, seq_lens=st["lens"])
        return [call], {"weights": st["w"]}
    pages2 = cq.PageTable(st["table2"], st["n_pages2"]) if case["paged"] else None
    select, kept, lens = cq.prepare_select_tokens(st["w"], t, case["keep"], case["sink"], case["recent"], seq_lens=st["lens"])
    move = cq.prepare_compact_cache(k, v, st["w"], fmt, kept, lens, t, t_cap, st["k2"].view(-1), st["v2"].view(-1), st["w2"], st["t_cap2"],
                                    pages=pages, pages_out=pages2)
    return [select, move], {"kept": kept, "lens": lens, "k": st["k2"], "v": st["v2"], "weights": st["w2"]}


def run(st):
    if own:
        if "calls" not in st:
            st["calls"], st["outputs"] = _call(st)
        for call in st["calls"]:
            call()
        return st["outputs"]
    op = st["case"]["op"]
    if op == "evict":
        return _plain_evict(st)
    return _plain_attention(st)


# ---------------------------------------------------------------- plain forms: elementary operations, 32 bits

def _read_tiles(st, codes, tiles):
    """Codes [batch, KV head, tokens, group] of the tiles `tiles` [batch, n] of every stream."""
    case = st["case"]
    batch, n = tiles.shape
    gh, hkv = HEAD // case["c"], case["hkv"]
    rows = torch.arange(batch, device="cuda")[:, None]
    if case["paged"]:
        raw = codes[st["table"].long()[rows, tiles]]
    else:
        raw = codes.view(batch, hkv, -1, codes.shape[-1])[rows, :, tiles]
    raw = raw.transpose(1, 2).contiguous()                                   # [batch, KV head, n, bytes]
    low = raw[..., :gh * TILE].view(batch, hkv, n, gh // 16, TILE, 16).transpose(3, 4).reshape(batch, hkv, n, TILE, gh)
    token, group = torch.arange(TILE, device="cuda")[:, None], torch.arange(gh, device="cuda")[None]
    slot = (group - token) % gh
    got = low.gather(-1, slot.expand(low.shape)).long()
    if case["b"] == 10:
        words = raw[..., gh * TILE:].contiguous().view(torch.int32).long()[..., None]
        got = got + ((words >> (2 * slot)) % 4) * 256
    return got.view(batch, hkv, n * TILE, gh)


def _dense(st, codes, cent):
    """fp32 [batch, KV head, tokens, 128] of codes in group order."""
    c, hkv = st["case"]["c"], st["case"]["hkv"]
    gh = HEAD // c
    cent = cent.view(hkv, gh, -1, c)
    h = torch.arange(hkv, device="cuda").view(1, hkv, 1, 1)
    return cent[h, torch.arange(gh, device="cuda"), codes].flatten(3).float()


def _plain_attention(st):
    case, q = st["case"], st["q"]
    m, hkv, t = case.get("m", 1), case["hkv"], case["t"]
    qper, batch = Q_HEADS // hkv, case["batch"]
    lens = torch.full((batch,), t, device="cuda") if st["lens"] is None else st["lens"].long()
    last = (lens - 1) // TILE
    n_tiles = -(-t // TILE)
    if "window" in case:
        # the tiles of the sinks that lie in front of the windows, then the windows'
        window, sink = case["window"], case["sink"]
        first = (lens - m - window + 1).clamp(min=0) // TILE
        head = min(n_tiles, -(-sink // TILE))
        count = min(n_tiles, (window + m + TILE - 2) // TILE + 1)
        i = torch.arange(head + count, device="cuda")[None]
        tiles = torch.where(i < head, i, first[:, None] + i - head)
        there = torch.where(i < head, i < first[:, None], tiles <= last[:, None])
    else:
        tiles = torch.arange(n_tiles, device="cuda")[None].expand(batch, -1)
        there = tiles <= last[:, None]
    tiles = tiles.clamp(max=n_tiles - 1)
    token = (tiles[..., None] * TILE + torch.arange(TILE, device="cuda")).view(batch, 1, -1)
    place = (lens - m)[:, None, None] + torch.arange(m, device="cuda")[None, :, None]
    seen = (token <= place) & there.repeat_interleave(TILE, 1)[:, None]
    if "window" in case:
        seen &= (token < sink) | (token > place - window)
    rows = q.view(batch, m, hkv, qper, HEAD).transpose(1, 2).reshape(batch, hkv, m * qper, HEAD).float()
    keys = _dense(st, _read_tiles(st, st["k"], tiles), st["ck"])
    s = torch.matmul(rows, keys.transpose(2, 3)) * SCALE
    s = s.masked_fill(~seen.repeat_interleave(qper, 1)[:, None], -math.inf)
    e = torch.exp(s - s.amax(-1, keepdim=True))
    total = e.sum(-1, keepdim=True)
    got = {}
    if "w" in st:
        w = st["w"]
        mine = (e / total).sum(2)[..., :w.shape[-1]]
        inside = (torch.arange(w.shape[-1], device="cuda") < lens[:, None])[:, None]
        w.copy_(torch.where(inside, DECAY * w + mine, w))
        got["weights"] = w
    if case["op"] != "chunk_weights":
        values = _dense(st, _read_tiles(st, st["v"], tiles), st["cv"])
        out = torch.matmul(e, values) / total
        got["out"] = out.view(batch, hkv, m, qper, HEAD).transpose(1, 2).reshape(q.shape).half()
    return got


def _plain_evict(st):
    case, w = st["case"], st["w"]
    batch, hkv, t, keep = case["batch"], case["hkv"], case["t"], case["keep"]
    lens = torch.full((batch,), t, device="cuda") if st["lens"] is None else st["lens"].long()
    i = torch.arange(t, device="cuda")
    n = lens[:, None, None]
    # class 2: kept whatever their weight; 1: by weight; 0: behind the sequence
    rank = torch.where(i < n, torch.where((i < case["sink"]) | (i >= n - case["recent"]), 2, 1), 0).expand(batch, hkv, t)
    value = torch.nan_to_num(w[..., :t], nan=-math.inf, posinf=math.inf, neginf=-math.inf)
    by = torch.sort(value, dim=-1, descending=True, stable=True).indices
    by = by.gather(-1, torch.sort(rank.gather(-1, by), dim=-1, descending=True, stable=True).indices)
    width = min(keep, t)
    count = lens.clamp(max=keep)[:, None, None]
    r = torch.arange(keep, device="cuda")
    chosen = torch.where(r[:width] < count, by[..., :width], t)
    chosen = torch.sort(chosen, dim=-1).values.clamp(max=t - 1)
    kept = torch.full((batch, hkv, keep), -1, dtype=torch.int32, device="cuda")
    kept[..., :width] = torch.where(r[:width] < count, chosen, -1).int()
    # everything is read, then written
    fresh = w.gather(-1, chosen)
    tiles = torch.arange(-(-t // TILE), device="cuda")[None].expand(batch, -1)
    pairs = [(_read_tiles(st, st[x], tiles).gather(2, chosen[..., None].expand(-1, -1, -1, HEAD // case["c"])), st[x + "2"]) for x in "kv"]
    inside = r[:width] < count
    [_write(st, codes, inside.expand(batch, hkv, width), to) for codes, to in pairs]
    end = min(t, st["t_cap2"])
    w2 = st["w2"]
    w2[..., :end] = 0
    w2[..., :width] = torch.where(inside, fresh, 0.0)
    return {"kept": kept, "lens": count.view(-1).int(), "k": st["k2"], "v": st["v2"], "weights": w2}


def _write(st, codes, inside, to):
    """Codes [batch, KV head, tokens, group] to positions 0 .. of every stream of `to`, where `inside`."""
    case = st["case"]
    batch, hkv, width, gh = codes.shape
    n = -(-width // TILE)
    pad = n * TILE - width
    codes = torch.nn.functional.pad(codes, (0, 0, 0, pad)).view(batch, hkv, n, TILE, gh)
    inside = torch.nn.functional.pad(inside, (0, pad)).view(batch, hkv, n, TILE)
    token, slot = torch.arange(TILE, device="cuda")[:, None], torch.arange(gh, device="cuda")[None]
    codes = codes.gather(-1, ((slot + token) % gh).expand(codes.shape))      # slot s of token u: group (s + u) mod gh
    rows = torch.arange(batch, device="cuda")[:, None]
    if case["paged"]:
        at = st["table2"].long()[:, :n]
        old = to[at].transpose(1, 2).contiguous()
    else:
        old = to.view(batch, hkv, -1, to.shape[-1])[:, :, :n].contiguous()
    low = old[..., :gh * TILE].view(batch, hkv, n, gh // 16, TILE, 16).transpose(3, 4).reshape(codes.shape)
    low = torch.where(inside[..., None], (codes % 256).to(torch.uint8), low)
    old[..., :gh * TILE] = low.view(batch, hkv, n, TILE, gh // 16, 16).transpose(3, 4).reshape(batch, hkv, n, -1)
    if case["b"] == 10:
        words = ((codes // 256) << (2 * slot)).sum(-1)
        words = torch.where(words >= 2 ** 31, words - 2 ** 32, words).int()
        before = old[..., gh * TILE:].contiguous().view(torch.int32)
        old[..., gh * TILE:] = torch.where(inside, words, before).view(torch.uint8)
    if case["paged"]:
        to[at] = old.transpose(1, 2).contiguous()
    else:
        to.view(batch, hkv, -1, to.shape[-1])[rows, :, torch.arange(n, device="cuda")[None]] = old.transpose(1, 2)


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    t, batch, hkv, m = case["t"], case["batch"], case["hkv"], case.get("m", 1)
    per_token = HEAD // case["c"] * case["b"] // 8                           # code bytes of a token and KV head
    book = hkv * HEAD * (1 << case["b"]) * 2
    mean = (0.5625 if case["ragged"] else 1.0) * t                           # lengths run from t / 8 to t
    streams = batch * hkv
    rows = batch * m * Q_HEADS
    if case["op"] == "evict":
        kept = min(mean, case["keep"])
        move = 2 * 2 * streams * kept * per_token if case["keep"] < mean or not case["inplace"] else 0
        return {"bytes": 4 * streams * (mean + 3 * kept) + move, "flops": 0}
    if "window" in case:
        every = min(mean, case["window"] + m - 1 + case["sink"])
        each = min(mean, case["window"] + case["sink"])
        return {"bytes": 2 * (streams * every * per_token + book) + 4 * rows * HEAD, "flops": 4 * rows * HEAD * each}
    if case["op"] == "weights":
        return {"bytes": 2 * (streams * mean * per_token + book) + 4 * rows * HEAD + 8 * streams * mean, "flops": 4 * rows * HEAD * mean}
    return {"bytes": streams * mean * per_token + book + 2 * rows * HEAD + 8 * streams * mean, "flops": 2 * rows * HEAD * max(1.0, mean - m / 2)}


# ---------------------------------------------------------------- the definitions, in 64 bits, stream by stream

def _stream(st, which, n, h, length, cent):
    """fp64 [length, 128]: what stream (n, h) of a cache stands for, byte by byte of its layout."""
    case = st["case"]
    gh, hkv, size = HEAD // case["c"], case["hkv"], _tile_bytes(case)
    i = torch.arange(length, device="cuda")
    if case["paged"]:
        base = (st["table"][n].long()[i // TILE] * hkv + h) * size
    else:
        base = ((n * hkv + h) * (st["t_cap"] // TILE) + i // TILE) * size
    u = i % TILE
    grp = torch.arange(gh, device="cuda")
    slot = (grp[None] - u[:, None]) % gh
    flat = st[which].view(-1)
    code = flat[base[:, None] + (slot // 16) * 1024 + u[:, None] * 16 + slot % 16].long()
    if case["b"] == 10:
        shift = 2 * slot
        byte = flat[base[:, None] + gh * TILE + 4 * u[:, None] + shift // 8].long()
        code = code + (torch.bitwise_right_shift(byte, shift % 8) & 3) * 256
    book = cent.view(hkv, gh, 1 << case["b"], case["c"])[h].double()
    return book[grp[None], code].reshape(length, HEAD)


def exact(case, seed):
    st = prepare(case, seed)
    batch, hkv, t = case["batch"], case["hkv"], case["t"]
    lens = [t] * batch if st["lens"] is None else st["lens"].tolist()
    if case["op"] == "evict":
        w2 = st["w2"].double().clone()
        w = st["w"].double()
        for n in range(batch):
            length = lens[n]
            count = min(length, case["keep"])
            for h in range(hkv):
                x = w[n, h, :length].clone()
                x[torch.isnan(x)] = -math.inf
                free = torch.ones(length, dtype=torch.bool, device="cuda")
                free[:case["sink"]] = False
                free[max(0, length - case["recent"]):] = False
                if count < length:
                    middle = torch.nonzero(free).view(-1)
                    best = torch.sort(x[middle], descending=True, stable=True).indices[:count - int((~free).sum())]
                    free[middle[best]] = False
                    at = torch.nonzero(~free).view(-1)
                else:
                    at = torch.arange(length, device="cuda")
                w2[n, h, :min(t, st["t_cap2"])] = 0
                w2[n, h, :count] = w[n, h, at]
        return {"kept": None, "lens": None, "k": None, "v": None, "weights": w2}
    m = case.get("m", 1)
    qper = Q_HEADS // hkv
    q = st["q"].view(batch, m, Q_HEADS, HEAD).double()
    out = torch.zeros(batch, m, Q_HEADS, HEAD, dtype=torch.float64, device="cuda")
    w = st["w"].double() if "w" in st else None
    for n in range(batch):
        length = lens[n]
        i = torch.arange(length, device="cuda")
        at = length - m + torch.arange(m, device="cuda")
        ok = i[None] <= at[:, None]
        if "window" in case:
            ok &= (i[None] < case["sink"]) | (at[:, None] - i[None] < case["window"])
        some = torch.nonzero(ok.any(0)).view(-1)
        ok = ok[:, some]
        for h in range(hkv):
            keys = _stream(st, "k", n, h, length, st["ck"])[some]
            values = _stream(st, "v", n, h, length, st["cv"])[some] if case["op"] != "chunk_weights" else None
            for j in range(qper):
                s = (q[n, :, h * qper + j] @ keys.T) * SCALE
                p = torch.softmax(s.masked_fill(~ok, -math.inf), -1)
                if values is not None:
                    out[n, :, h * qper + j] = p @ values
                if w is not None:
                    if j == 0:
                        w[n, h, :length] *= DECAY
                    w[n, h, some] += p.sum(0)
    got = {"weights": w} if w is not None else {}
    if case["op"] != "chunk_weights":
        got["out"] = out.view(st["q"].shape)
    return got
