"""The 8-bit block cache: sizes and refusals that need no GPU.  Every refused call returns before any launch."""
import ctypes

import pytest

import paper_2405_03917_amd as cq

E, UNSUPPORTED, SMALL = cq.CQ_ERR_INVALID_ARG, cq.CQ_ERR_UNSUPPORTED, cq.CQ_ERR_WORKSPACE_TOO_SMALL
BIG = 1 << 40
M = 1 << 20


def fmt_of(kind=1, head_dim=128, hkv=4):
    return cq._Q8Format(kind, head_dim, hkv)


def p(addr):
    return ctypes.c_void_p(addr)


def table(n_pages=64, max_tiles=8, row_stride=8, block_table=0x9000000):
    return cq._PageTable(n_pages, max_tiles, row_stride, block_table)


# (every array a MiB apart from the next, more than any of these calls uses but the pools, which lie at the end)
BASE = dict(k=0x100000000, v=0x200000000, ks=0x300000000, vs=0x400000000, batch=2, hq=8, m=5, t=300, cap=512, seq=None, scale=0.1, split=0,
            q=16 * M, out=32 * M, ws=48 * M, bytes=BIG, xk=64 * M, xv=80 * M, x_batch=5 * 512, x_row=512, rope=0, positions=0, qa=0, q_batch=5 * 1024,
            q_row=1024, q_out=0, ko=96 * M, vo=112 * M, o_batch=5 * 512, o_row=512)


def _cache(a):
    return cq._Q8Cache(a["k"], a["v"], a["ks"], a["vs"])


def _where(name, a, paged):
    if paged is None:
        return name, a["cap"]
    return name + "_paged", ctypes.byref(paged) if paged else None


def append(fmt=None, paged=None, **kw):
    a, f = {**BASE, **kw}, fmt or fmt_of()
    name, at = _where("cq_append_q8", a, paged)
    cache = _cache(a) if a.get("cache", 1) else None
    return int(getattr(cq.load(), name)(p(a["xk"]), p(a["xv"]), a["x_batch"], a["x_row"], cache, f, a["batch"], a["m"], a["t"], at, a["seq"], p(a["rope"]),
                                        a["positions"], p(a["qa"]), a["q_batch"], a["q_row"], a["hq"], p(a["q_out"]), None))


def dequantize(fmt=None, paged=None, **kw):
    a, f = {**BASE, **kw}, fmt or fmt_of()
    name, at = _where("cq_dequantize_q8", a, paged)
    cache = _cache(a) if a.get("cache", 1) else None
    return int(getattr(cq.load(), name)(cache, f, a["batch"], a["m"], a["t"], at, a["seq"], p(a["ko"]), p(a["vo"]), a["o_batch"], a["o_row"], None))


def chunk(fmt=None, paged=None, **kw):
    a, f = {**BASE, **kw}, fmt or fmt_of()
    name, at = _where("cq_chunk_attention_q8", a, paged)
    cache = _cache(a) if a.get("cache", 1) else None
    return int(getattr(cq.load(), name)(p(a["q"]), cache, a["scale"], f, a["batch"], a["hq"], a["m"], a["t"], at, a["seq"], a["split"], p(a["out"]),
                                        p(a["ws"]), a["bytes"], None))


def decode(fmt=None, paged=None, **kw):
    a, f = {**BASE, **kw}, fmt or fmt_of()
    name, at = _where("cq_decode_attention_q8", a, paged)
    cache = _cache(a) if a.get("cache", 1) else None
    return int(getattr(cq.load(), name)(p(a["q"]), cache, a["scale"], f, a["batch"], a["hq"], a["t"], at, a["seq"], a["split"], p(a["out"]), p(a["ws"]),
                                        a["bytes"], None))


CALLS = [(append, ("k", "v", "ks", "vs", "xk", "xv")), (dequantize, ("k", "v", "ks", "vs")), (chunk, ("k", "v", "ks", "vs", "q", "out", "ws")),
         (decode, ("k", "v", "ks", "vs", "q", "out", "ws"))]


@pytest.mark.parametrize("call,pointers", CALLS)
def test_pointers_shapes_and_formats(call, pointers):
    for name in pointers:
        assert call(**{name: 0}) == E, name
        assert call(**{name: BASE[name] + 8}) == E, name
    assert call(cache=0) == E
    for bad in (dict(batch=0), dict(batch=-1), dict(batch=32768), dict(t=0), dict(t=513), dict(cap=500), dict(cap=0), dict(cap=-64), dict(seq=p(0x7000002))):
        assert call(**bad) == E, bad
    if call is not decode:
        for bad in (dict(m=0), dict(m=-1), dict(m=301)):
            assert call(**bad) == E, bad
    for bad in (fmt_of(0), fmt_of(3), fmt_of(1, 0), fmt_of(1, -128), fmt_of(1, 128, 0), fmt_of(1, 128, 65536)):
        assert call(fmt=bad) == E
    assert call(fmt=fmt_of(1, 64)) == UNSUPPORTED
    assert call(paged=False) == E
    for bad in (table(n_pages=0), table(max_tiles=0), table(row_stride=7), table(block_table=0), table(block_table=0x9000002), table(max_tiles=4, row_stride=4),
                table(max_tiles=(1 << 24) + 1, row_stride=1 << 25)):
        assert call(paged=bad) == E


@pytest.mark.parametrize("call", [chunk, decode])
def test_attention(call):
    for bad in (dict(hq=6), dict(hq=0), dict(hq=-4), dict(scale=float("nan")), dict(scale=float("inf")), dict(split=100), dict(split=-64)):
        assert call(**bad) == E, bad
    for kind in (1, 2):
        fmt = cq.Q8Format(("", "int8", "e4m3")[kind], 128, 4)
        for split in (64, 128):
            m = BASE["m"] if call is chunk else 1
            need = cq.cq_attention_q8_workspace_bytes(fmt, 2, 8, m, 300, split)
            assert need == 4 * 2 * m * 8 * -(-300 // split) * 130
            assert call(fmt=fmt_of(kind), split=split, bytes=need - 1) == SMALL
    assert call(bytes=0) == SMALL
    # an output or workspace where something else is read or written
    for other in ("q", "ws", "k", "v", "ks", "vs"):
        assert call(out=BASE[other], split=64) == E, other
    for other in ("k", "v", "ks", "vs", "q"):
        assert call(ws=BASE[other], split=64) == E, other
    assert call(out=BASE["k"] + 4 * 2 * 8 * 8192 - 16) == E     # (its last tile)
    assert call(seq=p(BASE["out"] + 16)) == E


def test_append_arguments():
    for bad in (dict(x_row=511), dict(x_row=516), dict(x_row=504), dict(x_batch=5 * 512 - 8), dict(x_batch=5 * 512 + 4), dict(x_batch=0), dict(x_row=1 << 50)):
        assert append(**bad) == E, bad
    for bad in (dict(rope=0x5000008, positions=320), dict(rope=0x5000000, positions=0), dict(rope=0x5000000, positions=256), dict(rope=0x5000000, positions=330),
                dict(rope=0x5000000, positions=-64), dict(positions=320)):
        assert append(**bad) == E, bad
    q = dict(rope=130 * M, positions=320, qa=140 * M, q_out=150 * M)
    for bad in (dict(rope=0, positions=0), dict(qa=0), dict(q_out=0), dict(hq=6), dict(hq=0), dict(q_row=1016), dict(q_row=1028), dict(q_batch=5 * 1024 - 8),
                dict(qa=140 * M + 8), dict(q_out=150 * M + 8), dict(q_out=140 * M + 16), dict(q_out=BASE["xk"]), dict(q_out=130 * M), dict(q_out=BASE["k"]),
                dict(q_out=BASE["vs"]), dict(q_out=140 * M, q_row=1032, q_batch=5 * 1032), dict(q_out=140 * M, q_batch=6 * 1024)):
        assert append(**{**q, **bad}) == E, bad
    # arrays of the cache apart from each other and from what is read
    for pair in (("k", "v"), ("k", "ks"), ("ks", "vs"), ("v", "vs"), ("k", "xk"), ("vs", "xv"), ("ks", "xk")):
        assert append(**{pair[0]: BASE[pair[1]]}) == E, pair
    assert append(v=BASE["k"] + 2 * 4 * 8 * 8192 - 16) == E
    assert append(paged=table(block_table=BASE["ks"] + 64)) == E
    assert append(seq=p(BASE["ks"] + 64)) == E


def test_dequantize_arguments():
    for bad in (dict(ko=0, vo=0), dict(ko=96 * M + 8), dict(vo=112 * M + 8), dict(o_row=504), dict(o_row=516), dict(o_batch=5 * 512 - 8), dict(ko=BASE["k"]),
                dict(vo=BASE["vs"]), dict(vo=96 * M), dict(vo=96 * M + 512), dict(vo=96 * M + 1024), dict(vo=96 * M + 1024, o_row=1016, o_batch=5 * 1016),
                dict(vo=96 * M + 1024, m=1, o_batch=1016), dict(seq=p(96 * M))):
        assert dequantize(**bad) == E, bad


def test_sizes():
    lib = cq.load()
    fmt = cq.Q8Format("int8", 128, 4)
    assert cq.cq_q8_cache_bytes(fmt, 3, 256) == 3 * 4 * 256 * 128
    assert cq.cq_q8_cache_bytes(fmt, 3, 100) == cq.cq_q8_cache_bytes(fmt, 0, 64) == cq.cq_q8_cache_bytes(cq.Q8Format("e4m3", 64, 4), 3, 256) == 0
    assert cq.cq_q8_paged_cache_bytes(fmt, 7) == 7 * 4 * 8192 and cq.cq_q8_paged_cache_bytes(fmt, 0) == 0
    assert cq.cq_q8_cache_bytes(cq.Q8Format("e4m3", 128, 64), 512, 131072) == 512 * 64 * 131072 * 128
    assert lib.cq_q8_rope_table_bytes(128, 4096) == 16 * 64 * (64 + 64)
    assert lib.cq_q8_rope_table_bytes(128, 100) == lib.cq_q8_rope_table_bytes(64, 4096) == lib.cq_q8_rope_table_bytes(128, 0) == 0
    for bad in (lambda: cq.cq_attention_q8_workspace_bytes(fmt, 1, 6, 1, 100), lambda: cq.cq_attention_q8_workspace_bytes(fmt, 1, 8, 101, 100),
                lambda: cq.cq_attention_q8_workspace_bytes(fmt, 1, 8, 1, 100, 32), lambda: cq.cq_attention_q8_default_split(fmt, 0, 8, 1, 100)):
        assert bad() == 0
    with pytest.raises(ValueError):
        cq.cq_q8_cache_bytes(cq.Q8Format("int4", 128, 4), 1, 64)
    args = lambda **kw: [{**dict(base=1e4, d=128, n=320, at=0x1000, size=BIG), **kw}[x] for x in ("base", "d", "n", "at", "size")]  # noqa: E731
    for bad in (dict(base=0.0), dict(base=float("nan")), dict(base=float("inf")), dict(d=0), dict(n=0), dict(n=100), dict(at=0), dict(at=0x1008)):
        base, d, n, at, size = args(**bad)
        assert lib.cq_q8_rope_table(base, d, n, p(at), size, None) == E, bad
    assert lib.cq_q8_rope_table(1e4, 64, 320, p(0x1000), BIG, None) == UNSUPPORTED
    assert lib.cq_q8_rope_table(1e4, 128, 320, p(0x1000), 16 * 64 * (5 + 64) - 1, None) == SMALL


@pytest.mark.parametrize("hq,hkv", [(32, 32), (32, 8), (64, 1), (7, 7), (40, 8)])
def test_pieces_cover_the_context(hq, hkv):
    fmt = cq.Q8Format("int8", 128, hkv)
    for batch in (1, 3, 64):
        for m in (1, 2, 5, 64, 500, 4096):
            for t in (m, m + 1, m + 63, 4096, 131072):
                if t < m:
                    continue
                split = cq.cq_attention_q8_default_split(fmt, batch, hq, m, t)
                assert split > 0 and split % 64 == 0
                pieces = -(-(-(-t // 64)) // (split // 64))
                need = cq.cq_attention_q8_workspace_bytes(fmt, batch, hq, m, t)
                assert need == (16 if pieces == 1 else 4 * batch * m * hq * pieces * 130)
                # (a given split of the same length is the same call)
                assert need == cq.cq_attention_q8_workspace_bytes(fmt, batch, hq, m, t, split)
