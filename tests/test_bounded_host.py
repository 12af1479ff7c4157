"""Windows, attention weights and eviction: sizes and refusals that need no GPU.  Every refused call returns before any launch."""
import ctypes

import pytest

import paper_2405_03917_amd as cq

E, UNSUPPORTED, SMALL = cq.CQ_ERR_INVALID_ARG, cq.CQ_ERR_UNSUPPORTED, cq.CQ_ERR_WORKSPACE_TOO_SMALL
FORMATS = [(8, 8), (4, 8), (2, 8), (8, 10)]
BIG = 1 << 40


def fmt_of(c=8, b=8, hkv=4):
    return cq.CQFormat(c, b, 128, hkv)


def p(addr):
    return ctypes.c_void_p(addr)


def table(n_pages=64, max_tiles=8, row_stride=8, block_table=0x900000):
    return cq._PageTable(n_pages, max_tiles, row_stride, block_table)


DECODE = dict(q=0x10000, k=0x20000, v=0x30000, ck=0x40000, cv=0x50000, out=0x60000, ws=0x70000, xk=0x80000, xv=0x90000, w=0xa0000,
              scale=0.1, batch=2, hq=8, t=300, cap=512, seq=None, window=64, sink=4, split=0, bytes=BIG, stride=512, decay=1.0, row=None)


def window(fmt=None, paged=None, step=False, **kw):
    a, f = {**DECODE, **kw}, fmt or fmt_of()
    name = "cq_decode_step_window" if step else "cq_decode_attention_window"
    at = a["cap"]
    if paged is not None:
        name, at = name + "_paged", (ctypes.byref(paged) if paged else None)
    new = (p(a["xk"]), p(a["xv"]), f.channels if a["row"] is None else a["row"]) if step else ()
    return int(getattr(cq.load(), name)(p(a["q"]), *new, p(a["k"]), p(a["v"]), p(a["ck"]), p(a["cv"]), a["scale"], ctypes.byref(f._c()), a["batch"],
                                        a["hq"], a["t"], at, a["seq"], a["window"], a["sink"], a["split"], p(a["out"]), p(a["ws"]), a["bytes"], None))


def chunk_window(fmt=None, paged=None, m=3, **kw):
    a, f = {**DECODE, **kw}, fmt or fmt_of()
    name, at = ("cq_chunk_attention_window", a["cap"]) if paged is None else ("cq_chunk_attention_window_paged", ctypes.byref(paged) if paged else None)
    return int(getattr(cq.load(), name)(p(a["q"]), p(a["k"]), p(a["v"]), p(a["ck"]), p(a["cv"]), a["scale"], ctypes.byref(f._c()), a["batch"], a["hq"],
                                        m, a["t"], at, a["seq"], a["window"], a["sink"], a["split"], p(a["out"]), p(a["ws"]), a["bytes"], None))


def weights(fmt=None, paged=None, **kw):
    a, f = {**DECODE, **kw}, fmt or fmt_of()
    name, at = ("cq_decode_attention_weights", a["cap"]) if paged is None else ("cq_decode_attention_weights_paged", ctypes.byref(paged) if paged else None)
    return int(getattr(cq.load(), name)(p(a["q"]), p(a["k"]), p(a["v"]), p(a["ck"]), p(a["cv"]), a["scale"], ctypes.byref(f._c()), a["batch"], a["hq"],
                                        a["t"], at, a["seq"], a["split"], p(a["w"]), a["stride"], a["decay"], p(a["out"]), p(a["ws"]), a["bytes"], None))


def chunk_weights(fmt=None, paged=None, m=3, **kw):
    a, f = {**DECODE, **kw}, fmt or fmt_of()
    name, at = ("cq_chunk_weights", a["cap"]) if paged is None else ("cq_chunk_weights_paged", ctypes.byref(paged) if paged else None)
    return int(getattr(cq.load(), name)(p(a["q"]), p(a["k"]), p(a["ck"]), a["scale"], ctypes.byref(f._c()), a["batch"], a["hq"], m, a["t"], at, a["seq"],
                                        p(a["w"]), a["stride"], a["decay"], p(a["ws"]), a["bytes"], None))


@pytest.mark.parametrize("call,pointers", [
    (window, ("q", "k", "v", "ck", "cv", "out", "ws")),
    (lambda **kw: window(step=True, **kw), ("q", "k", "v", "ck", "cv", "out", "ws", "xk", "xv")),
    (lambda **kw: chunk_window(m=3, **kw), ("q", "k", "v", "ck", "cv", "out")),
    (weights, ("q", "k", "v", "ck", "cv", "out", "ws", "w")),
    (chunk_weights, ("q", "k", "ck", "ws", "w"))])
def test_pointers_shapes_and_scales(call, pointers):
    for name in pointers:
        assert call(**{name: 0}) == E, name
        assert call(**{name: DECODE[name] + 8}) == E, name
    for bad in (dict(batch=0), dict(hq=6), dict(hq=0), dict(t=0), dict(t=513), dict(cap=500), dict(cap=0), dict(scale=float("nan")), dict(scale=float("inf"))):
        assert call(**bad) == E, bad
    assert call(fmt=fmt_of(8, 9)) == UNSUPPORTED
    assert call(fmt=fmt_of(2, 4)) == UNSUPPORTED            # sub-byte formats are attended to as their fused format
    assert call(paged=False) == E
    for bad in (table(n_pages=0), table(max_tiles=0), table(row_stride=7), table(block_table=0), table(block_table=0x900002), table(max_tiles=4, row_stride=4)):
        assert call(paged=bad) == E


def test_windows():
    for call in (window, lambda **kw: window(step=True, **kw), chunk_window):
        assert call(window=0) == E
        assert call(window=-1) == E
        assert call(sink=-1) == E
        assert call(split=100) == E
        assert call(split=-64) == E
    assert window(step=True, row=fmt_of().channels - 8) == E
    assert window(step=True, row=fmt_of().channels + 4) == E
    assert window(step=True, v=DECODE["k"]) == E
    assert chunk_window(m=0) == E
    assert chunk_window(m=301) == E


def test_accumulators():
    for call in (weights, chunk_weights):
        assert call(stride=299) == E
        assert call(stride=-1) == E
        assert call(decay=float("nan")) == E
        assert call(decay=float("inf")) == E
    assert weights(split=100) == E
    assert weights(fmt=fmt_of(hkv=1), hq=4097) == UNSUPPORTED
    assert chunk_weights(m=0) == E
    assert chunk_weights(m=301) == E


@pytest.mark.parametrize("c,b", FORMATS)
def test_workspaces_are_checked_against_what_the_library_reports(c, b):
    f = fmt_of(c, b, 8)
    for batch, hq, t in ((1, 8, 5000), (24, 32, 511), (3, 64, 512)):
        cap = -(-t // 64) * 64
        w = dict(fmt=f, batch=batch, hq=hq, t=t, cap=cap)
        for win, sink in ((100, 0), (3000, 70)):
            need = cq.cq_decode_window_workspace_bytes(f, batch, hq, t, win, sink)
            assert need > 0
            assert window(**w, window=win, sink=sink, bytes=need - 1) == SMALL
            # no more than the whole context needs, by the library's split for as many tokens
            walked = min(-(-t // 64), -(-sink // 64) + (win + 62) // 64 + 1) * 64
            assert need == cq.cq_decode_workspace_bytes(f, batch, hq, walked)
            assert cq.cq_decode_window_default_split(f, batch, hq, t, win, sink) == cq.cq_decode_default_split(f, batch, hq, walked)
        need = cq.cq_decode_weights_workspace_bytes(f, batch, hq, t)
        assert need >= cq.cq_decode_workspace_bytes(f, batch, hq, t) + 4 * batch * hq * cap
        assert weights(**w, bytes=need - 1, stride=cap) == SMALL
        for m in (1, 40, 300):
            need = cq.cq_chunk_weights_workspace_bytes(f, batch, hq, m, t)
            assert need >= 8 * batch * hq * m
            assert chunk_weights(**w, m=m, bytes=need - 1, stride=cap) == SMALL
            need = cq.cq_chunk_window_workspace_bytes(f, batch, hq, m, t, 300, 4)
            if need > 4 * 130 * batch * m * hq:             # (a context in one piece needs none, whatever is reported)
                assert chunk_window(**w, m=m, window=300, sink=4, bytes=need - 4 * 130 * batch * m * hq) == SMALL


def test_sizes_of_bad_arguments_are_zero():
    f, bad = fmt_of(), fmt_of(8, 9)
    assert cq.cq_decode_window_workspace_bytes(f, 1, 8, 100, 0) == 0
    assert cq.cq_decode_window_workspace_bytes(f, 1, 8, 100, 5, -1) == 0
    assert cq.cq_decode_window_workspace_bytes(f, 1, 8, 0, 5) == 0
    assert cq.cq_decode_window_workspace_bytes(f, 1, 8, 100, 5, 0, 65) == 0
    assert cq.cq_decode_window_workspace_bytes(bad, 1, 8, 100, 5) == 0
    assert cq.cq_decode_window_default_split(f, 1, 8, 100, 0) == 0
    assert cq.cq_decode_weights_workspace_bytes(bad, 1, 8, 100) == 0
    assert cq.cq_decode_weights_workspace_bytes(f, 1, 8, 0) == 0
    assert cq.cq_chunk_window_workspace_bytes(f, 1, 8, 0, 100, 5) == 0
    assert cq.cq_chunk_window_workspace_bytes(f, 1, 8, 3, 100, 0) == 0
    assert cq.cq_chunk_weights_workspace_bytes(f, 1, 8, 101, 100) == 0
    assert cq.cq_chunk_weights_workspace_bytes(f, 1, 6, 1, 100) == 0
    assert cq.cq_select_workspace_bytes(0, 1, 1) == 0
    assert cq.cq_select_workspace_bytes(1, 1, 0) == 0
    assert cq.cq_select_workspace_bytes(2, 3, 100) > 0
    assert cq.cq_compact_workspace_bytes(bad, 1, 10) == 0
    assert cq.cq_compact_workspace_bytes(f, 1, 0) == 0


def test_a_window_needs_no_more_than_it_walks():
    f = fmt_of(4, 8, 8)
    assert cq.cq_decode_window_workspace_bytes(f, 4, 32, 1 << 20, 4096, 4) < cq.cq_decode_workspace_bytes(f, 4, 32, 1 << 20)
    # tokens beyond the context change nothing
    assert cq.cq_decode_window_workspace_bytes(f, 4, 32, 5000, 2 ** 31 - 1, 2 ** 31 - 1) == cq.cq_decode_workspace_bytes(f, 4, 32, 5000)


SELECT = dict(w=0x10000, stride=512, batch=2, hkv=4, t=300, seq=None, keep=100, sink=4, recent=10, kept=0x20000, lens=0x30000, ws=0x40000, bytes=BIG)


def select(**kw):
    a = {**SELECT, **kw}
    return int(cq.load().cq_select_tokens(p(a["w"]), a["stride"], a["batch"], a["hkv"], a["t"], a["seq"], a["keep"], a["sink"], a["recent"], p(a["kept"]),
                                          p(a["lens"]), p(a["ws"]), a["bytes"], None))


def test_selection():
    for name in ("w", "kept", "lens"):
        assert select(**{name: 0}) == E
        assert select(**{name: SELECT[name] + 4}) == E
    for bad in (dict(batch=0), dict(hkv=0), dict(t=0), dict(stride=299), dict(keep=0), dict(sink=-1), dict(recent=-1), dict(sink=95, recent=6)):
        assert select(**bad) == E, bad
    assert select(batch=1 << 16, hkv=1 << 15) == E
    need = cq.cq_select_workspace_bytes(2, 4, 100000)
    assert select(t=100000, stride=100000, bytes=need - 1) == SMALL
    assert select(t=100000, stride=100000, ws=0) == E
    assert select(t=100000, stride=100000, ws=0x40008) == E


COMPACT = dict(k=0x1000000, v=0x2000000, w=0x3000000, stride=512, batch=2, t=300, cap=512, kept=0x10000, lens=0x20000, keep=100, k2=0x4000000, v2=0x5000000,
               w2=0x6000000, stride2=512, cap2=128, ws=0x7000000, bytes=BIG)


def compact(fmt=None, pages=None, pages2=None, **kw):
    a, f = {**COMPACT, **kw}, fmt or fmt_of()
    name, at, at2 = "cq_compact_cache", a["cap"], a["cap2"]
    if pages is not None:
        name, at, at2 = name + "_paged", (ctypes.byref(pages) if pages else None), (ctypes.byref(pages2) if pages2 else None)
    return int(getattr(cq.load(), name)(p(a["k"]), p(a["v"]), p(a["w"]), a["stride"], ctypes.byref(f._c()), a["batch"], a["t"], at, p(a["kept"]), p(a["lens"]),
                                        a["keep"], p(a["k2"]), p(a["v2"]), p(a["w2"]), a["stride2"], at2, p(a["ws"]), a["bytes"], None))


def test_compaction():
    for name in ("k", "v", "kept", "lens", "k2", "v2"):
        assert compact(**{name: 0}) == E, name
        assert compact(**{name: COMPACT[name] + 8}) == E, name
    for bad in (dict(w=0), dict(w2=0), dict(w=COMPACT["w"] + 8), dict(batch=0), dict(t=0), dict(t=513), dict(cap=500), dict(cap2=100), dict(keep=0), dict(keep=129),
                dict(stride=299), dict(stride2=127), dict(batch=1 << 14)):
        assert compact(**bad) == E, bad
    assert compact(fmt=fmt_of(8, 9)) == UNSUPPORTED
    good, bad = table(), table(max_tiles=4, row_stride=4)
    assert compact(pages=False) == E
    assert compact(pages=good, pages2=False) == E
    assert compact(pages=bad, pages2=good) == E             # 256 positions, 300 tokens
    assert compact(pages=good, pages2=bad, keep=257) == E


def test_compaction_refuses_buffers_that_overlap():
    size = cq.cq_cache_bytes(fmt_of(), 2, 512)
    out = cq.cq_cache_bytes(fmt_of(), 2, 128)
    k, v, w = COMPACT["k"], COMPACT["v"], COMPACT["w"]
    assert compact(v=k + size - 16) == E                    # the inputs
    assert compact(v2=COMPACT["k2"] + out - 16) == E        # the outputs
    assert compact(k2=k + size - 16) == E                   # an output and an input, partly
    assert compact(k2=k + 16) == E
    assert compact(k2=k - out + 16) == E
    assert compact(k2=v) == E                               # an output and the other input
    assert compact(v2=k) == E
    assert compact(w2=w + 4 * 300) == E
    in_place = dict(k2=k, v2=v, cap2=512, w2=w)
    assert compact(**{**in_place, "cap2": 128}) == E        # in place: the same places
    assert compact(**in_place, stride2=600) == E
    need = cq.cq_compact_workspace_bytes(fmt_of(), 2, 100)
    assert compact(**in_place, bytes=need - 1) == SMALL
    assert compact(**in_place, ws=0) == E
    assert compact(**in_place, ws=COMPACT["ws"] + 8) == E
