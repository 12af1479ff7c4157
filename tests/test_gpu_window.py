"""Decode attention through a sliding window with sinks, and its fused step, against the 64-bit definition and, bit for
bit, against the calls they are made of."""
import numpy as np
import pytest
import torch

import paper_2405_03917_amd as cq
from bounded_util import FORMATS, SCALE, Cache, attention, queries
from gpu_util import check_attention

pytestmark = pytest.mark.gpu


def _run(cache, q, t, window, n_sink, lens=None, paged=False, split=0, table=None):
    sl = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
    if paged:
        return cq.cq_decode_attention_window_paged(q, *cache.pools, cache.ck, cache.cv, SCALE, cache.fmt, t, cache.pages(table),
                                                   window, n_sink, sl, split)
    return cq.cq_decode_attention_window(q, cache.k, cache.v, cache.ck, cache.cv, SCALE, cache.fmt, t, cache.t_cap, window, n_sink,
                                         sl, split)


def _check(cache, q, out, lens, window, n_sink):
    ref, _, _ = attention(cache, q[:, None], lens, window, n_sink)
    check_attention(out.cpu().numpy(), ref[:, 0].numpy())


# windows that start and end at tile borders and off them, of one token, longer than the context; sinks that end inside a
# tile, at its end, in the window's first tile, behind the window's start, behind the context
EDGES = [(1, 0), (1, 1), (64, 0), (64, 64), (65, 1), (63, 65), (200, 4), (200, 130), (300, 700), (5000, 3), (777, 0), (513, 128)]


@pytest.mark.parametrize("c,b", FORMATS)
@pytest.mark.parametrize("window,n_sink", EDGES)
def test_window_edges(c, b, window, n_sink):
    cache = Cache(c, b, 2, 5, 832, seed=window + n_sink + c)
    lens = [777, 1, 64, 65, 640]
    q = queries((5, 4, 128), 3 * window + n_sink)
    out = _run(cache, q, 777, window, n_sink, lens)
    _check(cache, q, out, lens, window, n_sink)
    assert torch.equal(out, _run(cache, q, 777, window, n_sink, lens, paged=True))


# (batch, query heads, KV heads, t): one head per workgroup, two, four; chunks of several tiles, several splits
SIZES = [(1, 8, 8, 9000), (16, 32, 16, 1500), (18, 32, 8, 300), (40, 8, 2, 2100), (3, 6, 2, 5000), (2, 5, 5, 20000), (70, 16, 4, 700)]


@pytest.mark.parametrize("c,b", FORMATS)
@pytest.mark.parametrize("batch,hq,hkv,t", SIZES)
def test_window_sizes_and_kernels(c, b, batch, hq, hkv, t):
    cache = Cache(c, b, hkv, batch, -(-t // 64) * 64, seed=t + batch)
    rng = np.random.default_rng(t)
    lens = [t] + [int(x) for x in rng.integers(1, t + 1, batch - 1)]
    q = queries((batch, hq, 128), t)
    for window, n_sink in ((t // 3 + 1, 5), (t, 0), (7, 70)):
        out = _run(cache, q, t, window, n_sink, lens, paged=bool(window % 2))
        _check(cache, q, out, lens, window, n_sink)


@pytest.mark.parametrize("c,b", FORMATS)
def test_a_window_over_everything_equals_the_whole_context(c, b):
    for batch, hq, hkv, t in ((2, 4, 2, 1000), (20, 32, 8, 500)):
        cache = Cache(c, b, hkv, batch, 1024, seed=c + b)
        q = queries((batch, hq, 128), 5)
        want = cq.cq_decode_attention(q, cache.k, cache.v, cache.ck, cache.cv, SCALE, cache.fmt, t, 1024)
        assert torch.equal(_run(cache, q, t, t, 0), want)
        assert torch.equal(_run(cache, q, t, 1, t), want)
        assert torch.equal(_run(cache, q, t, 2 ** 31 - 1, 2 ** 31 - 1), want)


@pytest.mark.parametrize("c,b", FORMATS)
def test_pages_outside_the_view_are_not_looked_at(c, b):
    cache = Cache(c, b, 8, 20, 1024, seed=9)
    q = queries((20, 32, 128), 7)
    lens = [1000] * 20
    want = _run(cache, q, 1000, 100, 70, lens, paged=True)
    # tiles 0, 1 hold sinks, 14, 15 the window; the others' entries name a page of other contents
    table = cache.table.copy()
    table[:, 2:14] = (set(range(cache.n_pages)) - set(cache.table.reshape(-1).tolist())).pop()
    assert torch.equal(_run(cache, q, 1000, 100, 70, lens, paged=True, table=table), want)


@pytest.mark.parametrize("split", [64, 128, 192, 1024])
@pytest.mark.parametrize("c,b", FORMATS)
def test_given_splits(c, b, split):
    cache = Cache(c, b, 4, 3, 1600, seed=split)
    q = queries((3, 4, 128), split)
    lens = [1555, 130, 700]
    out = _run(cache, q, 1555, 600, 66, lens, split=split)
    _check(cache, q, out, lens, 600, 66)


@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("c,b", FORMATS)
def test_step_is_encode_then_attention(c, b, paged):
    for batch, hq, hkv, t in ((3, 4, 2, 700), (20, 32, 8, 450), (9, 64, 32, 200)):
        cache = Cache(c, b, hkv, batch, 704, seed=t)
        fmt = cache.fmt
        rng = np.random.default_rng(t)
        lens = [t, 1] + [int(x) for x in rng.integers(1, t + 1, batch - 2)]
        sl = torch.tensor(lens, dtype=torch.int32, device="cuda")
        q = queries((batch, hq, 128), t)
        rows = [queries((batch, 2, fmt.channels), t + 1)[:, 0], queries((batch, 2, fmt.channels), t + 2)[:, 0]]    # rows apart
        k, v = (x.clone() for x in (cache.pools if paged else (cache.k, cache.v)))
        k2, v2 = k.clone(), v.clone()
        window, n_sink = 130, 5
        if paged:
            pages = cache.pages()
            out = cq.cq_decode_step_window_paged(q, *rows, k, v, cache.ck, cache.cv, SCALE, fmt, t, pages, window, n_sink, sl)
        else:
            out = cq.cq_decode_step_window(q, *rows, k, v, cache.ck, cache.cv, SCALE, fmt, t, 704, window, n_sink, sl)
        for n in range(batch):
            x = [r[n:n + 1, None] for r in rows]
            if paged:
                one = cq.PageTable(pages.block_table[n:n + 1], cache.n_pages)
                cq.cq_encode_kv_paged(*x, cache.ck, cache.cv, fmt, k2, v2, one, lens[n] - 1)
            else:
                size = k2.numel() // batch
                cq.cq_encode_kv(*x, cache.ck, cache.cv, fmt, k2[n * size:(n + 1) * size], v2[n * size:(n + 1) * size], lens[n] - 1, 704)
        if paged:
            want = cq.cq_decode_attention_window_paged(q, k2, v2, cache.ck, cache.cv, SCALE, fmt, t, pages, window, n_sink, sl)
        else:
            want = cq.cq_decode_attention_window(q, k2, v2, cache.ck, cache.cv, SCALE, fmt, t, 704, window, n_sink, sl)
        assert torch.equal(k, k2) and torch.equal(v, v2)
        assert torch.equal(out, want)


def test_lengths_out_of_range_are_clamped():
    cache = Cache(8, 8, 2, 3, 320, seed=4)
    q = queries((3, 2, 128), 4)
    assert torch.equal(_run(cache, q, 300, 100, 2, [0, -5, 1000]), _run(cache, q, 300, 100, 2, [1, 1, 300]))


def test_captured_and_on_another_stream():
    cache = Cache(8, 8, 4, 2, 4096, seed=1)
    q = queries((2, 4, 128), 1)
    want = _run(cache, q, 4000, 2000, 4)
    out = torch.empty_like(want)
    call, _ = cq.prepare_decode_attention_window(q, cache.k, cache.v, cache.ck, cache.cv, SCALE, cache.fmt, 4000, 4096, 2000, 4,
                                                 tokens_per_split=512, out=out)
    call()
    torch.cuda.synchronize()
    split = out.clone()
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        call()
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, split)
        eager = _run(cache, q, 4000, 2000, 4)
        assert torch.equal(eager, want)
