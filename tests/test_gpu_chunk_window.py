"""Causal attention of the last m tokens through sliding windows with sinks, in every kernel that serves it, against the
64-bit definition."""
import numpy as np
import pytest
import torch

import paper_2405_03917_amd as cq
from bounded_util import FORMATS, SCALE, Cache, attention, queries
from gpu_util import check_attention

pytestmark = pytest.mark.gpu


def _run(cache, q, t, window, n_sink, lens=None, paged=False, split=0, table=None, scale=SCALE):
    sl = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
    if paged:
        return cq.cq_chunk_attention_window_paged(q, *cache.pools, cache.ck, cache.cv, scale, cache.fmt, t, cache.pages(table), window,
                                                  n_sink, sl, split)
    return cq.cq_chunk_attention_window(q, cache.k, cache.v, cache.ck, cache.cv, scale, cache.fmt, t, cache.t_cap, window, n_sink, sl,
                                        split)


def _check(cache, q, out, lens, window, n_sink, scale=SCALE):
    ref, _, _ = attention(cache, q, lens, window, n_sink, scale)
    check_attention(out.cpu().numpy(), ref.numpy())


EDGES = [(1, 0), (1, 1), (64, 64), (63, 65), (65, 0), (200, 4), (200, 300), (5000, 3), (500, 128)]


# m x query heads per KV head: token by token, up to 4, 8, 16, 64, 128, 256 rows and more
@pytest.mark.parametrize("m,hq,hkv", [(1, 4, 2), (2, 4, 2), (3, 2, 2), (4, 2, 2), (7, 2, 2), (5, 6, 2), (9, 8, 2), (40, 2, 2), (33, 6, 2), (90, 6, 2)])
@pytest.mark.parametrize("c,b", FORMATS)
def test_rows_and_window_edges(c, b, m, hq, hkv):
    cache = Cache(c, b, hkv, 4, 896, seed=m + c)
    lens = [871, m, max(m, 64), 640]
    q = queries((4, m, hq, 128), m)
    for window, n_sink in EDGES:
        out = _run(cache, q, 871, window, n_sink, lens)
        _check(cache, q, out, lens, window, n_sink)
        assert torch.equal(out, _run(cache, q, 871, window, n_sink, lens, paged=True)), (window, n_sink)


@pytest.mark.parametrize("split", [64, 192, 512])
@pytest.mark.parametrize("m,hq,hkv", [(2, 4, 2), (4, 2, 2), (8, 2, 2), (20, 4, 2), (150, 4, 2)])
@pytest.mark.parametrize("c,b", FORMATS)
def test_given_splits_of_which_rows_see_nothing(c, b, m, hq, hkv, split):
    cache = Cache(c, b, hkv, 3, 1600, seed=split + m)
    lens = [1555, max(m, 130), 700]
    q = queries((3, m, hq, 128), split)
    for window, n_sink in ((5, 0), (40, 200), (900, 3)):
        _check(cache, q, _run(cache, q, 1555, window, n_sink, lens, split=split), lens, window, n_sink)


@pytest.mark.parametrize("c,b", FORMATS)
def test_long_contexts_large_batches(c, b):
    for batch, m, hq, hkv, t, window, n_sink in ((1, 300, 8, 2, 9000, 3000, 70), (20, 5, 8, 8, 2100, 1500, 4), (2, 6, 4, 4, 20000, 15000, 1)):
        cache = Cache(c, b, hkv, batch, -(-t // 64) * 64, seed=t)
        rng = np.random.default_rng(t)
        lens = [t] + [int(x) for x in rng.integers(m, t + 1, batch - 1)]
        q = queries((batch, m, hq, 128), t)
        _check(cache, q, _run(cache, q, t, window, n_sink, lens), lens, window, n_sink)


@pytest.mark.parametrize("m", [2, 5, 20, 100])
@pytest.mark.parametrize("c,b", FORMATS)
def test_pages_outside_the_view_are_not_looked_at(c, b, m):
    cache = Cache(c, b, 4, 3, 1024, seed=9)
    q = queries((3, m, 8, 128), 7)
    want = _run(cache, q, 1000, 100, 70, None, paged=True)
    first = (1000 - m - 100 + 1) // 64
    table = cache.table.copy()
    table[:, 2:first] = (set(range(cache.n_pages)) - set(cache.table.reshape(-1).tolist())).pop()
    assert torch.equal(_run(cache, q, 1000, 100, 70, None, paged=True, table=table), want)


@pytest.mark.parametrize("c,b", FORMATS)
def test_a_window_over_everything_equals_the_whole_context(c, b):
    for m in (1, 3, 8, 30, 200):
        cache = Cache(c, b, 2, 3, 1024, seed=m)
        q = queries((3, m, 4, 128), 5)
        want = cq.cq_chunk_attention(q, cache.k, cache.v, cache.ck, cache.cv, SCALE, cache.fmt, 1000, 1024)
        assert torch.equal(_run(cache, q, 1000, 1000, 0), want)
        assert torch.equal(_run(cache, q, 1000, 2 ** 31 - 1, 2 ** 31 - 1), want)


@pytest.mark.parametrize("m", [3, 8, 40, 130])
def test_large_scores_and_scales_of_either_sign(m):
    cache = Cache(8, 8, 2, 2, 704, seed=m, spread=30.0)
    q = queries((2, m, 4, 128), 5, 30.0)
    lens = [700, 500]
    for scale in (SCALE, -SCALE, 0.0):
        out = _run(cache, q, 700, 150, 5, lens, scale=scale).double().cpu()
        ref, _, largest = attention(cache, q, lens, 150, 5, scale)
        # Scores of this size (sum |q_i k_i| scale = `largest`, about 10^4) are not exact to small fractions in fp32: a
        # sum of 128 products rounds 132 times at most, by 2^-24 of `largest` each, E in all, and so does the reference of
        # the softmax; every weight is then off by a factor of at most e^(2 E), and the output, a mean of the values, by at most
        # (e^(2 E) - 1) times the distance of a value from it, 2 max |v|, behind the rounding to fp16.
        e = 132 * 2.0 ** -24 * largest
        room = np.expm1(2 * e) * 2 * float(cache.cv.abs().max())
        assert torch.isfinite(out).all()
        assert ((out - ref).abs() <= room + 2e-3 * torch.maximum(ref.abs(), 1e-3 * ref.abs().amax(-1, keepdim=True))).all()


def test_captured():
    cache = Cache(4, 8, 8, 2, 4096, seed=1)
    for m in (2, 5, 40):
        q = queries((2, m, 32, 128), 1)
        want = _run(cache, q, 4000, 2000, 4)
        call, out = cq.prepare_chunk_attention_window(q, cache.k, cache.v, cache.ck, cache.cv, SCALE, cache.fmt, 4000, 4096, 2000, 4)
        call()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        for _ in range(3):
            out.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want)
            assert torch.equal(_run(cache, q, 4000, 2000, 4), want)
