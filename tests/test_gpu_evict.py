"""Eviction: the tokens that stay against a sort, and the moved codes and accumulators against the layout, byte for byte,
with everything else left as it was."""
import numpy as np
import pytest
import torch

import paper_2405_03917_amd as cq
from bounded_util import FORMATS, SCALE, Cache, attention, queries, weight_tolerance
from gpu_util import check_attention
from oracle import code_layout as L

pytestmark = pytest.mark.gpu


def select_oracle(w, t, lens, keep, n_sink, n_recent):
    batch, hkv, _ = w.shape
    kept = np.full((batch, hkv, keep), -1, dtype=np.int32)
    new = np.zeros(batch, dtype=np.int32)
    for n in range(batch):
        length = min(max(lens[n], 0), t)
        new[n] = min(length, keep)
        for h in range(hkv):
            if length <= keep:
                kept[n, h, :length] = np.arange(length)
                continue
            lo, hi = n_sink, length - n_recent
            x = w[n, h, lo:hi].astype(np.float64)
            number = ~np.isnan(x)
            # heaviest first, equals by position; what is no number behind all numbers
            order = np.lexsort((np.arange(hi - lo), -np.where(number, x, 0.0), ~number))
            best = np.sort(order[:keep - n_sink - n_recent]) + lo
            kept[n, h] = np.concatenate([np.arange(lo), best, np.arange(hi, length)])
    return kept, new


def _weights(kind, shape, rng):
    if kind == "heavy":
        return (np.exp(2 * rng.standard_normal(shape)) * (rng.random(shape) > 0.3)).astype(np.float32)
    if kind == "ties":
        return rng.integers(0, 3, shape).astype(np.float32)
    if kind == "equal":
        return np.zeros(shape, dtype=np.float32)
    if kind == "close":                                    # neighbours in fp32
        return (np.float32(1.0).view(np.int32) + rng.integers(0, 2000, shape).astype(np.int32)).view(np.float32)
    w = rng.standard_normal(shape).astype(np.float32)      # "odd": both signs, zeros of both signs, infinities, NaN of both signs
    for value in (0.0, -0.0, np.inf, -np.inf, np.nan, np.copysign(np.nan, -1), 1e-45, -1e-45):
        w[rng.random(shape) < 0.06] = value
    return w


def _select(w, t, keep, n_sink, n_recent, lens=None):
    sl = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
    kept, new = cq.cq_select_tokens(torch.from_numpy(w).cuda(), t, keep, n_sink, n_recent, sl)
    return kept.cpu().numpy(), new.cpu().numpy()


@pytest.mark.parametrize("kind", ["heavy", "ties", "equal", "close", "odd"])
@pytest.mark.parametrize("t,keep,n_sink,n_recent", [(1, 1, 0, 0), (2, 1, 0, 1), (64, 63, 4, 5), (100, 10, 10, 0), (100, 10, 0, 10), (100, 11, 4, 6),
                                                    (1023, 500, 0, 0), (1025, 1024, 3, 1), (5000, 1, 0, 0), (5000, 77, 4, 64), (70000, 3000, 4, 32),
                                                    (300, 400, 200, 200), (131072, 131071, 0, 0)])
def test_select(kind, t, keep, n_sink, n_recent):
    rng = np.random.default_rng(t + keep)
    w = _weights(kind, (2, 3, t + keep % 5), rng)
    kept, new = _select(w, t, keep, n_sink, n_recent)
    want, want_new = select_oracle(w, t, [t, t], keep, n_sink, n_recent)
    assert np.array_equal(kept, want) and np.array_equal(new, want_new)


def test_select_ragged_lengths_and_many_streams():
    rng = np.random.default_rng(5)
    t, keep = 900, 128
    lens = [900, 0, 1, 127, 128, 129, 130, -3, 5000, 300] + [int(x) for x in rng.integers(1, 900, 30)]
    w = _weights("heavy", (40, 32, t), rng)
    kept, new = _select(w, t, keep, 4, 64, lens)
    want, want_new = select_oracle(w, t, lens, keep, 4, 64)
    assert np.array_equal(kept, want) and np.array_equal(new, want_new)


@pytest.mark.parametrize("kind", ["heavy", "ties", "equal", "close", "odd", "uniform", "mostly one"])
@pytest.mark.parametrize("batch,hkv,t,keep,n_sink,n_recent", [(1, 1, 600000, 5000, 4, 100), (3, 2, 50000, 4097, 0, 0), (100, 9, 9000, 300, 1, 7), (2, 1, 524289, 300000, 0, 9)])
def test_select_streams_of_many_runs(kind, batch, hkv, t, keep, n_sink, n_recent):
    """Longer than a workgroup's run, with few and many of them, at full length and ragged; weights of one value, of few, alike."""
    rng = np.random.default_rng(t)
    shape = (batch, hkv, t)
    if kind == "uniform":
        w = rng.random(shape, dtype=np.float32)
    elif kind == "mostly one":                              # with neighbours of the same first digits
        w = np.where(rng.random(shape) < 0.99, np.float32(0.3), rng.random(shape, dtype=np.float32) * np.float32(0.05) + np.float32(0.27))
    else:
        w = _weights(kind, shape, rng)
    lens = [t] + [int(x) for x in rng.integers(0, t, batch - 1)]
    kept, new = _select(w, t, keep, n_sink, n_recent, lens)
    want, want_new = select_oracle(w, t, lens, keep, n_sink, n_recent)
    assert np.array_equal(kept, want) and np.array_equal(new, want_new)
    again = _select(w, t, keep, n_sink, n_recent, lens)
    assert np.array_equal(again[0], kept)


def test_select_from_eight_million():
    t, keep = 8500000, 2000
    for w in (np.random.default_rng(1).random((1, 1, t), dtype=np.float32) ** 8, np.zeros((1, 1, t), dtype=np.float32)):
        kept, new = _select(w, t, keep, 4, 32)
        want, want_new = select_oracle(w, t, [t], keep, 4, 32)
        assert np.array_equal(kept, want) and np.array_equal(new, want_new)


def _moved(cache, which, kept, new, old):
    """Codes [B, t_cap_out, G] of a cache after the move, given those it held before."""
    f = cache.fmt
    gh = 128 // f.c
    want = old.copy()
    for n in range(kept.shape[0]):
        for h in range(f.n_kv_heads):
            g = slice(h * gh, (h + 1) * gh)
            want[n, :new[n], g] = cache.codes[which][n, kept[n, h, :new[n]], g]
    return want


def _unpack(buffer, f, batch, t_cap):
    return L.unpack(buffer.cpu().numpy().reshape(batch, f.n_kv_heads, t_cap // 64, -1), f.c, f.b, 128, f.n_kv_heads, t_cap)


def _moved_weights(w, out, kept, new, t, cap_out):
    want = out.copy()
    want[..., :min(t, cap_out)] = 0
    for n in range(kept.shape[0]):
        for h in range(kept.shape[1]):
            want[n, h, :new[n]] = w[n, h, kept[n, h, :new[n]]]
    return want


@pytest.mark.parametrize("inplace", [True, False])
@pytest.mark.parametrize("c,b", FORMATS)
@pytest.mark.parametrize("batch,hkv,t,keep", [(3, 2, 200, 70), (2, 4, 1000, 999), (1, 1, 64, 1), (5, 3, 777, 512), (40, 8, 150, 65), (2, 2, 130, 500)])
def test_compact(c, b, batch, hkv, t, keep, inplace):
    cap = 832 if t < 800 else 1024
    cache = Cache(c, b, hkv, batch, cap, seed=t + keep)
    f = cache.fmt
    rng = np.random.default_rng(t)
    lens = [t] + [int(x) for x in rng.integers(1, t + 1, batch - 1)]
    w = _weights("heavy", (batch, hkv, cap), rng)
    kept, new = select_oracle(w, t, lens, keep, 1 if keep > 1 else 0, min(5, keep - 1))
    kd, nd, wd = torch.from_numpy(kept).cuda(), torch.from_numpy(new).cuda(), torch.from_numpy(w).cuda()
    if inplace:
        old = cache.codes
        cq.cq_compact_cache(cache.k, cache.v, wd, f, kd, nd, t, cap)
        got, got_w, cap_out, before = (cache.k, cache.v), wd, cap, w
    else:
        cap_out = -(-keep // 64) * 64 + 64
        old = [rng.integers(0, 1 << b, (batch, cap_out, f.groups)).astype(np.uint16) for _ in range(2)]
        got = [torch.from_numpy(L.pack(x, c, b, 128, hkv, cap_out).reshape(-1)).cuda() for x in old]
        before = rng.random((batch, hkv, cap_out)).astype(np.float32)
        got_w = torch.from_numpy(before).cuda()
        untouched = cache.k.clone(), cache.v.clone()
        cq.cq_compact_cache(cache.k, cache.v, wd, f, kd, nd, t, cap, *got, got_w, cap_out)
        assert torch.equal(cache.k, untouched[0]) and torch.equal(cache.v, untouched[1]) and np.array_equal(wd.cpu().numpy(), w)
    for which in range(2):
        assert np.array_equal(_unpack(got[which], f, batch, cap_out), _moved(cache, which, kept, new, old[which]))
    assert np.array_equal(got_w.cpu().numpy(), _moved_weights(w, before, kept, new, t, cap_out))


@pytest.mark.parametrize("c,b", FORMATS)
@pytest.mark.parametrize("keep", [100, 640])
def test_compact_paged_in_place_equals_contiguous(c, b, keep):
    cache = Cache(c, b, 4, 6, 704, seed=keep)
    f, t = cache.fmt, 700
    rng = np.random.default_rng(keep)
    w = torch.from_numpy(_weights("heavy", (6, 4, t), rng)).cuda()
    w2 = w.clone()
    lens = torch.tensor([700, 90, 641, 640, 12, 333], dtype=torch.int32, device="cuda")
    kept, new = cq.cq_select_tokens(w, t, keep, 4, 32, lens)
    pools = [p.clone() for p in cache.pools]
    cq.cq_compact_cache_paged(*pools, w2, f, kept, new, t, cache.pages())
    cq.cq_compact_cache(cache.k, cache.v, w, f, kept, new, t, 704)
    assert torch.equal(w, w2)
    tb = L.tile_bytes(c, b, 128)
    at = torch.from_numpy(cache.table.astype(np.int64)).cuda()
    for pool, before, flat in zip(pools, cache.pools, (cache.k, cache.v)):
        pages = pool.view(cache.n_pages, 4, tb)
        assert torch.equal(pages[at].transpose(1, 2).reshape(-1), flat)
        others = torch.ones(cache.n_pages, dtype=torch.bool, device="cuda")
        others[at.view(-1)] = False
        assert torch.equal(pages[others], before.view(cache.n_pages, 4, tb)[others])


def test_compact_to_other_pages_of_the_same_pool():
    cache = Cache(4, 8, 2, 3, 512, seed=1)
    f = cache.fmt
    rng = np.random.default_rng(2)
    w = _weights("heavy", (3, 2, 512), rng)
    kept, new = select_oracle(w, 512, [512] * 3, 100, 0, 0)
    # the old last two tiles of each sequence, which other tokens still come from
    out = np.ascontiguousarray(cache.table[:, -2:])
    pools = [p.clone() for p in cache.pools]
    cq.cq_compact_cache_paged(*pools, None, f, torch.from_numpy(kept).cuda(), torch.from_numpy(new).cuda(), 512, cache.pages(),
                              pages_out=cache.pages(out))
    tb = L.tile_bytes(4, 8, 128)
    for which, pool in enumerate(pools):
        got = pool.view(cache.n_pages, 2, tb)[torch.from_numpy(out.astype(np.int64)).cuda()].transpose(1, 2).contiguous()
        assert np.array_equal(_unpack(got, f, 3, 128)[:, :100], _moved(cache, which, kept, new, cache.codes[which])[:, :100])


def test_without_accumulators_and_lists_out_of_range():
    cache = Cache(8, 8, 2, 2, 256, seed=3)
    f = cache.fmt
    kept = torch.tensor([[[-7, 3, 400], [5, 5, 255]], [[0, 1, 2], [9, 8, 7]]], dtype=torch.int32, device="cuda")
    lens = torch.tensor([9, -1], dtype=torch.int32, device="cuda")
    k2, v2 = cq.alloc_cache(f, 2, 64).zero_(), cq.alloc_cache(f, 2, 64).zero_()
    cq.cq_compact_cache(cache.k, cache.v, None, f, kept, lens, 200, 256, k2, v2, None, 64)
    want = np.zeros((2, 64, f.groups), dtype=np.uint16)
    clamped = kept.clamp(0, 199).cpu().numpy()
    assert np.array_equal(_unpack(k2, f, 2, 64), _moved(cache, 0, clamped, [3, 0], want))
    assert np.array_equal(_unpack(v2, f, 2, 64), _moved(cache, 1, clamped, [3, 0], want))


def test_sub_byte_formats_move_as_their_fused_format():
    fmt = cq.CQFormat(2, 4, 128, 2)
    cache = Cache(4, 8, 2, 2, 256, seed=3)
    kept, new = select_oracle(np.random.default_rng(1).random((2, 2, 256)).astype(np.float32), 256, [256, 256], 50, 0, 0)
    args = torch.from_numpy(kept).cuda(), torch.from_numpy(new).cuda(), 256, 256
    k, v = cache.k.clone(), cache.v.clone()
    cq.cq_compact_cache(k, v, None, fmt, *args)
    cq.cq_compact_cache(cache.k, cache.v, None, cache.fmt, *args)
    assert torch.equal(k, cache.k) and torch.equal(v, cache.v)


@pytest.mark.parametrize("c,b", FORMATS)
@pytest.mark.parametrize("batch,hkv,keep", [(1, 2, 4500), (2, 64, 4500), (1, 1, 4096)])
def test_long_lists_in_place_equal_those_moved_elsewhere(c, b, batch, hkv, keep):
    t, cap = 5001, 5056
    cache = Cache(c, b, hkv, batch, cap, seed=keep)
    weights = torch.rand(batch, hkv, cap, device="cuda")
    kept, lens = cq.cq_select_tokens(weights, t, keep, 3, 100, torch.tensor([t] + [4700] * (batch - 1), dtype=torch.int32, device="cuda"))
    k, v, w = cache.k.clone(), cache.v.clone(), weights.clone()
    cq.cq_compact_cache(cache.k, cache.v, weights, cache.fmt, kept, lens, t, cap, k, v, w, cap)
    cq.cq_compact_cache(cache.k, cache.v, weights, cache.fmt, kept, lens, t, cap)
    assert torch.equal(cache.k, k) and torch.equal(cache.v, v) and torch.equal(weights, w)


def test_captured():
    cache = Cache(4, 8, 4, 4, 1024, seed=8)
    f = cache.fmt
    start = [cache.k.clone(), cache.v.clone(), torch.rand(4, 4, 1024, device="cuda")]
    k, v, w = (x.clone() for x in start)
    select, kept, lens = cq.prepare_select_tokens(w, 1000, 300, 4, 50)
    move = cq.prepare_compact_cache(k, v, w, f, kept, lens, 1000, 1024)
    select()
    move()
    torch.cuda.synchronize()
    want = [x.clone() for x in (k, v, w, kept, lens)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        select()
        move()
    for _ in range(3):
        for x, s in zip((k, v, w), start):
            x.copy_(s)
        kept.zero_()
        lens.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip((k, v, w, kept, lens), want))
        select()
        move()
        torch.cuda.synchronize()


def test_what_a_call_on_another_stream_allocates_is_its_own():
    """Workspaces and outputs of a call on a stream, while the current stream fills freed memory of the same sizes."""
    cache = Cache(8, 8, 8, 2, 4096, seed=9)
    q, rows = queries((2, 8, 128), 1), queries((2, 5, 8, 128), 2)
    drawn = torch.rand(2, 8, 20000, device="cuda")
    side = torch.cuda.Stream()

    def all_of_them(stream):
        w, chunk = torch.zeros(2, 8, 4096, device="cuda"), torch.zeros(2, 8, 4096, device="cuda")
        if stream is not None:
            stream.wait_stream(torch.cuda.current_stream())
        args = (cache.k, cache.v, cache.ck, cache.cv, SCALE, cache.fmt, 4000, 4096)
        out = [cq.cq_decode_attention_window(q, *args, 3000, 5, stream=stream), cq.cq_decode_attention_weights(q, *args, w, stream=stream),
               cq.cq_chunk_attention_window(rows, *args, 3000, 5, stream=stream), *cq.cq_select_tokens(drawn, 20000, 500, 4, 32, stream=stream)]
        cq.cq_chunk_weights(rows, cache.k, cache.ck, SCALE, cache.fmt, 4000, 4096, chunk, stream=stream)
        return out + [w, chunk]

    want = all_of_them(None)
    torch.cuda.synchronize()
    sizes = [1 << k for k in range(9, 23)]
    for _ in range(10):
        held = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in sizes]
        del held
        got = all_of_them(side)
        for n in sizes:
            torch.empty(n, dtype=torch.uint8, device="cuda").fill_(255)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, want))


@pytest.mark.parametrize("c,b", FORMATS)
def test_a_bounded_cache_in_use(c, b):
    """Prompt, weights over some steps, eviction, more steps with the accumulators carried on, a second eviction, and a window
    over what is left: each output against the definition over the codes that the cache should hold."""
    batch, hkv, hq, cap = 3, 2, 4, 512
    cache = Cache(c, b, hkv, batch, cap, seed=11)
    f, gh = cache.fmt, 128 // c
    fresh = Cache(c, b, hkv, batch, cap, seed=12)                                   # tokens to come
    fresh.books, fresh.ck, fresh.cv = cache.books, cache.ck, cache.cv
    length = 300
    weights = torch.zeros(batch, hkv, cap, device="cuda")
    total = torch.zeros(batch, hkv, cap, dtype=torch.float64)
    room = torch.zeros(batch, hkv, cap, dtype=torch.float64)
    for step in range(60):
        # the new token's codes, as cq_encode_kv would leave them
        for which, buf in enumerate((cache.k, cache.v)):
            cache.codes[which][:, length] = fresh.codes[which][:, step]
            buf.copy_(torch.from_numpy(L.pack(cache.codes[which], c, b, 128, hkv, cap).reshape(-1)))
        length += 1
        q = queries((batch, hq, 128), step)
        out = cq.cq_decode_attention_weights(q, cache.k, cache.v, cache.ck, cache.cv, SCALE, f, length, cap, weights, 0.9)
        ref, sums, largest = attention(cache, q[:, None], [length] * batch)
        check_attention(out.cpu().numpy(), ref[:, 0].numpy())
        total = 0.9 * total + sums
        room = 0.9 * room + weight_tolerance(largest, 2) * sums + 2.0 ** -22 * total
        assert ((weights.double().cpu() - total).abs() <= room).all()
        if step in (20, 45):
            before = weights.clone()
            kept, lens = cq.cq_select_tokens(weights, length, 256, 4, 16)
            want, _ = select_oracle(before.cpu().numpy(), length, [length] * batch, 256, 4, 16)
            assert np.array_equal(kept.cpu().numpy(), want)
            cq.cq_compact_cache(cache.k, cache.v, weights, f, kept, lens, length, cap)
            for which, buf in enumerate((cache.k, cache.v)):
                cache.codes[which] = _moved(cache, which, want, [256] * batch, cache.codes[which])
                assert np.array_equal(_unpack(buf, f, batch, cap), cache.codes[which])
            at = torch.from_numpy(want.astype(np.int64))
            for x in (total, room):
                x[..., :256] = x.gather(-1, at)
                x[..., 256:] = 0
            length = 256
            assert (lens == 256).all()
    q = queries((batch, hq, 128), 99)
    out = cq.cq_decode_attention_window(q, cache.k, cache.v, cache.ck, cache.cv, SCALE, f, length, cap, 100, 4)
    ref, _, _ = attention(cache, q[:, None], [length] * batch, 100, 4)
    check_attention(out.cpu().numpy(), ref[:, 0].numpy())
