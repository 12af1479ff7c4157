"""The calls of the 8-bit block cache as a program makes them one behind the other: prompt, chunk, decode steps; captured, on other
streams, beyond 4 GiB."""
import numpy as np
import pytest
import torch

import paper_2405_03917_amd as cq
from q8_util import D, KINDS, SCALE, TILE, Cache, randn

pytestmark = pytest.mark.gpu
BASE = 10000.0
HQ, HKV = 8, 2


def _qkv(batch, m, seed):
    x = randn((batch, m, (HQ + 2 * HKV) * D), seed)
    q, k, v = x.split((HQ * D, HKV * D, HKV * D), dim=-1)
    return q.unflatten(-1, (HQ, D)), k, v


def _check(cache, q, out, t, lens=None):
    want, tol = cache.attention(q, t, lens)
    assert (np.abs(out.cpu().numpy().astype(np.float64) - want) <= tol).all()


@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("kind", KINDS)
def test_prompt_chunk_and_steps(kind, paged):
    """Ragged prompts, a chunk of five, ten steps: every call's output against the definition over the cache that the definition
    appended to, and the cache bit for bit at the end."""
    cache = Cache(kind, HKV, 3, 320, seed=1, paged=paged, fill=0xff)
    rope = cq.Q8RopeTable(BASE, 320)
    lens = np.array([200, 1, 77])
    for i, m in enumerate([200, 5] + [1] * 10):
        if i:
            lens = lens + m
        t = int(lens.max())
        q, k, v = _qkv(3, m, 100 + i)
        where = cache.where(lens.tolist())
        call, turned = cq.prepare_append_q8(k, v, cache.dev, cache.fmt, t, rope=rope, q=q, **where)
        call()
        cache.append(k.cpu().numpy(), v.cpu().numpy(), t, lens.tolist(), BASE)
        pad = [max(0, m - x) for x in lens]
        turned = torch.where(torch.arange(m, device="cuda")[None, :, None, None] >= torch.tensor(pad, device="cuda")[:, None, None, None], turned, 0)
        if m == 1:
            call, out = cq.prepare_decode_attention_q8(turned[:, 0].contiguous(), cache.dev, SCALE, cache.fmt, t, **where)
            call()
            _check(cache, turned, out[:, None], t, lens.tolist())
        else:
            call, out = cq.prepare_chunk_attention_q8(turned.contiguous(), cache.dev, SCALE, cache.fmt, t, **where)
            call()
            _check(cache, turned, out, t, lens.tolist())
    got = cache.download()
    for n, length in enumerate(lens):
        tile, u = divmod(int(length), TILE)
        assert np.array_equal(got[0][n, :, :tile], cache.k[n, :, :tile]) and np.array_equal(got[1][n, :, :tile], cache.v[n, :, :tile])
        assert np.array_equal(got[0][n, :, tile, :u], cache.k[n, :, tile, :u]) and np.array_equal(got[1][n, :, tile, :, :u], cache.v[n, :, tile, :, :u])
    k, v = (cq.cq_dequantize_q8_paged(cache.dev, cache.fmt, 3, 20, int(lens.max()), cache.pages(), where["seq_lens"]) if paged else
            cq.cq_dequantize_q8(cache.dev, cache.fmt, 3, 20, int(lens.max()), 320, where["seq_lens"]))
    for h in range(HKV):
        want = cache.dense(0, 2, h, int(lens[2]))[-20:]
        assert np.abs(k[2, :, h * D:(h + 1) * D].cpu().numpy() - want).max() <= 2.0 ** -11 * np.abs(want).max()


def _step(cache, rope, q, k, v, t, lens, split=0):
    """An append and the attention behind it, prepared: (calls, outputs)."""
    where = cache.where(None)
    where["seq_lens"] = lens
    append, turned = cq.prepare_append_q8(k, v, cache.dev, cache.fmt, t, rope=rope, q=q, **where)
    attend, out = cq.prepare_chunk_attention_q8(turned, cache.dev, SCALE, cache.fmt, t, tokens_per_split=split, **where)
    return (append, attend), out


def test_two_captured_steps_replayed():
    """Graphs of two batches, each with its own workspace, replayed in turn and at once on two streams, lengths that grow between replays;
    every replay against the eager calls on caches of their own."""
    rope = cq.Q8RopeTable(BASE, 4096)
    runs = []
    for i, kind in enumerate(KINDS):
        pair = [Cache(kind, HKV, 2, 4096, seed=20 + i, paged=bool(i)) for _ in range(2)]
        lens = torch.tensor([3000, 1000], dtype=torch.int32, device="cuda")
        buf = tuple(x.contiguous() for x in _qkv(2, 1, i))
        eager = _step(pair[0], rope, *buf, 4000, lens)
        replayed = _step(pair[1], rope, *buf, 4000, lens)
        torch.cuda.synchronize()
        graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        with torch.cuda.graph(graph, stream=side):
            for call in replayed[0]:
                call()
        runs.append((pair, lens, buf, eager, replayed, graph, torch.cuda.Stream()))
    for step in range(4):
        for pair, lens, buf, eager, replayed, graph, stream in runs:
            for b, x in zip(buf, _qkv(2, 1, 50 + step)):
                b.copy_(x)
            for call in eager[0]:
                call()
        torch.cuda.synchronize()
        for pair, lens, buf, eager, replayed, graph, stream in runs:
            with torch.cuda.stream(stream if step % 2 else torch.cuda.current_stream()):
                graph.replay()
        torch.cuda.synchronize()
        for pair, lens, buf, eager, replayed, graph, stream in runs:
            assert torch.equal(eager[1], replayed[1])
            for a, b in zip(pair[0].download(), pair[1].download()):
                assert np.ascontiguousarray(a).tobytes() == np.ascontiguousarray(b).tobytes()
            lens += 1
        torch.cuda.synchronize()


@pytest.mark.parametrize("hq,hkv,batch,m,t", [(32, 8, 1, 1, 2000), (32, 32, 2, 1, 2000), (8, 2, 3, 1, 1500), (2, 2, 4, 3, 4000), (12, 4, 2, 2, 900), (64, 2, 2, 1, 1000)])
def test_pieces_joined_inside_and_apart(hq, hkv, batch, m, t):
    """A captured call joins its pieces by a launch of its own, an eager one of few partial rows does not: the same bits, whatever
    order the workgroups ended in, on the stream of the capture and others."""
    cache = Cache("e4m3", hkv, batch, 4096, seed=t + hq)
    q = randn((batch, m, hq, D), hq, 2.0)
    lens = [t - 450 * n for n in range(batch)]
    assert t > cq.cq_attention_q8_default_split(cache.fmt, batch, hq, m, t)
    (eager, want), (captured, got) = (cq.prepare_chunk_attention_q8(q, cache.dev, SCALE, cache.fmt, t, **cache.where(lens)) for _ in range(2))
    eager()
    _check(cache, q, want, t, lens)
    first = want.clone()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        captured()
    for _ in range(4):
        got.zero_()
        want.zero_()
        graph.replay()
        eager()
        torch.cuda.synchronize()
        eager(side)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, first) and torch.equal(want, first)


def test_on_another_stream():
    cache = Cache("int8", HKV, 4, 2048, seed=30)
    rope = cq.Q8RopeTable(BASE, 2048)
    q, k, v = _qkv(4, 3, 1)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    q_out = cq.cq_append_q8(k, v, cache.dev, cache.fmt, 2000, 2048, rope=rope, q=q, stream=side)
    out = cq.cq_chunk_attention_q8(q_out, cache.dev, SCALE, cache.fmt, 2000, 2048, stream=side)
    one = cq.cq_decode_attention_q8(q_out[:, -1].contiguous(), cache.dev, SCALE, cache.fmt, 2000, 2048, stream=side) if side.synchronize() is None else None
    side.synchronize()
    cache.append(k.cpu().numpy(), v.cpu().numpy(), 2000, None, BASE)
    _check(cache, q_out, out, 2000)
    _check(cache, q_out[:, -1:], one[:, None], 2000)


def test_two_calls_at_once():
    """Calls on two streams at once, each with its own workspace, give what they give alone."""
    caches = [Cache(kind, HKV, 8, 4096, seed=31) for kind in KINDS]
    queries = [randn((8, 1, HQ, D), 1), randn((8, 40, HQ, D), 2)]
    calls = [cq.prepare_chunk_attention_q8(q, c.dev, SCALE, c.fmt, 4000, tokens_per_split=512, **c.where()) for c in caches for q in queries]
    want = []
    for call, out in calls:
        call()
        torch.cuda.synchronize()
        want.append(out.clone())
        out.zero_()
    streams = [torch.cuda.Stream() for _ in calls]
    torch.cuda.synchronize()
    for _ in range(5):
        for (call, _), s in zip(calls, streams):
            call(s)
    torch.cuda.synchronize()
    for (_, out), w in zip(calls, want):
        assert torch.equal(out, w)


@pytest.mark.parametrize("kind", KINDS)
def test_pools_of_more_than_4_gib(kind):
    """The last pages of pools of 4.5 GiB, and a contiguous stream behind 4 GiB of others."""
    hkv = 64
    n_pages = 9216                                           # 512 KiB of keys each
    fmt = cq.Q8Format(kind, D, hkv)
    pools = cq.alloc_q8_pools(fmt, n_pages)
    table = torch.tensor([[n_pages - 1, 3, n_pages - 2]], dtype=torch.int32, device="cuda")
    pages = cq.PageTable(table, n_pages)
    small = Cache(kind, hkv, 1, 192, seed=1, fill=0)
    x_k, x_v = randn((1, 150, hkv * D), 1), randn((1, 150, hkv * D), 2)
    q = randn((1, 4, hkv, D), 3)
    cq.cq_append_q8_paged(x_k, x_v, pools, fmt, 150, pages)
    cq.cq_append_q8(x_k, x_v, small.dev, fmt, 150, 192)
    want = cq.cq_chunk_attention_q8(q, small.dev, SCALE, fmt, 150, 192)
    assert torch.equal(cq.cq_chunk_attention_q8_paged(q, pools, SCALE, fmt, 150, pages), want)
    rows = cq.cq_dequantize_q8(small.dev, fmt, 1, 150, 150, 192)
    for a, b in zip(rows, cq.cq_dequantize_q8_paged(pools, fmt, 1, 150, 150, pages)):
        assert torch.equal(a, b)
    big = cq.Q8Cache(pools.k, pools.v, pools.k_scales, pools.v_scales)
    batch = n_pages // 3                                     # the same arrays as streams of three tiles
    lens = torch.zeros(batch, dtype=torch.int32, device="cuda")
    lens[-1] = 150
    wide_k, wide_v = (x.expand(batch, -1, -1) for x in (x_k, x_v))
    with pytest.raises(cq.CQError):                          # sequences that share their rows: refused
        cq.cq_append_q8(wide_k, wide_v, big, fmt, 150, 192, lens)
    one = cq.Q8Cache(*(x[-(x.numel() // batch):] for x in (pools.k, pools.v, pools.k_scales, pools.v_scales)))
    cq.cq_append_q8(x_k, x_v, one, fmt, 150, 192)
    out = cq.cq_chunk_attention_q8(q.expand(batch, -1, -1, -1).contiguous(), big, SCALE, fmt, 150, 192, lens)
    assert torch.equal(out[-1:], want) and (out[:-1] == 0).all()
