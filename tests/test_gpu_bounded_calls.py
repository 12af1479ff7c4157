"""Calls that keep a cache bounded, in the ways a program may make them that their other tests leave out."""
import pytest
import torch

import paper_2405_03917_amd as cq
from bounded_util import Cache

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("paged", [False, True])
def test_accumulators_in_place_under_another_tensor(paged):
    """The codes go elsewhere, the accumulators stay where they are, named by a view of the tensor they came in."""
    cache = Cache(4, 8, 2, 2, 512, seed=3)
    w = torch.rand(2, 2, 512, generator=torch.Generator().manual_seed(1)).cuda()
    kept, lens = cq.cq_select_tokens(w, 500, 130, 4, 20)
    k, v = cache.pools if paged else (cache.k, cache.v)

    def moved(weights, weights_out):
        k2, v2 = torch.zeros_like(k), torch.zeros_like(v)
        if paged:
            cq.cq_compact_cache_paged(k, v, weights, cache.fmt, kept, lens, 500, cache.pages(), k2, v2, weights_out)
        else:
            cq.cq_compact_cache(k, v, weights, cache.fmt, kept, lens, 500, 512, k2, v2, weights_out)
        return k2, v2, weights_out

    want = moved(w, w.clone())
    mine = w.clone()
    got = moved(mine, mine.view(2, 2, 512))
    assert all(torch.equal(x, y) for x, y in zip(got, want))


def test_tensors_dropped_behind_a_call_on_another_stream():
    """What a call on a busy stream reads and writes is dropped behind it, and the current stream fills memory of the same sizes."""
    cache = Cache(8, 8, 8, 2, 4096, seed=9)
    gen = torch.Generator().manual_seed(2)
    q, rows, new = ((torch.randn(*shape, generator=gen)).half() for shape in ((2, 8, 128), (2, 5, 8, 128), (2, cache.fmt.channels)))
    drawn, big = torch.rand(2, 8, 20000, generator=gen), torch.randn(8192, 8192, device="cuda").half()
    side = torch.cuda.Stream()
    args = (cache.ck, cache.cv, 0.09, cache.fmt)

    def all_of_them(stream):
        mine, mine_rows, x, w = q.cuda(), rows.cuda(), new.cuda(), drawn.cuda()
        k, v = cache.k.clone(), cache.v.clone()
        acc, chunk = torch.zeros(2, 8, 4096, device="cuda"), torch.zeros(2, 8, 4096, device="cuda")
        if stream is not None:
            stream.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(stream):
                for _ in range(8):
                    big @ big
        kept, lens = cq.cq_select_tokens(w, 20000, 500, 4, 32, stream=stream)
        cq.cq_chunk_weights(mine_rows, k, cache.ck, 0.09, cache.fmt, 4000, 4096, chunk, stream=stream)
        return [cq.cq_decode_step_window(mine, x, x, k, v, *args, 4000, 4096, 3000, 5, stream=stream),
                cq.cq_decode_attention_weights(mine, k, v, *args, 4000, 4096, acc, stream=stream),
                cq.cq_chunk_attention_window(mine_rows, k, v, *args, 4000, 4096, 3000, 5, stream=stream),
                cq.cq_decode_attention(mine, k, v, *args, 4000, 4096, stream=stream),
                cq.cq_chunk_attention(mine_rows, k, v, *args, 4000, 4096, stream=stream), kept, lens]

    want = all_of_them(None)
    torch.cuda.synchronize()
    sizes = [q.numel() * 2, rows.numel() * 2, new.numel() * 2, drawn.numel() * 4, cache.k.numel(), 2 * 8 * 4096 * 4]
    for _ in range(3):
        got = all_of_them(side)
        for _ in range(4):
            [torch.empty(n, dtype=torch.uint8, device="cuda").fill_(255) for n in sizes]
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, want))
