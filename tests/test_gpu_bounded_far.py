"""Calls that keep a cache bounded on a stream whose codes pass 4 GiB: what lies at its far end against a small cache that holds
the same tokens."""
import pytest
import torch

import paper_2405_03917_amd as cq
from bounded_util import weight_tolerance

pytestmark = pytest.mark.gpu

FMT = cq.CQFormat(2, 8, 128, 1)                             # 64 bytes a token
T = (1 << 26) + 5 * 64 + 17                                 # 4 GiB, and some tiles
CAP = -(-T // 64) * 64
NEAR = 4096                                                 # tokens of the small cache: the far end's, at the same places of their tiles
SHIFT = CAP - NEAR
SCALE = 0.09


@pytest.fixture(scope="module")
def far():
    g = torch.Generator(device="cuda").manual_seed(1)
    k, v = (torch.randint(0, 256, (CAP * 64,), generator=g, device="cuda", dtype=torch.uint8) for _ in range(2))
    ck, cv = (torch.randn(64, 256, 2, generator=g, device="cuda").half() for _ in range(2))
    near = [x[SHIFT * 64:].clone() for x in (k, v)]
    yield (k, v), near, ck, cv
    torch.cuda.empty_cache()


@pytest.mark.parametrize("m,window", [(0, 2000), (1, 3000), (5, 1000), (40, 1500), (300, 2000)])
def test_windows(far, m, window):
    (k, v), near, ck, cv = far
    g = torch.Generator(device="cuda").manual_seed(m)
    q = torch.randn(1, max(m, 1), 4, 128, generator=g, device="cuda").half()
    if m == 0:
        out = cq.cq_decode_attention_window(q[:, 0].contiguous(), k, v, ck, cv, SCALE, FMT, T, CAP, window)
        want = cq.cq_decode_attention_window(q[:, 0].contiguous(), *near, ck, cv, SCALE, FMT, T - SHIFT, NEAR, window)
    else:
        out = cq.cq_chunk_attention_window(q, k, v, ck, cv, SCALE, FMT, T, CAP, window)
        want = cq.cq_chunk_attention_window(q, *near, ck, cv, SCALE, FMT, T - SHIFT, NEAR, window)
    # the same tiles, walked in the same order
    assert torch.equal(out, want)


def test_weights(far):
    (k, v), near, ck, cv = far
    q = torch.randn(1, 1, 128, generator=torch.Generator(device="cuda").manual_seed(5), device="cuda").half()
    w, chunk, last = (torch.zeros(1, 1, n, device="cuda") for n in (CAP, CAP, NEAR))
    cq.cq_decode_attention_weights(q, k, v, ck, cv, SCALE, FMT, T, CAP, w, 0.0)
    cq.cq_chunk_weights(q[:, None], k, ck, SCALE, FMT, T, CAP, chunk, 0.0)
    cq.cq_decode_attention_weights(q, *near, ck, cv, SCALE, FMT, T - SHIFT, NEAR, last, 0.0)
    room = weight_tolerance(16.0, 1)                        # (sum |q_i k_i| scale: 128 terms of mean 0.64 0.09, below 16 for every token)
    assert all(abs(float(x.double().sum()) - 1) <= room for x in (w, chunk))
    # the last tokens' weights are those of the small cache times one factor
    n = T - SHIFT
    for got in (w[0, 0, SHIFT:T].double(), chunk[0, 0, SHIFT:T].double()):
        want = last[0, 0, :n].double()
        factor = got.sum() / want.sum()
        assert ((got - want * factor).abs() <= 4 * room * want * factor).all()      # (weights and factor, of both caches)


def test_selection_and_compaction(far):
    (k, v), near, _, _ = far
    w = torch.rand(1, 1, CAP, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda")
    w[..., SHIFT:T - 100] += 1                              # the heaviest: all of the far end
    keep = 3000
    kept, lens = cq.cq_select_tokens(w, T, keep, 0, 100)
    middle = torch.sort(w[0, 0, :T - 100], descending=True, stable=True).indices[:keep - 100].sort().values
    assert torch.equal(kept[0, 0].long(), torch.cat([middle, torch.arange(T - 100, T, device="cuda")]))
    assert int(kept.min()) >= SHIFT and int(lens[0]) == keep
    small = [torch.zeros(-(-keep // 64) * 64 * 64, dtype=torch.uint8, device="cuda") for _ in range(4)]
    w2, w3 = torch.zeros(1, 1, 3008, device="cuda"), torch.zeros(1, 1, 3008, device="cuda")
    cq.cq_compact_cache(k, v, w, FMT, kept, lens, T, CAP, small[0], small[1], w2, 3008)
    cq.cq_compact_cache(*near, w[..., SHIFT:].contiguous(), FMT, (kept - SHIFT).contiguous(), lens, T - SHIFT, NEAR, small[2], small[3], w3, 3008)
    assert torch.equal(small[0], small[2]) and torch.equal(small[1], small[3]) and torch.equal(w2, w3)
    # in place
    k2, v2, mine = k.clone(), v.clone(), w.clone()
    cq.cq_compact_cache(k2, v2, mine, FMT, kept, lens, T, CAP)
    assert torch.equal(k2[:46 * 4096], small[0][:46 * 4096]) and torch.equal(v2[:46 * 4096], small[1][:46 * 4096])
    assert torch.equal(mine[..., :keep], w2[..., :keep]) and not mine[..., keep:T].any()
    assert torch.equal(k2[48 * 4096:], k[48 * 4096:])
