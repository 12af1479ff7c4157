"""Attention over the 8-bit cache where rows and pages are not there: queries of padding rows that are no numbers, and pages outside the
pool, which are taken for its first and its last."""
import numpy as np
import pytest
import torch

import paper_2405_03917_amd as cq
from q8_util import D, KINDS, SCALE, Cache, randn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("split", [0, 64])
@pytest.mark.parametrize("m,t,hq,hkv", [(1, 200, 4, 4), (6, 300, 8, 2), (70, 300, 8, 2), (150, 300, 4, 2), (600, 4800, 1, 1)])
def test_queries_of_padding_rows_are_no_matter(kind, split, m, t, hq, hkv):
    lens = [0, 1, m - 1, m, t]
    cache = Cache(kind, hkv, len(lens), -(-t // 64) * 64, seed=m)
    q = randn((len(lens), m, hq, D), m, 2.0)
    call, out = cq.prepare_chunk_attention_q8(q, cache.dev, SCALE, cache.fmt, t, tokens_per_split=split, **cache.where(lens))
    call()
    want = out.clone()
    for n, length in enumerate(lens):
        pad = max(0, m - length)
        assert (want[n, :pad] == 0).all()
        for i, bad in enumerate((float("nan"), float("inf"), -float("inf"))):
            q[n, i:pad:3] = bad
    out.fill_(7.0)
    call()
    assert torch.equal(out, want)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("m", [1, 3, 90, 150])
def test_pages_outside_the_pool_are_its_ends(kind, m):
    cache = Cache(kind, 2, 2, 256, seed=6, paged=True)
    free = sorted(set(range(cache.n_pages)) - set(cache.table.reshape(-1).tolist()))
    for x in (cache.dev.k, cache.dev.v, cache.dev.k_scales, cache.dev.v_scales):
        pool = x.view(cache.n_pages, -1)
        pool[free] = pool[int(cache.table[0, 0])].clone()            # (a page that a sequence has: finite codes and scales)
    q = randn((2, m, 4, D), 1)
    outside, inside = cache.table.copy(), cache.table.copy()
    outside[:, 2:] = [[-1, 1 << 30], [2 ** 31 - 1, -2 ** 31]]
    inside[:, 2:] = [[0, cache.n_pages - 1], [cache.n_pages - 1, 0]]
    outs = [cq.cq_chunk_attention_q8_paged(q, cache.dev, SCALE, cache.fmt, 250, cq.PageTable(torch.from_numpy(x).cuda(), cache.n_pages)) for x in (outside, inside)]
    assert torch.isfinite(outs[1].float()).all() and torch.equal(*outs)
    rows = [cq.cq_dequantize_q8_paged(cache.dev, cache.fmt, 2, 150, 250, cq.PageTable(torch.from_numpy(x).cuda(), cache.n_pages)) for x in (outside, inside)]
    assert all(torch.equal(a, b) for a, b in zip(*rows))
    assert not np.array_equal(outside, inside)
