"""Chunks through windows over caches that are full to their last token, in splits that some rows' views do not reach, against
the 64-bit definition.  (Which tiles are requested there is checked on the host, test_view_tiles.py.)"""
import numpy as np
import pytest
import torch

import paper_2405_03917_amd as cq
from bounded_util import SCALE, Cache, attention, queries
from gpu_util import check_attention

pytestmark = pytest.mark.gpu


# (the second with the library's own split: pieces of 9 of at most 82 tiles, where some rows see 81)
@pytest.mark.parametrize("c,batch,hq,hkv,m,t,window,n_sink,split", [(8, 1, 8, 8, 5, 4096, 1024, 4, 128), (4, 2, 16, 4, 10, 23872, 5076, 4, 0),
                                                                   (8, 2, 16, 4, 10, 23872, 5076, 4, 576), (4, 3, 4, 4, 17, 1024, 200, 70, 64),
                                                                   (8, 2, 8, 2, 9, 640, 129, 0, 64), (4, 2, 4, 2, 3, 640, 130, 5, 64)])
def test_full_caches(c, batch, hq, hkv, m, t, window, n_sink, split):
    cache = Cache(c, 8, hkv, batch, t, seed=m)
    q = queries((batch, m, hq, 128), t)
    sl = [t] + [t - 63 if t > 64 else t] * (batch - 1)
    lens = torch.tensor(sl, dtype=torch.int32, device="cuda")
    args = (cache.ck, cache.cv, SCALE, cache.fmt, t)
    out = cq.cq_chunk_attention_window(q, cache.k, cache.v, *args, t, window, n_sink, lens, split)
    paged = cq.cq_chunk_attention_window_paged(q, *cache.pools, *args, cache.pages(), window, n_sink, lens, split)
    ref, _, _ = attention(cache, q, sl, window, n_sink)
    check_attention(out.cpu().numpy(), ref.numpy())
    assert np.array_equal(out.cpu().numpy(), paged.cpu().numpy())
