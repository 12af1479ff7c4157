"""Random coded caches and 64-bit definitions for the tests of windows, attention weights and eviction.

The definitions work on codes in group order, tokens x groups; the packed caches are made of them by the oracle's layout.
"""
from __future__ import annotations

import numpy as np
import torch

import paper_2405_03917_amd as cq
from oracle import code_layout as L

FORMATS = [(8, 8), (4, 8), (2, 8), (8, 10)]
SCALE = 1.0 / np.sqrt(128.0)


class Cache:
    """Codes, codebooks and packed caches (contiguous, and the same contents as shuffled pages) of `batch` sequences."""

    def __init__(self, c, b, hkv, batch, t_cap, seed, spread=1.0):
        rng = np.random.default_rng(seed)
        self.fmt = cq.CQFormat(c, b, 128, hkv)
        self.batch, self.t_cap, self.tiles = batch, t_cap, t_cap // 64
        g = self.fmt.groups
        self.codes = [np.minimum(*rng.integers(0, 1 << b, (2, batch, t_cap, g))).astype(np.uint16) for _ in range(2)]
        self.books = [(spread * rng.standard_normal((g, 1 << b, c))).astype(np.float16) for _ in range(2)]
        packed = [L.pack(x, c, b, 128, hkv, t_cap) for x in self.codes]
        self.k, self.v = (torch.from_numpy(x.reshape(-1)).cuda() for x in packed)
        self.ck, self.cv = (torch.from_numpy(x).cuda() for x in self.books)
        self.n_pages = batch * self.tiles + 3
        self.table = rng.permutation(self.n_pages)[:batch * self.tiles].reshape(batch, self.tiles).astype(np.int32)
        self.pools = []
        for x in packed:
            pool = rng.integers(0, 256, (self.n_pages, hkv, x.shape[-1])).astype(np.uint8)
            pool[self.table] = x.transpose(0, 2, 1, 3)
            self.pools.append(torch.from_numpy(pool.reshape(-1)).cuda())

    def pages(self, table=None):
        return cq.PageTable(torch.from_numpy(np.ascontiguousarray(self.table if table is None else table)).cuda(), self.n_pages)

    def dense(self, which, n, h, length):
        """fp64 [length, 128] of KV head h of sequence n: which = 0 keys, 1 values."""
        f = self.fmt
        gh = 128 // f.c
        codes = torch.from_numpy(self.codes[which][n, :length, h * gh:(h + 1) * gh].astype(np.int64)).cuda()
        book = (self.ck, self.cv)[which][h * gh:(h + 1) * gh].double()
        return book[torch.arange(gh, device="cuda")[None], codes].reshape(length, 128)


def queries(shape, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (scale * torch.randn(*shape, generator=g)).half().cuda()


def visible(length, m, window=None, n_sink=0):
    """bool [m, length]: what each of the last m tokens sees."""
    i, p = np.arange(length)[None], np.arange(length - m, length)[:, None]
    seen = i <= p
    if window is not None:
        seen &= (i > p - window) | (i < n_sink)
    return seen


def attention(cache, q, lens, window=None, n_sink=0, scale=SCALE):
    """(out fp64 [B, m, Hq, 128], weights fp64 [B, Hkv, t_cap] summed over rows and heads, bound on the error of a score in fp32):
    q [B, m, Hq, 128]."""
    batch, m, hq, _ = q.shape
    f = cache.fmt
    qper = hq // f.n_kv_heads
    out = torch.zeros(batch, m, hq, 128, dtype=torch.float64)
    sums = torch.zeros(batch, f.n_kv_heads, cache.t_cap, dtype=torch.float64)
    largest = 0.0
    for n, length in enumerate(lens):
        ok = torch.from_numpy(visible(length, m, window, n_sink)).cuda()
        for h in range(f.n_kv_heads):
            k, v = cache.dense(0, n, h, length), cache.dense(1, n, h, length)
            rows = q[n, :, h * qper:(h + 1) * qper].double()                       # [m, qper, 128]
            s = (rows @ k.T) * scale
            p = torch.softmax(s.masked_fill(~ok[:, None], -torch.inf), -1)
            out[n, :, h * qper:(h + 1) * qper] = (p @ v).cpu()
            sums[n, h, :length] = p.sum((0, 1)).cpu()
            largest = max(largest, float((rows.abs() @ k.abs().T).max()) * abs(scale))
    return out, sums, largest


def weight_tolerance(largest, n_rows):
    """Relative error of a sum of softmax weights.  A score is a sum of at most 128 products in fp32: the roundings of
    products and sums are at most (128 + 4) 2^-24 of sum |q_i k_i| scale = `largest`, wherever they fall, and as much for
    the reference of the sum; the exponential, sum of the context, reciprocal and sum over n_rows rows add less than
    (64 + n_rows) 2^-24."""
    return (2 * 132 * largest + 64 + n_rows) * 2.0 ** -24
