"""The 8-bit block cache in 64 bits, from its definition: caches as numpy arrays, appends token range by token range, dense rows and
attention.  Nothing here comes from the library but the byte order it documents."""
from __future__ import annotations

import numpy as np
import torch

import paper_2405_03917_amd as cq

D, TILE = 128, 64
SCALE = 1.0 / np.sqrt(128.0)
KINDS = ("int8", "e4m3")

_low = [f / 8 * 2.0 ** -6 if e == 0 else (1 + f / 8) * 2.0 ** (e - 7) for e in range(16) for f in range(8)]
_low[127] = np.nan
E4M3 = np.array(_low + [-x for x in _low])
_order = np.argsort(E4M3[:127])                              # magnitudes ascending: codes 0 .. 126
INT8 = np.arange(256) - 128.0


def values_of(kind, byte):
    return (INT8 if kind == "int8" else E4M3)[byte]


def code_of(kind, x):
    """Nearest code bytes of fp64 numbers in units of the scale, ties to the even code; zero, of either
    sign, has the code 0."""
    if kind == "int8":
        return (np.clip(np.rint(x), -127, 127) + 128).astype(np.uint8)
    grid = E4M3[:127]
    a = np.minimum(np.abs(x), 448.0)
    hi = np.clip(np.searchsorted(grid, a), 1, 126)
    below, above = a - grid[hi - 1], grid[hi] - a
    code = np.where((above < below) | ((above == below) & (hi % 2 == 0)), hi, hi - 1)
    return (code | np.where(x < 0, 128, 0)).astype(np.uint8)


def need(kind, largest):
    if kind == "int8":
        return np.float64(np.float32(largest / 127.0))
    if largest == 0:
        return 0.0
    part, e = np.frexp(largest / 448.0)
    return float(2.0 ** (e - 1 if part == 0.5 else e))


def rotated(x, pos, base):
    """fp64 [..., 128] rows rotated to positions [...]."""
    angle = np.asarray(pos, np.float64)[..., None] * base ** (-2.0 * np.arange(64) / 128)
    c, s = np.cos(angle), np.sin(angle)
    lo, hi = x[..., :64], x[..., 64:]
    return np.concatenate([lo * c - hi * s, hi * c + lo * s], -1)


class Cache:
    """Code bytes [batch][KV head][tile] of keys [64][128] and values [128][64] and their scales, with the device arrays of the
    same contents, contiguous or as shuffled pages."""

    def __init__(self, kind, hkv, batch, t_cap, seed, paged=False, fill=None):
        self.rng = np.random.default_rng(seed)
        self.kind, self.hkv, self.batch, self.t_cap, self.tiles, self.paged = kind, hkv, batch, t_cap, t_cap // TILE, paged
        self.fmt = cq.Q8Format(kind, D, hkv)
        shape = (batch, hkv, self.tiles)
        if fill is None:
            k, v = (code_of(kind, self.rng.standard_normal(shape + (TILE * D,)) * (31 if kind == "int8" else 70)) for _ in range(2))
            size = np.exp(0.4 * self.rng.standard_normal((2,) + shape))
            scales = (size / 31).astype(np.float32) if kind == "int8" else np.exp2(np.rint(np.log2(size / 70))).astype(np.float32)
        else:
            k, v = (np.full(shape + (TILE * D,), fill, np.uint8) for _ in range(2))
            scales = np.full((2,) + shape, np.nan, np.float32)
        self.k, self.v = k.reshape(shape + (TILE, D)), v.reshape(shape + (D, TILE))
        self.s = [scales[0].copy(), scales[1].copy()]
        self.n_pages = batch * self.tiles + 3
        self.table = self.rng.permutation(self.n_pages)[:batch * self.tiles].reshape(batch, self.tiles).astype(np.int32)
        self.upload()

    def upload(self):
        def place(x):
            if not self.paged:
                return torch.from_numpy(np.ascontiguousarray(x).reshape(-1)).cuda()
            flat = x.reshape(self.batch, self.hkv, self.tiles, -1).transpose(0, 2, 1, 3)
            pool = np.full((self.n_pages,) + flat.shape[2:], 0x7f, x.dtype)
            pool[self.table] = flat
            return torch.from_numpy(pool.reshape(-1)).cuda()
        self.dev = cq.Q8Cache(place(self.k), place(self.v), place(self.s[0]), place(self.s[1]))
        self.before = cq.Q8Cache(*(x.clone() for x in (self.dev.k, self.dev.v, self.dev.k_scales, self.dev.v_scales)))

    def pages(self):
        return cq.PageTable(torch.from_numpy(self.table).cuda(), self.n_pages) if self.paged else None

    def where(self, lens=None):
        return dict(t_cap=self.t_cap, pages=self.pages(), seq_lens=None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda"))

    def download(self):
        """(k, v, k_scales, v_scales) of the device arrays in the order of this object's."""
        def back(x, shape):
            x = x.cpu().numpy()
            if not self.paged:
                return x.reshape((self.batch, self.hkv, self.tiles) + shape)
            return x.reshape((self.n_pages, self.hkv) + shape)[self.table].swapaxes(1, 2)
        d = self.dev
        return back(d.k, (TILE, D)), back(d.v, (D, TILE)), back(d.k_scales, ()), back(d.v_scales, ())

    def unused_pages_are_untouched(self):
        if not self.paged:
            return True
        free = torch.tensor(sorted(set(range(self.n_pages)) - set(self.table.reshape(-1).tolist())), device="cuda")
        pairs = zip((self.dev.k, self.dev.v, self.dev.k_scales, self.dev.v_scales), (self.before.k, self.before.v, self.before.k_scales, self.before.v_scales))
        return all(torch.equal(a.view(self.n_pages, -1)[free].view(torch.uint8), b.view(self.n_pages, -1)[free].view(torch.uint8)) for a, b in pairs)

    def append(self, x_k, x_v, t, lens=None, base=None):
        """The definition: x fp16 [batch, m, hkv * 128]; returns how near to a border the nearest number was, in units of the gap."""
        m = x_k.shape[1]
        for n in range(self.batch):
            t_n = t if lens is None else min(max(lens[n], 0), t)
            start = max(t_n - m, 0)
            rows = range(m - (t_n - start), m)
            for which, x in enumerate((x_k, x_v)):
                x = x[n].astype(np.float64).reshape(m, self.hkv, D)[rows.start:]
                if which == 0 and base is not None:
                    x = rotated(x, np.arange(start, t_n)[:, None], base)
                for tile in range(start // TILE, -(-t_n // TILE)):
                    lo, hi = max(start - tile * TILE, 0), min(t_n - tile * TILE, TILE)
                    part = x[tile * TILE + lo - start:tile * TILE + hi - start]
                    for h in range(self.hkv):
                        codes = self.k[n, h, tile] if which == 0 else self.v[n, h, tile].T
                        had = np.float64(self.s[which][n, h, tile]) if lo else 0.0
                        s = max(had, need(self.kind, np.abs(part[:, h]).max()))
                        if s > had and lo:
                            codes[:lo] = code_of(self.kind, values_of(self.kind, codes[:lo]) * (had / s))
                        codes[lo:hi] = code_of(self.kind, part[:, h] / s if s else part[:, h])
                        self.s[which][n, h, tile] = s

    def dense(self, which, n, h, length):
        """fp64 [length, 128]"""
        tiles = -(-length // TILE)
        x = values_of(self.kind, (self.k if which == 0 else self.v.swapaxes(-1, -2))[n, h, :tiles])
        return (x * self.s[which][n, h, :tiles].astype(np.float64)[:, None, None]).reshape(-1, D)[:length]

    def attention(self, q, t, lens=None, scale=SCALE):
        """(out, tolerance) of q fp16 [batch, m, Hq, 128] (torch, any device): fp64, and what the kernel's arithmetic may be off."""
        batch, m, hq, _ = q.shape
        qper = hq // self.hkv
        out, tol = np.zeros(q.shape), np.zeros(q.shape)
        for n in range(batch):
            t_n = t if lens is None else min(max(lens[n], 0), t)
            p = t_n - m + np.arange(m)
            rows = np.nonzero(p >= 0)[0]
            if not rows.size:
                continue
            hidden = torch.from_numpy(np.arange(t_n)[None] > p[rows][:, None]).cuda()
            for h in range(self.hkv):
                k, v = (torch.from_numpy(self.dense(w, n, h, t_n)).cuda() for w in (0, 1))
                x = q[n, torch.from_numpy(rows).to(q.device), h * qper:(h + 1) * qper].double().cuda()      # [rows, qper, 128]
                s = torch.matmul(x, k.T.contiguous()) * scale
                w = torch.softmax(s.masked_fill(hidden[:, None], -torch.inf), -1)
                y, a = torch.matmul(w, v), torch.matmul(w, v.abs())
                largest = float(torch.matmul(x.abs(), k.abs().T.contiguous()).max()) * abs(scale)
                o = slice(h * qper, (h + 1) * qper)
                out[n, rows, o] = y.cpu().numpy()
                tol[n, rows, o] = tolerance(y, a, largest, t_n, float(v.abs().max())).cpu().numpy()
        return out, tol


def tolerance(y, a, largest, t, v_max):
    """What an output y = sum p v may be off, with a = sum p |v|.

    A score is a sum of 128 exact products in fp32: at most 132 2^-24 of scale sum |q k| <= `largest` off, and as much again for the
    reference (`scale` times log2 e and the block's scale are rounded too: 4 2^-24 more each).  Each weight is rounded to fp16
    once: 2^-11 of itself, or, below fp16's normal numbers, half its smallest, 2^-25, at weights of 2^-8 and more for the
    largest (the reference may lie 2^8 below it): 2^-17 2^-25 ... counted as 2^-32 of the largest weight for each of t tokens.  Sums
    over tiles in fp32: (64 + t / 16) 2^-24.  The output is rounded to fp16: 2^-11 of itself, 2^-25 for the smallest."""
    eps = 2.0 ** -24
    return a * (2.0 ** -11 + (2 * 140 * largest + 256 + t / 16) * eps) + t * 2.0 ** -31 * v_max + abs(y) * 2.0 ** -11 + 2.0 ** -25


def randn(shape, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (scale * torch.randn(*shape, generator=g)).half().cuda()
