"""Attention over the 8-bit block cache against the definition in 64 bits, with tolerances from the kernel's arithmetic (q8_util.tolerance)."""
import numpy as np
import pytest
import torch

import paper_2405_03917_amd as cq
from q8_util import D, KINDS, SCALE, TILE, Cache, randn

pytestmark = pytest.mark.gpu


def _chunk(cache, q, t, lens=None, scale=SCALE, **more):
    call, out = cq.prepare_chunk_attention_q8(q, cache.dev, scale, cache.fmt, t, **cache.where(lens), **more)
    call()
    return out


def _decode(cache, q, t, lens=None, scale=SCALE, **more):
    call, out = cq.prepare_decode_attention_q8(q, cache.dev, scale, cache.fmt, t, **cache.where(lens), **more)
    call()
    return out


def _check(cache, q, out, t, lens=None, scale=SCALE):
    want, tol = cache.attention(q, t, lens, scale)
    off = np.abs(out.cpu().numpy().astype(np.float64) - want)
    assert (off <= tol).all(), (float(np.nanmax(off / np.maximum(tol, 1e-30))), np.argwhere(~(off <= tol))[:4])


# heads of one, few and many queries: 1 to 32 rows of a KV head, more than a block of them, odd numbers
HEADS = [(4, 4), (8, 2), (3, 1), (32, 2), (17, 1), (40, 1), (64, 1)]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("hq,hkv", HEADS)
def test_decode_heads(kind, hq, hkv):
    cache = Cache(kind, hkv, 4, 512, seed=hq)
    q = randn((4, hq, D), hq, 2.0)
    lens = [500, 1, 64, 65]
    _check(cache, q[:, None], _decode(cache, q, 500, lens)[:, None], 500, lens)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("t", [1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 255, 256, 257, 1000, 5000, 20011])
def test_decode_lengths(kind, t):
    cache = Cache(kind, 2, 3, -(-t // 64) * 64, seed=t, paged=bool(t % 2))
    q = randn((3, 8, D), t, 2.0)
    lens = [t, max(1, t // 3), max(0, t - 64)]
    out = _decode(cache, q, t, lens)
    _check(cache, q[:, None], out[:, None], t, lens)
    _check(cache, q[:, None], _decode(cache, q, t)[:, None], t)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("hq,hkv", [(4, 4), (8, 2), (15, 5), (16, 1)])
@pytest.mark.parametrize("m,t", [(1, 70), (2, 2), (3, 64), (5, 700), (17, 300), (64, 64), (65, 129), (130, 130), (200, 1100), (333, 400)])
def test_chunk_sizes(kind, hq, hkv, m, t):
    cache = Cache(kind, hkv, 2, -(-t // 64) * 64, seed=t + m, paged=bool(m % 2))
    q = randn((2, m, hq, D), m, 2.0)
    lens = [t, max(m, t - 65)]
    _check(cache, q, _chunk(cache, q, t, lens), t, lens)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("m,hq,hkv", [(6, 4, 4), (70, 8, 2), (150, 2, 1), (300, 4, 4), (280, 4, 2)])
def test_padding_rows_are_zero(kind, m, hq, hkv):
    lens = [0, 1, m - 1, m, m + 1, 300, -5, 9999]
    cache = Cache(kind, hkv, len(lens), 320, seed=m)
    q = randn((len(lens), m, hq, D), m, 2.0)
    out = _chunk(cache, q, 300, lens)
    _check(cache, q, out, 300, lens)
    for n, length in enumerate(lens):
        pad = max(0, m - min(max(length, 0), 300))
        assert (out[n, :pad] == 0).all()
    one = _decode(cache, q[:, 0].contiguous(), 300, lens)
    assert (one[[0, 6]] == 0).all()
    _check(cache, q[:, :1], one[:, None], 300, lens)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("paged", [False, True])
def test_what_lies_behind_a_sequence_does_not_matter(kind, paged):
    """Codes behind the last token, whole tiles and their scales: any bytes (e4m3's no-number too), any scales (no numbers)."""
    lens = [130, 64, 1, 63, 190, 0]
    cache = Cache(kind, 2, 6, 320, seed=5, paged=paged)
    calls = [(randn((6, 8, D), 1, 2.0), _decode), (randn((6, 3, 8, D), 2, 2.0), _chunk), (randn((6, 90, 8, D), 3, 2.0), _chunk), (randn((6, 150, 8, D), 4, 2.0), _chunk)]
    want = [f(cache, q, 300, lens) for q, f in calls]
    for n, length in enumerate(lens):
        tile, u = length // TILE, length % TILE
        cache.k[n, :, tile, u:] = cache.v[n, :, tile, :, u:] = 0x7f
        cache.k[n, :, tile + 1:] = cache.v[n, :, tile + 1:] = 0xff
        for s in cache.s:
            s[n, :, tile + (u > 0):] = np.nan
    cache.upload()
    for (q, f), w in zip(calls, want):
        assert torch.equal(f(cache, q, 300, lens), w)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("split", [0, 640])
def test_long_contexts_in_front_of_many_rows(kind, paged, split):
    """600 rows behind up to 4200 tokens, ragged: all, some and none of the rows have tokens; then what lies behind the sequences changes."""
    lens = [4800, 650, 4736, 599, 64, 0]
    cache = Cache(kind, 1, 6, 4864, seed=21, paged=paged)
    q = randn((6, 600, 1, D), 5, 2.0)
    out = _chunk(cache, q, 4800, lens, tokens_per_split=split)
    _check(cache, q, out, 4800, lens)
    for n, length in enumerate(lens):
        tile, u = length // TILE, length % TILE
        cache.k[n, :, tile, u:] = cache.v[n, :, tile, :, u:] = 0x7f
        cache.k[n, :, tile + 1:] = cache.v[n, :, tile + 1:] = 0xff
        for x in cache.s:
            x[n, :, tile + (u > 0):] = np.nan
    cache.upload()
    assert torch.equal(_chunk(cache, q, 4800, lens, tokens_per_split=split), out)


@pytest.mark.parametrize("kind", KINDS)
def test_pages_outside_the_pool_cannot_be_reached(kind):
    """Entries are clamped to the pool, and entries of tiles behind a sequence are not used."""
    cache = Cache(kind, 2, 2, 256, seed=6, paged=True)
    q = randn((2, 3, 4, D), 1)
    lens = [100, 70]
    want = _chunk(cache, q, 200, lens)
    table = cache.table.copy()
    table[:, 2:] = [[-1, 1 << 30], [2 ** 31 - 1, -2 ** 31]]
    pages = cq.PageTable(torch.from_numpy(table).cuda(), cache.n_pages)
    sl = torch.tensor(lens, dtype=torch.int32, device="cuda")
    assert torch.equal(cq.cq_chunk_attention_q8_paged(q, cache.dev, SCALE, cache.fmt, 200, pages, sl), want)
    assert torch.isfinite(cq.cq_chunk_attention_q8_paged(q, cache.dev, SCALE, cache.fmt, 200, pages).float()).all() or kind == "e4m3"


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("split", [64, 128, 192, 320, 1024])
def test_given_splits(kind, split):
    cache = Cache(kind, 2, 3, 1088, seed=split)
    lens = [1055, 0, 700]
    for m in (1, 5, 150):
        q = randn((3, m, 8, D), m + split, 2.0)
        out = _chunk(cache, q, 1055, lens, tokens_per_split=split)
        _check(cache, q, out, 1055, lens)
    q = randn((3, 8, D), split, 2.0)
    _check(cache, q[:, None], _decode(cache, q, 1055, lens, tokens_per_split=split)[:, None], 1055, lens)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("m", [1, 150, 300])
def test_scales_of_every_sign(kind, m):
    cache = Cache(kind, 2, 2, 448, seed=11)
    q = randn((2, m, 4, D), m)
    for scale in (-0.3, 0.0, 1e-30, 3.0):
        _check(cache, q, _chunk(cache, q, 400, scale=scale), 400, scale=scale)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("m", [1, 150, 300])
def test_scores_far_beyond_the_24_bits_of_a_float(kind, m):
    """One token's score is larger by 2^20 than all others': its value is the output.  The largest number's own rounding must not
    show."""
    cache = Cache(kind, 1, 2, 320, seed=12)
    q = randn((2, m, 2, D), 3)
    cache.k[...] = 128 if kind == "int8" else 0
    code = 128 + 100 if kind == "int8" else 0x70                # 100, 128
    for n, tok in ((0, 77), (1, 5)):
        cache.k[n, 0, tok // 64, tok % 64, 9] = code
    cache.s[0][...] = 1.0
    cache.upload()
    q[..., 9] = 1000.0
    out = _chunk(cache, q, 320, scale=1000.3)
    pos = 320 - m + np.arange(m)
    for n, tok in ((0, 77), (1, 5)):
        rows = np.nonzero(pos >= tok)[0]
        want = np.broadcast_to(cache.dense(1, n, 0, 320)[tok], (rows.size, 2, D))
        got = out[n, torch.from_numpy(rows).cuda()].cpu().numpy()
        assert (np.abs(got - want) <= 2.0 ** -10 * np.abs(want) + 2.0 ** -25).all()     # weight and output, a rounding each


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("m", [1, 130, 600])
def test_many_small_weights_are_not_lost(kind, m):
    """The first token outweighs each of the others by 2^24.5; together they are a few thousandths of the sum, whose values alone are
    not zero in channel 1."""
    t = 65536
    cache = Cache(kind, 1, 1, t, seed=13, fill=128 if kind == "int8" else 0)
    one = 129 if kind == "int8" else 0x38                       # 1
    for s in cache.s:
        s[...] = 1.0
    cache.k[0, 0, 0, 0, 0] = one
    cache.v[0, 0, :, 1, :] = one
    cache.v[0, 0, 0, 1, 0] = 128 if kind == "int8" else 0
    cache.upload()
    q = torch.zeros(1, m, 1, D, dtype=torch.float16, device="cuda")
    q[..., 0] = 24.5 * np.log(2.0)
    _check(cache, q, _chunk(cache, q, t, scale=1.0), t, scale=1.0)


@pytest.mark.parametrize("kind", KINDS)
def test_growing_scores_move_the_reference(kind):
    """Scores that grow from tile to tile, by steps under and over what the reference tolerates, and that fall."""
    t = 1600
    for up in (1.0, -1.0):
        cache = Cache(kind, 1, 1, t, seed=14)
        ramp = np.zeros(t)
        ramp[:] = np.linspace(0, 100, t) + 3 * np.random.default_rng(1).standard_normal(t)
        cache.k[..., 0] = np.clip(np.rint(ramp), 0, 127).reshape(1, 1, -1, 64).astype(np.uint8) + 128 if kind == "int8" else cache.k[..., 0]
        if kind == "e4m3":
            from q8_util import code_of
            cache.k[..., 0] = code_of(kind, ramp).reshape(1, 1, -1, 64)
        cache.s[0][...] = 1.0
        cache.upload()
        for m in (1, 140):
            q = randn((1, m, 4, D), 2, 0.02)
            q[..., 0] = up
            _check(cache, q, _chunk(cache, q, t, scale=1.0), t, scale=1.0)


def test_blocks_whose_scales_are_far_apart():
    """Values of one block are 10^6 times those of another, which holds most of the weight."""
    for kind in KINDS:
        cache = Cache(kind, 2, 1, 512, seed=15)
        for s in cache.s:
            s[...] = np.exp2(np.rint(np.log2(s)))
        cache.s[1][0, :, 1::2] *= 2.0 ** -20
        cache.s[0][0, :, 3] = 0.0
        cache.upload()
        for m in (1, 150):
            q = randn((1, m, 8, D), 4, 3.0)
            _check(cache, q, _chunk(cache, q, 500), 500)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("m", [1, 200, 600])
@pytest.mark.parametrize("at", [0, 20])
def test_small_weights_beside_a_block_of_large_values_without_weight(kind, m, at):
    """A block whose values are 2^13 times the others' and whose weights are nothing; of the others one token outweighs each by 2^16.3, and
    the value of the many alone is not zero in channel 1."""
    t = 4096
    cache = Cache(kind, 1, 1, t, seed=17, fill=128 if kind == "int8" else 0)
    one, less = (129, 1) if kind == "int8" else (0x38, 0xf8)    # 1 and -127, 1 and -256
    for s in cache.s:
        s[...] = 1.0
    cache.k[0, 0, 30, 0, 0] = one
    cache.k[0, 0, at, :, 9] = less
    cache.v[0, 0, :, 1, :] = one
    cache.v[0, 0, 30, 1, 0] = 128 if kind == "int8" else 0
    q = torch.zeros(1, m, 1, D, dtype=torch.float16, device="cuda")
    q[..., 0] = 16.3 * np.log(2.0)
    q[..., 9] = 1.0
    want, tol = cache.attention(q, t, scale=1.0)             # (e^-127 of the weights: no scale of that block would be seen)
    cache.s[1][0, 0, at] = 2.0 ** 13
    cache.upload()
    for split in (0, t):                                     # (cut, few pieces meet the block)
        off = np.abs(_chunk(cache, q, t, scale=1.0, tokens_per_split=split).cpu().numpy().astype(np.float64) - want)
        assert (off <= tol).all(), (split, (off / tol).max())


@pytest.mark.parametrize("kind", KINDS)
def test_equal_calls_give_equal_bits_and_pages_are_no_matter(kind):
    a, b = (Cache(kind, 4, 5, 1024, seed=16, paged=x) for x in (False, True))
    lens = [1000, 1, 500, 64, 999]
    for m in (1, 9, 200):
        q = randn((5, m, 16, D), m)
        want = _chunk(a, q, 1000, lens)
        assert torch.equal(_chunk(a, q, 1000, lens), want)
        assert torch.equal(_chunk(b, q, 1000, lens), want)


def test_seeded_combinations():
    rng = np.random.default_rng(7)
    for i in range(60):
        kind = KINDS[i % 2]
        hkv, qper = int(rng.integers(1, 6)), int(rng.integers(1, 20))
        batch, t = int(rng.integers(1, 6)), int(np.exp(rng.uniform(0, 7.5)))
        m = int(min(t, np.exp(rng.uniform(0, 5.8)))) if i % 3 else 1
        cache = Cache(kind, hkv, batch, -(-t // 64) * 64, seed=i, paged=bool(rng.integers(2)))
        lens = [int(x) for x in rng.integers(0, t + 1, batch)] if rng.integers(2) else None
        q = randn((batch, m, hkv * qper, D), i, 1.5)
        split = int(rng.choice([0, 0, 64, 256]))
        _check(cache, q, _chunk(cache, q, t, lens, tokens_per_split=split), t, lens)
