"""cq_append_q8 and cq_dequantize_q8 against the definition in 64 bits: codes, scales and rows bit for bit."""
import numpy as np
import pytest
import torch

import paper_2405_03917_amd as cq
from q8_util import D, KINDS, TILE, Cache, E4M3, code_of, need, randn, rotated, values_of

pytestmark = pytest.mark.gpu
BASE = 10000.0


def _same(cache):
    """The device arrays against the object's; every byte, so what must not change has not."""
    k, v, ks, vs = cache.download()
    assert np.array_equal(ks.view(np.uint32), cache.s[0].view(np.uint32)) and np.array_equal(vs.view(np.uint32), cache.s[1].view(np.uint32))
    assert np.array_equal(k, cache.k), np.argwhere(k != cache.k)[:5]
    assert np.array_equal(v, cache.v), np.argwhere(v != cache.v)[:5]
    assert cache.unused_pages_are_untouched()


def _append(cache, x_k, x_v, t, lens=None, rope=None, **more):
    call, q_out = cq.prepare_append_q8(x_k, x_v, cache.dev, cache.fmt, t, rope=rope, **cache.where(lens), **more)
    call()
    cache.append(x_k.cpu().numpy(), x_v.cpu().numpy(), t, lens, None if rope is None else rope.base)
    return q_out


def _rows(batch, m, hkv, seed, big=1.0):
    """Keys and values side by side in rows of one projection, some channels larger."""
    x = randn((batch, m, 2 * hkv * D + 24), seed)
    x[..., 5] *= 9 * big
    x[..., hkv * D + 70] *= 5 * big
    return x[..., :hkv * D], x[..., hkv * D + 16:2 * hkv * D + 16]


# new tokens that begin and end at borders of blocks and off them, of one token and of several blocks; contexts from nothing
SIZES = [(1, 1), (1, 64), (1, 65), (2, 130), (63, 63), (64, 64), (64, 100), (65, 65), (65, 129), (66, 129), (130, 191), (200, 333), (320, 320)]


@pytest.mark.parametrize("rope", [False, True])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("m,t", SIZES)
def test_append_sizes(kind, m, t, rope):
    cache = Cache(kind, 3, 2, 320 + TILE, seed=m + t, paged=bool(t % 2))
    table = cq.Q8RopeTable(BASE, 384) if rope else None
    _append(cache, *_rows(2, m, 3, t), t, rope=table)
    _same(cache)


@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("kind", KINDS)
def test_ragged_lengths_and_padding(kind, paged):
    lens = [0, 1, 5, 63, 64, 65, 128, 129, 200, 199, -7, 1000]
    for m in (1, 6, 70):
        cache = Cache(kind, 2, len(lens), 256, seed=m, paged=paged)
        rope = cq.Q8RopeTable(BASE, 256)
        x_k, x_v = _rows(len(lens), m, 2, m)
        for n, length in enumerate(lens):                    # padding rows are not read
            pad = max(0, m - max(length, 0))
            x_k[n, :pad] = x_v[n, :pad] = float("nan")
        q = randn((len(lens), m, 4, D), 9)
        q_out = torch.full_like(q, 7.0)
        _append(cache, x_k, x_v, 200, lens, rope, q=q, q_out=q_out)
        _same(cache)
        for n, length in enumerate(lens):
            t_n = min(max(length, 0), 200)
            pad = max(0, m - t_n)
            assert (q_out[n, :pad] == 7).all()
            _check_queries(q_out[n, pad:], q[n, pad:], np.arange(t_n - m + pad, t_n))


def _check_queries(got, q, pos):
    want = rotated(q.cpu().numpy().astype(np.float64), np.asarray(pos)[:, None], BASE)
    # a rounding to fp16, and in fp32 two products, a sum and two roundings of the table
    x = np.abs(q.cpu().numpy().astype(np.float64))
    off = np.abs(got.cpu().numpy().astype(np.float64) - want)
    size = np.concatenate([x[..., :64] + x[..., 64:]] * 2, -1)
    assert (off <= 2.0 ** -11 * np.abs(want) + 2.0 ** -25 + 4 * 2.0 ** -24 * size).all()


@pytest.mark.parametrize("kind", KINDS)
def test_token_by_token_scales_grow(kind):
    cache = Cache(kind, 2, 3, 192, seed=4, fill=0x7f)        # (bytes and scales that mean nothing, e4m3's no-number among them)
    rope = cq.Q8RopeTable(BASE, 192)
    rng = np.random.default_rng(0)
    for t in range(1, 140):
        big = float(np.exp(rng.normal()))
        _append(cache, *_rows(3, 1, 2, t, big), t, rope=rope)
    _same(cache)


@pytest.mark.parametrize("kind", KINDS)
def test_cut_back_and_written_again(kind):
    cache = Cache(kind, 2, 2, 256, seed=8, paged=True)
    for m, t in ((100, 100), (7, 104), (30, 64), (80, 144), (2, 66), (1, 65), (70, 200)):
        _append(cache, *_rows(2, m, 2, t + m, 1 + t / 50), t)
    _same(cache)


@pytest.mark.parametrize("kind", KINDS)
def test_zeros_smallest_and_largest_numbers(kind):
    cache = Cache(kind, 4, 1, 128, seed=1)
    x = torch.zeros(1, 128, 4 * D, dtype=torch.float16, device="cuda")
    x[0, :64, D + 3] = 2.0 ** -24
    x[0, :, 2 * D:3 * D] = 65504.0 * torch.sign(randn((128, D), 3).float()).half()
    x[0, :, 3 * D:] = randn((128, D), 5)
    x[0, 64:, 3 * D + 1] = torch.exp2(torch.arange(64, device="cuda").float() / 3 - 12).half()
    _append(cache, x, x.flip(1).contiguous(), 128, rope=cq.Q8RopeTable(BASE, 128))
    _same(cache)
    # zero blocks grow from a scale of zero
    zero = Cache(kind, 1, 1, 64, seed=2)
    _append(zero, *(torch.zeros(1, 10, D, dtype=torch.float16, device="cuda") for _ in range(2)), 10)
    assert zero.s[0].item() == 0
    _append(zero, randn((1, 5, D), 3), randn((1, 5, D), 4), 15)
    _same(zero)


@pytest.mark.parametrize("kind", KINDS)
def test_numbers_at_the_borders_between_codes(kind):
    """Ties go to the even code.  Blocks whose largest number makes the scale a power of two, and every half step in them."""
    top = 127.0 if kind == "int8" else 448.0
    grid = np.arange(-127, 128) / 1.0 if kind == "int8" else np.concatenate([-E4M3[:127][::-1], E4M3[:127]])
    mid = (grid[1:] + grid[:-1]) / 2
    x = np.zeros((64, D))
    x.reshape(-1)[:mid.size] = mid
    x.reshape(-1)[mid.size:mid.size + grid.size] = grid
    x[63, 127] = top
    x = torch.from_numpy(x).half().cuda().view(1, 64, D)
    cache = Cache(kind, 1, 1, 64, seed=1)
    _append(cache, x, -x, 64)
    assert cache.s[0].item() == 1.0
    _same(cache)


@pytest.mark.parametrize("step", [1, 64])
@pytest.mark.parametrize("scale", [3.0, 5.0, 7.0 / 64])
def test_ties_under_scales_with_inexact_reciprocals(scale, step):
    """Integers: every code and every half step, exact in fp16, as single tokens and as a tile."""
    half_steps = np.arange(-253, 254) * scale / 2
    x = np.zeros((64, D))
    x.reshape(-1)[2 * D:2 * D + half_steps.size] = half_steps
    x[0, 127] = 127 * scale                                  # the scale from the first token on
    assert np.array_equal(x, x.astype(np.float16))
    x = torch.from_numpy(x).half().cuda().view(1, 64, D)
    cache = Cache("int8", 1, 1, 64, seed=1)
    for u in range(0, 64, step):
        _append(cache, x[:, u:u + step], -x[:, u:u + step], u + step)
    assert cache.s[0].item() == scale
    want = np.rint(half_steps / scale).astype(np.int64) + 128
    assert np.array_equal(cache.k.reshape(-1)[2 * D:2 * D + want.size], want)
    _same(cache)


@pytest.mark.parametrize("kind", KINDS)
def test_far_positions(kind):
    """Angles of positions near 2^20: the table's last blocks."""
    t = (1 << 20) - 3
    n_pages = 4
    fmt = cq.Q8Format(kind, D, 1)
    pools = cq.alloc_q8_pools(fmt, n_pages)
    pools.k_scales.zero_(), pools.v_scales.zero_()           # (the first block holds older tokens, whose scale counts)
    table = torch.zeros(1, 1 << 14, dtype=torch.int32, device="cuda")
    table[0, -2:] = torch.tensor([2, 1], dtype=torch.int32)
    pages = cq.PageTable(table, n_pages)
    x_k, x_v = randn((1, 70, D), 1), randn((1, 70, D), 2)
    q = randn((1, 70, 2, D), 3)
    rope = cq.Q8RopeTable(500000.0, 1 << 20)
    q_out = cq.cq_append_q8_paged(x_k, x_v, pools, fmt, t, pages, rope=rope, q=q)
    pos = np.arange(t - 70, t)
    want = rotated(x_k[0].cpu().numpy().astype(np.float64), pos, 500000.0)
    k = pools.k.view(n_pages, TILE, D).cpu().numpy()
    first = (1 << 20) - 128
    lo = t - 70 - first
    for page, rows in ((2, range(lo, 64)), (1, range(0, 61))):
        part = want[[first + (0 if page == 2 else 64) + u - (t - 70) for u in rows]]
        s = need(kind, np.abs(part).max())
        assert pools.k_scales.cpu().numpy()[page] == np.float32(s)
        # (angles of 2^20 in 64 bits are good to 2^-32: numbers that near to a border may go either way)
        got, ideal = values_of(kind, k[page, list(rows)]), part / s
        assert (np.abs(got - ideal) <= np.abs(values_of(kind, code_of(kind, ideal)) - ideal) + 1e-6 * np.abs(ideal) + 1e-9).all()
        assert (k[page, list(rows)] != code_of(kind, ideal)).mean() < 1e-3
    wantq = rotated(q[0].cpu().numpy().astype(np.float64), pos[:, None], 500000.0)
    assert np.abs(q_out[0].cpu().numpy() - wantq).max() <= 2.0 ** -11 * np.abs(wantq).max() + 2.0 ** -20


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("batch,m,t,hkv,hq", [(1, 1, 300, 32, 32), (40, 1, 500, 8, 64), (3, 700, 1000, 8, 24), (2, 1500, 1500, 16, 16), (5, 333, 700, 6, 42), (1, 9, 64, 1, 5)])
def test_queries_and_head_groups(kind, batch, m, t, hkv, hq):
    """Sizes at which a workgroup takes one head, several, and a thread several heads of queries; in place too."""
    cache = Cache(kind, hkv, batch, -(-t // 64) * 64, seed=t, paged=hkv == 8)
    rng = np.random.default_rng(t)
    lens = [t] + [int(x) for x in rng.integers(m, t + 1, batch - 1)]
    rope = cq.Q8RopeTable(BASE, cache.t_cap)
    x_k, x_v = _rows(batch, m, hkv, t)
    wide = randn((batch, m, hq * D + 40), 3)
    q = wide[..., 8:hq * D + 8].unflatten(-1, (hq, D))
    q_out = _append(cache, x_k, x_v, t, lens, rope, q=q)
    _same(cache)
    for n in {0, batch - 1}:
        _check_queries(q_out[n], q[n], np.arange(lens[n] - m, lens[n]))
    again = q.contiguous()
    call, out = cq.prepare_append_q8(x_k, x_v, cache.dev, cache.fmt, t, rope=rope, q=again, q_out=again, **cache.where(lens))
    call()
    assert out is again and torch.equal(again, q_out)
    _same(cache)                                             # (the same tokens once more: the same codes)


@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("m,t", [(1, 1), (1, 200), (63, 191), (64, 128), (65, 129), (130, 321), (321, 321)])
def test_dequantize(kind, m, t, paged):
    cache = Cache(kind, 3, 5, 384, seed=t, paged=paged)
    lens = [t, 0, max(1, t // 2), min(t, 64), 1]
    wide = torch.full((5, m, 2 * 3 * D + 16), 5.0, dtype=torch.float16, device="cuda")
    k_out, v_out = wide[..., :3 * D], wide[..., 3 * D + 8:6 * D + 8]
    call, *_ = cq.prepare_dequantize_q8(cache.dev, cache.fmt, 5, m, t, k_out, v_out, **cache.where(lens))
    call()
    for n, t_n in enumerate(lens):
        pad = max(0, m - t_n)
        for which, got in ((0, k_out), (1, v_out)):
            assert (got[n, :pad] == 5).all()
            for h in range(3):
                want = np.float32(values_of(kind, (cache.k if which == 0 else cache.v.swapaxes(-1, -2))[n, h])) * cache.s[which][n, h][:, None, None]
                want = want.reshape(-1, D)[max(0, t_n - m):t_n].astype(np.float16)
                assert np.array_equal(got[n, pad:, h * D:(h + 1) * D].cpu().numpy().view(np.uint16), want.view(np.uint16))
    assert (wide[..., 3 * D:3 * D + 8] == 5).all() and (wide[..., 6 * D + 8:] == 5).all()
    # one of the two alone
    for name, want in (("k_out", k_out), ("v_out", v_out)):
        one = torch.full((5, m, 3 * D), 5.0, dtype=torch.float16, device="cuda")
        call, *got = cq.prepare_dequantize_q8(cache.dev, cache.fmt, 5, m, t, **{name: one}, **cache.where(lens))
        call()
        assert torch.equal(one, want) and (got[0] is None) == (name == "v_out")


def test_one_shot_calls_on_both_kinds_of_cache():
    for paged in (False, True):
        cache = Cache("int8", 2, 2, 128, seed=3, paged=paged)
        x_k, x_v = _rows(2, 70, 2, 1)
        rope = cq.Q8RopeTable(BASE, 128)
        q = randn((2, 70, 4, D), 3)
        if paged:
            q_out = cq.cq_append_q8_paged(x_k, x_v, cache.dev, cache.fmt, 100, cache.pages(), rope=rope, q=q)
            k, v = cq.cq_dequantize_q8_paged(cache.dev, cache.fmt, 2, 70, 100, cache.pages())
        else:
            q_out = cq.cq_append_q8(x_k, x_v, cache.dev, cache.fmt, 100, 128, rope=rope, q=q)
            k, v = cq.cq_dequantize_q8(cache.dev, cache.fmt, 2, 70, 100, 128)
        cache.append(x_k.cpu().numpy(), x_v.cpu().numpy(), 100, None, BASE)
        _same(cache)
        _check_queries(q_out[1], q[1], np.arange(30, 100))
        for which, got in ((0, k), (1, v)):
            want = np.stack([cache.dense(which, 1, h, 100)[30:] for h in range(2)], 1).reshape(70, -1)
            assert np.abs(got[1].cpu().numpy() - want).max() <= 2.0 ** -11 * np.abs(want).max()
