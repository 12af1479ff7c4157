"""cq_dequantize_q8's two outputs as parts of one buffer: refused where rows meet, and only there."""
import random

import pytest
import torch

import paper_2405_03917_amd as cq
from test_q8_host import BASE, dequantize, fmt_of

E = cq.CQ_ERR_INVALID_ARG
W = 4 * 128                                                  # a row of four KV heads


def _meet(batch, m, batch_stride, row_stride, apart):
    """Whether a row of one output and a row of the other, `apart` elements on, share an element."""
    rows = [n * batch_stride + j * row_stride for n in range(batch) for j in range(m)]
    return any(abs(a - b - apart) < W for a in rows for b in rows)


def _cases():
    yield 2, 5, 5 * W, W, 0                                  # (what is refused, first)
    yield 2, 5, 5 * W, W, 5 * W                              # behind the first sequence's rows, where the second's begin
    yield 2, 5, 10 * W, W, 5 * W - 8
    yield 2, 5, 10 * W, W, 5 * W                             # [batch][2][m]
    yield 2, 5, 10 * W, W, -5 * W
    yield 2, 5, 10 * W, 2 * W, W                             # [batch][m][2]
    yield 2, 5, 10 * W, W, 15 * W                            # (one output ends inside the other's gap)
    yield 1, 5, 0, W, 5 * W
    yield 1, 5, 0, 3 * W, W + 8
    yield 3, 1, 2 * W, W, W
    yield 3, 1, 2 * W, W, W - 8
    rng = random.Random(3)
    for _ in range(300):
        batch, m = rng.randint(1, 4), rng.randint(1, 5)
        row = W + 8 * rng.randint(0, 96)
        stride = m * row + 8 * rng.randint(0, 3 * m * row // 8)
        yield batch, m, stride, row, 8 * rng.randint(-batch * stride // 8, batch * stride // 8)


@pytest.mark.skipif(torch.cuda.device_count() > 0, reason="addresses of nothing: an accepted call must not find a GPU")
def test_refused_where_rows_meet():
    met = []
    for batch, m, batch_stride, row_stride, apart in _cases():
        st = dequantize(fmt=fmt_of(hkv=4), batch=batch, m=m, o_batch=batch_stride, o_row=row_stride, vo=BASE["ko"] + 2 * apart, t=300,
                        k=1 << 40, v=1 << 41, ks=1 << 42, vs=1 << 43)
        met.append(_meet(batch, m, batch_stride, row_stride, apart))
        assert (st == E) == met[-1], (batch, m, batch_stride, row_stride, apart, st)
        assert met[-1] or st == cq.CQ_ERR_HIP                # (all checks passed; no GPU to launch on)
    assert 50 < sum(met) < len(met) - 50


@pytest.mark.gpu
@pytest.mark.parametrize("m", [1, 70])
@pytest.mark.parametrize("layout", ["batch, 2, m", "batch, m, 2", "2, batch, m"])
def test_both_outputs_in_one_buffer(layout, m):
    from q8_util import D, Cache
    cache = Cache("int8", 2, 3, 128, seed=4)
    want = cq.cq_dequantize_q8(cache.dev, cache.fmt, 3, m, 100, 128)
    at = layout.split(", ").index("2")
    shape = [3, m]
    buf = torch.full(shape[:at] + [2] + shape[at:] + [2 * D], 5.0, dtype=torch.float16, device="cuda")
    for k, v in (buf.unbind(at), buf.unbind(at)[::-1]):
        cq.cq_dequantize_q8(cache.dev, cache.fmt, 3, m, 100, 128, k_out=k, v_out=v)
        assert torch.equal(k, want[0]) and torch.equal(v, want[1])
