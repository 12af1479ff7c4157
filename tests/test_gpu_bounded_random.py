"""Seeded random combinations of format, heads, lengths, windows, splits, ragged and paged caches, over the calls of bounded caches."""
import numpy as np
import pytest
import torch

import paper_2405_03917_amd as cq
from bounded_util import FORMATS, Cache, attention, queries, weight_tolerance
from gpu_util import check_attention

pytestmark = pytest.mark.gpu


def _draw(seed):
    rng = np.random.default_rng(1000 + seed)
    pick = lambda *x: x[rng.integers(len(x))]  # noqa: E731
    c, b = FORMATS[seed % len(FORMATS)]
    hkv = int(pick(1, 2, 3, 4, 8))
    qper = int(pick(1, 1, 2, 3, 4, 5, 8))
    t = int(np.exp(rng.uniform(0, np.log(6000)))) + 1
    batch = int(pick(1, 2, 3, 7, 20)) if t < 1500 else int(pick(1, 2))
    m = min(t, int(pick(1, 1, 2, 3, 5, 8, 17, 33, 64, 130)))
    cap = -(-t // 64) * 64 + 64 * int(pick(0, 0, 1, 3))
    lens = None if rng.random() < 0.3 else [t] + [int(x) for x in rng.integers(m, t + 1, batch - 1)]
    return dict(c=c, b=b, hkv=hkv, hq=hkv * qper, t=t, batch=batch, m=m, cap=cap, lens=lens, paged=bool(rng.random() < 0.5),
                window=int(np.exp(rng.uniform(0, np.log(t + 64)))), n_sink=int(pick(0, 1, 4, 63, 64, 65, 200)), split=64 * int(pick(0, 0, 0, 1, 2, 5)),
                decay=float(pick(0.0, 0.5, 1.0)), scale=float(pick(0.02, 128 ** -0.5, -0.05)))


def _within(got, before, sums, largest, rows, decay, lens):
    got, before = got.double().cpu(), before.double().cpu()
    for n, length in enumerate(lens):
        kept = decay * before[n, :, :length] if decay else torch.zeros_like(before[n, :, :length])
        want = kept + sums[n, :, :length]
        # (the weights' own bound; an accumulator is rounded for its decay and once for every 256 rows)
        room = weight_tolerance(largest, rows) * sums[n, :, :length] + (2 + rows // 256) * 2.0 ** -24 * (kept.abs() + want.abs()) + 2.0 ** -126
        assert ((got[n, :, :length] - want).abs() <= room).all()
        assert torch.equal(got[n, :, length:], before[n, :, length:])


@pytest.mark.parametrize("seed", range(64))
def test_random(seed):
    d = _draw(seed)
    print(d, flush=True)
    cache = Cache(d["c"], d["b"], d["hkv"], d["batch"], d["cap"], seed=seed)
    t, lens, scale, paged = d["t"], d["lens"] or [d["t"]] * d["batch"], d["scale"], d["paged"]
    sl = None if d["lens"] is None else torch.tensor(d["lens"], dtype=torch.int32, device="cuda")
    books = (cache.ck, cache.cv, scale, cache.fmt, t)
    at = (cache.pages(),) if paged else (cache.t_cap,)
    k, v = cache.pools if paged else (cache.k, cache.v)
    call = lambda name: getattr(cq, name + ("_paged" if paged else ""))  # noqa: E731

    q = queries((d["batch"], d["m"], d["hq"], 128), seed)
    last = q[:, -1].contiguous()
    ref, _, _ = attention(cache, q, lens, d["window"], d["n_sink"], scale)
    out = call("cq_chunk_attention_window")(q, k, v, *books, *at, d["window"], d["n_sink"], sl, d["split"])
    check_attention(out.cpu().numpy(), ref.numpy())
    out = call("cq_decode_attention_window")(last, k, v, *books, *at, d["window"], d["n_sink"], sl, d["split"])
    check_attention(out.cpu().numpy(), ref[:, -1].numpy())

    start = torch.rand(d["batch"], d["hkv"], t + seed % 3, device="cuda")
    ref, sums, largest = attention(cache, last[:, None], lens, scale=scale)
    got = start.clone()
    out = call("cq_decode_attention_weights")(last, k, v, *books, *at, got, d["decay"], sl, d["split"])
    check_attention(out.cpu().numpy(), ref[:, 0].numpy())
    _within(got, start, sums, largest, d["hq"] // d["hkv"], d["decay"], lens)

    _, sums, largest = attention(cache, q, lens, scale=scale)
    got = start.clone()
    call("cq_chunk_weights")(q, k, cache.ck, scale, cache.fmt, t, *at, got, d["decay"], sl)
    _within(got, start, sums, largest, d["m"] * d["hq"] // d["hkv"], d["decay"], lens)

    # what stays by these weights, moved: attention over it is attention over those tokens, whatever their places
    keep = max(1, t // 3)
    kept, new = cq.cq_select_tokens(got, t, keep, min(4, keep), 0, sl)
    codes = [x[..., :].copy() for x in cache.codes]
    keep_cap = -(-keep // 64) * 64
    small = [cq.alloc_cache(cache.fmt, d["batch"], keep_cap) for _ in range(2)]
    if paged:
        table = torch.arange(d["batch"] * keep_cap // 64, dtype=torch.int32, device="cuda").flip(0).reshape(d["batch"], -1).contiguous()
        to = cq.PageTable(table, table.numel())
        cq.cq_compact_cache_paged(k, v, None, cache.fmt, kept, new, t, *at, *small, None, to)
        out = cq.cq_decode_attention_paged(last, *small, *books[:4], keep, to, new)
    else:
        cq.cq_compact_cache(k, v, None, cache.fmt, kept, new, t, *at, *small, None, keep_cap)
        out = cq.cq_decode_attention(last, *small, *books[:4], keep, keep_cap, new)
    gh = 128 // d["c"]
    moved = Cache.__new__(Cache)
    moved.__dict__.update(cache.__dict__, t_cap=keep_cap)
    moved.codes = [np.zeros((d["batch"], keep_cap, x.shape[2]), dtype=x.dtype) for x in codes]
    where, count = kept.cpu().numpy(), new.cpu().numpy()
    for n in range(d["batch"]):
        for h in range(d["hkv"]):
            for which in (0, 1):
                moved.codes[which][n, :count[n], h * gh:(h + 1) * gh] = codes[which][n, where[n, h, :count[n]], h * gh:(h + 1) * gh]
    ref, _, _ = attention(moved, last[:, None], [int(x) for x in count], scale=scale)
    check_attention(out.cpu().numpy(), ref[:, 0].numpy())
