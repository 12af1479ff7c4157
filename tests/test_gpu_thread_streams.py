"""hipStreamPerThread, a handle that is another stream in every host thread: calls of two threads at once, each cut into pieces that are
joined, give bit for bit what they give alone on the default stream."""
import math
import threading

import numpy as np
import pytest
import torch

import paper_2405_03917_amd as cq
import synth

from gpu_util import codes_to_cache, dev

pytestmark = pytest.mark.gpu
SCALE = 1.0 / math.sqrt(128)


class _PerThread:
    cuda_stream = 2                                          # hipStreamPerThread


def _coded(kind, seed):
    c, batch, hq, hkv, t, cap = 8, 2, 8, 8, 3000 + 64 * seed, 4096
    fmt = cq.CQFormat(c, 8, 128, hkv)
    rng = np.random.default_rng(seed)
    ck, cv = (dev(synth.sample_codebook(synth.tensor_recipe(1, seed, x, fmt.channels), c, 8)) for x in "kv")
    k, v = (codes_to_cache(rng.integers(0, 256, size=(batch, t, fmt.groups)).astype(np.uint16), fmt, cap) for _ in range(2))
    q = dev(rng.standard_normal((batch, hq, 128)).astype(np.float16))
    if kind == "decode":
        return cq.prepare_decode_attention(q, k, v, ck, cv, SCALE, fmt, t, cap, tokens_per_split=512)
    return cq.prepare_decode_attention_window(q, k, v, ck, cv, SCALE, fmt, t, cap, 2000, 4, tokens_per_split=512)


def _q8(seed):
    fmt, t = cq.Q8Format("int8", 128, 8), 2000 + 64 * seed
    cache = cq.alloc_q8_cache(fmt, 1, 4096)
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(2, 1, t, 8 * 128, generator=g, device="cuda").half()
    cq.cq_append_q8(x[0], x[1], cache, fmt, t, 4096)
    return cq.prepare_decode_attention_q8(x[0, :, -1].view(1, 8, 128).contiguous(), cache, SCALE, fmt, t, 4096)


@pytest.mark.parametrize("kind", ["decode", "window", "q8"])
def test_two_threads(kind):
    calls = [_q8(i) if kind == "q8" else _coded(kind, i) for i in range(2)]
    want = []
    for call, out in calls:
        call()
        torch.cuda.synchronize()
        want.append(out.clone())
    for _ in range(5):
        for _, out in calls:
            out.zero_()
        torch.cuda.synchronize()
        failed, ready = [], threading.Barrier(2)

        def work(call):
            try:
                ready.wait(timeout=30)
                for _ in range(40):
                    call(_PerThread)
            except Exception as e:  # noqa: BLE001
                failed.append(e)

        threads = [threading.Thread(target=work, args=(call,)) for call, _ in calls]
        for x in threads:
            x.start()
        for x in threads:
            x.join(timeout=60)
        torch.cuda.synchronize()
        assert not failed and not any(x.is_alive() for x in threads)
        for (_, out), w in zip(calls, want):
            assert torch.equal(out, w)
