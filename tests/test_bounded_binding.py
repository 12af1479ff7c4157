"""The binding of the calls that keep a cache bounded: what it prepares, without a GPU (its checks for device tensors are stood
in for; nothing is launched)."""
import pytest
import torch

import paper_2405_03917_amd as cq

FMT = cq.CQFormat(8, 8, 128, 4)


@pytest.fixture
def on_host(monkeypatch):
    monkeypatch.setattr(cq, "_dev", lambda t, dtype, what: t)
    monkeypatch.setattr(cq, "_same_device", lambda *tensors: None)


def _cache(tokens):
    return torch.zeros(cq.cq_cache_bytes(FMT, 2, tokens), dtype=torch.uint8)


@pytest.mark.parametrize("same", ["k", "v", "weights", "none"])
def test_an_output_that_is_its_input_under_another_tensor_has_a_workspace(on_host, same):
    k, v, w = _cache(512), _cache(512), torch.zeros(2, 4, 512)
    k2, v2, w2 = _cache(512), _cache(512), torch.zeros(2, 4, 512)
    k2, v2, w2 = (k.view(-1) if same == "k" else k2), (v.view(-1) if same == "v" else v2), (w.view(2, 4, 512) if same == "weights" else w2)
    kept, lens = torch.zeros(2, 4, 100, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    call = cq.prepare_compact_cache(k, v, w, FMT, kept, lens, 300, 512, k2, v2, w2)
    workspace, size = call._args[-2:]
    if same == "none":
        assert workspace is None and size == 0
    else:
        assert workspace and size == cq.cq_compact_workspace_bytes(FMT, 2, 100)


# ---------------------------------------------------------------- calls on another stream

class _Lib:
    """The library with its launches left out."""

    def __init__(self, real):
        self.real, self.launched, self.on = real, [], []

    def __getattr__(self, name):
        if name.endswith(("_bytes", "_split", "_check", "_format", "_string")):
            return getattr(self.real, name)

        def launch(*args):
            self.launched.append(name)
            self.on.append(args[-1])
            return cq.CQ_OK
        return launch


class _Stream:
    def __init__(self, cuda_stream=7):
        self.cuda_stream = cuda_stream


@pytest.fixture
def streams(on_host, monkeypatch):
    """(side stream, record of (address, stream) pairs, the library, what was the current stream at each allocation)."""
    current, records, lib = [_Stream()], set(), _Lib(cq.load())

    class Switch:
        def __init__(self, stream):
            self.stream = stream

        def __enter__(self):
            current.append(self.stream)

        def __exit__(self, *exc):
            current.pop()

    empty, allocated = torch.empty, []
    monkeypatch.setattr(cq, "load", lambda: lib)
    monkeypatch.setattr(torch.cuda, "Stream", _Stream)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: current[-1])
    monkeypatch.setattr(torch.cuda, "stream", Switch)
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda self, stream: records.add((self.data_ptr(), stream)))

    def allocate(*args, **kwargs):
        kwargs.pop("device", None)
        allocated.append(current[-1])
        return empty(*args, **kwargs)

    monkeypatch.setattr(torch, "empty", allocate)
    return _Stream(), current[0], records, lib, allocated


def _operands():
    half, i32 = torch.float16, torch.int32
    fmt = FMT
    x = dict(q=torch.zeros(2, 8, 128, dtype=half), rows=torch.zeros(2, 3, 8, 128, dtype=half), k=_cache(512), v=_cache(512),
             ck=torch.zeros(fmt.groups, 256, 8, dtype=half), cv=torch.zeros(fmt.groups, 256, 8, dtype=half), new=torch.zeros(2, fmt.channels, dtype=half),
             new_v=torch.zeros(2, fmt.channels, dtype=half), x=torch.zeros(2, 5, fmt.channels, dtype=half), x_v=torch.zeros(2, 5, fmt.channels, dtype=half),
             w=torch.zeros(2, 4, 512), lens=torch.full((2,), 300, dtype=i32), kept=torch.zeros(2, 4, 100, dtype=i32), new_lens=torch.zeros(2, dtype=i32),
             table=torch.zeros(2, 8, dtype=i32), rnd=torch.zeros(fmt.groups, 256, dtype=torch.int64))
    x["pages"] = cq.PageTable(x["table"], 16)
    return x


CALLS = {
    "window": (lambda o, s: cq.cq_decode_attention_window(o["q"], o["k"], o["v"], o["ck"], o["cv"], 0.1, FMT, 300, 512, 64, 4, o["lens"], stream=s),
               ("q", "k", "v", "ck", "cv", "lens")),
    "window_step_paged": (lambda o, s: cq.cq_decode_step_window_paged(o["q"], o["new"], o["new_v"], o["k"], o["v"], o["ck"], o["cv"], 0.1, FMT, 300,
                                                                      o["pages"], 64, stream=s), ("q", "new", "new_v", "k", "v", "ck", "cv", "table")),
    "chunk_window": (lambda o, s: cq.cq_chunk_attention_window(o["rows"], o["k"], o["v"], o["ck"], o["cv"], 0.1, FMT, 300, 512, 64, 4, stream=s),
                     ("rows", "k", "v", "ck", "cv")),
    "weights": (lambda o, s: cq.cq_decode_attention_weights(o["q"], o["k"], o["v"], o["ck"], o["cv"], 0.1, FMT, 300, 512, o["w"], stream=s),
                ("q", "k", "v", "ck", "cv", "w")),
    "chunk_weights": (lambda o, s: cq.cq_chunk_weights(o["rows"], o["k"], o["ck"], 0.1, FMT, 300, 512, o["w"], stream=s), ("rows", "k", "ck", "w")),
    "select": (lambda o, s: cq.cq_select_tokens(o["w"], 300, 100, seq_lens=o["lens"], stream=s), ("w", "lens")),
    "compact": (lambda o, s: cq.cq_compact_cache(o["k"], o["v"], o["w"], FMT, o["kept"], o["new_lens"], 300, 512, stream=s), ("k", "v", "w", "kept", "new_lens")),
    "encode": (lambda o, s: cq.cq_encode(o["x"], o["ck"], FMT, o["k"], 0, 512, s), ("x", "ck", "k")),
    "encode_kv_paged": (lambda o, s: cq.cq_encode_kv_paged(o["x"], o["x_v"], o["ck"], o["cv"], FMT, o["k"], o["v"], o["pages"], 0, s),
                        ("x", "x_v", "ck", "cv", "k", "v", "table")),
    "decode": (lambda o, s: cq.cq_decode_attention(o["q"], o["k"], o["v"], o["ck"], o["cv"], 0.1, FMT, 300, 512, o["lens"], stream=s),
               ("q", "k", "v", "ck", "cv", "lens")),
    "step_paged": (lambda o, s: cq.cq_decode_step_paged(o["q"], o["new"], o["new_v"], o["k"], o["v"], o["ck"], o["cv"], 0.1, FMT, 300, o["pages"], stream=s),
                   ("q", "new", "new_v", "k", "v", "ck", "cv", "table")),
    "chunk": (lambda o, s: cq.cq_chunk_attention(o["rows"], o["k"], o["v"], o["ck"], o["cv"], 0.1, FMT, 300, 512, stream=s), ("rows", "k", "v", "ck", "cv")),
    "dequantize": (lambda o, s: cq.cq_dequantize(o["k"], o["ck"], FMT, 2, 0, 10, 512, stream=s), ("k", "ck")),
    "kmeans": (lambda o, s: cq.cq_kmeans_fit(o["new"], FMT, 1, rnd=o["rnd"], stream=s), ("new", "rnd")),
    "rope_table": (lambda o, s: cq.RopeTable(1e4, 512, device="cpu", stream=s), ()),
}


@pytest.mark.parametrize("name", CALLS)
def test_a_call_on_another_stream_keeps_what_it_uses(streams, name):
    side, user, records, lib, allocated = streams
    call, used = CALLS[name]
    operands = _operands()
    result = call(operands, side)
    assert lib.launched
    for x in used:
        assert (operands[x].data_ptr(), side) in records, x
    assert all(s is side for s in allocated)                # from that stream's pool
    for x in cq._tensors(result):
        assert (x.data_ptr(), user) in records
    records.clear()
    call(operands, None)                                    # on the current stream: nothing to record
    assert not records


def test_a_stream_of_another_library(streams):
    class Theirs:
        cuda_stream = 11

    _, _, records, lib, _ = streams
    operands = _operands()
    cq.cq_decode_attention(operands["q"], operands["k"], operands["v"], operands["ck"], operands["cv"], 0.1, FMT, 300, 512, stream=Theirs())
    assert lib.launched and lib.on == [11]
    assert not records                                      # it may be gone when they are freed
