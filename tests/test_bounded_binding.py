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
