"""Calls that are handed a stream: whatever they allocate comes from that stream's pool (memory of another stream's pool may still be in
use there, and is given out again there while the call's kernels write it)."""
import pytest
import torch

import paper_2505_05950_amd as F
from paper_2505_05950_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")


def pool_of(t):
    """The stream that the caching allocator keeps a tensor's memory for."""
    for seg in torch.cuda.memory_snapshot():
        if seg["address"] <= t.data_ptr() < seg["address"] + seg["total_size"]:
            return seg["stream"]
    raise AssertionError("not the allocator's")


@pytest.fixture
def s():
    stream = torch.cuda.Stream()
    yield stream
    torch.cuda.synchronize()


@pytest.fixture
def spaces(monkeypatch):
    """Every workspace that is made."""
    made, make = [], B._workspace
    monkeypatch.setattr(B, "_workspace", lambda *a, **k: made.append(make(*a, **k)) or made[-1])
    return made


def all_of(s, *tensors):
    torch.cuda.synchronize()
    pools = [pool_of(t) for t in tensors]
    assert pools == [s.cuda_stream] * len(tensors), (pools, s.cuda_stream)


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def test_the_caches_calls(s, spaces):
    cache = F.KVCache(80, 2, 64, 32, device=DEV)
    n = 2000
    x = torch.randn((n, 2, 64), device=DEV).half()
    table, cu, before, after = i32([list(range(80))]), i32([0, n]), i32([0]), i32([n])
    torch.cuda.synchronize()
    table_of_angles = F.floe_rope_table(n, 64, device=DEV, stream=s)
    q = F.floe_kv_append(cache, x, x, cu, before, table, n, q=x, rope=F.Rope(table_of_angles), stream=s)
    k, v = F.floe_kv_gather(cache, before, cu, table, n, n, stream=s)
    one = q[-1:].contiguous()
    torch.cuda.synchronize()
    out, lse = F.floe_kv_attention(cache, one, i32([0, 1]), after, table, 1, n, want_lse=True, stream=s)  # one row of many chunks: a large workspace
    assert len(spaces) == 2
    all_of(s, table_of_angles, q, k, v, out, lse, *spaces)


def test_the_experts_calls(s, spaces):
    d, f, T = 512, 256, 3
    w, gd = torch.randn((f, d), device=DEV).half() * 0.05, torch.randn((f, 2, d), device=DEV).half() * 0.05
    x, tau, y = torch.randn((T, d), device=DEV).half(), torch.full((1,), 0.5, device=DEV), torch.zeros((T, d), device=DEV)
    weights = torch.ones(T, device=DEV)
    torch.cuda.synchronize()
    codes, scale, zero = F.floe_quantize_expert(w, 2, 64, stream=s)
    v = F.floe_up_gemv(codes, scale, zero, x, d, 2, 64, stream=s)
    idx, count = F.floe_select_channels(v, tau, stream=s)
    e = F.Expert(d, f, 2, 64, codes, scale, zero, gd)
    F.floe_gate_down_sparse(e, x, v, idx, count, weights, y, stream=s)
    _, idx2, count2 = F.floe_expert_ffn_sparse(e, x, tau, weights, y, stream=s)
    _, idx3, count3 = F.floe_expert_ffn_sparsified(e, F.SPARSIFY_GATE, x, tau, weights, y, stream=s)
    assert len(spaces) == 3
    all_of(s, codes, scale, zero, v, idx, count, idx2, count2, idx3, count3, *spaces)
    for i, c in ((idx, count), (idx2, count2), (idx3, count3)):  # lists end in -1
        behind = torch.arange(f, device=DEV)[None] >= c[:, None]
        assert bool(((i == -1) == behind).all())


def test_the_layers_calls(s, spaces):
    d, f, T = 512, 256, 3
    w, gd = torch.randn((f, d), device=DEV).half() * 0.05, torch.randn((f, 2, d), device=DEV).half() * 0.05
    experts = [F.Expert(d, f, 2, 64, *F.floe_quantize_expert(w, 2, 64), gd) for _ in range(2)]
    router, tau, x = torch.randn((2, d), device=DEV).half(), torch.full((2,), 0.5, device=DEV), torch.randn((T, d), device=DEV).half()
    torch.cuda.synchronize()
    layer = F.Layer(experts, 0, 1, True, router, tau, False, stream=s)
    y = F.floe_moe_layer_decode(layer, x, stream=s)
    assert len(spaces) == 1
    all_of(s, layer.table, y, *spaces)
    assert torch.equal(y, F.floe_moe_layer_decode(layer, x))
