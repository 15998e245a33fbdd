"""Attention with a window and first tokens that stay visible beside it, against the formula in 64 bits.  The tolerance is that of
test_gpu_kv_attention.py (`compare` of test_gpu_kv_limits.py): the kernels walk fewer tokens, the arithmetic is the same."""
import numpy as np
import pytest
import torch

import kv_reference as R
import paper_2505_05950_amd as F
from test_gpu_kv_attention import build
from test_gpu_kv_cache import DEV, cu_of, i32, to16
from test_gpu_kv_limits import blocks_of_size, compare

pytestmark = pytest.mark.gpu


def reference(q, k, v, there, length, causal, window, sinks, scale):
    n, H, D = q.shape
    out, size, lse = np.zeros((n, H, D)), np.zeros((n, H, D)), np.full((n, H), -np.inf)
    G, j = H // k.shape[1], np.arange(length)
    for i in range(n):
        pos = length - n + i
        see = j[there & (j <= pos if causal else j >= 0) & ((j > pos - window) | (j < sinks))]
        if not see.size:
            continue
        for h in range(H):
            s = (k[see, h // G] @ q[i, h]) * scale
            p = np.exp(s - s.max())
            out[i, h], size[i, h] = p @ v[see, h // G] / p.sum(), p @ np.abs(v[see, h // G]) / p.sum()
            lse[i, h] = s.max() + np.log(p.sum())
    return out, lse, size


def check(m, table, lens, n_q, qh, dtype, window, sinks, causal=True, max_len=None, scale=None, rng=None, fill=0x7f, cache=None):
    rng = rng or np.random.default_rng(0)
    D = m.D
    q = to16(rng.normal(0, 2.0, (sum(n_q), qh, D)).astype(np.float32), dtype)
    cache = m.device(dtype, DEV, fill) if cache is None else cache
    out, lse = F.floe_kv_attention(cache, q.to(DEV), cu_of(n_q), i32(list(lens)), i32(table), max(n_q), max(lens) if max_len is None else max_len,
                                   scale=scale, causal=causal, window=window, sinks=sinks, want_lse=True)
    torch.cuda.synchronize()
    at = 0
    for s, n in enumerate(n_q):
        k, there = m.value(0, lens[s], table[s])
        v, _ = m.value(1, lens[s], table[s])
        want, want_lse, size = reference(q[at:at + n].double().numpy(), k, v, there, lens[s], causal, window, sinks, D ** -0.5 if scale is None else scale)
        compare(out[at:at + n], lse[at:at + n], want, want_lse, size, dtype, s)
        at += n


def without_what_nobody_sees(table, lens, n_q, P, window, sinks):
    """The table without the pages that lie wholly between the first tokens and the first query's window."""
    out = [list(t) for t in table]
    for s, t in enumerate(out):
        first = lens[s] - n_q[s] - window + 1
        for b in range(len(t)):
            if b * P >= sinks and (b + 1) * P <= first:
                t[b] = -1
    return out


@pytest.mark.parametrize("fmt,dtype,D,P,heads,qh", [("int8", "fp16", 64, 32, 1, 1), ("e4m3", "bf16", 128, 64, 2, 8), ("int8", "bf16", 192, 128, 1, 3),
                                                    ("e4m3", "fp16", 256, 64, 2, 14), ("int8", "fp16", 128, 32, 3, 48)])
@pytest.mark.parametrize("window,sinks", [(1, 1), (7, 4), (33, 31), (64, 32), (100, 33), (31, 130), (500, 1), (90, 1 << 30), (1 << 30, 4)])
def test_one_token_per_sequence(fmt, dtype, D, P, heads, qh, window, sinks):
    rng = np.random.default_rng(D + heads)
    lens = [1, 0, 2, 31, 33, 64, 65, 96, 129, 131, 163, 500, 1030]
    m, table = build(rng, lens, heads, D, P, fmt, dtype)
    table = without_what_nobody_sees(table, lens, [1] * len(lens), P, window, sinks)
    check(m, table, lens, [1] * len(lens), qh, dtype, window, sinks, rng=rng)


@pytest.mark.parametrize("D,heads,qh,n_q", [(128, 2, 8, [3, 0, 1, 5, 2]), (64, 1, 7, [9, 8, 1, 0, 3]), (64, 1, 1, [17, 40, 1, 2, 33]), (192, 2, 6, [2, 11, 3, 1, 12])])
@pytest.mark.parametrize("causal,window,sinks", [(True, 1, 3), (True, 37, 40), (False, 20, 5), (True, 20, 64), (False, 3, 70)])
def test_several_tokens(D, heads, qh, n_q, causal, window, sinks):
    """Rows of one sequence whose windows begin before, among and behind the first tokens; rows before the sequence's first position."""
    rng = np.random.default_rng(window + D)
    lens = [40, 70, 1, 5, 210]
    m, table = build(rng, lens, heads, D, 32, "int8", "fp16")
    check(m, table, lens, n_q, qh, "fp16", window, sinks, causal, rng=rng)


@pytest.mark.parametrize("fmt,dtype,D,P,heads,qh", [("int8", "fp16", 128, 64, 1, 4), ("e4m3", "bf16", 64, 32, 1, 8), ("int8", "bf16", 256, 64, 1, 2),
                                                    ("e4m3", "fp16", 192, 128, 1, 3)])
@pytest.mark.parametrize("window,sinks,causal", [(50, 4, True), (1, 1, True), (90, 65, True), (33, 200, True), (70, 30, False)])
def test_chunks_of_prompts_beside_single_tokens(fmt, dtype, D, P, heads, qh, window, sinks, causal):
    rng = np.random.default_rng(7 + window)
    lens, n_q = [400, 129, 64, 700, 0, 300], [200, 65, 64, 140, 0, 1]
    m, table = build(rng, lens, heads, D, P, fmt, dtype)
    if causal:
        table = without_what_nobody_sees(table, lens, n_q, P, window, sinks)
    check(m, table, lens, n_q, qh, dtype, window, sinks, causal, rng=rng)
    check(m, table[3:4], lens[3:4], n_q[3:4], qh, dtype, window, sinks, causal, rng=rng, max_len=1, scale=-0.05)  # max_len only chooses


@pytest.mark.parametrize("D,qh,n", [(128, 4, 1), (64, 2, 3), (128, 4, 90), (256, 2, 200)])
@pytest.mark.parametrize("window,sinks", [(300, 90), (40, 600)])
def test_values_of_very_different_size_on_both_sides_of_the_gap(D, qh, n, window, sinks):
    rng = np.random.default_rng(3)
    sizes = [1e18, 1e-18, 1.0, 1e18, 1.0, 1e-18] * 4
    m, table, n_tokens = blocks_of_size(rng, sizes, 1, D, 32, "int8", 0.5)
    check(m, table, [n_tokens], [n], qh, "bf16", window, sinks, rng=rng, scale=0.02)


@pytest.mark.parametrize("n", [1, 6, 150])
def test_without_first_tokens_or_without_a_window_nothing_changes(n):
    rng = np.random.default_rng(5)
    lens = [300, 777]
    m, table = build(rng, lens, 2, 128, 64, "int8", "fp16")
    cache, q = m.device("fp16", DEV), to16(rng.normal(0, 2.0, (2 * n, 8, 128)).astype(np.float32), "fp16").to(DEV)
    args = cache, q, cu_of([n, n]), i32(lens), i32(table), n, 777
    for a, b in ((dict(window=100), dict(window=100, sinks=0)), (dict(), dict(sinks=40)), (dict(), dict(window=1000, sinks=40))):
        x, y = F.floe_kv_attention(*args, want_lse=True, **a), F.floe_kv_attention(*args, want_lse=True, **b)
        if b.get("window"):  # (another walk over the same tokens)
            assert float((x[0] - y[0]).abs().max()) <= 4e-3 and float((x[1] - y[1]).abs().max()) <= 2e-4
        else:
            assert torch.equal(x[0], y[0]) and torch.equal(x[1], y[1])


def test_a_scale_that_is_nan_counts_only_where_a_token_of_its_block_is_seen():
    rng = np.random.default_rng(11)
    lens = [600]
    m, table = build(rng, lens, 1, 128, 32, "e4m3", "fp16")
    for n in (1, 100):
        cache = m.device("fp16", DEV)
        cache.k_scale[table[0][7]] = float("nan")  # tokens 224 to 255: between the first tokens and every window
        cache.v_scale[table[0][8]] = float("nan")
        check(m, table, lens, [n], 4, "fp16", 60, 70, rng=rng, cache=cache)
        cache.v_scale[table[0][1]] = float("nan")  # the first tokens
        q = torch.randn((n, 4, 128), device=DEV).half()
        out = F.floe_kv_attention(cache, q, cu_of([n]), i32(lens), i32(table), n, 600, window=60, sinks=70)
        assert bool(out.isnan().all())


def test_a_captured_call_follows_the_lengths_on_the_device():
    rng = np.random.default_rng(12)
    lens = [700, 90]
    m, table = build(rng, lens, 2, 128, 32, "int8", "fp16")
    cache, q = m.device("fp16", DEV), torch.randn((2, 8, 128), device=DEV).half()
    length, cu, tab = i32(lens), cu_of([1, 1]), i32(table)
    out = torch.empty_like(q)
    call = lambda: F.floe_kv_attention(cache, q, cu, length, tab, 1, 700, window=80, sinks=40, out=out)  # noqa: E731
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for now in ([700, 90], [650, 1], [41, 89], [500, 0], [120, 60]):
        length.copy_(i32(now))
        graph.replay()
        got = out.clone()
        out.fill_(7)
        call()
        torch.cuda.synchronize()
        assert torch.equal(got, out), now
