"""Attention over the paged 8-bit cache against the formula in 64 bits (kv_reference.py).

Tolerance, per element: the final rounding (half a step of the 16-bit type) and, relative to sum p |v| / sum p, the rounding of the weights
to fp16 (2^-11) plus 1e-4 for what is done in binary32: exponents of at most 64 in size are formed with a handful of roundings
(8 * 64 * 2^-24 = 3e-5), and sums of a few thousand terms run in chains of at most 1000 (1000 * 2^-24 = 6e-5).  lse: the same 1e-4."""
import numpy as np
import pytest
import torch

import kv_reference as R
import paper_2505_05950_amd as F
from test_gpu_kv_cache import DEV, angles, cu_of, i32, tables, to16

pytestmark = pytest.mark.gpu


def build(rng, lens, heads, D, P, fmt, dtype, v_spread=0.0, k_size=1.0, spare=2):
    """A model cache with `lens` tokens per sequence, blocks of very different V scales with v_spread."""
    table, pages = tables(rng, lens, P, spare)
    m = R.Model(pages, heads, D, P, fmt)
    for s, n in enumerate(lens):
        for which in (0, 1):
            x = rng.normal(0, 1, (n, heads, D)).astype(np.float32) * np.float32(k_size if which == 0 else 1.0)
            if which == 1 and v_spread:
                x *= np.exp(rng.normal(0, v_spread, (-(-n // P), 1, 1)).repeat(P, 0)[:n]).astype(np.float32)
            m.append(which, x, 0, table[s])
    return m, table


def check(m, table, lens, n_q, qh, dtype, causal=True, window=0, scale=None, q_size=2.0, rng=None, fill=0x7f, max_len=None, q=None):
    rng = rng or np.random.default_rng(0)
    T, D = sum(n_q), m.D
    if q is None:
        q = to16((rng.normal(0, q_size, (T, qh, D))).astype(np.float32), dtype)
    cache = m.device(dtype, DEV, fill)
    max_q = max(n_q) if n_q else 0
    out, lse = F.floe_kv_attention(cache, q.to(DEV), cu_of(n_q), i32(list(lens)), i32(table), max_q, max(lens) if max_len is None else max_len,
                                   scale=scale, causal=causal, window=window, want_lse=True)
    torch.cuda.synchronize()
    out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    scale = D ** -0.5 if scale is None else scale
    at = 0
    for s, n in enumerate(n_q):
        k, there = m.value(0, lens[s], table[s])
        v, _ = m.value(1, lens[s], table[s])
        want, want_lse, size = R.attention(q[at:at + n].double().numpy(), k, v, there, lens[s], causal, window, scale)
        got, got_lse = out[at:at + n], lse[at:at + n]
        nan = np.isnan(want)
        assert np.array_equal(np.isnan(got), nan), (s, np.argwhere(np.isnan(got) != nan)[:5])
        bar = R.HALF_STEP[dtype] * np.abs(want) + (2.0 ** -11 + 1e-4) * size + 2.0 ** -25
        off = np.abs(got - want)
        bad = ~(off <= bar) & ~nan
        assert not bad.any(), (s, np.argwhere(bad)[:5], got[bad][:5], want[bad][:5], float((off / bar)[~nan].max()))
        assert np.array_equal(np.isneginf(got_lse), np.isneginf(want_lse)) and np.array_equal(np.isnan(got_lse), np.isnan(want_lse))
        ok = np.isfinite(want_lse)
        assert (np.abs(got_lse[ok] - want_lse[ok]) <= 1e-4 + 1e-6 * np.abs(want_lse[ok])).all()
        at += n


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("D,P,heads,qh", [(64, 32, 1, 1), (128, 64, 2, 8), (192, 128, 1, 3), (256, 64, 2, 14), (128, 32, 3, 48), (64, 128, 5, 5)])
def test_one_token_per_sequence(fmt, dtype, D, P, heads, qh):
    rng = np.random.default_rng(D + heads)
    lens = [1, 0, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 500, 1030]
    m, table = build(rng, lens, heads, D, P, fmt, dtype)
    check(m, table, lens, [1] * len(lens), qh, dtype, rng=rng)


@pytest.mark.parametrize("D,heads,qh,n_q", [(128, 2, 8, [3, 0, 1, 5, 2]), (64, 1, 7, [9, 8, 1, 0, 3]), (128, 1, 1, [17, 40, 1, 2, 33]),
                                            (256, 1, 4, [5, 1, 9, 2, 1]), (192, 2, 6, [2, 11, 3, 1, 12])])
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 1), (True, 37), (False, 20), (True, 4000)])
def test_several_tokens_masks_and_windows(D, heads, qh, n_q, causal, window):
    rng = np.random.default_rng(window + D)
    lens = [40, 70, 1, 5, 210]
    m, table = build(rng, lens, heads, D, 32, "int8", "fp16")
    check(m, table, lens, n_q, qh, "fp16", causal, window, rng=rng)


@pytest.mark.parametrize("fmt,dtype,D,P,heads,qh,window", [("int8", "fp16", 128, 64, 1, 4, 0), ("e4m3", "bf16", 128, 128, 2, 2, 50),
                                                           ("e4m3", "fp16", 64, 32, 1, 8, 0), ("int8", "bf16", 256, 64, 1, 2, 0),
                                                           ("int8", "fp16", 192, 64, 1, 3, 100)])
def test_chunks_of_prompts(fmt, dtype, D, P, heads, qh, window):
    rng = np.random.default_rng(7)
    lens, n_q = [300, 129, 64, 200], [300, 65, 64, 70]
    m, table = build(rng, lens, heads, D, P, fmt, dtype)
    check(m, table, lens, n_q, qh, dtype, True, window, rng=rng)


@pytest.mark.parametrize("D,heads,qh,P", [(64, 1, 2, 32), (128, 2, 8, 32), (192, 1, 3, 128), (256, 1, 2, 64)])
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 1), (True, 90), (False, 200)])
def test_long_and_short_chunks_in_one_call(D, heads, qh, P, causal, window):
    """Both kernels in one call; tiles of rows that are cut over their tokens, rows and tiles that are not full."""
    rng = np.random.default_rng(D + window)
    lens, n_q = [700, 90, 3, 0, 260, 130], [150, 90, 1, 0, 2, 129]
    m, table = build(rng, lens, heads, D, P, "e4m3" if D % 128 else "int8", "fp16")
    check(m, table, lens, n_q, qh, "fp16", causal, window, rng=rng)
    check(m, table[:1], [700], [150], qh, "bf16", causal, window, rng=rng)
    check(m, table[:1], [700], [150], qh, "fp16", causal, window, rng=rng, max_len=1, scale=-0.05)  # max_len only chooses


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_long_chunks_with_absent_pages_nan_blocks_and_extreme_scales(fmt):
    rng = np.random.default_rng(21)
    lens, n_q = [500, 330], [160, 200]
    m, table = build(rng, lens, 1, 128, 32, fmt, "bf16", v_spread=6.0)
    check(m, table, lens, n_q, 2, "bf16", rng=rng)
    check(m, table, lens, n_q, 2, "bf16", scale=0.0, rng=rng)
    table[0][2], table[1][0], table[1][9] = -1, 1 << 30, -7
    check(m, table, lens, n_q, 2, "bf16", rng=rng)
    check(m, [t[:5] for t in table], lens, n_q, 2, "bf16", rng=rng)
    m.scale[0][table[0][11], 0] = np.nan
    m.scale[1][table[1][4], 0] = np.nan
    check(m, table, lens, n_q, 2, "bf16", rng=rng)
    check(m, table, lens, n_q, 2, "bf16", window=40, rng=rng)
    check(m, table, [100, 20], [160, 200], 2, "bf16", rng=rng)  # more rows than tokens


@pytest.mark.parametrize("garbage", [0.0, -1.0, np.inf, np.nan, 1e-42])
def test_pages_of_nobody_hold_anything(garbage):
    """Codes and scales that no token has, page 0 among them, which an absent page's address falls on."""
    rng = np.random.default_rng(4)
    lens = [300, 200]
    table, pages = tables(rng, lens, 32)
    table = [[p + 1 if p >= 0 else p for p in t] for t in table]
    m = R.Model(pages + 1, 1, 128, 32, "e4m3")
    for s, n in enumerate(lens):
        for which in (0, 1):
            m.append(which, rng.normal(0, 1, (n, 1, 128)).astype(np.float32), 0, table[s])
    unused = ~m.known.any(axis=1)
    for scale in m.scale:
        scale[unused] = garbage
    table[0][4] = table[1][0] = table[1][1] = -1
    check(m, table, lens, [1, 2], 4, "fp16", rng=rng)
    check(m, table, lens, [150, 120], 2, "fp16", rng=rng)


def test_more_rows_than_tokens_and_absent_pages():
    rng = np.random.default_rng(3)
    lens = [3, 100, 130, 96]
    m, table = build(rng, lens, 2, 64, 32, "e4m3", "fp16")
    table[1] = [-1] * len(table[1])           # nothing is there
    table[2][1], table[3][0] = -5, 1 << 30    # a hole, a lost beginning
    check(m, table, lens, [8, 2, 2, 40], 4, "fp16", rng=rng)
    # the table ends before the sequence does
    check(m, [t[:2] for t in table], lens, [1, 1, 1, 1], 4, "fp16", rng=rng)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_blocks_of_very_different_size(fmt):
    """Scales of V over many powers of ten; a row whose weights lie where V is small; keys so large that one token has all weight."""
    rng = np.random.default_rng(5)
    lens = [400, 33]
    m, table = build(rng, lens, 1, 64, 32, fmt, "bf16", v_spread=8.0)
    check(m, table, lens, [1, 1], 4, "bf16", rng=rng)
    m, table = build(rng, lens, 1, 64, 32, fmt, "fp16", k_size=30.0)
    check(m, table, lens, [4, 1], 4, "fp16", scale=0.02, rng=rng)
    check(m, table, lens, [4, 1], 4, "fp16", scale=-0.02, rng=rng)
    check(m, table, lens, [4, 1], 4, "fp16", scale=0.0, rng=rng)


def test_queries_of_any_size_in_bf16():
    """Rows of 1e-30 and 1e30, subnormals and zeros: a power of two per row brings them into range."""
    rng = np.random.default_rng(9)
    lens = [70] * 5
    m, table = build(rng, lens, 1, 128, 64, "int8", "bf16")
    for size, scale in ((1e-30, 1e29), (1e30, 1e-31), (0.0, 1.0), (1e-39, 1e38), (300.0, 1e-3)):
        check(m, table, lens, [1] * 5, 2, "bf16", scale=scale, q_size=size, rng=rng)


def test_what_is_not_finite_stays_in_its_row_and_block():
    rng = np.random.default_rng(11)
    lens = [40, 100]
    m, table = build(rng, lens, 2, 64, 32, "int8", "fp16")
    q = to16(rng.normal(0, 2, (2, 4, 64)).astype(np.float32), "fp16")
    q[0, 1, 3], q[1, 2, 0] = float("nan"), float("inf")
    cache = m.device("fp16", DEV, 0x7f)
    out = F.floe_kv_attention(cache, q.to(DEV), cu_of([1, 1]), i32(lens), i32(table), 1, 100)
    nan = torch.isnan(out).all(-1).cpu()
    assert nan[0, 1] and nan[1, 2] and int(nan.sum()) == 2 and int(torch.isnan(out).any(-1).sum()) == 2
    # a block with a NaN scale: every row that sees one of its tokens, and no other (causal rows before it, windows behind it, other heads)
    m.scale[0][table[1][1], 0] = np.nan
    m.scale[1][table[1][2], 1] = np.nan
    check(m, table, lens, [3, 80], 4, "fp16", rng=rng)
    check(m, table, lens, [3, 80], 4, "fp16", window=3, rng=rng)
    check(m, table, [40, 32], [3, 30], 4, "fp16", rng=rng)   # block 1 holds nothing of the sequence now


def test_long_sequences_split_over_the_card_and_ragged_batches():
    """Against the same formula on the device in 64 bits: lengths over several shares, one long sequence beside many short ones."""
    for heads, qh, lens, dtype, fmt, D, P in ((2, 8, [20011], "fp16", "int8", 128, 64), (1, 1, [70001, 5, 0, 64], "bf16", "e4m3", 64, 128),
                                              (4, 4, [1500, 9000, 3, 1, 700] * 20, "fp16", "int8", 128, 32), (2, 10, [9000, 31], "fp16", "e4m3", 256, 64)):
        g = torch.Generator(device=DEV).manual_seed(len(lens))
        blocks = [-(-n // P) for n in lens]
        width, pages = max(blocks), sum(blocks)
        order = torch.randperm(pages, generator=g, device=DEV).int()
        table = torch.full((len(lens), width), -1, dtype=torch.int32, device=DEV)
        at = 0
        for s, b in enumerate(blocks):
            table[s, :b] = order[at:at + b]
            at += b
        cache = F.KVCache(pages, heads, D, P, F.KV_INT8 if fmt == "int8" else F.KV_E4M3, R.DTYPES[dtype], DEV)
        x = torch.randn((sum(lens), 2, heads, D), generator=g, device=DEV).to(R.DTYPES[dtype])
        cu = cu_of(lens)
        F.floe_kv_append(cache, x[:, 0], x[:, 1], cu, i32([0] * len(lens)), table, max(lens))
        # what the cache holds, in 64 bits
        kind = torch.int8 if fmt == "int8" else torch.float8_e4m3fn
        place = torch.from_numpy(R.v_index(P, D).ravel()).to(DEV)
        values = [cache.k.view(pages, heads, P, D).view(kind).double() * cache.k_scale.double()[..., None, None],
                  cache.v.view(pages, heads, P * D)[..., place].view(pages, heads, P, D).view(kind).double() * cache.v_scale.double()[..., None, None]]
        def of(which, s, head, upto):  # noqa: E306
            return values[which][table[s, :-(-upto // P)].long(), head].reshape(-1, D)[:upto]
        n_q = [2 if n else 1 for n in lens]
        q = torch.randn((sum(n_q), qh, D), generator=g, device=DEV).mul_(2).to(R.DTYPES[dtype])
        out, lse = F.floe_kv_attention(cache, q, cu_of(n_q), i32(lens), table, 2, max(lens), want_lse=True)
        row = 0
        for s, n in enumerate(lens):
            for i in range(n_q[s]):
                see = n - n_q[s] + i + 1
                for h in range(qh):
                    if see <= 0:
                        assert (out[row, h] == 0).all() and lse[row, h] == -float("inf")
                        continue
                    a = (of(0, s, h // (qh // heads), see) @ q[row, h].double()) / D ** 0.5
                    p, vv = a.softmax(0), of(1, s, h // (qh // heads), see)
                    bar = R.HALF_STEP[dtype] * (p @ vv).abs() + (2.0 ** -11 + 1e-4) * (p @ vv.abs()) + 2.0 ** -25
                    assert bool(((out[row, h].double() - p @ vv).abs() <= bar).all()), (s, i, h)
                    assert abs(float(lse[row, h]) - float(a.logsumexp(0))) <= 1e-4 + 1e-6 * abs(float(a.logsumexp(0)))
                row += 1


def test_results_do_not_depend_on_the_rest_of_the_batch_beyond_rounding_and_repeat_exactly():
    rng = np.random.default_rng(2)
    lens = [700, 3, 900, 64]
    m, table = build(rng, lens, 2, 128, 64, "int8", "fp16")
    cache = m.device("fp16", DEV)
    q = torch.randn((4, 8, 128), device=DEV).half()
    first = F.floe_kv_attention(cache, q, cu_of([1] * 4), i32(lens), i32(table), 1, 900)
    for _ in range(5):
        assert torch.equal(first, F.floe_kv_attention(cache, q, cu_of([1] * 4), i32(lens), i32(table), 1, 900))
    alone = F.floe_kv_attention(cache, q[2:3], cu_of([1]), i32(lens[2:3]), i32(table[2:3]), 1, 900)
    assert (alone - first[2:3]).abs().max() < 2e-3


def test_captured_step_follows_lengths_and_tables_that_change():
    """Append and attention in one graph; the lengths, the tables and the rows change between replays, eager calls run in between."""
    D, P, heads, qh, B = 128, 32, 2, 8, 3
    cache = F.KVCache(16, heads, D, P, F.KV_INT8, torch.float16, DEV)
    eager = F.KVCache(16, heads, D, P, F.KV_INT8, torch.float16, DEV)
    table = i32([[0, 1, 2], [5, 4, 3], [9, 8, 7]])
    cu, before, after = cu_of([1] * B), i32([0] * B), i32([1] * B)
    x = torch.zeros((B, qh + 2 * heads, D), dtype=torch.float16, device=DEV)
    rope = F.Rope(F.floe_rope_table(100, D, device=DEV))
    out = torch.empty((B, qh, D), dtype=torch.float16, device=DEV)

    def step(c, o):
        q = F.floe_kv_append(c, x[:, qh:qh + heads], x[:, qh + heads:], cu, before, table, 1, q=x[:, :qh], rope=rope)
        return F.floe_kv_attention(c, q, cu, after, table, 1, 96, out=o)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(cache, out)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(cache, out)
    g = torch.Generator(device=DEV).manual_seed(0)
    for t in range(70):
        before.fill_(t), after.fill_(t + 1)
        x.copy_(torch.randn(x.shape, generator=g, device=DEV))
        graph.replay()
        got = out.clone()
        want = step(eager, None)
        torch.cuda.synchronize()
        assert torch.equal(got, want), t
        assert torch.equal(cache.k_scale[[0, 5, 9]], eager.k_scale[[0, 5, 9]])


def test_calls_on_a_stream_of_their_own():
    rng = np.random.default_rng(2)
    lens = [300, 50]
    m, table = build(rng, lens, 1, 64, 32, "int8", "fp16")
    cache = m.device("fp16", DEV)
    q = torch.randn((2, 4, 64), device=DEV).half()
    args = (cache, q, cu_of([1, 1]), i32(lens), i32(table), 1, 300)
    want = F.floe_kv_attention(*args)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = F.floe_kv_attention(*args, stream=s)
    s.synchronize()
    assert torch.equal(got, want)


@pytest.mark.parametrize("D,fmt,dtype,heads,n,context", [
    (128, "int8", "fp16", 4, 2048, 2048), (128, "e4m3", "bf16", 2, 1600, 6000), (192, "e4m3", "fp16", 4, 1600, 1600), (192, "int8", "bf16", 2, 1600, 6000),
    (192, "int8", "fp16", 4, 1600, 2500), (256, "int8", "bf16", 4, 1000, 1000), (256, "e4m3", "fp16", 2, 1000, 4100), (256, "int8", "fp16", 1, 500, 3000)])
def test_prompts_that_fill_the_card(D, fmt, dtype, heads, n, context):
    # enough rows for the larger workgroups, with the context whole and cut; rows at the ends of their tiles and some between
    rng = np.random.default_rng(D + context)
    m, table = build(rng, [context], heads, D, 64, fmt, dtype)
    q = to16(rng.normal(0, 2.0, (n, 8 * heads, D)).astype(np.float32), dtype)
    out, lse = F.floe_kv_attention(m.device(dtype, DEV, 0x7f), q.to(DEV), cu_of([n]), i32([context]), i32(table), n, context, want_lse=True)
    torch.cuda.synchronize()
    k, there = m.value(0, context, table[0])
    v, _ = m.value(1, context, table[0])
    for i in [0, 1, 15, 16, 31, 32, 33, 63, 64, n // 2, n // 2 + 7, n - 33, n - 32, n - 2, n - 1]:
        seen = context - n + i + 1
        want, want_lse, size = R.attention(q[i:i + 1].double().numpy(), k[:seen], v[:seen], there[:seen], seen, True, 0, D ** -0.5)
        off = np.abs(out[i].double().cpu().numpy() - want[0])
        bar = R.HALF_STEP[dtype] * np.abs(want[0]) + (2.0 ** -11 + 1e-4) * size[0] + 2.0 ** -25
        assert (off <= bar).all(), (i, float((off / bar).max()))
        assert (np.abs(lse[i].double().cpu().numpy() - want_lse[0]) <= 1e-4 + 1e-6 * np.abs(want_lse[0])).all(), i


@pytest.mark.parametrize("D,heads,qh", [(128, 1, 128), (64, 2, 130), (256, 1, 80)])
def test_groups_of_more_heads_than_the_rows_kernel_takes(D, heads, qh):
    rng = np.random.default_rng(qh)
    lens = [1, 0, 33, 64, 200, 700]
    m, table = build(rng, lens, heads, D, 32, "int8", "fp16")
    check(m, table, lens, [1, 0, 1, 1, 1, 1], qh, "fp16", rng=rng)
    check(m, table, lens, [1, 0, 2, 1, 3, 0], qh, "fp16", rng=rng)
