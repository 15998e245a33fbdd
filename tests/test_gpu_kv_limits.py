"""Attention over the paged 8-bit cache at its limits: max_rows below a sequence's rows, values of V of very different size.  Formula in 64
bits from kv_reference.py; the tolerance is that of test_gpu_kv_attention.py."""
import numpy as np
import pytest
import torch

import kv_reference as R
import paper_2505_05950_amd as F
from test_gpu_kv_attention import build
from test_gpu_kv_cache import DEV, cu_of, i32, to16

pytestmark = pytest.mark.gpu


def compare(got, got_lse, want, want_lse, size, dtype, where):
    """Outputs of one sequence against the formula's: half a step of the type, fp16 weights and binary32 relative to sum p |v| / sum p."""
    got, got_lse = got.double().cpu().numpy(), got_lse.double().cpu().numpy()
    bar = R.HALF_STEP[dtype] * np.abs(want) + (2.0 ** -11 + 1e-4) * size + 2.0 ** -25
    off = np.abs(got - want)
    assert (off <= bar).all(), (where, np.argwhere(~(off <= bar))[:5], float((off / bar).max()))
    assert np.array_equal(np.isneginf(got_lse), np.isneginf(want_lse)), where
    ok = np.isfinite(want_lse)
    assert (np.abs(got_lse[ok] - want_lse[ok]) <= 1e-4 + 1e-6 * np.abs(want_lse[ok])).all(), where


@pytest.mark.parametrize("D,heads,qh,lens,n_q,most", [
    (128, 2, 8, [40, 70, 5, 210, 9], [12, 3, 0, 9, 11], 5),         # few rows
    (64, 1, 1, [900, 30], [64, 20], 1),
    (128, 2, 8, [700, 300, 64], [300, 129, 64], 70),                # many
    (256, 1, 2, [1500, 130], [700, 130], 129)])
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 7), (True, 90), (False, 50)])
def test_rows_behind_max_rows_are_left_out_and_those_before_keep_their_positions(D, heads, qh, lens, n_q, most, causal, window):
    rng = np.random.default_rng(D + window)
    m, table = build(rng, lens, heads, D, 32, "int8", "fp16")
    q = to16(rng.normal(0, 2.0, (sum(n_q), qh, D)).astype(np.float32), "fp16")
    out = torch.full((sum(n_q), qh, D), 5.0, dtype=torch.float16, device=DEV)
    lse = torch.full((sum(n_q), qh), 5.0, device=DEV)
    F.floe_kv_attention(m.device("fp16", DEV, 0x7f), q.to(DEV), cu_of(n_q), i32(lens), i32(table), most, max(lens), causal=causal, window=window,
                        out=out, lse=lse)
    torch.cuda.synchronize()
    at = 0
    for s, n in enumerate(n_q):
        k, there = m.value(0, lens[s], table[s])
        v, _ = m.value(1, lens[s], table[s])
        want, want_lse, size = R.attention(q[at:at + n].double().numpy(), k, v, there, lens[s], causal, window, D ** -0.5)
        c = min(n, most)
        compare(out[at:at + c], lse[at:at + c], want[:c], want_lse[:c], size[:c], "fp16", s)
        assert bool((out[at + c:at + n] == 5).all()) and bool((lse[at + c:at + n] == 5).all()), s
        at += n


def blocks_of_size(rng, sizes, heads, D, P, fmt, k_size):
    """One sequence whose blocks of P tokens have values of V of these sizes (0: a block of zeros, None: one whose scale is 0)."""
    n = P * len(sizes) - 5
    m = R.Model(len(sizes) + 1, heads, D, P, fmt)
    table = [[int(p) for p in rng.permutation(len(sizes) + 1)[:len(sizes)]]]
    m.append(0, (rng.normal(0, 1, (n, heads, D)) * k_size).astype(np.float32), 0, table[0])
    size = np.repeat([s or 0.0 for s in sizes], P)[:n, None, None]
    m.append(1, (rng.normal(0, 1, (n, heads, D)).clip(-3, 3) * size).astype(np.float32), 0, table[0])
    for page, s in zip(table[0], sizes):
        if s is None:
            m.scale[1][page] = 0.0
    return m, table, n


APART = [[1e37, 0.0], [0.0, 1e37], [0.0, 1e-15, 1e37, 1.0, 0.0], [1.0, None, 1.0], [1e37, None, None, 1.0], [None], [1e-25, 1e37, 0.0] * 3]


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("n_q,qh,copies", [(1, 4, 1), (1, 2, 40), (9, 4, 2), (200, 2, 1), (130, 2, 30)])
@pytest.mark.parametrize("k_size", [0.0, 0.5])
def test_tokens_count_in_the_softmax_whatever_the_size_of_their_values(fmt, n_q, qh, copies, k_size):
    """Scales of V that lie up to 181 powers of two apart, in one launch and joined from chunks: a token of small values, or of none, has
    its weight in the denominator and in the log-sum-exp beside one of large values."""
    for sizes in APART:
        rng = np.random.default_rng(len(sizes))
        m, table, n = blocks_of_size(rng, sizes * copies, 1, 64, 32, fmt, k_size)
        rows = min(n_q, n)
        q = to16(rng.normal(0, 2.0, (rows, qh, 64)).astype(np.float32), "bf16")
        out, lse = F.floe_kv_attention(m.device("bf16", DEV, 0x7f), q.to(DEV), cu_of([rows]), i32([n]), i32(table), rows, n, want_lse=True)
        torch.cuda.synchronize()
        k, there = m.value(0, n, table[0])
        v, _ = m.value(1, n, table[0])
        want, want_lse, size = R.attention(q.double().numpy(), k, v, there, n, True, 0, 64 ** -0.5)
        compare(out, lse, want, want_lse, size, "bf16", sizes)
