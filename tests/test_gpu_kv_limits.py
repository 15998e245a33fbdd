"""What the limits that a caller states do to attention over the paged 8-bit cache: max_rows below a sequence's rows.  Formula in 64 bits
from kv_reference.py; the tolerance is that of test_gpu_kv_attention.py."""
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
