"""The example that runs appending, attention and the MoE layer together: its captured steps, and the attention half against plain
arithmetic on the very cache that they left."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_the_example_decodes(fmt):
    import decode_block
    x, lengths = decode_block.main(tokens=6, batch=3, fmt=fmt, verbose=False)
    assert lengths.tolist() == [37 + 6, 248 + 6, 459 + 6]
    assert bool(torch.isfinite(x).all()) and float(x.float().square().mean()) == pytest.approx(1.0, rel=0.02)


def test_a_prompt_in_one_call_and_token_by_token_agree_on_the_rows_themselves():
    """Written at once or one by one, the cache stands for the same rows up to its own steps: half a step of the block's scale where
    rows are written at once, and at most one where the scale grew under them (by powers of two: 1/2 + 1/4 + ... of the last one)."""
    import paper_2505_05950_amd as F
    D, P, heads, n = 128, 64, 2, 150
    dev = "cuda"
    x = torch.randn((n, 2, heads, D), device=dev).half()
    table = torch.tensor([[2, 0, 1]], dtype=torch.int32, device=dev)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=dev)  # noqa: E731
    at_once, one_by_one = (F.KVCache(3, heads, D, P, F.KV_INT8, torch.float16, dev) for _ in range(2))
    F.floe_kv_append(at_once, x[:, 0], x[:, 1], i32([0, n]), i32([0]), table, n)
    for t in range(n):
        F.floe_kv_append(one_by_one, x[t:t + 1, 0], x[t:t + 1, 1], i32([0, 1]), i32([t]), table, 1)
    for cache, steps in ((at_once, 0.5), (one_by_one, 1.0)):
        for which, (got, scale) in enumerate(zip(F.floe_kv_gather(cache, i32([0]), i32([0, n]), table, n, n), (cache.k_scale, cache.v_scale))):
            per_row = scale[table[0].long()].repeat_interleave(P, 0)[:n, :, None]
            rounding = 2.0 ** -11 * got.float().abs()  # of the value read back
            assert bool(((got.float() - x[:, which].float()).abs() <= (steps + 1e-5) * per_row + rounding).all()), (which, steps)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_the_captured_step_appends_at_its_positions_and_attends_over_what_is_there(fmt, monkeypatch):
    """The last replay of the example's graph: its tensors are kept, and compared with the formulas in 64 bits over the cache it left."""
    import decode_block
    import kv_reference as R
    import numpy as np
    from test_gpu_kv_limits import compare
    F = decode_block.F
    appends, attends = [], []
    append, attention = F.floe_kv_append, F.floe_kv_attention

    def kept_append(cache, k, v, cu, before, table, most, q, rope):
        appends.append((cache, k, v, cu, before, table, q, rope, append(cache, k, v, cu, before, table, most, q=q, rope=rope)))
        return appends[-1][-1]

    def kept_attention(cache, q, cu, after, table, most, max_len):
        out, lse = attention(cache, q, cu, after, table, most, max_len, want_lse=True)
        attends.append((q, out, lse))
        return out
    monkeypatch.setattr(F, "floe_kv_append", kept_append)
    monkeypatch.setattr(F, "floe_kv_attention", kept_attention)
    _, lengths = decode_block.main(tokens=7, batch=3, fmt=fmt, verbose=False)
    torch.cuda.synchronize()
    assert len(appends) == len(attends) == 4  # the prompts, two eager steps, the captured one
    cache, k, v, _, _, table, q, rope, turned = appends[-1]
    of_graph, out, lse = attends[-1]
    assert of_graph is turned
    codes, scales = R.codes_of_device(cache)
    angles, table = rope.table.cpu().numpy(), table.cpu().numpy()
    heads, D, P = cache.kv_heads, cache.head_dim, cache.block
    for s, n in enumerate(lengths.tolist()):
        pages = table[s][:-(-n // P)]
        kk, vv = (np.concatenate([R.decode(c[p], fmt).astype(np.float64) * sc[p].astype(np.float64)[:, None, None] for p in pages], axis=1)[:, :n].transpose(1, 0, 2)
                  for c, sc in zip(codes, scales))
        # the appended token: rotated by its position, half a step of the code away (e4m3: 2^-4 of the value, or half its least step)
        for got, row, scale in ((kk[-1], R.rotate(k[s].float().cpu().numpy(), angles, n - 1, False), scales[0]), (vv[-1], v[s].float().cpu().numpy(), scales[1])):
            step = scale[pages[-1]][:, None].astype(np.float64)
            half = step / 2 if fmt == "int8" else np.maximum(np.abs(row) * 2.0 ** -4, step * 2.0 ** -10)
            assert (np.abs(got - row) <= half * (1 + 1e-5)).all(), s
        # its queries: the same rotation, rounded once
        want_q = R.rotate(q[s].float().cpu().numpy(), angles, n - 1, False)
        assert np.array_equal(turned[s].cpu().numpy(), want_q.astype(np.float16)), s
        want, want_lse, size = R.attention(turned[s:s + 1].double().cpu().numpy(), kk, vv, np.ones(n, bool), n, True, 0, D ** -0.5)
        compare(out[s:s + 1], lse[s:s + 1], want, want_lse, size, "fp16", s)
