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
