"""Appending to the paged 8-bit cache and reading it back, against the model in kv_reference.py: codes, scales and rotated queries are
defined bit for bit, so they are compared bit for bit."""
import numpy as np
import pytest
import torch

import kv_reference as R
import paper_2505_05950_amd as F

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def cu_of(n):
    return i32(np.concatenate([[0], np.cumsum(n)]).tolist())


def angles(n, rot, base=10000.0):
    a = np.arange(n)[:, None] * base ** (-2.0 * np.arange(rot // 2) / rot)
    return np.stack([np.cos(a), np.sin(a)], -1).astype(np.float32)


def to16(x, dtype):
    return torch.from_numpy(np.ascontiguousarray(x)).to(R.DTYPES[dtype])


def bits(t):
    return t.contiguous().view(torch.int16).cpu().numpy()


def tables(rng, lens, P, spare=2):
    """Pages in no order, -1 where a sequence has none."""
    blocks = [-(-t // P) for t in lens]
    order = rng.permutation(sum(blocks) + spare)
    width, at, out = max(1, max(blocks)), 0, []
    for b in blocks:
        out.append(list(order[at:at + b]) + [-1] * (width - b))
        at += b
    return out, len(order)


def check_cache(cache, model, untouched=None):
    codes, scales = R.codes_of_device(cache)
    for which, name in ((0, "K"), (1, "V")):
        used = model.known.any(axis=1)
        assert np.array_equal(scales[which][used].view(np.uint32) & 0x7fc00000, model.scale[which][used].view(np.uint32) & 0x7fc00000), name
        finite = np.isfinite(model.scale[which]) & used[:, None]
        assert np.array_equal(scales[which][finite], model.scale[which][finite]), f"{name} scales"
        assert np.isnan(scales[which][used[:, None] & ~finite]).all()
        ok = model.known[:, None, :, None] & finite[:, :, None, None]
        same = (codes[which] == model.codes[which]) | ~ok
        assert same.all(), f"{name}: {np.argwhere(~same)[:4]} {(~same).sum()} of {ok.sum()}"


CASES = [
    # fmt, dtype, D, P, kv heads, q heads, rot, interleaved, appends (new rows of each sequence, call after call)
    ("int8", "fp16", 64, 32, 1, 1, 64, False, [[1], [1], [1], [31], [1]]),
    ("int8", "bf16", 128, 64, 2, 8, 128, False, [[63, 0, 64, 65, 1], [1, 1, 1, 1, 1], [2, 200, 0, 63, 5]]),
    ("e4m3", "fp16", 128, 64, 3, 21, 64, True, [[1, 7], [1, 1], [1, 1], [1, 130]]),
    ("e4m3", "bf16", 192, 128, 2, 2, 192, False, [[5, 0, 300], [124, 1, 1], [1, 1, 0]]),
    ("int8", "fp16", 256, 128, 1, 5, 16, True, [[129], [1], [500]]),
    ("e4m3", "fp16", 64, 128, 5, 10, 48, False, [[200, 3], [1, 1]]),
    ("int8", "bf16", 192, 32, 2, 6, 96, True, [[33, 1, 2], [1, 1, 1], [1, 40, 1]]),
]


@pytest.mark.parametrize("fmt,dtype,D,P,heads,qh,rot,inter,appends", CASES)
def test_append_is_the_definition_bit_for_bit(fmt, dtype, D, P, heads, qh, rot, inter, appends):
    rng = np.random.default_rng(D + P)
    total = np.sum(appends, axis=0)
    table, pages = tables(rng, total, P)
    model = R.Model(pages, heads, D, P, fmt)
    cache = F.KVCache(pages, heads, D, P, F.KV_INT8 if fmt == "int8" else F.KV_E4M3, R.DTYPES[dtype], DEV)
    for t in (cache.k, cache.v):
        t.fill_(0x7f)  # whatever was there (NaN in e4m3)
    cache.k_scale.fill_(float("nan")), cache.v_scale.fill_(float("nan"))
    ang = angles(int(total.max()) + 1, rot)
    rope = F.Rope(torch.from_numpy(ang).to(DEV), inter)
    length = np.zeros(len(total), int)
    for call, n in enumerate(appends):
        T = int(np.sum(n))
        # every call brings larger rows than the one before to some blocks, so that scales grow
        x = rng.normal(0, 1, (T, qh + 2 * heads, D)) * np.exp(rng.normal(0, 1.5, (T, 1, 1))) * (1 + call)
        x16 = to16(x.astype(np.float32), dtype)
        xd, x32 = x16.to(DEV), x16.float().numpy()
        q, k, v = xd[:, :qh], xd[:, qh:qh + heads], xd[:, qh + heads:]  # views of one projection's output
        got = F.floe_kv_append(cache, k, v, cu_of(n), i32(length.tolist()), i32(table), max(n), q=q, rope=rope)
        torch.cuda.synchronize()
        at = 0
        for s, m in enumerate(n):
            rows = x32[at:at + m]
            pos = np.arange(length[s], length[s] + m)
            turned = np.stack([R.rotate(rows[i], ang, pos[i], inter) for i in range(m)]) if m else rows
            model.append(0, turned[:, qh:qh + heads], int(length[s]), table[s])
            model.append(1, rows[:, qh + heads:], int(length[s]), table[s])
            want = to16(turned[:, :qh], dtype)
            assert np.array_equal(bits(got[at:at + m]), bits(want)), f"q of sequence {s}, call {call}"
            at += m
        length += n
        check_cache(cache, model)
    # and back: code * scale, rounded once
    first = [int(t) // 3 for t in total]
    rows = [int(t) - f for t, f in zip(total, first)]
    k, v = F.floe_kv_gather(cache, i32(first), cu_of(rows), i32(table), sum(rows), max(rows))
    torch.cuda.synchronize()
    at = 0
    for s, m in enumerate(rows):
        for which, got in ((0, k), (1, v)):
            for t in range(m):
                page, o = table[s][(first[s] + t) // P], (first[s] + t) % P
                want = R.decode(model.codes[which][page, :, o], fmt) * model.scale[which][page][:, None]
                assert np.array_equal(bits(got[at + t]), bits(to16(want, dtype))), (s, t, which)
        at += m


@pytest.mark.parametrize("fmt,dtype,D,P,heads,rot,inter", [
    ("int8", "fp16", 64, 32, 1, 64, False), ("e4m3", "bf16", 128, 64, 3, 64, True), ("int8", "bf16", 192, 128, 2, 32, False),
    ("e4m3", "fp16", 256, 128, 1, 256, False)])
def test_single_tokens_into_every_place_of_a_block(fmt, dtype, D, P, heads, rot, inter):
    # one sequence from nothing through a whole block into the next, one behind a prompt, one that rests in most calls
    steps = [[1, 1, int(i % 7 == 0)] for i in range(P + 3)]
    test_append_is_the_definition_bit_for_bit(fmt, dtype, D, P, heads, 2, rot, inter, [[0, P // 2 + 5, 1]] + steps)


def test_a_single_token_that_is_not_finite_says_so_until_its_block_is_opened_again():
    cache = F.KVCache(3, 2, 128, 32, F.KV_INT8, torch.bfloat16, DEV)
    x = torch.ones((1, 2, 128), dtype=torch.bfloat16, device=DEV)
    table = i32([[2, 0]])
    for i in range(6):
        y = x * (1.0 + i)
        if i == 3:
            y[0, 1, 127] = float("inf")
        F.floe_kv_append(cache, x, y, cu_of([1]), i32([i]), table, 1)
    k, v = F.floe_kv_gather(cache, i32([0]), cu_of([6]), table, 6, 6)
    assert torch.isnan(v[:, 1]).all() and torch.isfinite(v[:, 0]).all() and torch.isfinite(k).all()
    F.floe_kv_append(cache, x, x, cu_of([1]), i32([0]), table, 1)
    k, v = F.floe_kv_gather(cache, i32([0]), cu_of([1]), table, 1, 1)
    assert torch.isfinite(v).all()


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_a_block_that_takes_a_value_that_is_not_finite_says_so_until_it_is_opened_again(fmt, bad):
    D, P = 64, 32
    cache = F.KVCache(2, 2, D, P, F.KV_INT8 if fmt == "int8" else F.KV_E4M3, torch.float16, DEV)
    x = torch.ones((4, 2, D), dtype=torch.float16, device=DEV)
    table = i32([[1, 0]])
    F.floe_kv_append(cache, x, x, cu_of([4]), i32([0]), table, 4)
    y = x.clone()
    y[2, 1, 5] = bad
    F.floe_kv_append(cache, y, x, cu_of([4]), i32([4]), table, 4)
    F.floe_kv_append(cache, x, x, cu_of([4]), i32([8]), table, 4)
    k, v = F.floe_kv_gather(cache, i32([0]), cu_of([12]), table, 12, 12)
    assert torch.isnan(k[:, 1]).all() and torch.isfinite(k[:, 0]).all() and torch.isfinite(v).all()
    F.floe_kv_append(cache, x, x, cu_of([4]), i32([0]), table, 4)
    k, v = F.floe_kv_gather(cache, i32([0]), cu_of([4]), table, 4, 4)
    assert torch.equal(k, x)


def test_zero_rows_extreme_rows_and_positions_of_ones_own():
    D, P = 64, 32
    rng = np.random.default_rng(1)
    model = R.Model(1, 1, D, P, "int8")
    cache = F.KVCache(1, 1, D, P, F.KV_INT8, torch.bfloat16, DEV)
    ang = angles(5000, 32)
    rope = F.Rope(torch.from_numpy(ang).to(DEV))
    # a block that opens with zeros (least scale), then 1e-30 (below it), 1.0, 1e30, and zeros again
    for t, size in enumerate((0.0, 1e-30, 1.0, 1e30, 0.0)):
        x16 = to16((rng.normal(0, 1, (1, 1, D)) * size).astype(np.float32), "bf16")
        pos = [4999, 0, 17, 3, 1][t]
        F.floe_kv_append(cache, x16.to(DEV), x16.to(DEV), cu_of([1]), i32([t]), i32([[0]]), 1, rope=rope, positions=i32([pos]))
        model.append(0, R.rotate(x16.float().numpy()[0], ang, pos, False)[None], t, [0])
        model.append(1, x16.float().numpy(), t, [0])
        check_cache(cache, model)
    # a position outside the table
    one = torch.ones((1, 1, D), dtype=torch.bfloat16, device=DEV)
    for pos in (-1, 5000):
        q = F.floe_kv_append(cache, one, one, cu_of([1]), i32([0]), i32([[0]]), 1, q=one, rope=rope, positions=i32([pos]))
        assert torch.isnan(cache.k_scale).all() and torch.isfinite(cache.v_scale).all()
        assert torch.isnan(q[..., :32]).all() and torch.equal(q[..., 32:], one[..., 32:])


def test_absent_pages_rows_of_nobody_and_limits_are_left_alone():
    D, P, pages = 64, 32, 6
    cache = F.KVCache(pages, 1, D, P, F.KV_E4M3, torch.float16, DEV)
    for t in (cache.k, cache.v):
        t.fill_(7)
    cache.k_scale.fill_(3.0), cache.v_scale.fill_(3.0)
    x = torch.randn((90, 1, D), device=DEV).half()
    q_out = torch.full((90, 1, D), 5.0, dtype=torch.float16, device=DEV)
    rope = F.Rope(torch.from_numpy(angles(200, 64)).to(DEV))
    # sequence 0: block 1 absent; sequence 1: runs out of the table; rows 80.. belong to nobody
    F.floe_kv_append(cache, x, x, i32([0, 70, 80]), i32([20, 60]), i32([[4, -1, 2], [9, 3, 1 << 30]]), 70, q=x, rope=rope, q_out=q_out)
    torch.cuda.synchronize()
    assert sorted({p for p in range(pages) if not (cache.k[p] == 7).all()}) == [2, 3, 4]
    assert (cache.k_scale[[0, 1, 5]] == 3).all() and (cache.v_scale[[0, 1, 5]] == 3).all()
    assert (q_out[80:] == 5).all() and (q_out[:80] != 5).any(dim=-1).all()
    k, v = F.floe_kv_gather(cache, i32([20, 60]), i32([0, 70, 80]), i32([[4, -1, 2], [9, 3, 1 << 30]]), 90, 70)
    assert (k[12:44] == 0).all() and (v[12:44] == 0).all()   # tokens 32 .. 63 of sequence 0
    # max_rows smaller than a sequence's rows: the rows behind are left out
    cache.k.fill_(7)
    F.floe_kv_append(cache, x, x, i32([0, 90]), i32([0]), i32([[0, 1, 5]]), 33)
    codes, _ = R.codes_of_device(cache)
    assert (codes[0][1, 0, 1:] == 7).all() and not (codes[0][1, 0, 0] == 7).all() and (codes[0][5] == 7).all()
    # nothing to do
    F.floe_kv_append(cache, x[:0], x[:0], i32([0]), i32([]), torch.zeros((0, 1), dtype=torch.int32, device=DEV), 0)
    F.floe_kv_append(cache, x, x, i32([0, 0]), i32([0]), i32([[-1]]), 5)


def test_rope_table_against_longer_arithmetic():
    n, rot, base = 300000, 64, 500000.0
    got = F.floe_rope_table(n, rot, base, DEV).cpu().numpy()
    rows = np.array([0, 1, 2, 1000, 65537, 299999])
    a = rows[:, None].astype(np.longdouble) * np.longdouble(base) ** (-2 * np.arange(rot // 2, dtype=np.longdouble) / rot)
    want = np.stack([np.cos(a), np.sin(a)], -1)
    # one rounding to binary32 (2^-24 of the value) and the angle's own error in binary64, 3e5 * 2^-52
    assert np.all(np.abs(got[rows] - want) <= 2.0 ** -24 * np.abs(want) + 3e5 * 2.0 ** -51)


def test_a_cache_whose_offsets_pass_32_bits():
    D, P, heads = 128, 64, 8
    pages = 5 * 2 ** 30 // (D * P * heads)
    cache = F.KVCache(pages, heads, D, P, F.KV_INT8, torch.float16, DEV)
    x = torch.randn((70, heads, D), device=DEV).half()
    table = i32([[pages - 1, pages // 2 + 3]])
    F.floe_kv_append(cache, x, x, cu_of([70]), i32([0]), table, 70)
    k, v = F.floe_kv_gather(cache, i32([0]), cu_of([70]), table, 70, 70)
    model = R.Model(2, heads, D, P, "int8")
    for which, got in ((0, k), (1, v)):
        model.append(which, x.float().cpu().numpy(), 0, [0, 1])
        for t in range(70):
            want = R.decode(model.codes[which][t // P, :, t % P], "int8") * model.scale[which][t // P][:, None]
            assert np.array_equal(bits(got[t]), bits(to16(want, "fp16"))), (which, t)
    o = F.floe_kv_attention(cache, x[-1:].repeat(1, 2, 1).contiguous(), cu_of([1]), i32([70]), table, 1, 70)
    for h2 in range(2 * heads):
        q = x[-1, h2 % heads].double().cpu()
        p = (k[:, h2 // 2].double().cpu() @ q / D ** 0.5).softmax(0)
        w = p @ v[:, h2 // 2].double().cpu()
        size = p @ v[:, h2 // 2].double().cpu().abs()  # weights rounded to fp16, K and V read back in fp16, one rounding at the end
        assert ((o[0, h2].double().cpu() - w).abs() <= 2.0 ** -9 * size).all()


def test_tensors_that_are_not_on_the_caches_device_are_refused():
    c = F.KVCache(2, 2, 64, 32, device=DEV)
    cu, n, table = cu_of([3]), i32([0]), i32([[0, 1]])
    x = torch.zeros((3, 2, 64), dtype=torch.float16, device=DEV)
    rope = F.Rope(torch.zeros((8, 32, 2), dtype=torch.float32))
    for args, more in (((x.cpu(), x, cu, n, table), {}), ((x, x.cpu(), cu, n, table), {}), ((x, x, cu.cpu(), n, table), {}),
                       ((x, x, cu, n.cpu(), table), {}), ((x, x, cu, n, table.cpu()), {}), ((x, x, cu, n, table), dict(rope=rope)),
                       ((x, x, cu, n, table), dict(positions=torch.zeros(3, dtype=torch.int32)))):
        with pytest.raises(ValueError):
            F.floe_kv_append(c, *args, 3, **more)
    for q, more in ((x.cpu(), {}), (x, dict(out=x.cpu())), (x, dict(lse=torch.zeros((3, 2)))), (x, dict(workspace=torch.zeros(1 << 20, dtype=torch.uint8)))):
        with pytest.raises(ValueError):
            F.floe_kv_attention(c, q, cu, i32([3]), table, 3, 3, **more)
    with pytest.raises(ValueError):
        F.floe_kv_gather(c, n, cu, table, 3, 3, k_out=x.cpu())
    with pytest.raises(ValueError):
        F.KVCache(2, 2, 64, 32, device=DEV, tensors=(c.k, c.v, c.k_scale.cpu(), c.v_scale))
