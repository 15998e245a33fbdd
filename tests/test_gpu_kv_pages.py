"""The pages of the cache: tables, counts and pairs against a plain model (kv_pool_reference.py), number by number; copies byte by byte."""
import random

import pytest
import torch

import paper_2505_05950_amd as F
from kv_pool_reference import Pool

pytestmark = pytest.mark.gpu
DEV = "cuda"


def i32(v, *shape):
    t = torch.tensor(v, dtype=torch.int32, device=DEV)
    return t.view(*shape) if shape else t


def device_pool(ref):
    return F.KVPool(ref.n, ref.block, refs=i32(ref.refs))


def refused(ref):
    """A pool of no pages (a state of empty sequences) is refused."""
    if ref.n:
        return False
    with pytest.raises(ValueError):
        device_pool(ref)
    return True


def cu_of(rows):
    out = [0]
    for n in rows:
        out.append(out[-1] + n)
    return i32(out)


def state(seed, n_seqs, block, most, spare, absent=0.0, share=False):
    """A pool and a table of sequences of up to `most` tokens with their pages in no order; `share`: some take over a prefix of another's."""
    rng = random.Random(seed)
    length = [rng.choice([0, 1, block - 1, block, block + 1, rng.randint(0, most)]) for _ in range(n_seqs)]
    width = most // block + 2
    need = sum(-(-n // block) for n in length)
    pages = list(range(need + spare))
    rng.shuffle(pages)
    table, at = [], 0
    for n in length:
        row = pages[at:at + -(-n // block)]
        at += len(row)
        table.append(row + [-1] * (width - len(row)))
    if share:
        for s in range(1, n_seqs, 2):
            k = rng.randint(0, min(length[s], length[s - 1]) // block)
            table[s][:k] = table[s - 1][:k]
    for row in table:
        for b in range(width):
            if rng.random() < absent:
                row[b] = rng.choice([-1, -7, len(pages), 1 << 30])
    return Pool(len(pages), block).count(table), table, length, rng


def same(pool, table, ref, want):
    torch.cuda.synchronize()
    assert table.tolist() == want
    assert pool.refs.tolist() == ref.refs


@pytest.mark.parametrize("seed", range(6))
@pytest.mark.parametrize("n_seqs,n_out,block,most", [(1, 1, 32, 40), (3, 17, 64, 900), (40, 40, 32, 300), (5, 2, 128, 5000), (200, 333, 64, 30000 // 40)])
def test_reorder(seed, n_seqs, n_out, block, most):
    ref, table, length, rng = state(seed, n_seqs, block, most, 5, 0.1 if seed % 2 else 0.0, share=seed > 2)
    parent = [rng.choice([rng.randrange(n_seqs), rng.randrange(n_seqs), 0, -1, n_seqs, 1 << 30]) for _ in range(n_out)]
    pool, t = device_pool(ref), i32(table)
    got, got_len = F.floe_kv_reorder(pool, t, i32(length), i32(parent))
    want, want_len = ref.reorder(table, length, parent)
    same(pool, got, ref, want)
    assert got_len.tolist() == want_len and t.tolist() == table


@pytest.mark.parametrize("seed", range(8))
@pytest.mark.parametrize("n_seqs,block,most,rows_most,spare", [(1, 32, 40, 1, 0), (7, 64, 900, 200, 40), (60, 32, 300, 1, 20), (1500, 32, 90, 3, 700), (3, 128, 20000, 9000, 300)])
def test_reserve(seed, n_seqs, block, most, rows_most, spare):
    ref, table, length, rng = state(seed, n_seqs, block, most, spare, 0.05 if seed % 2 else 0.0, share=seed > 3)
    if seed % 3 == 2:  # children of the same parents: their last blocks are shared too
        parent = [rng.randrange(max(1, n_seqs // 3)) for _ in range(n_seqs)]
        table, length = ref.reorder(table, length, parent)
    if seed in (4, 5, 6):  # drafts were rejected: rows go to blocks that others still read
        length = [max(0, x - rng.randint(0, 2 * block)) for x in length]
    rows = [rng.choice([0, 1, 1, rng.randint(0, rows_most)]) for _ in range(n_seqs)]
    if seed == 7:  # rows that go on behind the table
        rows[-1] = most + 5 * block
    if refused(ref):
        return
    pool, t = device_pool(ref), i32(table)
    pairs, missing = F.floe_kv_reserve(pool, t, i32(length), cu_of(rows))
    want_pairs, want_missing = ref.reserve(table, length, rows)
    same(pool, t, ref, table)
    assert pairs.tolist() == want_pairs and missing.tolist() == [want_missing]
    # again: nothing is left to do but what was missing
    before = t.clone()
    pairs, again = F.floe_kv_reserve(pool, t, i32(length), cu_of(rows))
    assert again.tolist() == [want_missing] and (want_missing or (torch.equal(before, t) and bool((pairs == -1).all())))


def test_reserve_gives_what_was_missing_when_pages_are_free_again():
    ref = Pool(6, 32)
    table, length = [[0, 1, -1, -1], [2, 3, -1, -1], [4, -1, -1, -1]], [64, 64, 20]
    ref.count(table)
    pool, t = device_pool(ref), i32(table)
    rows = [40, 1, 1]
    _, missing = F.floe_kv_reserve(pool, t, i32(length), cu_of(rows))
    assert missing.tolist() == [2] and t.tolist() == [[0, 1, 5, -1], [2, 3, -1, -1], [4, -1, -1, -1]]
    F.floe_kv_trim(pool, t, i32([64 + 32, 64, 0]))
    assert pool.refs.tolist() == [1, 1, 1, 1, 0, 1]
    _, missing = F.floe_kv_reserve(pool, t, i32(length), cu_of([32, 1, 0]))
    assert missing.tolist() == [0] and t.tolist() == [[0, 1, 5, -1], [2, 3, 4, -1], [-1, -1, -1, -1]]


@pytest.mark.parametrize("seed", range(4))
@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (1, 1), (31, 4), (33, 32), (64, 33), (100, 5), (700, 64), (1 << 30, 3), (5, 1 << 30)])
def test_trim(seed, window, sinks):
    ref, table, length, rng = state(seed, 30, 32, 600, 3, 0.1 if seed % 2 else 0.0, share=seed > 1)
    length = [rng.choice([n, n, 0, max(0, n - rng.randint(0, 100)), -5]) for n in length]  # finished ones, rejected drafts
    pool, t = device_pool(ref), i32(table)
    F.floe_kv_trim(pool, t, i32(length), window=window, sinks=sinks)
    ref.trim(table, length, window, sinks)
    same(pool, t, ref, table)


@pytest.mark.parametrize("seed", range(4))
@pytest.mark.parametrize("n_seqs,block,most,spare,moves", [(1, 32, 40, 0, 3), (20, 32, 500, 60, 1000), (20, 32, 500, 60, 7), (90, 64, 2900, 500, None), (4, 32, 60, 3000, None),
                                                           (3, 32, 70, 5, 0)])
def test_compact(seed, n_seqs, block, most, spare, moves):
    ref, table, length, rng = state(seed, n_seqs, block, most, spare, 0.05, share=seed % 2)
    gone = [n if rng.random() < 0.6 else 0 for n in length]
    if refused(ref):
        return
    pool, t = device_pool(ref), i32(table)
    F.floe_kv_trim(pool, t, i32(gone))
    ref.trim(table, gone, 0, 0)
    pairs, where = F.floe_kv_compact(pool, t, moves)
    want_pairs, want_where = ref.compact(table, ref.n if moves is None else moves)
    same(pool, t, ref, table)
    assert pairs.tolist() == want_pairs and where.tolist() == want_where


@pytest.mark.parametrize("fmt", [F.KV_INT8, F.KV_E4M3])
@pytest.mark.parametrize("heads,dim,block,layers", [(1, 64, 32, 1), (3, 192, 128, 2), (8, 128, 64, 5), (2, 64, 32, 67)])
def test_copied_pages_are_the_same_bytes_and_the_others_stay(fmt, heads, dim, block, layers):
    n = 9
    g = torch.Generator(device=DEV).manual_seed(1)
    caches = []
    for _ in range(layers):
        codes = [torch.randint(0, 256, (n, heads, block, dim), generator=g, device=DEV, dtype=torch.uint8) for _ in range(2)]
        scales = [torch.randint(-2 ** 31, 2 ** 31 - 1, (n, heads), generator=g, device=DEV, dtype=torch.int32).view(torch.float32) for _ in range(2)]
        caches.append(F.KVCache(n, heads, dim, block, fmt, tensors=(*codes, *scales)))
    want = [[t.clone() for t in (c.k, c.v, c.k_scale.view(torch.int32), c.v_scale.view(torch.int32))] for c in caches]
    pairs = [[0, 5], [0, 3], [-1, 2], [8, -1], [n, 1], [1, n], [4, 4], [7, 6], [1 << 30, 1 << 30]]
    for a, b in ((0, 5), (0, 3), (7, 6)):
        for layer in want:
            for t in layer:
                t[b] = t[a]
    F.floe_kv_copy_pages(caches if layers > 1 else caches[0], i32(pairs))
    torch.cuda.synchronize()
    for c, layer in zip(caches, want):
        for t, w in zip((c.k, c.v, c.k_scale.view(torch.int32), c.v_scale.view(torch.int32)), layer):
            assert torch.equal(t, w)


@pytest.mark.parametrize("seed", range(3))
def test_a_long_run_of_calls_keeps_counts_and_tables_together(seed):
    """Steps of a server: forks, appends, windows, ends and packing in turn, with the counts formed anew from the table after each."""
    rng = random.Random(seed)
    P, n_pages, width, n = 32, 400, 40, 12
    ref = Pool(n_pages, P)
    table, length = [[-1] * width for _ in range(n)], [0] * n
    pool, t, ln = device_pool(ref), i32(table), i32(length)
    for step in range(40):
        what = rng.choice(["append", "append", "fork", "trim", "compact", "end"])
        if what == "append":
            rows = [rng.choice([1, 1, 30, 70]) if x < (width - 3) * P else 0 for x in length]
            pairs, missing = F.floe_kv_reserve(pool, t, ln, cu_of(rows))
            want = ref.reserve(table, length, rows)
            assert pairs.tolist() == want[0] and missing.item() == want[1] == 0, step
            length = [a + b for a, b in zip(length, rows)]
        elif what == "fork":
            parent = [rng.randrange(-1, n) for _ in range(n)]
            t, ln = F.floe_kv_reorder(pool, t, ln, i32(parent))
            table, length = ref.reorder(table, length, parent)
            assert ln.tolist() == length
        elif what == "compact":
            F.floe_kv_compact(pool, t, 25)
            ref.compact(table, 25)
        else:
            if what == "end":
                length = [x if rng.random() < 0.7 else 0 for x in length]
            window, sinks = (100, 5) if what == "trim" else (0, 0)
            F.floe_kv_trim(pool, t, i32(length), window=window, sinks=sinks)
            ref.trim(table, length, window, sinks)
        ln = i32(length)
        same(pool, t, ref, table)
        assert Pool(n_pages, P).count(table).refs == ref.refs, (step, what)


def test_calls_of_nothing():
    pool = F.KVPool(4, 32)
    none, empty = torch.empty((0, 3), dtype=torch.int32, device=DEV), torch.empty((0,), dtype=torch.int32, device=DEV)
    t, ln = F.floe_kv_reorder(pool, none, empty, i32([0, -1]))
    assert t.tolist() == [[-1] * 3] * 2 and ln.tolist() == [0, 0]
    t, ln = F.floe_kv_reorder(pool, i32([[0, 1, -1]]), i32([40]), empty)
    assert t.shape == (0, 3) and pool.refs.tolist() == [-1, -1, 0, 0]  # (that table was never counted)
    pool.refs.zero_()
    pairs, missing = F.floe_kv_reserve(pool, none, empty, i32([0]))
    assert pairs.shape == (0, 2) and missing.tolist() == [0]
    pairs, missing = F.floe_kv_reserve(pool, torch.empty((2, 0), dtype=torch.int32, device=DEV), i32([0, 5]), i32([0, 1, 1]))
    assert pairs.tolist() == [[-1, -1]] * 2 and missing.tolist() == [1]
    F.floe_kv_trim(pool, none, empty)
    pairs, where = F.floe_kv_compact(pool, none, 2)
    assert pairs.tolist() == [[-1, -1]] * 2 and where.tolist() == [0, 1, 2, 3]
    F.floe_kv_copy_pages([], pairs)
    t, ln = F.floe_kv_reorder(pool, torch.empty((2, 0), dtype=torch.int32, device=DEV), i32([3, 4]), i32([1, 1, 0]))
    assert t.shape == (3, 0) and ln.tolist() == [4, 4, 3]


def test_a_large_pool_of_which_the_last_pages_are_free():
    n = 200_003
    refs = torch.ones((n,), dtype=torch.int32, device=DEV)
    free = [n - 1, n - 2, n - 3, 150_000, 5]
    refs[i32(free).long()] = 0
    pool, t = F.KVPool(n, 64, refs=refs), torch.full((4, 3), -1, dtype=torch.int32, device=DEV)
    _, missing = F.floe_kv_reserve(pool, t, i32([0, 0, 64, 0]), cu_of([64, 65, 1, 64]))
    assert missing.item() == 0 and t.tolist() == [[5, -1, -1], [150_000, n - 3, -1], [-1, n - 2, -1], [n - 1, -1, -1]]
    F.floe_kv_trim(pool, t, i32([0, 64, 128, 64]))
    pairs, where = F.floe_kv_compact(pool, t, 3)
    assert pairs.tolist() == [[n - 1, 5], [n - 2, n - 3], [-1, -1]]
    assert t.tolist() == [[-1, -1, -1], [150_000, -1, -1], [-1, n - 3, -1], [5, -1, -1]] and int(where[n - 1]) == 5
    assert int(pool.refs.sum()) == n - 2 and pool.refs[n - 2:].tolist() == [0, 0]


def test_a_captured_step_hands_out_the_same_pages_as_eager_ones():
    P, n = 32, 6
    ref = Pool(90, P)
    table, length = [[-1] * 20 for _ in range(n)], [0] * n
    pool = device_pool(ref)
    t, ln, other, other_ln = i32(table), i32(length), torch.empty((n, 20), dtype=torch.int32, device=DEV), torch.empty((n,), dtype=torch.int32, device=DEV)
    cu, parent = cu_of([7] * n), i32([0, 0, 1, 3, 3, 3])
    pairs, missing = torch.empty((n, 2), dtype=torch.int32, device=DEV), torch.empty((1,), dtype=torch.int32, device=DEV)

    def step():
        F.floe_kv_reserve(pool, t, ln, cu, pairs=pairs, missing=missing)
        ln.add_(7)
        F.floe_kv_reorder(pool, t, ln, parent, table_out=other, length_out=other_ln)
        t.copy_(other)
        ln.copy_(other_ln)
        F.floe_kv_trim(pool, t, ln, window=50, sinks=3)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    def model():
        nonlocal table, length
        want = ref.reserve(table, length, [7] * n)
        table, length = ref.reorder(table, [x + 7 for x in length], parent.tolist())
        ref.trim(table, length, 50, 3)
        return want
    model()
    for i in range(12):
        graph.replay() if i % 4 != 3 else step()
        want = model()
        same(pool, t, ref, table)
        assert pairs.tolist() == want[0] and missing.item() == want[1] == 0 and ln.tolist() == length


def test_two_streams_with_pools_of_their_own():
    streams = [torch.cuda.Stream() for _ in range(2)]
    refs, pools, tables = [], [], []
    for k in range(2):
        ref, table, length, rng = state(20 + k, 50, 32, 300, 200)
        refs.append((ref, table, length))
        pools.append(device_pool(ref))
        tables.append((i32(table), i32(length), cu_of([3] * 50)))
    torch.cuda.synchronize()
    for _ in range(5):
        for st, pool, (t, ln, cu) in zip(streams, pools, tables):
            F.floe_kv_reserve(pool, t, ln, cu, stream=st)
            with torch.cuda.stream(st):
                ln.add_(3)
    torch.cuda.synchronize()
    for (ref, table, length), pool, (t, ln, _) in zip(refs, pools, tables):
        for _ in range(5):
            ref.reserve(table, length, [3] * 50)
            length = [x + 3 for x in length]
        same(pool, t, ref, table)


@pytest.mark.parametrize("n_seqs,rows", [(40, 1200), (1024, 1), (1025, 1), (1024, 33), (16, 2048), (16, 2049), (2, 16384)])
@pytest.mark.parametrize("shared", [False, True])
def test_reserve_on_both_sides_of_what_a_workgroup_keeps_in_registers(n_seqs, rows, shared):
    """Up to 1024 sequences with up to 1024 blocks in all, and more of either; blocks that are begun, shared by some or by all of their writers."""
    P, width = 32, -(-(rows + 60) // 32) + 1
    length = [(13 * s) % 60 for s in range(n_seqs)]
    table, page = [[-1] * width for _ in range(n_seqs)], 0
    for s in range(n_seqs):
        if shared and s % 3:
            length[s], table[s] = length[s - 1], list(table[s - 1])
            continue
        for b in range(-(-length[s] // P)):
            table[s][b] = page
            page += 1
    ref = Pool(page + n_seqs * (rows // P + 2), P).count(table)
    count = [rows if not shared or s % 5 else 0 for s in range(n_seqs)]
    pool, t = device_pool(ref), i32(table)
    pairs, missing = F.floe_kv_reserve(pool, t, i32(length), cu_of(count))
    want = ref.reserve(table, length, count)
    same(pool, t, ref, table)
    assert pairs.tolist() == want[0] and missing.item() == want[1] == 0


@pytest.mark.parametrize("n_seqs,block,most,spare,moves", [(20, 32, 500, 9000, None), (700, 32, 400, 50, None), (700, 32, 400, 50, 77), (30, 32, 300, 7800, 3)])
def test_compact_on_both_sides_of_what_one_workgroup_takes(n_seqs, block, most, spare, moves):
    ref, table, length, rng = state(9, n_seqs, block, most, spare, 0.02)
    gone = [n if rng.random() < 0.5 else 0 for n in length]
    pool, t = device_pool(ref), i32(table)
    F.floe_kv_trim(pool, t, i32(gone))
    ref.trim(table, gone, 0, 0)
    moves = 400 if moves is None else moves
    pairs, where = F.floe_kv_compact(pool, t, moves)
    want_pairs, want_where = ref.compact(table, moves)
    same(pool, t, ref, table)
    assert pairs.tolist() == want_pairs and where.tolist() == want_where


def test_pages_that_lie_behind_32_bits_of_bytes():
    n, heads, dim, block = 70_000, 8, 128, 64
    cache = F.KVCache(n, heads, dim, block)
    g = torch.Generator(device=DEV).manual_seed(5)
    for t in (cache.k, cache.v):
        t[n - 2].copy_(torch.randint(0, 256, t[0].shape, generator=g, device=DEV, dtype=torch.uint8))
        t[3].copy_(torch.randint(0, 256, t[0].shape, generator=g, device=DEV, dtype=torch.uint8))
        t[n - 1].zero_()
        t[5].zero_()
    cache.k_scale[n - 2], cache.v_scale[n - 2] = 2.0, 3.0
    F.floe_kv_copy_pages(cache, i32([[n - 2, 5], [3, n - 1]]))
    torch.cuda.synchronize()
    for t in (cache.k, cache.v):
        assert torch.equal(t[5], t[n - 2]) and torch.equal(t[n - 1], t[3]) and int(t[5].sum()) > 0
    assert bool((cache.k_scale[5] == 2.0).all()) and bool((cache.v_scale[5] == 3.0).all())


@pytest.mark.parametrize("spare", [60, 9000])
def test_pages_that_the_caller_holds_are_followed_through_a_packing(spare):
    """Counts without a table entry: the lowest pages stay, a high one moves with its bytes to where the map says, and no reserve hands any of them out."""
    ref, table, length, rng = state(3, 12, 32, 300, spare)
    low, high = [0, 1, 2], [ref.n - 1, ref.n - 7]
    pages = iter([p for p in range(3, ref.n) if p not in high])
    table = [[next(pages) * 3 // 2 + 3 if e >= 0 else -1 for e in row] for row in table]  # (some free ones between)
    ref.count(table)
    for p in low + high:
        assert ref.refs[p] == 0
        ref.refs[p] = 1
    cache = F.KVCache(ref.n, 1, 64, 32)
    for t in (cache.k, cache.v):
        t.copy_(torch.randint(0, 256, t.shape, generator=torch.Generator(device=DEV).manual_seed(1), device=DEV, dtype=torch.uint8))
    held = [cache.k[p].clone() for p in low + high]
    pool, t = device_pool(ref), i32(table)
    pairs, where = F.floe_kv_compact(pool, t, 400)
    F.floe_kv_copy_pages(cache, pairs)
    want = ref.compact(table, 400)
    same(pool, t, ref, table)
    assert pairs.tolist() == want[0] and where.tolist() == want[1]
    now = [int(where[p]) for p in low + high]
    assert now[:3] == low and now[3] != high[0] and now[4] != high[1]
    assert all(torch.equal(cache.k[p], b) for p, b in zip(now, held))
    n = 40
    wide = torch.full((1, n), -1, dtype=torch.int32, device=DEV)
    _, missing = F.floe_kv_reserve(pool, wide, i32([0]), cu_of([32 * n]))
    assert missing.item() == 0 and not set(now) & set(wide[0].tolist())
