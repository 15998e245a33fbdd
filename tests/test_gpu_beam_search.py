"""Selection, tables, pages, copies, appends and attention together: the example's beam search, and streams that give their pages back."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu
DEV = "cuda"


def names_of(pool, table):
    t = table[(table >= 0) & (table < pool.n_pages)].long()
    return torch.bincount(t, minlength=pool.n_pages).int()


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("groups,beams", [(1, 1), (2, 4), (3, 7)])
def test_the_example_runs_captured(fmt, groups, beams):
    import beam_search
    search = beam_search.main(tokens=30, groups=groups, beams=beams, fmt=fmt, verbose=False)
    assert int(search.missing) == 0 and int(search.at) == 30
    assert search.length.tolist() == [45 + 90 * (i // beams) + 29 for i in range(groups * beams)]
    assert torch.equal(search.pool.refs, names_of(search.pool, search.table))
    score = search.score
    assert bool(torch.isfinite(score).all()) and bool((score[:, :-1] >= score[:, 1:]).all())
    rows = search.sequences()
    for g in range(groups):  # beams of a group are different continuations
        mine = [tuple(r) for r in rows[g * beams:(g + 1) * beams]]
        assert len(set(mine)) == beams and all(len(r) == 30 for r in mine)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_every_beam_holds_the_cache_of_its_own_history(fmt, monkeypatch):
    """The rows that each step appended, followed back over the parents and appended one by one to a cache of their own, give the codes and
    scales of the beam bit for bit: what was shared, copied on write and handed out again is nobody else's."""
    import beam_search
    F = beam_search.F
    kept, append = [], F.floe_kv_append

    def kept_append(cache, k, v, cu, before, table, most, q, rope):
        kept.append((k.clone(), v.clone(), rope))
        return append(cache, k, v, cu, before, table, most, q=q, rope=rope)
    monkeypatch.setattr(F, "floe_kv_append", kept_append)
    groups, beams, tokens = 2, 5, 25
    search = beam_search.main(tokens=tokens, groups=groups, beams=beams, fmt=fmt, captured=False, verbose=False)
    assert len(kept) == tokens and int(search.missing) == 0
    cache, parents, P = search.block.cache, search.parents.tolist(), search.block.cache.block
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    prompts = [45 + 90 * s for s in range(groups)]
    for beam in range(groups * beams):
        # the row of each step that this beam descends from: step t's rows are the beams after selection t
        rows, at = [], beam
        for t in reversed(range(tokens)):
            at = parents[t][at]
            rows.append(at)
        rows = rows[::-1]  # rows[0]: the prompt's group, rows[t]: the row of append t
        group = rows[0]
        n = -(-(prompts[group] + tokens - 1) // P)
        alone, table = F.KVCache(n, cache.kv_heads, cache.head_dim, P, cache.fmt), torch.arange(n, dtype=torch.int32, device=DEV)[None]
        lo = sum(prompts[:group])
        k, v, rope = kept[0]
        append(alone, k[lo:lo + prompts[group]], v[lo:lo + prompts[group]], i32([0, prompts[group]]), i32([0]), table, prompts[group], rope=rope)
        for t in range(1, tokens):
            k, v, rope = kept[t]
            append(alone, k[rows[t]:rows[t] + 1], v[rows[t]:rows[t] + 1], i32([0, 1]), i32([prompts[group] + t - 1]), table, 1, rope=rope)
        length = prompts[group] + tokens - 1
        assert int(search.length[beam]) == length
        got = F.floe_kv_gather(cache, i32([0]), i32([0, length]), search.table[beam:beam + 1].contiguous(), length, length)
        want = F.floe_kv_gather(alone, i32([0]), i32([0, length]), table, length, length)
        pages = search.table[beam, :n].long()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), beam
        assert torch.equal(cache.k_scale[pages], alone.k_scale) and torch.equal(cache.v_scale[pages], alone.v_scale), beam


@pytest.mark.parametrize("fmt", [0, 1])
def test_streams_that_give_their_pages_back_see_what_they_would_see_with_all_of_them(fmt):
    """Appends and attention with a window and first tokens over a small pool, pages given back and handed out again after every step, pages
    packed now and then, beside a cache that keeps everything: the outputs are the same bit for bit."""
    import paper_2505_05950_amd as F
    g = torch.Generator(device=DEV).manual_seed(4)
    B, P, heads, dim, qh, window, sinks, steps = 5, 32, 2, 64, 4, 70, 9, 60
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    width = 20
    small, large = F.KVCache(40, heads, dim, P, fmt), F.KVCache(B * width, heads, dim, P, fmt)
    small.k_scale.fill_(float("nan"))  # (what a page held before is nobody's)
    pool, table = F.KVPool(40, P), torch.full((B, width), -1, dtype=torch.int32, device=DEV)
    whole = torch.arange(B * width, dtype=torch.int32, device=DEV).view(B, width)
    length, most_used = i32([0] * B), 0
    for step in range(steps):
        new = [(3 * step + 5 * s) % 4 * 3 + (step == 0) * 40 for s in range(B)]
        cu = i32([sum(new[:s]) for s in range(B + 1)])
        rows, most = sum(new), max(new)
        k, v, q = (torch.randn((rows, h, dim), generator=g, device=DEV).half() for h in (heads, heads, qh))
        pairs, missing = F.floe_kv_reserve(pool, table, length, cu)
        assert int(missing) == 0 and bool((pairs == -1).all())
        F.floe_kv_append(small, k, v, cu, length, table, most)
        F.floe_kv_append(large, k, v, cu, length, whole, most)
        length = length + i32(new)
        out = [F.floe_kv_attention(c, q, cu, length, t, most, width * P, window=window, sinks=sinks, want_lse=True) for c, t in ((small, table), (large, whole))]
        assert torch.equal(out[0][0], out[1][0]) and torch.equal(out[0][1], out[1][1]), step
        F.floe_kv_trim(pool, table, length, window=window, sinks=sinks)
        if step % 7 == 6:
            pairs, _ = F.floe_kv_compact(pool, table, 5)
            F.floe_kv_copy_pages(small, pairs)
        assert torch.equal(pool.refs, names_of(pool, table))
        most_used = max(most_used, int((pool.refs > 0).sum()))
    assert int(length.max()) > 200 and most_used <= B * (-(-sinks // P) + window // P + 2)


@pytest.mark.parametrize("fmt", [0, 1])
def test_a_reserve_that_missed_pages_is_repeated_when_some_are_free(fmt):
    """Two sequences share a begun block, a third needs a page that is not there: what the first call named is copied, a fourth sequence ends,
    and the call is made again.  Each sequence then reads what a cache of its own holds, bit for bit."""
    import paper_2505_05950_amd as F
    P, heads, dim = 32, 2, 64
    g = torch.Generator(device=DEV).manual_seed(6)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    new = lambda n: [torch.randn((n, heads, dim), generator=g, device=DEV).half() for _ in range(2)]  # noqa: E731
    cache, pool = F.KVCache(5, heads, dim, P, fmt), F.KVPool(5, P)
    prompt, other, cu = new(20), new(64), i32([0, 20, 84, 94])
    k, v = (torch.cat(x) for x in zip(prompt, other, new(10)))
    t, before = torch.full((3, 4), -1, dtype=torch.int32, device=DEV), i32([0, 0, 0])
    F.floe_kv_reserve(pool, t, before, cu)
    F.floe_kv_append(cache, k, v, cu, before, t, 64)
    t, length = F.floe_kv_reorder(pool, t, i32([20, 64, 10]), i32([0, 0, 1, 2]))
    k, v = new(3)
    pairs, missing = F.floe_kv_reserve(pool, t, length, i32([0, 1, 2, 3, 3]))
    F.floe_kv_copy_pages(cache, pairs)
    assert missing.item() == 1 and pairs.tolist() == [[-1, -1], [0, 4], [-1, -1], [-1, -1]]
    F.floe_kv_trim(pool, t, i32([20, 20, 64, 0]))
    length = i32([20, 20, 64, 0])
    pairs, missing = F.floe_kv_reserve(pool, t, length, i32([0, 1, 2, 3, 3]))
    F.floe_kv_copy_pages(cache, pairs)
    assert missing.item() == 0 and bool((pairs == -1).all()) and t[:, 0].tolist() == [0, 4, 1, -1] and t[2, 2].item() == 3
    F.floe_kv_append(cache, k, v, i32([0, 1, 2, 3, 3]), length, t, 1)
    for s, (old_k, old_v) in enumerate((prompt, prompt, other)):
        alone, table, n = F.KVCache(3, heads, dim, P, fmt), i32([[0, 1, 2]]), old_k.shape[0]
        F.floe_kv_append(alone, old_k, old_v, i32([0, n]), i32([0]), table, n)
        F.floe_kv_append(alone, k[s:s + 1], v[s:s + 1], i32([0, 1]), i32([n]), table, 1)
        got = F.floe_kv_gather(cache, i32([0]), i32([0, n + 1]), t[s:s + 1].contiguous(), n + 1, n + 1)
        want = F.floe_kv_gather(alone, i32([0]), i32([0, n + 1]), table, n + 1, n + 1)
        assert all(torch.equal(a, b) for a, b in zip(got, want)), s


@pytest.mark.parametrize("sinks", [0, 5])
@pytest.mark.parametrize("fmt", [0, 1])
def test_windows_of_one_token_keep_the_block_that_is_begun(fmt, sinks):
    """Attention with a window of 1, pages given back with a window of 2: the scale of the begun block stays, and the outputs are those of a cache that
    keeps everything.  Pages that nobody has used hold NaN scales: an append to one of them that it takes for begun would show."""
    import paper_2505_05950_amd as F
    P, heads, dim, B, steps = 32, 2, 64, 3, 80
    g = torch.Generator(device=DEV).manual_seed(8)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    small, large = F.KVCache(40, heads, dim, P, fmt), F.KVCache(B * 5, heads, dim, P, fmt)
    small.k_scale.fill_(float("nan"))
    small.v_scale.fill_(float("nan"))
    pool, table, whole = F.KVPool(40, P), torch.full((B, 5), -1, dtype=torch.int32, device=DEV), torch.arange(B * 5, dtype=torch.int32, device=DEV).view(B, 5)
    length, cu = i32([0] * B), i32([0, 1, 2, 3])
    for step in range(steps):
        k, v, q = (torch.randn((B, h, dim), generator=g, device=DEV).half() * (1 + step % 7) for h in (heads, heads, 4))
        pairs, missing = F.floe_kv_reserve(pool, table, length, cu)
        assert int(missing) == 0 and bool((pairs == -1).all())
        for c, t in ((small, table), (large, whole)):
            F.floe_kv_append(c, k, v, cu, length, t, 1)
        length = length + 1
        out = [F.floe_kv_attention(c, q, cu, length, t, 1, 5 * P, window=1, sinks=sinks) for c, t in ((small, table), (large, whole))]
        assert torch.equal(*out) and bool(torch.isfinite(out[0]).all()), step
        F.floe_kv_trim(pool, table, length, window=2, sinks=sinks)
        assert int((pool.refs > 0).sum()) <= B * (2 if sinks else 1), step
