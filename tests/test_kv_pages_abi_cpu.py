"""Refusals of the calls on pages, of attention with first tokens and of the beam selection: every bad argument comes back as its status before
anything is enqueued (the pointers are made up and never followed), and the binding refuses tensors that do not fit."""
import ctypes as C
import os

import pytest
import torch

import paper_2505_05950_amd as F
from kv_pool_reference import Pool
from paper_2505_05950_amd import binding as B
from test_kv_abi_cpu import EHIP, EINVAL, ESHAPE, EUNSUPPORTED, EWORKSPACE, P, attn, cache, seqs

BIG = 1 << 40  # addresses this far apart do not overlap


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.lib_path()):
        from paper_2505_05950_amd import build
        build.build()
    return B.load()


def pool(n_pages=100, block=64, refs=P):
    return B._KvPool(n_pages, block, refs)


def reorder(lib, p=None, table=P, length=P, n=2, blocks=3, parent=P, table_out=BIG, length_out=2 * BIG, n_out=2):
    return lib.floe_kv_reorder(p or pool(), table, length, n, blocks, parent, table_out, length_out, n_out, None)


def reserve(lib, p=None, table=P, length=P, cu=P, n=2, blocks=3, pairs=P, missing=P, ws=P, size=BIG):
    return lib.floe_kv_reserve(p or pool(), table, length, cu, n, blocks, pairs, missing, ws, size, None)


def trim(lib, p=None, table=P, length=P, n=2, blocks=3, sinks=0, window=0):
    return lib.floe_kv_trim(p or pool(), table, length, n, blocks, sinks, window, None)


def compact(lib, p=None, table=P, n=2, blocks=3, pairs=P, n_pairs=5, page_map=P, ws=P, size=BIG):
    return lib.floe_kv_compact(p or pool(), table, n, blocks, pairs, n_pairs, page_map, ws, size, None)


@pytest.mark.parametrize("change,code", [(dict(n_pages=0), EINVAL), (dict(n_pages=-1), EINVAL), (dict(refs=None), EINVAL), (dict(refs=P + 4), EINVAL),
                                         (dict(block=16), EUNSUPPORTED), (dict(block=0), EUNSUPPORTED), (dict(n_pages=(1 << 24) + 1), EUNSUPPORTED)])
def test_a_bad_pool_is_refused_by_every_call(lib, change, code):
    for call in (reorder, reserve, trim, compact):
        assert call(lib, pool(**change)) == code
    assert lib.floe_kv_reserve_workspace_bytes(pool(**change)) == 0 and lib.floe_kv_compact_workspace_bytes(pool(**change), 3) == 0


@pytest.mark.parametrize("change,code", [(dict(n=-1), EINVAL), (dict(blocks=-1), EINVAL), (dict(n=65536), EUNSUPPORTED), (dict(blocks=(1 << 23) + 1), EUNSUPPORTED),
                                         (dict(n=1 << 12, blocks=1 << 20), EUNSUPPORTED), (dict(table=None), EINVAL), (dict(table=P + 2), EINVAL)])
def test_a_bad_table_is_refused_by_every_call(lib, change, code):
    for call in (reorder, reserve, trim, compact):
        assert call(lib, **change) == code, call


def test_reorder_refuses(lib):
    assert reorder(lib, parent=None) == EINVAL and reorder(lib, length=None) == EINVAL and reorder(lib, table_out=None) == EINVAL and reorder(lib, length_out=None) == EINVAL
    assert reorder(lib, parent=P + 1) == EINVAL and reorder(lib, length_out=BIG + 2) == EINVAL and reorder(lib, n_out=-1) == EINVAL and reorder(lib, n_out=65536) == EUNSUPPORTED
    # outputs that overlap what is read: by one entry, from either side, and the array itself
    assert reorder(lib, table=BIG + 20, table_out=BIG) == EINVAL and reorder(lib, table=BIG, table_out=BIG + 20) == EINVAL and reorder(lib, table=BIG) == EINVAL
    assert reorder(lib, length=2 * BIG) == EINVAL and reorder(lib, parent=2 * BIG + 4) == EINVAL and reorder(lib, parent=BIG + 20) == EINVAL
    assert reorder(lib, n=0, n_out=0, table=None, length=None, parent=None, table_out=None, length_out=None) == 0
    if not torch.cuda.is_available():
        assert reorder(lib, table=BIG + 24, table_out=BIG) == EHIP and reorder(lib) == EHIP and reorder(lib, n=0, table=None, length=None) == EHIP


def test_reserve_refuses(lib):
    need = lib.floe_kv_reserve_workspace_bytes(pool())
    assert need > 0 and reserve(lib, size=need - 1) == EWORKSPACE
    for change in (dict(length=None), dict(cu=None), dict(pairs=None), dict(missing=None), dict(ws=None), dict(length=P + 1), dict(cu=P + 2), dict(pairs=P + 1),
                   dict(missing=P + 2), dict(ws=P + 128)):
        assert reserve(lib, **change) == EINVAL, change
    if not torch.cuda.is_available():
        assert reserve(lib, size=need) == EHIP and reserve(lib, n=0, table=None, length=None, cu=None, pairs=None) == EHIP  # (missing is still written)


def test_trim_refuses(lib):
    assert trim(lib, length=None) == EINVAL and trim(lib, length=P + 2) == EINVAL and trim(lib, sinks=-1) == EINVAL and trim(lib, window=-1) == EINVAL
    assert trim(lib, sinks=(1 << 30) + 1) == EUNSUPPORTED and trim(lib, window=(1 << 30) + 1) == EUNSUPPORTED
    assert trim(lib, n=0, table=None, length=None) == 0 and trim(lib, blocks=0, table=None) == 0


def test_compact_refuses(lib):
    need = lib.floe_kv_compact_workspace_bytes(pool(), 5)
    assert need > 0 and compact(lib, size=need - 1) == EWORKSPACE and lib.floe_kv_compact_workspace_bytes(pool(), -1) == 0
    for change in (dict(pairs=None), dict(pairs=P + 2), dict(n_pairs=-1), dict(page_map=None), dict(page_map=P + 1), dict(ws=None), dict(ws=P + 64)):
        assert compact(lib, **change) == EINVAL, change
    # more moves than there are pages take no more scratch
    assert lib.floe_kv_compact_workspace_bytes(pool(), 100) == lib.floe_kv_compact_workspace_bytes(pool(), 1 << 30)


def test_copy_refuses(lib):
    def call(*caches, n=None, pairs=P, n_pairs=2):
        packed = b"".join(bytes(c) for c in caches)
        return lib.floe_kv_copy_pages(packed or None, len(caches) if n is None else n, pairs, n_pairs, None)
    assert call(cache(), n=-1) == EINVAL and call(cache(), n_pairs=-1) == EINVAL and call(n=1) == EINVAL
    assert call(cache(), pairs=None) == EINVAL and call(cache(), pairs=P + 2) == EINVAL
    assert call(cache(), cache(k=None)) == EINVAL and call(cache(), cache(head_dim=96)) == EUNSUPPORTED
    for other in (dict(n_pages=5), dict(kv_heads=1), dict(head_dim=64), dict(block=32), dict(fmt=1)):
        assert call(cache(), cache(**other)) == ESHAPE, other
    assert call(cache(n_pages=1 << 20, kv_heads=256, head_dim=256, block=128), n_pairs=1 << 20) == EUNSUPPORTED
    assert call(pairs=None) == 0 and call(cache(), pairs=None, n_pairs=0) == 0


def test_attention_with_first_tokens_refuses(lib):
    need = lib.floe_kv_attention_sinks_workspace_bytes(cache(), seqs(), attn(window=10), 4)
    def call(sinks, a=None, ws=P, n=1 << 40):
        return lib.floe_kv_attention_sinks(cache(), seqs(), a or attn(window=10), sinks, P, 1024, P, None, ws, n, None)
    assert need > 0 and call(4, n=need - 1) == EWORKSPACE
    assert call(-1) == EINVAL and call((1 << 30) + 1) == EUNSUPPORTED and call(-1, attn()) == EINVAL
    assert lib.floe_kv_attention_sinks_workspace_bytes(cache(), seqs(), attn(window=10), -1) == 0
    for a in (attn(), attn(window=7), attn(window=60, max_len=100000)):
        assert lib.floe_kv_attention_sinks_workspace_bytes(cache(), seqs(), a, 0) == lib.floe_kv_attention_workspace_bytes(cache(), seqs(), a)
    assert lib.floe_kv_attention_sinks_workspace_bytes(cache(), seqs(), attn(), 50) == lib.floe_kv_attention_workspace_bytes(cache(), seqs(), attn())


def beam(groups=2, beams=4, vocab=1000, take=4, dtype=0, eos=-1):
    return B._Beam(groups, beams, vocab, take, dtype, eos)


def test_selection_refuses(lib):
    def call(b=None, logits=P, stride=1000, score=P, done=None, so=P, parent=P, token=P, done_out=None, ws=P, n=1 << 40):
        return lib.floe_beam_select(b or beam(), logits, stride, score, done, so, parent, token, done_out, ws, n, None)
    for change, code in ((dict(groups=-1), EINVAL), (dict(beams=0), EINVAL), (dict(vocab=0), EINVAL), (dict(take=0), EINVAL), (dict(eos=-2), EINVAL), (dict(eos=1000), EINVAL),
                         (dict(take=65), EUNSUPPORTED), (dict(beams=257), EUNSUPPORTED), (dict(vocab=1 << 28), EUNSUPPORTED), (dict(groups=1 << 19), EUNSUPPORTED),
                         (dict(dtype=3), EUNSUPPORTED), (dict(dtype=-1), EUNSUPPORTED)):
        assert call(beam(**change), stride=1 << 30) == code, change
        assert lib.floe_beam_workspace_bytes(beam(**change)) == 0, change
    need = lib.floe_beam_workspace_bytes(beam())
    assert need > 0 and call(n=need - 1) == EWORKSPACE
    for change in (dict(logits=None), dict(score=None), dict(so=None), dict(parent=None), dict(token=None), dict(ws=None), dict(stride=999), dict(done=P),
                   dict(logits=P + 1), dict(score=P + 2), dict(parent=P + 1), dict(token=P + 2), dict(so=P + 3), dict(ws=P + 8), dict(b=beam(dtype=2), logits=P + 2)):
        assert call(**change) == EINVAL, change
    assert call(stride=(1 << 40) + 1) == EUNSUPPORTED and call(beam(groups=0), logits=None, ws=None) == 0 and lib.floe_beam_workspace_bytes(beam(groups=0)) == 0
    if not torch.cuda.is_available():
        assert call(n=need) == EHIP and call(beam(eos=5), done=P) == EHIP


@pytest.mark.parametrize("rows,vocab,take,dtype", [(1, 1, 1, 0), (4, 32000, 4, 0), (512, 131072, 64, 2), (1, (1 << 28) - 1, 64, 1), (1 << 20, 5, 1, 1), (3, 2049, 8, 2)])
def test_the_selection_s_workspace_stays_small_beside_the_logits(lib, rows, vocab, take, dtype):
    beams = 256 if rows == 1 << 20 else 1
    need = lib.floe_beam_workspace_bytes(beam(rows // beams, beams, vocab, take, dtype))
    assert 0 < need <= 512 + rows * (16 + 8 * take) * max(1, min(-(-vocab // 1024), 2048 // rows + 1))


def i32(*v):
    return torch.tensor(v, dtype=torch.int32)


def test_the_binding_refuses_tensors_of_the_host_before_the_library_sees_them():
    p, t, n = F.KVPool(4, 32, device="cpu"), torch.zeros((2, 3), dtype=torch.int32), i32(5, 6)
    c = F.KVCache(4, 1, 64, 32, device="cpu")
    for call in (lambda: F.floe_kv_reorder(p, t, n, n), lambda: F.floe_kv_reserve(p, t, n, i32(0, 1, 2)), lambda: F.floe_kv_trim(p, t, n), lambda: F.floe_kv_compact(p, t),
                 lambda: F.floe_kv_copy_pages([c, c], t[:, :2].contiguous()), lambda: F.floe_beam_select(torch.zeros((2, 8)), torch.zeros((1, 2)))):
        with pytest.raises(ValueError, match="GPU"):
            call()


def test_the_binding_refuses_tensors_that_do_not_fit(monkeypatch):
    for args in ((0, 32), (-3, 32)):
        with pytest.raises(ValueError):
            F.KVPool(*args, device="cpu")
    for refs in (torch.zeros(5, dtype=torch.int32), torch.zeros(4), torch.zeros(8, dtype=torch.int32)[::2], torch.zeros((4, 1), dtype=torch.int32)):
        with pytest.raises(ValueError):
            F.KVPool(4, 32, refs=refs)
    monkeypatch.setattr(B, "_launches_on", lambda *a: None)  # (the host stands in for the GPU up to the call)
    p, t, n = F.KVPool(4, 32, device="cpu"), torch.zeros((2, 3), dtype=torch.int32), i32(5, 6)
    bad_tables = (t.long(), t[0], t[:, ::2], t.float(), t[None])
    for x in bad_tables:
        for call in (lambda: F.floe_kv_reorder(p, x, n, n), lambda: F.floe_kv_reserve(p, x, n, i32(0, 1, 2)), lambda: F.floe_kv_trim(p, x, n), lambda: F.floe_kv_compact(p, x)):
            with pytest.raises(ValueError):
                call()
    for call in (lambda: F.floe_kv_reorder(p, t, i32(1), n), lambda: F.floe_kv_reorder(p, t, n, n.long()), lambda: F.floe_kv_reorder(p, t, n, n[None]),
                 lambda: F.floe_kv_reorder(p, t, n, n, table_out=torch.zeros((2, 2), dtype=torch.int32)), lambda: F.floe_kv_reorder(p, t, n, n, length_out=i32(1)),
                 lambda: F.floe_kv_reserve(p, t, n, i32(0, 1)), lambda: F.floe_kv_reserve(p, t, n, i32(0, 1, 2), pairs=torch.zeros((2, 3), dtype=torch.int32)),
                 lambda: F.floe_kv_reserve(p, t, n, i32(0, 1, 2), missing=torch.zeros(1)), lambda: F.floe_kv_trim(p, t, i32(1, 2, 3)),
                 lambda: F.floe_kv_compact(p, t, 2, pairs=torch.zeros((3, 2), dtype=torch.int32)), lambda: F.floe_kv_compact(p, t, 2, page_map=i32(1))):
        with pytest.raises(ValueError):
            call()
    c = F.KVCache(4, 1, 64, 32, device="cpu")
    for pairs in (i32(1, 2), torch.zeros((2, 3), dtype=torch.int32), torch.zeros((2, 2)), torch.zeros((2, 4), dtype=torch.int32)[:, ::2]):
        with pytest.raises(ValueError):
            F.floe_kv_copy_pages(c, pairs)
    x, s = torch.zeros((6, 8), dtype=torch.float16), torch.zeros((2, 3))
    for logits, score, more in ((x[:5], s, {}), (x.double(), s, {}), (x[None], s, {}), (x, s[0], {}), (x, s.half(), {}), (x, s.t().contiguous().t(), {}),
                                (x.t().contiguous().t(), s, {}), (x[:1].expand(6, 8), s, {}), (x, s, dict(done=torch.zeros((2, 3)))),
                                (x, s, dict(done=torch.zeros((2, 2), dtype=torch.uint8))), (x, s, dict(score_out=torch.zeros((2, 4)))),
                                (x, s, dict(parent=torch.zeros((2, 3)))), (x, s, dict(take=4, token=torch.zeros((2, 3), dtype=torch.int32))),
                                (x, s, dict(done_out=torch.zeros((2, 3), dtype=torch.int32)))):
        with pytest.raises(ValueError):
            F.floe_beam_select(logits, score, **more)


def test_a_pool_on_another_device_than_the_one_that_launches_is_refused(monkeypatch):
    p = F.KVPool(4, 32, device="cpu")
    p._device = 1
    monkeypatch.setattr(B, "_current_device", lambda: 0)
    with pytest.raises(ValueError, match="cuda:1"):
        F.floe_kv_trim(p, torch.zeros((2, 3), dtype=torch.int32), i32(1, 2))
    monkeypatch.setattr(B, "_current_device", lambda: 1)
    with pytest.raises(ValueError, match="cuda:1"):  # the pool's device launches, the table is elsewhere
        F.floe_kv_trim(p, torch.zeros((2, 3), dtype=torch.int32), i32(1, 2))


def test_the_model_of_the_pool_keeps_counts_and_tables_together():
    """The reference that the GPU is compared with: after every call its counts are those of its table, and no block that is written is shared."""
    import random
    rng = random.Random(0)
    n, P_, width, pages = 6, 32, 8, 60
    model = Pool(pages, P_)
    table, length = [[-1] * width for _ in range(n)], [0] * n
    for step in range(120):
        rows = [rng.choice([0, 1, 20]) if x < (width - 1) * P_ else 0 for x in length]
        pairs, missing = model.reserve(table, length, rows)
        assert missing == 0
        for s in range(n):
            if rows[s]:
                for b in range(length[s] // P_, (length[s] + rows[s] - 1) // P_ + 1):
                    assert sum(e == table[s][b] for row in table for e in row) == 1
        length = [a + b for a, b in zip(length, rows)]
        what = step % 3
        if what == 0:
            table, length = model.reorder(table, length, [rng.randrange(n) for _ in range(n)])
        elif what == 1:
            length = [x if rng.random() < 0.8 else 0 for x in length]
            model.trim(table, length, 70, 5)
        else:
            model.compact(table, 4)
        assert Pool(pages, P_).count(table).refs == model.refs


def test_a_selection_into_its_own_inputs_is_refused(monkeypatch):
    monkeypatch.setattr(B, "_launches_on", lambda *a: None)
    x, s, d = torch.zeros((6, 8), dtype=torch.float16), torch.zeros((2, 3)), torch.zeros((2, 3), dtype=torch.uint8)
    both = torch.zeros(9)
    for score, done, more in ((s, None, dict(score_out=s)), (s, d, dict(done_out=d)), (both[:6].view(2, 3), None, dict(score_out=both[3:].view(2, 3))),
                              (both[3:].view(2, 3), None, dict(score_out=both[:6].view(2, 3))), (s, None, dict(parent=s.view(torch.int32))),
                              (s, None, dict(take=1, token=s.view(torch.int32).flatten()[4:].view(2, 1)))):
        with pytest.raises(ValueError, match="over an input"):
            F.floe_beam_select(x, score, done=done, eos=1 if done is not None else -1, **more)


@pytest.mark.parametrize("n_pairs", [(1 << 30) + 1, (1 << 31) - 1])
def test_compact_refuses_more_pairs_than_32_bits_number(lib, n_pairs):
    """The kernels count pairs and their halves in 32 bits."""
    assert compact(lib, n_pairs=n_pairs) == EUNSUPPORTED and lib.floe_kv_compact_workspace_bytes(pool(), n_pairs) == 0
    if not torch.cuda.is_available():
        assert compact(lib, n_pairs=1 << 30) == EHIP  # (the most that is taken)


def test_a_pool_s_scratch_belongs_to_the_stream_of_the_call(monkeypatch):
    """Memory that a call on a stream uses without the caller's knowledge comes from that stream's pool: dropped with the pool, it is given out
    again in that stream's order.  One array per stream, made when the stream's first call needs it."""
    class Stream:
        def __init__(self, handle):
            self.cuda_stream = handle
    made, used = [], []
    make = lambda n, device, stream=None: made.append((stream, torch.empty((n + 256,), dtype=torch.uint8))) or made[-1][1]  # noqa: E731
    call = lambda *a: used.append(a[-3:]) or 0  # noqa: E731  (workspace, bytes, stream)
    monkeypatch.setattr(B, "_workspace", make)
    monkeypatch.setattr(B, "_launches_on", lambda *a: None)
    monkeypatch.setattr(B, "_stream", lambda stream: 7 if stream is None else stream.cuda_stream)
    monkeypatch.setattr(B, "_page_calls", lambda: (call,) * 5)
    p, t, n = F.KVPool(4, 32, device="cpu"), torch.zeros((2, 3), dtype=torch.int32), i32(5, 6)
    outs, moves = dict(pairs=torch.zeros((2, 2), dtype=torch.int32), missing=i32(0)), dict(pairs=torch.zeros((4, 2), dtype=torch.int32), page_map=i32(0, 0, 0, 0))
    one, two = Stream(11), Stream(12)
    for stream in (one, None, two, one, None):
        F.floe_kv_reserve(p, t, n, i32(0, 1, 2), **outs, stream=stream)
        F.floe_kv_compact(p, t, **moves, stream=stream)
    assert [s for s, _ in made] == [one, None, two]
    spaces = {11: made[0][1], 7: made[1][1], 12: made[2][1]}
    assert [st for _, _, st in used] == [11, 11, 7, 7, 12, 12, 11, 11, 7, 7]
    for at, size, st in used:
        assert spaces[st].data_ptr() <= at and at + size <= spaces[st].data_ptr() + spaces[st].numel() and at % 256 == 0
    own = torch.empty((4096,), dtype=torch.uint8)
    F.floe_kv_reserve(p, t, n, i32(0, 1, 2), **outs, workspace=own, stream=Stream(13))
    assert len(made) == 3 and own.data_ptr() <= used[-1][0] < own.data_ptr() + 256


def test_reorder_refuses_outputs_over_the_other_input_and_over_each_other(lib):
    """Some workgroups write both outputs while others still read the table, the lengths and the parents: no output lies over any of them."""
    # table_out (24 bytes) and length (8), length_out (8) and table (24), the two outputs
    for change in (dict(length=BIG), dict(length=BIG + 20), dict(length=BIG - 4), dict(table=2 * BIG - 20), dict(table=2 * BIG), dict(table=2 * BIG + 4),
                   dict(length_out=BIG), dict(length_out=BIG + 20), dict(length_out=BIG - 4)):
        assert reorder(lib, **change) == EINVAL, change
    if not torch.cuda.is_available():
        for change in (dict(length=BIG + 24), dict(length=BIG - 8), dict(table=2 * BIG - 24), dict(table=2 * BIG + 8), dict(length_out=BIG + 24), dict(length_out=BIG - 8)):
            assert reorder(lib, **change) == EHIP, change


def test_a_selection_whose_results_lie_over_each_other_is_refused(monkeypatch):
    monkeypatch.setattr(B, "_launches_on", lambda *a: None)
    x, s, room = torch.zeros((6, 8), dtype=torch.float16), torch.zeros((2, 3)), torch.zeros(20, dtype=torch.int32)
    part = lambda i: room[i:i + 6].view(2, 3)  # noqa: E731
    for more in (dict(parent=part(0), token=part(5)), dict(token=part(0), parent=part(5)), dict(score_out=part(3).view(torch.float32), token=part(0)),
                 dict(done_out=room.view(torch.uint8)[23:29].view(2, 3), parent=part(0)), dict(parent=part(2), token=part(2))):
        with pytest.raises(ValueError, match="over another result"):
            F.floe_beam_select(x, s, **more)


@pytest.mark.parametrize("value", [1 << 32, (1 << 32) + 3, 1 << 31, -(1 << 31) - 1, -(1 << 32)])
def test_the_binding_refuses_numbers_that_do_not_fit_the_call(monkeypatch, value):
    """ctypes cuts integers to 32 bits without a word: 2^32 first tokens would have been none."""
    monkeypatch.setattr(B, "_launches_on", lambda *a: None)
    reached = lambda *a: pytest.fail("the library was called")  # noqa: E731
    monkeypatch.setattr(B, "_page_calls", lambda: (reached,) * 5)
    monkeypatch.setattr(B, "_kv_calls", lambda: (reached,) * 4)
    monkeypatch.setattr(B, "_kv_seqs", lambda *a: b"")
    monkeypatch.setattr(B, "_stream", lambda s: 0)
    p, t, n = F.KVPool(4, 32, device="cpu"), torch.zeros((2, 3), dtype=torch.int32), i32(5, 6)
    c, q = F.KVCache(4, 1, 64, 32, device="cpu"), torch.zeros((1, 1, 64), dtype=torch.float16)
    for call in (lambda: F.floe_kv_attention(c, q, i32(0, 1), i32(1), t[:1], 1, 9, window=5, sinks=value), lambda: F.floe_kv_trim(p, t, n, sinks=value),
                 lambda: F.floe_kv_trim(p, t, n, window=value), lambda: F.floe_kv_compact(p, t, value), lambda: F.KVPool(4, value + 32 * (value > 0), refs=i32(0, 0, 0, 0))):
        with pytest.raises(ValueError, match="32 bits"):
            call()
    class Long:  # (a tensor of as many rows, as far as its sizes go)
        dtype, shape = torch.int32, (abs(value) + 2 ** 32, 3)
        is_contiguous, get_device, data_ptr, numel, dim = (lambda s: True), (lambda s: -1), (lambda s: 64), (lambda s: s.shape[0]), (lambda s: 2)
    for call in (lambda: F.floe_kv_trim(p, Long(), n), lambda: F.floe_kv_copy_pages(c, Long()), lambda: F.floe_kv_reorder(p, t, n, Long())):
        with pytest.raises(ValueError, match="32 bits"):
            call()
