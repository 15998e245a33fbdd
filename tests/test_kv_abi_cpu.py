"""Refusals of the calls on the paged 8-bit cache: every bad argument comes back as its status before anything is enqueued (the pointers
are made up and never followed), and the binding refuses tensors that do not fit."""
import ctypes as C
import os
import weakref

import pytest
import torch

import paper_2505_05950_amd as F
from paper_2505_05950_amd import binding as B

EINVAL, ESHAPE, EUNSUPPORTED, EWORKSPACE, EHIP = -1, -2, -3, -4, -5
P = 1 << 20  # an address that fits every alignment


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.lib_path()):
        from paper_2505_05950_amd import build
        build.build()
    return B.load()


def cache(n_pages=4, kv_heads=2, head_dim=128, block=64, fmt=0, dtype=0, k=P, v=P, ks=P, vs=P):
    return B._KvCache(n_pages, kv_heads, head_dim, block, fmt, dtype, k, v, ks, vs)


def seqs(n_seqs=2, n_rows=2, max_rows=1, max_blocks=3, cu=P, length=P, table=P):
    return B._KvSeqs(n_seqs, n_rows, max_rows, max_blocks, cu, length, table)


def attn(q_heads=8, causal=1, window=0, max_len=100, scale=0.1):
    return B._Attention(q_heads, causal, window, max_len, scale)


def rope(table=P, positions=None, n_positions=10, rot=128, interleaved=0):
    return B._Rope(table, positions, n_positions, rot, interleaved)


BAD_CACHES = [(dict(n_pages=0), EINVAL), (dict(kv_heads=0), EINVAL), (dict(k=None), EINVAL), (dict(v=P + 8), EINVAL), (dict(ks=None), EINVAL),
              (dict(vs=P + 2), EINVAL), (dict(head_dim=96), EUNSUPPORTED), (dict(head_dim=0), EUNSUPPORTED), (dict(head_dim=512), EUNSUPPORTED),
              (dict(block=16), EUNSUPPORTED), (dict(block=256), EUNSUPPORTED), (dict(kv_heads=257), EUNSUPPORTED), (dict(fmt=2), EUNSUPPORTED),
              (dict(dtype=2), EUNSUPPORTED), (dict(dtype=-1), EUNSUPPORTED)]
BAD_SEQS = [(dict(n_seqs=-1), EINVAL), (dict(n_rows=-1), EINVAL), (dict(max_rows=-1), EINVAL), (dict(max_blocks=0), EINVAL), (dict(cu=None), EINVAL),
            (dict(length=None), EINVAL), (dict(table=None), EINVAL), (dict(table=P + 2), EINVAL), (dict(n_seqs=65536), EUNSUPPORTED),
            (dict(n_rows=(1 << 24) + 1), EUNSUPPORTED)]


@pytest.mark.parametrize("c,s,code", [(c, {}, rc) for c, rc in BAD_CACHES] + [({}, s, rc) for s, rc in BAD_SEQS])
def test_a_bad_cache_or_batch_is_refused_by_every_call(lib, c, s, code):
    c, s = cache(**c), seqs(**s)
    assert lib.floe_kv_append(c, s, P, 256, P, 256, None, 0, 0, None, None, None) == code
    assert lib.floe_kv_gather(c, s, P, P, None) == code
    assert lib.floe_kv_attention(c, s, attn(), P, 1024, P, None, P, 1 << 40, None) == code


def test_append_refuses(lib):
    def call(k=P, ks=256, v=P, vs=256, q=None, qs=0, heads=0, out=None, r=None, s=None):
        return lib.floe_kv_append(cache(), s or seqs(), k, ks, v, vs, q, qs, heads, out, r, None)
    assert call(k=None) == EINVAL and call(v=None) == EINVAL and call(k=P + 8) == EINVAL
    assert call(ks=255) == EINVAL and call(ks=260) == EINVAL and call(vs=8) == EINVAL and call(ks=1 << 41) == EUNSUPPORTED
    assert call(r=rope(table=None)) == EINVAL and call(r=rope(table=P + 4)) == EINVAL and call(r=rope(n_positions=0)) == EINVAL
    assert call(r=rope(rot=24)) == ESHAPE and call(r=rope(rot=144)) == ESHAPE and call(r=rope(rot=0)) == EINVAL and call(r=rope(positions=P + 2)) == EINVAL
    good = dict(q=P, qs=1024, heads=8, out=P, r=rope())
    for change, rc in ((dict(r=None), EINVAL), (dict(out=None), EINVAL), (dict(heads=0), EINVAL), (dict(qs=1000), EINVAL), (dict(qs=1028), EINVAL),
                       (dict(q=P + 2), EINVAL), (dict(out=P + 8), EINVAL), (dict(heads=1025, qs=1 << 20), EUNSUPPORTED)):
        assert call(**{**good, **change}) == rc, change
    # launches that no grid holds
    assert call(s=seqs(n_seqs=65535, n_rows=1 << 24, max_rows=1 << 24)) == EUNSUPPORTED
    # nothing to do: nothing is looked at
    assert call(k=None, s=seqs(n_seqs=0)) == 0 and call(k=None, s=seqs(n_rows=0)) == 0 and call(k=None, s=seqs(max_rows=0, cu=None)) == 0


def test_attention_refuses(lib):
    need = lib.floe_kv_attention_workspace_bytes(cache(), seqs(), attn())
    assert need > 0
    def call(a=None, q=P, qs=1024, out=P, lse=None, ws=P, n=need, s=None):
        return lib.floe_kv_attention(cache(), s or seqs(), a or attn(), q, qs, out, lse, ws, n, None)
    for a, rc in ((dict(q_heads=0), EINVAL), (dict(q_heads=7), ESHAPE), (dict(window=-1), EINVAL), (dict(max_len=-1), EINVAL),
                  (dict(q_heads=1026), EUNSUPPORTED), (dict(window=(1 << 30) + 1), EUNSUPPORTED)):
        assert call(attn(**a), qs=1 << 20) == rc, a
        assert lib.floe_kv_attention_workspace_bytes(cache(), seqs(), attn(**a)) == 0
    assert call(q=None) == EINVAL and call(out=None) == EINVAL and call(ws=None) == EINVAL and call(qs=1020) == EINVAL and call(qs=512) == EINVAL
    assert call(ws=P + 128) == EINVAL and call(lse=P + 2) == EINVAL and call(q=P + 8) == EINVAL
    assert call(n=need - 1) == EWORKSPACE
    assert call(q=None, s=seqs(n_rows=0)) == 0
    if not torch.cuda.is_available():
        assert call() == EHIP


def test_rope_table_refuses(lib):
    def call(table=P, n=10, rot=64, base=1e4):
        return lib.floe_rope_table(table, n, rot, base, None)
    assert call(table=None) == EINVAL and call(n=-1) == EINVAL and call(rot=0) == EINVAL and call(base=0.0) == EINVAL and call(base=float("nan")) == EINVAL
    assert call(rot=24) == ESHAPE and call(rot=272) == EUNSUPPORTED and call(n=0) == 0


def test_the_binding_refuses_tensors_that_do_not_fit():
    c = F.KVCache(2, 2, 64, 32, device="cpu")
    cu, n, table = torch.tensor([0, 3], dtype=torch.int32), torch.tensor([3], dtype=torch.int32), torch.zeros((1, 2), dtype=torch.int32)
    x = torch.zeros((3, 2, 64), dtype=torch.float16)
    bad = [x.float(), x.bfloat16(), x[:, :1], torch.zeros((3, 2, 32), dtype=torch.float16), x.transpose(0, 1).contiguous().transpose(0, 1), x[0]]
    for t in bad:
        with pytest.raises(ValueError):
            F.floe_kv_append(c, t, x, cu, n, table, 3)
    with pytest.raises(ValueError):
        F.floe_kv_append(c, x, x[:2], cu, n, table, 3)
    for args in ((cu.long(), n, table), (cu, n.long(), table), (cu, torch.zeros(2, dtype=torch.int32), table), (cu, n, table[0]),
                 (cu, n, torch.zeros((2, 2), dtype=torch.int32)), (cu, n, torch.zeros((1, 4), dtype=torch.int32)[:, ::2].expand(1, 2).t().t()[:, :1].expand(1, 2))):
        with pytest.raises(ValueError):
            F.floe_kv_append(c, x, x, *args, 3)
    with pytest.raises(ValueError):
        F.floe_kv_attention(c, x, cu, n, table, 3, 3, out=torch.zeros((3, 2, 64)))
    with pytest.raises(ValueError):
        F.floe_kv_attention(c, x, cu, n, table, 3, 3, lse=torch.zeros((3, 1)))
    with pytest.raises(ValueError):
        F.floe_kv_gather(c, n, cu, table, 3, 3, k_out=torch.zeros((2, 2, 64), dtype=torch.float16))
    with pytest.raises(ValueError):
        F.KVCache(2, 2, 64, 32, dtype=torch.float32, device="cpu")
    with pytest.raises(ValueError):
        F.KVCache(2, 2, 64, 32, device="cpu", tensors=(c.k, c.v, c.k_scale, c.v_scale[:1]))
    with pytest.raises(ValueError):
        F.Rope(torch.zeros((4, 8), dtype=torch.float32))


def test_the_binding_refuses_tensors_of_the_host_before_the_library_sees_them():
    c = F.KVCache(2, 2, 64, 32, device="cpu")
    cu, n, table = torch.tensor([0, 3], dtype=torch.int32), torch.tensor([3], dtype=torch.int32), torch.zeros((1, 2), dtype=torch.int32)
    x = torch.zeros((3, 2, 64), dtype=torch.float16)
    for call in (lambda: F.floe_kv_append(c, x, x, cu, n, table, 3), lambda: F.floe_kv_attention(c, x, cu, n, table, 3, 3, workspace=c.k),
                 lambda: F.floe_kv_gather(c, n, cu, table, 3, 3)):
        with pytest.raises(ValueError, match="GPU"):
            call()


def test_a_workspace_that_was_outgrown_stays_for_the_graphs_that_hold_its_address():
    c = F.KVCache(1, 1, 64, 32, device="cpu")
    at, size = c.workspace(256, 7)
    assert c.workspace(size, 7) == (at, size)
    small = weakref.ref(c._ws[7][0])
    larger, more = c.workspace(size + 1, 7)
    assert larger != at and more >= 2 * size and c.workspace(256, 7) == (larger, more)
    assert small() is not None and small().data_ptr() <= at


class _On:
    """What the checks of a call's index arrays look at, of a tensor on any device."""
    dtype = torch.int32

    def __init__(self, device, *shape):
        self.device, self.shape = device, shape

    def get_device(self):
        return self.device

    def is_contiguous(self):
        return True

    def numel(self):
        return int(torch.Size(self.shape).numel())

    def data_ptr(self):
        return P


class _OnStream:
    def __init__(self, device):
        self.device_index = device


def test_a_cache_on_another_device_than_the_one_that_launches_is_refused(monkeypatch):
    c = F.KVCache(2, 2, 64, 32, device="cpu")
    c._device = 1
    arrays = _On(1, 3), _On(1, 2), _On(1, 2, 4)
    monkeypatch.setattr(B, "_current_device", lambda: 0)
    for stream in (None, _OnStream(0), _OnStream(1)):
        with pytest.raises(ValueError, match="cuda:1"):
            B._kv_seqs(c, *arrays, 3, 3, stream)
    monkeypatch.setattr(B, "_current_device", lambda: 1)
    with pytest.raises(ValueError, match="cuda:0"):
        B._kv_seqs(c, *arrays, 3, 3, _OnStream(0))
    assert B._kv_seqs(c, *arrays, 3, 3) == B._kv_seqs(c, *arrays, 3, 3, _OnStream(1))


def test_a_table_of_the_host_is_refused_before_a_kernel_writes_it(monkeypatch):
    with pytest.raises(ValueError, match="GPU"):
        F.floe_rope_table(4, 64, device="cpu")
    with pytest.raises(ValueError, match="GPU"):
        F.floe_rope_table(4, 64, device="meta")


def test_a_workspace_is_never_larger_than_its_tensor():
    """A view that ends before its first aligned byte holds nothing (as an unsigned size, less than nothing would be everything)."""
    whole = torch.empty(1024, dtype=torch.uint8)
    at = (-whole.data_ptr()) % 256  # first aligned byte
    for lo, hi in ((at + 1, at + 1), (at + 1, at + 100), (at + 1, at + 256), (at + 1, at + 300), (at, at), (at, at + 300)):
        ws = whole[lo:hi]
        start, size = B._aligned_ptr(ws)
        assert size == (max(0, whole.data_ptr() + hi - start) if hi > lo else 0) and start % 256 == 0  # (an empty tensor has the address 0)
    for ws in (whole[::2], whole[:1].expand(1 << 20), whole.view(32, 32).t()):
        with pytest.raises(ValueError):
            B._aligned_ptr(ws)


def test_attention_refuses_batches_whose_workgroups_no_launch_holds(lib):
    def need(dim, max_rows, n_seqs=128):
        return lib.floe_kv_attention_workspace_bytes(cache(kv_heads=32, head_dim=dim), seqs(n_seqs=n_seqs, n_rows=1 << 14, max_rows=max_rows),
                                                     attn(q_heads=1024))
    # 32 rows per token and KV head, 4096 sequences x heads; 2^32 threads are too many: at 256 dims a row has four, else two
    assert need(256, 8192) == 0 and need(256, 8180) > 0
    assert need(128, 16384) == 0 and need(128, 16300) > 0 and need(192, 8192) > 0 and need(64, 8192) > 0


def test_rope_table_refuses_more_pairs_than_a_launch_has_threads(lib):
    def call(n, rot):
        return lib.floe_rope_table(P, n, rot, 1e4, None)
    assert call(1 << 25, 256) == EUNSUPPORTED and call(1 << 28, 32) == EUNSUPPORTED and call((1 << 31) - 1, 16) == EUNSUPPORTED


@pytest.mark.parametrize("scale", [float("nan"), float("inf"), -float("inf")])
def test_attention_refuses_a_scale_that_is_not_finite(lib, scale):
    """The prompt kernel bounds the scale from below, which takes a NaN for a small one."""
    assert lib.floe_kv_attention_workspace_bytes(cache(), seqs(), attn(scale=scale)) == 0
    assert lib.floe_kv_attention(cache(), seqs(n_rows=0), attn(scale=scale), None, 1024, None, None, None, 0, None) == EINVAL


def test_index_arrays_hold_an_entry_per_sequence_and_no_more(monkeypatch):
    """Contiguous arrays are read one entry behind the other: what a second axis holds would be taken for the next sequence's."""
    c = F.KVCache(2, 2, 64, 32, device="cpu")
    c._device = 0
    monkeypatch.setattr(B, "_current_device", lambda: 0)
    for cu, length, table in (((3,), (2, 2), (2, 4)), ((3, 2), (2,), (2, 4)), ((3,), (2,), (2, 4, 1)), ((3,), (), (2, 4)), ((0,), (0,), (0, 4))):
        with pytest.raises(ValueError):
            B._kv_seqs(c, _On(0, *cu), _On(0, *length), _On(0, *table), 3, 3)
    assert B._kv_seqs(c, _On(0, 3), _On(0, 2, 1), _On(0, 2, 4), 3, 3) == B._kv_seqs(c, _On(0, 3, 1), _On(0, 2), _On(0, 2, 4), 3, 3)
