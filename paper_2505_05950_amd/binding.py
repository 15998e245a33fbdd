"""ctypes binding of include/floe.h.  Argument marshalling only: torch owns device memory and streams,
the functions below pass raw pointers and sizes to the C ABI under the same names.

A call runs on the current stream, or on `stream`: what it allocates then belongs to that stream, and the caller orders the stream
behind those that make its inputs, and before those that use its results or take its inputs' memory back."""
from __future__ import annotations

import ctypes as C
import os
import struct

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_NAME = "libfloe_hip.so"
_lib = None

SLOT_STAT_DTYPE = np.dtype([("expert", np.int32), ("count", np.int32), ("weight", np.float32), ("staged", np.int32)])


class FloeError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        msg = load().floe_status_string(status).decode()
        if status == -5:
            msg += f" [hipError {load().floe_last_hip_error()}]"
        super().__init__(f"{where}: {msg} (status {status})")


class _Shape(C.Structure):
    _fields_ = [("d", C.c_int32), ("f", C.c_int32), ("bits", C.c_int32), ("group", C.c_int32)]


class _Expert(C.Structure):
    _fields_ = [("s", _Shape), ("up_codes", C.c_void_p), ("up_scale", C.c_void_p), ("up_zero", C.c_void_p),
                ("gd", C.c_void_p), ("gd_is_staged", C.c_int32), ("gd_rows", C.c_int32)]


# The same fields for struct.pack: a call on a small expert is bound by the host, and a structure filled field by field cost it 2.3 us,
# a packed one 1.1 (it is built for every call, so that it always holds the tensors that the expert holds then)
_EXPERT_FIELDS = struct.Struct("4i4P2i")
assert _EXPERT_FIELDS.size == C.sizeof(_Expert)


class _Layer(C.Structure):
    _fields_ = [("n_experts", C.c_int32), ("top_k", C.c_int32), ("n_shared", C.c_int32), ("renormalize", C.c_int32),
                ("s", _Shape), ("router_cm", C.c_void_p), ("experts", C.POINTER(_Expert)), ("tau", C.c_void_p),
                ("tau_stride_t", C.c_int32), ("dev_table", C.c_void_p), ("gd_on_host", C.c_int32)]


class _Offload(C.Structure):
    _fields_ = [("staging", C.c_void_p), ("capacity_rows", C.c_int32), ("overflow", C.c_void_p),
                ("side_stream", C.c_void_p), ("ev_lists_ready", C.c_void_p), ("ev_staged", C.c_void_p)]


class _Prefetch(C.Structure):
    _fields_ = [("staging", C.c_void_p), ("capacity_rows", C.c_int32), ("pred_expert", C.c_void_p),
                ("pred_count", C.c_void_p), ("row_of", C.c_void_p), ("prefetch_stream", C.c_void_p),
                ("ev_inputs_ready", C.c_void_p), ("ev_prefetched", C.c_void_p)]


class _MissPath(C.Structure):
    _fields_ = [("miss_stream", C.c_void_p), ("ev_lists_ready", C.c_void_p), ("ev_staged", C.c_void_p),
                ("overflow", C.c_void_p)]


class _ChannelCache(C.Structure):
    _fields_ = [("pool", C.c_void_p), ("row_of", C.c_void_p), ("resident_rows", C.c_int32), ("capacity_rows", C.c_int32)]


class _KvCache(C.Structure):
    _fields_ = [("n_pages", C.c_int32), ("kv_heads", C.c_int32), ("head_dim", C.c_int32), ("block", C.c_int32),
                ("format", C.c_int32), ("dtype", C.c_int32), ("k", C.c_void_p), ("v", C.c_void_p), ("k_scale", C.c_void_p),
                ("v_scale", C.c_void_p)]


class _KvSeqs(C.Structure):
    _fields_ = [("n_seqs", C.c_int32), ("n_rows", C.c_int32), ("max_rows", C.c_int32), ("max_blocks", C.c_int32),
                ("cu_rows", C.c_void_p), ("len", C.c_void_p), ("block_table", C.c_void_p)]


class _Rope(C.Structure):
    _fields_ = [("table", C.c_void_p), ("positions", C.c_void_p), ("n_positions", C.c_int32), ("rot_dim", C.c_int32),
                ("interleaved", C.c_int32)]


class _KvPool(C.Structure):
    _fields_ = [("n_pages", C.c_int32), ("block", C.c_int32), ("refs", C.c_void_p)]


class _Beam(C.Structure):
    _fields_ = [("groups", C.c_int32), ("beams", C.c_int32), ("vocab", C.c_int32), ("take", C.c_int32), ("dtype", C.c_int32), ("eos", C.c_int32)]


class _Attention(C.Structure):
    _fields_ = [("q_heads", C.c_int32), ("causal", C.c_int32), ("window", C.c_int32), ("max_len", C.c_int32), ("scale", C.c_float)]


def lib_path() -> str:
    return os.path.join(_HERE, _LIB_NAME)


def load():
    """Loads the in-tree HIP library; raises if it has not been built (there is no fallback)."""
    global _lib
    if _lib is not None:
        return _lib
    path = lib_path()
    if not os.path.exists(path):
        raise ImportError(f"{path} is missing: run `python -c 'import __graft_entry__ as g; g.build()'` "
                          "(or python paper_2505_05950_amd/build.py) first; this package has no CPU fallback")
    lib = C.CDLL(path)
    vp, i32, sz = C.c_void_p, C.c_int, C.c_size_t
    lib.floe_status_string.restype = C.c_char_p
    lib.floe_status_string.argtypes = [i32]
    lib.floe_last_hip_error.restype = i32
    lib.floe_abi_version.restype = i32
    lib.floe_profile_kernel.argtypes = [i32, vp, vp]
    lib.floe_tuning.argtypes = [i32, i32]
    lib.floe_quantize_expert.argtypes = [C.POINTER(_Shape), vp, vp, vp, vp, vp]
    lib.floe_up_gemv.argtypes = [C.POINTER(_Shape), vp, vp, vp, vp, i32, vp, vp]
    lib.floe_select_channels.argtypes = [vp, i32, i32, vp, vp, vp, vp]
    lib.floe_expert_workspace_bytes.restype = sz
    lib.floe_expert_workspace_bytes.argtypes = [C.POINTER(_Shape), i32]
    lib.floe_gate_down_sparse.argtypes = [C.POINTER(_Expert), vp, i32, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.floe_expert_ffn_sparse.argtypes = [C.POINTER(_Expert), vp, i32, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.floe_expert_ffn_sparse_padded.argtypes = lib.floe_expert_ffn_sparse.argtypes
    lib.floe_expert_sparsified_workspace_bytes.restype = sz
    lib.floe_expert_sparsified_workspace_bytes.argtypes = [C.POINTER(_Shape), i32]
    lib.floe_expert_ffn_sparsified.argtypes = [C.POINTER(_Expert), i32, vp, i32, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.floe_layer_table_bytes.restype = sz
    lib.floe_layer_table_bytes.argtypes = [C.POINTER(_Layer)]
    lib.floe_layer_build_table.argtypes = [C.POINTER(_Layer), vp, sz, vp]
    lib.floe_layer_workspace_bytes.restype = sz
    lib.floe_layer_workspace_bytes.argtypes = [C.POINTER(_Layer), i32]
    lib.floe_moe_layer_decode.argtypes = [C.POINTER(_Layer), vp, i32, vp, vp, vp, sz, vp]
    lib.floe_moe_layer_decode_static.argtypes = [C.POINTER(_Layer), vp, i32, vp, vp, vp]
    lib.floe_moe_layer_decode_offloaded.argtypes = [C.POINTER(_Layer), C.POINTER(_Offload), vp, i32, vp, vp, vp, sz, vp]
    lib.floe_moe_layer_prefetch.argtypes = [C.POINTER(_Layer), C.POINTER(_Prefetch), vp, i32, vp, sz, vp]
    lib.floe_moe_layer_decode_prefetched.argtypes = [C.POINTER(_Layer), C.POINTER(_Prefetch), C.POINTER(_MissPath), vp, i32,
                                                     vp, vp, vp, vp, sz, vp]
    lib.floe_channel_cache_load.argtypes = [C.POINTER(_Layer), C.POINTER(_ChannelCache), i32, vp, vp, i32, i32, vp]
    lib.floe_moe_layer_decode_cached.argtypes = [C.POINTER(_Layer), C.POINTER(_ChannelCache), C.POINTER(_MissPath), vp, i32,
                                                 vp, vp, vp, vp, sz, vp]
    lib.floe_stage_channels.argtypes = [vp, i32, i32, vp, vp, i32, vp, vp, vp, vp]
    i64, kv, seqs, attn = C.c_int64, C.POINTER(_KvCache), C.POINTER(_KvSeqs), C.POINTER(_Attention)
    lib.floe_rope_table.argtypes = [vp, i32, i32, C.c_double, vp]
    lib.floe_kv_append.argtypes = [kv, seqs, vp, i64, vp, i64, vp, i64, i32, vp, C.POINTER(_Rope), vp]
    lib.floe_kv_gather.argtypes = [kv, seqs, vp, vp, vp]
    lib.floe_kv_attention_workspace_bytes.restype = sz
    lib.floe_kv_attention_workspace_bytes.argtypes = [kv, seqs, attn]
    lib.floe_kv_attention.argtypes = [kv, seqs, attn, vp, i64, vp, vp, vp, sz, vp]
    lib.floe_kv_attention_sinks_workspace_bytes.restype = sz
    lib.floe_kv_attention_sinks_workspace_bytes.argtypes = [kv, seqs, attn, i32]
    lib.floe_kv_attention_sinks.argtypes = [kv, seqs, attn, i32, vp, i64, vp, vp, vp, sz, vp]
    pool, beam = C.POINTER(_KvPool), C.POINTER(_Beam)
    lib.floe_kv_reorder.argtypes = [pool, vp, vp, i32, i32, vp, vp, vp, i32, vp]
    lib.floe_kv_trim.argtypes = [pool, vp, vp, i32, i32, i32, i32, vp]
    lib.floe_kv_reserve_workspace_bytes.restype = sz
    lib.floe_kv_reserve_workspace_bytes.argtypes = [pool]
    lib.floe_kv_reserve.argtypes = [pool, vp, vp, vp, i32, i32, vp, vp, vp, sz, vp]
    lib.floe_kv_compact_workspace_bytes.restype = sz
    lib.floe_kv_compact_workspace_bytes.argtypes = [pool, i32]
    lib.floe_kv_compact.argtypes = [pool, vp, i32, i32, vp, i32, vp, vp, sz, vp]
    lib.floe_kv_copy_pages.argtypes = [vp, i32, vp, i32, vp]
    lib.floe_beam_workspace_bytes.restype = sz
    lib.floe_beam_workspace_bytes.argtypes = [beam]
    lib.floe_beam_select.argtypes = [beam, vp, i64, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    _lib = lib
    return lib


def floe_status_string(status: int) -> str:
    return load().floe_status_string(status).decode()


KERNEL_IDS = {"none": 0, "quantize": 1, "router": 2, "up_gemv": 3, "select": 4, "gate_down": 5, "combine": 6, "stage": 7,
              "fused_ffn": 8, "kv_append": 9, "kv_gather": 10, "kv_attention": 11, "kv_join": 12, "kv_prompt": 13, "kv_reorder": 14, "kv_trim": 15, "kv_reserve": 16,
              "kv_compact": 17, "kv_copy": 18, "beam_rows": 19, "beam_groups": 20}


def floe_profile_kernel(kernel: str, start_event=None, stop_event=None):
    """Arms (or, with "none", disarms) the event bracket around one kernel; events are torch.cuda.Event
    objects created with enable_timing=True and recorded at least once (torch creates them lazily)."""
    kid = KERNEL_IDS[kernel]
    a = None if start_event is None else C.c_void_p(start_event.cuda_event)
    b = None if stop_event is None else C.c_void_p(stop_event.cuda_event)
    _check(load().floe_profile_kernel(kid, a, b), "floe_profile_kernel")


TUNE_UNION_KERNELS = 1
TUNE_STAGE_WORKGROUPS = 2
TUNE_GROUPED_GEMV = 3
TUNE_FUSED_TASKS = 4


def floe_tuning(key: int, value: int):
    """Process-wide tuning switch (see include/floe.h); Layer objects cache workspaces, so set it before building them."""
    _check(load().floe_tuning(int(key), int(value)), "floe_tuning")


def words_per_channel(d: int, bits: int) -> int:
    return d * bits // 32


def _ptr(t):
    if t is None:
        return None
    assert t.is_contiguous(), "tensors handed to the C ABI must be contiguous"
    return t.data_ptr()  # (ctypes makes a pointer of it; 0, an empty tensor's, is NULL)


# The current stream's handle without a Python object for it, 1 us a call (a name that torch does not promise: without it the object is made)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
# (torch.cuda.current_device without its look at whether torch has been initialised: a tensor on the GPU has seen to that)
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _stream(stream):
    if stream is None and _raw_stream is not None:
        return _raw_stream(_current_device())
    return (torch.cuda.current_stream() if stream is None else stream).cuda_stream


# What a call makes for the caller or for itself comes from the pool of the stream that it runs on: a block of another stream's pool may
# still be in use there, and would be given out again there while this call writes it.
def _empty(shape, dtype, device, stream):
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _check(rc: int, where: str):
    if rc != 0:
        raise FloeError(rc, where)


def _shape(d, f, bits, group) -> _Shape:
    return _Shape(int(d), int(f), int(bits), int(group))


class Expert:
    """Plain holder of one compressed expert's device tensors (no ownership semantics beyond Python refs)."""

    def __init__(self, d, f, bits, group, up_codes, up_scale, up_zero, gd, staged=False, gd_rows=None):
        self.d, self.f, self.bits, self.group = int(d), int(f), int(bits), int(group)
        self.up_codes, self.up_scale, self.up_zero, self.gd = up_codes, up_scale, up_zero, gd
        self.staged = bool(staged)
        self.gd_rows = int(gd_rows if gd_rows is not None else (gd.shape[0] if gd is not None else f))

    def c_struct(self) -> _Expert:
        codes, scale, zero, gd = self.up_codes, self.up_scale, self.up_zero, self.gd
        return _Expert.from_buffer_copy(_EXPERT_FIELDS.pack(
            self.d, self.f, self.bits, self.group, 0 if codes is None else codes.data_ptr(), 0 if scale is None else scale.data_ptr(),
            0 if zero is None else zero.data_ptr(), 0 if gd is None else gd.data_ptr(), self.staged, self.gd_rows))


def floe_quantize_expert(w_up_cm: torch.Tensor, bits: int, group: int, stream=None):
    """w_up_cm fp16 [f][d] on the GPU -> (codes int32-viewed-uint32 [f][d*bits/32], scale fp16, zero fp16)."""
    f, d = w_up_cm.shape
    dev = w_up_cm.device
    codes = _empty((f, max(1, d * bits // 32)), torch.int32, dev, stream)
    scale, zero = (_empty((f, max(1, d // group)), torch.float16, dev, stream) for _ in range(2))
    s = _shape(d, f, bits, group)
    _check(load().floe_quantize_expert(C.byref(s), _ptr(w_up_cm), _ptr(codes), _ptr(scale), _ptr(zero), _stream(stream)),
           "floe_quantize_expert")
    return codes, scale, zero


def floe_up_gemv(codes, scale, zero, x, d, bits, group, stream=None) -> torch.Tensor:
    f = codes.shape[0]
    T = x.shape[0]
    v = _empty((T, f), torch.float32, x.device, stream)
    s = _shape(d, f, bits, group)
    _check(load().floe_up_gemv(C.byref(s), _ptr(codes), _ptr(scale), _ptr(zero), _ptr(x), T, _ptr(v), _stream(stream)),
           "floe_up_gemv")
    return v


def _list(shape, device, stream):
    """Channel lists, -1 where the call writes none; filled on the stream that the call runs on."""
    if stream is None:
        return torch.full(shape, -1, dtype=torch.int32, device=device)
    with torch.cuda.stream(stream):
        return torch.full(shape, -1, dtype=torch.int32, device=device)


def floe_select_channels(v: torch.Tensor, tau: torch.Tensor, stream=None):
    T, f = v.shape
    idx = _list((T, f), v.device, stream)
    count = _empty((T,), torch.int32, v.device, stream)
    _check(load().floe_select_channels(_ptr(v), f, T, _ptr(tau), _ptr(idx), _ptr(count), _stream(stream)),
           "floe_select_channels")
    return idx, count


def floe_expert_workspace_bytes(d, f, bits, group, T) -> int:
    s = _shape(d, f, bits, group)
    return int(load().floe_expert_workspace_bytes(C.byref(s), int(T)))


def _workspace(nbytes: int, device, stream=None) -> torch.Tensor:
    return _empty((max(nbytes, 256) + 256,), torch.uint8, device, stream)


def _aligned_ptr(ws: torch.Tensor):
    if not ws.is_contiguous():
        raise ValueError(f"workspace: expected a contiguous tensor, got strides {ws.stride()}")
    base = ws.data_ptr()
    off = (-base) % 256
    return base + off, max(0, ws.numel() - off)


def floe_gate_down_sparse(e: Expert, x, v, idx, count, out_scale, y_acc, workspace=None, stream=None):
    T = x.shape[0]
    if workspace is None:
        workspace = _workspace(floe_expert_workspace_bytes(e.d, e.f, e.bits, e.group, T), x.device, stream)
    wp, wn = _aligned_ptr(workspace)
    es = e.c_struct()
    _check(load().floe_gate_down_sparse(C.byref(es), _ptr(x), T, _ptr(v), _ptr(idx), _ptr(count), _ptr(out_scale),
                                        _ptr(y_acc), wp, wn, _stream(stream)), "floe_gate_down_sparse")
    return y_acc


def floe_expert_ffn_sparse(e: Expert, x, tau, out_scale, y_acc, idx=None, count=None, workspace=None, stream=None,
                           want_list=True):
    """Alg. 1 for T tokens; returns (y_acc, idx, count); want_list=False passes no list buffers (idx, count = None)."""
    T = x.shape[0]
    call = load().floe_expert_ffn_sparse
    if want_list:
        if idx is None:  # a list of our own: the call that writes it also sets what lies behind its end
            call = load().floe_expert_ffn_sparse_padded
            idx = _empty((T, e.f), torch.int32, x.device, stream)
        if count is None:
            count = _empty((T,), torch.int32, x.device, stream)
    else:
        idx = count = None
    if workspace is None:
        workspace = _workspace(floe_expert_workspace_bytes(e.d, e.f, e.bits, e.group, T), x.device, stream)
    wp, wn = _aligned_ptr(workspace)
    es = e.c_struct()
    _check(call(C.byref(es), _ptr(x), T, _ptr(tau), _ptr(out_scale), _ptr(y_acc), _ptr(idx), _ptr(count), wp, wn,
                _stream(stream)), "floe_expert_ffn_sparse")
    return y_acc, idx, count


SPARSIFY_UP, SPARSIFY_GATE, SPARSIFY_DOWN = 0, 1, 2


def floe_expert_ffn_sparsified(e: Expert, which: int, x, tau, out_scale, y_acc, workspace=None, stream=None):
    """Eq. 1 with the sparsity function on a_up / a_gate / a_down (Sec. 3.2.1); returns (y_acc, idx, count)."""
    T = x.shape[0]
    idx = _list((T, e.f), x.device, stream)
    count = _empty((T,), torch.int32, x.device, stream)
    if workspace is None:
        s = _shape(e.d, e.f, e.bits, e.group)
        workspace = _workspace(int(load().floe_expert_sparsified_workspace_bytes(C.byref(s), T)), x.device, stream)
    wp, wn = _aligned_ptr(workspace)
    es = e.c_struct()
    _check(load().floe_expert_ffn_sparsified(C.byref(es), int(which), _ptr(x), T, _ptr(tau), _ptr(out_scale), _ptr(y_acc),
                                             _ptr(idx), _ptr(count), wp, wn, _stream(stream)), "floe_expert_ffn_sparsified")
    return y_acc, idx, count


class Layer:
    """One MoE layer: routed experts first, shared experts last; builds the HBM pointer table once."""

    def __init__(self, experts, n_shared, top_k, renormalize, router_cm, tau, tau_per_token: bool, stream=None,
                 gd_on_host: bool = False):
        self.experts = list(experts)
        e0 = self.experts[0]
        self.d, self.f, self.bits, self.group = e0.d, e0.f, e0.bits, e0.group
        self.n_shared, self.top_k, self.renormalize = int(n_shared), int(top_k), bool(renormalize)
        self.n_experts = len(self.experts) - self.n_shared
        self.router_cm, self.tau = router_cm, tau
        self.tau_stride = len(self.experts) if tau_per_token else 0
        self._arr = (_Expert * len(self.experts))(*[e.c_struct() for e in self.experts])
        self._c = _Layer(self.n_experts, self.top_k, self.n_shared, int(self.renormalize),
                         _shape(self.d, self.f, self.bits, self.group),
                         None if router_cm is None else router_cm.data_ptr(), self._arr, tau.data_ptr(),
                         self.tau_stride, None, int(gd_on_host))
        self.gd_on_host = bool(gd_on_host)
        nbytes = floe_layer_table_bytes(self)
        self.table = _empty((nbytes + 256,), torch.uint8, tau.device, stream)
        tp, tn = _aligned_ptr(self.table)
        floe_layer_build_table(self, tp, tn, stream)
        self._c.dev_table = tp
        self._ws = {}

    def set_tau(self, tau, tau_per_token: bool):
        self.tau = tau
        self.tau_stride = len(self.experts) if tau_per_token else 0
        self._c.tau = tau.data_ptr()
        self._c.tau_stride_t = self.tau_stride

    def new_workspace(self, T: int) -> torch.Tensor:
        """A workspace of its own (e.g. for a prefetch that runs beside a decode call)."""
        return _workspace(floe_layer_workspace_bytes(self, T), self.tau.device)

    def workspace(self, T: int, stream=None) -> torch.Tensor:
        if T not in self._ws:
            self._ws[T] = _workspace(floe_layer_workspace_bytes(self, T), self.tau.device, stream)
        return self._ws[T]


def floe_layer_table_bytes(L: Layer) -> int:
    return int(load().floe_layer_table_bytes(C.byref(L._c)))


def floe_layer_build_table(L: Layer, table_ptr, table_bytes, stream=None):
    _check(load().floe_layer_build_table(C.byref(L._c), table_ptr, table_bytes, _stream(stream)), "floe_layer_build_table")


def floe_layer_workspace_bytes(L: Layer, T: int) -> int:
    return int(load().floe_layer_workspace_bytes(C.byref(L._c), int(T)))


def floe_moe_layer_decode(L: Layer, x: torch.Tensor, y: torch.Tensor = None, stats: torch.Tensor = None,
                          workspace=None, stream=None):
    """x fp16 [T][d] -> y fp16 [T][d]; stats (optional) int32 [T][slots][4] viewed as floe_slot_stat."""
    T = x.shape[0]
    if y is None:
        y = _empty((T, L.d), torch.float16, x.device, stream)
    if workspace is None:
        workspace = L.workspace(T, stream)
    wp, wn = _aligned_ptr(workspace)
    _check(load().floe_moe_layer_decode(C.byref(L._c), _ptr(x), T, _ptr(y), _ptr(stats), wp, wn, _stream(stream)),
           "floe_moe_layer_decode")
    return y


STATIC_SCRATCH_BYTES = 16 << 20


def floe_moe_layer_decode_static(L: Layer, x: torch.Tensor, y: torch.Tensor, stats: torch.Tensor = None, stream=None):
    """floe_moe_layer_decode on the library's own scratch array; y must be supplied (nothing is allocated here)."""
    _check(load().floe_moe_layer_decode_static(C.byref(L._c), _ptr(x), x.shape[0], _ptr(y), _ptr(stats), _stream(stream)),
           "floe_moe_layer_decode_static")
    return y


def floe_moe_layer_decode_offloaded(L: Layer, x, staging, capacity_rows, side_stream, ev_lists_ready, ev_staged,
                                    y=None, stats=None, overflow=None, workspace=None, stream=None):
    """Offloaded layer: experts' gd are pinned host tensors; staging dev [T*slots][capacity_rows][2][d]."""
    T = x.shape[0]
    if y is None:
        y = _empty((T, L.d), torch.float16, x.device, stream)
    if workspace is None:
        workspace = L.workspace(T, stream)
    wp, wn = _aligned_ptr(workspace)
    cur = stream if stream is not None else torch.cuda.current_stream()
    # torch creates the hipEvent_t lazily on the first record(); the library records both again
    ev_lists_ready.record(cur)
    ev_staged.record(side_stream)
    off = _Offload(staging.data_ptr(), int(capacity_rows), None if overflow is None else overflow.data_ptr(),
                   side_stream.cuda_stream, ev_lists_ready.cuda_event, ev_staged.cuda_event)
    _check(load().floe_moe_layer_decode_offloaded(C.byref(L._c), C.byref(off), _ptr(x), T, _ptr(y), _ptr(stats), wp, wn,
                                                  _stream(stream)), "floe_moe_layer_decode_offloaded")
    return y


PREFETCH_STAT_DTYPE = np.dtype([("expert_predicted", np.int32), ("predicted", np.int32), ("hits", np.int32),
                                ("misses", np.int32)])


class Prefetch:
    """Buffers and events of one floe_prefetch object (two of them alternate between neighbouring layers):
    staging [2*T*slots][capacity][2][d], predicted expert / count per task, row map [T*slots][f]."""

    def __init__(self, L: "Layer", T: int, capacity_rows: int, prefetch_stream, device=None):
        dev = device if device is not None else L.tau.device
        slots = L.top_k + L.n_shared
        n = T * slots
        self.T, self.capacity_rows, self.stream = T, int(capacity_rows), prefetch_stream
        self.staging = torch.empty((2 * n, capacity_rows, 2, L.d), dtype=torch.float16, device=dev)
        self.pred_expert = torch.full((n,), -1, dtype=torch.int32, device=dev)
        self.pred_count = torch.zeros((n,), dtype=torch.int32, device=dev)
        self.row_of = torch.full((n, L.f), -1, dtype=torch.int32, device=dev)
        self.ev_inputs_ready, self.ev_prefetched = torch.cuda.Event(), torch.cuda.Event()
        # torch creates the hipEvent_t lazily on the first record(); after this the library alone records them
        self.ev_inputs_ready.record(torch.cuda.current_stream())
        self.ev_prefetched.record(prefetch_stream)
        self._c = _Prefetch(self.staging.data_ptr(), self.capacity_rows, self.pred_expert.data_ptr(),
                            self.pred_count.data_ptr(), self.row_of.data_ptr(), prefetch_stream.cuda_stream,
                            self.ev_inputs_ready.cuda_event, self.ev_prefetched.cuda_event)


class MissPath:
    """Stream and events on which the channels that were not predicted are copied."""

    def __init__(self, miss_stream, n_tasks: int, device):
        self.stream = miss_stream
        self.overflow = torch.zeros((n_tasks,), dtype=torch.int32, device=device)
        self.ev_lists_ready, self.ev_staged = torch.cuda.Event(), torch.cuda.Event()
        self.ev_lists_ready.record(torch.cuda.current_stream())
        self.ev_staged.record(miss_stream)
        self._c = _MissPath(miss_stream.cuda_stream, self.ev_lists_ready.cuda_event, self.ev_staged.cuda_event,
                            self.overflow.data_ptr())


def floe_moe_layer_prefetch(L: Layer, P: Prefetch, x_cur, workspace, stream=None):
    """Predicts layer L's experts and channels from x_cur and copies their chunks ahead (on P.stream)."""
    T = x_cur.shape[0]
    wp, wn = _aligned_ptr(workspace)
    _check(load().floe_moe_layer_prefetch(C.byref(L._c), C.byref(P._c), _ptr(x_cur), T, wp, wn, _stream(stream)),
           "floe_moe_layer_prefetch")


def floe_moe_layer_decode_prefetched(L: Layer, P: Prefetch, M: MissPath, x, y=None, stats=None, prefetch_stats=None,
                                     workspace=None, stream=None):
    """Layer decode on staging rows that floe_moe_layer_prefetch has (partly) filled; only the misses are copied now."""
    T = x.shape[0]
    if y is None:
        y = _empty((T, L.d), torch.float16, x.device, stream)
    if workspace is None:
        workspace = L.workspace(T, stream)
    wp, wn = _aligned_ptr(workspace)
    _check(load().floe_moe_layer_decode_prefetched(C.byref(L._c), C.byref(P._c), C.byref(M._c), _ptr(x), T, _ptr(y),
                                                   _ptr(stats), _ptr(prefetch_stats), wp, wn, _stream(stream)),
           "floe_moe_layer_decode_prefetched")
    return y


class ChannelCache:
    """Buffers of a floe_channel_cache: the pool (resident rows, then one slab per (token, slot)) and the row map."""

    def __init__(self, L: "Layer", T: int, resident_rows: int, capacity_rows: int, device=None):
        dev = device if device is not None else L.tau.device
        n = T * (L.top_k + L.n_shared)
        self.resident_rows, self.capacity_rows = int(resident_rows), int(capacity_rows)
        self.pool = torch.empty((self.resident_rows + n * self.capacity_rows, 2, L.d), dtype=torch.float16, device=dev)
        self.row_of = torch.full((len(L.experts), L.f), -1, dtype=torch.int32, device=dev)
        self._c = _ChannelCache(self.pool.data_ptr(), self.row_of.data_ptr(), self.resident_rows, self.capacity_rows)


def floe_channel_cache_load(L: Layer, cache: ChannelCache, expert: int, idx, count, first_row: int, max_rows: int, stream=None):
    _check(load().floe_channel_cache_load(C.byref(L._c), C.byref(cache._c), int(expert), _ptr(idx), _ptr(count), int(first_row),
                                          int(max_rows), _stream(stream)), "floe_channel_cache_load")


def floe_moe_layer_decode_cached(L: Layer, cache: ChannelCache, M: MissPath, x, y=None, stats=None, cache_stats=None,
                                 workspace=None, stream=None):
    T = x.shape[0]
    if y is None:
        y = _empty((T, L.d), torch.float16, x.device, stream)
    if workspace is None:
        workspace = L.workspace(T, stream)
    wp, wn = _aligned_ptr(workspace)
    _check(load().floe_moe_layer_decode_cached(C.byref(L._c), C.byref(cache._c), C.byref(M._c), _ptr(x), T, _ptr(y),
                                               _ptr(stats), _ptr(cache_stats), wp, wn, _stream(stream)),
           "floe_moe_layer_decode_cached")
    return y


def floe_stage_channels(host_gd: torch.Tensor, idx, count, capacity_rows: int, hbm_dst, overflow=None,
                        side_stream=None, done_event=None):
    """host_gd: pinned CPU fp16 tensor [f][2][d]; idx/count device; hbm_dst device [capacity][2][d]."""
    assert host_gd.is_pinned(), "host_gd must be pinned host memory"
    d = host_gd.shape[-1]
    f = host_gd.shape[0]
    ev = None
    if done_event is not None:
        # torch creates the underlying hipEvent_t lazily on the first record(); force that now.
        # The library records the same event again after the copy, which supersedes this one.
        done_event.record(side_stream if side_stream is not None else torch.cuda.current_stream())
        ev = C.c_void_p(done_event.cuda_event)
    _check(load().floe_stage_channels(C.c_void_p(host_gd.data_ptr()), d, f, _ptr(idx), _ptr(count), int(capacity_rows),
                                      _ptr(hbm_dst), _ptr(overflow), _stream(side_stream), ev), "floe_stage_channels")
    return hbm_dst


# ---- attention in front of the MoE layer: the paged cache in 8 bits (layout and arithmetic in include/floe.h)
KV_INT8, KV_E4M3 = 0, 1
_KV_DTYPES = {torch.float16: 0, torch.bfloat16: 1}


class KVCache:
    """Pages of `block` tokens: codes of K and V (uint8) and one fp32 scale per page and head for each.  tensors=(k, v, k_scale,
    v_scale) wraps arrays that exist; otherwise they are allocated (and need no initialising).  dtype: of the 16-bit tensors of the calls."""

    def __init__(self, n_pages: int, kv_heads: int, head_dim: int, block: int = 64, fmt: int = KV_INT8, dtype=torch.float16,
                 device="cuda", tensors=None):
        self.n_pages, self.kv_heads, self.head_dim, self.block = int(n_pages), int(kv_heads), int(head_dim), int(block)
        self.fmt, self.dtype = int(fmt), dtype
        if dtype not in _KV_DTYPES:
            raise ValueError(f"KVCache: dtype is torch.float16 or torch.bfloat16, not {dtype}")
        n = self.n_pages * self.kv_heads
        if tensors is None:
            codes = [torch.empty((self.n_pages, self.kv_heads, self.block, self.head_dim), dtype=torch.uint8, device=device) for _ in range(2)]
            tensors = (*codes, *(torch.empty((self.n_pages, self.kv_heads), dtype=torch.float32, device=device) for _ in range(2)))
        self.k, self.v, self.k_scale, self.v_scale = tensors
        for t, size, kind in ((self.k, n * self.block * self.head_dim, torch.uint8), (self.v, n * self.block * self.head_dim, torch.uint8),
                              (self.k_scale, n, torch.float32), (self.v_scale, n, torch.float32)):
            if t.numel() != size or t.dtype != kind or not t.is_contiguous():
                raise ValueError(f"KVCache: expected a contiguous {kind} tensor of {size} elements, got {t.dtype} {tuple(t.shape)}")
        self._device = self.k.get_device()  # (-1 for tensors of the host; a look at t.device costs twice as much)
        if any(t.get_device() != self._device for t in tensors):
            raise ValueError("KVCache: the four arrays are on one device")
        self._c = _KvCache(self.n_pages, self.kv_heads, self.head_dim, self.block, self.fmt, _KV_DTYPES[dtype], self.k.data_ptr(),
                           self.v.data_ptr(), self.k_scale.data_ptr(), self.v_scale.data_ptr())
        self._at = C.addressof(self._c)
        self._ws = {}

    def workspace(self, nbytes: int, stream: int, pool=None):
        """(address, bytes) of scratch for the attention calls on a stream: an array per stream, since the calls on one are ordered.
        An array that was too small stays (a captured graph may hold its address); each is twice the one before or more.  pool: the
        stream as an object, where it is not the current one."""
        ws = self._ws.get(stream)
        if ws is None or ws[2] < nbytes:
            array = _workspace(max(nbytes, 2 * ws[2]) if ws else nbytes, self.k.device, pool)
            ws = self._ws[stream] = (array, *_aligned_ptr(array), ws)
        return ws[1], ws[2]


class Rope:
    """The rotation that an append applies: table fp32 [positions][rot_dim / 2][2] of (cos, sin)."""

    def __init__(self, table: torch.Tensor, interleaved: bool = False):
        if table.dtype != torch.float32 or table.dim() != 3 or table.shape[2] != 2 or not table.is_contiguous():
            raise ValueError("Rope: table is a contiguous fp32 tensor [positions][rot_dim / 2][2]")
        self.table, self.interleaved = table, bool(interleaved)
        self.n_positions, self.rot_dim = int(table.shape[0]), 2 * int(table.shape[1])

    def _packed(self, positions):
        return _ROPE_FIELDS.pack(self.table.data_ptr(), 0 if positions is None else positions.data_ptr(), self.n_positions, self.rot_dim,
                                 self.interleaved)


def _fits(n: int, name: str) -> int:
    """A number for a 32-bit argument (ctypes would hand over its lower bits)."""
    if -0x80000000 <= n <= 0x7fffffff:
        return n
    raise ValueError(f"{name}: {n} does not fit 32 bits")


def _launches_on(device: int, stream, what: str):
    """The library launches on the current device, and a stream is one device's: both have to be the one that the memory is on."""
    if device < 0:
        raise ValueError(f"{what} is not on a GPU")
    if device != _current_device() or (stream is not None and stream.device_index != device):
        on = f"cuda:{_current_device()}" + ("" if stream is None else f", the stream of cuda:{stream.device_index}")
        raise ValueError(f"{what} is on cuda:{device}, the current device is {on}: call it under torch.cuda.device({device})")


def floe_rope_table(n_positions: int, rot_dim: int, base: float = 10000.0, device="cuda", stream=None) -> torch.Tensor:
    table = _empty((int(n_positions), int(rot_dim) // 2, 2), torch.float32, device, stream)
    _launches_on(table.get_device(), stream, "floe_rope_table: the table")
    _check(load().floe_rope_table(_ptr(table), int(n_positions), int(rot_dim), float(base), _stream(stream)), "floe_rope_table")
    return table


# A decode step of one sequence is bound by the host: what these calls hand over is packed at once (a structure filled field by field
# costs a microsecond more), their functions take plain integers, and what is right is seen in one look (_kv_wrong says what is not).
_SEQS_FIELDS, _ROPE_FIELDS, _ATTENTION_FIELDS = struct.Struct("4i3P"), struct.Struct("2P3i4x"), struct.Struct("4if")
assert [f.size for f in (_SEQS_FIELDS, _ROPE_FIELDS, _ATTENTION_FIELDS)] == [C.sizeof(t) for t in (_KvSeqs, _Rope, _Attention)]
_kv_functions = None


def _kv_calls():
    global _kv_functions
    if _kv_functions is None:
        lib, vp, i64, i32, packed, sz = load(), C.c_void_p, C.c_int64, C.c_int, C.c_char_p, C.c_size_t
        append, gather, attention, need = (lib[n] for n in ("floe_kv_append", "floe_kv_gather", "floe_kv_attention_sinks",
                                                            "floe_kv_attention_sinks_workspace_bytes"))
        append.argtypes = [vp, packed, vp, i64, vp, i64, vp, i64, i32, vp, packed, vp]
        gather.argtypes = [vp, packed, vp, vp, vp]
        attention.argtypes = [vp, packed, packed, i32, vp, i64, vp, vp, vp, sz, vp]
        need.argtypes, need.restype = [vp, packed, packed, i32], sz
        _kv_functions = append, gather, attention, need
    return _kv_functions


def _kv_seqs(cache, cu_rows, length, block_table, n_rows, max_rows, stream=None) -> bytes:
    device, n, i32 = cache._device, cu_rows.numel() - 1, torch.int32
    shape = block_table.shape
    if not (cu_rows.dtype is i32 and length.dtype is i32 and block_table.dtype is i32 and cu_rows.is_contiguous() and length.is_contiguous()
            and block_table.is_contiguous()):
        raise ValueError("cu_rows, lengths and block_table are contiguous int32 tensors")
    if length.numel() != n or len(shape) != 2 or shape[0] != n:
        raise ValueError(f"{n} sequences in cu_rows, {tuple(length.shape)} lengths, block_table {tuple(shape)}")
    if cu_rows.get_device() != device or length.get_device() != device or block_table.get_device() != device or device < 0:
        raise ValueError("cu_rows, lengths and block_table are on the cache's GPU")
    _launches_on(device, stream, "the cache")
    return _SEQS_FIELDS.pack(n, n_rows, max_rows, shape[1], cu_rows.data_ptr(), length.data_ptr(), block_table.data_ptr())


def _kv_wrong(t, cache, heads, n_rows, name):
    shape = tuple(t.shape)
    if t.dtype != cache.dtype or len(shape) != 3 or shape[1:] != (heads, cache.head_dim):
        raise ValueError(f"{name}: expected {cache.dtype} [rows][{heads}][{cache.head_dim}], got {t.dtype} {shape}")
    if shape[0] != n_rows:
        raise ValueError(f"{name}: {shape[0]} rows, expected {n_rows}")
    if t.get_device() != cache._device:
        raise ValueError(f"{name}: on {t.device}, the cache is on {cache.k.device}")
    raise ValueError(f"{name}: the heads of a row lie one behind the other (strides {t.stride()})")


def _kv_rows(t, cache: KVCache, heads, n_rows, name: str):
    """Row stride of a 16-bit tensor [n_rows][heads][head_dim] whose rows may lie anywhere."""
    shape, D = t.shape, cache.head_dim
    if t.dtype is not cache.dtype or len(shape) != 3 or shape[2] != D or shape[1] != heads or shape[0] != n_rows or t.get_device() != cache._device:
        _kv_wrong(t, cache, heads, n_rows, name)
    stride = t.stride()
    if (stride[2] != 1 or (stride[1] != D and heads > 1)) and n_rows:
        _kv_wrong(t, cache, heads, n_rows, name)
    return stride[0] if n_rows > 1 else heads * D


def _kv_out(t, cache, shape, dtype, like, name, stream):
    """An output tensor: the caller's, if it fits, or a new one beside `like` (which saves 1 us where it has the same form)."""
    if t is None:
        if stream is not None:
            return _empty(shape, dtype, like.device, stream)
        if like.dtype is dtype and like.shape == shape and like.is_contiguous():
            return torch.empty_like(like)
        return like.new_empty(shape, dtype=dtype)
    if tuple(t.shape) != tuple(shape) or t.dtype != dtype or not t.is_contiguous() or t.get_device() != cache._device:
        raise ValueError(f"{name}: expected a contiguous {dtype} tensor {tuple(shape)} on {like.device}, got {t.dtype} {tuple(t.shape)} on {t.device}")
    return t


def floe_kv_append(cache: KVCache, k, v, cu_rows, length, block_table, max_rows: int, q=None, rope: Rope = None, positions=None,
                   q_out=None, stream=None):
    """Appends k, v [rows][kv_heads][head_dim] behind the first length[s] tokens of each sequence; rope turns k, and q
    [rows][q_heads][head_dim] into q_out, which is returned (None without q).  max_rows: at least the rows of any sequence."""
    n_rows = k.shape[0]
    ks, vs = _kv_rows(k, cache, cache.kv_heads, n_rows, "k"), _kv_rows(v, cache, cache.kv_heads, n_rows, "v")
    qs = heads = q_at = q_out_at = 0
    if q is not None:
        shape = q.shape
        heads = shape[1] if len(shape) == 3 else 0
        qs, q_at = _kv_rows(q, cache, heads, n_rows, "q"), q.data_ptr()
        q_out = _kv_out(q_out, cache, shape, cache.dtype, q, "q_out", stream)
        q_out_at = q_out.data_ptr()
    if positions is not None and (positions.dtype != torch.int32 or positions.shape != (n_rows,) or not positions.is_contiguous()
                                  or positions.get_device() != cache._device):
        raise ValueError(f"positions: expected contiguous int32 [{n_rows}] on {cache.k.device}")
    if rope is not None and rope.table.get_device() != cache._device:
        raise ValueError(f"rope: its table is on {rope.table.device}, the cache on {cache.k.device}")
    rc = _kv_calls()[0](cache._at, _kv_seqs(cache, cu_rows, length, block_table, n_rows, max_rows, stream), k.data_ptr(), ks, v.data_ptr(), vs, q_at, qs,
                        heads, q_out_at, None if rope is None else rope._packed(positions), _stream(stream))
    if rc:
        _check(rc, "floe_kv_append")
    return q_out if q is not None else None


def floe_kv_gather(cache: KVCache, first, cu_rows, block_table, n_rows: int, max_rows: int, k_out=None, v_out=None, stream=None):
    """Rows cu_rows[s] .. cu_rows[s + 1) are tokens first[s], first[s] + 1, ... of sequence s: (k, v) 16-bit [n_rows][kv_heads][head_dim]."""
    shape = (n_rows, cache.kv_heads, cache.head_dim)
    k_out = _kv_out(k_out, cache, shape, cache.dtype, cache.k, "k_out", stream)
    v_out = _kv_out(v_out, cache, shape, cache.dtype, k_out, "v_out", stream)
    rc = _kv_calls()[1](cache._at, _kv_seqs(cache, cu_rows, first, block_table, n_rows, max_rows, stream), k_out.data_ptr(), v_out.data_ptr(), _stream(stream))
    if rc:
        _check(rc, "floe_kv_gather")
    return k_out, v_out


def floe_kv_attention(cache: KVCache, q, cu_rows, length, block_table, max_rows: int, max_len: int, scale: float = None,
                      causal: bool = True, window: int = 0, want_lse: bool = False, out=None, lse=None, workspace=None, stream=None,
                      sinks: int = 0):
    """Attention of q [rows][q_heads][head_dim] over the cache; length[s] counts the rows' own tokens.  Returns out, or (out, lse) with
    want_lse.  scale: 1 / sqrt(head_dim) by default.  sinks: first tokens that rows see beside their window.  max_len: at least every length; far above them, small batches take longer (floe.h).
    workspace: the cache's own (one per stream) unless handed over; a captured call keeps the one of the stream it was captured on, so
    graphs that run side by side, or beside eager calls on that stream, are captured on different streams or bring theirs."""
    shape = q.shape
    n_rows, heads = shape[0], shape[1] if len(shape) == 3 else 0
    qs = _kv_rows(q, cache, heads, n_rows, "q")
    out = _kv_out(out, cache, shape, cache.dtype, q, "out", stream)
    if want_lse or lse is not None:
        lse = _kv_out(lse, cache, (n_rows, heads), torch.float32, q, "lse", stream)
    call, need = _kv_calls()[2:]
    if sinks:
        _fits(sinks, "sinks")
    s = _kv_seqs(cache, cu_rows, length, block_table, n_rows, max_rows, stream)
    a = _ATTENTION_FIELDS.pack(heads, causal, window, max_len, cache.head_dim ** -0.5 if scale is None else scale)
    if workspace is not None and workspace.get_device() != cache._device:
        raise ValueError(f"workspace: on {workspace.device}, the cache is on {cache.k.device}")
    st = _stream(stream)
    at, size = cache.workspace(256, st, stream) if workspace is None else _aligned_ptr(workspace)
    args = cache._at, s, a, sinks, q.data_ptr(), qs, out.data_ptr(), None if lse is None else lse.data_ptr()
    rc = call(*args, at, size, st)
    if rc == -4 and workspace is None:  # refused before anything is enqueued: the cache's workspace has to grow
        at, size = cache.workspace(need(cache._at, s, a, sinks), st, stream)
        rc = call(*args, at, size, st)
    if rc:
        _check(rc, "floe_kv_attention")
    return (out, lse) if lse is not None else out


# ---- the pages of such caches: handed out, shared, given back, packed, copied (include/floe.h)
_page_functions = None


def _page_calls():
    """The pages' functions with plain integers for addresses (these calls are bound by the host too)."""
    global _page_functions
    if _page_functions is None:
        lib, vp, i32, sz = load(), C.c_void_p, C.c_int, C.c_size_t
        reorder, reserve, trim, compact, copy = (lib["floe_kv_" + n] for n in ("reorder", "reserve", "trim", "compact", "copy_pages"))
        reorder.argtypes = [vp, vp, vp, i32, i32, vp, vp, vp, i32, vp]
        reserve.argtypes = [vp, vp, vp, vp, i32, i32, vp, vp, vp, sz, vp]
        trim.argtypes = [vp, vp, vp, i32, i32, i32, i32, vp]
        compact.argtypes = [vp, vp, i32, i32, vp, i32, vp, vp, sz, vp]
        copy.argtypes = [vp, i32, vp, i32, vp]
        _page_functions = reorder, reserve, trim, compact, copy
    return _page_functions


def _i32(t, shape, device: int, name: str) -> int:
    """Address of a contiguous int32 tensor of this shape on the pool's GPU."""
    if t.dtype is torch.int32 and t.shape == shape and t.is_contiguous() and t.get_device() == device:
        return t.data_ptr()
    if t.get_device() != device:
        raise ValueError(f"{name}: on {t.device}, expected cuda:{device}")
    raise ValueError(f"{name}: expected contiguous int32 {tuple(shape)}, got {t.dtype} {tuple(t.shape)}, strides {t.stride()}")


def _new(like, shape, dtype, stream):
    return like.new_empty(shape, dtype=dtype) if stream is None else _empty(shape, dtype, like.device, stream)


class KVPool:
    """How many table entries name each of a cache's pages: refs int32 [n_pages], zeros at the start (refs=: an array that exists).  One
    pool serves the caches of all layers, which share their tables.  Its calls are ordered by the caller, captured ones too.  Captured calls
    hold the addresses of refs and, unless handed a workspace, of the pool's own: the pool lives as long as their graphs."""

    def __init__(self, n_pages: int, block: int = 64, refs=None, device="cuda"):
        self.n_pages, self.block = _fits(int(n_pages), "KVPool: n_pages"), _fits(int(block), "KVPool: block")
        if self.n_pages < 1:
            raise ValueError(f"KVPool: at least one page, not {n_pages}")
        if refs is None:
            refs = torch.zeros((self.n_pages,), dtype=torch.int32, device=device)
        if refs.dtype is not torch.int32 or refs.shape != (self.n_pages,) or not refs.is_contiguous():
            raise ValueError(f"KVPool: refs is a contiguous int32 tensor [{self.n_pages}], got {refs.dtype} {tuple(refs.shape)}")
        self.refs, self._device = refs, refs.get_device()
        self._c = _KvPool(self.n_pages, self.block, refs.data_ptr())
        self._at = C.addressof(self._c)
        lib, at = load(), C.byref(self._c)
        self._need = max(lib.floe_kv_reserve_workspace_bytes(at), lib.floe_kv_compact_workspace_bytes(at, self.n_pages))
        self._ws = {}

    def _workspace(self, given, st: int, stream):
        """(address, bytes) of scratch: an array per stream, from that stream's pool of memory, which takes it back in the order of the
        stream when the pool is dropped while calls are still queued."""
        if given is None:
            ws = self._ws.get(st)
            if ws is None:
                array = _workspace(self._need, self.refs.device, stream)
                ws = self._ws[st] = (*_aligned_ptr(array), array)
            return ws[0], ws[1]
        if given.get_device() != self._device:
            raise ValueError(f"workspace: on {given.device}, the pool is on {self.refs.device}")
        return _aligned_ptr(given)

    def _table(self, table, stream):
        """Address and sizes of a table, on the device that launches."""
        shape = table.shape
        if len(shape) != 2:
            raise ValueError(f"table: expected int32 [sequences][blocks], got {tuple(shape)}")
        _launches_on(self._device, stream, "the pool")
        return _i32(table, shape, self._device, "table"), _fits(shape[0], "table: sequences"), _fits(shape[1], "table: blocks")


def _given_or_new(t, shape, pool, like, name, stream):
    if t is None:
        return _new(like, shape, torch.int32, stream)
    _i32(t, shape, pool._device, name)
    return t


def floe_kv_reorder(pool: KVPool, table, length, parent, table_out=None, length_out=None, stream=None):
    """Sequence i takes over the pages and the length of sequence parent[i] (outside the table: none); `table` is no longer in use afterwards.
    Returns (table_out, length_out)."""
    at, n, blocks = pool._table(table, stream)
    m = _fits(parent.numel(), "parent")
    length_at, parent_at = _i32(length, (n,), pool._device, "length"), _i32(parent, (m,), pool._device, "parent")
    table_out = _given_or_new(table_out, (m, blocks), pool, table, "table_out", stream)
    length_out = _given_or_new(length_out, (m,), pool, table, "length_out", stream)
    rc = _page_calls()[0](pool._at, at, length_at, n, blocks, parent_at, table_out.data_ptr(), length_out.data_ptr(), m, _stream(stream))
    if rc:
        _check(rc, "floe_kv_reorder")
    return table_out, length_out


def floe_kv_reserve(pool: KVPool, table, length, cu_rows, pairs=None, missing=None, workspace=None, stream=None):
    """Gives every block that an append of cu_rows behind `length` tokens writes to a page that only its sequence names.  Returns (pairs
    int32 [sequences][2], what floe_kv_copy_pages has to copy before the append and before any other call on the pool; missing int32 [1],
    blocks that got no page: nothing is appended then, but what the pairs name is copied all the same)."""
    at, n, blocks = pool._table(table, stream)
    length_at, cu_at = _i32(length, (n,), pool._device, "length"), _i32(cu_rows, (n + 1,), pool._device, "cu_rows")
    pairs = _given_or_new(pairs, (n, 2), pool, table, "pairs", stream)
    missing = _given_or_new(missing, (1,), pool, table, "missing", stream)
    st = _stream(stream)
    wp, wn = pool._workspace(workspace, st, stream)
    rc = _page_calls()[1](pool._at, at, length_at, cu_at, n, blocks, pairs.data_ptr(), missing.data_ptr(), wp, wn, st)
    if rc:
        _check(rc, "floe_kv_reserve")
    return pairs, missing


def floe_kv_trim(pool: KVPool, table, length, window: int = 0, sinks: int = 0, stream=None):
    """Gives back the blocks of `table` that no query behind `length` tokens sees: all behind the end, and with a window those before it
    that hold none of the first `sinks` tokens.  Sequences that go on: a window of 2 or more, which keeps the block that is begun (floe.h)."""
    at, n, blocks = pool._table(table, stream)
    rc = _page_calls()[2](pool._at, at, _i32(length, (n,), pool._device, "length"), n, blocks, _fits(sinks, "sinks"), _fits(window, "window"),
                          _stream(stream))
    if rc:
        _check(rc, "floe_kv_trim")


def floe_kv_compact(pool: KVPool, table, max_moves: int = None, pairs=None, page_map=None, workspace=None, stream=None):
    """Moves the highest used pages to the lowest free ones (max_moves at most: as many as there are pages by default); the pool and `table`
    follow at once.  Returns (pairs int32 [max_moves][2], what floe_kv_copy_pages has to copy; page_map int32 [n_pages], where each page went:
    also those that the caller holds by a count of its own, or by other tables)."""
    at, n, blocks = pool._table(table, stream)
    moves = pool.n_pages if max_moves is None else _fits(int(max_moves), "max_moves")
    pairs = _given_or_new(pairs, (moves, 2), pool, table, "pairs", stream)
    page_map = _given_or_new(page_map, (pool.n_pages,), pool, table, "page_map", stream)
    st = _stream(stream)
    wp, wn = pool._workspace(workspace, st, stream)
    rc = _page_calls()[3](pool._at, at, n, blocks, pairs.data_ptr(), moves, page_map.data_ptr(), wp, wn, st)
    if rc:
        _check(rc, "floe_kv_compact")
    return pairs, page_map


def floe_kv_copy_pages(caches, pairs, stream=None):
    """Copies page pairs[i][0] to page pairs[i][1] (-1: none) in each of the caches, the layers of a model."""
    caches = [caches] if isinstance(caches, KVCache) else list(caches)
    if not caches:
        return
    dev = caches[0]._device
    if any(c._device != dev for c in caches):
        raise ValueError("floe_kv_copy_pages: the caches are on one device")
    _launches_on(dev, stream, "the cache")
    n = _fits(pairs.shape[0], "pairs") if pairs.dim() else 0
    at = _i32(pairs, (n, 2), dev, "pairs")
    rc = _page_calls()[4](b"".join([bytes(c._c) for c in caches]), len(caches), at, n, _stream(stream))
    if rc:
        _check(rc, "floe_kv_copy_pages")


# ---- beam search
_BEAM_DTYPES = {torch.float16: 0, torch.bfloat16: 1, torch.float32: 2}
_BEAM_FIELDS = struct.Struct("6i")
assert _BEAM_FIELDS.size == C.sizeof(_Beam)
_beam_functions = None


def _beam_calls():
    global _beam_functions
    if _beam_functions is None:
        lib, vp, packed = load(), C.c_void_p, C.c_char_p
        select, need = lib["floe_beam_select"], lib["floe_beam_workspace_bytes"]
        select.argtypes = [packed, vp, C.c_int64, vp, vp, vp, vp, vp, vp, vp, C.c_size_t, vp]
        need.argtypes, need.restype = [packed], C.c_size_t
        _beam_functions = select, need
    return _beam_functions


# Scratch of a call: the caller's, or its own from the pool of its stream, given back when the call has been enqueued.  No two calls, and no two
# captured graphs, share an array that outlives them.  Returns the tensor, an address and the bytes behind it.
def _scratch(given, like, nbytes: int, stream):
    if given is None:
        given = _new(like, (nbytes + 256,), torch.uint8, stream)
        return (given, given.data_ptr(), nbytes) if given.data_ptr() % 256 == 0 else (given, *_aligned_ptr(given))
    if given.get_device() != like.get_device():
        raise ValueError(f"workspace: on {given.device}, expected {like.device}")
    return (given, *_aligned_ptr(given))


def _beam_out(t, shape, dtype, like, name, stream):
    if t is None:
        return _new(like, shape, dtype, stream)
    if t.dtype is not dtype or t.shape != shape or not t.is_contiguous() or t.get_device() != like.get_device():
        raise ValueError(f"{name}: expected contiguous {dtype} {shape} on {like.device}, got {t.dtype} {tuple(t.shape)} on {t.device}")
    return t


def _overlap(a, b) -> bool:
    """Whether two contiguous tensors share bytes."""
    x, y = a.data_ptr(), b.data_ptr()
    return x < y + b.numel() * b.element_size() and y < x + a.numel() * a.element_size()


def floe_beam_select(logits, score, take: int = None, done=None, eos: int = -1, score_out=None, parent=None, token=None, done_out=None, workspace=None,
                     stream=None):
    """The `take` best continuations (as many as beams by default) of each group: logits [groups * beams][vocab] fp16, bf16 or fp32 (rows may lie
    anywhere), score fp32 [groups][beams], done uint8 [groups][beams] (rows that offer `eos` alone).  Returns (score, parent, token, done), all
    [groups][take]; parent is the row that a continuation comes from, -1 behind the last one (include/floe.h)."""
    kind, shape, sizes = _BEAM_DTYPES.get(logits.dtype), logits.shape, score.shape
    if kind is None or len(shape) != 2 or len(sizes) != 2 or shape[0] != sizes[0] * sizes[1]:
        raise ValueError(f"floe_beam_select: logits fp16, bf16 or fp32 [groups * beams][vocab], got {logits.dtype} {tuple(shape)}, score {tuple(sizes)}")
    (rows, vocab), (groups, beams), strides = shape, sizes, logits.stride()
    if (vocab > 1 and rows and strides[1] != 1) or (rows > 1 and strides[0] < vocab):
        raise ValueError(f"floe_beam_select: the logits of a row lie one behind the other, and rows apart (strides {strides})")
    _launches_on(logits.get_device(), stream, "floe_beam_select: logits")
    for t, dtype, name in ((score, torch.float32, "score"), (done, torch.uint8, "done")):
        if t is not None:
            _beam_out(t, sizes, dtype, logits, name, stream)
    take = beams if take is None else take
    out = groups, take
    given = (score_out, "score_out"), (parent, "parent"), (token, "token"), (done_out, "done_out")
    score_out = _beam_out(score_out, out, torch.float32, logits, "score_out", stream)
    parent = _beam_out(parent, out, torch.int32, logits, "parent", stream)
    token = _beam_out(token, out, torch.int32, logits, "token", stream)
    done_out = _beam_out(done_out, out, torch.uint8, logits, "done_out", stream)
    for t, name in given:
        if t is not None and any(i is not None and _overlap(t, i) for i in (score, done)):
            raise ValueError(f"floe_beam_select: {name} lies over an input (score and done stay as they are)")
        if t is not None and any(o is not t and _overlap(t, o) for o in (score_out, parent, token, done_out)):
            raise ValueError(f"floe_beam_select: {name} lies over another result")
    b, (call, need) = _BEAM_FIELDS.pack(groups, beams, vocab, take, kind, eos), _beam_calls()
    workspace, wp, wn = _scratch(workspace, logits, need(b), stream)
    rc = call(b, logits.data_ptr(), strides[0] if rows > 1 else vocab, score.data_ptr(), None if done is None else done.data_ptr(), score_out.data_ptr(),
              parent.data_ptr(), token.data_ptr(), done_out.data_ptr(), wp, wn, _stream(stream))
    if rc:
        _check(rc, "floe_beam_select")
    return score_out, parent, token, done_out
