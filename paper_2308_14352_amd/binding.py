"""Thin ctypes binding of libmoeq.so: same names as include/moeq.h, argument marshalling only.

torch is used for device memory and streams; every step of the path runs in the library's HIP
kernels. There is no fallback: if the library is missing the import of a compute call raises.
"""
import ctypes as C
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
# MOEQ_LIB lets a developer point the binding at another build of the same library.
LIB_PATH = os.environ.get("MOEQ_LIB") or os.path.join(_HERE, "libmoeq.so")

MOEQ_OK, MOEQ_EINVAL, MOEQ_EUNSUPPORTED, MOEQ_EWORKSPACE, MOEQ_EDEVICE = range(5)
MOEQ_ACT_RELU, MOEQ_ACT_SWIGLU = 0, 1
MOEQ_F32, MOEQ_BF16, MOEQ_F16 = 0, 1, 2
MOEQ_OUT_CANONICAL, MOEQ_OUT_COLUMNS = 0, 1
MOEQ_IN_CANONICAL, MOEQ_IN_STREAM = 0, 1
MOEQ_KEEP_NONE, MOEQ_KEEP_OWN, MOEQ_KEEP_8 = 0, 1, 8


class MoeqError(RuntimeError):
    def __init__(self, status, what):
        self.status = int(status)
        super().__init__(f"{what}: {status_str(status)} (status {int(status)})")


class moeq_expert(C.Structure):
    _fields_ = [("bits", C.c_int32),
                ("q_in", C.c_void_p), ("s_in", C.c_void_p),
                ("q_gate", C.c_void_p), ("s_gate", C.c_void_p),
                ("q_out", C.c_void_p), ("s_out", C.c_void_p)]


class moeq_layer_desc(C.Structure):
    _fields_ = [("d_model", C.c_int32), ("d_ff", C.c_int32), ("n_experts", C.c_int32),
                ("top_k", C.c_int32), ("group", C.c_int32), ("act", C.c_int32),
                ("renorm", C.c_int32), ("x_dtype", C.c_int32),
                ("router_w", C.c_void_p), ("router_bias", C.c_void_p),
                ("experts", C.POINTER(moeq_expert)), ("out_layout", C.c_int32), ("in_layout", C.c_int32),
                ("group_in", C.c_int32), ("group_out", C.c_int32)]


class moeq_adapters(C.Structure):
    _fields_ = [("n_adapters", C.c_int32), ("rank", C.c_int32), ("d_in", C.c_int32), ("d_out", C.c_int32), ("dtype", C.c_int32),
                ("a", C.c_void_p), ("b", C.c_void_p), ("scale", C.c_void_p)]


class moeq_gated_ffn(C.Structure):
    _fields_ = [("d_model", C.c_int32), ("d_ff", C.c_int32), ("dtype", C.c_int32),
                ("w_in", C.c_void_p), ("w_gate", C.c_void_p), ("w_out", C.c_void_p)]


_lib = None


def lib():
    """Loads libmoeq.so (building it first only if no built library exists)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        from . import build as _build
        _build.build()
    L = C.CDLL(LIB_PATH)
    vp, i32, i64, sz = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t
    L.moe_status_str.restype = C.c_char_p
    L.moe_status_str.argtypes = [C.c_int]
    L.moe_layer_table_bytes.restype = sz
    L.moe_layer_table_bytes.argtypes = [i32]
    L.moe_packed_bytes.restype = sz
    L.moe_packed_bytes.argtypes = [i64, i64, i32, i32, C.POINTER(sz)]
    L.moe_layer_create.restype = C.c_int
    L.moe_layer_create.argtypes = [C.POINTER(moeq_layer_desc), vp, sz, C.POINTER(vp)]
    L.moe_layer_destroy.restype = None
    L.moe_layer_destroy.argtypes = [vp]
    L.moe_layer_profile_kernel.restype = C.c_int
    L.moe_layer_profile_kernel.argtypes = [vp, i32, vp, vp]
    L.moe_workspace_bytes.restype = sz
    L.moe_workspace_bytes.argtypes = [vp, i32]
    L.moe_layer_path.restype = i32
    L.moe_layer_path.argtypes = [vp, i32]
    L.moe_router_topk.restype = C.c_int
    L.moe_router_topk.argtypes = [vp, vp, i32, vp, vp, vp, vp, sz, vp]
    L.moe_expert_ffn_q.restype = C.c_int
    L.moe_expert_ffn_q.argtypes = [vp, i32, vp, i32, vp, i32, vp, vp, sz, vp]
    L.moe_layer_forward.restype = C.c_int
    L.moe_layer_forward.argtypes = [vp, vp, i32, vp, vp, vp, vp, sz, vp]
    L.moe_static_scratch_bytes.restype = sz
    L.moe_static_scratch_bytes.argtypes = []
    L.moe_layer_forward_static.restype = C.c_int
    L.moe_layer_forward_static.argtypes = [vp, vp, i32, vp, vp, vp, vp]
    L.moe_layer_forward_routed.restype = C.c_int
    L.moe_layer_forward_routed.argtypes = [vp, vp, i32, vp, vp, vp, vp, sz, vp]
    L.moe_quantize_pack.restype = C.c_int
    L.moe_quantize_pack.argtypes = [vp, i64, i64, i32, i32, vp, vp, vp]
    L.moe_unpack_codes.restype = C.c_int
    L.moe_unpack_codes.argtypes = [vp, i64, i64, i32, vp, vp]
    L.moe_dequantize.restype = C.c_int
    L.moe_dequantize.argtypes = [vp, vp, i64, i64, i32, i32, vp, vp]
    L.moe_stream_bytes.restype = sz
    L.moe_stream_bytes.argtypes = [i64, i64, i32, i32]
    L.moe_prepare_in.restype = C.c_int
    L.moe_prepare_in.argtypes = [vp, vp, i64, i64, i32, i32, vp, vp]
    L.moe_unprepare_in.restype = C.c_int
    L.moe_unprepare_in.argtypes = [vp, i64, i64, i32, i32, vp, vp, vp]
    for fn in (L.moe_prepare_out, L.moe_unprepare_out):
        fn.restype = C.c_int
        fn.argtypes = [vp, vp, i64, i64, i32, i32, vp, vp, vp]
    f32 = C.c_float
    for name, res, args in (
            ("moe_sort_bytes", sz, [i32, i32, i32]),
            ("moe_sort_pairs", C.c_int, [vp, i32, i32, i32, vp, vp, vp, vp, sz, vp]),
            ("moe_gather_rows", C.c_int, [vp, i32, i32, i32, i32, vp, i64, vp, i64, vp]),
            ("moe_combine_rows", C.c_int, [vp, vp, i32, i32, i32, i32, vp, i64, i32, vp, i64, vp]),
            ("moe_combine_rows_backward", C.c_int, [vp, vp, i32, i32, i32, i32, vp, i64, i32, vp, i64, vp, i64, vp, vp]),
            ("moe_adapters_workspace_bytes", sz, [vp, i32, i32]),
            ("moe_adapters_forward", C.c_int, [vp, vp, i64, vp, i32, vp, i64, i32, vp, i64, vp, sz, vp]),
            ("moe_adapters_backward", C.c_int, [vp, vp, i64, vp, i32, i32, vp, i64, vp, i64, vp, i64, vp, vp, vp, sz, vp]),
            ("moe_distill_workspace_bytes", sz, [i32, i32, i32]),
            ("moe_distill_forward", C.c_int, [vp, i64, i32, i32, i32, vp, vp, i32, f32, vp, vp, vp, vp, sz, vp]),
            ("moe_distill_backward", C.c_int, [vp, i64, i32, i32, i32, vp, vp, i32, f32, vp, vp, vp, vp, i64, vp]),
            ("moe_distill_loss_grad", C.c_int, [vp, i64, i32, i32, i32, vp, vp, i32, f32, vp, vp, vp, i64, vp, sz, vp]),
            ("moe_block_norms_forward", C.c_int, [i32, i32, f32, f32, i32, vp, i64, i32, vp, i64, vp, vp, vp, vp, i64, i32, vp, i64, vp]),
            ("moe_block_norms_workspace_bytes", sz, [i32, i32]),
            ("moe_block_norms_backward", C.c_int, [i32, i32, f32, f32, i32, vp, i64, i32, vp, i64, vp, i64, i32, vp, i64, vp, vp, vp, vp, i64,
                                                   vp, i64, vp, vp, vp, vp, sz, vp]),
            ("moe_pack8", C.c_int, [vp, i64, i32, i32, i32, vp, vp, vp]),
            ("moe_unpack8", C.c_int, [vp, vp, i32, i32, i32, vp, i64, vp]),
            ("moe_gated_ffn_workspace_bytes", sz, [vp, i32, i32, i32, i32]),
            ("moe_gated_ffn_forward", C.c_int, [vp, vp, i64, i32, vp, i64, i32, vp, i64, i32, vp, vp, vp, sz, vp]),
            ("moe_gated_ffn_backward", C.c_int, [vp, vp, i64, vp, vp, i32, vp, i64, i32, vp, vp, vp, i64, vp, vp, vp, vp, sz, vp]),
            ("moe_q8_pitch", i64, [i32]),
            ("moe_quantize_rows", C.c_int, [vp, i64, i32, i32, i32, vp, vp, vp]),
            ("moe_matmul_q8_workspace_bytes", sz, [i32, i32, i32]),
            ("moe_matmul_q8", C.c_int, [vp, vp, i32, vp, vp, i32, i32, vp, i64, i32, vp, i64, vp, sz, vp])):
        fn = getattr(L, name)
        fn.restype, fn.argtypes = res, args
    _lib = L
    return L


EXPORTS = ["moe_status_str", "moe_layer_profile_kernel", "moe_layer_table_bytes", "moe_packed_bytes", "moe_layer_create",
           "moe_layer_destroy", "moe_workspace_bytes", "moe_layer_path", "moe_router_topk", "moe_expert_ffn_q",
           "moe_layer_forward", "moe_layer_forward_routed", "moe_layer_forward_static", "moe_static_scratch_bytes", "moe_quantize_pack", "moe_unpack_codes", "moe_dequantize", "moe_prepare_out",
           "moe_unprepare_out", "moe_prepare_in", "moe_unprepare_in", "moe_stream_bytes",
           "moe_sort_bytes", "moe_sort_pairs", "moe_gather_rows", "moe_combine_rows", "moe_combine_rows_backward",
           "moe_adapters_workspace_bytes", "moe_adapters_forward", "moe_adapters_backward",
           "moe_distill_workspace_bytes", "moe_distill_forward", "moe_distill_backward", "moe_distill_loss_grad",
           "moe_block_norms_forward", "moe_block_norms_workspace_bytes", "moe_block_norms_backward", "moe_pack8", "moe_unpack8",
           "moe_gated_ffn_workspace_bytes", "moe_gated_ffn_forward", "moe_gated_ffn_backward", "moe_q8_pitch", "moe_quantize_rows",
           "moe_matmul_q8_workspace_bytes", "moe_matmul_q8"]


def status_str(st):
    return lib().moe_status_str(int(st)).decode()


def _check(st, what):
    if st != MOEQ_OK:
        raise MoeqError(st, what)


def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream(stream):
    # (the handle of the current stream without a Stream object around it: 2.8 -> 0.2 us of a call of about 15)
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice()) if stream is None else stream.cuda_stream


MOEQ_KERNEL_FFN_IN, MOEQ_KERNEL_FFN_OUT, MOEQ_KERNEL_FUSED = 1, 2, 3
MOEQ_PATH_TWO_KERNELS, MOEQ_PATH_ONE_KERNEL, MOEQ_PATH_ONE_KERNEL_MX, MOEQ_PATH_GROUPED_GEMM, MOEQ_PATH_STREAM = 0, 1, 2, 3, 4


def moe_layer_profile_kernel(layer, which, start_event=None, stop_event=None):
    """which: 0 (off) or one of the MOEQ_KERNEL_* ids; events are raw hipEvent_t handles (ints)."""
    _check(lib().moe_layer_profile_kernel(layer.handle, int(which), C.c_void_p(start_event), C.c_void_p(stop_event)),
           "moe_layer_profile_kernel")


def moe_packed_bytes(rows, cols, bits, group):
    """(code bytes, scale bytes) of a packed [rows][cols] matrix; (0, 0) for an invalid shape."""
    sb = C.c_size_t(0)
    qb = lib().moe_packed_bytes(rows, cols, bits, group, C.byref(sb))
    return int(qb), int(sb.value)


def moe_layer_table_bytes(n_experts):
    return int(lib().moe_layer_table_bytes(n_experts))


def moe_quantize_pack(w, bits, group, stream=None):
    """w: device fp32 [rows][cols] -> (codes uint8 [rows][cols*bits/8], scales int16-typed fp16 bits [rows][cols/group])."""
    assert w.is_cuda and w.dtype == torch.float32 and w.is_contiguous() and w.dim() == 2
    rows, cols = w.shape
    qb, sb = moe_packed_bytes(rows, cols, bits, group)
    if qb == 0:
        raise MoeqError(MOEQ_EINVAL, "moe_quantize_pack")
    q = torch.empty((rows, cols * bits // 8), dtype=torch.uint8, device=w.device)
    s = torch.empty((rows, cols // group), dtype=torch.float16, device=w.device)
    _check(lib().moe_quantize_pack(_ptr(w), rows, cols, bits, group, _ptr(q), _ptr(s), _stream(stream)),
           "moe_quantize_pack")
    return q, s


def moe_unpack_codes(q, cols, bits, stream=None):
    rows = q.shape[0]
    out = torch.empty((rows, cols), dtype=torch.int8, device=q.device)
    _check(lib().moe_unpack_codes(_ptr(q), rows, cols, bits, _ptr(out), _stream(stream)), "moe_unpack_codes")
    return out


def moe_dequantize(q, s, cols, bits, group, stream=None):
    rows = q.shape[0]
    out = torch.empty((rows, cols), dtype=torch.float32, device=q.device)
    _check(lib().moe_dequantize(_ptr(q), _ptr(s), rows, cols, bits, group, _ptr(out), _stream(stream)),
           "moe_dequantize")
    return out


def moe_prepare_out(q, s, cols, bits, group, stream=None):
    """Canonical W_out (codes [rows][cols*bits/8], scales [rows][cols/group]) -> dword-column-major copies
    (codes uint8 [cols*bits/32][rows*4], scales [cols/group][rows])."""
    rows = q.shape[0]
    qc = torch.empty((cols * bits // 32, rows * 4), dtype=torch.uint8, device=q.device)
    sc = torch.empty((cols // group, rows), dtype=torch.float16, device=q.device)
    _check(lib().moe_prepare_out(_ptr(q), _ptr(s), rows, cols, bits, group, _ptr(qc), _ptr(sc), _stream(stream)),
           "moe_prepare_out")
    return qc, sc


def moe_unprepare_out(qc, sc, cols, bits, group, stream=None):
    """Inverse of moe_prepare_out."""
    rows = sc.shape[1]
    q = torch.empty((rows, cols * bits // 8), dtype=torch.uint8, device=qc.device)
    s = torch.empty((rows, cols // group), dtype=torch.float16, device=qc.device)
    _check(lib().moe_unprepare_out(_ptr(qc), _ptr(sc), rows, cols, bits, group, _ptr(q), _ptr(s), _stream(stream)),
           "moe_unprepare_out")
    return q, s


def moe_stream_bytes(rows, cols, bits, group):
    return int(lib().moe_stream_bytes(rows, cols, bits, group))


def moe_prepare_in(q, s, cols, bits, group, stream=None):
    """Canonical W_in / W_gate (codes [rows][cols*bits/8], scales [rows][cols/group]) -> one stream buffer (uint8)."""
    rows = q.shape[0]
    n = moe_stream_bytes(rows, cols, bits, group)
    if n == 0:
        raise MoeqError(MOEQ_EUNSUPPORTED, "moe_prepare_in")
    buf = torch.empty(n, dtype=torch.uint8, device=q.device)
    _check(lib().moe_prepare_in(_ptr(q), _ptr(s), rows, cols, bits, group, _ptr(buf), _stream(stream)), "moe_prepare_in")
    return buf


def moe_unprepare_in(buf, rows, cols, bits, group, stream=None):
    """Inverse of moe_prepare_in: (codes, scales) in the canonical format."""
    q = torch.empty((rows, cols * bits // 8), dtype=torch.uint8, device=buf.device)
    s = torch.empty((rows, cols // group), dtype=torch.float16, device=buf.device)
    _check(lib().moe_unprepare_in(_ptr(buf), rows, cols, bits, group, _ptr(q), _ptr(s), _stream(stream)),
           "moe_unprepare_in")
    return q, s


class PackedExpert:
    """Device tensors of one expert in the boundary format (keeps them alive). q_out/s_out are in the
    layout the owning Layer is created with."""

    def __init__(self, bits, q_in, s_in, q_out, s_out, q_gate=None, s_gate=None):
        self.bits = int(bits)
        self.q_in, self.s_in, self.q_out, self.s_out = q_in, s_in, q_out, s_out
        self.q_gate, self.s_gate = q_gate, s_gate

    def with_out_columns(self, d_ff, group):
        """A copy of this expert (canonical W_out) whose W_out is in the dword-column-major layout."""
        qc, sc = moe_prepare_out(self.q_out, self.s_out, d_ff, self.bits, group)
        return PackedExpert(self.bits, self.q_in, self.s_in, qc, sc, self.q_gate, self.s_gate)

    def with_stream_layout(self, d_model, d_ff, group):
        """A copy of this expert (canonical) for a MOEQ_IN_STREAM layer: W_in / W_gate as stream buffers (their
        scales inside), W_out in the dword-column-major layout."""
        qc, sc = moe_prepare_out(self.q_out, self.s_out, d_ff, self.bits, group)
        b_in = moe_prepare_in(self.q_in, self.s_in, d_model, self.bits, group)
        b_gate = None if self.q_gate is None else moe_prepare_in(self.q_gate, self.s_gate, d_model, self.bits, group)
        return PackedExpert(self.bits, b_in, None, qc, sc, b_gate, None)

    def nbytes(self):
        ts = [self.q_in, self.s_in, self.q_out, self.s_out, self.q_gate, self.s_gate]
        return sum(t.numel() * t.element_size() for t in ts if t is not None)

    def c_struct(self):
        return moeq_expert(self.bits, _ptr(self.q_in), _ptr(self.s_in), _ptr(self.q_gate), _ptr(self.s_gate),
                           _ptr(self.q_out), _ptr(self.s_out))


class Layer:
    """Owner of a moeq_layer handle and of the device tensors it borrows."""

    def __init__(self, d_model, d_ff, top_k, group, act, renorm, x_dtype, router_w, router_bias, experts,
                 out_layout=MOEQ_OUT_CANONICAL, in_layout=MOEQ_IN_CANONICAL, group_in=0, group_out=0):
        self.out_layout = out_layout
        self.in_layout = in_layout
        self.group_in, self.group_out = group_in or group, group_out or group
        self.d_model, self.d_ff, self.top_k, self.group = d_model, d_ff, top_k, group
        self.n_experts = len(experts)
        self.experts = list(experts)
        self.router_w, self.router_bias = router_w, router_bias
        self.x_dtype = x_dtype
        dev = router_w.device
        self._table = torch.empty(max(moe_layer_table_bytes(self.n_experts), 16), dtype=torch.uint8, device=dev)
        arr = (moeq_expert * self.n_experts)(*[e.c_struct() for e in self.experts])
        desc = moeq_layer_desc(d_model, d_ff, self.n_experts, top_k, group, act, int(bool(renorm)), x_dtype,
                               _ptr(router_w), _ptr(router_bias), arr, out_layout, in_layout, group_in, group_out)
        h = C.c_void_p()
        _check(lib().moe_layer_create(C.byref(desc), _ptr(self._table), self._table.numel(), C.byref(h)),
               "moe_layer_create")
        self._h = h
        self._ws = None

    def __del__(self):
        h = getattr(self, "_h", None)
        if h and callable(lib):          # at interpreter shutdown the module's names may already be gone
            lib().moe_layer_destroy(h)
            self._h = None

    @property
    def handle(self):
        return self._h

    def workspace_bytes(self, max_tokens):
        return int(lib().moe_workspace_bytes(self._h, max_tokens))

    def path(self, n_tokens):
        """MOEQ_PATH_* constant: the kernels a layer call with n_tokens tokens runs."""
        return int(lib().moe_layer_path(self._h, n_tokens))

    def workspace(self, n_tokens):
        need = self.workspace_bytes(n_tokens)
        if self._ws is None or self._ws.numel() < need:
            self._ws = torch.empty(need, dtype=torch.uint8, device=self.router_w.device)
        return self._ws


def moe_router_topk(layer, x, want_probs=False, ws=None, stream=None):
    T = x.shape[0]
    dev = x.device
    if ws is None:
        ws = layer.workspace(T)
    idx = torch.empty((T, layer.top_k), dtype=torch.int32, device=dev)
    gate = torch.empty((T, layer.top_k), dtype=torch.float32, device=dev)
    probs = torch.empty((T, layer.n_experts), dtype=torch.float32, device=dev) if want_probs else None
    _check(lib().moe_router_topk(layer.handle, _ptr(x), T, _ptr(idx), _ptr(gate), _ptr(probs), _ptr(ws), ws.numel(),
                                 _stream(stream)), "moe_router_topk")
    return (idx, gate, probs) if want_probs else (idx, gate)


def moe_expert_ffn_q(layer, expert, x, gate=None, y=None, accumulate=False, ws=None, stream=None):
    T = x.shape[0]
    if y is None:
        y = torch.empty((T, layer.d_model), dtype=torch.float32, device=x.device)
    if ws is None:
        ws = layer.workspace(T)
    _check(lib().moe_expert_ffn_q(layer.handle, expert, _ptr(x), T, _ptr(gate), int(bool(accumulate)), _ptr(y),
                                  _ptr(ws), ws.numel(), _stream(stream)), "moe_expert_ffn_q")
    return y


def moe_layer_forward(layer, x, y=None, want_routing=False, ws=None, stream=None):
    T = x.shape[0]
    dev = x.device
    if y is None:
        y = torch.empty((T, layer.d_model), dtype=torch.float32, device=dev)
    idx = gate = None
    if want_routing:
        idx = torch.empty((T, layer.top_k), dtype=torch.int32, device=dev)
        gate = torch.empty((T, layer.top_k), dtype=torch.float32, device=dev)
    if ws is None:
        ws = layer.workspace(T)
    _check(lib().moe_layer_forward(layer.handle, _ptr(x), T, _ptr(y), _ptr(idx), _ptr(gate), _ptr(ws), ws.numel(),
                                   _stream(stream)), "moe_layer_forward")
    return (y, idx, gate) if want_routing else y


def moe_static_scratch_bytes():
    return int(lib().moe_static_scratch_bytes())


def moe_layer_forward_static(layer, x, y=None, want_routing=False, stream=None):
    """moe_layer_forward without a workspace argument (the library's fixed scratch array is used)."""
    T = x.shape[0]
    dev = x.device
    if y is None:
        y = torch.empty((T, layer.d_model), dtype=torch.float32, device=dev)
    idx = gate = None
    if want_routing:
        idx = torch.empty((T, layer.top_k), dtype=torch.int32, device=dev)
        gate = torch.empty((T, layer.top_k), dtype=torch.float32, device=dev)
    _check(lib().moe_layer_forward_static(layer.handle, _ptr(x), T, _ptr(y), _ptr(idx), _ptr(gate), _stream(stream)),
           "moe_layer_forward_static")
    return (y, idx, gate) if want_routing else y


def moe_layer_forward_routed(layer, x, idx, gate, y=None, ws=None, stream=None):
    """The layer with the routing given by the caller: idx [T][top_k] int32, gate [T][top_k] fp32 (device)."""
    T = x.shape[0]
    if y is None:
        y = torch.empty((T, layer.d_model), dtype=torch.float32, device=x.device)
    if ws is None:
        ws = layer.workspace(T)
    _check(lib().moe_layer_forward_routed(layer.handle, _ptr(x), T, _ptr(idx), _ptr(gate), _ptr(y), _ptr(ws),
                                          ws.numel(), _stream(stream)), "moe_layer_forward_routed")
    return y


# ---- operators beside the layer ----------------------------------------------------------------------------------------------
# The checks of their tensors, the memory of their outputs and the C ABI calls are in the extension module _calls (csrc/calls.cpp):
# most of these calls are a kernel or two of a few microseconds. Nothing is recorded for autograd: tensors that require gradients are taken as
# they are, and gradients come from the backward calls.

_DTYPES = {torch.float32: MOEQ_F32, torch.bfloat16: MOEQ_BF16, torch.float16: MOEQ_F16}
_native = None


def _stream_on(device):
    """The handle of the current stream, where `device` (that of a call's tensors) is the current one."""
    if torch._C._cuda_getDevice() != device:
        raise MoeqError(MOEQ_EINVAL, "tensors on a device that is not the current one")
    return torch._C._cuda_getCurrentRawStream(device)


def _load():
    global _native
    L = lib()
    if not os.path.exists(os.path.join(_HERE, "_calls.so")):
        from . import build as _build
        _build.build()
    from . import _calls
    names = ("moe_sort_bytes", "moe_sort_pairs", "moe_gather_rows", "moe_combine_rows", "moe_combine_rows_backward",
             "moe_adapters_workspace_bytes", "moe_adapters_forward", "moe_adapters_backward", "moe_distill_workspace_bytes",
             "moe_distill_forward", "moe_distill_backward", "moe_distill_loss_grad", "moe_block_norms_forward",
             "moe_block_norms_workspace_bytes", "moe_block_norms_backward", "moe_pack8", "moe_unpack8", "moe_gated_ffn_workspace_bytes",
             "moe_gated_ffn_forward", "moe_gated_ffn_backward", "moe_q8_pitch", "moe_quantize_rows", "moe_matmul_q8_workspace_bytes",
             "moe_matmul_q8")
    _calls.bind(MoeqError, _stream_on, *[C.cast(getattr(L, n), C.c_void_p).value for n in names])
    _native = _calls
    return _calls


def _need(ok, what):
    if not ok:
        raise MoeqError(MOEQ_EINVAL, what)


class PairSort:
    """The order of a call's (token, choice) pairs by expert: int32 tensors offsets [n_experts + 1], order [pairs] (the pair in
    every place) and slot [pairs] (the place of every pair); pairs without an expert come last, as ~pair and ~place."""

    __slots__ = ("offsets", "order", "slot", "n_tokens", "top_k", "n_experts")

    def __init__(self, offsets, order, slot, n_tokens, top_k, n_experts):
        self.offsets, self.order, self.slot = offsets, order, slot
        self.n_tokens, self.top_k, self.n_experts = n_tokens, top_k, n_experts


def moe_sort_pairs(idx, n_experts, stream=None):
    """idx: device int32 [T][k], the experts that a router chose (outside [0, n_experts): none) -> PairSort."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return moe_sort_pairs(idx, n_experts)
    return PairSort(*(_native or _load()).sort_pairs(idx, n_experts))


def moe_gather_rows(sort, x, rows=None, stream=None):
    """The tokens' rows [T][d] in the order of the sort: rows [pairs][d] (zeros for pairs without an expert)."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return moe_gather_rows(sort, x, rows)
    return (_native or _load()).gather_rows(sort.slot, sort.n_tokens, sort.top_k, x, rows)


def moe_combine_rows(sort, rows, gate=None, dtype=None, y=None, stream=None):
    """Rows in the order of the sort back to tokens: y[t] = sum of gate[t][j] * row (gate None: ones, the gradient of
    moe_gather_rows). dtype: of y, the rows' own (default) or fp32."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return moe_combine_rows(sort, rows, gate, dtype, y)
    return (_native or _load()).combine_rows(sort.slot, sort.n_tokens, sort.top_k, rows, gate, dtype, y)


def moe_combine_rows_backward(sort, dy, rows, gate=None, drows=None, stream=None):
    """The gradient of moe_combine_rows: (drows [pairs][d] in the rows' dtype, dgate [T][k] fp32)."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return moe_combine_rows_backward(sort, dy, rows, gate, drows)
    return (_native or _load()).combine_rows_backward(sort.slot, sort.n_tokens, sort.top_k, dy, rows, gate, drows)


class Adapters:
    """Low-rank adapters a [n][rank][d_in], b [n][d_out][rank] (one dtype) with scale [n] fp32: device tensors that are borrowed,
    not copied, so that an update in place is seen by the next call."""

    def __init__(self, a, b, scale):
        what = "Adapters"
        _need(a.dim() == 3 and b.dim() == 3 and scale.dim() == 1 and a.dtype in _DTYPES and b.dtype is a.dtype, what)
        n, r, d_in = a.shape
        _need(b.shape[0] == n and b.shape[2] == r and scale.shape[0] == n and scale.dtype is torch.float32, what)
        _need(all(t.is_cuda and t.is_contiguous() and t.device == a.device for t in (a, b, scale)), what)
        self.a, self.b, self.scale = a, b, scale
        self.n_adapters, self.rank, self.d_in, self.d_out, self.dtype = n, r, d_in, b.shape[1], a.dtype
        self._desc = moeq_adapters(n, r, d_in, self.d_out, _DTYPES[a.dtype], a.data_ptr(), b.data_ptr(), scale.data_ptr())
        self.handle = C.addressof(self._desc)
        self._ws = None               # the last call's own workspace, held until the next one

    def workspace_bytes(self, max_tokens, backward=False):
        return int(lib().moe_adapters_workspace_bytes(self.handle, max_tokens, int(backward)))

    def workspace(self, max_tokens, backward=False):
        """A workspace for calls of up to max_tokens rows, for callers who pass one (`ws`) and order the calls that share it."""
        return torch.empty(max(self.workspace_bytes(max_tokens, backward), 16), dtype=torch.uint8, device=self.a.device)


def moe_adapters_forward(adapters, x, ids, base=None, y=None, ws=None, stream=None):
    """y[t] = base[t] + scale_a B_a A_a x[t] with a = ids[t] (int32; outside [0, n): no adapter). base: [T][d_out] or None
    (zeros), may be y itself. y: in the adapters' dtype or fp32 (default: the base's, or the adapters'). ws: a workspace that the
    caller keeps; calls that share one have to be ordered. Without it a call has its own."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return moe_adapters_forward(adapters, x, ids, base, y, ws)
    y, used = (_native or _load()).adapters_forward(adapters.handle, x, ids, base, y, ws, adapters.a)
    if ws is None:
        adapters._ws = used
    return y


def moe_adapters_backward(adapters, x, ids, dy, dx_base=None, dx=None, want_dx=True, ws=None, stream=None):
    """The gradient of moe_adapters_forward: (dx [T][d_in] in dy's dtype, dA [n][rank][d_in] fp32, dB [n][d_out][rank] fp32).
    dx_base: added to dx (the gradient through the shared projection), may be dx itself."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return moe_adapters_backward(adapters, x, ids, dy, dx_base, dx, want_dx, ws)
    dx, dA, dB, used = (_native or _load()).adapters_backward(adapters.handle, x, ids, dy, dx_base, dx, bool(want_dx), ws, adapters.a)
    if ws is None:
        adapters._ws = used
    return dx, dA, dB


def moe_distill_forward(logits, top_idx, top_logits, temperature=1.0, weight=None, stream=None):
    """Distillation from a teacher's top logits [T][K] fp32 at top_idx [T][K] int32 (outside [0, V): no entry): (loss [T], lse [T])
    with loss = w tau^2 KL(softmax(top_logits / tau) || softmax(logits / tau)) and lse = log sum exp(logits / tau)."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return moe_distill_forward(logits, top_idx, top_logits, temperature, weight)
    return (_native or _load()).distill_forward(logits, top_idx, top_logits, temperature, weight)


def moe_distill_backward(logits, top_idx, top_logits, lse, dloss, temperature=1.0, weight=None, dlogits=None, stream=None):
    """dlogits [T][V] in the logits' dtype from the forward's lse and the gradients of the losses, both [T] fp32."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return moe_distill_backward(logits, top_idx, top_logits, lse, dloss, temperature, weight, dlogits)
    return (_native or _load()).distill_backward(logits, top_idx, top_logits, temperature, weight, lse, dloss, dlogits)


def moe_distill_loss_grad(logits, top_idx, top_logits, temperature=1.0, weight=None, dlogits=None, stream=None):
    """(loss [T], the gradient of the losses' sum with respect to the logits [T][V]) in one call."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return moe_distill_loss_grad(logits, top_idx, top_logits, temperature, weight, dlogits)
    return (_native or _load()).distill_loss_grad(logits, top_idx, top_logits, temperature, weight, dlogits)


def moe_block_norms_forward(f, r, gate=None, w_after=None, w_before=None, residual_scale=1.0, eps=1e-5, dtype=None, y=None, n=None,
                            stream=None):
    """The norms around a block: y = residual_scale r + gate N(f; w_after) and n = N(y; w_before) with N(v; w) = v / sqrt(mean v^2 + eps) w
    over the rows of f (the block's output) and r (the residual), [T][d]: (y in r's dtype, n in `dtype`, r's by default). gate [T],
    w_after [d] and w_before [d] are fp32; without w_after f itself is added, without w_before n is None. y may be r, n may be f."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return moe_block_norms_forward(f, r, gate, w_after, w_before, residual_scale, eps, dtype, y, n)
    return (_native or _load()).block_norms_forward(f, r, gate, w_after, w_before, residual_scale, eps, dtype, y, n)


def moe_block_norms_backward(f, y, dy, dn=None, gate=None, w_after=None, w_before=None, residual_scale=1.0, eps=1e-5, df=None, dr=None,
                             stream=None):
    """The gradient of moe_block_norms_forward from f, the forward's y and the gradients of y and n (y and dn may be None without
    w_before): (df, dr, dgate [T], dw_after [d], dw_before [d]), the last three fp32 and None where their input is."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return moe_block_norms_backward(f, y, dy, dn, gate, w_after, w_before, residual_scale, eps, df, dr)
    return (_native or _load()).block_norms_backward(f, y, dy, dn, gate, w_after, w_before, residual_scale, eps, df, dr)


class Packed8:
    """A tensor kept in 8 bits: codes int8 [..., d] and exps int8 [..., ceil(d / 32)], one power of two for 32 columns of a row;
    dtype: of the tensor it was."""

    __slots__ = ("codes", "exps", "dtype")

    def __init__(self, codes, exps, dtype):
        self.codes, self.exps, self.dtype = codes, exps, dtype

    @property
    def shape(self):
        return self.codes.shape

    def nbytes(self):
        return self.codes.numel() + self.exps.numel()


def moe_pack8(x, packed=None, stream=None):
    """x [T][d] -> Packed8, 33/64 of the bytes of 16-bit elements. A block with a NaN or an infinity comes back as NaN. packed: a
    Packed8 of this shape and dtype that is written again."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return moe_pack8(x, packed)
    _need(packed is None or packed.dtype is x.dtype, "moe_pack8")
    codes, exps = (_native or _load()).pack8(x, packed and packed.codes, packed and packed.exps)
    return packed or Packed8(codes, exps, x.dtype)


def moe_unpack8(packed, x=None, stream=None):
    """The tensor in its dtype: the values that the codes stand for, exactly. x: rows [T][d] to write to."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return moe_unpack8(packed, x)
    return (_native or _load()).unpack8(packed.codes, packed.exps, packed.dtype, x)


class GatedFfn:
    """The weights of a gated feed-forward block, w_in and w_gate [d_ff][d_model] and w_out [d_model][d_ff] of one dtype: device
    tensors that are borrowed, not copied, so that an update in place is seen by the next call."""

    def __init__(self, w_in, w_gate, w_out):
        what = "GatedFfn"
        _need(all(t.dim() == 2 and t.dtype in _DTYPES and t.dtype is w_in.dtype for t in (w_in, w_gate, w_out)), what)
        f, d = w_in.shape
        _need(tuple(w_gate.shape) == (f, d) and tuple(w_out.shape) == (d, f) and f > 0 and d > 0, what)
        _need(all(t.is_cuda and t.is_contiguous() and t.device == w_in.device for t in (w_in, w_gate, w_out)), what)
        self.w_in, self.w_gate, self.w_out = w_in, w_gate, w_out
        self.d_model, self.d_ff, self.dtype = d, f, w_in.dtype
        self._desc = moeq_gated_ffn(d, f, _DTYPES[w_in.dtype], w_in.data_ptr(), w_gate.data_ptr(), w_out.data_ptr())
        self.handle = C.addressof(self._desc)

    def workspace_bytes(self, max_tokens, backward=False, x_packed=False, keep=None):
        return int(lib().moe_gated_ffn_workspace_bytes(self.handle, max_tokens, int(backward), int(x_packed), _keep(keep)))

    def workspace(self, max_tokens, backward=False, x_packed=False, keep=None):
        """A workspace for calls of up to max_tokens rows, for callers who pass one (`ws`) and order the calls that share it."""
        return torch.empty(max(self.workspace_bytes(max_tokens, backward, x_packed, keep), 16), dtype=torch.uint8, device=self.w_in.device)


def _keep(keep):
    _need(keep is None or keep == "own" or keep == 8, "keep: None, \"own\" or 8")
    return MOEQ_KEEP_NONE if keep is None else MOEQ_KEEP_OWN if keep == "own" else MOEQ_KEEP_8


def moe_gated_ffn_forward(ffn, x, keep=None, base=None, dtype=None, y=None, ws=None, stream=None):
    """y = base + (silu(x w_in^T) * (x w_gate^T)) w_out^T, x [T][d_model] in the weights' dtype. base: [T][d_model] or None (zeros), may
    be y itself; y in the weights' dtype or fp32 (`dtype`; default: the base's, or the weights'). keep: what the backward pass finds of
    the products a = x w_in^T and b = x w_gate^T: None (y alone is returned), "own" ((y, ab [2][T][d_ff])) or 8 ((y, ab as Packed8))."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return moe_gated_ffn_forward(ffn, x, keep, base, dtype, y, ws)
    y, ab, exps = (_native or _load()).gated_ffn_forward(ffn.handle, x, base, dtype, y, _keep(keep), ws, ffn.w_in)
    if keep is None:
        return y
    return y, ab if keep == "own" else Packed8(ab, exps, x.dtype)


def moe_gated_ffn_backward(ffn, x, dy, ab=None, dx=None, want_dx=True, ws=None, stream=None):
    """The gradient of moe_gated_ffn_forward: (dx [T][d_model], dw_in, dw_gate, dw_out) in the weights' dtype. x: the forward's, or a
    Packed8 of it. ab: what the forward pass kept (a tensor or a Packed8), None: computed again."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return moe_gated_ffn_backward(ffn, x, dy, ab, dx, want_dx, ws)
    x8, ab8 = isinstance(x, Packed8), isinstance(ab, Packed8)
    _need((not x8 or x.dtype is ffn.dtype) and (not ab8 or ab.dtype is ffn.dtype), "moe_gated_ffn_backward")
    keep = MOEQ_KEEP_NONE if ab is None else MOEQ_KEEP_8 if ab8 else MOEQ_KEEP_OWN
    return (_native or _load()).gated_ffn_backward(ffn.handle, x.codes if x8 else x, x.exps if x8 else None, dy, keep, ab.codes if ab8 else ab,
                                                   ab.exps if ab8 else None, dx, bool(want_dx), ws, ffn.w_in)


class QuantRows:
    """Rows of k codes int8 with a scale each (value = code * scale): codes [n][pitch], pitch = k up to a multiple of 128 with zeros
    behind column k, scale [n] fp32. Codes [n][k] of another pitch are copied into such rows once, here; with the right one they are
    borrowed."""

    def __init__(self, codes, scale, k=None):
        what = "QuantRows"
        _need(codes.dim() == 2 and codes.dtype is torch.int8 and scale.dim() == 1 and scale.dtype is torch.float32, what)
        _need(codes.is_cuda and scale.is_cuda and scale.is_contiguous() and scale.device == codes.device, what)
        n, width = codes.shape
        k = width if k is None else k
        pitch = (k + 127) // 128 * 128
        _need(scale.shape[0] == n and k > 0 and width in (k, pitch), what)
        if width != pitch or not codes.is_contiguous() or codes.data_ptr() % 16:
            wide = torch.zeros((n, pitch), dtype=torch.int8, device=codes.device)
            wide[:, :k] = codes[:, :k]
            codes = wide
        self.codes, self.scale, self.k = codes, scale, k

    @classmethod
    def _of(cls, codes, scale, k):
        rows = cls.__new__(cls)
        rows.codes, rows.scale, rows.k = codes, scale, k
        return rows


def moe_quantize_rows(x, stream=None):
    """x [T][k] -> QuantRows: scale = max |x[t]| / 127, code = rint(x / scale). A row with a NaN or an infinity has the scale NaN."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return moe_quantize_rows(x)
    codes, scale = (_native or _load()).quantize_rows(x)
    return QuantRows._of(codes, scale, x.shape[1])


def moe_matmul_q8(rows, weights, base=None, dtype=None, y=None, stream=None):
    """y[t][n] = base[t][n] + the product of row t of `rows` and row n of `weights` (both QuantRows of the same k): whole numbers summed
    exactly, times both scales. base: [T][n] or None (zeros), may be y itself; y in `dtype` (default: the base's, or fp32)."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return moe_matmul_q8(rows, weights, base, dtype, y)
    _need(rows.k == weights.k, "moe_matmul_q8")
    return (_native or _load()).matmul_q8(rows.k, rows.codes, rows.scale, weights.codes, weights.scale, base, dtype, y)
