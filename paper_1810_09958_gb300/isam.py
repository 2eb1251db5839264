"""Thin Python binding of libisam.so (include/isam.h): argument marshalling only.

Each function takes torch tensors that already live on the current CUDA
device, checks dtype/shape/contiguity, points the library at torch's current
stream and passes raw device pointers through the C ABI.  Every step of the
computation runs in the library's CUDA kernels; there is no fallback.  If the
library has not been built, loading it raises.
"""
from __future__ import annotations

import ctypes
import os
import re
import threading

PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(PKG, "libisam.so")
HEADER = os.path.join(os.path.dirname(PKG), "include", "isam.h")

ISAM_OK, ISAM_ERR_INVALID_ARG, ISAM_ERR_UNSUPPORTED, ISAM_ERR_CUDA, ISAM_ERR_TIMEOUT = range(5)

_lock = threading.Lock()
_lib = None


class IsamError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"isam error {code}: {msg}")
        self.code = code


def declared_functions() -> list[str]:
    """Names of every function declared in include/isam.h."""
    with open(HEADER) as f:
        text = f.read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    return sorted(set(re.findall(r"\b(isam_[a-z0-9_]+)\s*\(", text)))


def load():
    """Loads libisam.so (raises if it has not been built)."""
    global _lib
    with _lock:
        if _lib is not None:
            return _lib
        if not os.path.exists(LIB_PATH):
            raise ImportError(
                f"{LIB_PATH} is missing: build it with `python -c 'import __graft_entry__ as g; g.build()'`")
        lib = ctypes.CDLL(LIB_PATH)
        i, f, P = ctypes.c_int, ctypes.c_float, ctypes.c_void_p
        lib.isam_version.argtypes = []
        lib.isam_set_stream.argtypes = [P]
        lib.isam_sync.argtypes = []
        lib.isam_last_error_string.argtypes = []
        lib.isam_last_error_string.restype = ctypes.c_char_p
        lib.isam_shutdown.argtypes = []
        lib.isam_gemm.argtypes = [i, i, i, i, i, f, P, P, f, P]
        lib.isam_gemm_plan_info.argtypes = [i, i, i, i, i, f, P]
        lib.isam_gemm_plan_info2.argtypes = [i, i, i, i, i, f, P]
        lib.isam_gemm_grouped.argtypes = [i, P, P, P, P, P, P, P, P, P, P]
        lib.isam_gemm_fp8.argtypes = [i, i, i, f, P, P, f, P]
        lib.isam_gemm_grouped_fp8.argtypes = [i, P, P, P, P, P, P, P, P]
        lib.isam_gemm_mxfp8.argtypes = [i, i, i, f, P, P, P, P, f, P]
        lib.isam_gemm_grouped_mxfp8.argtypes = [i, P, P, P, P, P, P, P, P, P, P]
        lib.isam_gru_forward.argtypes = [i, i, i, P, P, P, P, P, P]
        lib.isam_gru_forward_reset_before.argtypes = [i, i, i, P, P, P, P, P, P]
        lib.isam_gru_forward_stack.argtypes = [i, i, i, i, i, P, P, P, P, P, P]
        lib.isam_dwsep_conv.argtypes = [i, i, i, i, i, P, P, P, P]
        lib.isam_depthwise_conv3x3.argtypes = [i, i, i, i, P, P, P]
        lib.isam_dwsep_plan_info.argtypes = [i, i, i, P]
        lib.isam_dwsep_plan_for.argtypes = [i, i, i, i, P]
        lib.isam_gemm_plan_for.argtypes = [i, i, i, i, i, f, i, i, P, P]
        lib.isam_gru_plan_info.argtypes = [i, i, i, i, P]
        lib.isam_gru_plan_for.argtypes = [i, i, i, i, i, i, P]
        lib.isam_glr_forward.argtypes = [i, i, i, i, P, P, P, i, P, P]
        lib.isam_glr_backward.argtypes = [i, i, i, i, P, P, P, i, P, P, P, P, P]
        lib.isam_glr_step.argtypes = [i, i, i, i, P, P, P, P, i, P]
        lib.isam_glu_forward.argtypes = [i, i, i, i, P, P, P]
        lib.isam_glu_backward_workspace.argtypes = [i, i, i, P]
        lib.isam_glu_backward.argtypes = [i, i, i, i, P, P, P, P, P, P]
        lib.isam_w4_pack.argtypes = [i, i, i, P, P, P, P]
        lib.isam_gemv_w4.argtypes = [i, i, i, i, P, P, P, P]
        for name in ("isam_version", "isam_set_stream", "isam_sync", "isam_shutdown", "isam_gemm",
                     "isam_gemm_plan_info", "isam_gemm_plan_info2", "isam_gemm_grouped", "isam_gemm_fp8", "isam_gemm_grouped_fp8",
                     "isam_gemm_mxfp8", "isam_gemm_grouped_mxfp8",
                     "isam_gru_forward", "isam_gru_forward_reset_before",
                     "isam_gru_forward_stack",
                     "isam_dwsep_conv", "isam_dwsep_plan_info", "isam_dwsep_plan_for", "isam_depthwise_conv3x3",
                     "isam_gru_plan_info", "isam_gru_plan_for", "isam_gemm_plan_for",
                     "isam_glr_forward", "isam_glr_backward", "isam_glr_step",
                     "isam_glu_forward", "isam_glu_backward_workspace", "isam_glu_backward",
                     "isam_w4_pack", "isam_gemv_w4"):
            getattr(lib, name).restype = ctypes.c_int
        _lib = lib
        return lib


def last_error() -> str:
    return load().isam_last_error_string().decode(errors="replace")


def check(rc: int) -> None:
    if rc != ISAM_OK:
        raise IsamError(rc, last_error())


def _ptr(t):
    return None if t is None else t.data_ptr()


def _dev(t, dtype, numel, name):
    import torch
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if t.numel() != numel:
        raise ValueError(f"{name} has {t.numel()} elements, expected {numel}")
    if t.get_device() != torch.cuda.current_device():
        raise ValueError(f"{name} is not on the current device")


_raw_stream = None


def _stream_getter():
    global _raw_stream
    import torch
    if _raw_stream is None:
        # Where torch has it, 3 us cheaper than building a Stream object.
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        _raw_stream = raw if raw else lambda _: torch.cuda.current_stream().cuda_stream
    return _raw_stream


# The library's stream is one for the whole process: a thread holds this from
# setting it to the end of the call that is to run there.
_stream_lock = threading.Lock()


def _on_current_stream(fn, *args):
    """fn(*args), an entry of the library, on torch's current stream."""
    import torch
    stream = _stream_getter()(torch.cuda.current_device())
    with _stream_lock:
        _lib.isam_set_stream(stream)
        rc = fn(*args)
    check(rc)


def sync() -> None:
    """isam_sync: waits for the stream of the last call (of any thread) and
    raises what its kernels reported."""
    check(load().isam_sync())


def shutdown() -> None:
    check(load().isam_shutdown())


def gemm(M, N, K, transA, transB, alpha, A, B, beta, C) -> None:
    """isam_gemm: C = alpha op(A) op(B) + beta C (A, B bf16; C fp32)."""
    import torch
    lib = load()
    _dev(A, torch.bfloat16, M * K, "A")
    _dev(B, torch.bfloat16, K * N, "B")
    _dev(C, torch.float32, M * N, "C")
    _on_current_stream(lib.isam_gemm, M, N, K, int(transA), int(transB), float(alpha), _ptr(A), _ptr(B),
                       float(beta), _ptr(C))


def gemm_fp8(M, N, K, alpha, A, B, beta, C) -> None:
    """isam_gemm_fp8: C = alpha A B^T + beta C (A: M x K, B: N x K, E4M3 bytes as
    torch.uint8 or torch.float8_e4m3fn; C fp32)."""
    import torch
    lib = load()
    for t, n, name in ((A, M * K, "A"), (B, N * K, "B")):
        if t.dtype not in (torch.uint8, getattr(torch, "float8_e4m3fn", torch.uint8)):
            raise ValueError(f"{name} must hold E4M3 bytes (uint8 or float8_e4m3fn), got {t.dtype}")
        _dev(t, t.dtype, n, name)
    _dev(C, torch.float32, M * N, "C")
    _on_current_stream(lib.isam_gemm_fp8, M, N, K, float(alpha), _ptr(A), _ptr(B), float(beta), _ptr(C))


def _e4m3_dev(t, n, name):
    import torch
    if t.dtype not in (torch.uint8, getattr(torch, "float8_e4m3fn", torch.uint8)):
        raise ValueError(f"{name} must hold E4M3 bytes (uint8 or float8_e4m3fn), got {t.dtype}")
    _dev(t, t.dtype, n, name)


def mx_scale_bytes(rows, K) -> int:
    """Bytes of an atom-major scale array: ceil(K/128) x rows x 4."""
    return (K + 127) // 128 * rows * 4


def gemm_mxfp8(M, N, K, alpha, A, SA, B, SB, beta, C) -> None:
    """isam_gemm_mxfp8: C = alpha (SA o A)(SB o B)^T + beta C with A (M x K) and
    B (N x K) E4M3 bytes, SA and SB E8M0 bytes (torch.uint8) in the atom-major
    layout [ceil(K/128)][rows][4] (include/isam.h), C fp32."""
    import torch
    lib = load()
    _e4m3_dev(A, M * K, "A")
    _e4m3_dev(B, N * K, "B")
    _dev(SA, torch.uint8, mx_scale_bytes(M, K), "SA")
    _dev(SB, torch.uint8, mx_scale_bytes(N, K), "SB")
    _dev(C, torch.float32, M * N, "C")
    _on_current_stream(lib.isam_gemm_mxfp8, M, N, K, float(alpha), _ptr(A), _ptr(SA), _ptr(B), _ptr(SB), float(beta),
                       _ptr(C))


class GroupedGemmMxfp8:
    """Marshalled arguments of one isam_gemm_grouped_mxfp8 call over a list of
    (M, N, K, alpha, A, SA, B, SB, beta, C); SA, SB atom-major (mx_scale_bytes)."""

    def __init__(self, problems):
        import torch
        n = len(problems)
        ia = lambda vals: (ctypes.c_int * n)(*vals)
        fa = lambda vals: (ctypes.c_float * n)(*vals)
        pa = lambda vals: (ctypes.c_void_p * n)(*vals)
        for (M, N, K, alpha, A, SA, B, SB, beta, C) in problems:
            _e4m3_dev(A, M * K, "A")
            _e4m3_dev(B, N * K, "B")
            _dev(SA, torch.uint8, mx_scale_bytes(M, K), "SA")
            _dev(SB, torch.uint8, mx_scale_bytes(N, K), "SB")
            _dev(C, torch.float32, M * N, "C")
        cols = list(zip(*problems))
        self.n = n
        ptrs = lambda col: pa([t.data_ptr() for t in col])
        self.args = (ia(cols[0]), ia(cols[1]), ia(cols[2]), fa(cols[3]), ptrs(cols[4]), ptrs(cols[5]),
                     ptrs(cols[6]), ptrs(cols[7]), fa(cols[8]), ptrs(cols[9]))

    def __call__(self):
        lib = load()
        _on_current_stream(lib.isam_gemm_grouped_mxfp8, self.n, *self.args)


class GroupedGemm:
    """Marshalled argument arrays of one isam_gemm_grouped call (build once,
    call many times: the arrays keep the ctypes buffers alive)."""

    def __init__(self, problems):
        import torch
        n = len(problems)
        ia = lambda vals: (ctypes.c_int * n)(*vals)
        fa = lambda vals: (ctypes.c_float * n)(*vals)
        pa = lambda vals: (ctypes.c_void_p * n)(*vals)
        for (M, N, K, tA, tB, alpha, A, B, beta, C) in problems:
            _dev(A, torch.bfloat16, M * K, "A")
            _dev(B, torch.bfloat16, K * N, "B")
            _dev(C, torch.float32, M * N, "C")
        cols = list(zip(*problems))
        self.n = n
        self.args = (ia(cols[0]), ia(cols[1]), ia(cols[2]), ia(cols[3]), ia(cols[4]), fa(cols[5]),
                     pa([t.data_ptr() for t in cols[6]]), pa([t.data_ptr() for t in cols[7]]), fa(cols[8]),
                     pa([t.data_ptr() for t in cols[9]]))

    def __call__(self):
        lib = load()
        _on_current_stream(lib.isam_gemm_grouped, self.n, *self.args)


class GroupedGemmFp8:
    """Marshalled arguments of one isam_gemm_grouped_fp8 call over a list of
    (M, N, K, alpha, A, B, beta, C); A, B E4M3 bytes (uint8 / float8_e4m3fn)."""

    def __init__(self, problems):
        import torch
        n = len(problems)
        ia = lambda vals: (ctypes.c_int * n)(*vals)
        fa = lambda vals: (ctypes.c_float * n)(*vals)
        pa = lambda vals: (ctypes.c_void_p * n)(*vals)
        for (M, N, K, alpha, A, B, beta, C) in problems:
            _dev(A, A.dtype, M * K, "A")
            _dev(B, B.dtype, N * K, "B")
            _dev(C, torch.float32, M * N, "C")
        cols = list(zip(*problems))
        self.n = n
        self.args = (ia(cols[0]), ia(cols[1]), ia(cols[2]), fa(cols[3]), pa([t.data_ptr() for t in cols[4]]),
                     pa([t.data_ptr() for t in cols[5]]), fa(cols[6]), pa([t.data_ptr() for t in cols[7]]))

    def __call__(self):
        lib = load()
        _on_current_stream(lib.isam_gemm_grouped_fp8, self.n, *self.args)


def gemm_grouped(problems) -> None:
    """isam_gemm_grouped over a list of (M, N, K, transA, transB, alpha, A, B, beta, C)."""
    GroupedGemm(problems)()


def gemm_plan(M, N, K, transA, transB, beta=0.0, num_sms=None, smem_optin=None, cluster_caps=None) -> dict:
    """The tile plan the library's cost model picks (nothing is launched);
    with num_sms, smem_optin and cluster_caps (resident clusters of 2, 4, 8
    CTAs), isam_gemm_plan_for on those limits (no GPU)."""
    lib = load()
    out = (ctypes.c_int * 8)()
    if num_sms is None:
        check(lib.isam_gemm_plan_info2(M, N, K, int(transA), int(transB), float(beta), out))
    else:
        caps = (ctypes.c_int * 3)(*cluster_caps)
        check(lib.isam_gemm_plan_for(M, N, K, int(transA), int(transB), float(beta), num_sms, smem_optin, caps, out))
    return dict(zip(("BN", "split", "stages", "group_m", "grid", "smem", "tile_m", "cta_pair"), list(out)))


def gru_forward(T, batch, hidden, x, W, U, b, h0, h_out, reset_before=False) -> None:
    """isam_gru_forward, or isam_gru_forward_reset_before with reset_before
    (x, W, U bf16; b, h0, h_out fp32; h0 may be None)."""
    import torch
    lib = load()
    H = hidden
    _dev(x, torch.bfloat16, T * batch * H, "x")
    _dev(W, torch.bfloat16, 3 * H * H, "W")
    _dev(U, torch.bfloat16, 3 * H * H, "U")
    _dev(b, torch.float32, 6 * H, "b")
    if h0 is not None:
        _dev(h0, torch.float32, batch * H, "h0")
    _dev(h_out, torch.float32, T * batch * H, "h_out")
    fn = lib.isam_gru_forward_reset_before if reset_before else lib.isam_gru_forward
    _on_current_stream(fn, T, batch, H, _ptr(x), _ptr(W), _ptr(U), _ptr(b), _ptr(h0), _ptr(h_out))


def gru_forward_stack(layers, T, batch, hidden, x, W, U, b, h0, h_out, reset_before=False) -> None:
    """isam_gru_forward_stack: x [T,batch,H] bf16; W, U [layers,3H,H] bf16;
    b [layers,6H], h0 [layers,batch,H] (or None), h_out [layers,T,batch,H] fp32."""
    import torch
    lib = load()
    H, L = hidden, layers
    _dev(x, torch.bfloat16, T * batch * H, "x")
    _dev(W, torch.bfloat16, L * 3 * H * H, "W")
    _dev(U, torch.bfloat16, L * 3 * H * H, "U")
    _dev(b, torch.float32, L * 6 * H, "b")
    if h0 is not None:
        _dev(h0, torch.float32, L * batch * H, "h0")
    _dev(h_out, torch.float32, L * T * batch * H, "h_out")
    _on_current_stream(lib.isam_gru_forward_stack, L, T, batch, H, int(bool(reset_before)), _ptr(x), _ptr(W),
                       _ptr(U), _ptr(b), _ptr(h0), _ptr(h_out))


def dwsep_conv(N, H, W, Cin, Cout, x, dw_w, pw_w, out) -> None:
    """isam_dwsep_conv: NHWC 3x3 depthwise (pad 1) then 1x1 pointwise."""
    import torch
    lib = load()
    _dev(x, torch.bfloat16, N * H * W * Cin, "x")
    _dev(dw_w, torch.bfloat16, 9 * Cin, "dw_w")
    _dev(pw_w, torch.bfloat16, Cin * Cout, "pw_w")
    _dev(out, torch.float32, N * H * W * Cout, "out")
    _on_current_stream(lib.isam_dwsep_conv, N, H, W, Cin, Cout, _ptr(x), _ptr(dw_w), _ptr(pw_w), _ptr(out))


def depthwise_conv3x3(N, H, W, C, x, dw_w, y) -> None:
    """isam_depthwise_conv3x3: NHWC 3x3 depthwise (pad 1), bf16 in and out."""
    import torch
    lib = load()
    _dev(x, torch.bfloat16, N * H * W * C, "x")
    _dev(dw_w, torch.bfloat16, 9 * C, "dw_w")
    _dev(y, torch.bfloat16, N * H * W * C, "y")
    _on_current_stream(lib.isam_depthwise_conv3x3, N, H, W, C, _ptr(x), _ptr(dw_w), _ptr(y))


_DWSEP_PLAN_KEYS = ("kernel", "rows_per_tile", "blocks", "block_cout")
_GRU_PLAN_KEYS = ("splits", "atoms", "batch_pad", "ctas", "smem", "path", "chunks")


def dwsep_plan(W, Cin, Cout, smem_optin=None) -> dict:
    """isam_dwsep_plan_info: the kernel, tile rows and output-channel blocks
    isam_dwsep_conv takes for this width and channel counts (nothing is
    launched); with smem_optin, isam_dwsep_plan_for on those limits (no GPU)."""
    lib = load()
    out = (ctypes.c_int * 4)()
    if smem_optin is None:
        check(lib.isam_dwsep_plan_info(W, Cin, Cout, out))
    else:
        check(lib.isam_dwsep_plan_for(W, Cin, Cout, smem_optin, out))
    return dict(zip(_DWSEP_PLAN_KEYS, list(out)))


def gru_plan(layers, batch, hidden, reset_before=False, num_sms=None, smem_optin=None) -> dict:
    """isam_gru_plan_info: K splits, padded batch, CTAs, shared memory and the
    layer schedule of a GRU call (nothing is launched); with num_sms and
    smem_optin, isam_gru_plan_for on those limits (no GPU)."""
    lib = load()
    out = (ctypes.c_int * 7)()
    if num_sms is None:
        check(lib.isam_gru_plan_info(layers, batch, hidden, int(bool(reset_before)), out))
    else:
        check(lib.isam_gru_plan_for(layers, batch, hidden, int(bool(reset_before)), num_sms, smem_optin, out))
    return dict(zip(_GRU_PLAN_KEYS, list(out)))


# The calls below run for single tokens, where a few microseconds of checks count:
# one look at the current device and stream a call, and the checks of a tensor
# in one expression that falls back to _dev for its message.

class _Call:
    """The library, torch, and the current device and stream set for one call."""

    __slots__ = ("lib", "torch", "device")

    def __init__(self):
        if _torch is None:
            _first_call()
        self.torch = _torch
        self.lib = _lib
        self.device = _current_device()

    def ptr(self, t, dtype, numel, name):
        """The address of a tensor that is what it has to be."""
        # (a CPU tensor's device is -1, which no current device is)
        if not (t.dtype is dtype and t.get_device() == self.device and t.numel() == numel and t.is_contiguous()):
            _dev(t, dtype, numel, name)
        return t.data_ptr()

    def opt(self, t, dtype, numel, name):
        return None if t is None else self.ptr(t, dtype, numel, name)

    def kind(self, t, name):
        """ISAM_F32 or ISAM_BF16 of a tensor."""
        code = _kinds.get(t.dtype)
        if code is None:
            raise ValueError(f"{name} must be torch.float32 or torch.bfloat16, got {t.dtype}")
        return code

    def run(self, fn, *args):
        stream = _raw_stream(self.device)
        with _stream_lock:
            self.lib.isam_set_stream(stream)
            rc = fn(*args)
        if rc != ISAM_OK:
            check(rc)


_torch = None
_kinds = {}


def _current_device():
    """-2 until torch has set CUDA up: no tensor is on a device then."""
    global _current_device
    if not _torch.cuda.is_initialized():
        return -2
    # Where torch has it, without torch's check that CUDA is set up.
    _current_device = getattr(_torch._C, "_cuda_getDevice", _torch.cuda.current_device)
    return _current_device()


def _with_workspace(device, size, call):
    """call(address of `size` bytes of torch's allocator on the current stream,
    given back behind the call, to later work of that stream)."""
    # Where torch has it: 1 us a call, a tensor 5 to 8.
    alloc = getattr(_torch._C, "_cuda_cudaCachingAllocator_raw_alloc", None)
    free = getattr(_torch._C, "_cuda_cudaCachingAllocator_raw_delete", None)
    if alloc is None or free is None:
        held = _torch.empty(size, dtype=_torch.uint8, device=f"cuda:{device}")
        call(held.data_ptr())
        return
    at = alloc(size, _raw_stream(device))
    try:
        call(at)
    finally:
        free(at)


def _first_call():
    global _torch
    import torch
    load()
    _stream_getter()
    _kinds.update({torch.float32: 0, torch.bfloat16: 1})
    _torch = torch


def glr_forward(T, batch, hidden, g, h0, lengths, h_out, h_last=None) -> None:
    """isam_glr_forward: h_t = z h_{t-1} + (1 - z) n over T steps, z = sigmoid of
    the first and n the second half of g's rows (g [T,batch,2H] and h_out
    [T,batch,H] fp32 or bf16; h0, h_last [batch,H] fp32 or None; lengths
    [batch] int32 or None)."""
    c = _Call()
    f32, n = c.torch.float32, T * batch * hidden
    gt, ht = c.kind(g, "g"), c.kind(h_out, "h_out")
    c.run(c.lib.isam_glr_forward, T, batch, hidden, gt, c.ptr(g, g.dtype, 2 * n, "g"),
          c.opt(h0, f32, batch * hidden, "h0"), c.opt(lengths, c.torch.int32, batch, "lengths"), ht,
          c.ptr(h_out, h_out.dtype, n, "h_out"), c.opt(h_last, f32, batch * hidden, "h_last"))


def glr_backward(T, batch, hidden, g, h0, lengths, h_out, dh_out, dh_last, dg, dh0=None) -> None:
    """isam_glr_backward: gradients dg (g's shape and type) and dh0 [batch,H]
    fp32 (or None) of glr_forward from dh_out (h_out's shape and type, or None)
    and dh_last [batch,H] fp32 (or None)."""
    c = _Call()
    f32, n, edge = c.torch.float32, T * batch * hidden, batch * hidden
    gt, ht = c.kind(g, "g"), c.kind(h_out, "h_out")
    c.run(c.lib.isam_glr_backward, T, batch, hidden, gt, c.ptr(g, g.dtype, 2 * n, "g"), c.opt(h0, f32, edge, "h0"),
          c.opt(lengths, c.torch.int32, batch, "lengths"), ht, c.ptr(h_out, h_out.dtype, n, "h_out"),
          c.opt(dh_out, h_out.dtype, n, "dh_out"), c.opt(dh_last, f32, edge, "dh_last"),
          c.ptr(dg, g.dtype, 2 * n, "dg"), c.opt(dh0, f32, edge, "dh0"))


def glr_step(batch, hidden, slots, g, slot_ids, state, new_state, h) -> None:
    """isam_glr_step: one token for `batch` sequences whose fp32 states are rows
    slot_ids (int32, or None for row b) of state [slots,H]; new_state may be
    state; h [batch,H] fp32 or bf16."""
    c = _Call()
    f32, n = c.torch.float32, batch * hidden
    gt, ht = c.kind(g, "g"), c.kind(h, "h")
    c.run(c.lib.isam_glr_step, batch, hidden, slots, gt, c.ptr(g, g.dtype, 2 * n, "g"),
          c.opt(slot_ids, c.torch.int32, batch, "slot_ids"), c.ptr(state, f32, slots * hidden, "state"),
          c.ptr(new_state, f32, slots * hidden, "new_state"), ht, c.ptr(h, h.dtype, n, "h"))


ACTIVATIONS = {"silu": 0, "gelu": 1, "relu": 2, "sigmoid": 3}


def _act_code(act):
    if act not in ACTIVATIONS:
        raise ValueError(f"act must be one of {sorted(ACTIVATIONS)}, got {act!r}")
    return ACTIVATIONS[act]


def glu_forward(T, D, F, act, x, W, h) -> None:
    """isam_glu_forward: h = act(x Wg^T) * (x Wu^T) (x [T,D], W [2F,D] with the
    gate rows first, h [T,F], all bf16; act "silu", "gelu", "relu" or "sigmoid")."""
    code, c = _act_code(act), _Call()
    bf16 = c.torch.bfloat16
    c.run(c.lib.isam_glu_forward, T, D, F, code, c.ptr(x, bf16, T * D, "x"), c.ptr(W, bf16, 2 * F * D, "W"),
          c.ptr(h, bf16, T * F, "h"))


def glu_backward_workspace(T, D, F) -> int:
    """isam_glu_backward_workspace: bytes of glu_backward's workspace."""
    out = ctypes.c_size_t()
    check(load().isam_glu_backward_workspace(T, D, F, ctypes.byref(out)))
    return out.value


def glu_backward(T, D, F, act, x, W, dh, dx, dW, workspace=None) -> None:
    """isam_glu_backward: dx [T,D] and dW [2F,D] (bf16, either may be None) of
    glu_forward from dh [T,F]; workspace a uint8 tensor of
    glu_backward_workspace bytes, or None to take one from torch's allocator
    on the current stream."""
    code, c = _act_code(act), _Call()
    bf16, u8 = c.torch.bfloat16, c.torch.uint8
    args = (c.ptr(x, bf16, T * D, "x"), c.ptr(W, bf16, 2 * F * D, "W"), c.ptr(dh, bf16, T * F, "dh"))
    out = (c.opt(dx, bf16, T * D, "dx"), c.opt(dW, bf16, 2 * F * D, "dW"))
    need = glu_backward_workspace(T, D, F)
    if workspace is None:
        _with_workspace(c.device, need, lambda ws: c.run(c.lib.isam_glu_backward, T, D, F, code, *args, ws, *out))
        return
    ws = c.ptr(workspace, u8, workspace.numel(), "workspace")
    if workspace.numel() < need:
        raise ValueError(f"workspace has {workspace.numel()} bytes, {need} are needed")
    c.run(c.lib.isam_glu_backward, T, D, F, code, *args, ws, *out)


def w4_tiled_bytes(N, K) -> int:
    """Bytes of the tiled codes of an N x K matrix."""
    return (N + 15) // 16 * ((K + 127) // 128) * 1024


def w4_tiled_scales(N, K, group) -> int:
    """Elements of the tiled scales of an N x K matrix."""
    return (N + 15) // 16 * ((K + 127) // 128) * 16 * (128 // group)


def w4_pack(N, K, group, codes, scales, tiled, tiled_scales) -> None:
    """isam_w4_pack: codes [N,K/2] (uint8, even k in the low half) and scales
    [N,ceil(K/group)] (bf16) into the tiled order gemv_w4 reads (uint8
    w4_tiled_bytes, bf16 w4_tiled_scales)."""
    if group not in (32, 64, 128):
        raise ValueError(f"group must be 32, 64 or 128, got {group}")
    c = _Call()
    bf16, u8 = c.torch.bfloat16, c.torch.uint8
    c.run(c.lib.isam_w4_pack, N, K, group, c.ptr(codes, u8, N * (K // 2), "codes"),
          c.ptr(scales, bf16, N * ((K + group - 1) // group), "scales"),
          c.ptr(tiled, u8, w4_tiled_bytes(N, K), "tiled"),
          c.ptr(tiled_scales, bf16, w4_tiled_scales(N, K, group), "tiled_scales"))


def gemv_w4(M, N, K, group, x, tiled, tiled_scales, y) -> None:
    """isam_gemv_w4: y [M,N] fp32 = x [M,K] bf16 times 4-bit weights in
    w4_pack's order, M <= 32."""
    if group not in (32, 64, 128):
        raise ValueError(f"group must be 32, 64 or 128, got {group}")
    c = _Call()
    bf16 = c.torch.bfloat16
    c.run(c.lib.isam_gemv_w4, M, N, K, group, c.ptr(x, bf16, M * K, "x"),
          c.ptr(tiled, c.torch.uint8, w4_tiled_bytes(N, K), "tiled"),
          c.ptr(tiled_scales, bf16, w4_tiled_scales(N, K, group), "tiled_scales"),
          c.ptr(y, c.torch.float32, M * N, "y"))