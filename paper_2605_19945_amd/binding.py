"""ctypes binding of include/moe.h.  Argument marshalling only.

PyTorch is used for device memory and streams: tensors are passed as raw device pointers
(`data_ptr()`), the stream as the raw handle of the current one.
"""
from __future__ import annotations

import ctypes as C
import functools
import os
import struct

_PKG = os.path.dirname(os.path.abspath(__file__))
_LIB_NAME = "libmoe_gfx950.so"
_lib = None
torch = None  # set by load_library (the mapping search and the argument checks need neither)
_BF16 = _F32 = _I32T = _U8 = _device = _stream_of = _wrote = None  # torch's types, current device, raw stream and note of a write, set with it

FLAG_STAGE_EVENTS = 1
STAGE_NAMES = ("route", "permute", "gemm1", "gemm2", "combine")
_STATUS = {0: "MOE_OK", 1: "MOE_ERR_INVALID_ARG", 2: "MOE_ERR_UNSUPPORTED_SHAPE",
           3: "MOE_ERR_WORKSPACE_TOO_SMALL", 4: "MOE_ERR_DEVICE"}


class MoEError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        lib = load_library()
        msg = lib.moe_status_string(status).decode()
        if status in (3, 4) and lib.moe_last_device_error():
            msg += ": " + lib.moe_last_device_error().decode()
        super().__init__(f"{what}: {_STATUS.get(status, status)} ({msg})")


class _Shape(C.Structure):
    _fields_ = [("T_max", C.c_int32), ("d", C.c_int32), ("f", C.c_int32), ("E", C.c_int32),
                ("k", C.c_int32), ("e_lo", C.c_int32), ("E_local", C.c_int32), ("flags", C.c_uint32)]


def library_path() -> str:
    return os.path.join(_PKG, _LIB_NAME)


_VP, _I32, _I64, _SZ = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t
_SIGNATURES = {
    "moe_status_string": (C.c_char_p, [C.c_int]),
    "moe_last_device_error": (C.c_char_p, []),
    "moe_workspace_bytes": (_SZ, [C.POINTER(_Shape)]),
    "moe_create": (C.c_int, [C.POINTER(_VP), C.POINTER(_Shape), _VP, _SZ]),
    "moe_destroy": (None, [_VP]),
    "moe_rows_capacity": (_I64, [C.POINTER(_Shape), _I32]),
    "moe_packed_router_bytes": (_SZ, [C.POINTER(_Shape)]),
    "moe_pack_router": (C.c_int, [_VP, _VP, _VP, _VP]),
    "moe_packed_weight_bytes": (_SZ, [C.POINTER(_Shape)]),
    "moe_pack_weights": (C.c_int, [_VP, _VP, _VP, _VP, _VP, _VP]),
    "moe_route": (C.c_int, [_VP, _VP, _VP, _VP, _I32, _VP, _VP, _VP, _VP]),
    "moe_permute": (C.c_int, [_VP, _VP, _VP, _I32, _VP, _VP, _VP, _VP, _VP]),
    "moe_permute_noalloc": (C.c_int, [_VP, _VP, _I32, _I32, _I32, _I32, _I32, _I32, _VP, _VP, _VP, _VP, _VP]),
    "moe_grouped_ffn": (C.c_int, [_VP, _VP, _VP, _I32, _VP, _VP, _VP]),
    "moe_combine": (C.c_int, [_VP, _VP, _VP, _VP, _I32, _VP, _VP]),
    "moe_layer_forward": (C.c_int, [_VP, _VP, _VP, _VP, _VP, _I32, _VP, _VP, _VP]),
    "moe_stage_times": (C.c_int, [_VP, C.POINTER(C.c_float)]),
    "moe_profile_ffn": (C.c_int, [_VP, _VP, _VP, _VP, C.POINTER(_I32), _I32, _I32, _I32, C.POINTER(C.c_float), _VP]),
    "moe_gem_score": (C.c_int, [_VP, _I32, _I32, _I32, _VP, _VP, _VP, _VP, C.POINTER(C.c_double)]),
    "moe_gem_place": (C.c_int, [_VP, _I32, _I32, _I32, _VP, _VP, _VP, _VP, _I32, _VP, C.POINTER(C.c_double),
                                C.POINTER(_I32)]),
    "moe_curve_sample_counts": (C.c_int, [_I32, _I32, _I32, _I32, _I32, _VP, _I32, C.POINTER(_I32)]),
    "moe_curve_eval": (C.c_int, [_VP, _VP, _I32, _VP, _I32, _VP]),
    "moe_curve_sum": (C.c_int, [_VP, _VP, _I32, _I32, _I32, C.POINTER(C.c_double)]),
    "moe_trace_mean_utilisation": (C.c_int, [_VP, _I32, _I32, _VP]),
    "moe_trace_correlation": (C.c_int, [_VP, _I32, _I32, _VP]),
    "moe_measure_mfma_rate": (C.c_int, [_I32, _I32, C.POINTER(C.c_float), _VP]),
    "moe_measure_mfma_rate_of": (C.c_int, [_I32, _I32, _I32, C.POINTER(C.c_float), _VP]),
    "moe_measure_hbm_read_rate": (C.c_int, [_VP, C.c_size_t, _I32, _I32, C.POINTER(C.c_float), _VP]),
    "moe_ffn_refused_flag": (C.c_int, [_VP, C.POINTER(_VP)]),
    "moe_tile_rows": (_I32, [_VP]),
    "moe_set_tile_class": (C.c_int, [_VP, _I32]),
    "moe_grouped_gemm_workspace_bytes": (_SZ, [_I32, _I32, _I32, _I32, _I32]),
    "moe_grouped_gemm": (C.c_int, [_VP, _I64, _VP, _I32, _VP, _I32, _I32, _I32, _I32, _VP, _I64, _VP, _SZ, _VP]),
    "moe_grouped_gemm_wgrad_workspace_bytes": (_SZ, [_I32, _I32, _I32, _I32]),
    "moe_grouped_gemm_wgrad": (C.c_int, [_VP, _I64, _VP, _I64, _VP, _I32, _I32, _I32, _I32, _VP, _I32, _I32, _VP, _SZ, _VP]),
    "moe_swiglu": (C.c_int, [_VP, _I64, _VP, _I32, _I32, _VP, _I64, _VP]),
    "moe_swiglu_backward": (C.c_int, [_VP, _I64, _VP, _I64, _VP, _I32, _I32, _VP, _I64, _VP, _I64, _VP]),
    "moe_grad_norm_workspace_bytes": (_SZ, [_I32]),
    "moe_grad_norm": (C.c_int, [_VP, _VP, _VP, _I32, _VP, _SZ, _VP, _VP]),
    "moe_clip_grad_norm": (C.c_int, [_VP, _VP, _VP, _VP, _I32, C.c_float, _VP, _SZ, _VP, _VP]),
    "moe_mxfp4_scale_cols": (_I32, [_I32]),
    "moe_mxfp4_quantize": (C.c_int, [_VP, _I32, _I64, _VP, _I32, _I32, _VP, _VP, _VP]),
    "moe_mxfp4_quantize_weights": (C.c_int, [_VP, _I32, _I32, _I32, _VP, _VP, _VP]),
    "moe_mxfp4_dequantize": (C.c_int, [_VP, _VP, _I64, _I32, _VP, _I64, _VP]),
    "moe_mxfp4_grouped_gemm_workspace_bytes": (_SZ, [_I32, _I32, _I32, _I32]),
    "moe_mxfp4_grouped_gemm": (C.c_int, [_VP, _VP, _VP, _VP, _VP, _I32, _I32, _I32, _I32, _VP, _I64, _VP, _SZ, _VP]),
    "moe_rms_norm": (C.c_int, [_VP, _I32, _I64, _VP, _I32, C.c_float, _VP, _I32, _I32, _VP, _I32, _I64, _VP]),
    "moe_norm_backward_workspace_bytes": (_SZ, [_I32, _I32]),
    "moe_rms_norm_backward": (C.c_int, [_VP, _I32, _I64, _VP, _I32, _I64, _VP, _I32, C.c_float, _VP, _I64, _VP, _I32, _I32, _VP, _I64,
                                        _VP, _VP, _SZ, _VP]),
    "moe_residual_norm": (C.c_int, [_VP, _I32, _I64, _VP, _I32, _I64, _VP, _I32, _I32, _VP, _I64, C.c_float, _VP, C.c_float, _VP, _I32,
                                    _I32, _VP, _I64, _VP, _I64, _VP]),
    "moe_residual_norm_backward": (C.c_int, [_VP, _I64, _VP, _I64, _VP, _I32, _I64, _VP, _I32, _I64, _VP, _I32, _I32, _VP, _I64,
                                             C.c_float, _VP, C.c_float, _VP, _I32, _I32, _VP, _I64, _VP, _I64, _VP, _I64, _VP, _VP, _VP,
                                             _SZ, _VP]),
    "moe_orthogonalize_workspace_bytes": (_SZ, [_I32, _I32, _I32]),
    "moe_orthogonalize": (C.c_int, [_VP, _I32, _I64, _I64, _I32, _I32, _I32, _VP, _I32, C.c_float, C.c_float, _VP, _I32, _I64, _I64, _VP, _SZ,
                                    _VP]),
    "moe_layer_intermediates": (C.c_int, [_VP, C.POINTER(_VP), C.POINTER(_VP), C.POINTER(_VP), C.POINTER(_VP)]),
}


def exported_symbols():
    return tuple(_SIGNATURES)


def load_library():
    """Loads libmoe_gfx950.so from the package directory.  Raises if it has not been built."""
    global _lib, torch, _BF16, _F32, _I32T, _U8, _device, _stream_of, _wrote
    if _lib is not None:
        return _lib
    # PyTorch ships its own HIP runtime; import it first so that the library binds to that one
    # instance instead of bringing a second runtime into the process.
    import torch
    _BF16, _F32, _I32T, _U8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8
    _device, _stream_of = torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream
    _wrote = torch.autograd.graph.increment_version  # (a saved tensor that a call writes over is then noticed)
    path = library_path()
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is missing: build it with `python -m paper_2605_19945_amd.build` "
                           "(there is no fallback path)")
    lib = C.CDLL(path)
    for name, (res, args) in _SIGNATURES.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    _lib = lib
    return lib


# A call's arguments are marshalled as plain integers (argtypes makes pointers of them), and the stream is asked for
# as the raw handle: building the Stream object of torch.cuda.current_stream() took 3.0 us of the 12 us that a program
# spent on a small routing call, the handle takes 0.2.
def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream():
    return _stream_of(torch.cuda.current_device())


class MoEContext:
    """One moe_ctx plus its device workspace.  Methods carry the C entry points' names."""

    def __init__(self, T_max, d, f, E, k, e_lo=0, E_local=-1, flags=0, device="cuda:0"):
        self.lib = load_library()
        if E_local < 0:
            E_local = E
        self.shape = _Shape(T_max, d, f, E, k, e_lo, E_local, flags)
        self.T_max, self.d, self.f, self.E, self.k, self.e_lo, self.E_local = T_max, d, f, E, k, e_lo, E_local
        self.device = torch.device(device)
        self._ctx = C.c_void_p()
        nbytes = self.lib.moe_workspace_bytes(C.byref(self.shape))
        if nbytes == 0:
            raise MoEError(2, "moe_workspace_bytes")
        torch.cuda.set_device(self.device)
        self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        st = self.lib.moe_create(C.byref(self._ctx), C.byref(self.shape), _ptr(self.workspace), nbytes)
        if st != 0:
            raise MoEError(st, "moe_create")

    def close(self):
        if getattr(self, "_ctx", None) is not None and self._ctx.value:
            self.lib.moe_destroy(self._ctx)
            self._ctx = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # ---- helpers -------------------------------------------------------------------------------
    def rows_capacity(self, T):
        return int(self.lib.moe_rows_capacity(C.byref(self.shape), T))

    def _check(self, st, what):
        if st != 0:
            raise MoEError(st, what)

    def _empty(self, shape, dtype):
        return torch.empty(shape, dtype=dtype, device=self.device)

    # ---- load time -----------------------------------------------------------------------------
    def moe_pack_router(self, Wg):
        rp = self._empty(self.lib.moe_packed_router_bytes(C.byref(self.shape)) // 2, torch.bfloat16)
        self._check(self.lib.moe_pack_router(self._ctx, _ptr(Wg), _ptr(rp), _stream()), "moe_pack_router")
        return rp

    def moe_pack_weights(self, W1, W3, W2):
        packed = self._empty(self.lib.moe_packed_weight_bytes(C.byref(self.shape)) // 2, torch.bfloat16)
        self._check(self.lib.moe_pack_weights(self._ctx, _ptr(W1), _ptr(W3), _ptr(W2), _ptr(packed), _stream()),
                    "moe_pack_weights")
        return packed

    # ---- hot path ------------------------------------------------------------------------------
    def moe_route(self, x, router_packed, bias=None, T=None, idx=None, w=None, counts=None):
        """idx / w / counts: optional caller-provided outputs (e.g. one row of a trace matrix)."""
        T = x.shape[0] if T is None else T
        idx = self._empty((T, self.k), torch.int32) if idx is None else idx
        w = self._empty((T, self.k), torch.float32) if w is None else w
        counts = self._empty((self.E,), torch.int32) if counts is None else counts
        if T == 0:
            counts.zero_()
        self._check(self.lib.moe_route(self._ctx, _ptr(x), _ptr(router_packed), _ptr(bias), T, _ptr(idx), _ptr(w),
                                       _ptr(counts), _stream()), "moe_route")
        return idx, w, counts

    def moe_permute(self, x, topk_idx, T=None, copy_rows=True):
        T = topk_idx.shape[0] if T is None else T
        cap = max(1, self.rows_capacity(T))
        xp = self._empty((cap, self.d), torch.bfloat16) if copy_rows else None
        offsets = self._empty((self.E_local + 1,), torch.int32)
        row_of = self._empty((T, self.k), torch.int32)
        tok_of = self._empty((cap,), torch.int32)
        if T == 0:
            offsets.zero_()
        self._check(self.lib.moe_permute(self._ctx, _ptr(x), _ptr(topk_idx), T, _ptr(xp), _ptr(offsets),
                                         _ptr(row_of), _ptr(tok_of), _stream()), "moe_permute")
        return xp, offsets, row_of, tok_of

    def moe_grouped_ffn(self, xp, offsets, n_rows_cap, packed, y=None):
        if y is None:
            y = self._empty((max(1, n_rows_cap), self.d), torch.bfloat16)
        self._check(self.lib.moe_grouped_ffn(self._ctx, _ptr(xp), _ptr(offsets), n_rows_cap, _ptr(packed), _ptr(y),
                                             _stream()), "moe_grouped_ffn")
        return y

    def moe_combine(self, y, row_of, topk_w, T=None, out=None):
        T = row_of.shape[0] if T is None else T
        if out is None:
            out = self._empty((T, self.d), torch.bfloat16)
        self._check(self.lib.moe_combine(self._ctx, _ptr(y), _ptr(row_of), _ptr(topk_w), T, _ptr(out), _stream()),
                    "moe_combine")
        return out

    def moe_layer_forward(self, x, router_packed, bias, packed, T=None, out=None, counts_out=None):
        T = x.shape[0] if T is None else T
        if out is None:
            out = self._empty((T, self.d), torch.bfloat16)
        self._check(self.lib.moe_layer_forward(self._ctx, _ptr(x), _ptr(router_packed), _ptr(bias), _ptr(packed),
                                               T, _ptr(out), _ptr(counts_out), _stream()), "moe_layer_forward")
        return out

    # ---- introspection -------------------------------------------------------------------------
    def moe_stage_times(self):
        ms = (C.c_float * len(STAGE_NAMES))()
        self._check(self.lib.moe_stage_times(self._ctx, ms), "moe_stage_times")
        return dict(zip(STAGE_NAMES, (float(v) for v in ms)))

    def moe_profile_ffn(self, xp, packed, token_counts, warmup=3, iters=20, y=None):
        """Mean milliseconds of the isolated expert kernels at each token count (blocking)."""
        counts = [int(n) for n in token_counts]
        if y is None:
            y = self._empty((max(max(counts, default=0), 1), self.d), torch.bfloat16)
        arr = (_I32 * len(counts))(*counts)
        ms = (C.c_float * len(counts))()
        self._check(self.lib.moe_profile_ffn(self._ctx, _ptr(xp), _ptr(packed), _ptr(y), arr, len(counts), warmup,
                                             iters, ms, _stream()), "moe_profile_ffn")
        return [float(v) for v in ms]

    def moe_ffn_refused(self):
        """True if the most recent expert-FFN call on this context refused its offsets (blocks until it is done)."""
        p = C.c_void_p()
        self._check(self.lib.moe_ffn_refused_flag(self._ctx, C.byref(p)), "moe_ffn_refused_flag")
        off = p.value - self.workspace.data_ptr()
        torch.cuda.synchronize()
        return bool(self.workspace[off:off + 4].view(torch.int32).item())

    def moe_tile_rows(self):
        return int(self.lib.moe_tile_rows(self._ctx))

    def moe_set_tile_class(self, cls):
        self._check(self.lib.moe_set_tile_class(self._ctx, cls), "moe_set_tile_class")

    def moe_layer_intermediates(self, T):
        """Copies of topk_idx [T,k], topk_w [T,k], offsets [E_local+1], row_of [T,k] of the last layer call."""
        p = [C.c_void_p() for _ in range(4)]
        self._check(self.lib.moe_layer_intermediates(self._ctx, *[C.byref(q) for q in p]), "moe_layer_intermediates")
        base = self.workspace.data_ptr()

        def view(ptr, n, dtype):
            off = ptr.value - base
            return self.workspace[off:off + 4 * n].view(dtype).clone()

        A = T * self.k
        return (view(p[0], A, torch.int32).view(T, self.k), view(p[1], A, torch.float32).view(T, self.k),
                view(p[2], self.E_local + 1, torch.int32), view(p[3], A, torch.int32).view(T, self.k))


def moe_permute_noalloc(x, topk_idx, E, e_lo=0, E_local=-1, xp=None, offsets=None, row_of=None, tok_of=None):
    """moe_permute without a context (scratch in the library's static device array).  The outputs are
    allocated here unless the caller passes them; the library call itself allocates nothing."""
    lib = load_library()
    T, k = topk_idx.shape
    E_local = E if E_local < 0 else E_local
    d = x.shape[1] if x is not None else 0
    cap = max(1, T * min(k, E_local))
    dev = topk_idx.device
    if xp is None and x is not None:
        xp = torch.empty((cap, d), dtype=torch.bfloat16, device=dev)
    offsets = torch.empty(E_local + 1, dtype=torch.int32, device=dev) if offsets is None else offsets
    row_of = torch.empty((T, k), dtype=torch.int32, device=dev) if row_of is None else row_of
    tok_of = torch.empty(cap, dtype=torch.int32, device=dev) if tok_of is None else tok_of
    if T == 0:
        offsets.zero_()
    st = lib.moe_permute_noalloc(_ptr(x), _ptr(topk_idx), T, d, E, k, e_lo, E_local, _ptr(xp), _ptr(offsets),
                                 _ptr(row_of), _ptr(tok_of), _stream())
    if st != 0:
        raise MoEError(st, "moe_permute_noalloc")
    return xp, offsets, row_of, tok_of


# ---- operators around the experts' weights (no context) -----------------------------------------------
# Tensors are checked here for what the C entry points cannot see: type, device, shape, strides, and whether torch would lose a
# gradient (no call records a graph; norms and clipping, like torch's, and 4-bit codes have none to lose).  Small calls are bound by this
# code, so each one first asks whether all is as it should be, in one expression, and only otherwise goes through the
# checks one by one, which find what to say or let an unusual layout pass, such as a single row, whose distance to the next one means
# nothing (a product 7.6 -> 6.3 us of host time, SwiGLU 6.6 -> 5.4).
def _refuse(what, why):
    raise MoEError(1, f"{what}: {why}")


def _no_graph(what):
    """A call was given tensors that require gradients: it would lose them where torch records a graph."""
    if torch.is_grad_enabled():
        _refuse(what, "the operators record no graph: pass detached tensors, or call them under torch.no_grad()")


def _launch_device(what, t, *others):
    """The device of all these tensors, which has to be the current one."""
    dev = t.get_device()
    if dev < 0:
        _refuse(what, "tensors have to be on the GPU")
    for o in others:
        if o is not None and o.get_device() != dev:
            _refuse(what, "tensors have to be on one device")
    if _device() != dev:
        _refuse(what, f"tensors have to be on the current device, cuda:{_device()}")
    return dev


def _rows(what, name, t, dtype, width=None):
    """Values between two rows of the matrix t, whose own values are contiguous."""
    if t.dtype is not dtype or t.dim() != 2:
        _refuse(what, f"{name} has to be a matrix of {dtype}")
    rows, w = t.shape
    if width is not None and w != width:
        _refuse(what, f"{name} has to have {width} columns, not {w}")
    ld, step = t.stride()
    if step != 1 and w > 1:
        _refuse(what, f"the rows of {name} have to be contiguous")
    return ld if rows > 1 else max(w, 1)


def _whole(what, name, t, dtype, shape):
    if t.dtype is not dtype or t.shape != shape or not t.is_contiguous():
        _refuse(what, f"{name} has to be a contiguous tensor of {dtype}, {tuple(shape)}")


def _groups(what, offsets, E):
    if offsets.dtype is not torch.int32 or offsets.shape != (E + 1,) or not offsets.is_contiguous():
        _refuse(what, f"offsets has to be a contiguous vector of {E + 1} int32")


def _live(what, offsets):
    """Address of the number of rows that there are, the last of the offsets (None: all rows)."""
    if offsets is None:
        return None
    if offsets.dtype is not torch.int32 or offsets.dim() != 1 or offsets.shape[0] < 1 or not offsets.is_contiguous():
        _refuse(what, "offsets has to be a contiguous vector of int32")
    return offsets.data_ptr() + 4 * (offsets.shape[0] - 1)


def _out_rows(what, name, out, rows, width):
    """Values between the rows of the output `out`, bf16 [rows, width]."""
    ld = _rows(what, name, out, torch.bfloat16, width)
    if out.shape[0] != rows:
        _refuse(what, f"{name} has to have {rows} rows")
    return ld


def _done(st, what):
    if st != 0:
        raise MoEError(st, what)


@functools.lru_cache(maxsize=4096)
def _workspace_bytes(name, *sizes):
    """What a call of these sizes needs (it follows from them alone)."""
    return getattr(load_library(), name)(*sizes)


def _workspace(t, name, *sizes):
    """(workspace or None, its address, its bytes) for a call on t's device."""
    n = _workspace_bytes(name, *sizes)
    if n == 0:
        return None, None, 0
    ws = t.new_empty(n, dtype=_U8)
    return ws, ws.data_ptr(), n


def _grouped_checked(what, x, K, w, E, offsets, out):
    """(values between the rows of x, device), or what is wrong."""
    if w.dim() != 3 or w.dtype is not _BF16 or not w.is_contiguous():
        _refuse(what, "w has to be a contiguous tensor of bfloat16 with three dimensions")
    ldx = _rows(what, "x", x, _BF16, K)
    _groups(what, offsets, E)
    return ldx, _launch_device(what, x, w, offsets, out)


def moe_grouped_gemm(x, w, offsets, transpose_w=False, out=None):
    """y[r] = x[r] @ w[e] (transpose_w: @ w[e].T) for the rows r of every expert e.  x [rows, K] bf16; w [E, K, N]
    (transpose_w: [E, N, K]) bf16; offsets [E + 1] int32.  Rows from offsets[E] on are left as they are.
    out shares no memory with the inputs."""
    lib, what = _lib or load_library(), "moe_grouped_gemm"
    if w.dim() != 3 or x.dim() != 2:
        _grouped_checked(what, x, None, w, -1, offsets, out)
        _refuse(what, "w has to have three dimensions, x two")
    if x.requires_grad or w.requires_grad or out is not None and out.requires_grad:
        _no_graph(what)
    E, K, N = w.shape
    t = 0
    if transpose_w:
        K, N, t = N, K, 1
    (rows, width), (ldx, step), dev = x.shape, x.stride(), x.get_device()
    if not (x.dtype is _BF16 and w.dtype is _BF16 and offsets.dtype is _I32T and width == K and step == 1
            and (ldx == K or ldx > K and rows > 1) and w.is_contiguous() and offsets.shape == (E + 1,) and offsets.is_contiguous()
            and dev >= 0 and w.get_device() == dev and offsets.get_device() == dev and _device() == dev):
        ldx, dev = _grouped_checked(what, x, K, w, E, offsets, out)
    y = out
    if out is None:
        y, ldy = x.new_empty(rows, N), N
    else:
        ldy = _out_rows(what, "out", out, rows, N)
        _launch_device(what, x, out)
    ws, at, n = _workspace(x, "moe_grouped_gemm_workspace_bytes", rows, E, K, N, t)
    st = lib.moe_grouped_gemm(x.data_ptr(), ldx, w.data_ptr(), t, offsets.data_ptr(), rows, E, K, N, y.data_ptr(), ldy, at, n,
                              _stream_of(dev))
    if st != 0:
        raise MoEError(st, what)
    if out is not None:
        _wrote(out)
    return y


def moe_grouped_gemm_wgrad(x, dy, offsets, dtype=None, out=None, accumulate=False):
    """dw[e] = x[r].T @ dy[r] summed over the rows r of expert e: [E, K, N] of `dtype` (fp32, the default, or bf16).
    accumulate: add to `out` (fp32).  out shares no memory with the inputs."""
    lib, what = _lib or load_library(), "moe_grouped_gemm_wgrad"
    if x.requires_grad or dy.requires_grad or out is not None and out.requires_grad:
        _no_graph(what)
    ldx, lddy = _rows(what, "x", x, _BF16), _rows(what, "dy", dy, _BF16)
    rows, K = x.shape
    if dy.shape[0] != rows:
        _refuse(what, "x and dy have to have as many rows")
    E, N = offsets.shape[0] - 1 if offsets.dim() == 1 else -1, dy.shape[1]
    _groups(what, offsets, E)
    if out is not None:
        if out.dtype not in (_F32, _BF16) or (dtype is not None and out.dtype is not dtype):
            _refuse(what, "out has to be of dtype, float32 or bfloat16")
        _whole(what, "out", out, out.dtype, (E, K, N))
    elif accumulate:
        _refuse(what, "accumulate needs out")
    elif dtype not in (None, _F32, _BF16):
        _refuse(what, "dtype has to be float32 or bfloat16")
    dev = _launch_device(what, x, dy, offsets, out)
    dw = out
    if out is None:
        dw = x.new_empty((max(E, 0), K, N), dtype=dtype or _F32)
    ws, at, n = _workspace(x, "moe_grouped_gemm_wgrad_workspace_bytes", rows, E, K, N)
    st = lib.moe_grouped_gemm_wgrad(x.data_ptr(), ldx, dy.data_ptr(), lddy, offsets.data_ptr(), rows, E, K, N, dw.data_ptr(),
                                    1 if dw.dtype is _F32 else 0, 1 if accumulate else 0, at, n, _stream_of(dev))
    if st != 0:
        raise MoEError(st, what)
    if out is not None:
        _wrote(out)
    return dw


def moe_swiglu(gu, offsets=None, out=None):
    """silu(gu[:, :f]) * gu[:, f:] (bf16).  offsets: rows from its last value on are left as they are.  out may be gu[:, :f] or
    gu[:, f:]."""
    lib, what = _lib or load_library(), "moe_swiglu"
    if gu.requires_grad or out is not None and out.requires_grad:
        _no_graph(what)
    live = None if offsets is None else _live(what, offsets)
    if gu.dim() != 2:
        _refuse(what, "gu has to be a matrix")
    (rows, f2), (ldgu, step), dev = gu.shape, gu.stride(), gu.get_device()
    if f2 & 1:
        _refuse(what, "gu has to have an even number of columns")
    if not (gu.dtype is _BF16 and step == 1 and (ldgu == f2 or ldgu > f2 and rows > 1) and dev >= 0
            and _device() == dev) or offsets is not None:
        ldgu, dev = _rows(what, "gu", gu, _BF16), _launch_device(what, gu, offsets, out)
    f = f2 >> 1
    h = out
    if out is None:
        h, ldh = gu.new_empty(rows, f), f
    else:
        ldh = _out_rows(what, "out", out, rows, f)
        _launch_device(what, gu, out)
    st = lib.moe_swiglu(gu.data_ptr(), ldgu, live, rows, f, h.data_ptr(), ldh, _stream_of(dev))
    if st != 0:
        raise MoEError(st, what)
    if out is not None:
        _wrote(out)
    return h


def moe_swiglu_backward(dh, gu, offsets=None, out=None, h=None):
    """The gradient of gu [rows, 2f] from that of moe_swiglu's result.  h: a matrix [rows, f] that gets that result
    again.  out may be gu itself, h may be dh or a half of gu."""
    lib, what = _lib or load_library(), "moe_swiglu_backward"
    if dh.requires_grad or gu.requires_grad or out is not None and out.requires_grad or h is not None and h.requires_grad:
        _no_graph(what)
    live = None if offsets is None else _live(what, offsets)
    if dh.dim() != 2 or gu.dim() != 2:
        _refuse(what, "dh and gu have to be matrices")
    (rows, f), (lddh, s1), (ldgu, s2), dev = dh.shape, dh.stride(), gu.stride(), gu.get_device()
    if not (dh.dtype is _BF16 and gu.dtype is _BF16 and s1 == 1 and s2 == 1 and gu.shape == (rows, 2 * f)
            and (lddh == f or lddh > f and rows > 1) and (ldgu == 2 * f or ldgu > 2 * f and rows > 1) and dev >= 0
            and dh.get_device() == dev and _device() == dev) or offsets is not None:
        lddh, ldgu = _rows(what, "dh", dh, _BF16), _rows(what, "gu", gu, _BF16, 2 * f)
        if gu.shape[0] != rows:
            _refuse(what, "dh and gu have to have as many rows")
        dev = _launch_device(what, dh, gu, offsets, out, h)
    ldh, at = f, None
    if h is not None:
        ldh, at = _out_rows(what, "h", h, rows, f), h.data_ptr()
        _launch_device(what, gu, h)
    dgu = out
    if out is None:
        dgu, lddgu = gu.new_empty(rows, 2 * f), 2 * f
    else:
        lddgu = _out_rows(what, "out", out, rows, 2 * f)
        _launch_device(what, gu, out)
    st = lib.moe_swiglu_backward(dh.data_ptr(), lddh, gu.data_ptr(), ldgu, live, rows, f, dgu.data_ptr(), lddgu, at, ldh, _stream_of(dev))
    if st != 0:
        raise MoEError(st, what)
    if out is not None:
        _wrote(out)
    if h is not None:
        _wrote(h)
    return dgu


@functools.lru_cache(maxsize=64)
def _packers(n):
    return tuple(struct.Struct(f"={n}{c}").pack for c in "Qqi")


def _grad_list(what, tensors):
    """Host arrays (bytes) of the addresses, sizes and types of a list of gradients, and their devices.  (map over the unbound
    methods, and struct instead of array: a list of a thousand tensors is bound by this.)"""
    T, f32 = torch.Tensor, torch.float32
    types = [t.dtype for t in tensors]
    if not all(map(T.is_contiguous, tensors)) or not {f32, torch.bfloat16}.issuperset(types):
        _refuse(what, "gradients have to be contiguous tensors of float32 or bfloat16")
    pointers, sizes, flags = _packers(len(types))
    return (pointers(*map(T.data_ptr, tensors)), sizes(*map(T.numel, tensors)), flags(*[t is f32 for t in types]),
            set(map(T.get_device, tensors)))


def _norm_of(what, tensors, devices, call):
    n = _workspace_bytes("moe_grad_norm_workspace_bytes", len(tensors))
    if tensors:
        like = tensors[0]
        dev = like.get_device()
        if len(devices) > 1 or dev < 0 or _device() != dev:
            _launch_device(what, like)
            _refuse(what, "tensors have to be on one device")
    else:
        dev = torch.cuda.current_device()
        like = torch.empty(0, device=torch.device("cuda", dev))
    # (memory of its own for the norm: programs keep it longer than the workspace)
    ws, norm = like.new_empty(n, dtype=_U8), like.new_empty((), dtype=_F32)
    st = call(ws.data_ptr(), n, norm.data_ptr(), _stream_of(dev))
    if st != 0:
        raise MoEError(st, what)
    return norm


def moe_grad_norm(grads):
    """Norm over all values of a list of gradients (float32 or bfloat16), as a tensor on the GPU.  Records no graph."""
    lib, what = _lib or load_library(), "moe_grad_norm"
    grads = list(grads)
    ptrs, counts, types, devices = _grad_list(what, grads)
    return _norm_of(what, grads, devices, lambda ws, n, norm, st: lib.moe_grad_norm(ptrs, counts, types, len(grads), ws, n, norm, st))


def moe_clip_grad_norm(grads, max_norm, out=None):
    """Scales the gradients by min(1, max_norm / (norm + 1e-6)) in place, or into the tensors of `out` (of the same
    types and sizes, overlapping nothing).  Returns the norm before, as a tensor on the GPU.  Records no graph."""
    lib, what = _lib or load_library(), "moe_clip_grad_norm"
    grads = list(grads)
    ptrs, counts, types, devices = _grad_list(what, grads)
    outs, targets = ptrs, grads
    if out is not None:
        targets = list(out)
        outs, n_out, out_types, others = _grad_list(what, targets)
        devices |= others
        if n_out != counts or out_types != types:
            _refuse(what, "out has to hold as many tensors of the same types and sizes")
    norm = _norm_of(what, grads, devices,
                    lambda ws, n, norm, st: lib.moe_clip_grad_norm(ptrs, outs, counts, types, len(grads), max_norm, ws, n, norm, st))
    _wrote(targets)
    return norm


def _mx_pair(what, t, lead, K):
    cols = _workspace_bytes("moe_mxfp4_scale_cols", K)
    if cols == 0:
        raise MoEError(2, what)
    return t.new_empty((*lead, K // 2), dtype=_U8), t.new_empty((*lead, cols), dtype=_U8)


def moe_mxfp4_quantize(x, offsets=None):
    """Rows [n, K] (bf16 or fp32) -> (values [n, K / 2], scales [n, S]), uint8.  offsets: rows from its last value on
    are not quantised."""
    lib, what = _lib or load_library(), "moe_mxfp4_quantize"
    live = None if offsets is None else _live(what, offsets)
    if x.dim() != 2:
        _refuse(what, "x has to be a matrix")
    f32 = x.dtype is _F32
    (rows, K), (ldx, step), dev = x.shape, x.stride(), x.get_device()
    if not ((f32 or x.dtype is _BF16) and step == 1 and (ldx == K or ldx > K and rows > 1) and dev >= 0
            and _device() == dev) or offsets is not None:
        ldx, dev = _rows(what, "x", x, _F32 if f32 else _BF16), _launch_device(what, x, offsets)
    cols = _workspace_bytes("moe_mxfp4_scale_cols", K)
    if cols == 0:
        raise MoEError(2, what)
    values, scales = x.new_empty(rows, K // 2, dtype=_U8), x.new_empty(rows, cols, dtype=_U8)
    st = lib.moe_mxfp4_quantize(x.data_ptr(), 1 if f32 else 0, ldx, live, rows, K, values.data_ptr(), scales.data_ptr(), _stream_of(dev))
    if st != 0:
        raise MoEError(st, what)
    return values, scales


def moe_mxfp4_quantize_weights(w):
    """Weights [E, K, N] (bf16) -> (values [E, N, K / 2], scales [E, N, S]), uint8, blocks along K."""
    lib, what = _lib or load_library(), "moe_mxfp4_quantize_weights"
    if w.dim() != 3 or w.dtype is not torch.bfloat16 or not w.is_contiguous():
        _refuse(what, "w has to be a contiguous tensor of bfloat16 with three dimensions")
    E, K, N = w.shape
    dev = _launch_device(what, w)
    values, scales = _mx_pair(what, w, (E, N), K)
    _done(lib.moe_mxfp4_quantize_weights(w.data_ptr(), E, K, N, values.data_ptr(), scales.data_ptr(),
                                         _stream_of(dev)), what)
    return values, scales


def _mx_check(what, name, values, scales):
    """K of a pair of codes and scales."""
    if values.dim() < 2 or values.dtype is not torch.uint8 or not values.is_contiguous():
        _refuse(what, f"the values of {name} have to be a contiguous tensor of uint8")
    K = 2 * values.shape[-1]
    cols = _workspace_bytes("moe_mxfp4_scale_cols", K)
    if cols == 0:
        raise MoEError(2, what)
    if scales.dtype is not torch.uint8 or scales.shape != (*values.shape[:-1], cols) or not scales.is_contiguous():
        _refuse(what, f"the scales of {name} have to be a contiguous tensor of uint8, {(*values.shape[:-1], cols)}")
    return K


def moe_mxfp4_dequantize(values, scales):
    """The bf16 values [..., K] that codes [..., K / 2] and scales [..., S] stand for."""
    lib, what = _lib or load_library(), "moe_mxfp4_dequantize"
    K = _mx_check(what, "x", values, scales)
    dev = _launch_device(what, values, scales)
    out = values.new_empty((*values.shape[:-1], K), dtype=torch.bfloat16)
    _done(lib.moe_mxfp4_dequantize(values.data_ptr(), scales.data_ptr(), out.numel() // K, K, out.data_ptr(), K,
                                   _stream_of(dev)), what)
    return out


def moe_mxfp4_grouped_gemm(x_values, x_scales, w_values, w_scales, offsets, out=None):
    """y[r] = x[r] @ w[e].T on 4-bit rows [n, K / 2] and weights [E, N, K / 2] with their scales; bf16 [n, N]."""
    lib, what = _lib or load_library(), "moe_mxfp4_grouped_gemm"
    if out is not None and out.requires_grad:
        _no_graph(what)
    if x_values.dim() != 2 or w_values.dim() != 3:
        _refuse(what, "x_values has to have two dimensions, w_values three")
    (rows, half), (E, N, w_half), dev = x_values.shape, w_values.shape, x_values.get_device()
    K = 2 * half
    cols = _workspace_bytes("moe_mxfp4_scale_cols", K)
    if not (x_values.dtype is _U8 and x_scales.dtype is _U8 and w_values.dtype is _U8 and w_scales.dtype is _U8
            and offsets.dtype is _I32T and half == w_half and cols and x_scales.shape == (rows, cols) and w_scales.shape == (E, N, cols)
            and offsets.shape == (E + 1,) and x_values.is_contiguous() and x_scales.is_contiguous() and w_values.is_contiguous()
            and w_scales.is_contiguous() and offsets.is_contiguous() and dev >= 0 and x_scales.get_device() == dev
            and w_values.get_device() == dev and w_scales.get_device() == dev and offsets.get_device() == dev and _device() == dev):
        _mx_check(what, "x", x_values, x_scales)
        if _mx_check(what, "w", w_values, w_scales) != K:
            _refuse(what, "x and w have to have the same K")
        _groups(what, offsets, E)
        dev = _launch_device(what, x_values, x_scales, w_values, w_scales, offsets)
    y = out
    if out is None:
        y, ldy = x_values.new_empty(rows, N, dtype=_BF16), N
    else:
        ldy = _out_rows(what, "out", out, rows, N)
        _launch_device(what, x_values, out)
    ws, at, n = _workspace(x_values, "moe_mxfp4_grouped_gemm_workspace_bytes", rows, E, K, N)
    st = lib.moe_mxfp4_grouped_gemm(x_values.data_ptr(), x_scales.data_ptr(), w_values.data_ptr(), w_scales.data_ptr(),
                                    offsets.data_ptr(), rows, E, K, N, y.data_ptr(), ldy, at, n, _stream_of(dev))
    if st != 0:
        raise MoEError(st, what)
    if out is not None:
        _wrote(out)
    return y


# ---- norms around a block ----
def _norm_matrix(what, name, t, rows, d, dtype=None):
    """Values between the rows of t [rows, d], float32 or bfloat16."""
    if t.dtype not in (_F32, _BF16) or (dtype is not None and t.dtype is not dtype):
        _refuse(what, f"{name} has to be of {dtype or 'float32 or bfloat16'}")
    ld = _rows(what, name, t, t.dtype, d)
    if t.shape[0] != rows:
        _refuse(what, f"{name} has to have {rows} rows")
    return ld


def _norm_weights(what, d, *weights):
    """Type of the weights [d], which have to agree (None: ones)."""
    dtype = None
    for w in weights:
        if w is None:
            continue
        if w.dtype not in (_F32, _BF16) or (dtype is not None and w.dtype is not dtype):
            _refuse(what, "weights have to be float32 or bfloat16, all alike")
        dtype = w.dtype
        if w.shape != (d,) or not w.is_contiguous():
            _refuse(what, f"weights have to be contiguous vectors of {d} values")
    return 0 if dtype is _BF16 else 1


def _norm_types(what, stream, block):
    if stream not in (_F32, _BF16) or not (block is stream or block is _BF16):
        _refuse(what, "streams are float32 or bfloat16; what goes into and comes out of a block has their type or is bfloat16")


def _no_graphs(what, *tensors):
    for t in tensors:
        if t is not None and t.requires_grad:
            return _no_graph(what)


def _plain(t, dev):
    return t.is_contiguous() and t.get_device() == dev


def _fits(stream, block):
    return (stream is _BF16 or stream is _F32) and (block is stream or block is _BF16)


def _weight_ok(w, d, dev):
    return (w.dtype is _F32 or w.dtype is _BF16) and w.shape == (d,) and w.is_contiguous() and w.get_device() == dev


def _gate_of(what, gate, rows, d, block):
    """(address, values between its rows; 0: a number for each row) of a gate or its gradient."""
    if gate is None:
        return None, 0
    if gate.dim() == 1:
        _whole(what, "a gate of rows", gate, _F32, (rows,))
        return gate.data_ptr(), 0
    return gate.data_ptr(), _norm_matrix(what, "a gate of values", gate, rows, d, block)


def moe_rms_norm(x, weight=None, eps=1e-6, offsets=None, out=None, dtype=None):
    """x / sqrt(mean(x^2) + eps) * weight for every row of x [rows, d] (float32 or bfloat16), of `dtype`: x's, the default, or bfloat16.
    offsets: rows from its last value on are left as they are.  out may be x."""
    lib, what = _lib or load_library(), "moe_rms_norm"
    if x.requires_grad or weight is not None and weight.requires_grad or out is not None and out.requires_grad:
        _no_graph(what)
    live = None if offsets is None else _live(what, offsets)
    if x.dim() != 2:
        _refuse(what, "x has to be a matrix")
    (rows, d), (ldx, step), dev, stream = x.shape, x.stride(), x.get_device(), x.dtype
    block = dtype or (out.dtype if out is not None else stream)
    wide = weight is None or weight.dtype is _F32
    if not ((stream is _BF16 or stream is _F32) and (block is stream or block is _BF16) and step == 1 and (ldx == d or ldx > d and rows > 1)
            and dev >= 0 and _device() == dev and (weight is None or (wide or weight.dtype is _BF16) and weight.shape == (d,)
                                                   and weight.is_contiguous() and weight.get_device() == dev)) or offsets is not None:
        ldx = _norm_matrix(what, "x", x, rows, d)
        _norm_types(what, stream, block)
        _norm_weights(what, d, weight)
        dev = _launch_device(what, x, weight, offsets, out)
    h, ldh = out, d
    if out is None:
        h = x.new_empty(rows, d, dtype=block)
    else:
        ldh = _norm_matrix(what, "out", out, rows, d, block)
        _launch_device(what, x, out)
    st = lib.moe_rms_norm(x.data_ptr(), 1 if stream is _F32 else 0, ldx, None if weight is None else weight.data_ptr(), 1 if wide else 0, eps,
                          live, rows, d, h.data_ptr(), 1 if block is _F32 else 0, ldh, _stream_of(dev))
    if st != 0:
        raise MoEError(st, what)
    if out is not None:
        _wrote(out)
    return h


def moe_rms_norm_backward(dh, x, weight=None, eps=1e-6, dres=None, offsets=None, out=None):
    """(gradient of x, gradient of the weight in float32; None without a weight) from that of moe_rms_norm's result.  dres: what x gets by another
    way (the residual's), added.  out: where the gradient of x goes; it may be dh, x or dres."""
    lib, what = _lib or load_library(), "moe_rms_norm_backward"
    if (x.requires_grad or dh.requires_grad or weight is not None and weight.requires_grad or dres is not None and dres.requires_grad
            or out is not None and out.requires_grad):
        _no_graph(what)
    live = None if offsets is None else _live(what, offsets)
    if x.dim() != 2:
        _refuse(what, "x has to be a matrix")
    (rows, d), dev, stream, block = x.shape, x.get_device(), x.dtype, dh.dtype
    if (offsets is None and out is None and dh.shape == (rows, d) and _plain(x, dev) and _plain(dh, dev) and _fits(stream, block) and dev >= 0
            and _device() == dev and (weight is None or _weight_ok(weight, d, dev))
            and (dres is None or dres.dtype is stream and dres.shape == (rows, d) and _plain(dres, dev))):
        ldx = lddh = lddres = d
        wt = 0 if weight is not None and weight.dtype is _BF16 else 1
    else:
        ldx, lddh = _norm_matrix(what, "x", x, rows, d), _norm_matrix(what, "dh", dh, rows, d)
        _norm_types(what, stream, block)
        wt = _norm_weights(what, d, weight)
        lddres = 0 if dres is None else _norm_matrix(what, "dres", dres, rows, d, stream)
        dev = _launch_device(what, x, dh, weight, dres, offsets, out)
    dx, lddx = out, d
    if out is None:
        dx = x.new_empty(rows, d)
    else:
        lddx = _norm_matrix(what, "out", out, rows, d, x.dtype)
    dw, at, ws, n = None, None, None, 0
    if weight is not None:
        dw = x.new_empty(d, dtype=_F32)
        ws, at, n = _workspace(x, "moe_norm_backward_workspace_bytes", rows, d)
    st = lib.moe_rms_norm_backward(dh.data_ptr(), 1 if dh.dtype is _F32 else 0, lddh, x.data_ptr(), 1 if x.dtype is _F32 else 0, ldx,
                                   None if weight is None else weight.data_ptr(), wt, eps, None if dres is None else dres.data_ptr(), lddres,
                                   live, rows, d, dx.data_ptr(), lddx, None if dw is None else dw.data_ptr(), at, n, _stream_of(dev))
    if st != 0:
        raise MoEError(st, what)
    if out is not None:
        _wrote(out)
    return dx, dw


def moe_residual_norm(x, y, weight=None, norm=True, gate=None, scale=1.0, next_weight=None, eps=1e-6, offsets=None, out=None, h=None):
    """The end of a block: n = y * weight, with `norm` y / sqrt(mean(y^2) + eps) * weight; out = scale * x + gate * n; and, with
    next_weight, h = out / sqrt(mean(out^2) + eps) * next_weight, what the next block begins with.  Returns (out, h), h None without
    next_weight.  x [rows, d] is the residual stream, y the block's output (of x's type or bfloat16); gate [rows] float32 or [rows, d] of
    y's type.  offsets: rows from its last value on are left as they are.  out and h may each be x, y or a gate of values."""
    lib, what = _lib or load_library(), "moe_residual_norm"
    if (x.requires_grad or y.requires_grad or weight is not None and weight.requires_grad or gate is not None and gate.requires_grad
            or next_weight is not None and next_weight.requires_grad or out is not None and out.requires_grad or h is not None and h.requires_grad):
        _no_graph(what)
    live = None if offsets is None else _live(what, offsets)
    if x.dim() != 2:
        _refuse(what, "x has to be a matrix")
    (rows, d), dev, stream, block = x.shape, x.get_device(), x.dtype, y.dtype
    if (offsets is None and out is None and h is None and (gate is None or gate.dtype is _F32 and gate.shape == (rows,) and _plain(gate, dev)) and y.shape == (rows, d) and _plain(x, dev) and _plain(y, dev)
            and _fits(stream, block) and dev >= 0 and _device() == dev and (weight is None or _weight_ok(weight, d, dev))
            and (next_weight is None or _weight_ok(next_weight, d, dev) and (weight is None or weight.dtype is next_weight.dtype))):
        ldx = ldy = d
        some = weight if weight is not None else next_weight
        wt, gate_at, ldgate = 0 if some is not None and some.dtype is _BF16 else 1, None if gate is None else gate.data_ptr(), 0
    else:
        ldx, ldy = _norm_matrix(what, "x", x, rows, d), _norm_matrix(what, "y", y, rows, d)
        _norm_types(what, stream, block)
        wt = _norm_weights(what, d, weight, next_weight)
        gate_at, ldgate = _gate_of(what, gate, rows, d, block)
        dev = _launch_device(what, x, y, weight, gate, next_weight, offsets, out, h)
    if h is not None and next_weight is None:
        _refuse(what, "h needs next_weight")
    o, ldo, n, ldh = out, d, h, d
    if out is None:
        o = x.new_empty(rows, d)
    else:
        ldo = _norm_matrix(what, "out", out, rows, d, stream)
    if h is not None:
        ldh = _norm_matrix(what, "h", h, rows, d, block)
    elif next_weight is not None:
        n = y.new_empty(rows, d)
    st = lib.moe_residual_norm(x.data_ptr(), 1 if stream is _F32 else 0, ldx, y.data_ptr(), 1 if block is _F32 else 0, ldy,
                               None if weight is None else weight.data_ptr(), wt, 1 if norm else 0, gate_at, ldgate, scale,
                               None if next_weight is None else next_weight.data_ptr(), eps, live, rows, d, o.data_ptr(), ldo,
                               None if n is None else n.data_ptr(), ldh, _stream_of(dev))
    if st != 0:
        raise MoEError(st, what)
    if out is not None:
        _wrote(out)
    if h is not None:
        _wrote(h)
    return o, n


def moe_residual_norm_backward(dout, y, weight=None, out=None, dh=None, norm=True, gate=None, scale=1.0, next_weight=None, eps=1e-6,
                               offsets=None, dx=None, dy=None):
    """Gradients (of x, y, weight, next_weight, gate) from those of moe_residual_norm's results: dout [rows, d] of the stream's type (None:
    zeros) and dh (with next_weight, which needs `out`, the stream that moe_residual_norm returned; None: h was not used).  Weights' gradients
    are float32; where there is no weight or gate, None.  dx and dy: where the first two go; they may be dout, dh, out, y or a gate of
    values, not each other."""
    lib, what = _lib or load_library(), "moe_residual_norm_backward"
    if (y.requires_grad or dout is not None and dout.requires_grad or weight is not None and weight.requires_grad or out is not None and out.requires_grad
            or dh is not None and dh.requires_grad or gate is not None and gate.requires_grad or next_weight is not None and next_weight.requires_grad
            or dx is not None and dx.requires_grad or dy is not None and dy.requires_grad):
        _no_graph(what)
    live = None if offsets is None else _live(what, offsets)
    if y.dim() != 2:
        _refuse(what, "y has to be a matrix")
    if (dh is None) != (next_weight is None):
        _refuse(what, "dh and next_weight come together")
    if dh is not None and out is None:
        _refuse(what, "dh needs out")
    if dout is None and dh is None:
        _refuse(what, "dout or dh has to be there")
    (rows, d), dev, block, stream = y.shape, y.get_device(), y.dtype, (dout if dout is not None else out).dtype
    if (offsets is None and dx is None and dy is None and dout is not None and dout.shape == (rows, d) and _plain(y, dev) and _plain(dout, dev)
            and _fits(stream, block) and dev >= 0 and _device() == dev and (weight is None or _weight_ok(weight, d, dev))
            and (dh is None or dh.dtype is block and out.dtype is stream and dh.shape == (rows, d) and out.shape == (rows, d) and _plain(dh, dev)
                 and _plain(out, dev) and _weight_ok(next_weight, d, dev) and (weight is None or weight.dtype is next_weight.dtype))
            and (gate is None or _plain(gate, dev) and (gate.dtype is _F32 and gate.shape == (rows,) or gate.dtype is block and gate.shape == (rows, d)))):
        ldy = lddout = ldo = lddh = d
        some = weight if weight is not None else next_weight
        wt = 0 if some is not None and some.dtype is _BF16 else 1
        gate_at, ldgate = (None, 0) if gate is None else (gate.data_ptr(), 0 if gate.dim() == 1 else d)
    else:
        ldy = _norm_matrix(what, "y", y, rows, d)
        _norm_types(what, stream, block)
        lddout = 0 if dout is None else _norm_matrix(what, "dout", dout, rows, d, stream)
        ldo, lddh = (0, 0) if dh is None else (_norm_matrix(what, "out", out, rows, d, stream), _norm_matrix(what, "dh", dh, rows, d, block))
        wt = _norm_weights(what, d, weight, next_weight)
        gate_at, ldgate = _gate_of(what, gate, rows, d, block)
        dev = _launch_device(what, y, dout, weight, out, dh, gate, next_weight, offsets, dx, dy)
    gx, lddx, gy, lddy = dx, d, dy, d
    if dx is None:
        gx = y.new_empty(rows, d, dtype=stream)
    else:
        lddx = _norm_matrix(what, "dx", dx, rows, d, stream)
    if dy is None:
        gy = y.new_empty(rows, d)
    else:
        lddy = _norm_matrix(what, "dy", dy, rows, d, block)
    dgate = None if gate is None else gate.new_empty(gate.shape)
    dw = None if weight is None else y.new_empty(d, dtype=_F32)
    dnext = None if next_weight is None else y.new_empty(d, dtype=_F32)
    ws, at, n = (None, None, 0) if dw is None and dnext is None else _workspace(y, "moe_norm_backward_workspace_bytes", rows, d)

    def ptr(t):
        return None if t is None else t.data_ptr()

    st = lib.moe_residual_norm_backward(ptr(dout), lddout, ptr(dh), lddh, ptr(out) if dh is not None else None, 1 if stream is _F32 else 0, ldo,
                                        y.data_ptr(), 1 if block is _F32 else 0, ldy, ptr(weight), wt, 1 if norm else 0, gate_at, ldgate, scale,
                                        ptr(next_weight), eps, live, rows, d, gx.data_ptr(), lddx, gy.data_ptr(), lddy, ptr(dgate), d, ptr(dw),
                                        ptr(dnext), at, n, _stream_of(dev))
    if st != 0:
        raise MoEError(st, what)
    if dx is not None:
        _wrote(dx)
    if dy is not None:
        _wrote(dy)
    return gx, gy, dw, dnext, dgate


# ---- orthogonalised updates ----
@functools.lru_cache(maxsize=64)
def _packed(triples):
    return struct.pack(f"={3 * len(triples)}f", *[v for t in triples for v in t])


def _coefficients(what, values, steps):
    """Host array (bytes) of the coefficients [steps][3].  They are turned into numbers before they are looked up: tensors would be found by identity."""
    if not isinstance(steps, int) or not 1 <= steps <= 64:
        _refuse(what, "steps has to be an integer from 1 to 64")
    try:
        try:
            triples = (tuple(map(float, values)),) * steps
        except (TypeError, ValueError, RuntimeError):
            triples = tuple(tuple(map(float, t)) for t in values)
        if len(triples) == steps and all(len(t) == 3 for t in triples):
            return _packed(triples)
    except (TypeError, ValueError, RuntimeError, OverflowError):
        pass
    _refuse(what, "coefficients have to be three numbers, or three for each step")


def _stack(what, name, t):
    """(E, rows, cols, values between matrices, between rows) of a matrix or a stack of them, float32 or bfloat16."""
    if t.dim() not in (2, 3) or t.dtype not in (_F32, _BF16):
        _refuse(what, f"{name} has to be a matrix or a stack of matrices, float32 or bfloat16")
    E, rows, cols = t.shape if t.dim() == 3 else (1, *t.shape)
    *first, ld, step = t.stride()
    if step != 1 and cols > 1:
        _refuse(what, f"the rows of {name} have to be contiguous")
    return E, rows, cols, first[0] if first and E > 1 else 0, ld if rows > 1 else max(cols, 1)


def moe_orthogonalize(g, steps=5, scale=1.0, eps=1e-7, coefficients=(3.4445, -4.7750, 2.0315), out=None, dtype=None):
    """Each matrix of g [rows, cols] or [E, rows, cols] (float32 or bfloat16) near the orthogonal matrix next to it: X = g / (|g| + eps),
    then `steps` times X = a X + (b S + c S S) X with S = X X^T (rows > cols: on the transpose), times scale; of `dtype`, g's by default.
    coefficients: (a, b, c), or one such triple for each step; |a| up to 4000.  out may be g.  Views whose last dimension is contiguous are taken as they are."""
    lib, what = _lib or load_library(), "moe_orthogonalize"
    _no_graphs(what, g, out)
    E, rows, cols, stride, ld = _stack(what, "g", g)
    dtype = dtype or (out.dtype if out is not None else g.dtype)
    if dtype not in (_F32, _BF16):
        _refuse(what, "dtype has to be float32 or bfloat16")
    abc = _coefficients(what, coefficients, steps)
    dev = _launch_device(what, g, out)
    x, ostride, ldo = out, rows * cols, cols
    if out is None:
        x = g.new_empty(g.shape, dtype=dtype)
    else:
        if out.shape != g.shape or out.dtype is not dtype:
            _refuse(what, "out has to be of g's shape and of dtype")
        *_, ostride, ldo = _stack(what, "out", out)
    if g.numel() == 0:
        return x
    ws, at, n = _workspace(g, "moe_orthogonalize_workspace_bytes", E, rows, cols)
    st = lib.moe_orthogonalize(g.data_ptr(), 1 if g.dtype is _F32 else 0, stride, ld, E, rows, cols, abc, steps, eps, scale, x.data_ptr(),
                               1 if dtype is _F32 else 0, ostride, ldo, at, n, _stream_of(dev))
    if st != 0:
        raise MoEError(st, what)
    if out is not None:
        _wrote(out)
    return x


# ---- host-side mapping search (no context, no GPU) ------------------------------------------------
def _curve_arrays(curves):
    import numpy as np
    counts = np.concatenate([np.asarray(c, dtype=np.int32) for c, _ in curves])
    ms = np.concatenate([np.asarray(m, dtype=np.float32) for _, m in curves])
    off = np.zeros(len(curves) + 1, dtype=np.int32)
    off[1:] = np.cumsum([len(c) for c, _ in curves])
    return counts, ms, off


def moe_measure_mfma_rate(iters_per_wave=2500, launches=5, shape=1):
    """Sustained bf16 MFMA rate (TFLOP/s) of the current device under an MFMA-only load; shape 1: 16x16x32
    (the grouped GEMM's instruction), 0: 32x32x16."""
    lib = load_library()
    out = C.c_float()
    st = lib.moe_measure_mfma_rate_of(shape, iters_per_wave, launches, C.byref(out),
                                      torch.cuda.current_stream().cuda_stream)
    if st != 0:
        raise MoEError(st, "moe_measure_mfma_rate_of")
    return out.value


def moe_measure_hbm_read_rate(buf, nontemporal=True, launches=10):
    """GB/s at which a read-only kernel streams the device tensor `buf` (plain or non-temporal loads)."""
    lib = load_library()
    out = C.c_float()
    st = lib.moe_measure_hbm_read_rate(buf.data_ptr(), buf.numel() * buf.element_size(), 1 if nontemporal else 0,
                                       launches, C.byref(out), torch.cuda.current_stream().cuda_stream)
    if st != 0:
        raise MoEError(st, "moe_measure_hbm_read_rate")
    return out.value


def moe_gem_score(trace, curves, mapping):
    """Eq. 1 score of `mapping` (GPU of each expert); trace [S][E] ints; curves: per GPU (counts, ms)."""
    import numpy as np
    lib = load_library()
    t = np.ascontiguousarray(trace, dtype=np.int32)
    counts, ms, off = _curve_arrays(curves)
    m = np.ascontiguousarray(mapping, dtype=np.int32)
    out = C.c_double()
    st = lib.moe_gem_score(t.ctypes.data, t.shape[0], t.shape[1], len(curves), counts.ctypes.data, ms.ctypes.data,
                           off.ctypes.data, m.ctypes.data, C.byref(out))
    if st != 0:
        raise MoEError(st, "moe_gem_score")
    return out.value


def moe_gem_place(trace, curves, noise=None, K=1):
    """The paper's mapping search; returns (mapping [E], score, swaps of the winning restart)."""
    import numpy as np
    lib = load_library()
    t = np.ascontiguousarray(trace, dtype=np.int32)
    counts, ms, off = _curve_arrays(curves)
    nz = np.ascontiguousarray(noise, dtype=np.float32) if noise is not None else None
    mapping = np.zeros(t.shape[1], dtype=np.int32)
    score, swaps = C.c_double(), _I32()
    st = lib.moe_gem_place(t.ctypes.data, t.shape[0], t.shape[1], len(curves), counts.ctypes.data, ms.ctypes.data,
                           off.ctypes.data, nz.ctypes.data if nz is not None else None, K, mapping.ctypes.data,
                           C.byref(score), C.byref(swaps))
    if st != 0:
        raise MoEError(st, "moe_gem_place")
    return mapping, score.value, swaps.value
