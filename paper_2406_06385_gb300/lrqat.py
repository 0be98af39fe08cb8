"""Python binding of liblrqat (the C ABI in include/lrqat.h).

Argument marshalling only: every function here forwards torch tensor pointers
and the current CUDA stream to the C entry point of the same name and raises
``LrqatError`` on a non-OK status.  All computation happens in the library's
CUDA kernels; there is no fallback when the library is missing.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional

PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(PKG, "_lib", "liblrqat.so")

PHI_QFIXED = 0
PHI_INT_PACKED = 1
PHI_BF16 = 2
PHI_FP16 = 3
PHI_FP8_E4M3 = 4
PHI_FP8_E5M2 = 5

STATUS = {0: "LRQAT_OK", -1: "LRQAT_ERR_INVALID_ARG", -2: "LRQAT_ERR_UNSUPPORTED", -3: "LRQAT_ERR_ALIGNMENT",
          -4: "LRQAT_ERR_WORKSPACE", -5: "LRQAT_ERR_CUDA", -6: "LRQAT_ERR_TIMEOUT", -7: "LRQAT_ERR_RANGE"}


class LrqatError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{STATUS.get(status, status)}: {message}")
        self.status = status


class Layer(ctypes.Structure):
    """Mirror of the C struct lrqat_layer."""
    _fields_ = [("m", ctypes.c_int64), ("k", ctypes.c_int64), ("r", ctypes.c_int32), ("alpha", ctypes.c_float),
                ("bits", ctypes.c_int32), ("group_size", ctypes.c_int32), ("phi_format", ctypes.c_int32),
                ("act_bits", ctypes.c_int32), ("zero", ctypes.c_void_p), ("act_per_token", ctypes.c_int32),
                ("u_bf16", ctypes.c_int32)]

    @classmethod
    def from_spec(cls, spec, zero: int = 0) -> "Layer":
        """`zero`: device address of the zero offsets (asymmetric weights), 0 for none."""
        return cls(spec.m, spec.k, spec.r, spec.alpha, spec.bits, spec.group_size, spec.phi_format, spec.act_bits,
                   zero or None, int(getattr(spec, "act_per_token", False)), int(getattr(spec, "u_bf16", False)))


class AdamW(ctypes.Structure):
    """Mirror of lrqat_adamw (App. B, Table B1 defaults)."""
    _fields_ = [("lr_ab", ctypes.c_float), ("lr_s", ctypes.c_float), ("beta1", ctypes.c_float),
                ("beta2", ctypes.c_float), ("eps", ctypes.c_float), ("weight_decay_ab", ctypes.c_float),
                ("weight_decay_s", ctypes.c_float), ("max_grad_norm", ctypes.c_float), ("step", ctypes.c_int32)]

    @classmethod
    def make(cls, lr_ab: float, lr_s: float, step: int, beta1: float = 0.9, beta2: float = 0.95, eps: float = 1e-8,
             weight_decay_ab: float = 0.0, weight_decay_s: float = 0.0, max_grad_norm: float = 1.0) -> "AdamW":
        return cls(lr_ab, lr_s, beta1, beta2, eps, weight_decay_ab, weight_decay_s, max_grad_norm, step)


class AdamWState(ctypes.Structure):
    """Mirror of lrqat_adamw_state: device addresses of the fp32 masters and moments."""
    _fields_ = [(n, ctypes.c_void_p) for n in ("A32", "B32", "mA", "vA", "mB", "vB", "ms", "vs")]


class Norm(ctypes.Structure):
    """Mirror of lrqat_norm."""
    _fields_ = [("k", ctypes.c_int64), ("eps", ctypes.c_float), ("act_bits", ctypes.c_int32)]


_types = None


def _dtypes():
    """(int8, float32, int32, types of a bf16 row array: bf16 or its bits as 16-bit whole numbers) of torch."""
    global _types
    if _types is None:
        import torch
        _types = (torch.int8, torch.float32, torch.int32, frozenset((torch.bfloat16, torch.int16, torch.uint16)))
    return _types


class KVCache(ctypes.Structure):
    """Mirror of lrqat_kv_cache."""
    _fields_ = [("n_blocks", ctypes.c_int64), ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("block", ctypes.c_int32), ("k_codes", ctypes.c_void_p), ("v_codes", ctypes.c_void_p),
                ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p)]
    device = None                      # get_device() of the tensors, where `of` has seen them

    @classmethod
    def of(cls, k_codes, v_codes, k_scale, v_scale) -> "KVCache":
        """`k_codes`, `v_codes`: int8 [n_blocks, n_kv_heads, block, head_dim]; `k_scale`, `v_scale`: fp32
        [n_blocks, n_kv_heads]; all dense.  The cache keeps the tensors alive."""
        shape, scales = k_codes.shape, k_scale.shape
        if (len(shape) != 4 or v_codes.shape != shape or scales != shape[:2] or v_scale.shape != scales
                or not (k_codes.is_contiguous() and v_codes.is_contiguous() and k_scale.is_contiguous()
                        and v_scale.is_contiguous())):
            raise LrqatError(-1, "cache tensors must be dense and of matching shapes")
        i8, f32, _, _ = _types or _dtypes()
        if not (k_codes.dtype is v_codes.dtype is i8 and k_scale.dtype is v_scale.dtype is f32):
            raise LrqatError(-1, "cache codes must be int8 and scales float32")
        if not k_codes.device == v_codes.device == k_scale.device == v_scale.device:
            raise LrqatError(-1, "cache tensors must lie on one device")
        n_blocks, heads, block, d = shape
        cache = cls(n_blocks, heads, d, block, k_codes.data_ptr(), v_codes.data_ptr(), k_scale.data_ptr(),
                    v_scale.data_ptr())
        cache.tensors = (k_codes, v_codes, k_scale, v_scale)
        cache.device = k_codes.get_device()
        return cache


class KVBatch(ctypes.Structure):
    """Mirror of lrqat_kv_batch."""
    _fields_ = [("n_seqs", ctypes.c_int32), ("max_blocks", ctypes.c_int32), ("len", ctypes.c_void_p),
                ("row_start", ctypes.c_void_p), ("block_table", ctypes.c_void_p), ("rows", ctypes.c_int64),
                ("max_rows", ctypes.c_int32), ("max_len", ctypes.c_int32)]
    device = None                      # get_device() of the tensors, where `of` has seen them

    @classmethod
    def of(cls, lens, row_start, block_table, rows: int, max_rows: int, max_len: int) -> "KVBatch":
        """`lens` int32 [n_seqs], `row_start` int32 [n_seqs + 1], `block_table` int32 [n_seqs, max_blocks], all
        dense device tensors, which the batch keeps alive; `rows`, `max_rows`, `max_len`: the host's bounds."""
        n_seqs, max_blocks = block_table.shape
        if (lens.shape != (n_seqs,) or row_start.shape != (n_seqs + 1,)
                or not (lens.is_contiguous() and row_start.is_contiguous() and block_table.is_contiguous())):
            raise LrqatError(-1, "lens, row_start and block_table must be dense, of n_seqs, n_seqs + 1 and n_seqs rows")
        if not lens.dtype is row_start.dtype is block_table.dtype is (_types or _dtypes())[2]:
            raise LrqatError(-1, "lens, row_start and block_table must be int32")
        if not lens.device == row_start.device == block_table.device:
            raise LrqatError(-1, "lens, row_start and block_table must lie on one device")
        batch = cls(n_seqs, max_blocks, lens.data_ptr(), row_start.data_ptr(), block_table.data_ptr(), rows, max_rows,
                    max_len)
        batch.tensors = (lens, row_start, block_table)
        batch.device = lens.get_device()
        return batch


_lib = None


def lib() -> ctypes.CDLL:
    """Loads liblrqat.so; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2406_06385_gb300.build`")
        L = ctypes.CDLL(LIB_PATH)
        vp, i64, sz, ip = ctypes.c_void_p, ctypes.c_int64, ctypes.c_size_t, ctypes.c_int
        lp = ctypes.POINTER(Layer)
        L.lrqat_last_error.restype = ctypes.c_char_p
        L.lrqat_last_error.argtypes = []
        sigs = {
            "lrqat_range_minmax": [lp, vp, vp, vp],
            "lrqat_downcast": [lp, vp, vp, vp, vp],
            "lrqat_linear_fwd": [lp, i64, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp],
            "lrqat_linear_fwd_noalloc": [lp, i64, vp, vp, vp, vp, vp, vp, vp, vp],
            "lrqat_linear_bwd": [lp, i64, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, ip, vp, sz, vp],
            "lrqat_linear_fwd_quantized": [lp, i64, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp],
            "lrqat_linear_bwd_quantized": [lp, i64, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, ip, vp, sz, vp],
            "lrqat_merge": [lp, vp, vp, vp, vp, vp],
            "lrqat_get_device_status": [vp],
            "lrqat_grad_sqnorm": [lp, vp, vp, vp, vp, vp],
            "lrqat_range_lp": [lp, vp, ctypes.c_float, ctypes.c_int32, vp, vp],
            "lrqat_act_quant": [lp, ctypes.c_int64, vp, vp, vp, vp, vp],
            "lrqat_adamw_step": [lp, ctypes.POINTER(AdamW), vp, vp, vp, vp, ctypes.POINTER(AdamWState), vp, vp, vp,
                                 vp],
        }
        np_, cp, bp = ctypes.POINTER(Norm), ctypes.POINTER(KVCache), ctypes.POINTER(KVBatch)
        i32, f32 = ctypes.c_int32, ctypes.c_float
        sigs.update({
            "lrqat_add_rmsnorm_fwd": [np_, i64, vp, vp, vp, vp, vp, vp, vp, vp],
            "lrqat_add_rmsnorm_bwd": [np_, i64, vp, vp, vp, vp, vp, vp, ip, vp, sz, vp],
            "lrqat_act_dequant": [np_, i64, vp, vp, vp, vp],
            "lrqat_kv_write": [cp, bp, vp, i64, vp, i64, vp],
            "lrqat_kv_read": [cp, bp, vp, i64, vp, i64, vp],
            "lrqat_kv_attn": [cp, bp, i32, f32, i32, vp, i64, vp, i64, vp, sz, vp],
        })
        for name, args in sigs.items():
            fn = getattr(L, name)
            fn.argtypes = args
            fn.restype = ctypes.c_int
        for name in ("lrqat_get_gemm_variant", "lrqat_get_dw_schedule", "lrqat_get_lowrank_path"):
            getattr(L, name).argtypes = []
            getattr(L, name).restype = ctypes.c_int
        L.lrqat_set_gemm_variant.argtypes = [ip]
        L.lrqat_set_gemm_variant.restype = ctypes.c_int
        L.lrqat_set_dw_schedule.argtypes = [ip]
        L.lrqat_set_dw_schedule.restype = ctypes.c_int
        L.lrqat_set_lowrank_path.argtypes = [ip]
        L.lrqat_set_lowrank_path.restype = ctypes.c_int
        L.lrqat_trace_enable.argtypes = [ip]
        L.lrqat_trace_enable.restype = ctypes.c_int
        L.lrqat_trace_read.argtypes = [ip, ctypes.POINTER(ctypes.c_char_p), ctypes.POINTER(ctypes.c_int64),
                                       ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_int)]
        L.lrqat_trace_read.restype = ctypes.c_int
        for name in ("lrqat_fwd_workspace_bytes", "lrqat_bwd_workspace_bytes"):
            fn = getattr(L, name)
            fn.argtypes = [lp, i64]
            fn.restype = ctypes.c_size_t
        L.lrqat_add_rmsnorm_bwd_workspace_bytes.argtypes = [np_, i64]
        L.lrqat_add_rmsnorm_bwd_workspace_bytes.restype = ctypes.c_size_t
        L.lrqat_kv_attn_workspace_bytes.argtypes = [cp, bp, i32, i32]
        L.lrqat_kv_attn_workspace_bytes.restype = ctypes.c_size_t
        _lib = L
    return _lib


def _check(status: int) -> None:
    if status != 0:
        raise LrqatError(status, lib().lrqat_last_error().decode())


def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


_current_stream = None


def _current_stream_source():
    """The handle of torch's current stream.  torch's own raw accessors take a tenth of the time of
    torch.cuda.current_stream(), but are not part of its public interface: without them the public one serves."""
    import torch
    device, raw = getattr(torch._C, "_cuda_getDevice", None), getattr(torch._C, "_cuda_getCurrentRawStream", None)
    if device is None or raw is None:
        return lambda: torch.cuda.current_stream().cuda_stream
    return lambda: raw(device())


def _stream(stream) -> Optional[int]:
    if stream is not None:
        return stream if isinstance(stream, int) else stream.cuda_stream
    global _current_stream
    if _current_stream is None:
        _current_stream = _current_stream_source()
    return _current_stream()


def last_error() -> str:
    return lib().lrqat_last_error().decode()


def range_minmax(layer: Layer, W0, s0, stream=None) -> None:
    _check(lib().lrqat_range_minmax(ctypes.byref(layer), _ptr(W0), _ptr(s0), _stream(stream)))


def downcast(layer: Layer, W0, s0, Phi0, stream=None) -> None:
    _check(lib().lrqat_downcast(ctypes.byref(layer), _ptr(W0), _ptr(s0), _ptr(Phi0), _stream(stream)))


def fwd_workspace_bytes(layer: Layer, T: int) -> int:
    return int(lib().lrqat_fwd_workspace_bytes(ctypes.byref(layer), T))


def bwd_workspace_bytes(layer: Layer, T: int) -> int:
    return int(lib().lrqat_bwd_workspace_bytes(ctypes.byref(layer), T))


def linear_fwd(layer: Layer, T: int, X, Phi0, s, A, B, s_x, Y, workspace, stream=None) -> None:
    nbytes = workspace.numel() * workspace.element_size() if workspace is not None else 0
    _check(lib().lrqat_linear_fwd(ctypes.byref(layer), T, _ptr(X), _ptr(Phi0), _ptr(s), _ptr(A), _ptr(B), _ptr(s_x),
                                  _ptr(Y), _ptr(workspace), nbytes, _stream(stream)))


def linear_fwd_noalloc(layer: Layer, T: int, X, Phi0, s, A, B, s_x, Y, stream=None) -> None:
    """Forward that takes its scratch from the library's fixed device array (no workspace argument)."""
    _check(lib().lrqat_linear_fwd_noalloc(ctypes.byref(layer), T, _ptr(X), _ptr(Phi0), _ptr(s), _ptr(A), _ptr(B),
                                          _ptr(s_x), _ptr(Y), _stream(stream)))


def linear_bwd(layer: Layer, T: int, dY, X, Phi0, s, A, B, s_x, dX, dA, dB, ds, accumulate: bool, workspace,
               stream=None) -> None:
    nbytes = workspace.numel() * workspace.element_size() if workspace is not None else 0
    _check(lib().lrqat_linear_bwd(ctypes.byref(layer), T, _ptr(dY), _ptr(X), _ptr(Phi0), _ptr(s), _ptr(A), _ptr(B),
                                  _ptr(s_x), _ptr(dX), _ptr(dA), _ptr(dB), _ptr(ds), 1 if accumulate else 0,
                                  _ptr(workspace), nbytes, _stream(stream)))


def linear_fwd_quantized(layer: Layer, T: int, X_q, Phi0, s, A, B, s_x, Y, workspace, stream=None) -> None:
    """Forward on the output of act_quant (per tensor: codes; per token: X_hat)."""
    nbytes = workspace.numel() * workspace.element_size() if workspace is not None else 0
    _check(lib().lrqat_linear_fwd_quantized(ctypes.byref(layer), T, _ptr(X_q), _ptr(Phi0), _ptr(s), _ptr(A), _ptr(B),
                                            _ptr(s_x), _ptr(Y), _ptr(workspace), nbytes, _stream(stream)))


def linear_bwd_quantized(layer: Layer, T: int, dY, X_q, mask, Phi0, s, A, B, s_x, dX, dA, dB, ds, accumulate: bool,
                         workspace, stream=None) -> None:
    """Backward on the output of act_quant and its clip mask (per tensor; None per token)."""
    nbytes = workspace.numel() * workspace.element_size() if workspace is not None else 0
    _check(lib().lrqat_linear_bwd_quantized(ctypes.byref(layer), T, _ptr(dY), _ptr(X_q), _ptr(mask), _ptr(Phi0),
                                            _ptr(s), _ptr(A), _ptr(B), _ptr(s_x), _ptr(dX), _ptr(dA), _ptr(dB),
                                            _ptr(ds), 1 if accumulate else 0, _ptr(workspace), nbytes,
                                            _stream(stream)))


def merge(layer: Layer, Phi0, A, B, W_Z, stream=None) -> None:
    _check(lib().lrqat_merge(ctypes.byref(layer), _ptr(Phi0), _ptr(A), _ptr(B), _ptr(W_Z), _stream(stream)))


def act_quant(layer: Layer, T: int, X, s_x, X_out, mask=None, stream=None) -> None:
    """Activation quantizer on its own (per tensor: codes + optional mask; per token: X_hat)."""
    _check(lib().lrqat_act_quant(ctypes.byref(layer), T, _ptr(X), _ptr(s_x), _ptr(X_out), _ptr(mask),
                                 _stream(stream)))


def range_lp(layer: Layer, W0, s0, p_norm: float, n_candidates: int = 100, stream=None) -> None:
    """L^p range setting over n_candidates scaled min-max scales (symmetric grids)."""
    _check(lib().lrqat_range_lp(ctypes.byref(layer), _ptr(W0), p_norm, n_candidates, _ptr(s0), _stream(stream)))


def grad_sqnorm(layer: Layer, dA, dB, ds, sqnorm, stream=None) -> None:
    """Adds the squared L2 norm of the layer's gradients to the device scalar sqnorm."""
    _check(lib().lrqat_grad_sqnorm(ctypes.byref(layer), _ptr(dA), _ptr(dB), _ptr(ds), _ptr(sqnorm), _stream(stream)))


def adamw_step(layer: Layer, opt: AdamW, sqnorm, dA, dB, ds, state: dict, s, A, B, stream=None) -> None:
    """One clipped AdamW step; `state` maps A32, B32, mA, vA, mB, vB, ms, vs to device tensors."""
    st = AdamWState(*[_ptr(state[n]) for n, _ in AdamWState._fields_])
    _check(lib().lrqat_adamw_step(ctypes.byref(layer), ctypes.byref(opt), _ptr(sqnorm), _ptr(dA), _ptr(dB), _ptr(ds),
                                  ctypes.byref(st), _ptr(s), _ptr(A), _ptr(B), _stream(stream)))


def add_rmsnorm_fwd(norm: Norm, T: int, X, R, gamma, H, Y, Y_q, s_y, stream=None) -> None:
    """h = X + R (R and H may be None), y = gamma h / rms(h).  act_bits 0: Y = bf16(y); act_bits 8: per-token
    codes Y_q with scales s_y and / or their values Y (the X_q of linear_fwd_quantized)."""
    _check(lib().lrqat_add_rmsnorm_fwd(ctypes.byref(norm), T, _ptr(X), _ptr(R), _ptr(gamma), _ptr(H), _ptr(Y),
                                       _ptr(Y_q), _ptr(s_y), _stream(stream)))


def add_rmsnorm_bwd_workspace_bytes(norm: Norm, T: int) -> int:
    return int(lib().lrqat_add_rmsnorm_bwd_workspace_bytes(ctypes.byref(norm), T))


def add_rmsnorm_bwd(norm: Norm, T: int, dY, dH, H, gamma, dX, dgamma, accumulate: bool, workspace,
                    stream=None) -> None:
    """Gradient of add_rmsnorm_fwd at the residual stream H (dH and dgamma may be None; without dgamma the
    workspace may be None)."""
    nbytes = workspace.numel() * workspace.element_size() if workspace is not None else 0
    _check(lib().lrqat_add_rmsnorm_bwd(ctypes.byref(norm), T, _ptr(dY), _ptr(dH), _ptr(H), _ptr(gamma), _ptr(dX),
                                       _ptr(dgamma), 1 if accumulate else 0, _ptr(workspace), nbytes,
                                       _stream(stream)))


def act_dequant(norm: Norm, T: int, codes, s, X_hat, stream=None) -> None:
    """X_hat = bf16(s codes): the values of activations kept as 8-bit codes and per-token scales."""
    _check(lib().lrqat_act_dequant(ctypes.byref(norm), T, _ptr(codes), _ptr(s), _ptr(X_hat), _stream(stream)))


def _rows(t, heads: int, d: int, rows: int = 0) -> int:
    """Distance in elements of consecutive rows of a [rows or more, heads, head_dim] tensor or view."""
    shape, stride = t.shape, t.stride()
    if (len(shape) != 3 or shape[1] != heads or shape[2] != d or shape[0] < rows or stride[2] != 1
            or (heads > 1 and stride[1] != d)):
        raise LrqatError(-1, f"{rows} rows of {heads} heads by {d} expected, dense within a row")
    return stride[0] if shape[0] > 1 else heads * d        # a single row's distance to the next one has no meaning


def _device(cache: KVCache, batch: KVBatch):
    """The CUDA device of a cache and a batch, None where both were filled by hand."""
    a, b = cache.device, batch.device
    if a != b and a is not None and b is not None:
        raise LrqatError(-1, "the cache and the batch must lie on one device")
    if a is None:
        a = b
    if a == -1:
        raise LrqatError(-1, "the cache and the batch must lie on a CUDA device")
    return a


def _row_array(t, heads: int, d: int, rows: int, device) -> int:
    """Checks a row array of a call and returns its row distance (see _rows)."""
    if t.dtype not in (_types or _dtypes())[3]:
        raise LrqatError(-1, "row arrays must be bf16 (or its bits as 16-bit whole numbers)")
    if t.get_device() != device and (device is not None or not t.is_cuda):
        raise LrqatError(-1, "row arrays must lie on the device of the cache and the batch")
    return _rows(t, heads, d, rows)


def kv_write(cache: KVCache, batch: KVBatch, K, V, stream=None) -> None:
    """Quantizes the batch's new keys and values, bf16 [rows, n_kv_heads, head_dim], into the cache."""
    h, d, rows, device = cache.n_kv_heads, cache.head_dim, batch.rows, _device(cache, batch)
    ldk, ldv = _row_array(K, h, d, rows, device), _row_array(V, h, d, rows, device)
    _check(lib().lrqat_kv_write(ctypes.byref(cache), ctypes.byref(batch), _ptr(K), ldk, _ptr(V), ldv, _stream(stream)))


def kv_read(cache: KVCache, batch: KVBatch, K, V, stream=None) -> None:
    """Reads the batch's rows back into K and V, bf16 [rows, n_kv_heads, head_dim]."""
    h, d, rows, device = cache.n_kv_heads, cache.head_dim, batch.rows, _device(cache, batch)
    ldk, ldv = _row_array(K, h, d, rows, device), _row_array(V, h, d, rows, device)
    _check(lib().lrqat_kv_read(ctypes.byref(cache), ctypes.byref(batch), _ptr(K), ldk, _ptr(V), ldv, _stream(stream)))


def kv_attn_workspace_bytes(cache: KVCache, batch: KVBatch, n_heads: int, window: int = 0) -> int:
    return int(lib().lrqat_kv_attn_workspace_bytes(ctypes.byref(cache), ctypes.byref(batch), n_heads, window))


def kv_attn(cache: KVCache, batch: KVBatch, Q, softmax_scale: float, window: int, O, workspace, stream=None) -> None:
    """Causal attention of the batch's rows Q over the cache into O, both bf16 [rows, n_heads, head_dim]."""
    nbytes, device = 0, _device(cache, batch)
    if workspace is not None:
        nbytes = workspace.numel() * workspace.element_size()
        if not workspace.is_cuda:
            raise LrqatError(-1, "the workspace must lie on the device")
    shape, d, rows = Q.shape, cache.head_dim, batch.rows
    heads = shape[1] if len(shape) == 3 else 0
    ldq, ldo = _row_array(Q, heads, d, rows, device), _row_array(O, heads, d, rows, device)
    _check(lib().lrqat_kv_attn(ctypes.byref(cache), ctypes.byref(batch), heads, softmax_scale, window, _ptr(Q), ldq,
                               _ptr(O), ldo, _ptr(workspace), nbytes, _stream(stream)))


def get_device_status(stream=None) -> None:
    _check(lib().lrqat_get_device_status(_stream(stream)))


DW_SCHEDULES = {"auto": 0, "split": 1, "tail": 2}


def set_dw_schedule(schedule: str) -> None:
    """Process-wide schedule of the weight-gradient work: "auto", "split" or "tail"."""
    _check(lib().lrqat_set_dw_schedule(DW_SCHEDULES[schedule]))


GEMM_VARIANTS = {"auto": 0, "single": 1, "pair": 2}


def set_gemm_variant(variant: str) -> None:
    """Process-wide kernels of the forward, dX and dW GEMMs: "auto" (CTA pairs where they were
    measured faster, the default), "single" (one SM per tile) or "pair" (CTA pairs wherever
    the shapes allow)."""
    _check(lib().lrqat_set_gemm_variant(GEMM_VARIANTS[variant]))


def gemm_variant() -> str:
    return {v: k for k, v in GEMM_VARIANTS.items()}[lib().lrqat_get_gemm_variant()]


def dw_schedule() -> str:
    return {v: k for k, v in DW_SCHEDULES.items()}[lib().lrqat_get_dw_schedule()]


LOWRANK_PATHS = {"auto": 0, "tile": 1, "codes": 2}


def set_lowrank_path(path: str) -> None:
    """Process-wide source of the low-rank term in the forward and dX GEMMs: "auto" (the
    default), "tile" (computed inside each GEMM stage; ranks up to 64) or "codes" (one pass per
    call writes the codes of every weight, which the GEMMs read)."""
    _check(lib().lrqat_set_lowrank_path(LOWRANK_PATHS[path]))


def lowrank_path() -> str:
    return {v: k for k, v in LOWRANK_PATHS.items()}[lib().lrqat_get_lowrank_path()]


def trace_enable(enable: bool = True) -> None:
    _check(lib().lrqat_trace_enable(1 if enable else 0))


def trace_read(max_entries: int = 32):
    """Per-kernel {name: (launches, total_ms)} recorded since trace_enable(True)."""
    names = (ctypes.c_char_p * max_entries)()
    launches = (ctypes.c_int64 * max_entries)()
    ms = (ctypes.c_double * max_entries)()
    count = ctypes.c_int(0)
    _check(lib().lrqat_trace_read(max_entries, names, launches, ms, ctypes.byref(count)))
    return {names[i].decode(): (int(launches[i]), float(ms[i])) for i in range(min(count.value, max_entries))}
