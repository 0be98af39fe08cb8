"""Python binding of liblrqat (the C ABI in include/lrqat.h).

Argument marshalling only: every function here forwards torch tensor pointers
and the current CUDA stream to the C entry point of the same name and raises
``LrqatError`` on a non-OK status.  All computation happens in the library's
CUDA kernels; there is no fallback when the library is missing.

The calls of a serving step first try a short way (csrc/binding.cpp), which looks at the same arguments in
compiled code and returns None for whatever it does not find in order; the checks here then say what is wrong.
"""
from __future__ import annotations

import ctypes
import os
import sys
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


def _fits(**numbers) -> None:
    """Refuses whole numbers beyond the 32 bits of the C interface, whose lower bits ctypes would pass."""
    for name, v in numbers.items():
        if not -1 << 31 <= v < 1 << 31:
            raise LrqatError(-1, f"{name} must fit 32 bits (got {v})")


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
        if _short is not None:
            cache = cls()
            device = _short.fill_cache(cache, k_codes, v_codes, k_scale, v_scale)
            if device is not None:
                cache.tensors = (k_codes, v_codes, k_scale, v_scale)
                cache.device = device
                return cache
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
        if _short is not None:
            batch = cls()
            device = _short.fill_batch(batch, lens, row_start, block_table, rows, max_rows, max_len)
            if device is not None:
                batch.tensors = (lens, row_start, block_table)
                batch.device = device
                return batch
        n_seqs, max_blocks = block_table.shape
        if (lens.shape != (n_seqs,) or row_start.shape != (n_seqs + 1,)
                or not (lens.is_contiguous() and row_start.is_contiguous() and block_table.is_contiguous())):
            raise LrqatError(-1, "lens, row_start and block_table must be dense, of n_seqs, n_seqs + 1 and n_seqs rows")
        if not lens.dtype is row_start.dtype is block_table.dtype is (_types or _dtypes())[2]:
            raise LrqatError(-1, "lens, row_start and block_table must be int32")
        if not lens.device == row_start.device == block_table.device:
            raise LrqatError(-1, "lens, row_start and block_table must lie on one device")
        _fits(max_rows=max_rows, max_len=max_len)
        batch = cls(n_seqs, max_blocks, lens.data_ptr(), row_start.data_ptr(), block_table.data_ptr(), rows, max_rows,
                    max_len)
        batch.tensors = (lens, row_start, block_table)
        batch.device = lens.get_device()
        return batch


class QKRope(ctypes.Structure):
    """Mirror of lrqat_qk_rope."""
    _fields_ = [("n_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("rot_dim", ctypes.c_int32), ("neighbours", ctypes.c_int32), ("eps", ctypes.c_float),
                ("turns", ctypes.c_void_p)]
    device = None                      # get_device() of the turns, where `of` has seen them

    @classmethod
    def of(cls, n_heads: int, n_kv_heads: int, head_dim: int, turns, neighbours: bool = False,
           eps: float = 1e-6) -> "QKRope":
        """`turns`: rope_turns of the frequencies on the device (int64, one for each pair that rotates), or None; it is
        kept alive."""
        if turns is not None:
            import torch
            if turns.dtype is not torch.int64 or turns.dim() != 1 or not turns.is_contiguous() or not turns.is_cuda:
                raise LrqatError(-1, "turns must be a dense int64 vector on the device")
        _fits(n_heads=n_heads, n_kv_heads=n_kv_heads, head_dim=head_dim)
        rope = cls(n_heads, n_kv_heads, head_dim, 0 if turns is None else 2 * turns.numel(), int(neighbours), eps,
                   _ptr(turns))
        rope.turns_tensor = turns
        if turns is not None:
            rope.device = turns.get_device()
        return rope


class KVBlocks(ctypes.Structure):
    """Mirror of lrqat_kv_blocks."""
    _fields_ = [("n_seqs", ctypes.c_int32), ("max_blocks", ctypes.c_int32), ("block", ctypes.c_int32),
                ("pinned", ctypes.c_int32), ("capacity", ctypes.c_int64), ("block_table", ctypes.c_void_p),
                ("free_ids", ctypes.c_void_p)]
    device = None                      # get_device() of the tensors, where `of` has seen them

    @classmethod
    def of(cls, block_table, free_ids, block: int, pinned: int = 0) -> "KVBlocks":
        """`block_table` int32 [n_seqs, max_blocks], `free_ids` int32 [capacity], dense device tensors, which are kept
        alive."""
        if _short is not None:
            blocks = cls()
            device = _short.fill_blocks(blocks, block_table, free_ids, block, pinned)
            if device is not None:
                blocks.tensors = (block_table, free_ids)
                blocks.device = device
                return blocks
        i32 = (_types or _dtypes())[2]
        if block_table.dim() != 2 or free_ids.dim() != 1 or not (block_table.is_contiguous() and free_ids.is_contiguous()):
            raise LrqatError(-1, "block_table and free_ids must be dense, of two and one dimensions")
        if not block_table.dtype is free_ids.dtype is i32:
            raise LrqatError(-1, "block_table and free_ids must be int32")
        if block_table.device != free_ids.device or not block_table.is_cuda:
            raise LrqatError(-1, "block_table and free_ids must lie on one device")
        _fits(block=block, pinned=pinned)
        n_seqs, max_blocks = block_table.shape
        blocks = cls(n_seqs, max_blocks, block, pinned, free_ids.shape[0], block_table.data_ptr(), free_ids.data_ptr())
        blocks.tensors = (block_table, free_ids)
        blocks.device = block_table.get_device()
        return blocks


_lib = None
_short = None                          # csrc/binding.cpp
_short_tried = False


def _load_short():
    """The short way, where it has been built for the torch that is running and loads with it."""
    from importlib.machinery import ExtensionFileLoader
    from importlib.util import module_from_spec, spec_from_file_location
    import torch
    path = os.path.join(os.path.dirname(LIB_PATH), f"lrqat_binding-{torch.__version__.split('+')[0]}-{sys.implementation.cache_tag}.so")
    if not os.path.exists(path):
        return None
    spec = spec_from_file_location("lrqat_binding", path, loader=ExtensionFileLoader("lrqat_binding", path))
    try:
        module = module_from_spec(spec)
        spec.loader.exec_module(module)
    except ImportError:                # built for a torch of this version with libraries that this one lacks
        return None
    module.structures(QKRope, KVCache, KVBatch, KVBlocks)
    return module


def lib() -> ctypes.CDLL:
    """Loads liblrqat.so; raises if it has not been built."""
    global _lib, _short, _short_tried
    if _lib is not None and not _short_tried and "torch" in sys.modules:
        _short_tried = True
        _short = _load_short()
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
        rp, tp = ctypes.POINTER(QKRope), ctypes.POINTER(KVBlocks)
        i32, f32 = ctypes.c_int32, ctypes.c_float
        sigs.update({
            "lrqat_add_rmsnorm_fwd": [np_, i64, vp, vp, vp, vp, vp, vp, vp, vp],
            "lrqat_add_rmsnorm_bwd": [np_, i64, vp, vp, vp, vp, vp, vp, ip, vp, sz, vp],
            "lrqat_act_dequant": [np_, i64, vp, vp, vp, vp],
            "lrqat_rope_turns": [vp, i32, vp],
            "lrqat_qk_rope_fwd": [rp, i64, vp, vp, i64, vp, i64, vp, vp, vp, i64, vp, i64, vp],
            "lrqat_qk_rope_bwd": [rp, i64, vp, vp, i64, vp, i64, vp, i64, vp, i64, vp, vp, vp, i64, vp, i64, vp, vp, ip,
                                  vp, sz, vp],
            "lrqat_kv_extend": [tp, vp, vp, vp, i64, vp, vp, vp, vp, vp, vp, vp, sz, vp],
            "lrqat_kv_truncate": [tp, vp, vp, vp, vp, vp, vp, sz, vp],
            "lrqat_kv_write": [cp, bp, vp, i64, vp, i64, vp],
            "lrqat_kv_read": [cp, bp, vp, i64, vp, i64, vp],
            "lrqat_kv_attn": [cp, bp, i32, f32, i32, vp, i64, vp, i64, vp, sz, vp],
            "lrqat_kv_attn_sinks": [cp, bp, i32, f32, i32, i32, vp, i64, vp, i64, vp, sz, vp],
            "lrqat_kv_attn_shared": [cp, bp, vp, i32, i32, f32, vp, i64, vp, i64, vp, sz, vp],
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
        L.lrqat_qk_rope_bwd_workspace_bytes.argtypes = [rp, i64]
        L.lrqat_qk_rope_bwd_workspace_bytes.restype = ctypes.c_size_t
        L.lrqat_kv_blocks_workspace_bytes.argtypes = [tp]
        L.lrqat_kv_blocks_workspace_bytes.restype = ctypes.c_size_t
        L.lrqat_kv_attn_workspace_bytes.argtypes = [cp, bp, i32, i32]
        L.lrqat_kv_attn_workspace_bytes.restype = ctypes.c_size_t
        L.lrqat_kv_attn_sinks_workspace_bytes.argtypes = [cp, bp, i32, i32, i32]
        L.lrqat_kv_attn_sinks_workspace_bytes.restype = ctypes.c_size_t
        L.lrqat_kv_attn_shared_workspace_bytes.argtypes = [cp, bp, i32, i32]
        L.lrqat_kv_attn_shared_workspace_bytes.restype = ctypes.c_size_t
        _lib = L
        return lib()
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


_current_device = None


def _on_current(device: int) -> None:
    """Refuses tensors of another device than the current one, on which the library launches."""
    global _current_device
    if _current_device is None:
        import torch
        _current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
    if device != _current_device():
        raise LrqatError(-1, f"the tensors lie on device {device}, which is not the current one")


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


def _scratch(workspace, device):
    """(address, bytes) of a workspace on the call's device (None: any); its bytes are there where it is dense."""
    if workspace is None:
        return None, 0
    at = workspace.get_device()
    if at < 0 or (device is not None and at != device):
        raise LrqatError(-1, "the workspace must lie on the device of the call's other arrays")
    if not workspace.is_contiguous():
        raise LrqatError(-1, "the workspace must be dense")
    return workspace.data_ptr(), workspace.numel() * workspace.element_size()


def rope_turns(freq):
    """The frequencies `freq` (radians a position: base ** (-2 i / rot_dim), or a scaled variant) as the fractions of a turn
    that QKRope takes: an int64 host tensor."""
    import torch
    freq = torch.as_tensor(freq, dtype=torch.float64, device="cpu").contiguous()
    turns = torch.empty(freq.shape, dtype=torch.int64)
    _check(lib().lrqat_rope_turns(freq.data_ptr(), freq.numel(), turns.data_ptr()))
    return turns


def _vector(t, n: int, dtype, device, name: str) -> Optional[int]:
    """Address of a dense vector of at least n elements on the call's device (None: none)."""
    if t is None:
        return None
    if t.dtype is not dtype or t.numel() < n or not t.is_contiguous():
        raise LrqatError(-1, f"{name} must be dense, {dtype}, of at least {n} elements")
    if t.get_device() != device or not t.is_cuda:
        raise LrqatError(-1, f"{name} must lie on the device of the call's other arrays")
    return t.data_ptr()


def _head_rows(t, heads: int, d: int, rows, device, name: str):
    """(address, row distance, rows, device) of a row array [rows, heads, head_dim] of a call whose rows and device
    are given, or None; no heads: no array."""
    if heads == 0:
        return None, 0, rows, device
    if t is None:
        raise LrqatError(-1, f"{name} must be given")
    at = t.get_device()
    if t.dtype not in (_types or _dtypes())[3] or at < 0 or (device is not None and at != device):
        raise LrqatError(-1, f"{name} must be bf16 (or its bits as 16-bit whole numbers), on the device of the other arrays")
    n = t.shape[0]
    if rows is not None and n != rows:
        raise LrqatError(-1, f"{name} must have as many rows as the other arrays ({rows})")
    return t.data_ptr(), _rows(t, heads, d), n, at


def _rope_on(rope: QKRope, device) -> None:
    """Refuses a rotation whose turns lie on another device than a call's arrays, which have to be on the current one."""
    _on_current(device)
    if rope.device is not None and rope.device != device:
        raise LrqatError(-1, f"the turns lie on device {rope.device}, the call's arrays on device {device}")


def _gamma(t, d: int, device) -> Optional[int]:
    if t is None:
        return None
    if t.dtype not in (_types or _dtypes())[3]:
        raise LrqatError(-1, "gamma must be bf16 (or its bits as 16-bit whole numbers)")
    return _vector(t, d, t.dtype, device, "gamma")


def qk_rope_fwd(rope: QKRope, pos, Q, K, gamma_q, gamma_k, Q_out, K_out, stream=None) -> None:
    """Norm of each head (where its gamma is not None) and rotation by position of Q, bf16 [T, n_heads, head_dim], and
    K, bf16 [T, n_kv_heads, head_dim], into Q_out and K_out (which may be Q and K).  pos: int32 [T], or None for row t at
    position t; rows at negative positions are left as they are."""
    if stream is None and _short is not None:
        status = _short.qk_rope_fwd(rope, pos, Q, K, gamma_q, gamma_k, Q_out, K_out)
        if status is not None:
            return _check(status)
    hq, hk, d = rope.n_heads, rope.n_kv_heads, rope.head_dim
    q, ldq, rows, device = _head_rows(Q, hq, d, None, None, "Q")
    k, ldk, rows, device = _head_rows(K, hk, d, rows, device, "K")
    qo, ldqo, _, _ = _head_rows(Q_out, hq, d, rows, device, "Q_out")
    ko, ldko, _, _ = _head_rows(K_out, hk, d, rows, device, "K_out")
    _rope_on(rope, device)
    if pos is not None:
        pos = _vector(pos, rows, (_types or _dtypes())[2], device, "pos")
    _check(lib().lrqat_qk_rope_fwd(ctypes.byref(rope), rows, pos, q, ldq, k, ldk, _gamma(gamma_q, d, device),
                                   _gamma(gamma_k, d, device), qo, ldqo, ko, ldko, _stream(stream)))


def qk_rope_bwd_workspace_bytes(rope: QKRope, T: int) -> int:
    if _short is not None:
        size = _short.qk_rope_bwd_workspace_bytes(rope, T)
        if size is not None:
            return size
    return int(lib().lrqat_qk_rope_bwd_workspace_bytes(ctypes.byref(rope), T))


def qk_rope_bwd(rope: QKRope, pos, dQ_out, dK_out, Q, K, gamma_q, gamma_k, dQ, dK, dgamma_q, dgamma_k, accumulate: bool,
                workspace, stream=None) -> None:
    """Gradient of qk_rope_fwd at its inputs Q and K (None where there is no gamma).  dgamma_q, dgamma_k: fp32 [head_dim] or
    None (without both the workspace may be None)."""
    if stream is None and _short is not None:
        status = _short.qk_rope_bwd(rope, pos, dQ_out, dK_out, Q, K, gamma_q, gamma_k, dQ, dK, dgamma_q, dgamma_k, accumulate,
                                    workspace)
        if status is not None:
            return _check(status)
    hq, hk, d = rope.n_heads, rope.n_kv_heads, rope.head_dim
    _, f32, i32, _ = _types or _dtypes()
    gq, ldgq, rows, device = _head_rows(dQ_out, hq, d, None, None, "dQ_out")
    gk, ldgk, rows, device = _head_rows(dK_out, hk, d, rows, device, "dK_out")
    _rope_on(rope, device)
    # the inputs of heads without a norm are not read
    q, ldq, _, _ = _head_rows(Q, 0 if gamma_q is None else hq, d, rows, device, "Q")
    k, ldk, _, _ = _head_rows(K, 0 if gamma_k is None else hk, d, rows, device, "K")
    dq, lddq, _, _ = _head_rows(dQ, hq, d, rows, device, "dQ")
    dk, lddk, _, _ = _head_rows(dK, hk, d, rows, device, "dK")
    _check(lib().lrqat_qk_rope_bwd(ctypes.byref(rope), rows, _vector(pos, rows, i32, device, "pos"), gq, ldgq, gk, ldgk,
                                   q, ldq, k, ldk, _gamma(gamma_q, d, device), _gamma(gamma_k, d, device), dq, lddq, dk,
                                   lddk, _vector(dgamma_q, d, f32, device, "dgamma_q"),
                                   _vector(dgamma_k, d, f32, device, "dgamma_k"), 1 if accumulate else 0,
                                   *_scratch(workspace, device), _stream(stream)))


def kv_blocks_workspace_bytes(blocks: KVBlocks) -> int:
    if _short is not None:
        size = _short.kv_blocks_workspace_bytes(blocks)
        if size is not None:
            return size
    return int(lib().lrqat_kv_blocks_workspace_bytes(ctypes.byref(blocks)))


def _blocks_arrays(blocks: KVBlocks, names, arrays, sizes):
    """Addresses of int32 arrays of at least `sizes` elements on the blocks' device, which has to be the current one."""
    i32, device, out = (_types or _dtypes())[2], blocks.device, []
    for name, t, n in zip(names, arrays, sizes):
        if t is None:
            raise LrqatError(-1, f"{name} must be given")
        at = t.get_device()
        if device is None:
            device = at
        if t.dtype is not i32 or t.numel() < n or not t.is_contiguous() or at != device or at < 0:
            raise LrqatError(-1, f"{name} must be dense, int32, of at least {n} elements, on the blocks' device")
        out.append(t.data_ptr())
    _on_current(device)
    return out, device


def kv_extend(blocks: KVBlocks, lens, add, free_count, lens_out, free_out, batch_lens, row_start, pos, slot, workspace,
              stream=None) -> None:
    """Room for add[b] > 0 new tokens behind sequence b's lens[b], or -add[b] rows of padding: blocks from the free list into
    the tables, and the batch's layout.  lens, add, lens_out, batch_lens: int32 [n_seqs]; free_count, free_out: int32 [1];
    row_start: int32 [n_seqs + 1]; pos: int32 [rows]; slot: int64 [rows] or None.  lens_out may be lens, free_out
    free_count."""
    if stream is None and _short is not None:
        status = _short.kv_extend(blocks, lens, add, free_count, lens_out, free_out, batch_lens, row_start, pos, slot, workspace)
        if status is not None:
            return _check(status)
    n, rows = blocks.n_seqs, 0 if pos is None else pos.numel()
    p, device = _blocks_arrays(
        blocks, ("lens", "add", "free_count", "lens_out", "free_out", "batch_lens", "row_start", "pos"),
        (lens, add, free_count, lens_out, free_out, batch_lens, row_start, pos), (n, n, 1, n, 1, n, n + 1, rows))
    if slot is not None:
        import torch
        slot = _vector(slot, rows, torch.int64, device, "slot")
    _check(lib().lrqat_kv_extend(ctypes.byref(blocks), *p[:3], rows, *p[3:], slot, *_scratch(workspace, device),
                                 _stream(stream)))


def kv_truncate(blocks: KVBlocks, lens, keep, free_count, lens_out, free_out, workspace, stream=None) -> None:
    """Shortens sequence b to keep[b] tokens and appends the blocks it no longer needs to the free list.  lens, keep,
    lens_out: int32 [n_seqs]; free_count, free_out: int32 [1]; lens_out may be lens, free_out free_count."""
    if stream is None and _short is not None:
        status = _short.kv_truncate(blocks, lens, keep, free_count, lens_out, free_out, workspace)
        if status is not None:
            return _check(status)
    n = blocks.n_seqs
    p, device = _blocks_arrays(blocks, ("lens", "keep", "free_count", "lens_out", "free_out"),
                               (lens, keep, free_count, lens_out, free_out), (n, n, 1, n, 1))
    _check(lib().lrqat_kv_truncate(ctypes.byref(blocks), *p, *_scratch(workspace, device), _stream(stream)))


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
    if (n_heads | window) >> 31:       # 0.04 us, the call 0.24
        _fits(n_heads=n_heads, window=window)
    return int(lib().lrqat_kv_attn_workspace_bytes(ctypes.byref(cache), ctypes.byref(batch), n_heads, window))


def kv_attn(cache: KVCache, batch: KVBatch, Q, softmax_scale: float, window: int, O, workspace, stream=None) -> None:
    """Causal attention of the batch's rows Q over the cache into O, both bf16 [rows, n_heads, head_dim]."""
    if window >> 31:
        _fits(window=window)
    device = _device(cache, batch)
    room, nbytes = _scratch(workspace, device)
    shape, d, rows = Q.shape, cache.head_dim, batch.rows
    heads = shape[1] if len(shape) == 3 else 0
    ldq, ldo = _row_array(Q, heads, d, rows, device), _row_array(O, heads, d, rows, device)
    _check(lib().lrqat_kv_attn(ctypes.byref(cache), ctypes.byref(batch), heads, softmax_scale, window, _ptr(Q), ldq,
                               _ptr(O), ldo, room, nbytes, _stream(stream)))


def _attn_rows(cache: KVCache, batch: KVBatch, Q, O, workspace):
    """(query heads, row distances of Q and O, workspace and its bytes, device) of an attention call, checked."""
    device = _device(cache, batch)
    room, nbytes = _scratch(workspace, device)
    if device is not None:
        _on_current(device)
    heads = Q.shape[1] if len(Q.shape) == 3 else 0
    return (heads, _row_array(Q, heads, cache.head_dim, batch.rows, device),
            _row_array(O, heads, cache.head_dim, batch.rows, device), room, nbytes, device)


def kv_attn_sinks_workspace_bytes(cache: KVCache, batch: KVBatch, n_heads: int, window: int, sinks: int) -> int:
    if _short is not None:
        size = _short.kv_attn_sinks_workspace_bytes(cache, batch, n_heads, window, sinks)
        if size is not None:
            return size
    _fits(n_heads=n_heads, window=window, sinks=sinks)
    return int(lib().lrqat_kv_attn_sinks_workspace_bytes(ctypes.byref(cache), ctypes.byref(batch), n_heads, window, sinks))


def kv_attn_sinks(cache: KVCache, batch: KVBatch, Q, softmax_scale: float, window: int, sinks: int, O, workspace,
                  stream=None) -> None:
    """kv_attn through a window that leaves the first `sinks` tokens visible."""
    if stream is None and _short is not None:
        status = _short.kv_attn_sinks(cache, batch, Q, softmax_scale, window, sinks, O, workspace)
        if status is not None:
            return _check(status)
    _fits(window=window, sinks=sinks)
    heads, ldq, ldo, room, nbytes, _ = _attn_rows(cache, batch, Q, O, workspace)
    _check(lib().lrqat_kv_attn_sinks(ctypes.byref(cache), ctypes.byref(batch), heads, softmax_scale, window, sinks, _ptr(Q),
                                     ldq, _ptr(O), ldo, room, nbytes, _stream(stream)))


def kv_attn_shared_workspace_bytes(cache: KVCache, batch: KVBatch, n_heads: int, prefix: int) -> int:
    if _short is not None:
        size = _short.kv_attn_shared_workspace_bytes(cache, batch, n_heads, prefix)
        if size is not None:
            return size
    _fits(n_heads=n_heads, prefix=prefix)
    return int(lib().lrqat_kv_attn_shared_workspace_bytes(ctypes.byref(cache), ctypes.byref(batch), n_heads, prefix))


def kv_attn_shared(cache: KVCache, batch: KVBatch, prefix_table, prefix: int, Q, softmax_scale: float, O, workspace,
                   stream=None) -> None:
    """Causal attention of a batch whose sequences start with the same `prefix` tokens (a multiple of the block), which lie
    in the cache blocks prefix_table, int32 [prefix / block]."""
    if stream is None and _short is not None:
        status = _short.kv_attn_shared(cache, batch, prefix_table, prefix, Q, softmax_scale, O, workspace)
        if status is not None:
            return _check(status)
    _fits(prefix=prefix)
    heads, ldq, ldo, room, nbytes, device = _attn_rows(cache, batch, Q, O, workspace)
    columns = -(-prefix // cache.block) if prefix > 0 and cache.block > 0 else 0
    if columns and prefix_table is None:
        raise LrqatError(-1, "prefix_table must be given")
    if prefix_table is not None and device is None:
        device = prefix_table.get_device()
    table = _vector(prefix_table, columns, (_types or _dtypes())[2], device, "prefix_table")
    _check(lib().lrqat_kv_attn_shared(ctypes.byref(cache), ctypes.byref(batch), table, prefix, heads, softmax_scale,
                                      _ptr(Q), ldq, _ptr(O), ldo, room, nbytes, _stream(stream)))


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
