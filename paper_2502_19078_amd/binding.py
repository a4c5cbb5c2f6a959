"""ctypes binding of libclada (argument marshalling only; no arithmetic here).

Function names mirror the C ABI in ``include/clada.h``.  Tensors are torch CUDA
tensors; kernels are enqueued on torch's current stream of the tensor's device.
"""
from __future__ import annotations

import ctypes as C
import os
from dataclasses import dataclass

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libclada.so")
_lib = None

F32, BF16 = 0, 1
_STATUS = ["CLADA_OK", "CLADA_ERR_NULL", "CLADA_ERR_SHAPE", "CLADA_ERR_DTYPE", "CLADA_ERR_ALIGN",
           "CLADA_ERR_WORKSPACE", "CLADA_ERR_VALUE", "CLADA_ERR_HIP"]


class CladaError(RuntimeError):
    def __init__(self, status: int, text: str):
        self.status = status
        name = _STATUS[status] if 0 <= status < len(_STATUS) else f"status {status}"
        super().__init__(f"{name}: {text}")


SWIGLU, RELU, GEGLU = 0, 1, 2      # clada_ffn_kind


class _CLayer(C.Structure):
    _fields_ = [("w_gate", C.c_void_p), ("w_up", C.c_void_p), ("w_down", C.c_void_p),
                ("d", C.c_int32), ("d_ff", C.c_int32), ("dtype", C.c_int), ("kind", C.c_int),
                ("b_in", C.c_void_p), ("b_out", C.c_void_p)]


class _CPrefixOut(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in
                ("sum_abs_act", "sum_sq_act", "max_abs_act", "sum_sq_h", "A", "abs_act_pool")]


class _CHeads(C.Structure):
    _fields_ = [("data", C.c_void_p), ("stride_b", C.c_int64), ("stride_t", C.c_int64), ("stride_h", C.c_int64)]


class _CKvCache(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("stride_b", C.c_int64), ("stride_h", C.c_int64), ("stride_n", C.c_int64),
                ("batch", C.c_int32), ("heads", C.c_int32), ("d", C.c_int32), ("capacity", C.c_int32), ("dtype", C.c_int32),
                ("n_sink", C.c_int32), ("ring", C.c_int32)]


ROPE_HALF, ROPE_PAIRS = 0, 1       # clada_rope_layout
ROPE_SCALE_NONE, ROPE_SCALE_LINEAR, ROPE_SCALE_BASE, ROPE_SCALE_BANDS, ROPE_SCALE_RAMP = range(5)      # clada_rope_scale


class _CRope(C.Structure):
    _fields_ = [("turns", C.c_void_p), ("rotary_dim", C.c_int32), ("layout", C.c_int32), ("magnitude", C.c_float)]


class _CRopeScaling(C.Structure):
    _fields_ = [(n, C.c_double) for n in ("theta", "factor", "original_len", "low", "high")] + [("kind", C.c_int32)]


class _CHeadNorm(C.Structure):
    _fields_ = [("q_weight", C.c_void_p), ("k_weight", C.c_void_p), ("eps", C.c_float), ("offset", C.c_float)]


def lib_path() -> str:
    return _LIB_PATH


def load_library() -> C.CDLL:
    """Load libclada.so; raises if it has not been built (there is no fallback)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise RuntimeError(f"{_LIB_PATH} is missing: build it with "
                           f"`python -m paper_2502_19078_amd.build` (hipcc, gfx950)")
    lib = C.CDLL(_LIB_PATH)
    vp, i32, f32 = C.c_void_p, C.c_int32, C.c_float
    lib.clada_create.argtypes = [C.POINTER(vp), C.c_int, C.c_size_t]
    lib.clada_destroy.argtypes = [vp]
    lib.clada_destroy.restype = None
    lib.clada_status_str.argtypes = [C.c_int]
    lib.clada_status_str.restype = C.c_char_p
    lib.clada_last_error.argtypes = [vp]
    lib.clada_last_error.restype = C.c_char_p
    lib.clada_set_option.argtypes = [vp, C.c_char_p, i32]
    lib.clada_workspace_bytes.argtypes = [i32] * 5
    lib.clada_workspace_bytes.restype = C.c_size_t
    lib.clada_prefix_stats.argtypes = [vp, C.POINTER(_CLayer), vp, i32, vp, C.POINTER(_CPrefixOut), vp]
    lib.clada_threshold_calibrate.argtypes = [vp, vp, C.c_int64, f32, vp, vp]
    lib.clada_cognitive_signals.argtypes = [vp, vp, C.c_int, i32, i32, vp, vp, vp, vp]
    lib.clada_threshold.argtypes = [vp, vp, vp, vp, i32, vp, vp, i32, f32, f32, vp, vp]
    lib.clada_cognitive_signals_static.argtypes = [vp, vp, C.c_int, i32, i32, vp, vp, vp, vp]
    lib.clada_cognitive_signals_static.restype = C.c_int
    lib.clada_signals_threshold.argtypes = [vp, vp, C.c_int, i32, i32, vp, vp, vp, vp, i32, f32, f32, vp, vp, vp, vp]
    lib.clada_sparse_ffn_decode.argtypes = [vp, C.POINTER(_CLayer), vp, i32, vp, vp, vp, vp, vp, vp]
    lib.clada_dense_ffn_decode.argtypes = [vp, C.POINTER(_CLayer), vp, i32, vp, vp]
    lib.clada_sparse_ffn_stack_decode.argtypes = [vp, C.POINTER(_CLayer), i32, vp, i32, vp, vp, vp, vp]
    lib.clada_sparse_ffn_stack_decode.restype = C.c_int
    lib.clada_dense_ffn_stack_decode.argtypes = [vp, C.POINTER(_CLayer), i32, vp, i32, vp, vp]
    lib.clada_dense_ffn_stack_decode.restype = C.c_int
    lib.clada_diag_stream_read.argtypes = [vp, vp, C.c_size_t, i32, vp]
    lib.clada_diag_copy.argtypes = [vp, vp, vp, C.c_size_t, vp]
    lib.clada_threshold_search_cett.argtypes = [vp, C.POINTER(_CLayer), vp, i32, C.c_float, i32, vp, vp, vp]
    lib.clada_cett_eval.argtypes = [vp, C.POINTER(_CLayer), vp, i32, C.c_float, vp, vp, vp]
    lib.clada_static_mask_threshold.argtypes = [vp, vp, i32, vp, vp, vp, vp]
    lib.clada_static_mask_topk.argtypes = [vp, vp, i32, i32, vp, vp, vp]
    lib.clada_static_ffn_decode.argtypes = [vp, C.POINTER(_CLayer), vp, i32, vp, vp, vp, vp]
    lib.clada_mask_pack.argtypes = [vp, vp, vp, i32, vp, vp]
    lib.clada_mask_unpack.argtypes = [vp, vp, i32, vp, vp, vp]
    lib.clada_mask_sparse_max_bytes.argtypes = [i32]
    lib.clada_mask_sparse_max_bytes.restype = C.c_size_t
    lib.clada_mask_sparse_encode.argtypes = [vp, vp, vp, i32, vp, i32, vp, vp]
    lib.clada_mask_sparse_encode.restype = C.c_int
    lib.clada_mask_sparse_decode.argtypes = [vp, vp, vp, i32, vp, i32, vp, vp]
    lib.clada_mask_sparse_decode.restype = C.c_int
    lib.clada_mask_sparse_encode_batch.argtypes = [vp, vp, vp, C.c_int64, i32, i32, vp, i32, vp, vp]
    lib.clada_mask_sparse_encode_batch.restype = C.c_int
    lib.clada_mask_sparse_decode_batch.argtypes = [vp, vp, vp, C.c_int64, i32, vp, C.c_int64, i32, i32, vp, vp]
    lib.clada_mask_sparse_decode_batch.restype = C.c_int
    lib.clada_device_fault.argtypes = [vp, C.POINTER(C.c_int32)]
    lib.clada_graph_begin.argtypes = [vp, vp]
    lib.clada_graph_end.argtypes = [vp, vp, C.POINTER(vp)]
    lib.clada_graph_launch.argtypes = [vp, vp, vp]
    lib.clada_graph_destroy.argtypes = [vp]
    lib.clada_graph_destroy.restype = None
    lib.clada_diag_kernel_times.argtypes = [vp, C.POINTER(C.c_float), C.POINTER(C.c_float)]
    lib.clada_rope_turns.argtypes = [vp, i32, C.POINTER(_CRopeScaling), vp, C.POINTER(C.c_float)]
    lib.clada_qk_rope.argtypes = [vp, vp, vp, i32, i32, i32, vp, vp, vp, vp, vp, vp, vp, vp]
    lib.clada_window_attn.argtypes = [vp, vp, vp, vp, vp, i32, i32, i32, i32, i32, f32, vp, vp, vp]
    lib.clada_shared_prefix_attn.argtypes = [vp, vp, vp, i32, vp, vp, i32, i32, f32, vp, vp, vp]
    lib.clada_attn_workspace_bytes.argtypes = [i32] * 4
    lib.clada_attn_workspace_bytes.restype = C.c_size_t
    for name in ("clada_diag_stream_read", "clada_diag_copy", "clada_diag_kernel_times", "clada_device_fault",
                 "clada_threshold_search_cett", "clada_cett_eval", "clada_static_mask_threshold",
                 "clada_static_mask_topk", "clada_static_ffn_decode", "clada_mask_pack", "clada_mask_unpack", "clada_create", "clada_set_option", "clada_prefix_stats", "clada_threshold_calibrate",
                 "clada_cognitive_signals", "clada_threshold", "clada_signals_threshold", "clada_sparse_ffn_decode",
                 "clada_dense_ffn_decode", "clada_rope_turns", "clada_qk_rope", "clada_window_attn", "clada_shared_prefix_attn"):
        getattr(lib, name).restype = C.c_int
    _lib = lib
    return lib


def workspace_bytes(d: int, d_ff: int, B: int, T: int, V: int) -> int:
    return int(load_library().clada_workspace_bytes(d, d_ff, B, T, V))


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return F32
    if t.dtype == torch.bfloat16:
        return BF16
    raise TypeError(f"unsupported dtype {t.dtype}")


def _ptr(t):
    return None if t is None else t.data_ptr()


# The raw handle of torch's current stream on a device (0.2 us; torch.cuda.current_stream builds a Stream object, 2.1 us of
# the 13 us that a single-token call of a small layer spends on the host).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(t: torch.Tensor):
    if not t.is_cuda:                                        # (the raw call takes a host tensor's -1 for the current device)
        raise ValueError(f"expected a tensor on the GPU, got one on {t.device}")
    if _raw_stream is not None:
        return _raw_stream(t.get_device())
    return torch.cuda.current_stream(t.device).cuda_stream


class Context:
    """Owns a libclada context (its device workspace)."""

    def __init__(self, device: int = 0, workspace_bytes: int = 0):
        self._lib = load_library()
        h = C.c_void_p()
        st = self._lib.clada_create(C.byref(h), int(device), int(workspace_bytes))
        if st != 0:
            raise CladaError(st, self._lib.clada_last_error(None).decode())
        self._h = h
        self.device = device

    def close(self):
        if getattr(self, "_h", None):
            self._lib.clada_destroy(self._h)
            self._h = None

    __del__ = close

    def check(self, st: int):
        if st != 0:
            raise CladaError(st, self._lib.clada_last_error(self._h).decode())

    def device_fault(self) -> bool:
        """True once a balanced decode kernel of this context has given up its bounded wait."""
        f = C.c_int32()
        self.check(self._lib.clada_device_fault(self._h, C.byref(f)))
        return f.value != 0

    def set_option(self, name: str, value: int):
        self.check(self._lib.clada_set_option(self._h, name.encode(), int(value)))


@dataclass
class Layer:
    """Neuron-major weights of one FFN layer, each [d_ff][d] on the GPU.  kind = SWIGLU or GEGLU (gated, sigma = SiLU or tanh-form GELU:
    w_gate, w_up, w_down) or RELU (non-gated, OPT family: w_gate = W_in, w_up = None, w_down = W_out
    neuron-major, optional fp32 biases b_in [d_ff], b_out [d])."""
    w_gate: torch.Tensor
    w_up: torch.Tensor | None
    w_down: torch.Tensor
    kind: int = 0
    b_in: torch.Tensor | None = None
    b_out: torch.Tensor | None = None

    def c_struct(self) -> _CLayer:
        wg, wu, wd = self.w_gate, self.w_up, self.w_down
        shape, dtype = wg.shape, wg.dtype
        F, d = shape
        assert wg.is_cuda and wg.is_contiguous()
        assert wd.is_cuda and wd.is_contiguous() and wd.shape == shape and wd.dtype == dtype
        if self.kind != RELU:
            assert wu.is_cuda and wu.is_contiguous() and wu.shape == shape and wu.dtype == dtype
        b_in, b_out = self.b_in, self.b_out
        assert b_in is None or (b_in.is_cuda and b_in.is_contiguous() and b_in.dtype == torch.float32 and b_in.numel() == F)
        assert b_out is None or (b_out.is_cuda and b_out.is_contiguous() and b_out.dtype == torch.float32 and b_out.numel() == d)
        return _CLayer(wg.data_ptr(), _ptr(wu), wd.data_ptr(), d, F, _dtype_code(wg), self.kind, _ptr(b_in), _ptr(b_out))


@dataclass
class PrefixStats:
    sum_abs_act: torch.Tensor
    sum_sq_act: torch.Tensor
    max_abs_act: torch.Tensor
    sum_sq_h: torch.Tensor
    A: torch.Tensor
    abs_act_pool: torch.Tensor | None
    y: torch.Tensor | None


def prefix_stats(ctx: Context, layer: Layer, x: torch.Tensor, want_y: bool = True,
                 want_pool: bool = True) -> PrefixStats:
    cl = layer.c_struct()
    T = x.shape[0]
    assert x.is_cuda and x.is_contiguous() and x.shape == (T, cl.d) and x.dtype == layer.w_gate.dtype
    f = lambda *s: torch.empty(*s, dtype=torch.float32, device=x.device)
    stats = [f(cl.d_ff) for _ in range(5)]
    pool = f(T, cl.d_ff) if want_pool else None
    y = torch.empty_like(x) if want_y else None
    out = _CPrefixOut(*[s.data_ptr() for s in stats], pool.data_ptr() if want_pool else None)
    ctx.check(ctx._lib.clada_prefix_stats(ctx._h, C.byref(cl), _ptr(x), T, _ptr(y), C.byref(out), _stream(x)))
    return PrefixStats(*stats, pool, y)


def threshold_calibrate(ctx: Context, abs_act_pool: torch.Tensor, target_sparsity: float,
                        out: torch.Tensor | None = None) -> torch.Tensor:
    p = abs_act_pool
    assert p.is_cuda and p.is_contiguous() and p.dtype == torch.float32
    if out is None:
        out = torch.empty(1, dtype=torch.float32, device=p.device)
    ctx.check(ctx._lib.clada_threshold_calibrate(ctx._h, _ptr(p), p.numel(), float(target_sparsity),
                                                 _ptr(out), _stream(p)))
    return out


def threshold_search_cett(ctx: Context, layer: Layer, x_val: torch.Tensor, bound: float = 0.2,
                          n_probes: int = 31, out: torch.Tensor | None = None):
    """(tau_base [1], mean CETT at tau_base [1]) of the error-bounded base-threshold search."""
    cl = layer.c_struct()
    T = x_val.shape[0]
    assert x_val.is_cuda and x_val.is_contiguous() and x_val.shape == (T, cl.d) and x_val.dtype == layer.w_gate.dtype
    if out is None:
        out = torch.empty(1, dtype=torch.float32, device=x_val.device)
    mean = torch.empty(1, dtype=torch.float32, device=x_val.device)
    ctx.check(ctx._lib.clada_threshold_search_cett(ctx._h, C.byref(cl), _ptr(x_val), T, float(bound), int(n_probes),
                                                   _ptr(out), _ptr(mean), _stream(x_val)))
    return out, mean


def cett_eval(ctx: Context, layer: Layer, x_val: torch.Tensor, eps: float):
    """(per-token CETT [T], mean [1]) at cut threshold eps."""
    cl = layer.c_struct()
    T = x_val.shape[0]
    assert x_val.is_cuda and x_val.is_contiguous() and x_val.shape == (T, cl.d) and x_val.dtype == layer.w_gate.dtype
    c = torch.empty(T, dtype=torch.float32, device=x_val.device)
    mean = torch.empty(1, dtype=torch.float32, device=x_val.device)
    ctx.check(ctx._lib.clada_cett_eval(ctx._h, C.byref(cl), _ptr(x_val), T, float(eps), _ptr(c), _ptr(mean),
                                       _stream(x_val)))
    return c, mean


def cognitive_signals(ctx: Context, logits: torch.Tensor, token_ids: torch.Tensor):
    B, V = logits.shape
    assert logits.is_cuda and logits.is_contiguous()
    assert token_ids.is_cuda and token_ids.dtype == torch.int32 and token_ids.numel() == B
    s = torch.empty(B, dtype=torch.float32, device=logits.device)
    h = torch.empty(B, dtype=torch.float32, device=logits.device)
    ctx.check(ctx._lib.clada_cognitive_signals(ctx._h, _ptr(logits), _dtype_code(logits), B, V,
                                               _ptr(token_ids), _ptr(s), _ptr(h), _stream(logits)))
    return s, h


def cognitive_signals_static(ctx: Context, logits: torch.Tensor, token_ids: torch.Tensor,
                             out: tuple[torch.Tensor, torch.Tensor] | None = None):
    """clada_cognitive_signals_static: scratch inside the library, nothing allocated by the call when `out`
    = (surprisal, entropy) is given."""
    B, V = logits.shape
    assert logits.is_cuda and logits.is_contiguous()
    assert token_ids.is_cuda and token_ids.dtype == torch.int32 and token_ids.numel() == B
    if out is None:
        out = (torch.empty(B, dtype=torch.float32, device=logits.device),
               torch.empty(B, dtype=torch.float32, device=logits.device))
    s, h = out
    ctx.check(ctx._lib.clada_cognitive_signals_static(ctx._h, _ptr(logits), _dtype_code(logits), B, V,
                                                      _ptr(token_ids), _ptr(s), _ptr(h), _stream(logits)))
    return s, h


def threshold(ctx: Context, tau_base, lam, gam, surprisal, entropy, tau_s: float, tau_H: float,
              out: torch.Tensor | None = None) -> torch.Tensor:
    L, B = tau_base.numel(), surprisal.numel()
    for t in (tau_base, lam, gam, surprisal, entropy):
        assert t.is_cuda and t.dtype == torch.float32 and t.is_contiguous()
    assert lam.numel() == L and gam.numel() == L and entropy.numel() == B
    if out is None:
        out = torch.empty(L, B, dtype=torch.float32, device=tau_base.device)
    ctx.check(ctx._lib.clada_threshold(ctx._h, _ptr(tau_base), _ptr(lam), _ptr(gam), L, _ptr(surprisal),
                                       _ptr(entropy), B, float(tau_s), float(tau_H), _ptr(out),
                                       _stream(tau_base)))
    return out


def signals_threshold(ctx: Context, logits: torch.Tensor, token_ids: torch.Tensor, tau_base, lam, gam,
                      tau_s: float, tau_H: float, out: torch.Tensor | None = None):
    """(surprisal [B], entropy [B], tau_final [L][B]) from one launch."""
    B, V = logits.shape
    L = tau_base.numel()
    assert logits.is_cuda and logits.is_contiguous()
    assert token_ids.is_cuda and token_ids.dtype == torch.int32 and token_ids.numel() == B
    for t in (tau_base, lam, gam):
        assert t.is_cuda and t.dtype == torch.float32 and t.is_contiguous() and t.numel() == L
    s = torch.empty(B, dtype=torch.float32, device=logits.device)
    h = torch.empty(B, dtype=torch.float32, device=logits.device)
    if out is None:
        out = torch.empty(L, B, dtype=torch.float32, device=logits.device)
    ctx.check(ctx._lib.clada_signals_threshold(ctx._h, _ptr(logits), _dtype_code(logits), B, V, _ptr(token_ids),
                                               _ptr(tau_base), _ptr(lam), _ptr(gam), L, float(tau_s), float(tau_H),
                                               _ptr(s), _ptr(h), _ptr(out), _stream(logits)))
    return s, h, out


def sparse_ffn_decode(ctx: Context, layer: Layer, x: torch.Tensor, tau_final: torch.Tensor,
                      y: torch.Tensor | None = None, want_lists: bool = False):
    """Returns y, or (y, active_idx, n_active, mask_bits) when want_lists."""
    cl = layer.c_struct()
    B = x.shape[0]
    assert x.is_cuda and x.is_contiguous() and x.shape == (B, cl.d) and x.dtype == layer.w_gate.dtype
    assert tau_final.is_cuda and tau_final.dtype == torch.float32 and tau_final.numel() == B
    assert tau_final.is_contiguous()
    if y is None:
        y = torch.empty_like(x)
    idx = cnt = bits = None
    if want_lists:
        idx = torch.full((cl.d_ff,), -1, dtype=torch.int32, device=x.device)
        cnt = torch.empty(1 + B, dtype=torch.int32, device=x.device)
        bits = torch.empty(B, (cl.d_ff + 31) // 32, dtype=torch.int32, device=x.device)
    ctx.check(ctx._lib.clada_sparse_ffn_decode(ctx._h, C.byref(cl), _ptr(x), B, _ptr(tau_final), _ptr(y),
                                               _ptr(idx), _ptr(cnt), _ptr(bits), _stream(x)))
    return (y, idx, cnt, bits) if want_lists else y


def dense_ffn_decode(ctx: Context, layer: Layer, x: torch.Tensor, y: torch.Tensor | None = None):
    cl = layer.c_struct()
    B = x.shape[0]
    assert x.is_cuda and x.is_contiguous() and x.shape == (B, cl.d) and x.dtype == layer.w_gate.dtype
    if y is None:
        y = torch.empty_like(x)
    ctx.check(ctx._lib.clada_dense_ffn_decode(ctx._h, C.byref(cl), _ptr(x), B, _ptr(y), _stream(x)))
    return y


def layer_array(layers):
    """Host array of clada_layer structs for the whole-stack calls (keep it alive while calls use it)."""
    return (_CLayer * len(layers))(*[l.c_struct() for l in layers])


def _stack_batch(layers, x):
    L = len(layers)
    assert x.is_cuda and x.is_contiguous() and x.shape[0] == L and x.dim() in (2, 3) and x.dtype == layers[0].w_gate.dtype
    return L, (1 if x.dim() == 2 else x.shape[1])


def sparse_ffn_stack_decode(ctx: Context, layers, x: torch.Tensor, tau_final: torch.Tensor,
                            y: torch.Tensor | None = None, want_counts: bool = False, c_layers=None):
    """x [L][d] or [L][B][d], tau_final [L] or [L][B] -> y like x (and n_active [L][1+B] int32 with
    want_counts): the L layers of a stack in one call."""
    L, B = _stack_batch(layers, x)
    arr = c_layers if c_layers is not None else layer_array(layers)
    assert tau_final.is_cuda and tau_final.dtype == torch.float32 and tau_final.numel() == L * B and tau_final.is_contiguous()
    if y is None:
        y = torch.empty_like(x)
    cnt = torch.empty(L, 1 + B, dtype=torch.int32, device=x.device) if want_counts else None
    ctx.check(ctx._lib.clada_sparse_ffn_stack_decode(ctx._h, arr, L, _ptr(x), B, _ptr(tau_final), _ptr(y), _ptr(cnt), _stream(x)))
    return (y, cnt) if want_counts else y


def dense_ffn_stack_decode(ctx: Context, layers, x: torch.Tensor, y: torch.Tensor | None = None, c_layers=None):
    L, B = _stack_batch(layers, x)
    arr = c_layers if c_layers is not None else layer_array(layers)
    if y is None:
        y = torch.empty_like(x)
    ctx.check(ctx._lib.clada_dense_ffn_stack_decode(ctx._h, arr, L, _ptr(x), B, _ptr(y), _stream(x)))
    return y


def static_mask_threshold(ctx: Context, A: torch.Tensor, tau_final: torch.Tensor):
    """(active_idx [F] int32, n_active [1] int32): ascending neurons with A_j >= tau_final[0]."""
    assert A.is_cuda and A.dtype == torch.float32 and A.is_contiguous()
    assert tau_final.is_cuda and tau_final.dtype == torch.float32 and tau_final.numel() >= 1
    idx = torch.empty(A.numel(), dtype=torch.int32, device=A.device)
    n = torch.empty(1, dtype=torch.int32, device=A.device)
    ctx.check(ctx._lib.clada_static_mask_threshold(ctx._h, _ptr(A), A.numel(), _ptr(tau_final), _ptr(idx), _ptr(n),
                                                   _stream(A)))
    return idx, n


def static_mask_topk(ctx: Context, score: torch.Tensor, k: int):
    """(active_idx [F] int32, n_active [1] int32): ascending indices of the k largest scores."""
    assert score.is_cuda and score.dtype == torch.float32 and score.is_contiguous()
    idx = torch.empty(score.numel(), dtype=torch.int32, device=score.device)
    n = torch.empty(1, dtype=torch.int32, device=score.device)
    ctx.check(ctx._lib.clada_static_mask_topk(ctx._h, _ptr(score), score.numel(), int(k), _ptr(idx), _ptr(n),
                                              _stream(score)))
    return idx, n


def mask_pack(ctx: Context, active_idx: torch.Tensor, n_active: torch.Tensor, d_ff: int) -> torch.Tensor:
    """Ascending list -> packed bit mask [ceil(d_ff/32)] int32."""
    assert active_idx.is_cuda and active_idx.dtype == torch.int32 and n_active.dtype == torch.int32
    bits = torch.empty((d_ff + 31) // 32, dtype=torch.int32, device=active_idx.device)
    ctx.check(ctx._lib.clada_mask_pack(ctx._h, _ptr(active_idx), _ptr(n_active), int(d_ff), _ptr(bits),
                                       _stream(active_idx)))
    return bits


def mask_unpack(ctx: Context, mask_bits: torch.Tensor, d_ff: int):
    """Packed bit mask -> (active_idx [d_ff] int32, n_active [1] int32)."""
    assert mask_bits.is_cuda and mask_bits.dtype == torch.int32 and mask_bits.numel() >= (d_ff + 31) // 32
    idx = torch.empty(d_ff, dtype=torch.int32, device=mask_bits.device)
    n = torch.empty(1, dtype=torch.int32, device=mask_bits.device)
    ctx.check(ctx._lib.clada_mask_unpack(ctx._h, _ptr(mask_bits), int(d_ff), _ptr(idx), _ptr(n), _stream(mask_bits)))
    return idx, n


def mask_sparse_encode(ctx: Context, mask_bits: torch.Tensor, ref_bits: torch.Tensor | None, d_ff: int,
                       capacity: int | None = None):
    """Bit mask (against a reference mask or None) -> (stream uint8 [capacity], n int32 [2] = bytes or -1, positions)."""
    words = (d_ff + 31) // 32
    assert mask_bits.is_cuda and mask_bits.dtype == torch.int32 and mask_bits.numel() >= words and mask_bits.is_contiguous()
    assert ref_bits is None or (ref_bits.is_cuda and ref_bits.dtype == torch.int32 and ref_bits.numel() >= words
                                and ref_bits.is_contiguous())
    if capacity is None:
        capacity = int(ctx._lib.clada_mask_sparse_max_bytes(int(d_ff)))
    stream = torch.empty(max(capacity, 1), dtype=torch.uint8, device=mask_bits.device)
    n = torch.empty(2, dtype=torch.int32, device=mask_bits.device)
    ctx.check(ctx._lib.clada_mask_sparse_encode(ctx._h, _ptr(mask_bits), _ptr(ref_bits), int(d_ff), _ptr(stream),
                                                int(capacity), _ptr(n), _stream(mask_bits)))
    return stream, n


def mask_sparse_decode(ctx: Context, stream: torch.Tensor, n_bytes: torch.Tensor, ref_bits: torch.Tensor | None,
                       d_ff: int, out: torch.Tensor | None = None) -> torch.Tensor:
    """Stream (+ the reference it was coded against) -> bit mask [ceil(d_ff/32)] int32."""
    assert stream.is_cuda and stream.dtype == torch.uint8 and stream.is_contiguous()
    assert n_bytes.is_cuda and n_bytes.dtype == torch.int32 and n_bytes.numel() >= 1
    if out is None:
        out = torch.empty((d_ff + 31) // 32, dtype=torch.int32, device=stream.device)
    ctx.check(ctx._lib.clada_mask_sparse_decode(ctx._h, _ptr(stream), _ptr(n_bytes), int(stream.numel()), _ptr(ref_bits),
                                                int(d_ff), _ptr(out), _stream(stream)))
    return out


def _ref_stride(ref_bits, n, words):
    if ref_bits is None or ref_bits.dim() == 1:
        return 0
    assert ref_bits.shape == (n, words)
    return words


def mask_sparse_encode_batch(ctx: Context, mask_bits: torch.Tensor, ref_bits: torch.Tensor | None, d_ff: int,
                             capacity: int | None = None):
    """mask_bits [n][words] against ref_bits ([words] shared, [n][words] one each, or None)
    -> (streams uint8 [n][capacity], n_out int32 [n][2])."""
    words = (d_ff + 31) // 32
    assert mask_bits.is_cuda and mask_bits.dtype == torch.int32 and mask_bits.dim() == 2 and mask_bits.shape[1] == words
    assert mask_bits.is_contiguous() and (ref_bits is None or (ref_bits.is_cuda and ref_bits.dtype == torch.int32
                                                               and ref_bits.is_contiguous()))
    n = mask_bits.shape[0]
    if capacity is None:
        capacity = int(ctx._lib.clada_mask_sparse_max_bytes(int(d_ff)))
    streams = torch.empty(n, max(capacity, 1), dtype=torch.uint8, device=mask_bits.device)
    n_out = torch.empty(n, 2, dtype=torch.int32, device=mask_bits.device)
    ctx.check(ctx._lib.clada_mask_sparse_encode_batch(ctx._h, _ptr(mask_bits), _ptr(ref_bits), _ref_stride(ref_bits, n, words),
                                                      int(d_ff), n, _ptr(streams), int(streams.shape[1]), _ptr(n_out),
                                                      _stream(mask_bits)))
    return streams, n_out


def mask_sparse_decode_batch(ctx: Context, streams: torch.Tensor, n_out: torch.Tensor, ref_bits: torch.Tensor | None,
                             d_ff: int) -> torch.Tensor:
    """Streams [n][capacity] with the encoder's n_out [n][2] -> bit masks [n][words] int32."""
    words = (d_ff + 31) // 32
    assert streams.is_cuda and streams.dtype == torch.uint8 and streams.dim() == 2 and streams.is_contiguous()
    n = streams.shape[0]
    assert n_out.is_cuda and n_out.dtype == torch.int32 and n_out.shape == (n, 2) and n_out.is_contiguous()
    out = torch.empty(n, words, dtype=torch.int32, device=streams.device)
    ctx.check(ctx._lib.clada_mask_sparse_decode_batch(ctx._h, _ptr(streams), _ptr(n_out), 2, int(streams.shape[1]),
                                                      _ptr(ref_bits), _ref_stride(ref_bits, n, words), int(d_ff), n,
                                                      _ptr(out), _stream(streams)))
    return out


def static_ffn_decode(ctx: Context, layer: Layer, x: torch.Tensor, active_idx: torch.Tensor,
                      n_active: torch.Tensor, y: torch.Tensor | None = None) -> torch.Tensor:
    cl = layer.c_struct()
    B = x.shape[0]
    assert x.is_cuda and x.is_contiguous() and x.shape == (B, cl.d) and x.dtype == layer.w_gate.dtype
    assert active_idx.is_cuda and active_idx.dtype == torch.int32 and active_idx.is_contiguous()
    assert n_active.is_cuda and n_active.dtype == torch.int32 and n_active.numel() >= 1
    if y is None:
        y = torch.empty_like(x)
    ctx.check(ctx._lib.clada_static_ffn_decode(ctx._h, C.byref(cl), _ptr(x), B, _ptr(active_idx), _ptr(n_active),
                                               _ptr(y), _stream(x)))
    return y


def attn_workspace_bytes(B: int, T: int, Hq: int, d: int) -> int:
    return int(load_library().clada_attn_workspace_bytes(B, T, Hq, d))


class KVCache:
    """Keys and values [batch][heads][capacity][d] on the GPU: two tensors (views with any strides, d contiguous) of one shape and one
    set of strides.  ring = 0: row n holds position n.  ring > 0: positions from n_sink on share `ring` rows behind the first n_sink."""
    __slots__ = ("k", "v", "n_sink", "ring", "heads", "d", "dtype", "device_index", "_c", "_ref")

    def __init__(self, k: torch.Tensor, v: torch.Tensor, n_sink: int = 0, ring: int = 0):
        shape, stride, dtype = k.shape, k.stride(), k.dtype
        assert k.is_cuda and len(shape) == 4 and v.shape == shape and v.dtype is dtype and v.get_device() == k.get_device()
        assert stride[3] == 1 and v.stride() == stride, "k and v need one set of strides, the values of a head contiguous"
        B, H, N, D = shape
        self.k, self.v, self.n_sink, self.ring = k, v, n_sink, ring
        self.heads, self.d, self.dtype, self.device_index = H, D, dtype, k.get_device()
        self._c = _CKvCache(k.data_ptr(), v.data_ptr(), stride[0] if B > 1 else 0, stride[1] if H > 1 else 0, stride[2] if N > 1 else 0,
                            B, H, D, N, _dtype_code(k), n_sink, ring)
        self._ref = C.byref(self._c)


def _heads(x: torch.Tensor, shape, cache: KVCache, what: str):
    """clada_heads of x [B][T][H][d], whose shape is `shape`.  (A dimension of one row has no stride to speak of.)"""
    sb, st, sh, sd = x.stride()
    assert x.get_device() == cache.device_index and x.dtype is cache.dtype and sd == 1 and shape[3] == cache.d, \
        f"{what}: type, device, head size or strides do not fit the cache"
    return C.byref(_CHeads(x.data_ptr(), sb if shape[0] > 1 else 0, st if shape[1] > 1 else 0, sh if shape[2] > 1 else 0))


def _ints(x: torch.Tensor, n: int, cache: KVCache, what: str):
    assert x.dtype is torch.int32 and x.numel() == n and x.is_contiguous() and x.get_device() == cache.device_index, \
        f"{what}: expected {n} contiguous int32 on the cache's device"
    return x.data_ptr()


@dataclass
class RopePlan:
    """Frequencies of a rotation: turns [R/2] int64 on the GPU (the bits of clada_rope.turns), how values pair up, and the factor
    of cosines and sines.  rope_plan computes one."""
    turns: torch.Tensor
    layout: int = ROPE_HALF
    magnitude: float = 1.0


def rope_plan(ctx: Context, rotary_dim: int, theta: float = 10000.0, layout: int = ROPE_HALF, scaling: int = ROPE_SCALE_NONE,
              factor: float = 1.0, original_len: float = 0.0, low: float = 1.0, high: float = 4.0) -> RopePlan:
    """Frequencies theta^(-2i/R), scaled for long contexts as clada_rope_turns says (low and high in waves that fit original_len)."""
    host = torch.empty(max(rotary_dim, 2) // 2, dtype=torch.int64)
    m = C.c_float()
    ctx.check(ctx._lib.clada_rope_turns(ctx._h, int(rotary_dim), C.byref(_CRopeScaling(theta, factor, original_len, low, high, scaling)),
                                        host.data_ptr(), C.byref(m)))
    return RopePlan(host.to(f"cuda:{ctx.device}"), layout, m.value)


def qk_rope(ctx: Context, plan: RopePlan, q: torch.Tensor | None, k: torch.Tensor | None, v: torch.Tensor | None, positions: torch.Tensor,
            cache: KVCache, slots: torch.Tensor | None = None, q_norm: torch.Tensor | None = None, k_norm: torch.Tensor | None = None,
            eps: float = 1e-6, norm_offset: float = 0.0, norm: bool | None = None, out: torch.Tensor | None = None):
    """Norm for each head (norm None: where a weight is given; True without weights: the bare norm), rotation, and keys and values into the cache.  q [B][T][Hq][d], k and v
    [B][T][heads][d] (any strides, d contiguous), positions [B][T] int32 -> rotated queries (None without q)."""
    x = q if q is not None else k
    shape = x.shape
    B, T, Hq, _ = shape
    cq = co = ck = cv = c_norm = None
    if q is not None:
        if out is None:
            out = torch.empty_like(q)
        else:
            assert out.shape == shape
        cq, co = _heads(q, shape, cache, "q"), _heads(out, shape, cache, "out")
    if k is not None:
        kshape = k.shape
        assert v is not None and v.shape == kshape and kshape[0] == B and kshape[1] == T and kshape[2] == cache.heads
        ck, cv = _heads(k, kshape, cache, "k"), _heads(v, kshape, cache, "v")
    turns = plan.turns
    assert turns.get_device() == cache.device_index and turns.dtype is torch.int64 and turns.is_contiguous()
    if norm or (norm is None and (q_norm is not None or k_norm is not None)):
        for w in (q_norm, k_norm):
            assert w is None or (w.get_device() == cache.device_index and w.dtype is cache.dtype and w.is_contiguous() and w.numel() == cache.d)
        c_norm = C.byref(_CHeadNorm(_ptr(q_norm), _ptr(k_norm), eps, norm_offset))
    ctx.check(ctx._lib.clada_qk_rope(ctx._h, C.byref(_CRope(turns.data_ptr(), 2 * turns.numel(), plan.layout, plan.magnitude)), c_norm, B, T, Hq, cq,
                                     ck, cv, _ints(positions, B * T, cache, "positions"),
                                     None if slots is None else _ints(slots, B * T, cache, "slots"), co, cache._ref, _stream(x)))
    return out if q is not None else None


def window_attn(ctx: Context, q: torch.Tensor, cache: KVCache, lens: torch.Tensor, q_lens: torch.Tensor | None = None, window: int = 0,
                sinks: int = 0, scale: float | None = None, out: torch.Tensor | None = None, want_lse: bool = False):
    """Causal attention of q [B][T][Hq][d] over the cache; lens [B] int32 tokens held (the call's own among them), q_lens [B] int32
    queries of every sequence (None: T).  window 0: everything is visible.  scale None: d^-0.5.  Returns out, or (out, lse [B][T][Hq])."""
    shape = q.shape
    B, T, Hq, D = shape
    if out is None:
        out = torch.empty_like(q)
    else:
        assert out.shape == shape
    lse = torch.empty((B, T, Hq), dtype=torch.float32, device=q.device) if want_lse else None
    ctx.check(ctx._lib.clada_window_attn(ctx._h, _heads(q, shape, cache, "q"), cache._ref, _ints(lens, B, cache, "lens"),
                                         None if q_lens is None else _ints(q_lens, B, cache, "q_lens"), B, T, Hq, window, sinks,
                                         D ** -0.5 if scale is None else scale, _heads(out, shape, cache, "out"), _ptr(lse), _stream(q)))
    return (out, lse) if want_lse else out


def shared_prefix_attn(ctx: Context, q: torch.Tensor, prefix: KVCache, prefix_len: int, cache: KVCache, lens: torch.Tensor,
                       scale: float | None = None, out: torch.Tensor | None = None, want_lse: bool = False):
    """One query a sequence, q [B][Hq][d], over the first prefix_len rows of `prefix` (one sequence) and the first lens[b] rows of the
    sequence's own in `cache`.  Returns out, or (out, lse [B][Hq])."""
    B, Hq, D = q.shape
    if out is None:
        out = torch.empty_like(q)
    else:
        assert out.shape == q.shape
    assert prefix.device_index == cache.device_index
    lse = torch.empty((B, Hq), dtype=torch.float32, device=q.device) if want_lse else None
    shape = (B, 1, Hq, D)
    ctx.check(ctx._lib.clada_shared_prefix_attn(ctx._h, _heads(q.unsqueeze(1), shape, cache, "q"), prefix._ref, prefix_len, cache._ref,
                                                _ints(lens, B, cache, "lens"), B, Hq, D ** -0.5 if scale is None else scale,
                                                _heads(out.unsqueeze(1), shape, cache, "out"), _ptr(lse), _stream(q)))
    return (out, lse) if want_lse else out


def diag_stream_read(ctx: Context, src: torch.Tensor, blocks_per_cu: int = 1):
    ctx.check(ctx._lib.clada_diag_stream_read(ctx._h, _ptr(src), src.numel() * src.element_size(),
                                              blocks_per_cu, _stream(src)))


class Graph:
    """One captured decode step (clada_graph_*).  The calls issued on torch's current stream between
    graph_begin and graph_end are recorded; launch() replays them on the current stream."""

    def __init__(self, ctx: Context, handle):
        self._ctx, self._g = ctx, handle

    def launch(self):
        st = C.c_void_p(torch.cuda.current_stream().cuda_stream)
        self._ctx.check(self._ctx._lib.clada_graph_launch(self._ctx._h, self._g, st))

    def __del__(self):
        if getattr(self, "_g", None):
            self._ctx._lib.clada_graph_destroy(self._g)
            self._g = None


def graph_begin(ctx: Context):
    ctx.check(ctx._lib.clada_graph_begin(ctx._h, C.c_void_p(torch.cuda.current_stream().cuda_stream)))


def graph_end(ctx: Context) -> Graph:
    g = C.c_void_p()
    ctx.check(ctx._lib.clada_graph_end(ctx._h, C.c_void_p(torch.cuda.current_stream().cuda_stream), C.byref(g)))
    return Graph(ctx, g)


def diag_copy(ctx: Context, src: torch.Tensor, dst: torch.Tensor):
    assert src.numel() * src.element_size() == dst.numel() * dst.element_size()
    ctx.check(ctx._lib.clada_diag_copy(ctx._h, _ptr(src), _ptr(dst), src.numel() * src.element_size(),
                                       _stream(src)))


def diag_kernel_times(ctx: Context):
    """(main_us, finalize_us) of the context's last decode call; needs option diag.kernel_events = 1."""
    a, b = C.c_float(), C.c_float()
    ctx.check(ctx._lib.clada_diag_kernel_times(ctx._h, C.byref(a), C.byref(b)))
    return a.value, b.value
