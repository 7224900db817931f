"""ctypes binding of include/hero.h.  Marshals arguments; every step runs in libhero.so.

Tensors are torch CUDA tensors used purely as device buffers (data_ptr / shape / stride); the
stream is torch's current CUDA stream unless one is passed.
"""
import ctypes as C
import os
import sys

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libhero.so")

OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_ALIGNMENT, ERR_WORKSPACE, ERR_CUDA, ERR_DEVICE_TIMEOUT = range(7)
I8, U8, I32, F16, BF16, F32 = range(6)
GRAN_NONE, GRAN_TWQ, GRAN_FWQ, GRAN_SQ = range(4)
ACT_NONE, ACT_GELU_ERF, ACT_GELU_TANH, ACT_SILU = range(4)
MASK_NONE, MASK_CAUSAL = range(2)
POST_LN, PRE_LN = range(2)
MODE_INT8, MODE_FP = range(2)
PRESET_FP, PRESET_M1, PRESET_M2, PRESET_M3 = range(4)
MODULES = ("qkv", "attn", "attn_out", "fc1", "fc2")

F8 = 6                      # e4m3 payload of the FP8 variant
_DT = {torch.int8: I8, torch.uint8: U8, torch.int32: I32, torch.float16: F16, torch.bfloat16: BF16,
       torch.float32: F32, torch.float8_e4m3fn: F8}
GRAN = {"none": GRAN_NONE, "twq": GRAN_TWQ, "fwq": GRAN_FWQ, "sq": GRAN_SQ, "fp": GRAN_NONE}
ACT = {"none": ACT_NONE, "gelu_erf": ACT_GELU_ERF, "gelu_tanh": ACT_GELU_TANH, "silu": ACT_SILU}   # silu: hero_moe_linear only
MASK = {"none": MASK_NONE, "causal": MASK_CAUSAL}
FPDT = {"f16": F16, "bf16": BF16}
TORCH_FP = {"f16": torch.float16, "bf16": torch.bfloat16}


class HeroError(RuntimeError):
    def __init__(self, status, msg):
        super().__init__("hero status %d: %s" % (status, msg))
        self.status = status


class Tensor(C.Structure):
    _fields_ = [("data", C.c_void_p), ("dtype", C.c_int32), ("gran", C.c_int32), ("rows", C.c_int64),
                ("cols", C.c_int64), ("ld", C.c_int64), ("scale", C.c_void_p)]


class LnArgs(C.Structure):
    _fields_ = [("residual", Tensor), ("branch", Tensor), ("extra", Tensor), ("token_ids", C.c_void_p),
                ("type_ids", C.c_void_p), ("seq_len", C.c_int32), ("n_tokens", C.c_int64), ("gamma", C.c_void_p),
                ("beta", C.c_void_p), ("eps", C.c_float), ("out", Tensor), ("fp_out", Tensor),
                ("out_col_absmax", C.c_void_p)]


class LinearArgs(C.Structure):
    _fields_ = [("A", Tensor), ("W", C.c_void_p), ("N", C.c_int64), ("ldw", C.c_int64), ("w_scale", C.c_void_p),
                ("bias", C.c_void_p), ("act", C.c_int32), ("post_scale", C.c_void_p), ("out", Tensor),
                ("out_col_absmax", C.c_void_p)]


class AttnArgs(C.Structure):
    _fields_ = [("q", C.c_void_p), ("k", C.c_void_p), ("v", C.c_void_p), ("dtype", C.c_int32), ("ld", C.c_int64),
                ("B", C.c_int32), ("S", C.c_int32), ("nh", C.c_int32), ("dh", C.c_int32), ("s_q", C.c_float),
                ("s_k", C.c_float), ("s_v", C.c_float), ("s_p", C.c_float), ("mask", C.c_int32),
                ("key_len", C.c_void_p), ("out", Tensor), ("p_absmax", C.c_void_p), ("p_mode", C.c_int32),
                ("out_col_absmax", C.c_void_p)]


class AttnProbe(C.Structure):
    _fields_ = [("scores", C.c_void_p), ("p_codes", C.c_void_p), ("acc", C.c_void_p)]


class DecodeAttnArgs(C.Structure):
    _fields_ = [("q", C.c_void_p), ("ld_q", C.c_int64), ("k_cache", C.c_void_p), ("v_cache", C.c_void_p),
                ("ld_kv", C.c_int64), ("batch_stride", C.c_int64), ("k_new", C.c_void_p), ("v_new", C.c_void_p),
                ("ld_new", C.c_int64), ("len", C.c_void_p), ("max_len", C.c_int32), ("B", C.c_int32), ("nh", C.c_int32),
                ("dh", C.c_int32), ("s_q", C.c_float), ("s_k", C.c_float), ("s_v", C.c_float), ("s_p", C.c_float),
                ("p_mode", C.c_int32), ("out", Tensor)]


class LinearParams(C.Structure):
    _fields_ = [("W", C.c_void_p), ("w_scale", C.c_void_p), ("bias", C.c_void_p), ("post_scale", C.c_void_p)]


class LayerDesc(C.Structure):
    _fields_ = [("arch", C.c_int32), ("B", C.c_int32), ("S", C.c_int32), ("H", C.c_int32), ("nh", C.c_int32),
                ("F", C.c_int32), ("act", C.c_int32), ("eps", C.c_float), ("mask", C.c_int32),
                ("fp_dtype", C.c_int32), ("mode", C.c_int32 * 5), ("gran_in", C.c_int32), ("gran_mid", C.c_int32),
                ("gran_attn", C.c_int32), ("gran_out", C.c_int32), ("s_in", C.c_void_p), ("s_mid", C.c_void_p),
                ("s_attn", C.c_void_p), ("s_o", C.c_void_p), ("s_x2", C.c_void_p), ("s_out", C.c_void_p),
                ("s_q", C.c_float), ("s_k", C.c_float), ("s_v", C.c_float), ("s_p", C.c_float),
                ("qkv", LinearParams), ("o", LinearParams), ("fc1", LinearParams), ("fc2", LinearParams),
                ("ln1_g", C.c_void_p), ("ln1_b", C.c_void_p), ("ln2_g", C.c_void_p), ("ln2_b", C.c_void_p),
                ("p_mode", C.c_int32), ("payload", C.c_int32)]


class StackDesc(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("layers", C.POINTER(LayerDesc)), ("edges", C.POINTER(Tensor)),
                ("pending", C.POINTER(Tensor)), ("entry_in", Tensor), ("entry_gamma", C.c_void_p), ("entry_beta", C.c_void_p),
                ("entry_eps", C.c_float)]


class KvCache(C.Structure):
    _fields_ = [("k_cache", C.c_void_p), ("v_cache", C.c_void_p), ("ld_kv", C.c_int64), ("batch_stride", C.c_int64),
                ("len", C.c_void_p), ("max_len", C.c_int32)]


class BlockCache(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("k_scale", C.c_void_p), ("v_scale", C.c_void_p), ("dtype", C.c_int32),
                ("page", C.c_int32), ("n_pages", C.c_int64), ("page_stride", C.c_int64), ("head_stride", C.c_int64),
                ("ld", C.c_int64), ("table", C.c_void_p), ("ld_table", C.c_int64), ("len", C.c_void_p), ("max_len", C.c_int32),
                ("B", C.c_int32), ("nkv", C.c_int32), ("dh", C.c_int32)]


class BlockRowsArgs(C.Structure):
    _fields_ = [("k", Tensor), ("v", Tensor), ("row_start", C.c_void_p), ("max_rows", C.c_int32)]


class BlockAttnArgs(C.Structure):
    _fields_ = [("q", Tensor), ("out", Tensor), ("row_start", C.c_void_p), ("max_rows", C.c_int32), ("nq", C.c_int32),
                ("scale", C.c_float), ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t)]


class QkNormRopeArgs(C.Structure):
    _fields_ = [("q", Tensor), ("k", Tensor), ("q_out", Tensor), ("k_out", Tensor), ("nq", C.c_int32), ("nkv", C.c_int32),
                ("dh", C.c_int32), ("rot", C.c_int32), ("pairing", C.c_int32), ("eps", C.c_float), ("q_gamma", C.c_void_p),
                ("k_gamma", C.c_void_p), ("pos", C.c_void_p), ("cos", C.c_void_p), ("sin", C.c_void_p), ("n_pos", C.c_int64)]


class MoeRouteArgs(C.Structure):
    _fields_ = [("logits", Tensor), ("n_tokens", C.c_void_p), ("select_bias", C.c_void_p), ("top_k", C.c_int32), ("score", C.c_int32),
                ("renorm", C.c_int32), ("scale", C.c_float), ("expert", C.c_void_p), ("weight", C.c_void_p), ("offset", C.c_void_p),
                ("token", C.c_void_p), ("row", C.c_void_p), ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t)]


class MoeLinearArgs(C.Structure):
    _fields_ = [("A", Tensor), ("token", C.c_void_p), ("offset", C.c_void_p), ("W", C.c_void_p), ("N", C.c_int64), ("ldw", C.c_int64),
                ("expert_stride", C.c_int64), ("n_experts", C.c_int32), ("w_scale", C.c_void_p), ("bias", C.c_void_p), ("act", C.c_int32),
                ("gated", C.c_int32), ("post_scale", C.c_void_p), ("out", Tensor), ("out_col_absmax", C.c_void_p)]


class MoeCombineArgs(C.Structure):
    _fields_ = [("y", Tensor), ("row", C.c_void_p), ("weight", C.c_void_p), ("expert", C.c_void_p), ("top_k", C.c_int32), ("n_experts", C.c_int32),
                ("residual", Tensor), ("shared", Tensor), ("gamma", C.c_void_p), ("beta", C.c_void_p), ("eps", C.c_float), ("out", Tensor),
                ("fp_out", Tensor)]


class LayerLayout(C.Structure):
    _fields_ = [(n, C.c_size_t) for n in ("qkv", "x_attn", "x_o", "x_mid", "x_mid_scale", "a", "x_2", "x_in", "x_in_scale",
                                          "h_in", "h_mid", "total")]


P_MODE = {"static": 0, "rowmax": 1}
PAIRING = {"halves": 0, "adjacent": 1}
SCORE = {"softmax": 0, "sigmoid": 1}
HIST_BINS = 2048

EXPORTS = ("hero_create", "hero_destroy", "hero_last_error", "hero_check", "hero_launch_count",
           "hero_layernorm_quant", "hero_w8a8_linear", "hero_int8_attention", "hero_mode_preset",
           "hero_layer_workspace_bytes", "hero_layer_workspace_layout", "hero_layer_forward", "hero_layer_forward_host", "hero_layer_forward_host_async", "hero_profile_begin",
           "hero_profile_end", "hero_layer_forward_static", "hero_absmax_observe", "hero_quantize_weight", "hero_abs_histogram",
           "hero_int8_decode_attention", "hero_layer_decode", "hero_static_check", "hero_int8_attention_probe", "hero_stack_forward",
           "hero_stack_forward_host_async", "hero_quantize_weight_f8", "hero_block_cache_append", "hero_block_cache_read",
           "hero_block_attention_workspace_bytes", "hero_block_attention", "hero_qk_norm_rope", "hero_moe_route_workspace_bytes",
           "hero_moe_route", "hero_moe_linear", "hero_moe_combine")

_lib = None


def lib():
    """The loaded CUDA library.  Missing library = hard error (there is no other implementation)."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise RuntimeError("libhero.so is not built (%s); run `python -m paper_2310_17723_b200.build`. "
                               "There is no fallback path." % _LIB_PATH)
        try:                                     # a library older than its sources is loaded all the same, but said
            from . import build as _build
            if os.path.exists(_build.STAMP) and open(_build.STAMP).read().strip() != _build._digest():
                sys.stderr.write("hero: libhero.so was built from other sources than those in csrc/ now; "
                                 "run `python -m paper_2310_17723_b200.build`\n")
        except OSError:
            pass
        L = C.CDLL(_LIB_PATH)
        L.hero_last_error.restype = C.c_char_p
        L.hero_launch_count.restype = C.c_int64
        L.hero_launch_count.argtypes = [C.c_void_p]
        L.hero_create.argtypes = [C.POINTER(C.c_void_p)]
        L.hero_destroy.argtypes = [C.c_void_p]
        L.hero_check.argtypes = [C.c_void_p, C.c_void_p]
        L.hero_layernorm_quant.argtypes = [C.c_void_p, C.POINTER(LnArgs), C.c_void_p]
        L.hero_w8a8_linear.argtypes = [C.c_void_p, C.POINTER(LinearArgs), C.c_void_p]
        L.hero_int8_attention.argtypes = [C.c_void_p, C.POINTER(AttnArgs), C.c_void_p]
        L.hero_int8_attention_probe.argtypes = [C.c_void_p, C.POINTER(AttnArgs), C.POINTER(AttnProbe), C.c_void_p]
        L.hero_int8_decode_attention.argtypes = [C.c_void_p, C.POINTER(DecodeAttnArgs), C.c_void_p]
        L.hero_mode_preset.argtypes = [C.c_int32, C.POINTER(C.c_int32 * 5)]
        L.hero_layer_workspace_bytes.argtypes = [C.POINTER(LayerDesc), C.c_int64, C.POINTER(C.c_size_t)]
        L.hero_absmax_observe.argtypes = [C.c_void_p, C.POINTER(Tensor), C.c_void_p, C.c_void_p, C.c_void_p]
        L.hero_abs_histogram.argtypes = [C.c_void_p, C.POINTER(Tensor), C.c_float, C.c_void_p, C.c_void_p]
        L.hero_quantize_weight.argtypes = [C.c_void_p, C.c_void_p, C.c_int64, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p,
                                           C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p, C.c_void_p]
        L.hero_quantize_weight_f8.argtypes = L.hero_quantize_weight.argtypes
        L.hero_layer_workspace_layout.argtypes = [C.POINTER(LayerDesc), C.c_int64, C.POINTER(LayerLayout)]
        L.hero_layer_forward.argtypes = [C.c_void_p, C.POINTER(LayerDesc), C.POINTER(Tensor), C.POINTER(Tensor),
                                         C.POINTER(Tensor), C.c_void_p, C.c_size_t, C.c_void_p]
        L.hero_layer_decode.argtypes = [C.c_void_p, C.POINTER(LayerDesc), C.POINTER(KvCache), C.POINTER(Tensor), C.POINTER(Tensor),
                                        C.POINTER(Tensor), C.c_void_p, C.c_size_t, C.c_void_p]
        L.hero_layer_forward_host_async.argtypes = [C.c_void_p, C.POINTER(LayerDesc)] + [C.POINTER(Tensor)] * 4 + \
            [C.c_void_p, C.c_size_t, C.c_void_p]
        L.hero_layer_forward_host.argtypes = [C.c_void_p, C.POINTER(LayerDesc)] + [C.POINTER(Tensor)] * 4 + \
            [C.c_void_p, C.c_size_t, C.c_void_p]
        L.hero_layer_forward_static.argtypes = [C.POINTER(LayerDesc), C.POINTER(Tensor), C.POINTER(Tensor),
                                                C.POINTER(Tensor), C.c_void_p]
        L.hero_static_check.argtypes = [C.c_void_p]
        L.hero_stack_forward.argtypes = [C.c_void_p, C.POINTER(StackDesc), C.c_void_p, C.c_size_t, C.c_void_p]
        L.hero_stack_forward_host_async.argtypes = [C.c_void_p, C.POINTER(StackDesc), C.POINTER(Tensor), C.POINTER(Tensor),
                                                    C.c_void_p, C.c_size_t, C.c_void_p]
        L.hero_block_cache_append.argtypes = [C.c_void_p, C.POINTER(BlockCache), C.POINTER(BlockRowsArgs), C.c_void_p]
        L.hero_block_cache_read.argtypes = L.hero_block_cache_append.argtypes
        L.hero_block_attention_workspace_bytes.argtypes = [C.c_void_p, C.POINTER(BlockCache), C.c_int32, C.c_int64, C.c_int32,
                                                           C.POINTER(C.c_size_t)]
        L.hero_block_attention.argtypes = [C.c_void_p, C.POINTER(BlockCache), C.POINTER(BlockAttnArgs), C.c_void_p]
        L.hero_qk_norm_rope.argtypes = [C.c_void_p, C.POINTER(QkNormRopeArgs), C.c_void_p]
        L.hero_moe_route_workspace_bytes.argtypes = [C.c_void_p, C.c_int64, C.c_int32, C.c_int32, C.POINTER(C.c_size_t)]
        L.hero_moe_route.argtypes = [C.c_void_p, C.POINTER(MoeRouteArgs), C.c_void_p]
        L.hero_moe_linear.argtypes = [C.c_void_p, C.POINTER(MoeLinearArgs), C.c_void_p]
        L.hero_moe_combine.argtypes = [C.c_void_p, C.POINTER(MoeCombineArgs), C.c_void_p]
        L.hero_profile_begin.argtypes = [C.c_void_p, C.c_int32]
        L.hero_profile_end.argtypes = [C.c_void_p, C.POINTER(C.c_float), C.POINTER(C.c_int32), C.POINTER(C.c_int32)]
        _lib = L
    return _lib


def _check(status):
    if status != OK:
        raise HeroError(status, lib().hero_last_error().decode())


def _ptr(t):
    return None if t is None else C.c_void_p(t.data_ptr())


def _stream(stream):
    if stream is None:
        stream = torch.cuda.current_stream()
    return C.c_void_p(stream.cuda_stream)


def tensor(t, gran="none", scale=None):
    """hero_tensor view of a 2-D torch CUDA tensor (row-major, unit inner stride); None -> absent."""
    if t is None:
        return Tensor(None, 0, 0, 0, 0, 0, None)
    assert t.is_cuda and t.dim() == 2 and t.stride(1) == 1, "need a 2-D row-major CUDA tensor"
    if scale is not None:
        assert scale.is_cuda and scale.dtype == torch.float32 and scale.is_contiguous()
    g = GRAN[gran] if isinstance(gran, str) else gran
    ld = t.stride(0) if t.shape[0] > 1 else max(t.stride(0), t.shape[1])
    T = Tensor(t.data_ptr(), _DT[t.dtype], g, t.shape[0], t.shape[1], ld, None if scale is None else scale.data_ptr())
    T._keep = (t, scale)      # the struct holds raw pointers: keep the buffers alive as long as it lives
    T._device = t.get_device()
    return T


def _vector(t, dtype, name):
    """Address of a contiguous CUDA vector (or table) of the given type; None -> absent."""
    if t is None:
        return None
    if not (t.is_cuda and t.dtype == dtype and t.is_contiguous()):
        raise HeroError(ERR_INVALID_ARG, "%s: a contiguous CUDA tensor of %s is needed" % (name, dtype))
    return t.data_ptr()


def block_cache(k, v, k_scale, v_scale, table, lens, max_len):
    """hero_block_cache over k, v: int8 / float8_e4m3fn [n_pages, nkv, page, dh] views of equal strides (feature stride 1;
    a [n_pages, page, nkv, dh] buffer is passed as buffer.transpose(1, 2)); k_scale, v_scale: float32 [n_pages, nkv];
    table: int32 [B, pages per sequence]; lens: int32 [B].  The struct keeps the tensors alive; it can be kept and used for
    every call on the cache, `lens` and `table` being read on the device each time."""
    need = lambda ok, what: None if ok else _refuse(what)      # noqa: E731
    need(k.dim() == 4 and k.shape == v.shape and k.stride() == v.stride() and k.stride(3) == 1, "k, v: [n_pages, nkv, page, dh] views of equal strides")
    need(k.dtype == v.dtype and k.dtype in (torch.int8, torch.float8_e4m3fn), "k, v: int8 or float8_e4m3fn")
    need(k_scale.shape == v_scale.shape == k.shape[:2], "k_scale, v_scale: [n_pages, nkv]")
    need(table.dim() == 2 and lens.shape == (table.shape[0],), "table: [B, pages], lens: [B]")
    need(len({t.device for t in (k, v, k_scale, v_scale, table, lens)}) == 1 and k.is_cuda, "all tensors of a cache live on one CUDA device")
    n, nkv, page, dh = k.shape
    s = BlockCache(k.data_ptr(), v.data_ptr(), _vector(k_scale, torch.float32, "k_scale"), _vector(v_scale, torch.float32, "v_scale"),
                   _DT[k.dtype], page, n, k.stride(0) if n > 1 else max(k.stride(0), dh), k.stride(1) if nkv > 1 else max(k.stride(1), dh),
                   k.stride(2), _vector(table, torch.int32, "table"), table.shape[1], _vector(lens, torch.int32, "lens"), int(max_len),
                   table.shape[0], nkv, dh)
    s._keep = (k, v, k_scale, v_scale, table, lens)
    s._device = k.get_device()
    return s


def _refuse(what):
    raise HeroError(ERR_INVALID_ARG, what)


def _current_raw_stream(device):
    """Address of torch's current stream on `device` (what torch.cuda.current_stream(device).cuda_stream holds, without the
    stream object)."""
    return torch._C._cuda_getCurrentRawStream(device)


_ABSENT = tensor(None)


def _scaled_rows(t, name):
    """A token-wise scale has to reach the tensor's last row (the kernels read one entry per row)."""
    scale = getattr(t, "_keep", (None, None))[1]
    if t.gran == GRAN_TWQ and scale is not None and scale.numel() < t.rows:
        _refuse("%s: a token-wise scale of %d entries for %d rows" % (name, scale.numel(), t.rows))


class Handle:
    """Owns a hero_handle on the current CUDA device."""

    def __init__(self):
        if not torch.cuda.is_available():
            raise RuntimeError("hero needs a CUDA device (sm_100a); none is visible")
        self._h = C.c_void_p()
        _check(lib().hero_create(C.byref(self._h)))
        self._device, self._lib = torch.cuda.current_device(), lib()

    def close(self):
        if self._h:
            lib().hero_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def check(self, stream=None):
        _check(lib().hero_check(self._h, _stream(stream)))

    @property
    def launches(self):
        return int(lib().hero_launch_count(self._h))

    # ---- the four calls of the boundary, same names as the C entry points ----
    def hero_layernorm_quant(self, residual, gamma, beta, eps, out, branch=None, extra=None, fp_out=None,
                             token_ids=None, type_ids=None, seq_len=0, n_tokens=0, out_col_absmax=None, stream=None):
        """residual / branch / extra / out / fp_out are hero.Tensor structs (see `tensor`); out_col_absmax: float32 [H]
        running per-column absolute maximum of the FP tensor the call stores (calibration observer)."""
        a = LnArgs(residual, branch or tensor(None), extra or tensor(None), _ptr(token_ids), _ptr(type_ids),
                   int(seq_len), int(n_tokens), _ptr(gamma), _ptr(beta), float(eps), out or tensor(None),
                   fp_out or tensor(None), _ptr(out_col_absmax))
        _check(lib().hero_layernorm_quant(self._h, C.byref(a), _stream(stream)))

    def hero_w8a8_linear(self, A, W, out, w_scale=None, bias=None, act="none", post_scale=None, out_col_absmax=None,
                         stream=None):
        """A, out: hero.Tensor; W: torch tensor [N, K] (K contiguous); out_col_absmax: float32 [N] running per-column
        absolute maximum of an FP16 / BF16 output (calibration observer fused into the epilogue)."""
        assert W.dim() == 2 and W.stride(1) == 1
        _scaled_rows(A, "A")
        a = LinearArgs(A, W.data_ptr(), W.shape[0], W.stride(0), _ptr(w_scale), _ptr(bias),
                       ACT[act] if isinstance(act, str) else act, _ptr(post_scale), out, _ptr(out_col_absmax))
        _check(lib().hero_w8a8_linear(self._h, C.byref(a), _stream(stream)))

    def hero_int8_attention(self, q, k, v, B, S, nh, dh, out, s_q=1.0, s_k=1.0, s_v=1.0, s_p=1.0 / 255,
                            mask="none", key_len=None, p_absmax=None, p_mode="static", probe=None, out_col_absmax=None,
                            stream=None):
        """q, k, v: 2-D torch views [B*S, nh*dh] sharing one leading dimension; out: hero.Tensor; p_absmax: float32[1]
        running maximum of the softmax probabilities (F16 / BF16 core only).  probe = (scores int32 [B*nh, S, S] | None,
        p_codes uint8 [B*nh, S, S] | None, acc int32 [B*S, nh*dh] | None) calls hero_int8_attention_probe instead."""
        assert q.stride(0) == k.stride(0) == v.stride(0) and q.dtype == k.dtype == v.dtype
        a = AttnArgs(q.data_ptr(), k.data_ptr(), v.data_ptr(), _DT[q.dtype], q.stride(0), B, S, nh, dh, s_q, s_k,
                     s_v, s_p, MASK[mask] if isinstance(mask, str) else mask, _ptr(key_len), out, _ptr(p_absmax),
                     P_MODE[p_mode] if isinstance(p_mode, str) else p_mode, _ptr(out_col_absmax))
        if probe is not None:
            scores, codes, acc = probe
            pr = AttnProbe(_ptr(scores), _ptr(codes), _ptr(acc))
            _check(lib().hero_int8_attention_probe(self._h, C.byref(a), C.byref(pr), _stream(stream)))
            return
        _check(lib().hero_int8_attention(self._h, C.byref(a), _stream(stream)))

    def hero_int8_decode_attention(self, q, k_cache, v_cache, lens, max_len, nh, dh, out, s_q=1.0, s_k=1.0, s_v=1.0,
                                   s_p=1.0 / 255, k_new=None, v_new=None, p_mode="static", stream=None):
        """q: int8 [B, nh*dh] view; k_cache, v_cache: int8 [B, S_max, nh*dh] views (feature stride 1, equal strides);
        lens: int32 [B] device tensor; k_new / v_new: optional int8 [B, nh*dh] views of equal pitch (appended at
        lens[b] - 1); out: hero.Tensor [B, nh*dh]."""
        assert q.dim() == 2 and k_cache.dim() == 3 and k_cache.stride() == v_cache.stride() and k_cache.stride(2) == 1
        assert q.dtype == k_cache.dtype == v_cache.dtype == torch.int8 and lens.dtype == torch.int32 and lens.is_cuda
        ld_new = 0
        if k_new is not None:
            assert k_new.stride(0) == v_new.stride(0) and k_new.dtype == torch.int8
            ld_new = k_new.stride(0) if k_new.shape[0] > 1 else max(k_new.stride(0), k_new.shape[1])
        ld_q = q.stride(0) if q.shape[0] > 1 else max(q.stride(0), q.shape[1])
        a = DecodeAttnArgs(q.data_ptr(), ld_q, k_cache.data_ptr(), v_cache.data_ptr(), k_cache.stride(1), k_cache.stride(0),
                           _ptr(k_new), _ptr(v_new), ld_new, lens.data_ptr(), int(max_len), q.shape[0], nh, dh, s_q, s_k, s_v,
                           s_p, P_MODE[p_mode] if isinstance(p_mode, str) else p_mode, out)
        _check(lib().hero_int8_decode_attention(self._h, C.byref(a), _stream(stream)))

    def hero_absmax_observe(self, x, col_absmax=None, tensor_absmax=None, stream=None):
        """x: hero.Tensor (F16 / BF16); col_absmax float32[cols] / tensor_absmax float32[1]: running maxima, updated."""
        _check(lib().hero_absmax_observe(self._h, C.byref(x), _ptr(col_absmax), _ptr(tensor_absmax), _stream(stream)))

    def hero_abs_histogram(self, x, bound, hist, stream=None):
        """x: hero.Tensor (F16 / BF16); hist: int64 / uint64 [2048] device tensor, accumulated."""
        assert hist.numel() == HIST_BINS and hist.element_size() == 8
        _check(lib().hero_abs_histogram(self._h, C.byref(x), float(bound), C.c_void_p(hist.data_ptr()), _stream(stream)))

    def hero_quantize_weight(self, W, Wq, w_scale, in_scale=None, out_scale=None, bias=None, bias_out=None, stream=None):
        """W: float32 [N, K]; Wq: int8 [N, K], or float8_e4m3fn [N, K] for the FP8 variant (hero_quantize_weight_f8);
        w_scale: float32 [N]; optional folds in_scale [K], out_scale [N]."""
        assert W.dim() == 2 and W.stride(1) == 1 and Wq.stride(1) == 1 and W.dtype == torch.float32
        assert Wq.dtype in (torch.int8, torch.float8_e4m3fn)
        fn = lib().hero_quantize_weight if Wq.dtype == torch.int8 else lib().hero_quantize_weight_f8
        _check(fn(self._h, C.c_void_p(W.data_ptr()), W.stride(0), W.shape[0], W.shape[1],
                                          _ptr(in_scale), _ptr(out_scale), _ptr(bias), C.c_void_p(Wq.data_ptr()),
                                          Wq.stride(0), _ptr(w_scale), _ptr(bias_out), _stream(stream)))

    # ---- serving over an 8-bit block cache (a decode step is a few microseconds of GPU time: these methods are kept lean)
    def _address(self, t, dtype, name):
        """Address of a contiguous vector (or table) of the given type on the handle's device; None -> absent."""
        if t is None:
            return None
        if t.dtype is not dtype or not t.is_contiguous() or t.get_device() != self._device:
            _refuse("%s: a contiguous tensor of %s on CUDA device %d is needed" % (name, dtype, self._device))
        return t.data_ptr()

    def _here(self, *descs):
        """Every hero.Tensor of a call lives on the handle's device."""
        for d in descs:
            if d is not None and getattr(d, "_device", None) != self._device:
                _refuse("a tensor is not on the handle's device %d" % self._device)

    def _raw_stream(self, stream):
        return _current_raw_stream(self._device) if stream is None else stream.cuda_stream

    def _rows(self, cache, row_start):
        if cache._device != self._device:
            _refuse("the cache is not on the handle's device %d" % self._device)
        if row_start is not None and row_start.numel() != cache.B + 1:
            _refuse("row_start has B + 1 = %d entries" % (cache.B + 1))
        return self._address(row_start, torch.int32, "row_start")

    def hero_block_cache_append(self, cache, k, v, row_start=None, max_rows=1, stream=None):
        """cache: hero.block_cache; k, v: hero.Tensor (F16 / BF16 [rows, nkv*dh]) of the new tokens; row_start: int32 [B + 1]
        (None: one row per sequence); max_rows: upper bound on a sequence's rows.  `lens` already counts the new tokens."""
        self._here(k, v)
        a = BlockRowsArgs(k, v, self._rows(cache, row_start), max_rows)
        _check(self._lib.hero_block_cache_append(self._h, C.byref(cache), C.byref(a), self._raw_stream(stream)))

    def hero_block_cache_read(self, cache, k, v, row_start=None, max_rows=1, stream=None):
        """k, v: hero.Tensor (F16 / BF16 [rows, nkv*dh]) to be written, either may be None: the values of the last tokens of each
        sequence, as many as it has rows."""
        self._here(k, v)
        a = BlockRowsArgs(k or _ABSENT, v or _ABSENT, self._rows(cache, row_start), max_rows)
        _check(self._lib.hero_block_cache_read(self._h, C.byref(cache), C.byref(a), self._raw_stream(stream)))

    def hero_block_attention_workspace_bytes(self, cache, nq, rows, max_rows=1):
        """Bytes that serve every call on this cache with these heads and at most max_rows rows a sequence."""
        n = C.c_size_t()
        _check(self._lib.hero_block_attention_workspace_bytes(self._h, C.byref(cache), nq, rows, max_rows, C.byref(n)))
        return int(n.value)

    def hero_block_attention(self, cache, q, out, nq, row_start=None, max_rows=1, scale=0.0, workspace=None, stream=None):
        """q: hero.Tensor (F16 / BF16 [rows, nq*dh]); out: hero.Tensor of the same shape (F16 / BF16, or I8 / F8 with a
        feature-wise or static scale); workspace: 1-D uint8 CUDA tensor of hero_block_attention_workspace_bytes (may be empty or
        None when that is 0); scale 0: 1 / sqrt(dh)."""
        self._here(q, out)
        ws, n = None, 0
        if workspace is not None and workspace.numel():
            ws, n = self._address(workspace, torch.uint8, "workspace"), workspace.numel()
        a = BlockAttnArgs(q, out, self._rows(cache, row_start), max_rows, nq, scale, ws, n)
        _check(self._lib.hero_block_attention(self._h, C.byref(cache), C.byref(a), self._raw_stream(stream)))

    def hero_qk_norm_rope(self, q, k, q_out, k_out, nq, nkv, pos=None, cos=None, sin=None, q_gamma=None, k_gamma=None, eps=1e-6,
                          pairing="halves", stream=None):
        """q, k, q_out, k_out: hero.Tensor ([rows, nq*dh] / [rows, nkv*dh]; k and k_out None with nkv = 0; an output may be its
        input); pos: int32 [rows]; cos, sin: float32 [n_pos, rot / 2] (None: no rotation); gammas: float32 [dh] (None: no norm)."""
        self._here(q, k, q_out, k_out)
        dh, rot, n_pos = q.cols // max(nq, 1), 0, 0
        if cos is not None:
            n_pos, half = cos.shape if cos.dim() == 2 else _refuse("cos, sin: [n_pos, rot / 2]")
            rot = 2 * half
            if sin is None or sin.numel() != n_pos * half or pos is None or pos.numel() < q.rows:
                _refuse("cos, sin: [n_pos, rot / 2], pos: [rows]")
        if (q_gamma is not None and q_gamma.numel() != dh) or (k_gamma is not None and k_gamma.numel() != dh):
            _refuse("a gamma has dh = %d entries" % dh)
        f32, at = torch.float32, self._address
        a = QkNormRopeArgs(q, k or _ABSENT, q_out, k_out or _ABSENT, nq, nkv, dh, rot, PAIRING[pairing] if isinstance(pairing, str) else pairing,
                           eps, at(q_gamma, f32, "q_gamma"), at(k_gamma, f32, "k_gamma"), at(pos, torch.int32, "pos"), at(cos, f32, "cos"),
                           at(sin, f32, "sin"), n_pos)
        _check(self._lib.hero_qk_norm_rope(self._h, C.byref(a), self._raw_stream(stream)))

    # ---- a mixture of experts (lean for the same reason)
    def _pairs(self, t, dtype, shape, name):
        """Address of a contiguous table of the given type and shape on the handle's device; None -> absent."""
        if t is None:
            return None
        if t.shape != shape or t.dtype is not dtype or not t.is_contiguous() or t.get_device() != self._device:
            _refuse("%s: a contiguous tensor of %s, shape %s, on CUDA device %d is needed, got %s of %s" % (name, dtype, shape, self._device, tuple(t.shape), t.dtype))
        return t.data_ptr()

    def hero_moe_route_workspace_bytes(self, tokens, n_experts, top_k):
        """Bytes that serve every call with these experts and at most this many tokens."""
        n = C.c_size_t()
        _check(self._lib.hero_moe_route_workspace_bytes(self._h, tokens, n_experts, top_k, C.byref(n)))
        return int(n.value)

    def hero_moe_route(self, logits, expert, weight, offset, token, row, score="softmax", renorm=True, scale=1.0, select_bias=None,
                       n_tokens=None, workspace=None, stream=None):
        """logits: hero.Tensor (F32 / F16 / BF16 [tokens, experts]); written: expert, row int32 [tokens, k], weight float32 [tokens, k],
        offset int32 [experts + 1], token int32 [tokens * k]; select_bias: float32 [experts]; n_tokens: int32 [1] device tensor (a padded
        batch); workspace: 1-D uint8 tensor of hero_moe_route_workspace_bytes (may be empty or None when that is 0)."""
        self._here(logits)
        T, E, at, i32 = logits.rows, logits.cols, self._pairs, torch.int32
        if expert.dim() != 2 or expert.shape[0] != T:
            _refuse("expert: [tokens, k]")
        k, ws, n = expert.shape[1], None, 0
        if workspace is not None and workspace.numel():
            ws, n = self._address(workspace, torch.uint8, "workspace"), workspace.numel()
        a = MoeRouteArgs(logits, at(n_tokens, i32, (1,), "n_tokens"), at(select_bias, torch.float32, (E,), "select_bias"), k,
                         SCORE[score] if isinstance(score, str) else score, int(renorm), scale, at(expert, i32, (T, k), "expert"),
                         at(weight, torch.float32, (T, k), "weight"), at(offset, i32, (E + 1,), "offset"), at(token, i32, (T * k,), "token"),
                         at(row, i32, (T, k), "row"), ws, n)
        _check(self._lib.hero_moe_route(self._h, C.byref(a), self._raw_stream(stream)))

    def hero_moe_linear(self, A, W, out, offset, token=None, w_scale=None, bias=None, act="none", gated=False, post_scale=None,
                        out_col_absmax=None, stream=None):
        """A, out: hero.Tensor; W: [experts, N, K] of A's type (K contiguous); offset: int32 [experts + 1]; token: int32 [rows of out] (None: A is in
        sorted order); w_scale, bias: float32 [experts, N]; post_scale, out_col_absmax: float32 [experts, columns of out]."""
        self._here(A, out)
        _scaled_rows(A, "A")
        if W.dim() != 3 or W.stride(2) != 1 or W.shape[2] != A.cols or W.get_device() != self._device or _DT.get(W.dtype) != A.dtype:
            _refuse("W: [experts, N, K = %d] of A's type on the handle's device, K contiguous" % A.cols)
        E, N, K = W.shape
        at, f32 = self._pairs, torch.float32
        a = MoeLinearArgs(A, at(token, torch.int32, (out.rows,), "token"), at(offset, torch.int32, (E + 1,), "offset"), W.data_ptr(), N,
                          W.stride(1) if N > 1 else max(W.stride(1), K), W.stride(0), E, at(w_scale, f32, (E, N), "w_scale"), at(bias, f32, (E, N), "bias"),
                          ACT[act] if isinstance(act, str) else act, int(gated), at(post_scale, f32, (E, out.cols), "post_scale"), out,
                          at(out_col_absmax, f32, (E, out.cols), "out_col_absmax"))
        _check(self._lib.hero_moe_linear(self._h, C.byref(a), self._raw_stream(stream)))

    def hero_moe_combine(self, y, row, weight, expert=None, residual=None, shared=None, out=None, fp_out=None, gamma=None, beta=None, eps=1e-5,
                         stream=None):
        """y: hero.Tensor of the sorted rows (F16 / BF16, or I8 / F8 with a static scale or, "fwq", one of [experts, H]); row, expert: int32 [tokens, k],
        weight: float32 [tokens, k], as hero_moe_route leaves them; residual, shared, out, fp_out: hero.Tensor [tokens, H] or None;
        gamma, beta: float32 [H], with out."""
        self._here(y, *(t for t in (residual, shared, out, fp_out) if t is not None))
        like, at, i32, f32 = out or fp_out, self._pairs, torch.int32, torch.float32
        if like is None or row.dim() != 2 or row.shape[0] != like.rows:
            _refuse("out or fp_out is needed, row: [tokens, k]")
        E, shape = 0, tuple(row.shape)
        if y.gran == GRAN_FWQ:
            scale = y._keep[1]
            if scale is None or scale.dim() != 2 or scale.shape[1] != y.cols:
                _refuse("y: the feature-wise scale is [experts, H]")
            E = scale.shape[0]
        for t, n in ((residual, like.rows), (shared, like.rows), (out, like.rows)):
            if t is not None and t.gran in (GRAN_TWQ, GRAN_FWQ) and t._keep[1] is not None and t._keep[1].numel() != (n if t.gran == GRAN_TWQ else t.cols):
                _refuse("a token-wise scale has one entry per token, a feature-wise one per feature")
        a = MoeCombineArgs(y, at(row, i32, shape, "row"), at(weight, f32, shape, "weight"), at(expert, i32, shape, "expert"), shape[1], E,
                           residual or _ABSENT, shared or _ABSENT, at(gamma, f32, (like.cols,), "gamma"), at(beta, f32, (like.cols,), "beta"), eps,
                           out or _ABSENT, fp_out or _ABSENT)
        _check(self._lib.hero_moe_combine(self._h, C.byref(a), self._raw_stream(stream)))

    def hero_layer_workspace_bytes(self, desc, M):
        n = C.c_size_t()
        _check(lib().hero_layer_workspace_bytes(C.byref(desc), int(M), C.byref(n)))
        return int(n.value)

    def hero_layer_workspace_layout(self, desc, M):
        lay = LayerLayout()
        _check(lib().hero_layer_workspace_layout(C.byref(desc), int(M), C.byref(lay)))
        return lay

    def hero_layer_forward_host_async(self, desc, in_host, out_host, in_dev, out_dev, workspace, stream=None):
        """Host-buffer variant without the final synchronisation (out_host is valid after the stream is synchronised)."""
        _check(lib().hero_layer_forward_host_async(self._h, C.byref(desc), C.byref(in_host), C.byref(out_host),
                                                   C.byref(in_dev), C.byref(out_dev), C.c_void_p(workspace.data_ptr()),
                                                   workspace.numel(), _stream(stream)))

    def hero_layer_forward_host(self, desc, in_host, out_host, in_dev, out_dev, workspace, stream=None):
        """Host-buffer variant: copies in, runs the layer, copies out, synchronizes."""
        _check(lib().hero_layer_forward_host(self._h, C.byref(desc), C.byref(in_host), C.byref(out_host),
                                             C.byref(in_dev), C.byref(out_dev), C.c_void_p(workspace.data_ptr()),
                                             workspace.numel(), _stream(stream)))

    def hero_stack_forward(self, stack_desc, workspace, stream=None):
        """stack_desc: hero.StackDesc (see `stack_desc`); one C call runs the entry LN^quant (if any) and every layer."""
        _check(lib().hero_stack_forward(self._h, C.byref(stack_desc), C.c_void_p(workspace.data_ptr()), workspace.numel(),
                                        _stream(stream)))

    def hero_stack_forward_host_async(self, stack_desc, in_host, out_host, workspace, stream=None):
        """Host-buffer variant: H2D of in_host, the stack, D2H into out_host, all enqueued on the stream."""
        _check(lib().hero_stack_forward_host_async(self._h, C.byref(stack_desc), C.byref(in_host), C.byref(out_host),
                                                   C.c_void_p(workspace.data_ptr()), workspace.numel(), _stream(stream)))

    def profile_begin(self, max_launches):
        self._prof_cap = int(max_launches)
        _check(lib().hero_profile_begin(self._h, self._prof_cap))

    def profile_end(self):
        """[(kernel family, milliseconds), ...] for every launch since profile_begin, in order."""
        ms = (C.c_float * self._prof_cap)()
        tag = (C.c_int32 * self._prof_cap)()
        n = C.c_int32()
        _check(lib().hero_profile_end(self._h, ms, tag, C.byref(n)))
        return [(int(tag[i]), float(ms[i])) for i in range(n.value)]

    def hero_layer_forward(self, desc, x_in, out, workspace, pending=None, stream=None):
        """x_in / out / pending: hero.Tensor; workspace: 1-D torch uint8 CUDA tensor."""
        pend = C.byref(pending) if pending is not None else None
        _check(lib().hero_layer_forward(self._h, C.byref(desc), C.byref(x_in), pend, C.byref(out),
                                        C.c_void_p(workspace.data_ptr()), workspace.numel(), _stream(stream)))

    def hero_layer_decode(self, desc, k_cache, v_cache, lens, max_len, x_in, out, workspace, pending=None, stream=None):
        """One decode step: k_cache / v_cache int8 [B, S_max, H] views of equal strides (the new key / value are stored at
        lens[b] - 1), lens int32 [B]; x_in / out / pending: hero.Tensor with B rows."""
        assert k_cache.dim() == 3 and k_cache.stride() == v_cache.stride() and k_cache.stride(2) == 1
        assert k_cache.dtype == v_cache.dtype == torch.int8 and lens.dtype == torch.int32 and lens.is_cuda
        kv = KvCache(k_cache.data_ptr(), v_cache.data_ptr(), k_cache.stride(1), k_cache.stride(0), lens.data_ptr(), int(max_len))
        pend = C.byref(pending) if pending is not None else None
        _check(lib().hero_layer_decode(self._h, C.byref(desc), C.byref(kv), C.byref(x_in), pend, C.byref(out),
                                       C.c_void_p(workspace.data_ptr()), workspace.numel(), _stream(stream)))


def stack_desc(layer_descs, edges, entry_in=None, entry_gamma=None, entry_beta=None, entry_eps=0.0):
    """hero_stack_desc over a list of LayerDesc and a list of len(layer_descs) + 1 hero.Tensor edges (device tensors)."""
    n = len(layer_descs)
    assert len(edges) == n + 1
    sd = StackDesc()
    layers = (LayerDesc * n)(*layer_descs)
    e = (Tensor * (n + 1))(*edges)
    sd.n_layers, sd.layers, sd.edges, sd.pending = n, layers, e, None
    sd.entry_in = entry_in if entry_in is not None else tensor(None)
    sd.entry_gamma, sd.entry_beta, sd.entry_eps = _ptr(entry_gamma), _ptr(entry_beta), float(entry_eps)
    sd._keep = (layers, e, list(layer_descs), list(edges), entry_in, entry_gamma, entry_beta)
    return sd


def host_tensor(t, gran="none", scale=None):
    """hero_tensor view of a 2-D (pinned) host torch tensor, for hero_layer_forward_host."""
    assert not t.is_cuda and t.dim() == 2 and t.stride(1) == 1
    g = GRAN[gran] if isinstance(gran, str) else gran
    T = Tensor(t.data_ptr(), _DT[t.dtype], g, t.shape[0], t.shape[1], t.stride(0), None if scale is None else scale.data_ptr())
    T._keep = (t, scale)
    return T


def hero_layer_forward_static(desc, x_in, out, pending=None, stream=None):
    """The layer forward without handle or workspace, for callers that may not allocate device memory: the
    scratch is a fixed 64 MiB array inside libhero.so (larger layers are refused).  Calls share that array, so
    do not let two of them overlap on the GPU."""
    pend = C.byref(pending) if pending is not None else None
    _check(lib().hero_layer_forward_static(C.byref(desc), C.byref(x_in), pend, C.byref(out), _stream(stream)))


def hero_static_check(stream=None):
    """Synchronizes the stream and raises if a kernel of hero_layer_forward_static left a code in its error word."""
    _check(lib().hero_static_check(_stream(stream)))


def mode_preset(preset):
    m = (C.c_int32 * 5)()
    _check(lib().hero_mode_preset(int(preset), C.byref(m)))
    return list(m)
