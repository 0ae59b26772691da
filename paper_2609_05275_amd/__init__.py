"""Python binding of liblayerdrop (MI355X / gfx950 layer-dropout hot path).

Argument marshalling only: every function here has the name of a C entry
point in include/layerdrop.h, converts torch tensors to device pointers and
the current torch stream to a hipStream_t, calls the library, and raises
LdError on a non-zero status.  All computation happens in the HIP kernels;
there is no fallback -- importing fails loudly when the library is not built.
"""

import ctypes as C
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "liblayerdrop.so")

LD_F32, LD_BF16 = 0, 1
LD_KV8_E4M3, LD_KV8_INT8 = 0, 1
LD_W4_E2M1, LD_W4_INT4 = 0, 1
LD_GRAN_LAYER_SEQ, LD_GRAN_SUBLAYER_SEQ, LD_GRAN_LAYER_BATCH, LD_GRAN_SUBLAYER_BATCH = 0, 1, 2, 3
UNIFORM, ILD, ALD = 0, 1, 2
CONSTANT, ITS, DTS = 0, 1, 2

WEIGHT_KEYS = ("g_attn", "w_qkv", "w_o", "g_mlp", "w_gate_up", "w_down")


class LdError(RuntimeError):
    def __init__(self, status, msg):
        super().__init__(f"{status_name(status)}: {msg}")
        self.status = status


class ld_config(C.Structure):
    _fields_ = [("batch", C.c_int32), ("seq", C.c_int32), ("d_model", C.c_int32),
                ("n_heads", C.c_int32), ("d_ff", C.c_int32), ("dtype", C.c_int32),
                ("rms_eps", C.c_float), ("rescale", C.c_int32), ("res_scale", C.c_float),
                ("block_kind", C.c_int32), ("granularity", C.c_int32)]


class ld_kv8(C.Structure):
    _fields_ = [(k, C.c_int32) for k in ("format", "block", "n_seq", "n_kv_heads", "d_head", "s_max")] + \
               [("codes", C.c_void_p), ("scales", C.c_void_p)]
    device = None     # the tensors' GPU, where kv8() was given tensors
    tensors = ()


class ld_w4(C.Structure):
    _fields_ = [(k, C.c_int32) for k in ("format", "group", "n", "k")] + [("codes", C.c_void_p), ("scales", C.c_void_p)]
    device = None     # the tensors' GPU, where w4() was given tensors
    tensors = ()


class ld_kv4(C.Structure):
    _fields_ = [(k, C.c_int32) for k in ("n_seq", "n_kv_heads", "d_head", "s_max")] + \
               [("codes", C.c_void_p), ("scales", C.c_void_p), ("sums", C.c_void_p)]
    device = None     # the tensors' GPU, where kv4() was given tensors
    tensors = ()


class ld_weights_w4(C.Structure):
    _fields_ = [("g_attn", C.c_void_p), ("g_mlp", C.c_void_p)] + \
               [(k, ld_w4) for k in ("w_qkv", "w_o", "w_gate_up", "w_down")]


class ld_weights(C.Structure):
    _fields_ = [(k, C.c_void_p) for k in WEIGHT_KEYS]


class ld_grads(C.Structure):
    _fields_ = [(k, C.c_void_p) for k in WEIGHT_KEYS]


if not os.path.exists(LIB_PATH):
    raise ImportError(f"{LIB_PATH} is not built; run `python paper_2609_05275_amd/build.py`")
_lib = C.CDLL(LIB_PATH)

_vp, _i32, _i64, _u64, _f32, _sz = C.c_void_p, C.c_int32, C.c_int64, C.c_uint64, C.c_float, C.c_size_t
_PCFG = C.POINTER(ld_config)
_PKV8 = C.POINTER(ld_kv8)
_PKV4 = C.POINTER(ld_kv4)
_PW4 = C.POINTER(ld_w4)
_SIGS = {
    "ld_status_string": (C.c_char_p, [C.c_int]),
    "ld_last_error": (C.c_char_p, []),
    "ld_schedule_p": (C.c_int, [_i32, _i32, _f32, _i32, _i32, _i64, _i64, C.POINTER(_f32)]),
    "ld_masks": (C.c_int, [_i32, _i32, C.POINTER(_f32), _i32, _u64, _u64, _vp, _vp, _vp, _vp]),
    "ld_masks_granular": (C.c_int, [_i32, _i32, _i32, C.POINTER(_f32), _i32, _u64, _u64, _vp, _vp,
                                    _vp, _vp]),
    "ld_gather_rows": (C.c_int, [_PCFG, _vp, _vp, _vp, _vp, _vp]),
    "ld_scatter_add_rows": (C.c_int, [_PCFG, _vp, _vp, _f32, _vp, _vp, _vp]),
    "ld_layer_ctx_bytes": (_sz, [_PCFG]),
    "ld_layer_ws_bytes": (_sz, [_PCFG]),
    "ld_stack_ws_bytes": (_sz, [_PCFG, _i32]),
    "ld_layer_fwd": (C.c_int, [_PCFG, C.POINTER(ld_weights), _i32, _f32, _u64, _u64, _vp, _vp,
                               _vp, _sz, _vp, _vp]),
    "ld_layer_bwd": (C.c_int, [_PCFG, C.POINTER(ld_weights), _vp, _vp, C.POINTER(ld_grads), _vp,
                               _sz, _vp]),
    "ld_stack_step": (C.c_int, [_PCFG, _i32, C.POINTER(ld_weights), C.POINTER(_f32), _u64, _u64,
                                _vp, _vp, C.POINTER(ld_grads), _vp, _sz, _vp, _vp, _vp, _vp, _vp]),
    "ld_rmsnorm_fwd": (C.c_int, [_i32, _i32, _i32, _f32, _vp, _vp, _vp, _vp, _vp]),
    "ld_rmsnorm_bwd_ws_bytes": (_sz, [_i32, _i32]),
    "ld_rmsnorm_bwd": (C.c_int, [_i32, _i32, _i32, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _sz,
                                 _vp]),
    "ld_relu2_fwd": (C.c_int, [_i32, _i32, _i32, _vp, _vp, _vp]),
    "ld_relu2_bwd": (C.c_int, [_i32, _i32, _i32, _vp, _vp, _vp, _vp]),
    "ld_alibi_slope": (C.c_float, [_i32, _i32]),
    "ld_swiglu_fwd": (C.c_int, [_i32, _i32, _i32, _vp, _vp, _vp]),
    "ld_swiglu_bwd": (C.c_int, [_i32, _i32, _i32, _vp, _vp, _vp, _vp]),
    "ld_gemm_ws_bytes": (_sz, [_i32, _i32, _i32, _i32, _i32, _i32, _i32, _i32]),
    "ld_gemm": (C.c_int, [_i32, _i32, _i32, _i32, _i32, _i32, _vp, _i32, _vp, _i32, _vp, _i32,
                          _i32, _f32, _vp, _i32, _vp, _sz, _vp]),
    "ld_attn_fwd": (C.c_int, [_i32, _i32, _i32, _i32, _i32, _i32, _vp, _vp, _vp, _vp]),
    "ld_attn_bwd_ws_bytes": (_sz, [_i32, _i32, _i32]),
    "ld_attn_bwd": (C.c_int, [_i32, _i32, _i32, _i32, _i32, _i32, _vp, _vp, _vp, _vp, _vp, _vp,
                              _sz, _vp]),
    "ld_attn_bwd_noalloc": (C.c_int, [_i32, _i32, _i32, _i32, _i32, _i32, _vp, _vp, _vp, _vp, _vp,
                                      _vp]),
    "ld_eval_ws_bytes": (_sz, [_PCFG]),
    "ld_stack_eval": (C.c_int, [_PCFG, _i32, C.POINTER(ld_weights), _vp, _vp, _vp, _vp, _i32, _vp,
                                _sz, _vp]),
    "ld_decode_ws_bytes": (_sz, [_PCFG, _i32, _i32]),
    "ld_stack_decode": (C.c_int, [_PCFG, _i32, C.POINTER(ld_weights), _vp, _vp, _vp, _vp, _i32,
                                  _i32, _i32, _vp, _sz, _vp]),
    "ld_gemm_skinny_ws_bytes": (_sz, [_i32, _i32, _i32]),
    "ld_gemm_skinny": (C.c_int, [_i32, _i32, _i32, _vp, _i32, _vp, _i32, _vp, _i32, _f32, _vp, _i32,
                                 _vp, _sz, _vp]),
    "ld_gemm_dec": (C.c_int, [_i32, _i32, _i32, _vp, _i32, _vp, _f32, _vp, _i32, _vp, _i32, _f32, _vp, _i32,
                              _i32, _vp]),
    "ld_kv_store": (C.c_int, [_i32, _i32, _i32, _i32, _vp, _vp, _i32, _vp]),
    "ld_attn_decode_ws_bytes": (_sz, [_i32, _i32, _i32, _i32]),
    "ld_attn_decode": (C.c_int, [_i32, _i32, _i32, _i32, _i32, _i32, _vp, _vp, _i32, _vp, _vp, _sz,
                                 _vp]),
    "ld_stack_eval_kv8": (C.c_int, [_PCFG, _i32, C.POINTER(ld_weights), _vp, _vp, _vp, _PKV8, _vp, _sz, _vp]),
    "ld_decode_kv8_ws_bytes": (_sz, [_PCFG, _i32, _i32]),
    "ld_stack_decode_kv8": (C.c_int, [_PCFG, _i32, C.POINTER(ld_weights), _vp, _vp, _vp, _PKV8, _i32, _vp, _i32,
                                      _vp, _sz, _vp]),
    "ld_kv8_code_bytes": (_sz, [_PKV8]),
    "ld_kv8_scale_bytes": (_sz, [_PKV8]),
    "ld_kv8_store": (C.c_int, [_PKV8, _i32, _i32, _i32, _vp, _vp, _vp]),
    "ld_kv8_load": (C.c_int, [_PKV8, _i32, _i32, _vp, _vp, _vp]),
    "ld_attn_decode_kv8_ws_bytes": (_sz, [_PKV8, _i32, _i32]),
    "ld_attn_decode_kv8": (C.c_int, [_PKV8, _i32, _i32, _i32, _vp, _i32, _vp, _vp, _vp, _sz, _vp]),
    "ld_stack_eval_kv4": (C.c_int, [_PCFG, _i32, C.POINTER(ld_weights), _vp, _vp, _vp, _PKV4, _vp, _sz, _vp]),
    "ld_decode_kv4_ws_bytes": (_sz, [_PCFG, _i32, _i32, _i32]),
    "ld_stack_decode_kv4": (C.c_int, [_PCFG, _i32, C.POINTER(ld_weights), _vp, _vp, _vp, _PKV4, _i32, _vp, _i32,
                                      _vp, _sz, _vp]),
    "ld_stack_decode_w4": (C.c_int, [_PCFG, _i32, C.POINTER(ld_weights_w4), _vp, _vp, _vp, _PKV4, _i32, _vp, _i32,
                                     _vp, _sz, _vp]),
    "ld_w4_code_bytes": (_sz, [_PW4]),
    "ld_w4_scale_bytes": (_sz, [_PW4]),
    "ld_w4_pack": (C.c_int, [_PW4, _vp, _i32, _vp]),
    "ld_w4_load": (C.c_int, [_PW4, _vp, _i32, _vp]),
    "ld_gemm_w4_ws_bytes": (_sz, [_PW4, _i32, _i32]),
    "ld_gemm_w4": (C.c_int, [_i32, _vp, _i32, _vp, _f32, _PW4, _vp, _i32, _f32, _vp, _i32, _i32, _vp, _sz, _vp]),
    "ld_kv4_code_bytes": (_sz, [_PKV4]),
    "ld_kv4_scale_bytes": (_sz, [_PKV4]),
    "ld_kv4_store": (C.c_int, [_PKV4, _i32, _i32, _i32, _vp, _vp, _vp]),
    "ld_kv4_load": (C.c_int, [_PKV4, _i32, _i32, _vp, _vp, _vp]),
    "ld_attn_decode_kv4_ws_bytes": (_sz, [_PKV4, _i32, _i32]),
    "ld_attn_decode_kv4": (C.c_int, [_PKV4, _i32, _i32, _i32, _vp, _i32, _vp, _vp, _vp, _sz, _vp]),
    "ld_kv4_evict_ws_bytes": (_sz, [_PKV4, _i32, _i32]),
    "ld_kv4_evict": (C.c_int, [_PKV4, _PKV4, _i32, _vp, _i32, _i32, _vp, _vp, _sz, _vp]),
    "ld_prof_start": (C.c_int, [C.c_char_p]),
    "ld_prof_stop": (C.c_int, []),
    "ld_prof_result": (C.c_int, [C.POINTER(_i64), C.POINTER(C.c_double), C.POINTER(C.c_double),
                                 C.POINTER(C.c_double)]),
}
for _name, (_res, _args) in _SIGS.items():
    _fn = getattr(_lib, _name)
    _fn.restype = _res
    _fn.argtypes = _args

EXPORTED = tuple(_SIGS)


def status_name(status):
    return _lib.ld_status_string(status).decode()


def last_error():
    return _lib.ld_last_error().decode()


def _check(status):
    if status != 0:
        raise LdError(status, last_error())


def _ptr(t, name="tensor", inner=False):
    """Device address of t.  A torch tensor must live on the GPU and be
    contiguous (with inner=True, for calls that take a leading dimension,
    only its last dimension must be); anything else -- a raw address (int) or
    an object with data_ptr() -- is passed through for the library to check."""
    if t is None:
        return None
    if isinstance(t, int):
        return t
    if isinstance(t, torch.Tensor):
        if not t.is_cuda:
            raise ValueError(f"{name}: a device tensor is required, got one on {t.device}")
        if inner:
            if t.dim() and t.stride(-1) != 1 and t.numel() > 1:
                raise ValueError(f"{name}: the last dimension must be contiguous")
        elif not t.is_contiguous():
            raise ValueError(f"{name}: a contiguous tensor is required")
    return t.data_ptr()


_TORCH_OF = {LD_F32: torch.float32, LD_BF16: torch.bfloat16}


def _need(t, name, dtype=None, numel=None, min_bytes=None):
    """Checks a torch tensor argument against what the call reads or writes
    (dtype, element count, byte size) before anything is launched; other
    objects pass through to the library's own checks."""
    if not isinstance(t, torch.Tensor):
        return
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name}: dtype {t.dtype}, expected {dtype}")
    if numel is not None and t.numel() != numel:
        raise ValueError(f"{name}: {t.numel()} elements, expected {numel}")
    if min_bytes is not None and t.numel() * t.element_size() < min_bytes:
        raise ValueError(f"{name}: {t.numel() * t.element_size()} bytes, at least {min_bytes} needed")


def _n_masks(cfg):
    return 2 if cfg.granularity & LD_GRAN_SUBLAYER_SEQ else 1


def _weight_numel(cfg):
    d, f = cfg.d_model, cfg.d_ff
    return dict(g_attn=d, w_qkv=3 * d * d, w_o=d * d, g_mlp=d,
                w_gate_up=(2 if cfg.block_kind == 0 else 1) * f * d, w_down=d * f)


def _check_layer_tensors(cfg, w=None, dw=None, acts=()):
    dt = _TORCH_OF.get(cfg.dtype)
    n = _weight_numel(cfg)
    for k in WEIGHT_KEYS:
        if w is not None:
            _need(w[k], k, dt, n[k])
        if dw is not None:
            _need(dw[k], "grad " + k, torch.float32, n[k])
    for name, t in acts:
        _need(t, name, dt, cfg.batch * cfg.seq * cfg.d_model)


# torch.cuda.current_stream() builds a Stream object, 2.8 us of a call's 9; its
# handle alone takes 0.1
_current_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream, device=None):
    """The hipStream_t of a stream argument: None is the current one (of the
    current device, whose index the caller may give)."""
    if stream is None:
        if device is not None and _current_raw_stream is not None:
            return _current_raw_stream(device)
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _dtype_code(t):
    if t.dtype == torch.bfloat16:
        return LD_BF16
    if t.dtype == torch.float32:
        return LD_F32
    raise TypeError(f"unsupported dtype {t.dtype}")


def config(batch, seq, d_model, n_heads, d_ff, dtype=LD_BF16, rms_eps=1e-5, rescale=True,
           res_scale=1.0, block_kind=0, granularity=0):
    return ld_config(batch, seq, d_model, n_heads, d_ff, dtype, rms_eps, int(bool(rescale)),
                     res_scale, block_kind, granularity)


def weights(w):
    """ld_weights from a dict of device tensors keyed by WEIGHT_KEYS."""
    return ld_weights(*[_ptr(w[k], k) for k in WEIGHT_KEYS])


def _stack_weights(cfg, ws_list, active, other=None, device=None):
    """The layers' weights for a call that reads those of the active ones (_u8_array), whose
    tensors are checked as _check_layer_tensors does, or by other(tensor, name, dtype,
    numel) where they are not as expected and on `device`."""
    dt, n = _TORCH_OF.get(cfg.dtype), _weight_numel(cfg)
    sizes = [(k, n[k]) for k in WEIGHT_KEYS]
    out = (ld_weights * len(ws_list))()
    for l, w in enumerate(ws_list):
        if active is not None and not active[l]:
            out[l] = weights(w)
            continue
        p = []
        for k, m in sizes:
            t = w[k]
            if type(t) is torch.Tensor and t.dtype is dt and t.numel() == m and t.is_contiguous() and \
                    (t.is_cuda if other is None else t.get_device() == device):
                p.append(t.data_ptr())     # the usual case, 0.3 us a layer sooner
            elif other is not None:
                p.append(other(t, k, dt, m))
            else:
                _need(t, k, dt, m)
                p.append(_ptr(t, k))
        out[l] = ld_weights(*p)
    return out


def grads(g):
    return ld_grads(*[_ptr(g[k], "grad " + k) for k in WEIGHT_KEYS])


# ------------------------------------------------------------------ entry points

def ld_schedule_p(dist, sched, p_max, layer, n_layers, t, n_steps):
    out = C.c_float()
    _check(_lib.ld_schedule_p(dist, sched, p_max, layer, n_layers, t, n_steps, C.byref(out)))
    return out.value


def ld_masks(p, seed, step, keep, idx, count, first_layer=0, stream=None):
    n = len(p)
    arr = (C.c_float * n)(*[float(v) for v in p])
    B = keep.shape[-1]
    _need(keep, "keep", torch.uint8, n * B)
    _need(idx, "idx", torch.int32, n * B)
    _need(count, "count", torch.int32, n)
    _check(_lib.ld_masks(n, B, arr, first_layer, seed, step, _ptr(keep, "keep"), _ptr(idx, "idx"),
                         _ptr(count, "count"), _stream(stream)))


def ld_masks_granular(granularity, p, seed, step, keep, idx, count, first_layer=0, stream=None):
    n = len(p)
    arr = (C.c_float * n)(*[float(v) for v in p])
    B = keep.shape[-1]
    nm = 2 if granularity in (LD_GRAN_SUBLAYER_SEQ, LD_GRAN_SUBLAYER_BATCH) else 1
    _need(keep, "keep", torch.uint8, n * nm * B)
    _need(idx, "idx", torch.int32, n * nm * B)
    _need(count, "count", torch.int32, n * nm)
    _check(_lib.ld_masks_granular(granularity, n, B, arr, first_layer, seed, step,
                                  _ptr(keep, "keep"), _ptr(idx, "idx"), _ptr(count, "count"),
                                  _stream(stream)))


def ld_gather_rows(cfg, idx, count, x, xk, stream=None):
    _need(idx, "idx", torch.int32, cfg.batch)
    _need(count, "count", torch.int32, 1)
    _check_layer_tensors(cfg, acts=(("x", x), ("xk", xk)))
    _check(_lib.ld_gather_rows(C.byref(cfg), _ptr(idx, "idx"), _ptr(count, "count"), _ptr(x, "x"),
                               _ptr(xk, "xk"), _stream(stream)))


def ld_scatter_add_rows(cfg, idx, count, r, yk, x, stream=None):
    _need(idx, "idx", torch.int32, cfg.batch)
    _need(count, "count", torch.int32, 1)
    _check_layer_tensors(cfg, acts=(("yk", yk), ("x", x)))
    _check(_lib.ld_scatter_add_rows(C.byref(cfg), _ptr(idx, "idx"), _ptr(count, "count"), r,
                                    _ptr(yk, "yk"), _ptr(x, "x"), _stream(stream)))


def ld_layer_ctx_bytes(cfg):
    return _lib.ld_layer_ctx_bytes(C.byref(cfg))


def ld_layer_ws_bytes(cfg):
    return _lib.ld_layer_ws_bytes(C.byref(cfg))


def ld_stack_ws_bytes(cfg, n_layers):
    return _lib.ld_stack_ws_bytes(C.byref(cfg), n_layers)


def ld_layer_fwd(cfg, w, layer, p, seed, step, x, ctx, ws=None, keep_override=None, stream=None):
    _check_layer_tensors(cfg, w=w, acts=(("x", x),))
    _need(ctx, "ctx", min_bytes=ld_layer_ctx_bytes(cfg))
    _need(keep_override, "keep_override", torch.uint8, _n_masks(cfg) * cfg.batch)
    wb = weights(w)
    ws_bytes = 0 if ws is None else ws.numel() * ws.element_size()
    _check(_lib.ld_layer_fwd(C.byref(cfg), C.byref(wb), layer, p, seed, step, _ptr(x), _ptr(ctx),
                             _ptr(ws), ws_bytes, _ptr(keep_override), _stream(stream)))


def ld_layer_bwd(cfg, w, ctx, dx, dw, ws, stream=None):
    _check_layer_tensors(cfg, w=w, dw=dw, acts=(("dx", dx),))
    _need(ctx, "ctx", min_bytes=ld_layer_ctx_bytes(cfg))
    wb, gb = weights(w), grads(dw)
    _check(_lib.ld_layer_bwd(C.byref(cfg), C.byref(wb), _ptr(ctx), _ptr(dx), C.byref(gb),
                             _ptr(ws), ws.numel() * ws.element_size(), _stream(stream)))


def ld_stack_step(cfg, ws_list, p, seed, step, x, dx, dw_list, ws, keep_override=None,
                  keep_out=None, idx_out=None, count_out=None, stream=None):
    L = len(ws_list)
    if len(dw_list) != L or len(p) != L:
        raise ValueError(f"{L} layers of weights, {len(dw_list)} of gradients, {len(p)} rates")
    for l in range(L):
        _check_layer_tensors(cfg, w=ws_list[l], dw=dw_list[l])
    _check_layer_tensors(cfg, acts=(("x", x), ("dx", dx)))
    nmb = L * _n_masks(cfg) * cfg.batch
    _need(keep_override, "keep_override", torch.uint8, nmb)
    _need(keep_out, "keep_out", torch.uint8, nmb)
    _need(idx_out, "idx_out", torch.int32, nmb)
    _need(count_out, "count_out", torch.int32, L * _n_masks(cfg))
    wa = (ld_weights * L)(*[weights(w) for w in ws_list])
    ga = (ld_grads * L)(*[grads(g) for g in dw_list])
    pa = (C.c_float * L)(*[float(v) for v in p])
    _check(_lib.ld_stack_step(C.byref(cfg), L, wa, pa, seed, step, _ptr(x), _ptr(dx), ga, _ptr(ws),
                              ws.numel() * ws.element_size(), _ptr(keep_override), _ptr(keep_out),
                              _ptr(idx_out), _ptr(count_out), _stream(stream)))


def _u8_array(v, n):
    if v is None:
        return None
    return (C.c_uint8 * n)(*[1 if a else 0 for a in v])


def _f32_array(v, n):
    if v is None:
        return None
    if isinstance(v, (int, float)):
        v = [v] * n
    return (C.c_float * n)(*[float(a) for a in v])


def _ptr_array(v, n):
    if v is None:
        return None
    return (C.c_void_p * n)(*[_ptr(t) for t in v])


def ld_eval_ws_bytes(cfg):
    return _lib.ld_eval_ws_bytes(C.byref(cfg))


def ld_stack_eval(cfg, ws_list, x, ws, active=None, r_eval=None, kv=None, s_max=0, stream=None):
    """Forward-only evaluation form over the active layers; kv: list of
    per-layer caches (None entries allowed for inactive layers)."""
    L = len(ws_list)
    act, rr, kk = _u8_array(active, L), _f32_array(r_eval, L), _ptr_array(kv, L)
    wa = _stack_weights(cfg, ws_list, act)
    _check(_lib.ld_stack_eval(C.byref(cfg), L, wa, act, rr, _ptr(x), kk, s_max, _ptr(ws),
                              ws.numel() * ws.element_size(), _stream(stream)))


def ld_decode_ws_bytes(cfg, n_new, s_max):
    return _lib.ld_decode_ws_bytes(C.byref(cfg), n_new, s_max)


def ld_stack_decode(cfg, ws_list, x, kv, s_max, pos, n_new, ws, active=None, r_eval=None,
                    stream=None):
    L = len(ws_list)
    act, rr, kk = _u8_array(active, L), _f32_array(r_eval, L), _ptr_array(kv, L)
    wa = _stack_weights(cfg, ws_list, act)
    _check(_lib.ld_stack_decode(C.byref(cfg), L, wa, act, rr, _ptr(x), kk, s_max, pos, n_new,
                                _ptr(ws), ws.numel() * ws.element_size(), _stream(stream)))


def ld_gemm_skinny_ws_bytes(M, N, K):
    return _lib.ld_gemm_skinny_ws_bytes(M, N, K)


def ld_gemm_skinny(A, W, C_out, alpha=1.0, R=None, ws=None, stream=None):
    M, K = A.shape
    N = W.shape[0]
    _check(_lib.ld_gemm_skinny(M, N, K, _ptr(A, "A", inner=True), A.stride(0),
                               _ptr(W, "W", inner=True), W.stride(0), _ptr(C_out, "C_out", inner=True),
                               C_out.stride(0), alpha, _ptr(R, "R", inner=True),
                               0 if R is None else R.stride(0), _ptr(ws, "ws"),
                               0 if ws is None else ws.numel() * ws.element_size(), _stream(stream)))


DEC_ACT_NONE, DEC_ACT_SWIGLU, DEC_ACT_RELU2 = 0, 1, 2


def ld_gemm_dec(A, W, C_out, g=None, eps=1e-5, alpha=1.0, R=None, act=DEC_ACT_NONE, stream=None):
    """Fused decoding projection (M <= 8 rows): C = act(R + alpha A' W^T), A'
    the RMSNorm of A's rows with gain g when g is given; with SwiGLU W holds
    the gate rows then the up rows and C has half as many columns."""
    M, K = A.shape
    N = C_out.shape[1]
    _check(_lib.ld_gemm_dec(M, N, K, _ptr(A, "A", inner=True), A.stride(0), _ptr(g, "g"), eps,
                            _ptr(W, "W", inner=True), W.stride(0), _ptr(C_out, "C_out", inner=True),
                            C_out.stride(0), alpha, _ptr(R, "R", inner=True),
                            0 if R is None else R.stride(0), act, _stream(stream)))


def ld_kv_store(n_seq, n_new, d_model, pos, qkv, kv, s_max, stream=None):
    _check(_lib.ld_kv_store(n_seq, n_new, d_model, pos, _ptr(qkv), _ptr(kv), s_max, _stream(stream)))


def ld_attn_decode_ws_bytes(n_seq, n_heads, d_head, s_max):
    return _lib.ld_attn_decode_ws_bytes(n_seq, n_heads, d_head, s_max)


def ld_attn_decode(n_seq, n_heads, d_head, pos, n_new, qkv, kv, s_max, o, ws, alibi=0, stream=None):
    _check(_lib.ld_attn_decode(n_seq, n_heads, d_head, alibi, pos, n_new, _ptr(qkv), _ptr(kv), s_max,
                               _ptr(o), _ptr(ws), ws.numel() * ws.element_size(), _stream(stream)))


def kv8(codes, scales, format, block, n_seq, n_kv_heads, d_head, s_max):
    """ld_kv8 over device tensors: codes (uint8) and scales (float32), of
    ld_kv8_code_bytes and ld_kv8_scale_bytes bytes; None for a descriptor that
    only those two are asked about.  It keeps the tensors."""
    kv = ld_kv8(format, block, n_seq, n_kv_heads, d_head, s_max)
    if codes is not None or scales is not None:
        n, m = ld_kv8_code_bytes(kv), ld_kv8_scale_bytes(kv)
        if n:   # an invalid descriptor is refused by the call that takes it
            _need(codes, "codes", torch.uint8, n)
            _need(scales, "scales", torch.float32, m // 4)
        kv.codes, kv.scales = _ptr(codes, "codes"), _ptr(scales, "scales")
        if isinstance(codes, torch.Tensor) and isinstance(scales, torch.Tensor):
            if codes.device != scales.device:
                raise ValueError(f"codes on {codes.device}, scales on {scales.device}")
            kv.device = codes.device.index
        kv.tensors = (codes, scales)
    return kv


def ld_kv8_code_bytes(kv):
    return _lib.ld_kv8_code_bytes(C.byref(kv))


def ld_kv8_scale_bytes(kv):
    return _lib.ld_kv8_scale_bytes(C.byref(kv))


def _kv8_device(kv):
    """The current device, on which the cache (or 4-bit weights) and the stream
    have to be; None for one given by addresses."""
    if kv.device is not None and kv.device != torch.cuda.current_device():
        raise ValueError(f"codes: on cuda:{kv.device}, which is not the current device")
    return kv.device


def _kv8_ptr(t, name, device, dtype=None, numel=None):
    """_need and _ptr of an argument on `device`."""
    if t is None:
        return None
    if type(t) is torch.Tensor and t.get_device() == device and t.is_contiguous() and \
            (dtype is None or (t.dtype is dtype and t.numel() == numel)):
        return t.data_ptr()     # the usual case, 0.3 us sooner
    if isinstance(t, torch.Tensor):
        if dtype is not None:
            _need(t, name, dtype, numel)
        if t.is_cuda and t.device.index != (torch.cuda.current_device() if device is None else device):
            raise ValueError(f"{name}: on {t.device}, which is not the current device")
    return _ptr(t, name)


def _stack_weights_on(cfg, ws_list, active, device):
    return _stack_weights(cfg, ws_list, active, lambda t, name, dtype, numel: _kv8_ptr(t, name, device, dtype, numel),
                          device)


def _kv8_rows(kv, n_heads, n_new, qkv, device):
    return _kv8_ptr(qkv, "qkv", device, torch.bfloat16,
                    kv.n_seq * n_new * (n_heads + 2 * kv.n_kv_heads) * kv.d_head)


def ld_kv8_store(kv, n_heads, n_new, pos, qkv, seq_pos=None, stream=None):
    """Quantise the keys and values of qkv rows into the cache at positions
    pos (or seq_pos[b] <= pos) onwards."""
    dev = _kv8_device(kv)
    _check(_lib.ld_kv8_store(C.byref(kv), n_heads, n_new, pos,
                             _kv8_ptr(seq_pos, "seq_pos", dev, torch.int32, kv.n_seq),
                             _kv8_rows(kv, n_heads, n_new, qkv, dev), _stream(stream, dev)))


def ld_kv8_load(kv, pos, n, out, seq_len=None, stream=None):
    """Positions pos .. pos + n - 1 back to bfloat16 rows [n_seq, n, 2 n_kv_heads d_head]."""
    dev = _kv8_device(kv)
    _check(_lib.ld_kv8_load(C.byref(kv), pos, n, _kv8_ptr(seq_len, "seq_len", dev, torch.int32, kv.n_seq),
                            _kv8_ptr(out, "out", dev, torch.bfloat16, kv.n_seq * n * 2 * kv.n_kv_heads * kv.d_head),
                            _stream(stream, dev)))


def ld_attn_decode_kv8_ws_bytes(kv, n_heads, n_new):
    return _lib.ld_attn_decode_kv8_ws_bytes(C.byref(kv), n_heads, n_new)


def ld_attn_decode_kv8(kv, n_heads, pos, n_new, qkv, o, ws, seq_pos=None, alibi=0, stream=None):
    """Attention of n_new rows per sequence at positions pos (or seq_pos[b])
    onwards over the cache, which already holds them."""
    dev = _kv8_device(kv)
    _check(_lib.ld_attn_decode_kv8(C.byref(kv), n_heads, int(alibi), pos,
                                   _kv8_ptr(seq_pos, "seq_pos", dev, torch.int32, kv.n_seq), n_new,
                                   _kv8_rows(kv, n_heads, n_new, qkv, dev),
                                   _kv8_ptr(o, "o", dev, torch.bfloat16, kv.n_seq * n_new * n_heads * kv.d_head),
                                   _kv8_ptr(ws, "ws", dev), ws.numel() * ws.element_size(), _stream(stream, dev)))


def _kv8_array(kv, n):
    """Descriptors of n layers; None (an inactive layer's) as an empty one.  And
    the device that the other arguments have to be on (_kv8_device)."""
    if len(kv) != n:
        raise ValueError(f"{n} layers of weights, {len(kv)} of caches")
    device = None
    for k in kv:
        if k is not None:
            d = _kv8_device(k)
            device = d if device is None else device
    return (ld_kv8 * n)(*[k if k is not None else ld_kv8() for k in kv]), device


def ld_stack_eval_kv8(cfg, ws_list, x, ws, kv, active=None, r_eval=None, stream=None):
    """ld_stack_eval that writes 8-bit caches; kv: a kv8() per layer (None
    allowed for inactive layers)."""
    L = len(ws_list)
    act, rr, (kk, dev) = _u8_array(active, L), _f32_array(r_eval, L), _kv8_array(kv, L)
    wa = _stack_weights_on(cfg, ws_list, act, dev)
    px = _kv8_ptr(x, "x", dev, torch.bfloat16, cfg.batch * cfg.seq * cfg.d_model)
    _check(_lib.ld_stack_eval_kv8(C.byref(cfg), L, wa, act, rr, px, kk, _kv8_ptr(ws, "ws", dev),
                                  ws.numel() * ws.element_size(), _stream(stream, dev)))


def ld_decode_kv8_ws_bytes(cfg, n_new, s_max):
    return _lib.ld_decode_kv8_ws_bytes(C.byref(cfg), n_new, s_max)


def ld_stack_decode_kv8(cfg, ws_list, x, kv, pos, n_new, ws, seq_pos=None, active=None, r_eval=None,
                        stream=None):
    """ld_stack_decode over 8-bit caches; seq_pos: int32 [batch] positions on
    the device (at most pos), where they differ or the call is captured."""
    L = len(ws_list)
    act, rr, (kk, dev) = _u8_array(active, L), _f32_array(r_eval, L), _kv8_array(kv, L)
    wa = _stack_weights_on(cfg, ws_list, act, dev)
    px = _kv8_ptr(x, "x", dev, torch.bfloat16, cfg.batch * n_new * cfg.d_model)
    _check(_lib.ld_stack_decode_kv8(C.byref(cfg), L, wa, act, rr, px, kk, pos,
                                    _kv8_ptr(seq_pos, "seq_pos", dev, torch.int32, cfg.batch), n_new,
                                    _kv8_ptr(ws, "ws", dev), ws.numel() * ws.element_size(), _stream(stream, dev)))


def _on_one_device(obj, tensors):
    """Notes the device of a descriptor's tensors, which it keeps."""
    devs = {t.device for t in tensors if isinstance(t, torch.Tensor)}
    if len(devs) > 1:
        raise ValueError("the descriptor's tensors are on " + " and ".join(sorted(map(str, devs))))
    if devs:
        obj.device = devs.pop().index
    obj.tensors = tensors
    return obj


def w4(codes, scales, format, group, n, k):
    """ld_w4 over device tensors: codes (uint8) and scales (uint8 for e2m1,
    bfloat16 for int4), of ld_w4_code_bytes and ld_w4_scale_bytes bytes; None for
    a descriptor that only those two are asked about.  It keeps the tensors."""
    w = ld_w4(format, group, n, k)
    if codes is None and scales is None:
        return w
    nb, sb = ld_w4_code_bytes(w), ld_w4_scale_bytes(w)
    if nb:   # an invalid descriptor is refused by the call that takes it
        _need(codes, "codes", torch.uint8, nb)
        if format == LD_W4_E2M1:
            _need(scales, "scales", torch.uint8, sb)
        else:
            _need(scales, "scales", torch.bfloat16, sb // 2)
    w.codes, w.scales = _ptr(codes, "codes"), _ptr(scales, "scales")
    return _on_one_device(w, (codes, scales))


def ld_w4_code_bytes(w):
    return _lib.ld_w4_code_bytes(C.byref(w))


def ld_w4_scale_bytes(w):
    return _lib.ld_w4_scale_bytes(C.byref(w))


def _w4_rows(w, t, name, device):
    """A matrix [n, k] in bfloat16 whose rows may be apart."""
    if isinstance(t, torch.Tensor):
        if t.dtype != torch.bfloat16 or tuple(t.shape) != (w.n, w.k):
            raise ValueError(f"{name}: {t.dtype} {tuple(t.shape)}, expected bfloat16 {(w.n, w.k)}")
        if t.is_cuda and device is not None and t.device.index != device:
            raise ValueError(f"{name}: on {t.device}, the descriptor's tensors on cuda:{device}")
    return _ptr(t, name, inner=True), t.stride(0) if w.n > 1 else w.k


def ld_w4_pack(w, src, stream=None):
    """bfloat16 weights [n, k] to 4 bits."""
    dev = _kv8_device(w)
    p, ld = _w4_rows(w, src, "src", dev)
    _check(_lib.ld_w4_pack(C.byref(w), p, ld, _stream(stream, dev)))


def ld_w4_load(w, dst, stream=None):
    """4-bit weights back to bfloat16 [n, k]."""
    dev = _kv8_device(w)
    p, ld = _w4_rows(w, dst, "dst", dev)
    _check(_lib.ld_w4_load(C.byref(w), p, ld, _stream(stream, dev)))


def ld_gemm_w4_ws_bytes(w, M, act=DEC_ACT_NONE):
    return _lib.ld_gemm_w4_ws_bytes(C.byref(w), M, act)


def _rows_2d(t, name, device, shape):
    """Address and row distance of a bfloat16 matrix whose rows may be apart."""
    if t is None:
        return None, 0
    if type(t) is torch.Tensor and t.get_device() == device and t.dtype is torch.bfloat16 and t.shape == shape:
        ld, step = t.stride()
        if step == 1:
            return t.data_ptr(), ld if shape[0] > 1 else shape[1]   # the usual case, 0.3 us sooner
    if isinstance(t, torch.Tensor):
        if t.dtype is not torch.bfloat16 or t.dim() != 2 or t.shape[0] != shape[0] or t.shape[1] != shape[1]:
            raise ValueError(f"{name}: {t.dtype} {tuple(t.shape)}, expected bfloat16 {tuple(shape)}")
        if t.get_device() != (torch.cuda.current_device() if device is None else device):
            raise ValueError(f"{name}: on {t.device}, which is not the current device")
        if shape[1] > 1 and t.stride(1) != 1:
            raise ValueError(f"{name}: the last dimension must be contiguous")
    return t.data_ptr(), t.stride(0) if shape[0] > 1 else shape[1]


def _ws(ws, device):
    """Address and bytes of a workspace."""
    if ws is None:
        return None, 0
    return _kv8_ptr(ws, "ws", device), ws.numel() * ws.element_size()


def ld_gemm_w4(w, A, C_out, ws=None, g=None, eps=1e-5, alpha=1.0, R=None, act=DEC_ACT_NONE, stream=None):
    """Projection of up to 64 rows by 4-bit weights, C = act(R + alpha A' W^T), A' the
    RMSNorm of A's rows with gain g when g is given; with SwiGLU w holds the gate
    rows then the up rows and C has half as many columns."""
    dev = _kv8_device(w)
    M, N = A.shape[0], w.n // 2 if act == DEC_ACT_SWIGLU else w.n
    pa, lda = _rows_2d(A, "A", dev, (M, w.k))
    pc, ldc = _rows_2d(C_out, "C_out", dev, (M, N))
    pr, ldr = _rows_2d(R, "R", dev, (M, N))
    pw, wsb = _ws(ws, dev)
    _check(_lib.ld_gemm_w4(M, pa, lda, _kv8_ptr(g, "g", dev, torch.bfloat16, w.k),
                           eps, C.byref(w), pc, ldc, alpha, pr, ldr, act, pw, wsb, _stream(stream, dev)))


def kv4(codes, scales, n_seq, n_kv_heads, d_head, s_max, sums=None):
    """ld_kv4 over device tensors: codes and scales (uint8) of ld_kv4_code_bytes and
    ld_kv4_scale_bytes bytes, sums None or float32 [n_seq, n_kv_heads, s_max]; None for
    a descriptor that only sizes are asked about.  It keeps the tensors."""
    kv = ld_kv4(n_seq, n_kv_heads, d_head, s_max)
    if codes is None and scales is None and sums is None:
        return kv
    n, m = ld_kv4_code_bytes(kv), ld_kv4_scale_bytes(kv)
    if n:   # an invalid descriptor is refused by the call that takes it
        _need(codes, "codes", torch.uint8, n)
        _need(scales, "scales", torch.uint8, m)
        _need(sums, "sums", torch.float32, n_seq * n_kv_heads * s_max)
    kv.codes, kv.scales, kv.sums = _ptr(codes, "codes"), _ptr(scales, "scales"), _ptr(sums, "sums")
    return _on_one_device(kv, (codes, scales, sums))


def ld_kv4_code_bytes(kv):
    return _lib.ld_kv4_code_bytes(C.byref(kv))


def ld_kv4_scale_bytes(kv):
    return _lib.ld_kv4_scale_bytes(C.byref(kv))


def ld_kv4_store(kv, n_heads, n_new, pos, qkv, seq_pos=None, stream=None):
    """Quantise the keys and values of qkv rows into the cache at positions
    pos (or seq_pos[b] <= pos) onwards."""
    dev = _kv8_device(kv)
    _check(_lib.ld_kv4_store(C.byref(kv), n_heads, n_new, pos,
                             _kv8_ptr(seq_pos, "seq_pos", dev, torch.int32, kv.n_seq),
                             _kv8_rows(kv, n_heads, n_new, qkv, dev), _stream(stream, dev)))


def ld_kv4_load(kv, pos, n, out, seq_len=None, stream=None):
    """Positions pos .. pos + n - 1 back to bfloat16 rows [n_seq, n, 2 n_kv_heads d_head]."""
    dev = _kv8_device(kv)
    _check(_lib.ld_kv4_load(C.byref(kv), pos, n, _kv8_ptr(seq_len, "seq_len", dev, torch.int32, kv.n_seq),
                            _kv8_ptr(out, "out", dev, torch.bfloat16, kv.n_seq * n * 2 * kv.n_kv_heads * kv.d_head),
                            _stream(stream, dev)))


def ld_attn_decode_kv4_ws_bytes(kv, n_heads, n_new):
    return _lib.ld_attn_decode_kv4_ws_bytes(C.byref(kv), n_heads, n_new)


def ld_attn_decode_kv4(kv, n_heads, pos, n_new, qkv, o, ws, seq_pos=None, alibi=0, stream=None):
    """Attention of n_new rows per sequence at positions pos (or seq_pos[b])
    onwards over the cache, which already holds them; its weights are added to
    the cache's sums, if it has some."""
    dev = _kv8_device(kv)
    pw, wsb = _ws(ws, dev)
    _check(_lib.ld_attn_decode_kv4(C.byref(kv), n_heads, int(alibi), pos,
                                   _kv8_ptr(seq_pos, "seq_pos", dev, torch.int32, kv.n_seq), n_new,
                                   _kv8_rows(kv, n_heads, n_new, qkv, dev),
                                   _kv8_ptr(o, "o", dev, torch.bfloat16, kv.n_seq * n_new * n_heads * kv.d_head),
                                   pw, wsb, _stream(stream, dev)))


def ld_kv4_evict_ws_bytes(kv, length, keep):
    return _lib.ld_kv4_evict_ws_bytes(C.byref(kv), length, keep)


def ld_kv4_evict(src, dst, length, keep, recent, idx, ws=None, seq_len=None, stream=None):
    """Of each head's first `length` (or seq_len[b] <= length) positions of src the last
    `recent` and the keep - recent others with the largest sums, to dst; idx: int32
    [n_seq, n_kv_heads, keep], their positions."""
    dev = _kv8_device(src)
    if dst.device is not None and dev is not None and dst.device != dev:
        raise ValueError(f"dst: on cuda:{dst.device}, src on cuda:{dev}")
    pw, wsb = _ws(ws, dev)
    _check(_lib.ld_kv4_evict(C.byref(src), C.byref(dst), length,
                             _kv8_ptr(seq_len, "seq_len", dev, torch.int32, src.n_seq), keep, recent,
                             _kv8_ptr(idx, "idx", dev, torch.int32, src.n_seq * src.n_kv_heads * max(keep, 0)),
                             pw, wsb, _stream(stream, dev)))


def weights_w4(w):
    """ld_weights_w4 from a dict keyed by WEIGHT_KEYS: gains as device tensors
    (bfloat16, of as many elements as w_qkv has k), matrices as w4()s."""
    d, dev = w["w_qkv"].k, w["w_qkv"].device
    return ld_weights_w4(*[_kv8_ptr(w[k], k, dev, torch.bfloat16, d) for k in ("g_attn", "g_mlp")],
                         *[w[k] for k in ("w_qkv", "w_o", "w_gate_up", "w_down")])


def _kv4_array(kv, n):
    """Descriptors of n layers and their device, as _kv8_array's."""
    if len(kv) != n:
        raise ValueError(f"{n} layers of weights, {len(kv)} of caches")
    device = None
    for k in kv:
        if k is not None:
            d = _kv8_device(k)
            device = d if device is None else device
    return (ld_kv4 * n)(*[k if k is not None else ld_kv4() for k in kv]), device


def ld_stack_eval_kv4(cfg, ws_list, x, ws, kv, active=None, r_eval=None, stream=None):
    """ld_stack_eval that writes 4-bit caches; kv: a kv4() per layer (None
    allowed for inactive layers)."""
    L = len(ws_list)
    act, rr, (kk, dev) = _u8_array(active, L), _f32_array(r_eval, L), _kv4_array(kv, L)
    wa = _stack_weights_on(cfg, ws_list, act, dev)
    px = _kv8_ptr(x, "x", dev, torch.bfloat16, cfg.batch * cfg.seq * cfg.d_model)
    pw, wsb = _ws(ws, dev)
    _check(_lib.ld_stack_eval_kv4(C.byref(cfg), L, wa, act, rr, px, kk, pw, wsb, _stream(stream, dev)))


def ld_decode_kv4_ws_bytes(cfg, n_new, s_max, sums=False):
    return _lib.ld_decode_kv4_ws_bytes(C.byref(cfg), n_new, s_max, int(sums))


def _stack_decode_4(call, weights_of, cfg, ws_list, x, kv, pos, n_new, ws, seq_pos, active, r_eval, stream):
    L = len(ws_list)
    act, rr, (kk, dev) = _u8_array(active, L), _f32_array(r_eval, L), _kv4_array(kv, L)
    wa = weights_of(cfg, ws_list, act, dev)
    px = _kv8_ptr(x, "x", dev, torch.bfloat16, cfg.batch * n_new * cfg.d_model)
    pw, wsb = _ws(ws, dev)
    _check(call(C.byref(cfg), L, wa, act, rr, px, kk, pos, _kv8_ptr(seq_pos, "seq_pos", dev, torch.int32, cfg.batch),
                n_new, pw, wsb, _stream(stream, dev)))


def ld_stack_decode_kv4(cfg, ws_list, x, kv, pos, n_new, ws, seq_pos=None, active=None, r_eval=None,
                        stream=None):
    """ld_stack_decode over 4-bit caches; seq_pos as in ld_stack_decode_kv8."""
    _stack_decode_4(_lib.ld_stack_decode_kv4, _stack_weights_on, cfg, ws_list, x, kv, pos, n_new, ws, seq_pos,
                    active, r_eval, stream)


def _stack_weights_w4(cfg, ws_list, active, device):
    for w in ws_list:
        for k in ("w_qkv", "w_o", "w_gate_up", "w_down"):
            _kv8_device(w[k])
    return (ld_weights_w4 * len(ws_list))(*[weights_w4(w) for w in ws_list])


def ld_stack_decode_w4(cfg, ws_list, x, kv, pos, n_new, ws, seq_pos=None, active=None, r_eval=None,
                       stream=None):
    """ld_stack_decode_kv4 with the layers' matrices in 4 bits; ws_list: a dict
    for weights_w4() per layer."""
    _stack_decode_4(_lib.ld_stack_decode_w4, _stack_weights_w4, cfg, ws_list, x, kv, pos, n_new, ws, seq_pos,
                    active, r_eval, stream)


def ld_rmsnorm_fwd(x, g, y, rstd, eps=1e-5, stream=None):
    rows, d = x.shape
    _check(_lib.ld_rmsnorm_fwd(_dtype_code(x), rows, d, eps, _ptr(x), _ptr(g), _ptr(y), _ptr(rstd),
                               _stream(stream)))


def ld_rmsnorm_bwd_ws_bytes(rows, d):
    return _lib.ld_rmsnorm_bwd_ws_bytes(rows, d)


def ld_rmsnorm_bwd(x, g, rstd, gy, gres, gx, dg, ws, stream=None):
    rows, d = x.shape
    _check(_lib.ld_rmsnorm_bwd(_dtype_code(x), rows, d, _ptr(x), _ptr(g), _ptr(rstd), _ptr(gy),
                               _ptr(gres), _ptr(gx), _ptr(dg), _ptr(ws),
                               ws.numel() * ws.element_size(), _stream(stream)))


def ld_relu2_fwd(u, s, stream=None):
    rows, f = u.shape
    _check(_lib.ld_relu2_fwd(_dtype_code(u), rows, f, _ptr(u), _ptr(s), _stream(stream)))


def ld_relu2_bwd(u, gs, gu, stream=None):
    rows, f = u.shape
    _check(_lib.ld_relu2_bwd(_dtype_code(u), rows, f, _ptr(u), _ptr(gs), _ptr(gu),
                             _stream(stream)))


def ld_alibi_slope(h, n_heads):
    return _lib.ld_alibi_slope(h, n_heads)


def ld_swiglu_fwd(uv, s, stream=None):
    rows, f2 = uv.shape
    _check(_lib.ld_swiglu_fwd(_dtype_code(uv), rows, f2 // 2, _ptr(uv), _ptr(s), _stream(stream)))


def ld_swiglu_bwd(uv, gs, guv, stream=None):
    rows, f2 = uv.shape
    _check(_lib.ld_swiglu_bwd(_dtype_code(uv), rows, f2 // 2, _ptr(uv), _ptr(gs), _ptr(guv),
                              _stream(stream)))


def ld_gemm_ws_bytes(dtype, a_kcontig, b_kcontig, M, N, K, ldc, c_f32):
    return _lib.ld_gemm_ws_bytes(dtype, int(a_kcontig), int(b_kcontig), M, N, K, ldc, int(c_f32))


def ld_gemm(a_kcontig, b_kcontig, M, N, K, A, lda, B, ldb, Cm, ldc, alpha=1.0, R=None, ldr=0,
            c_f32=False, dtype=None, ws=None, stream=None):
    dt = _dtype_code(A) if dtype is None else dtype
    ws_bytes = 0 if ws is None else ws.numel() * ws.element_size()
    _check(_lib.ld_gemm(dt, int(a_kcontig), int(b_kcontig), M, N, K, _ptr(A, "A", inner=True), lda,
                        _ptr(B, "B", inner=True), ldb, _ptr(Cm, "C", inner=True), ldc, int(c_f32), alpha,
                        _ptr(R, "R", inner=True), ldr, _ptr(ws, "ws"), ws_bytes, _stream(stream)))


def ld_attn_fwd(n_seq, seq, n_heads, d_head, qkv, o, lse, stream=None, alibi=0):
    _check(_lib.ld_attn_fwd(_dtype_code(qkv), n_seq, seq, n_heads, d_head, int(alibi), _ptr(qkv),
                            _ptr(o), _ptr(lse), _stream(stream)))


def ld_attn_bwd_ws_bytes(n_seq, seq, n_heads):
    return _lib.ld_attn_bwd_ws_bytes(n_seq, seq, n_heads)


def ld_attn_bwd(n_seq, seq, n_heads, d_head, qkv, o, lse, go, gqkv, ws, stream=None, alibi=0):
    _check(_lib.ld_attn_bwd(_dtype_code(qkv), n_seq, seq, n_heads, d_head, int(alibi), _ptr(qkv),
                            _ptr(o), _ptr(lse), _ptr(go), _ptr(gqkv), _ptr(ws),
                            ws.numel() * ws.element_size(), _stream(stream)))


def ld_attn_bwd_noalloc(n_seq, seq, n_heads, d_head, qkv, o, lse, go, gqkv, stream=None, alibi=0):
    _check(_lib.ld_attn_bwd_noalloc(_dtype_code(qkv), n_seq, seq, n_heads, d_head, int(alibi),
                                    _ptr(qkv, "qkv"), _ptr(o, "o"), _ptr(lse, "lse"), _ptr(go, "go"),
                                    _ptr(gqkv, "gqkv"), _stream(stream)))


def ld_prof_start(kernel_name):
    _check(_lib.ld_prof_start(kernel_name.encode()))


def ld_prof_stop():
    _check(_lib.ld_prof_stop())


def ld_prof_result():
    n, ms, fl, by = C.c_int64(), C.c_double(), C.c_double(), C.c_double()
    _check(_lib.ld_prof_result(C.byref(n), C.byref(ms), C.byref(fl), C.byref(by)))
    return dict(launches=n.value, ms=ms.value, flops=fl.value, bytes=by.value)
