"""Binding of include/accerl.h (ctypes; forwards, V-trace and the KL indicators through the compiled accerl_args): same names, argument marshalling only."""
import contextlib
import ctypes as C
import os
import threading

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
_SO = os.path.join(_HERE, "libaccerl.so")
_BUILD = "run `python -c 'import __graft_entry__ as g; g.build()'` (or paper_2211_15023_amd/build.py)"
_lib = None
torch = None            # set by load_library
_args = None            # accerl_args, set by _loaded

INT8, FP32, BF16 = 0, 1, 2
OBS_U8, OBS_F32 = 0, 1
TAP_ACC, TAP_ACT, TAP_ACC_A, TAP_ACT_A = 0, 1, 2, 3
MAX_LAYERS = 48
_KINDS = {"conv": 1, "dense": 2, "maxpool": 3, "resblock": 4, "relu": 5, "flatten": 6, "lstm": 7}
_PREC = {"int8": INT8, "fp32": FP32, "bf16": BF16}


class AccerlError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"accerl status {code}: {msg}")
        self.code = code


class _Layer(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("kind", "cin", "cout", "k", "stride", "pad", "relu", "reserved")]


class _Arch(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("obs_dtype", "obs_c", "obs_h", "obs_w", "n_actions", "precision", "n_layers")] + \
               [("layers", _Layer * MAX_LAYERS)]


class _PolicyLossArgs(C.Structure):
    _fields_ = [("B", C.c_int64), ("A", C.c_int64), ("dtype", C.c_int32), ("kl_kind", C.c_int32), ("logits", C.c_void_p), ("ld_logits", C.c_int64),
                ("ref_logits", C.c_void_p), ("ld_ref", C.c_int64), ("grad_logits", C.c_void_p), ("ld_grad", C.c_int64),
                ("mask", C.c_void_p), ("ld_mask", C.c_int64)] + \
               [(n, C.c_void_p) for n in ("actions", "old_logp", "advantages", "weights", "ref_logp")] + \
               [(n, C.c_double) for n in ("clip_low", "clip_high", "kl_coef", "entropy_coef", "scale")] + \
               [(n, C.c_void_p) for n in ("out_loss", "out_logp", "out_kl", "out_entropy", "out_stats", "workspace")] + [("workspace_bytes", C.c_int64)]


def load_library():
    """Load libaccerl.so (after torch, so that both share one HIP runtime).  No fallback exists."""
    global _lib, torch
    if _lib is not None:
        return _lib
    import torch as _torch  # brings in the HIP runtime the library links against
    torch = _torch
    _CODES.update({torch.float32: 0, torch.bfloat16: 1, torch.float16: 2})
    if not os.path.exists(_SO):
        raise ImportError(f"{_SO} is missing: {_BUILD}; there is no CPU fallback")
    lib = C.CDLL(_SO)
    vp, i64, i32 = C.c_void_p, C.c_int64, C.c_int32
    lib.accerl_blob_sizes.argtypes = [C.POINTER(_Arch), C.POINTER(i64), C.POINTER(i64)]
    lib.accerl_policy_create.argtypes = [C.POINTER(_Arch), vp, i64, vp, i64, C.POINTER(vp)]
    lib.accerl_policy_destroy.argtypes = [vp]
    lib.accerl_policy_destroy.restype = None
    fwd = [vp, vp, i64, vp, vp, vp, vp, vp]
    lib.accerl_actor_forward.argtypes = fwd
    lib.accerl_actor_forward_teacher.argtypes = fwd
    lib.accerl_actor_forward_recurrent.argtypes = [vp, vp, i64, vp, vp, vp, vp, vp, vp, vp, vp]
    lib.accerl_actor_forward_debug.argtypes = [vp, vp, i64, i32, i32, vp, i64, vp]
    lib.accerl_plan_describe.argtypes = [C.POINTER(_Arch), vp, i64, vp, i64, C.c_char_p, i64]
    lib.accerl_plan_describe.restype = C.c_int
    lib.accerl_profile_begin.argtypes = [vp]
    lib.accerl_profile_end.argtypes = [vp, i32, vp, vp, vp, vp, vp]
    lib.accerl_monitor_kl.argtypes = [vp, vp, i64, i32, vp, vp, vp, vp]
    lib.accerl_vtrace.argtypes = [vp, vp, vp, vp, vp, vp, vp, i64, i64, i32, C.c_float, C.c_float, vp, vp, vp, vp]
    lib.accerl_monitor_kl.restype = C.c_int
    lib.accerl_monitor_kl_noalloc.argtypes = [vp, vp, i64, i32, vp, vp, vp, vp]
    lib.accerl_monitor_kl_noalloc.restype = C.c_int
    lib.accerl_probe_mfma.argtypes = [i32, i32, vp, vp]
    lib.accerl_probe_mfma.restype = C.c_int
    lib.accerl_probe_copy.argtypes = [vp, vp, i64, vp]
    lib.accerl_probe_copy.restype = C.c_int
    lib.accerl_probe_empty.argtypes = [vp]
    lib.accerl_probe_empty.restype = C.c_int
    lib.accerl_actor_forward_mixture.argtypes = [vp, vp, vp, i64, vp, vp, vp, vp, vp, vp]
    lib.accerl_actor_forward_mixture.restype = C.c_int
    lib.accerl_mixture_alpha.argtypes = [C.c_double, C.c_double, C.c_double]
    lib.accerl_mixture_alpha.restype = C.c_double
    lib.accerl_distill_loss.argtypes = [vp, vp, vp, vp, i64, i32, C.c_float, vp, vp, vp]
    lib.accerl_distill_loss.restype = C.c_int
    lib.accerl_vtrace.restype = C.c_int
    lib.accerl_packed_rows_bytes.argtypes = [i64, i64]
    lib.accerl_packed_rows_bytes.restype = i64
    lib.accerl_quantize_rows.argtypes = [vp, i32, i64, i64, i64, vp, vp, vp]
    lib.accerl_pack_rows_i8.argtypes = [vp, i64, i64, i64, vp, vp]
    lib.accerl_unpack_rows_i8.argtypes = [vp, i64, i64, vp, i64, vp]
    lib.accerl_dense_i8.argtypes = [vp, vp, vp, vp, vp, i64, i64, i64, i32, vp, i32, i64, vp]
    lib.accerl_dense_i8_workspace.argtypes = [i64, i64]
    lib.accerl_dense_i8_workspace.restype = i64
    lib.accerl_dense_i8_dynamic.argtypes = [vp, i32, i64, vp, vp, vp, i64, i64, i64, i32, vp, i32, i64, vp, i64, vp]
    lib.accerl_policy_loss_workspace.argtypes = []
    lib.accerl_policy_loss_workspace.restype = i64
    lib.accerl_action_logprob.argtypes = [vp, i32, i64, vp, i64, vp, i64, i64, vp, vp, vp, i64, vp]
    lib.accerl_policy_loss.argtypes = [C.POINTER(_PolicyLossArgs), vp]
    lib.accerl_last_error.restype = C.c_char_p
    for f in ("accerl_blob_sizes", "accerl_policy_create", "accerl_actor_forward", "accerl_actor_forward_teacher",
              "accerl_actor_forward_recurrent", "accerl_actor_forward_debug", "accerl_profile_begin",
              "accerl_profile_end"):
        getattr(lib, f).restype = C.c_int
    _lib = lib
    try:
        _loaded()                            # here and not in the first call that needs it, which says it if there is none
    except ImportError:
        pass
    return lib


def _loaded():
    """accerl_args, for the calls that go through it; the others, and host-only ones, do without it."""
    global _args
    load_library()                           # accerl_args links against torch and the library
    try:
        from . import accerl_args
    except ImportError as e:
        raise ImportError(f"accerl_args.so is missing or of another torch or Python ({e}): {_BUILD}") from e
    accerl_args.init(C.c_void_p)
    _args = accerl_args
    return _args


def accerl_last_error():
    return load_library().accerl_last_error().decode()


def _check(rc):
    if rc != 0:
        raise AccerlError(rc, accerl_last_error())


def make_arch(net, precision):
    """net: object with obs_dtype ("u8"/"f32"), obs_shape, n_actions, layers (list of dicts)."""
    a = _Arch()
    a.obs_dtype = OBS_U8 if net.obs_dtype == "u8" else OBS_F32
    shp = tuple(net.obs_shape)
    a.obs_c, a.obs_h, a.obs_w = (shp[0], 1, 1) if len(shp) == 1 else shp
    a.n_actions = net.n_actions
    a.precision = _PREC[precision] if isinstance(precision, str) else int(precision)
    if len(net.layers) > MAX_LAYERS:
        raise ValueError("too many layers")
    a.n_layers = len(net.layers)
    for i, L in enumerate(net.layers):
        l = a.layers[i]
        l.kind = _KINDS[L["kind"]]
        if L["kind"] == "resblock":
            l.cin = l.cout = L["ch"]
        elif L["kind"] == "lstm":
            l.cin, l.cout = L["cin"], L["hidden"]
        else:
            l.cin, l.cout = L.get("cin", 0), L.get("cout", 0)
        l.k, l.stride, l.pad = L.get("k", 0), L.get("stride", 0), L.get("pad", 0)
        l.relu = int(bool(L.get("relu", False)))
    return a


def blob_sizes(arch):
    wb, ns = C.c_int64(), C.c_int64()
    _check(load_library().accerl_blob_sizes(C.byref(arch), C.byref(wb), C.byref(ns)))
    return wb.value, ns.value


def pack_weights(tensors):
    """tensors: blob-order list of dicts with "wq" (int8) or "w" (fp32) and "b" (fp32 or None).
    For an LSTM the pair is (W_ih with the bias, W_hh without).  Returns a uint8 array."""
    out = bytearray()

    def put(arr):
        pad = (-len(out)) % 16
        out.extend(b"\0" * pad)
        out.extend(np.ascontiguousarray(arr).tobytes())

    for t in tensors:
        if "wq" in t:
            put(np.asarray(t["wq"], np.int8))
        else:
            put(np.asarray(t["w"], np.float32))
        if t.get("b") is not None:
            put(np.asarray(t["b"], np.float32))
    return np.frombuffer(bytes(out), np.uint8)


def pack_scales(act_scales, tensors):
    parts = [np.asarray(act_scales, np.float32).reshape(-1)]
    parts += [np.asarray(t["s_w"], np.float32).reshape(-1) for t in tensors if "wq" in t]
    return np.ascontiguousarray(np.concatenate(parts))


def accerl_policy_create(arch, weights, quant_scales=None):
    """weights: uint8 numpy blob; quant_scales: float32 numpy array or None.  Returns an opaque handle."""
    lib = load_library()
    weights = np.ascontiguousarray(weights, np.uint8)
    ns, sp = 0, None
    if quant_scales is not None and len(quant_scales):
        quant_scales = np.ascontiguousarray(quant_scales, np.float32)
        ns, sp = quant_scales.size, quant_scales.ctypes.data_as(C.c_void_p)
    h = C.c_void_p()
    _check(lib.accerl_policy_create(C.byref(arch), weights.ctypes.data_as(C.c_void_p), weights.size, sp, ns, C.byref(h)))
    return h


def accerl_plan_describe(arch, weights, quant_scales=None):
    """Text description of the launch plan (host only, no GPU needed)."""
    lib = load_library()
    weights = np.ascontiguousarray(weights, np.uint8)
    ns, sp = 0, None
    if quant_scales is not None and len(quant_scales):
        quant_scales = np.ascontiguousarray(quant_scales, np.float32)
        ns, sp = quant_scales.size, quant_scales.ctypes.data_as(C.c_void_p)
    buf = C.create_string_buffer(1 << 16)
    _check(lib.accerl_plan_describe(C.byref(arch), weights.ctypes.data_as(C.c_void_p), weights.size, sp, ns, buf, len(buf)))
    return buf.value.decode()


def accerl_policy_destroy(handle):
    load_library().accerl_policy_destroy(handle)


# Marshalling is most of what a small call costs the host (32 states of the 64-unit MLP, time between calls: 5.8 us through ctypes from
# the code below, 3.6 through accerl_args; the kernel takes 2.5).  A policy's forwards, V-trace and the KL indicators go through
# accerl_args and come here where it returns None, because an argument is not a plain tensor: an error to raise, a subclass of torch.Tensor,
# a stream object.  The mixture and the distillation loss always come here.  DenseInt8 and PolicyLoss go through accerl_args, which makes their
# outputs too, on the current stream.
def _ptr(t, dtype=None):
    if t is None:
        return None
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("device tensors must be contiguous CUDA/HIP tensors")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"expected {dtype}, got {t.dtype}")
    return t.data_ptr()


def _stream(stream):
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def accerl_actor_forward(handle, states, uniforms, out_logits, out_value, out_action, stream=None):
    rc = (_args or _loaded()).forward(handle, states, uniforms, out_logits, out_value, out_action, stream)
    if rc is not None:
        if rc:
            _check(rc)
        return
    B = states.shape[0]
    _check(load_library().accerl_actor_forward(handle, _ptr(states), B, _ptr(uniforms, torch.float32),
                                               _ptr(out_logits, torch.float32), _ptr(out_value, torch.float32),
                                               _ptr(out_action, torch.int32), _stream(stream)))


def accerl_actor_forward_teacher(handle, states, uniforms, out_logits, out_value, out_action, stream=None):
    rc = (_args or _loaded()).forward_teacher(handle, states, uniforms, out_logits, out_value, out_action, stream)
    if rc is not None:
        if rc:
            _check(rc)
        return
    B = states.shape[0]
    _check(load_library().accerl_actor_forward_teacher(handle, _ptr(states), B, _ptr(uniforms, torch.float32),
                                                       _ptr(out_logits, torch.float32), _ptr(out_value, torch.float32),
                                                       _ptr(out_action, torch.int32), _stream(stream)))


def accerl_actor_forward_recurrent(handle, states, uniforms, done, h, c, out_logits, out_value, out_action, stream=None):
    rc = (_args or _loaded()).forward_recurrent(handle, states, uniforms, done, h, c, out_logits, out_value, out_action, stream)
    if rc is not None:
        if rc:
            _check(rc)
        return
    B = states.shape[0]
    _check(load_library().accerl_actor_forward_recurrent(
        handle, _ptr(states), B, _ptr(uniforms, torch.float32), _ptr(done, torch.uint8), _ptr(h, torch.float32),
        _ptr(c, torch.float32), _ptr(out_logits, torch.float32), _ptr(out_value, torch.float32),
        _ptr(out_action, torch.int32), _stream(stream)))


def accerl_actor_forward_debug(handle, states, layer, tap, out, stream=None):
    B = states.shape[0]
    _check(load_library().accerl_actor_forward_debug(handle, _ptr(states), B, int(layer), int(tap), _ptr(out),
                                                     out.numel() * out.element_size(), _stream(stream)))


def accerl_actor_forward_mixture(smaller, original, states, uniforms, use_smaller, out_logits, out_value, out_action, stream=None):
    """use_smaller: host uint8 array [B] (numpy); the other tensors live on the device."""
    import numpy as np
    B = states.shape[0]
    flags = np.ascontiguousarray(use_smaller, dtype=np.uint8)
    if flags.shape != (B,):
        raise ValueError("use_smaller must be a host array of B flags")
    _check(load_library().accerl_actor_forward_mixture(smaller, original, _ptr(states), B, _ptr(uniforms, torch.float32),
                                                       flags.ctypes.data_as(C.c_void_p), _ptr(out_logits, torch.float32),
                                                       _ptr(out_value, torch.float32), _ptr(out_action, torch.int32),
                                                       _stream(stream)))


def accerl_mixture_alpha(kl_mean, kl_lo, kl_hi):
    return float(load_library().accerl_mixture_alpha(kl_mean, kl_lo, kl_hi))


def accerl_probe_mfma(bf16, iters, sink, stream=None):
    import torch
    _check(load_library().accerl_probe_mfma(int(bool(bf16)), int(iters), _ptr(sink, torch.int32), _stream(stream)))


def accerl_probe_copy(src, dst, stream=None):
    n = src.numel() * src.element_size()
    _check(load_library().accerl_probe_copy(_ptr(src), _ptr(dst), n, _stream(stream)))


def accerl_probe_empty(stream=None):
    _check(load_library().accerl_probe_empty(_stream(stream)))


def accerl_monitor_kl(logits_original, logits_smaller, out_kl, out_entropy, out_stats, stream=None):
    """out_stats: float64 device tensor [4] = KL mean, KL max, KL variance, entropy mean."""
    rc = (_args or _loaded()).monitor_kl(logits_original, logits_smaller, out_kl, out_entropy, out_stats, stream)
    if rc is not None:
        if rc:
            _check(rc)
        return
    import torch
    B, A = logits_original.shape
    if tuple(logits_smaller.shape) != (B, A):
        raise ValueError("logit tables differ in shape")
    _check(load_library().accerl_monitor_kl(_ptr(logits_original, torch.float32), _ptr(logits_smaller, torch.float32), B, A,
                                            _ptr(out_kl, torch.float32), _ptr(out_entropy, torch.float32),
                                            _ptr(out_stats, torch.float64), _stream(stream)))


def accerl_monitor_kl_noalloc(logits_original, logits_smaller, out_kl, out_entropy, out_stats, stream=None):
    """accerl_monitor_kl on the library's fixed partial-sum array: no device allocation, at most 2^24 rows."""
    rc = (_args or _loaded()).monitor_kl_noalloc(logits_original, logits_smaller, out_kl, out_entropy, out_stats, stream)
    if rc is not None:
        if rc:
            _check(rc)
        return
    import torch
    B, A = logits_original.shape
    if tuple(logits_smaller.shape) != (B, A):
        raise ValueError("logit tables differ in shape")
    _check(load_library().accerl_monitor_kl_noalloc(_ptr(logits_original, torch.float32), _ptr(logits_smaller, torch.float32), B, A,
                                                    _ptr(out_kl, torch.float32), _ptr(out_entropy, torch.float32),
                                                    _ptr(out_stats, torch.float64), _stream(stream)))


def accerl_distill_loss(logits_original, logits_smaller, value_original, value_smaller, beta, out_loss, out_mean, stream=None):
    import torch
    B, A = logits_original.shape
    if tuple(logits_smaller.shape) != (B, A) or tuple(value_original.shape) != (B,) or tuple(value_smaller.shape) != (B,):
        raise ValueError("shapes differ")
    _check(load_library().accerl_distill_loss(_ptr(logits_original, torch.float32), _ptr(logits_smaller, torch.float32),
                                              _ptr(value_original, torch.float32), _ptr(value_smaller, torch.float32), B, A,
                                              float(beta), _ptr(out_loss, torch.float32), _ptr(out_mean, torch.float64),
                                              _stream(stream)))


def accerl_vtrace(logits_original, logits_smaller, actions, rewards, discounts, values, bootstrap,
                  rho_bar, c_bar, out_vs, out_pg_adv, out_rho, stream=None):
    rc = (_args or _loaded()).vtrace(logits_original, logits_smaller, actions, rewards, discounts, values, bootstrap, rho_bar, c_bar, out_vs, out_pg_adv, out_rho, stream)
    if rc is not None:
        if rc:
            _check(rc)
        return
    import torch
    T, B, A = logits_original.shape
    if tuple(logits_smaller.shape) != (T, B, A):
        raise ValueError("logit tables differ in shape")
    for t in (actions, rewards, discounts, values, out_vs, out_rho):
        if tuple(t.shape) != (T, B):
            raise ValueError("per-step tensors must be [T, B]")
    _check(load_library().accerl_vtrace(_ptr(logits_original, torch.float32), _ptr(logits_smaller, torch.float32),
                                        _ptr(actions, torch.int32), _ptr(rewards, torch.float32), _ptr(discounts, torch.float32),
                                        _ptr(values, torch.float32), _ptr(bootstrap, torch.float32), T, B, A,
                                        float(rho_bar), float(c_bar), _ptr(out_vs, torch.float32),
                                        _ptr(out_pg_adv, torch.float32), _ptr(out_rho, torch.float32), _stream(stream)))


# ---------------------------------------------------------------- operators of wide policies
KL_KINDS = {"none": 0, "sampled": 1, "forward": 2, "reverse": 3}


def _dtype(t):
    try:
        return {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}[t.dtype]
    except KeyError:
        raise ValueError(f"expected float32, bfloat16 or float16, got {t.dtype}") from None


_SAME = contextlib.nullcontext()


def _device_of(*tensors):
    """The device that all of them lie on (the first is no None), as a context: kernels are launched on the current one."""
    at = tensors[0].get_device()                     # (-1 on the host)
    for t in tensors:
        if t is not None and t.get_device() != at:
            raise ValueError(f"tensors of one call lie on different devices: {tensors[0].device} and {t.device}")
    return _SAME if at < 0 or at == torch._C._cuda_getDevice() else torch.cuda.device(at)


def _rows(t, what):
    """Pointer and row stride of a device matrix whose rows are contiguous."""
    if t is None:
        return None, 0
    if not t.is_cuda or t.dim() != 2:
        raise ValueError(f"{what} must be a CUDA/HIP matrix")
    rows, cols = t.shape
    ld = t.stride(0) if rows > 1 else cols
    if (cols > 1 and t.stride(1) != 1) or ld < cols:
        raise ValueError(f"the rows of {what} must be contiguous and must not overlap")
    return t.data_ptr(), ld


def _vector(t, dtype, n, what):
    if t is None:
        return None
    if tuple(t.shape) != (n,):
        raise ValueError(f"{what} must be a vector of {n}")
    return _ptr(t, dtype)


def _packed(t, rows, cols, what):
    if t.numel() * t.element_size() < packed_rows_bytes(rows, cols):
        raise ValueError(f"{what} is smaller than the packed rows of {rows} x {cols}")
    return _ptr(t, torch.int8)


def _count(n):
    if n < 0:
        _check(n)
    return n


def packed_rows_bytes(rows, cols):
    """Size of the buffer of accerl_quantize_rows and accerl_pack_rows_i8 (a flat int8 tensor)."""
    return _count(load_library().accerl_packed_rows_bytes(rows, cols))


def accerl_quantize_rows(x, out_packed, out_scale, stream=None):
    lib = load_library()
    p, ld = _rows(x, "x")
    R, K = x.shape
    with _device_of(x, out_packed, out_scale):
        _check(lib.accerl_quantize_rows(p, _dtype(x), R, K, ld, _packed(out_packed, R, K, "out_packed"), _vector(out_scale, torch.float32, R, "out_scale"),
                                        _stream(stream)))


def accerl_pack_rows_i8(q, out_packed, stream=None):
    lib = load_library()
    if q.dtype != torch.int8:
        raise ValueError(f"expected torch.int8, got {q.dtype}")
    p, ld = _rows(q, "q")
    R, K = q.shape
    with _device_of(q, out_packed):
        _check(lib.accerl_pack_rows_i8(p, R, K, ld, _packed(out_packed, R, K, "out_packed"), _stream(stream)))


def accerl_unpack_rows_i8(packed, out_q, stream=None):
    lib = load_library()
    if out_q.dtype != torch.int8:
        raise ValueError(f"expected torch.int8, got {out_q.dtype}")
    p, ld = _rows(out_q, "out_q")
    R, K = out_q.shape
    with _device_of(packed, out_q):
        _check(lib.accerl_unpack_rows_i8(_packed(packed, R, K, "packed"), R, K, p, ld, _stream(stream)))


def accerl_dense_i8(x_packed, x_scale, w_packed, w_scale, bias, K, out, relu=False, stream=None):
    """out [M, N] from packed tokens [M, K] and packed features [N, K]."""
    lib = load_library()
    po, ld = _rows(out, "out")
    M, N = out.shape
    with _device_of(x_packed, x_scale, w_packed, w_scale, bias, out):
        _check(lib.accerl_dense_i8(_packed(x_packed, M, K, "x_packed"), _vector(x_scale, torch.float32, M, "x_scale"), _packed(w_packed, N, K, "w_packed"),
                                   _vector(w_scale, torch.float32, N, "w_scale"), _vector(bias, torch.float32, N, "bias"), M, N, K, int(bool(relu)),
                                   po, _dtype(out), ld, _stream(stream)))


def accerl_dense_i8_workspace(M, K):
    return _count(load_library().accerl_dense_i8_workspace(M, K))


def accerl_dense_i8_dynamic(x, w_packed, w_scale, bias, out, workspace, relu=False, stream=None):
    """out [M, N] from floating-point tokens x [M, K]; workspace: uint8 tensor of accerl_dense_i8_workspace(M, K) bytes."""
    lib = load_library()
    px, ldx = _rows(x, "x")
    po, ld = _rows(out, "out")
    (M, K), N = x.shape, out.shape[1]
    if out.shape[0] != M:
        raise ValueError("x and out differ in rows")
    with _device_of(x, w_packed, w_scale, bias, out, workspace):
        _check(lib.accerl_dense_i8_dynamic(px, _dtype(x), ldx, _packed(w_packed, N, K, "w_packed"), _vector(w_scale, torch.float32, N, "w_scale"),
                                           _vector(bias, torch.float32, N, "bias"), M, N, K, int(bool(relu)), po, _dtype(out), ld,
                                           _ptr(workspace, torch.uint8), workspace.numel(), _stream(stream)))


def accerl_policy_loss_workspace():
    return load_library().accerl_policy_loss_workspace()


def _mask_rows(mask, B, A):
    """uint8 [B, A], or [1, A] for all rows."""
    if mask is None:
        return None, 0
    if mask.dtype != torch.uint8:
        raise ValueError(f"expected torch.uint8, got {mask.dtype}")
    if mask.dim() != 2 or mask.shape[1] != A or mask.shape[0] not in (1, B):
        raise ValueError("the mask must be [B, A] or [1, A]")
    p, ld = _rows(mask, "mask")
    return p, 0 if mask.shape[0] == 1 else ld


def accerl_action_logprob(logits, mask, actions, out_logp, out_entropy, workspace, stream=None):
    """mask: uint8 [B, A], [1, A] for all rows, or None; workspace: uint8 tensor of accerl_policy_loss_workspace() bytes."""
    lib = load_library()
    p, ld = _rows(logits, "logits")
    B, A = logits.shape
    pm, ldm = _mask_rows(mask, B, A)
    with _device_of(logits, mask, actions, out_logp, out_entropy, workspace):
        _check(lib.accerl_action_logprob(p, _dtype(logits), ld, pm, ldm, _vector(actions, torch.int32, B, "actions"), B, A,
                                         _vector(out_logp, torch.float32, B, "out_logp"), _vector(out_entropy, torch.float32, B, "out_entropy"),
                                         _ptr(workspace, torch.uint8), workspace.numel(), _stream(stream)))


def accerl_policy_loss(logits, actions, old_logp, advantages, workspace, mask=None, weights=None, kl="none", ref_logits=None, ref_logp=None,
                       clip_low=0.2, clip_high=0.2, kl_coef=0.0, entropy_coef=0.0, scale=1.0, grad_logits=None, out_loss=None, out_logp=None,
                       out_kl=None, out_entropy=None, out_stats=None, stream=None):
    """kl: "none", "sampled" (ref_logp), "forward" or "reverse" (ref_logits).  Every output may be None."""
    lib = load_library()
    B, A = logits.shape
    for t, what in ((ref_logits, "ref_logits"), (grad_logits, "grad_logits")):
        if t is not None and (t.shape != logits.shape or t.dtype != logits.dtype):
            raise ValueError(f"{what} differs from the logits in shape or type")
    a = _PolicyLossArgs()
    a.B, a.A, a.dtype, a.kl_kind = B, A, _dtype(logits), KL_KINDS[kl] if isinstance(kl, str) else int(kl)
    a.logits, a.ld_logits = _rows(logits, "logits")
    a.ref_logits, a.ld_ref = _rows(ref_logits, "ref_logits")
    a.grad_logits, a.ld_grad = _rows(grad_logits, "grad_logits")
    a.mask, a.ld_mask = _mask_rows(mask, B, A)
    a.actions = _vector(actions, torch.int32, B, "actions")
    for n, t in (("old_logp", old_logp), ("advantages", advantages), ("weights", weights), ("ref_logp", ref_logp), ("out_loss", out_loss),
                 ("out_logp", out_logp), ("out_kl", out_kl), ("out_entropy", out_entropy)):
        setattr(a, n, _vector(t, torch.float32, B, n))
    a.out_stats = _vector(out_stats, torch.float32, 4, "out_stats")
    a.clip_low, a.clip_high, a.kl_coef, a.entropy_coef, a.scale = clip_low, clip_high, kl_coef, entropy_coef, scale
    a.workspace, a.workspace_bytes = _ptr(workspace, torch.uint8), workspace.numel()
    with _device_of(logits, actions, old_logp, advantages, workspace, mask, weights, ref_logits, ref_logp, grad_logits, out_loss, out_logp, out_kl, out_entropy, out_stats):
        _check(lib.accerl_policy_loss(C.byref(a), _stream(stream)))


_CODES = {None: -1}         # output types of accerl_args, filled by load_library


def _logits(t):
    if not t.is_cuda or t.dim() != 2:
        raise ValueError("logits must be a CUDA/HIP matrix")
    return t.detach()


def _captured(stream):
    """Whether what the current stream, this one, is given now goes into a graph (0.3 us; the default stream, 0, cannot be captured)."""
    return stream != 0 and torch._C._cuda_isCurrentStreamCapturing()


class _Workspaces:
    """A buffer for each thread and stream, allocated on the stream: a call is several launches that meet in it, and another thread's may come
    between them.  A buffer that grows is given back in the order of the stream that used it, and so are a thread's when it ends.  A call that
    torch.cuda.graph captures gets one of the graph's own memory, as its outputs do: no other graph, no eager call and nothing that is allocated
    later has it."""

    def __init__(self):
        self._own = threading.local()

    def __reduce__(self):
        return _Workspaces, ()                # a copy begins with none

    def kept(self, stream, index):
        """What this thread has on a stream of the device of this index, or None."""
        return self._own.__dict__.get((index, stream)) if stream == 0 or not _captured(stream) else None

    def get(self, nbytes, stream, device):
        t = self.kept(stream, device.index)
        if t is None or t.numel() < nbytes:
            t = torch.empty(nbytes, dtype=torch.uint8, device=device)
            if not _captured(stream):
                self._own.__dict__[device.index, stream] = t
        return t


class _On:
    """The stream that a call runs on, and its device: what is allocated inside belongs to it."""

    def __init__(self, stream, device):
        self.other = None
        if stream is None:
            self.raw = torch._C._cuda_getCurrentRawStream(device.index)
            if device.index != torch._C._cuda_getDevice():
                self.other = torch.cuda.device(device)
        else:
            s = stream if isinstance(stream, torch.cuda.Stream) else torch.cuda.ExternalStream(int(stream), device=device)
            if s.device != device:
                raise ValueError(f"the stream is one of {s.device}, the tensors lie on {device}")
            self.raw, self.other = s.cuda_stream, torch.cuda.stream(s)

    def __enter__(self):
        if self.other is not None:
            self.other.__enter__()
        return self.raw

    def __exit__(self, *e):
        if self.other is not None:
            self.other.__exit__(*e)


class DenseInt8:
    """Int8 dense layer with a scale for each token and channel: owner of packed weights, workspaces and outputs.

    w: int8 [N, K] with w_scale [N], or a float matrix that is quantised here, a scale for each row; bias [N] or None.  Threads and streams may
    share a layer: each has a workspace of its own in it (accerl_dense_i8_workspace bytes, for as long as the thread and the layer live).
    """

    def __init__(self, w, w_scale=None, bias=None, relu=False):
        load_library()
        self.N, self.K = w.shape
        if bias is not None and tuple(bias.shape) != (self.N,):
            raise ValueError(f"the bias must be a vector of {self.N}")
        self.relu = bool(relu)
        self._relu = int(self.relu)
        self.w = torch.empty(packed_rows_bytes(self.N, self.K), dtype=torch.int8, device=w.device)
        self.w_scale = torch.empty(self.N, dtype=torch.float32, device=w.device)
        self.bias = None if bias is None else bias.detach().to(w.device, torch.float32, copy=True).contiguous()
        self._work = _Workspaces()
        self.update(w, w_scale)

    def update(self, w, w_scale=None, bias=None):
        """New weights of the same shape (a learner's, after its step), and bias if given, on the current stream.  Forwards of other streams or
        threads that are not ordered with it may see some of both."""
        if tuple(w.shape) != (self.N, self.K) or (bias is not None and (self.bias is None or bias.shape != self.bias.shape)):
            raise ValueError("the weights or the bias differ in shape from the layer's")
        if w.dtype == torch.int8:
            if w_scale is None or tuple(w_scale.shape) != (self.N,):
                raise ValueError(f"int8 weights need a vector of {self.N} scales")
            self.w_scale.copy_(w_scale.detach())
            accerl_pack_rows_i8(w, self.w)
        elif w_scale is not None:
            raise ValueError("scales belong to int8 weights; a float matrix is quantised with scales of its own")
        else:
            accerl_quantize_rows(w.detach(), self.w, self.w_scale)
        if bias is not None:
            self.bias.copy_(bias.detach())

    def forward(self, x, dtype=None, out=None, stream=None):
        """x [M, K] -> [M, N] in `dtype` (x's own if None)."""
        if stream is None and out is None and x.is_cuda:
            at = x.get_device()
            raw = torch._C._cuda_getCurrentRawStream(at)
            ws = self._work.kept(raw, at)
            r = None if ws is None else (_args or _loaded()).dense_dynamic(x, self.N, self.K, self.w, self.w_scale, self.bias, self._relu, _CODES.get(dtype, 3),
                                                                           ws, raw)
            if r is not None:
                if r[0]:
                    _check(r[0])
                return r[1]
        if not x.is_cuda or x.dim() != 2 or x.shape[1] != self.K:
            raise ValueError(f"x must be a CUDA/HIP matrix of {self.K} columns")
        if out is not None and tuple(out.shape) != (x.shape[0], self.N):
            raise ValueError(f"out must be [{x.shape[0]}, {self.N}]")
        M = x.shape[0]
        with _On(stream, x.device) as raw:
            if out is None:
                out = torch.empty((M, self.N), dtype=x.dtype if dtype is None else dtype, device=x.device)
            ws = self._work.get(accerl_dense_i8_workspace(M, self.K), raw, x.device)
            accerl_dense_i8_dynamic(x, self.w, self.w_scale, self.bias, out, ws, self.relu, raw)
        return out


class PolicyLoss:
    """Clipped policy loss with KL and entropy terms: owner of the coefficients, workspaces and outputs.

    forward returns the per-row outputs, the batch's sums and the gradient by the logits: `logits.backward(r.grad)` continues it into
    whatever made the logits.  Threads and streams may share one, as they may a DenseInt8.
    """

    class Result:
        __slots__ = ("loss", "logp", "kl", "entropy", "stats", "grad")

    def __init__(self, clip_low=0.2, clip_high=0.2, kl="none", kl_coef=0.0, entropy_coef=0.0):
        load_library()
        self.how = dict(clip_low=clip_low, clip_high=clip_high, kl=kl, kl_coef=kl_coef, entropy_coef=entropy_coef)
        self._how = (KL_KINDS[kl], float(clip_low), float(clip_high), float(kl_coef), float(entropy_coef))
        self._bytes = accerl_policy_loss_workspace()
        self._work = _Workspaces()

    def forward(self, logits, actions, old_logp, advantages, mask=None, weights=None, scale=None, ref_logits=None, ref_logp=None,
                grad=True, stream=None):
        """scale: None for the mean over all rows; grad: a table to write the gradient to (the logits themselves too), True for a new one,
        False for the value only."""
        if stream is None and (grad is True or grad is False) and logits.is_cuda:
            at = logits.get_device()
            raw = torch._C._cuda_getCurrentRawStream(at)
            ws = self._work.kept(raw, at)
            t = (_args or _loaded()).policy_loss(logits, actions, old_logp, advantages, mask, weights, ref_logits, ref_logp, int(grad), *self._how,
                                                 1.0 / max(1, logits.shape[0]) if scale is None else float(scale),
                                                 self._work.get(self._bytes, raw, logits.device) if ws is None else ws, raw)
            if t is not None:
                if t[0]:
                    _check(t[0])
                r = self.Result()
                _, r.loss, r.logp, r.kl, r.entropy, r.stats, *g = t
                r.grad = g[0] if grad else None
                return r
        logits = _logits(logits)
        B = logits.shape[0]
        r = self.Result()
        with _On(stream, logits.device) as raw:
            rows = torch.empty((4, B), dtype=torch.float32, device=logits.device)
            r.loss, r.logp, r.kl, r.entropy = rows.unbind(0)
            r.stats = torch.empty(4, dtype=torch.float32, device=logits.device) if B else torch.zeros(4, dtype=torch.float32, device=logits.device)
            r.grad = torch.empty(logits.shape, dtype=logits.dtype, device=logits.device) if grad is True else None if grad is False else grad
            accerl_policy_loss(logits, actions, old_logp, advantages, self._work.get(self._bytes, raw, logits.device), mask=mask, weights=weights,
                               ref_logits=ref_logits, ref_logp=ref_logp, scale=1.0 / max(1, B) if scale is None else scale, grad_logits=r.grad,
                               out_loss=r.loss, out_logp=r.logp, out_kl=r.kl, out_entropy=r.entropy, out_stats=r.stats, stream=raw, **self.how)
        return r

    def logprob(self, logits, actions, mask=None, stream=None):
        """log pi(a) and entropy, each [B]."""
        if stream is None and logits.is_cuda:
            at = logits.get_device()
            raw = torch._C._cuda_getCurrentRawStream(at)
            ws = self._work.kept(raw, at)
            t = (_args or _loaded()).action_logprob(logits, actions, mask, self._work.get(self._bytes, raw, logits.device) if ws is None else ws, raw)
            if t is not None:
                if t[0]:
                    _check(t[0])
                return t[1], t[2]
        logits = _logits(logits)
        with _On(stream, logits.device) as raw:
            logp, ent = torch.empty((2, logits.shape[0]), dtype=torch.float32, device=logits.device).unbind(0)
            accerl_action_logprob(logits, mask, actions, logp, ent, self._work.get(self._bytes, raw, logits.device), raw)
        return logp, ent


STEP_KINDS = ("mlp_fused", "quant_obs", "conv", "gemm", "gemm_f32", "maxpool", "lstm_pack", "sample", "heads")


def accerl_profile_begin(handle):
    _check(load_library().accerl_profile_begin(handle))


def accerl_profile_end(handle):
    """Returns a list of dicts: step, layer, kind, launches, total_ms."""
    cap = 256
    n = C.c_int32()
    ms = (C.c_float * cap)()
    cnt = (C.c_int64 * cap)()
    layer = (C.c_int32 * cap)()
    kind = (C.c_int32 * cap)()
    _check(load_library().accerl_profile_end(handle, cap, C.byref(n), ms, cnt, layer, kind))
    return [dict(step=i, layer=layer[i], kind=STEP_KINDS[kind[i]], launches=cnt[i], total_ms=ms[i])
            for i in range(n.value)]


class Policy:
    """Convenience owner of a policy handle plus output allocation through torch."""

    def __init__(self, net, precision, tensors, act_scales=None):
        self.net = net
        self.precision = precision
        self.arch = make_arch(net, precision)
        blob = pack_weights(tensors)
        scales = pack_scales(act_scales, tensors) if precision == "int8" else None
        self.handle = accerl_policy_create(self.arch, blob, scales)
        self.recurrent = any(L["kind"] == "lstm" for L in net.layers)

    def close(self):
        if self.handle is not None:
            accerl_policy_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def alloc_outputs(self, B, device="cuda"):
        import torch
        A = self.net.n_actions
        return (torch.empty((B, A), dtype=torch.float32, device=device),
                torch.empty((B,), dtype=torch.float32, device=device),
                torch.empty((B,), dtype=torch.int32, device=device))

    def forward(self, states, uniforms, done=None, h=None, c=None, outputs=None, stream=None):
        logits, value, action = outputs if outputs is not None else self.alloc_outputs(states.shape[0], states.device)
        if self.recurrent:
            accerl_actor_forward_recurrent(self.handle, states, uniforms, done, h, c, logits, value, action, stream)
        elif self.precision == "int8":
            accerl_actor_forward(self.handle, states, uniforms, logits, value, action, stream)
        else:
            accerl_actor_forward_teacher(self.handle, states, uniforms, logits, value, action, stream)
        return logits, value, action

    def tap(self, states, layer, tap, shape, dtype, stream=None):
        import torch
        out = torch.empty(shape, dtype=dtype, device=states.device)
        accerl_actor_forward_debug(self.handle, states, layer, tap, out, stream)
        return out
