"""ctypes binding of libprism.so (see include/prism.h).  Argument marshalling only: every
step of the path runs in the HIP kernels.  PyTorch supplies device memory and the stream.

The library must have been built (python -m paper_2601_22137_amd.build); there is no fallback.
"""
import collections
import ctypes
import os
import struct

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libprism.so")

F32, BF16 = 0, 1
FN_POLAR, FN_SQRT, FN_INV_ROOT, FN_SIGN, FN_INVERSE, FN_SQRT_NEWTON = 1, 2, 3, 4, 5, 6
MAX_ITERS = 64
FLAG_BF16_PLAIN_ITERATE = 1
FLAG_SHARED_GPU = 2
FLAG_SINGLE_STREAM = 4
FLAG_FIT_NO_WAIT = 8
OK, EINVAL, EUNSUPPORTED, ENOMEM, EHIP = 0, 1, 2, 3, 4
INFO_CONVERGED, INFO_BUDGET, INFO_NONFINITE, INFO_ZERO, INFO_DIVERGED = 0, 1, 2, 3, 4

INFO_DTYPE = np.dtype([("iters", np.int32), ("status", np.int32),
                       ("residual", np.float32, (MAX_ITERS + 1,)), ("alpha", np.float32, (MAX_ITERS,))])

EXPORTS = ("prism_workspace_bytes", "prism_release_workspaces", "prism_polar", "prism_polar_ex", "prism_polar_static", "prism_sqrt", "prism_sqrt_ex",
           "prism_inv_root", "prism_inv_root_ex", "prism_sign", "prism_sign_ex", "prism_inverse", "prism_inverse_ex", "prism_sqrt_newton", "prism_sqrt_newton_ex", "prism_spd_inverse", "prism_run_grouped", "prism_run_grouped_from",
           "prism_dropout", "prism_qk_norm_rope", "prism_qk_norm_rope_backward", "prism_norm_rope_workspace_bytes",
           "prism_attention", "prism_attention_backward", "prism_attention_workspace_bytes",
           "prism_embedding", "prism_embedding_backward", "prism_embedding_workspace_bytes",
           "prism_layer_norm", "prism_layer_norm_backward", "prism_layer_norm_workspace_bytes",
           "prism_token_logprob", "prism_token_logprob_backward", "prism_policy_loss", "prism_policy_loss_workspace_bytes",
           "prism_sketch", "prism_gauss_parts", "prism_chain_product", "prism_chain_product_bf16", "prism_gemm_f32", "prism_gemm_f32_planes",
           "prism_gemm_f64a", "prism_gemm_bf16_nt", "prism_profile_enable", "prism_profile_collect",
           "prism_last_error")

PROFILE_KINDS = ("prep", "final", "sketch", "chain", "solve", "f32_resid", "f32_polyq", "f32_apply", "f32_store",
                 "f64_mnext", "make_t", "bf16_gram", "bf16_polyq", "bf16_apply", "bf16_store", "spd_inverse", "db_moments",
                 "db_update_m", "f32_small_polar", "moments", "fit_square", "flow", "small_root",
                 "dropout", "norm_rope", "norm_rope_backward", "attention", "attention_join", "attention_docs", "attention_dq", "attention_dkv",
                 "embedding", "embedding_sort", "embedding_backward", "layer_norm", "layer_norm_backward", "logprob", "logprob_backward", "policy_loss", "loss_sum")


class Options(ctypes.Structure):
    _fields_ = [("flags", ctypes.c_uint32), ("warm_iters", ctypes.c_int32), ("workspace", ctypes.c_void_p),
                ("workspace_bytes", ctypes.c_size_t), ("info", ctypes.c_void_p),
                ("alpha_schedule", ctypes.POINTER(ctypes.c_float)), ("schedule_len", ctypes.c_int32)]


class Group(ctypes.Structure):
    _fields_ = [("x", ctypes.c_void_p), ("inv_out", ctypes.c_void_p), ("info", ctypes.c_void_p),
                ("batch", ctypes.c_int32), ("m", ctypes.c_int32), ("n", ctypes.c_int32)]


class Strides(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int64), ("token", ctypes.c_int64), ("head", ctypes.c_int64)]


class NormRopeDesc(ctypes.Structure):
    _fields_ = ([(f, ctypes.c_int32) for f in ("batch", "len", "q_heads", "k_heads", "head_dim", "rot_dim", "norm", "interleaved", "start")]
                + [("eps", ctypes.c_float), ("scale", ctypes.c_float)]
                + [(f, ctypes.c_void_p) for f in ("positions", "inv_freq", "q_weight", "k_weight")]
                + [(f, Strides) for f in ("q", "k", "q_out", "k_out", "dq", "dk")]
                + [("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t)])


class AttentionDesc(ctypes.Structure):
    _fields_ = ([(f, ctypes.c_int32) for f in ("batch", "q_len", "k_len", "q_heads", "k_heads", "head_dim", "causal")]
                + [("scale", ctypes.c_float), ("softcap", ctypes.c_float)]
                + [(f, ctypes.c_void_p) for f in ("slopes", "prefix", "k_lens", "q_doc", "k_doc")]
                + [(f, Strides) for f in ("q", "k", "v", "out", "dout", "dq", "dk", "dv")]
                + [("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t)])


class EmbeddingDesc(ctypes.Structure):
    _fields_ = [("count", ctypes.c_int64), ("rows", ctypes.c_int64), ("width", ctypes.c_int32), ("wide_tokens", ctypes.c_int32), ("scale", ctypes.c_float),
                ("table_stride", ctypes.c_int64), ("out_stride", ctypes.c_int64), ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t)]


class LayerNormDesc(ctypes.Structure):
    _fields_ = ([("rows", ctypes.c_int64), ("width", ctypes.c_int32), ("center", ctypes.c_int32), ("eps", ctypes.c_float)]
                + [(f, ctypes.c_int64) for f in ("x", "residual", "total", "y", "dy", "dtotal", "dx")]
                + [("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t)])


class LogitsDesc(ctypes.Structure):
    _fields_ = ([("rows", ctypes.c_int64), ("vocabulary", ctypes.c_int32), ("wide_tokens", ctypes.c_int32), ("scale", ctypes.c_double),
                 ("logits_stride", ctypes.c_int64), ("dlogits_stride", ctypes.c_int64)]
                + [(f, ctypes.c_double) for f in ("clip_low", "clip_high", "kl")]
                + [(f, ctypes.c_void_p) for f in ("advantages", "old_logp", "ref_logp", "weights", "workspace")] + [("workspace_bytes", ctypes.c_size_t)])


class PrismError(RuntimeError):
    pass


_lib = None


def lib():
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise PrismError("libprism.so is not built: run `python -m paper_2601_22137_amd.build`")
        L = ctypes.CDLL(LIB_PATH)
        vp, i, u64, dbl = ctypes.c_void_p, ctypes.c_int, ctypes.c_uint64, ctypes.c_double
        L.prism_last_error.restype = ctypes.c_char_p
        L.prism_workspace_bytes.argtypes = [i, i, i, i, i, i, i, i, ctypes.POINTER(ctypes.c_size_t)]
        L.prism_polar.argtypes = [vp, i, i, i, i, i, i, i, u64, dbl, vp]
        L.prism_polar_ex.argtypes = L.prism_polar.argtypes + [ctypes.POINTER(Options)]
        L.prism_polar_static.argtypes = L.prism_polar_ex.argtypes
        L.prism_sqrt.argtypes = [vp, vp, i, i, i, i, i, i, i, u64, dbl, vp]
        L.prism_sqrt_ex.argtypes = L.prism_sqrt.argtypes + [ctypes.POINTER(Options)]
        L.prism_inv_root.argtypes = [vp, i, i, i, i, i, i, i, i, u64, dbl, vp]
        L.prism_inv_root_ex.argtypes = L.prism_inv_root.argtypes + [ctypes.POINTER(Options)]
        L.prism_sign.argtypes = [vp, i, i, i, i, i, i, i, u64, dbl, vp]
        L.prism_sign_ex.argtypes = L.prism_sign.argtypes + [ctypes.POINTER(Options)]
        L.prism_inverse.argtypes = [vp, i, i, i, i, i, i, u64, dbl, vp]
        L.prism_inverse_ex.argtypes = L.prism_inverse.argtypes + [ctypes.POINTER(Options)]
        L.prism_sqrt_newton.argtypes = [vp, vp, i, i, i, i, i, i, dbl, vp]
        L.prism_sqrt_newton_ex.argtypes = L.prism_sqrt_newton.argtypes + [ctypes.POINTER(Options)]
        L.prism_spd_inverse.argtypes = [vp, vp, i, i, vp]
        L.prism_run_grouped.argtypes = [i, ctypes.POINTER(Group), i, i, i, i, i, i, u64, dbl, vp, ctypes.POINTER(Options)]
        L.prism_run_grouped_from.argtypes = [i, ctypes.POINTER(Group), vp, i, i, i, i, i, i, u64, dbl, vp, ctypes.POINTER(Options)]
        L.prism_dropout.argtypes = [vp, vp, vp, ctypes.c_int64, i, dbl, u64, ctypes.c_uint32, vp]
        L.prism_qk_norm_rope.argtypes = [vp, vp, vp, vp, i, vp, vp]
        L.prism_qk_norm_rope_backward.argtypes = [vp] * 8 + [i, vp, vp]
        L.prism_norm_rope_workspace_bytes.argtypes = [i, vp, ctypes.POINTER(ctypes.c_size_t)]
        L.prism_attention.argtypes = [vp] * 5 + [i, vp, vp]
        L.prism_attention_backward.argtypes = [vp] * 9 + [i, vp, vp]
        L.prism_attention_workspace_bytes.argtypes = [i, vp, i, ctypes.POINTER(ctypes.c_size_t)]
        size_p = ctypes.POINTER(ctypes.c_size_t)
        L.prism_embedding.argtypes = L.prism_embedding_backward.argtypes = [vp, vp, vp, i, vp, vp]
        L.prism_embedding_workspace_bytes.argtypes = L.prism_layer_norm_workspace_bytes.argtypes = [i, vp, size_p]
        L.prism_layer_norm.argtypes = [vp] * 7 + [i, vp, vp]
        L.prism_layer_norm_backward.argtypes = [vp] * 8 + [i, vp, vp]
        L.prism_token_logprob.argtypes = [vp] * 4 + [i, vp, vp]
        L.prism_token_logprob_backward.argtypes = [vp] * 5 + [i, vp, vp]
        L.prism_policy_loss.argtypes = [vp] * 7 + [i, vp, vp]
        L.prism_policy_loss_workspace_bytes.argtypes = [vp, size_p]
        L.prism_sketch.argtypes = [vp, i, i, u64, i, i, vp]
        L.prism_gauss_parts.argtypes = [ctypes.c_uint32, ctypes.c_uint32, vp, vp, vp, vp]
        L.prism_chain_product.argtypes = [vp, vp, vp, i, i, i, vp]
        L.prism_chain_product_bf16.argtypes = [vp, vp, vp, vp, vp, i, i, i, vp]
        L.prism_gemm_f32.argtypes = [vp, vp, vp, i, i, i, i, i, vp]
        L.prism_gemm_f32_planes.argtypes = L.prism_gemm_f32.argtypes
        L.prism_gemm_f64a.argtypes = [vp, vp, vp, i, i, i, i, vp]
        L.prism_gemm_bf16_nt.argtypes = [vp, vp, vp, i, i, i, i, i, vp]
        L.prism_profile_enable.argtypes = [i]
        L.prism_profile_collect.argtypes = [ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_longlong), i]
        _lib = L
    return _lib


def _check(rc):
    if rc != OK:
        names = {EINVAL: "PRISM_EINVAL", EUNSUPPORTED: "PRISM_EUNSUPPORTED", ENOMEM: "PRISM_ENOMEM", EHIP: "PRISM_EHIP"}
        raise PrismError("%s (%s)" % (names.get(rc, rc), lib().prism_last_error().decode()))


def _stream():
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


def _dtype_code(t):
    if t.dtype == torch.float32:
        return F32
    if t.dtype == torch.bfloat16:
        return BF16
    raise PrismError("unsupported dtype %s" % t.dtype)


def _batched(t):
    if not (t.is_cuda and t.is_contiguous() and t.dim() == 3):
        raise PrismError("expected a contiguous CUDA tensor [batch, m, n]")
    return t.shape


class _Info:
    def __init__(self, batch, device):
        self.buf = torch.empty(batch * INFO_DTYPE.itemsize, dtype=torch.uint8, device=device)

    def read(self):
        """Synchronises and returns a numpy structured array (one record per matrix)."""
        return self.buf.cpu().numpy().view(INFO_DTYPE).copy()


def _options(info, flags, warm_iters, workspace, alpha_schedule=None):
    o = Options()
    if alpha_schedule is not None and len(alpha_schedule) > 0:
        o._sched = (ctypes.c_float * len(alpha_schedule))(*[float(a) for a in alpha_schedule])   # kept alive by o
        o.alpha_schedule = ctypes.cast(o._sched, ctypes.POINTER(ctypes.c_float))
        o.schedule_len = len(alpha_schedule)
    o.flags = flags
    o.warm_iters = warm_iters
    o.workspace = workspace.data_ptr() if workspace is not None else None
    o.workspace_bytes = workspace.numel() * workspace.element_size() if workspace is not None else 0
    o.info = info.buf.data_ptr()
    return o


def workspace_bytes(fn, batch, m, n, dtype_code, degree, sketch_dim, root_p=0):
    out = ctypes.c_size_t(0)
    _check(lib().prism_workspace_bytes(fn, batch, m, n, dtype_code, degree, sketch_dim, root_p, ctypes.byref(out)))
    return out.value


def polar(x, degree=5, max_iters=30, sketch_dim=8, seed=22137, tol=1e-6, flags=0, warm_iters=0, workspace=None,
          alpha_schedule=None):
    """In place: x[batch, m, n] <- polar factor.  Returns an info handle (.read() synchronises)."""
    b, m, n = _batched(x)
    info = _Info(b, x.device)
    o = _options(info, flags, warm_iters, workspace, alpha_schedule)
    _check(lib().prism_polar_ex(x.data_ptr(), b, m, n, _dtype_code(x), degree, max_iters, sketch_dim, seed, tol,
                                _stream(), ctypes.byref(o)))
    return info


STATIC_SCRATCH_BYTES = 32 << 20


def new_info(batch, device="cuda"):
    """An info handle made ahead of time, for calls that must not allocate (polar_static)."""
    return _Info(batch, device)


def polar_static(x, degree=5, max_iters=30, sketch_dim=8, seed=22137, tol=1e-6, flags=0, warm_iters=0, info=None,
                 alpha_schedule=None):
    """polar() through the entry point that allocates nothing: the library's intermediates live in
    its static device array (STATIC_SCRATCH_BYTES; larger calls raise PRISM_EUNSUPPORTED).  `info` is
    a handle from new_info() made beforehand, or None; nothing is allocated here either."""
    b, m, n = _batched(x)
    o = Options()
    if alpha_schedule is not None and len(alpha_schedule) > 0:
        o._sched = (ctypes.c_float * len(alpha_schedule))(*[float(a) for a in alpha_schedule])
        o.alpha_schedule = ctypes.cast(o._sched, ctypes.POINTER(ctypes.c_float))
        o.schedule_len = len(alpha_schedule)
    o.flags = flags
    o.warm_iters = warm_iters
    o.info = info.buf.data_ptr() if info is not None else None
    _check(lib().prism_polar_static(x.data_ptr(), b, m, n, _dtype_code(x), degree, max_iters, sketch_dim, seed, tol,
                                    _stream(), ctypes.byref(o)))
    return info


def sqrt(a, degree=5, max_iters=30, sketch_dim=8, seed=22137, tol=1e-6, warm_iters=0, workspace=None,
         alpha_schedule=None, flags=0):
    """In place: a <- A^(1/2); returns (A^(-1/2), info handle)."""
    b, m, n = _batched(a)
    inv = torch.empty_like(a)
    info = _Info(b, a.device)
    o = _options(info, flags, warm_iters, workspace, alpha_schedule)
    _check(lib().prism_sqrt_ex(a.data_ptr(), inv.data_ptr(), b, m, n, _dtype_code(a), degree, max_iters, sketch_dim,
                               seed, tol, _stream(), ctypes.byref(o)))
    return inv, info


def inv_root(a, root_p, max_iters=30, sketch_dim=8, seed=22137, tol=1e-6, warm_iters=0, workspace=None,
             alpha_schedule=None, flags=0):
    """In place: a <- A^(-1/root_p).  Returns an info handle."""
    b, m, n = _batched(a)
    info = _Info(b, a.device)
    o = _options(info, flags, warm_iters, workspace, alpha_schedule)
    _check(lib().prism_inv_root_ex(a.data_ptr(), root_p, b, m, n, _dtype_code(a), 3, max_iters, sketch_dim, seed,
                                   tol, _stream(), ctypes.byref(o)))
    return info


def sign(x, degree=5, max_iters=30, sketch_dim=8, seed=22137, tol=1e-6, warm_iters=0, workspace=None,
         alpha_schedule=None, flags=0):
    """In place: x[batch, n, n] <- sign(x).  Returns an info handle."""
    b, m, n = _batched(x)
    info = _Info(b, x.device)
    o = _options(info, flags, warm_iters, workspace, alpha_schedule)
    _check(lib().prism_sign_ex(x.data_ptr(), b, m, n, _dtype_code(x), degree, max_iters, sketch_dim, seed, tol,
                               _stream(), ctypes.byref(o)))
    return info


def inverse(a, max_iters=30, sketch_dim=8, seed=22137, tol=1e-6, warm_iters=0, workspace=None, alpha_schedule=None, flags=0):
    """In place: a[batch, n, n] <- a^(-1) by the Chebyshev iteration.  Returns an info handle."""
    b, m, n = _batched(a)
    info = _Info(b, a.device)
    o = _options(info, flags, warm_iters, workspace, alpha_schedule)
    _check(lib().prism_inverse_ex(a.data_ptr(), b, m, n, _dtype_code(a), max_iters, sketch_dim, seed, tol,
                                  _stream(), ctypes.byref(o)))
    return info


def sqrt_newton(a, max_iters=30, tol=1e-6, fit=True, workspace=None, alpha_schedule=None, flags=0):
    """In place: a <- A^(1/2) by the DB Newton iteration; returns (A^(-1/2), info handle)."""
    b, m, n = _batched(a)
    inv = torch.empty_like(a)
    info = _Info(b, a.device)
    o = _options(info, flags, 0, workspace, alpha_schedule)
    _check(lib().prism_sqrt_newton_ex(a.data_ptr(), inv.data_ptr(), b, m, n, _dtype_code(a), max_iters, int(bool(fit)), tol,
                                      _stream(), ctypes.byref(o)))
    return inv, info


def run_grouped(fn, xs, degree=5, max_iters=30, sketch_dim=8, seed=22137, tol=1e-6, root_p=0, flags=0, warm_iters=0,
                alpha_schedule=None, sources=None):
    """One call over tensors of different shapes (each [batch, m, n], all of one dtype), in place.  sources: per tensor
    of xs a list of `batch` contiguous [m, n] tensors that are read instead; xs then only takes the results, and no such tensor may
    overlap any part of xs but its own place.
    Returns (inverse outputs or None per group, info handles per group)."""
    if len(xs) == 0:
        _check(lib().prism_run_grouped(fn, None, 0, root_p, F32, degree, max_iters, sketch_dim, seed, tol, _stream(), None))
        return [], []
    groups = (Group * len(xs))()
    infos, invs = [], []
    two_outputs = fn in (FN_SQRT, FN_SQRT_NEWTON)
    for g, x in zip(groups, xs):
        b, m, n = _batched(x)
        info = _Info(b, x.device)
        inv = torch.empty_like(x) if two_outputs else None
        g.x, g.inv_out, g.info = x.data_ptr(), (inv.data_ptr() if two_outputs else None), info.buf.data_ptr()
        g.batch, g.m, g.n = b, m, n
        infos.append(info)
        invs.append(inv)
    o = Options()
    o.flags, o.warm_iters = flags, warm_iters
    if alpha_schedule is not None and len(alpha_schedule) > 0:
        o._sched = (ctypes.c_float * len(alpha_schedule))(*[float(a) for a in alpha_schedule])
        o.alpha_schedule = ctypes.cast(o._sched, ctypes.POINTER(ctypes.c_float))
        o.schedule_len = len(alpha_schedule)
    rest = (len(xs), root_p, _dtype_code(xs[0]), degree, max_iters, sketch_dim, seed, tol, _stream(), ctypes.byref(o))
    if sources is None:
        _check(lib().prism_run_grouped(fn, groups, *rest))
        return invs, infos
    for x, ts in zip(xs, sources):
        if len(ts) != x.shape[0] or any(t.shape != x.shape[1:] or t.dtype != x.dtype or t.device != x.device or not t.is_contiguous() for t in ts):
            raise PrismError("expected per group one contiguous tensor [m, n] per matrix, of the dtype and on the device of the results")
    if len(sources) != len(xs):
        raise PrismError("expected sources for every group")
    lists = [(ctypes.c_void_p * len(ts))(*[t.data_ptr() for t in ts]) for ts in sources]
    _check(lib().prism_run_grouped_from(fn, groups, (ctypes.c_void_p * len(lists))(*[ctypes.addressof(a) for a in lists]), *rest))
    return invs, infos


def read_reports(infos):
    """The reports of the groups of one grouped call, read by one copy (synchronises): a structured array per group.  One copy per
    group costs its round trip each: eight groups 0.3 ms."""
    if not infos:
        return []
    whole = torch.cat([h.buf for h in infos]).cpu().numpy()
    out, at = [], 0
    for h in infos:
        out.append(whole[at:at + h.buf.numel()].view(INFO_DTYPE).copy())
        at += h.buf.numel()
    return out


# ---- operators of a transformer layer ----
#
# Arrays of heads are tensors [batch, token, head, dim]; dim has to be contiguous, the other strides are free (views into one
# projection, transposed views).  These calls take a few microseconds on the GPU when they are small, so their descriptions are
# packed in one step (the layouts of prism_norm_rope_desc and prism_attention_desc) and every tensor is asked once.

_NORM_ROPE = struct.Struct("@9i2f4P18qPN")
_ATTENTION = struct.Struct("@7i2f5P24qPN")
_NO_NUMBER = (struct.error, OverflowError)      # of pack: what a field does not hold
_NO_STRIDES = (0, 0, 0)
_NONE = (None, None)
_raw_stream = torch._C._cuda_getCurrentRawStream if hasattr(torch._C, "_cuda_getCurrentRawStream") else (lambda i: torch.cuda.current_stream(i).cuda_stream)


def _device(t):
    """Index of a CUDA tensor's device."""
    i = t.get_device()
    if i < 0:
        raise PrismError("expected CUDA tensors")
    return i


def _on(dev, call, *args):
    """The library call on that device's current stream (passed last); the caller's device stays the current one."""
    if torch.cuda.current_device() == dev:
        _check(call(*args, _raw_stream(dev)))
    else:
        with torch.cuda.device(dev):
            _check(call(*args, _raw_stream(dev)))


def _heads(t, name, dtype, dev, shape):
    """Strides of batch, token and head of an array of heads."""
    if t.shape != shape:
        raise PrismError("%s: expected shape %s" % (name, tuple(shape)))
    s = t.stride()
    if t.dtype is not dtype or t.get_device() != dev or (s[3] != 1 and shape[3] > 1):
        raise PrismError("%s: expected the dtype and device of the other arrays, and contiguous dim" % name)
    return s[:3]


def _plain(t, name, dtype, dev, shape):
    """The address of an optional contiguous array."""
    if t is None:
        return 0
    if t.dtype is not dtype or t.shape != shape or t.get_device() != dev or not t.is_contiguous():
        raise PrismError("%s: expected a contiguous %s tensor of shape %s on the device of the others" % (name, dtype, tuple(shape)))
    return t.data_ptr()


def _given(workspace, dev):
    if workspace is None:
        return 0, 0
    if workspace.get_device() != dev:
        raise PrismError("workspace: expected a tensor on the device of the others")
    return workspace.data_ptr(), workspace.numel() * workspace.element_size()


def dropout(x, p, seed, offset=0, residual=None, out=None):
    """residual + dropout(x): every element is kept with probability 1 - p (rounded to 16 bits) and then divided by it.  The mask is a function
    of (seed modulo 2^64, offset modulo 2^32, index) and is not stored: the gradient with respect to x is dropout(dy, p, seed, offset).  out may be x or residual."""
    y = torch.empty_like(x) if out is None else out
    dev = _device(x)
    for t in (x, y) if residual is None else (x, y, residual):
        if t.shape != x.shape or t.dtype is not x.dtype or t.get_device() != dev or not t.is_contiguous():
            raise PrismError("expected contiguous tensors of one shape, dtype and device")
    _on(dev, lib().prism_dropout, x.data_ptr(), None if residual is None else residual.data_ptr(), y.data_ptr(), x.numel(), _dtype_code(x), p, seed, offset)
    return y


def rope_frequencies(rot_dim, base=10000.0, scaling=None, factor=1.0, original_len=None, fast=32.0, slow=1.0, device=None):
    """(inv_freq, scale) for qk_norm_rope: base^(-2i / rot_dim), for contexts `factor` times longer than trained on
       "linear"    every frequency divided by factor
       "base"      a larger base, so that the lowest frequency is divided by factor and the highest kept
       "by_turns"  frequencies that turn less than `slow` times in original_len divided by factor, more than `fast` times kept, a ramp
                   between; the rotated part is scaled by 0.1 ln(factor) + 1."""
    if rot_dim < 2 or rot_dim % 2 or not 0 < factor < np.inf or not 0 < base < np.inf:
        raise PrismError("rot_dim has to be even and positive, factor and base positive and finite")
    half = rot_dim // 2
    if scaling == "base":
        base = base * factor ** (rot_dim / (rot_dim - 2)) if rot_dim > 2 else base
    f = base ** (-np.arange(half) / half)
    scale = 1.0
    if scaling == "linear":
        f = f / factor
    elif scaling == "by_turns":
        if not original_len or original_len < 0 or not fast > slow:
            raise PrismError("by_turns needs a positive original_len, and fast above slow")
        keep = np.clip((original_len * f / (2 * np.pi) - slow) / (fast - slow), 0.0, 1.0)
        f = f * keep + f / factor * (1.0 - keep)
        scale = 0.1 * np.log(factor) + 1.0 if factor > 1.0 else 1.0
    elif scaling not in (None, "base"):
        raise PrismError("unknown scaling %r" % (scaling,))
    return torch.tensor(f, dtype=torch.float32, device=device), float(scale)


def _norm_rope_desc(q, k, results, grads, inv_freq, positions, start, q_weight, k_weight, norm, interleaved, scale, eps, workspace):
    """(a tensor of the call, its device, the packed description).  results: the arrays of the forward results (or their gradients), grads: those of the backward ones."""
    some = q if q is not None else k
    if some is None or some.dim() != 4:
        raise PrismError("expected queries or keys [batch, token, head, dim]")
    dev, dtype, (b, n, h, d) = _device(some), some.dtype, some.shape
    heads, strides = [0, 0], []
    for x, t in enumerate((q, k)):
        if t is not None:
            if t.dim() != 4:
                raise PrismError("expected [batch, token, head, dim]")
            heads[x] = t.shape[2]
    for arrays, names in (((q, k), ("q", "k")), (results, ("q_out", "k_out")), (grads, ("dq", "dk"))):
        for x, t in enumerate(arrays):
            if (t is None) != ((q, k)[x] is None) and arrays is not _NONE:
                raise PrismError("%s: goes with its input" % names[x])
            strides += _NO_STRIDES if t is None else _heads(t, names[x], dtype, dev, (b, n, heads[x], d))
    rot = 0 if inv_freq is None else 2 * inv_freq.numel()
    try:
        return some, dev, _NORM_ROPE.pack(
            b, n, heads[0], heads[1], d, rot, 1 if norm else 0, 1 if interleaved else 0, start, eps, scale, _plain(positions, "positions", torch.int32, dev, (b, n)),
            _plain(inv_freq, "inv_freq", torch.float32, dev, (rot // 2,)), _plain(q_weight, "q_weight", torch.float32, dev, (d,)),
            _plain(k_weight, "k_weight", torch.float32, dev, (d,)), *strides, *_given(workspace, dev))
    except _NO_NUMBER as e:
        raise PrismError("a number is out of range: %s" % e) from None


def _ptr(t):
    return None if t is None else t.data_ptr()


def _new(t):
    return None if t is None else t.new_empty(t.shape)


def qk_norm_rope(q, k, inv_freq=None, positions=None, start=0, q_weight=None, k_weight=None, norm=True, interleaved=False, scale=1.0, eps=1e-6,
                 out=None):
    """RMS norm of every head of q and k [batch, token, head, dim] times q_weight / k_weight (fp32 [dim], None: ones), then the rotation of
    its first 2 * len(inv_freq) entries by positions (int32 [batch, token], None: from `start` on).  norm=False: rotation only; inv_freq=None: norm only.
    q or k may be None.  out: the tensors for the results (q and k themselves are allowed).  Returns (q, k)."""
    qo, ko = (_new(q), _new(k)) if out is None else out
    some, dev, desc = _norm_rope_desc(q, k, (qo, ko), _NONE, inv_freq, positions, start, q_weight, k_weight, norm, interleaved, scale, eps, None)
    _on(dev, lib().prism_qk_norm_rope, _ptr(q), _ptr(k), _ptr(qo), _ptr(ko), _dtype_code(some), desc)
    return qo, ko


def qk_norm_rope_backward(dq_out, dk_out, q, k, inv_freq=None, positions=None, start=0, q_weight=None, k_weight=None, norm=True, interleaved=False,
                          scale=1.0, eps=1e-6, out=None, workspace=None):
    """Gradients of qk_norm_rope from those of its results: (dq, dk, dq_weight, dk_weight), the last two fp32 [dim], or None without the norm.
    q and k are the inputs of the forward call.  out: tensors for dq and dk."""
    dq, dk = (_new(q), _new(k)) if out is None else out
    some, dev, desc = _norm_rope_desc(q, k, (dq_out, dk_out), (dq, dk), inv_freq, positions, start, q_weight, k_weight, norm, interleaved, scale, eps, workspace)
    dqw, dkw = [None if t is None or not norm else (t.new_empty if t.numel() else t.new_zeros)(t.shape[3], dtype=torch.float32) for t in (q, k)]
    _on(dev, lib().prism_qk_norm_rope_backward, _ptr(dq_out), _ptr(dk_out), _ptr(q), _ptr(k), _ptr(dq), _ptr(dk), _ptr(dqw), _ptr(dkw), _dtype_code(some), desc)
    return dq, dk, dqw, dkw


def _attention_desc(q, k, v, out, back, scale, causal, softcap, slopes, prefix, k_lens, q_doc, k_doc, workspace):
    """(device, the packed description).  back: dout, dq, dk, dv, or ()."""
    if q.dim() != 4 or k.dim() != 4:
        raise PrismError("expected [batch, token, head, dim]")
    dev, dtype, rows, cells = _device(q), q.dtype, q.shape, k.shape
    b, n, hq, d = rows
    m, hk = cells[1], cells[2]
    if cells[0] != b or cells[3] != d:
        raise PrismError("k: expected the batch and dim of q")
    strides = _heads(q, "q", dtype, dev, rows) + _heads(k, "k", dtype, dev, cells) + _heads(v, "v", dtype, dev, cells) + _heads(out, "out", dtype, dev, rows)
    if back:
        dout, dq, dk, dv = back
        strides += _heads(dout, "dout", dtype, dev, rows) + _heads(dq, "dq", dtype, dev, rows) + _heads(dk, "dk", dtype, dev, cells) + _heads(dv, "dv", dtype, dev, cells)
    else:
        strides += 4 * _NO_STRIDES
    i32 = torch.int32
    try:
        return dev, _ATTENTION.pack(
            b, n, m, hq, hk, d, 1 if causal else 0, d ** -0.5 if scale is None else scale, softcap, _plain(slopes, "slopes", torch.float32, dev, (hq,)),
            _plain(prefix, "prefix", i32, dev, (b,)), _plain(k_lens, "k_lens", i32, dev, (b,)), _plain(q_doc, "q_doc", i32, dev, (b, n)),
            _plain(k_doc, "k_doc", i32, dev, (b, m)), *strides, *_given(workspace, dev))
    except _NO_NUMBER as e:
        raise PrismError("a number is out of range: %s" % e) from None


def attention(q, k, v, scale=None, causal=False, softcap=0.0, slopes=None, prefix=None, k_lens=None, q_doc=None, k_doc=None, out=None, workspace=None):
    """Attention of q [batch, n, q_heads, dim] over k and v [batch, m, k_heads, dim].  scores = scale q.k (scale None: dim^-1/2), capped by softcap tanh(. / softcap),
    less slopes[head] * distance.  Masks: causal (the last query sits at the last key), prefix [batch] (keys that all see), k_lens [batch] (keys there are), q_doc / k_doc
    [batch, n] / [batch, m] (documents; negative: padding).  Returns (out, lse); a query that sees nothing gets 0 and -inf."""
    y = q.new_empty(q.shape) if out is None else out
    dev, desc = _attention_desc(q, k, v, y, (), scale, causal, softcap, slopes, prefix, k_lens, q_doc, k_doc, workspace)
    lse = q.new_empty((q.shape[0], q.shape[2], q.shape[1]), dtype=torch.float32)
    _on(dev, lib().prism_attention, q.data_ptr(), k.data_ptr(), v.data_ptr(), y.data_ptr(), lse.data_ptr(), _dtype_code(q), desc)
    return y, lse


def attention_backward(dout, q, k, v, out, lse, scale=None, causal=False, softcap=0.0, slopes=None, prefix=None, k_lens=None, q_doc=None, k_doc=None,
                       grads=None, workspace=None):
    """(dq, dk, dv) from dout; out and lse as attention() returned them for the same arguments.  grads: tensors for the three results."""
    dq, dk, dv = (q.new_empty(q.shape), k.new_empty(k.shape), v.new_empty(v.shape)) if grads is None else grads
    dev, desc = _attention_desc(q, k, v, out, (dout, dq, dk, dv), scale, causal, softcap, slopes, prefix, k_lens, q_doc, k_doc, workspace)
    _plain(lse, "lse", torch.float32, dev, (q.shape[0], q.shape[2], q.shape[1]))
    _on(dev, lib().prism_attention_backward, dout.data_ptr(), q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), lse.data_ptr(), dq.data_ptr(), dk.data_ptr(),
        dv.data_ptr(), _dtype_code(q), desc)
    return dq, dk, dv


# ---- operators at the ends of a model ----
#
# Arrays of rows are tensors [..., width] whose rows follow each other at one stride, their entries next to each other; tokens are contiguous int64 or int32 tensors.  Scratch
# memory comes from PyTorch's allocator, for the stream (and graph) of the call.

_EMBEDDING = struct.Struct("@2q2if2qPN")
_LAYER_NORM = struct.Struct("@q2if7qPN")
_LOGITS = struct.Struct("@q2id2q3d5PN")


def _rows(t, name, dtype, dev, shape):
    """The stride between the rows of an array of rows."""
    if t.shape != shape or t.dtype is not dtype or t.get_device() != dev:
        raise PrismError("%s: expected shape %s, and the dtype and device of the other arrays" % (name, tuple(shape)))
    if t.is_contiguous():
        return shape[-1]
    if t.dim() == 2 and t.stride(1) == 1:
        return t.stride(0)
    try:
        flat = t.view(-1, shape[-1])
    except RuntimeError:
        flat = None
    if flat is None or (flat.stride(1) != 1 and shape[-1] > 1):
        raise PrismError("%s: expected rows at one stride, their entries next to each other" % name)
    return flat.stride(0)


def _tokens(t, dev, shape=None):
    """Whether they are int64."""
    if t.dtype is not torch.int64 and t.dtype is not torch.int32:
        raise PrismError("tokens: expected int64 or int32")
    if t.get_device() != dev or not t.is_contiguous() or (shape is not None and t.shape != shape):
        raise PrismError("tokens: expected a contiguous tensor%s on the device of the others" % ("" if shape is None else " of shape %s" % (tuple(shape),)))
    return 1 if t.dtype is torch.int64 else 0


def _pack(layout, *fields):
    try:
        return layout.pack(*fields)
    except _NO_NUMBER as e:
        raise PrismError("a number is out of range: %s" % e) from None


def _scratch(query, dev, workspace, layout, fields):
    """(the packed description, the tensor of its workspace).  query: the library's size for a description."""
    if workspace is None:
        n = ctypes.c_size_t(0)
        _check(query(_pack(layout, *fields, 0, 0), ctypes.byref(n)))
        workspace = torch.empty(n.value, dtype=torch.uint8, device="cuda:%d" % dev)
    return _pack(layout, *fields, *_given(workspace, dev)), workspace


def embedding(tokens, table, scale=1.0, out=None):
    """scale * table[tokens], [..., width]; a token that is no row of the table [rows, width] (padding) gives zeros."""
    dev = _device(table)
    size = table.shape
    if len(size) != 2:
        raise PrismError("table: expected [rows, width]")
    wide, (rows, width) = _tokens(tokens, dev), size
    shape = tokens.shape + (width,)
    if out is None:
        y, stride = table.new_empty(shape), width
    else:
        y, stride = out, _rows(out, "out", table.dtype, dev, shape)
    desc = _pack(_EMBEDDING, tokens.numel(), rows, width, wide, scale, _rows(table, "table", table.dtype, dev, size), stride, 0, 0)
    _on(dev, lib().prism_embedding, table.data_ptr(), tokens.data_ptr(), y.data_ptr(), _dtype_code(table), desc)
    return y


def embedding_backward(dout, tokens, rows, scale=1.0, out=None, workspace=None):
    """The gradient of embedding() with respect to its table, [rows, width], whole: rows that no token names are zeros."""
    dev, width, dtype = _device(dout), dout.shape[-1] if dout.dim() else 0, dout.dtype
    if dout.dim() < 1 or rows < 0:
        raise PrismError("expected dout [..., width] and a table's rows")
    d = dout.new_empty((rows, width)) if out is None else out
    fields = (tokens.numel(), rows, width, _tokens(tokens, dev, dout.shape[:-1]), scale, _rows(d, "out", dtype, dev, torch.Size((rows, width))),
              _rows(dout, "dout", dtype, dev, dout.shape))
    code = _dtype_code(dout)
    desc, workspace = _scratch(lambda *a: lib().prism_embedding_workspace_bytes(code, *a), dev, workspace, _EMBEDDING, fields)
    _on(dev, lib().prism_embedding_backward, dout.data_ptr(), tokens.data_ptr(), d.data_ptr(), code, desc)
    return d


def layer_norm(x, weight=None, bias=None, residual=None, center=True, eps=1e-5, out=None):
    """(y, total, stats): total = x + residual (x itself without one), y its rows [..., width] less their mean (center=False: as they are) over the root of their mean square
    and eps, times weight, plus bias (fp32 [width]); stats [rows, 2] for the gradients.  out: the tensors for y and total (None without a residual)."""
    dev, dtype, shape = _device(x), x.dtype, x.shape
    if x.dim() < 1:
        raise PrismError("expected [..., width]")
    width = shape[-1]
    sx, sr = _rows(x, "x", dtype, dev, shape), 0 if residual is None else _rows(residual, "residual", dtype, dev, shape)
    if out is None:
        y, total, sy, st = x.new_empty(shape), None if residual is None else x.new_empty(shape), width, width
    else:
        y, total = out
        if (total is None) != (residual is None):
            raise PrismError("total: goes with residual")
        sy, st = _rows(y, "out", dtype, dev, shape), 0 if total is None else _rows(total, "total", dtype, dev, shape)
    rows = x.numel() // width if width else 0
    stats = x.new_empty((rows, 2), dtype=torch.float32)
    f32 = torch.float32
    w, b = _plain(weight, "weight", f32, dev, (width,)), _plain(bias, "bias", f32, dev, (width,))
    desc = _pack(_LAYER_NORM, rows, width, 1 if center else 0, eps, sx, sr, st, sy, 0, 0, 0, 0, 0)
    _on(dev, lib().prism_layer_norm, x.data_ptr(), _ptr(residual), w, b, y.data_ptr(), _ptr(total), stats.data_ptr(), _dtype_code(x), desc)
    return y, x if total is None else total, stats


def layer_norm_backward(dy, total, stats, weight=None, dtotal=None, center=True, bias=True, out=None, workspace=None):
    """(dx, dweight, dbias) of layer_norm() from the gradient of y and, where not None, of total; total and stats as it returned them.  dx is the gradient of x and of the
    residual; dbias is None where bias is False."""
    dev, dtype, shape = _device(total), total.dtype, total.shape
    if total.dim() < 1:
        raise PrismError("expected [..., width]")
    width = shape[-1]
    dx = total.new_empty(shape) if out is None else out
    rows = total.numel() // width if width else 0
    dw = total.new_empty((width,), dtype=torch.float32)
    db = total.new_empty((width,), dtype=torch.float32) if bias else None
    w, at = _plain(weight, "weight", torch.float32, dev, (width,)), _plain(stats, "stats", torch.float32, dev, (rows, 2))
    fields = (rows, width, 1 if center else 0, 0.0, 0, 0, _rows(total, "total", dtype, dev, shape), 0, _rows(dy, "dy", dtype, dev, shape),
              0 if dtotal is None else _rows(dtotal, "dtotal", dtype, dev, shape), _rows(dx, "out", dtype, dev, shape))
    code = _dtype_code(total)
    desc, workspace = _scratch(lambda *a: lib().prism_layer_norm_workspace_bytes(code, *a), dev, workspace, _LAYER_NORM, fields)
    _on(dev, lib().prism_layer_norm_backward, dy.data_ptr(), total.data_ptr(), at, w, _ptr(dtotal), dx.data_ptr(), dw.data_ptr(), _ptr(db), code, desc)
    return dx, dw, db


def _logits(logits, tokens, scale, out, more=(0.0, 0.0, 0.0, 0, 0, 0, 0)):
    """(device, dtype code, the description's fields before the workspace)."""
    dev = _device(logits)
    if logits.dim() < 1:
        raise PrismError("expected logits [..., vocabulary]")
    shape = logits.shape
    return dev, _dtype_code(logits), (tokens.numel(), shape[-1], _tokens(tokens, dev, shape[:-1]), scale, _rows(logits, "logits", logits.dtype, dev, shape),
                                      0 if out is None else _rows(out, "out", logits.dtype, dev, shape)) + more


def token_logprob(logits, tokens, scale=1.0):
    """(logp, lse), fp32 in the shape of tokens: the logarithm of the softmax of scale * logits [..., vocabulary] at each row's token, and of the sum of its exponentials.  A token
    outside the vocabulary (padding) gives 0 in both."""
    dev, code, fields = _logits(logits, tokens, scale, None)
    logp, lse = logits.new_empty(tokens.shape, dtype=torch.float32), logits.new_empty(tokens.shape, dtype=torch.float32)
    _on(dev, lib().prism_token_logprob, logits.data_ptr(), tokens.data_ptr(), logp.data_ptr(), lse.data_ptr(), code, _pack(_LOGITS, *fields, 0, 0))
    return logp, lse


def token_logprob_backward(dlogp, logits, tokens, lse, scale=1.0, out=None):
    """The gradient with respect to the logits from that of logp; lse as token_logprob() (or policy_loss()) returned it.  out may be logits."""
    d = torch.empty_like(logits, memory_format=torch.contiguous_format) if out is None else out
    dev, code, fields = _logits(logits, tokens, scale, d)
    given = [_plain(t, n, torch.float32, dev, tokens.shape) for t, n in ((dlogp, "dlogp"), (lse, "lse"))]
    _on(dev, lib().prism_token_logprob_backward, given[0], logits.data_ptr(), tokens.data_ptr(), given[1], d.data_ptr(), code, _pack(_LOGITS, *fields, 0, 0))
    return d


PolicyLoss = collections.namedtuple("PolicyLoss", "loss logp lse dlogp dlogits")


def policy_loss(logits, tokens, advantages=None, old_logp=None, ref_logp=None, weights=None, clip=(0.2, 0.2), kl=0.0, scale=1.0, gradient=True, out=None, workspace=None):
    """The loss of a policy on the tokens it took, and its gradient, in one pass over the logits [..., vocabulary]:
    the sum over rows of weight * (-min(r A, clip(r) A) + kl (exp(f) - f - 1)), r = exp(logp - old_logp) held between 1 - clip[0] and 1 + clip[1], f = ref_logp - logp.
    Without old_logp -A logp takes the first part's place; without advantages A = 1 (with neither: cross entropy); weights None: the mean over the rows that have a token.
    Everything given for a row is fp32 in the shape of tokens; a token outside the vocabulary (padding) is left out.
    Returns (loss, logp, lse, dlogp, dlogits): dlogp the gradient with respect to logp, dlogits None with gradient=False; out: the tensor for dlogits (logits itself is allowed)."""
    if gradient:
        out = torch.empty_like(logits, memory_format=torch.contiguous_format) if out is None else out
    elif out is not None:
        raise PrismError("out: goes with gradient")
    low, high = clip
    rows = tokens.shape
    dev = _device(logits)
    _, code, fields = _logits(logits, tokens, scale, out, (low, high, kl) + tuple(
        _plain(t, n, torch.float32, dev, rows) for t, n in ((advantages, "advantages"), (old_logp, "old_logp"), (ref_logp, "ref_logp"), (weights, "weights"))))
    loss = logits.new_empty((), dtype=torch.float32)
    logp = logits.new_empty(rows, dtype=torch.float32)
    lse, dlogp = torch.empty_like(logp), torch.empty_like(logp)       # (not views of one allocation: what is written to one of them would count for all)
    desc, workspace = _scratch(lib().prism_policy_loss_workspace_bytes, dev, workspace, _LOGITS, fields)
    _on(dev, lib().prism_policy_loss, logits.data_ptr(), tokens.data_ptr(), loss.data_ptr(), logp.data_ptr(), lse.data_ptr(), dlogp.data_ptr(), _ptr(out), code, desc)
    return PolicyLoss(loss, logp, lse, dlogp, out)


# ---- single steps (unit tests, profiling) ----

def spd_inverse(a):
    batch, n, _ = a.shape
    out = torch.empty_like(a)
    _check(lib().prism_spd_inverse(a.data_ptr(), out.data_ptr(), batch, n, _stream()))
    return out


def sketch(n, sketch_dim, seed, k, fn, device="cuda"):
    out = torch.empty((n, sketch_dim), dtype=torch.float32, device=device)
    _check(lib().prism_sketch(out.data_ptr(), n, sketch_dim, seed, k, fn, _stream()))
    return out


def gauss_parts(first, count, device="cuda"):
    r = torch.empty(count, dtype=torch.float64, device=device)
    c = torch.empty_like(r)
    s = torch.empty_like(r)
    _check(lib().prism_gauss_parts(first, count, r.data_ptr(), c.data_ptr(), s.data_ptr(), _stream()))
    return r, c, s


def chain_product(R, V):
    batch, n, ld = V.shape
    out = torch.empty_like(V)
    _check(lib().prism_chain_product(R.data_ptr(), V.data_ptr(), out.data_ptr(), batch, n, ld, _stream()))
    return out


def release_workspaces():
    """Free the library's cached workspaces (nothing may be in flight, no captured graph may be replayed)."""
    torch.cuda.synchronize()
    _check(lib().prism_release_workspaces())


def chain_product_bf16(Rb, R, V, return_planes=False):
    """out = (Rb + diag(R - Rb)) V.  With return_planes also the scratch array of the call: bf16 bit
    patterns [2][batch][n / 256][3][ld][32 units, low four bits xor-ed with the column][8], the planes of V and of out (zeros where the launch is
    small enough for the kernel that does not use them)."""
    batch, n, ld = V.shape
    out = torch.empty_like(V)
    planes = torch.zeros((2, batch, n * ld * 3), dtype=torch.int16, device=V.device)
    _check(lib().prism_chain_product_bf16(Rb.data_ptr(), R.data_ptr(), V.data_ptr(), out.data_ptr(), planes.data_ptr(),
                                          batch, n, ld, _stream()))
    return (out, planes) if return_planes else out


def gemm_f32(A, B, a_km=False, sym=False):
    batch = A.shape[0]
    M, K = (A.shape[2], A.shape[1]) if a_km else (A.shape[1], A.shape[2])
    N = B.shape[2]
    C = torch.empty((batch, M, N), dtype=torch.float32, device=A.device)
    _check(lib().prism_gemm_f32(A.data_ptr(), B.data_ptr(), C.data_ptr(), batch, M, N, K, int(a_km) | (2 if sym else 0), _stream()))
    return C


def gemm_f32_planes(A, B, C=None):
    """C + A B (A [batch][M][K]), or without C: I - A^T B (A stored [batch][K][M], the product symmetric), from three bf16 planes per operand."""
    batch, a, b = A.shape
    M, K = (b, a) if C is None else (a, b)
    N = B.shape[2]
    out = torch.empty((batch, M, N), dtype=torch.float32, device=A.device) if C is None else C.clone()
    _check(lib().prism_gemm_f32_planes(A.data_ptr(), B.data_ptr(), out.data_ptr(), batch, M, N, K, int(C is None), _stream()))
    return out


def gemm_f64a(A, B):
    batch, M, K = A.shape
    N = B.shape[2]
    C = torch.empty((batch, M, N), dtype=torch.float64, device=A.device)
    _check(lib().prism_gemm_f64a(A.data_ptr(), B.data_ptr(), C.data_ptr(), batch, M, N, K, _stream()))
    return C


def gemm_bf16_nt(A, B, tile, km=0):
    """C = A B^T.  km = 0: A [batch][M][K], B [batch][N][K]; km = 2: B is stored [batch][K][N];
    km = 3: A is stored [batch][K][M] and B [batch][K][N]."""
    if km not in (0, 2, 3):
        raise ValueError("km must be 0, 2 or 3")
    batch = A.shape[0]
    K, M = (A.shape[1], A.shape[2]) if km == 3 else (A.shape[2], A.shape[1])
    N = B.shape[2] if km else B.shape[1]
    if (B.shape[1] if km else B.shape[2]) != K or B.shape[0] != batch:
        raise ValueError("operand shapes do not match")
    tile = tile + (10000 if km == 3 else 20000 if km == 2 else 0)
    C = torch.empty((batch, M, N), dtype=torch.float32, device=A.device)
    _check(lib().prism_gemm_bf16_nt(A.data_ptr(), B.data_ptr(), C.data_ptr(), batch, M, N, K, tile, _stream()))
    return C


def profile_enable(on):
    _check(lib().prism_profile_enable(int(on)))


def profile_collect():
    """{kind: (milliseconds, launches)} summed over everything recorded since profile_enable(True)."""
    n = len(PROFILE_KINDS)
    ms = (ctypes.c_double * n)()
    cnt = (ctypes.c_longlong * n)()
    _check(lib().prism_profile_collect(ms, cnt, n))
    return {k: (ms[j], cnt[j]) for j, k in enumerate(PROFILE_KINDS)}
