"""Thin ctypes binding of libdpgrad.so (declared in include/dpgrad.h).

Each function has the name and argument order of its C entry point and only
marshals arguments: device pointers may be given as torch tensors (their
``data_ptr()``), raw integer addresses or None; ``ws_bytes`` is taken from the
workspace tensor; ``stream`` defaults to torch's current HIP stream.  A status
other than DP_OK raises :class:`DPError`.  There is no fallback: if the
library is not built, loading fails loudly.  The functions of the
language-model operators (dp_embedding_lookup, dp_clip_accumulate_tokens,
dp_gated_ffn_*, dp_clip_global_norm_many, dp_rotary, dp_attention_*,
dp_distill_loss) also check their tensors: dense, on one GPU, of the declared
type and at least the declared size, else ValueError or TypeError; they are
enqueued on the tensors' GPU, and a torch stream of another one is refused
(ValueError).  Where a call takes the values from one position to the next
(ldx, ldq and the like), a tensor may be a view of [N][T] positions with those
strides, such as a section of a fused projection's output.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional

PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(PKG, "libdpgrad.so")

DP_OK, DP_EINVAL, DP_EDTYPE, DP_EUNSUPPORTED, DP_ECAP, DP_EHIP = range(6)
DP_F32, DP_BF16 = 0, 1
DP_FLAG_BAD_INDEX, DP_FLAG_NONFINITE, DP_FLAG_CAP, DP_FLAG_WAIT = 1, 2, 4, 8

# (name, restype, argtypes) of every exported entry point
_P = ctypes.c_void_p
_I64 = ctypes.c_int64
_F = ctypes.c_float
_SZ = ctypes.c_size_t
_I32 = ctypes.c_int32
_U32 = ctypes.c_uint32
_U64 = ctypes.c_uint64
_ST = ctypes.c_int

SIGNATURES = {
    "dp_status_string": (ctypes.c_char_p, [_ST]),
    "dp_abi_version": (ctypes.c_int, []),
    "dp_grad_sample_linear_workspace_bytes": (_SZ, [_I64, _I64, _I64, _I64, _ST]),
    "dp_grad_sample_linear": (_ST, [_P, _P, _ST, _I64, _I64, _I64, _I64, _F, _P, _P, _P, _P, _P, _SZ, _P]),
    "dp_grad_sample_linear_noalloc_max_bytes": (_SZ, []),
    "dp_grad_sample_linear_noalloc": (_ST, [_P, _P, _ST, _I64, _I64, _I64, _I64, _F, _P, _P, _P, _P, _P]),
    "dp_grad_sample_conv2d_workspace_bytes": (_SZ, [_I64] * 11),
    "dp_grad_sample_conv2d": (_ST, [_P, _P, _ST] + [_I64] * 16 + [_F, _P, _P, _P, _P, _P, _SZ, _P]),
    "dp_conv2d_set_path": (ctypes.c_int, [ctypes.c_int]),
    "dp_conv2d_kernel_choice": (_I32, [_I64] * 11),
    "dp_grad_sample_many_grouped": (_I32, [_P, _ST, _I64]),
    "dp_grad_sample_many_workspace_bytes": (_SZ, [_P, _I32, _ST, _I64]),
    "dp_grad_sample_many": (_ST, [_P, _I32, _ST, _I64, _P, _P, _SZ, _P]),
    "dp_grad_sample_embedding_workspace_bytes": (_SZ, [_I64, _I64]),
    "dp_grad_sample_embedding": (_ST, [_P, _P, _ST, _I64, _I64, _I64, _I64, _F, _P, _P, _P, _I64, _P,
                                       _P, _P, _SZ, _P]),
    "dp_embedding_lookup": (_ST, [_P, _P, _ST, _I64, _I64, _I64, _I64, _F, _P, _ST, _P, _P]),
    "dp_gated_ffn_forward_workspace_bytes": (_SZ, [_I64, _I64, _I64, _ST]),
    "dp_gated_ffn_forward": (_ST, [_P, _P, _P, _ST, _I64, _I64, _I64, _ST, _P, _P, _P, _P, _SZ, _P]),
    "dp_gated_ffn_backward_workspace_bytes": (_SZ, [_I64, _I64, _I64, _ST]),
    "dp_gated_ffn_backward": (_ST, [_P, _P, _P, _P, _P, _ST, _I64, _I64, _I64, _ST, _P, _P, _P, _P, _SZ, _P]),
    "dp_rotary": (_ST, [_P, _ST, _I64, _I64, _I64, _I64, _I64, _P, _P, _I32, _P, _ST, _I32, _P, _I64, _P]),
    "dp_attention_forward_workspace_bytes": (_SZ, [_P]),
    "dp_attention_forward": (_ST, [_P, _P, _P, _P, _P, _P, _P, _SZ, _P]),
    "dp_attention_backward_workspace_bytes": (_SZ, [_P]),
    "dp_attention_backward": (_ST, [_P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _SZ, _P]),
    "dp_distill_loss_workspace_bytes": (_SZ, [_I64, _I64, _I64, _ST]),
    "dp_distill_loss": (_ST, [_P, _ST, _I64, _I64, _P, _P, _I64, _P, _F, _F, _P, _P, _P, _P, _P, _SZ, _P]),
    "dp_grad_sample_layernorm_workspace_bytes": (_SZ, [_I64, _I64, _I64]),
    "dp_grad_sample_layernorm": (_ST, [_P, _P, _ST, _I64, _I64, _I64, _F, _P, _P, _P, _P, _P, _SZ, _P]),
    "dp_grad_sample_groupnorm_workspace_bytes": (_SZ, [_I64, _I64, _I64]),
    "dp_grad_sample_groupnorm": (_ST, [_P, _P, _ST, _I64, _I64, _I64, _F, _P, _P, _P, _P, _P, _SZ, _P]),
    "dp_lstm_backward": (_ST, [_P, _P, _P, _P, _P, _I64, _I64, _I64, _P, _P, _P]),
    "dp_per_sample_norms": (_ST, [_P, _I32, _I64, _P, _P, _P]),
    "dp_per_sample_norms_active": (_ST, [_P, _I32, _I64, _P, _P, _P, _P]),
    "dp_ghost_norm_linear_workspace_bytes": (_SZ, [_I64, _I64, _I64, _I64]),
    "dp_ghost_norm_linear": (_ST, [_P, _P, _ST, _I64, _I64, _I64, _I64, _F, _I32, _P, _P, _P, _SZ, _P]),
    "dp_ghost_norm_linear_many_workspace_bytes": (_SZ, [_P, _I32, _I64]),
    "dp_grad_sample_layernorm_many_workspace_bytes": (_SZ, [_P, _I32, _I64, _ST]),
    "dp_grad_sample_layernorm_many": (_ST, [_P, _I32, _ST, _I64, _P, _P, _SZ, _P]),
    "dp_ghost_norm_linear_many": (_ST, [_P, _I32, _ST, _I64, _P, _P, _SZ, _P]),
    "dp_sqnorm_from_grads": (_ST, [_P, _I64, _I64, _P, _P, _P]),
    "dp_clip_factors": (_ST, [_P, _I64, _F, _P, _P, _P]),
    "dp_clip_accumulate_workspace_bytes": (_SZ, [_I64, _I64]),
    "dp_clip_accumulate": (_ST, [_P, _P, _F, _I64, _I64, _P, _P, _P, _P, _SZ, _P]),
    "dp_clip_accumulate_linear_workspace_bytes": (_SZ, [_I64, _I64, _I64, _I64, _ST]),
    "dp_clip_accumulate_linear": (_ST, [_P, _P, _ST, _I64, _I64, _I64, _I64, _F, _P, _F, _P, _P, _P, _P,
                                        _SZ, _P]),
    "dp_clip_accumulate_linear_many_workspace_bytes": (_SZ, [_P, _I32, _ST, _I64]),
    "dp_clip_accumulate_linear_many": (_ST, [_P, _I32, _ST, _I64, _P, _F, _P, _P, _SZ, _P]),
    "dp_clip_accumulate_embedding_workspace_bytes": (_SZ, [_I64, _I64]),
    "dp_clip_accumulate_embedding": (_ST, [_P, _P, _P, _I64, _P, _F, _I64, _I64, _I64, _P, _P, _P, _SZ, _P]),
    "dp_clip_accumulate_tokens_workspace_bytes": (_SZ, [_I64, _I64, _I64, _I64, _ST]),
    "dp_clip_accumulate_tokens": (_ST, [_P, _P, _ST, _I64, _I64, _I64, _I64, _F, _P, _F, _P, _P, _P, _SZ, _P]),
    "dp_clip_global_norm_many_workspace_bytes": (_SZ, [_P, _I32]),
    "dp_clip_global_norm_many": (_ST, [_P, _I32, _F, _P, _P, _P, _SZ, _P]),
    "dp_clip_noise_many_workspace_bytes": (_SZ, [_P, _I32, _I64]),
    "dp_clip_noise_many": (_ST, [_P, _I32, _I64, _P, _F, _U64, _U64, _P, _F, _F, _P, _P, _SZ, _P]),
    "dp_norms_clip_noise_workspace_bytes": (_SZ, [_P, _I32, _I64]),
    "dp_norms_clip_noise": (_ST, [_P, _I32, _P, _I32, _I64, _P, _F, _U64, _U64, _P, _F, _F, _P, _P, _SZ, _P]),
    "dp_norms_clip_noise_sched": (_ST, [_P, _I32, _P, _I32, _I64, _P, _F, _U64, _U64, _P, _P, _I64, _P, _F, _P, _P,
                                        _SZ, _P]),
    "dp_step_advance": (_ST, [_P, _U64, _P]),
    "dp_add_noise": (_ST, [_P, _P, _I64, _U64, _U64, _U32, _F, _F, _F, _P, _P]),
    "dp_philox_normals": (_ST, [_P, _P, _I64, _U64, _U64, _U32, _P]),
}


class DPParam(ctypes.Structure):
    """struct dp_param of dpgrad.h."""
    _fields_ = [("grad_sample", ctypes.c_void_p), ("sum", ctypes.c_void_p), ("out", ctypes.c_void_p),
                ("numel", ctypes.c_int64), ("param_index", ctypes.c_uint32), ("flags", ctypes.c_uint32),
                ("accum", ctypes.c_void_p)]


DP_PARAM_REDUCE = 1


def _item_array(kind, entries):
    """Items of a grouped call, one per entry.  The array keeps the entries, and with them the tensors whose addresses it
    holds."""
    arr = (kind * max(len(entries), 1))()
    arr.entries = list(entries)
    return arr


def make_params(entries):
    """A dp_param array from (grad_sample, sum, out, numel, param_index[, accum]) tuples.

    grad_sample None means the sum is already formed (no DP_PARAM_REDUCE);
    an empty tensor (N = 0) still asks for the reduction.  accum (optional,
    default None) is the running sum of a virtual step."""
    arr = _item_array(DPParam, entries)
    for i, ent in enumerate(entries):
        g, s, o, numel, pidx = ent[:5]
        arr[i].accum = _ptr(ent[5]) if len(ent) > 5 else None
        arr[i].grad_sample = _ptr(g)
        arr[i].sum = _ptr(s)
        arr[i].out = _ptr(o)
        arr[i].numel = int(numel)
        arr[i].param_index = int(pidx)
        arr[i].flags = DP_PARAM_REDUCE if g is not None else 0
    return arr


class DPLinearClip(ctypes.Structure):
    """struct dp_linear_clip of dpgrad.h."""
    _fields_ = [("A", ctypes.c_void_p), ("B", ctypes.c_void_p), ("T", ctypes.c_int64), ("d_in", ctypes.c_int64),
                ("d_out", ctypes.c_int64), ("scale", ctypes.c_float), ("sumW", ctypes.c_void_p),
                ("sumb", ctypes.c_void_p)]


def make_linear_clips(entries):
    """A dp_linear_clip array from (A, B, T, d_in, d_out, scale, sumW, sumb) tuples."""
    arr = _item_array(DPLinearClip, entries)
    for i, (A, B, T, d_in, d_out, scale, sumW, sumb) in enumerate(entries):
        arr[i].A = _ptr(A)
        arr[i].B = _ptr(B)
        arr[i].T, arr[i].d_in, arr[i].d_out = int(T), int(d_in), int(d_out)
        arr[i].scale = float(scale)
        arr[i].sumW = _ptr(sumW)
        arr[i].sumb = _ptr(sumb)
    return arr


DP_LAYER_LINEAR, DP_LAYER_CONV2D = 0, 1


class DPLayerGrad(ctypes.Structure):
    """struct dp_layer_grad of dpgrad.h."""
    _fields_ = [("kind", ctypes.c_int32), ("A", ctypes.c_void_p), ("B", ctypes.c_void_p)] + \
               [(f, ctypes.c_int64) for f in ("T", "d_in", "d_out", "Cin", "H", "W", "Cout", "Ho", "Wo", "kh", "kw",
                                              "sh", "sw", "ph", "pw")] + \
               [("scale", ctypes.c_float), ("gW", ctypes.c_void_p), ("gb", ctypes.c_void_p),
                ("sqnorm", ctypes.c_void_p)]


def linear_grad_item(A, B, T, d_in, d_out, scale, gW, gb=None, sqnorm=None):
    """The dp_layer_grad fields of a Linear layer (a dict for make_layer_grads)."""
    return dict(kind=DP_LAYER_LINEAR, A=A, B=B, T=T, d_in=d_in, d_out=d_out, scale=scale, gW=gW, gb=gb,
                sqnorm=sqnorm)


def conv2d_grad_item(X, GY, Cin, H, W, Cout, Ho, Wo, kh, kw, sh, sw, ph, pw, scale, gW, gb=None, sqnorm=None):
    """The dp_layer_grad fields of a Conv2d layer (a dict for make_layer_grads)."""
    return dict(kind=DP_LAYER_CONV2D, A=X, B=GY, Cin=Cin, H=H, W=W, Cout=Cout, Ho=Ho, Wo=Wo, kh=kh, kw=kw, sh=sh,
                sw=sw, ph=ph, pw=pw, scale=scale, gW=gW, gb=gb, sqnorm=sqnorm)


def make_layer_grads(entries):
    """A dp_layer_grad array from linear_grad_item / conv2d_grad_item dicts."""
    arr = _item_array(DPLayerGrad, entries)
    for i, e in enumerate(entries):
        for k, v in e.items():
            if k in ("A", "B", "gW", "gb", "sqnorm"):
                setattr(arr[i], k, _ptr(v))
            elif k == "scale":
                arr[i].scale = float(v)
            else:
                setattr(arr[i], k, int(v))
    return arr


class DPGhostLayer(ctypes.Structure):
    """struct dp_ghost_layer of dpgrad.h."""
    _fields_ = [("A", ctypes.c_void_p), ("B", ctypes.c_void_p), ("T", ctypes.c_int64), ("d_in", ctypes.c_int64),
                ("d_out", ctypes.c_int64), ("scale", ctypes.c_float), ("bias", ctypes.c_int32),
                ("sqnorm", ctypes.c_void_p)]


def make_ghost_layers(entries):
    """A dp_ghost_layer array from (A, B, T, d_in, d_out, scale, bias, sqnorm) tuples."""
    arr = _item_array(DPGhostLayer, entries)
    for i, (A, B, T, d_in, d_out, scale, bias, sqnorm) in enumerate(entries):
        arr[i].A = _ptr(A)
        arr[i].B = _ptr(B)
        arr[i].T, arr[i].d_in, arr[i].d_out = int(T), int(d_in), int(d_out)
        arr[i].scale = float(scale)
        arr[i].bias = 1 if bias else 0
        arr[i].sqnorm = _ptr(sqnorm)
    return arr


class DPLayerNormLayer(ctypes.Structure):
    """struct dp_layernorm_layer of dpgrad.h."""
    _fields_ = [("xhat", ctypes.c_void_p), ("B", ctypes.c_void_p), ("T", ctypes.c_int64), ("D", ctypes.c_int64),
                ("scale", ctypes.c_float), ("ggamma", ctypes.c_void_p), ("gbeta", ctypes.c_void_p),
                ("sqnorm", ctypes.c_void_p)]


def make_layernorm_layers(entries):
    """A dp_layernorm_layer array from (xhat, B, T, D, scale, ggamma, gbeta, sqnorm) tuples."""
    arr = _item_array(DPLayerNormLayer, entries)
    for i, (xh, B, T, D, scale, gg, gb, sq) in enumerate(entries):
        arr[i].xhat = _ptr(xh)
        arr[i].B = _ptr(B)
        arr[i].T, arr[i].D = int(T), int(D)
        arr[i].scale = float(scale)
        arr[i].ggamma = _ptr(gg)
        arr[i].gbeta = _ptr(gb)
        arr[i].sqnorm = _ptr(sq)
    return arr


class DPGradTensor(ctypes.Structure):
    """struct dp_grad_tensor of dpgrad.h."""
    _fields_ = [("g", ctypes.c_void_p), ("out", ctypes.c_void_p), ("numel", ctypes.c_int64),
                ("dtype", ctypes.c_int32)]


def make_grad_tensors(entries):
    """A dp_grad_tensor array from (g, out, numel, dtype) tuples; out None: the tensor counts in the norm only.  Takes
    about 1 us of the host's time per tensor: keep the array while the buffers stay."""
    arr = _item_array(DPGradTensor, entries)
    dev, ptrs = _tensors("make_grad_tensors", *[(n, x, _tdtype(dt), numel) for g, out, numel, dt in entries
                                                for n, x in (("g", g), ("out", out))])
    for i, (g, out, numel, dt) in enumerate(entries):
        arr[i].g, arr[i].out = ptrs[2 * i], ptrs[2 * i + 1]
        arr[i].numel = int(numel)
        arr[i].dtype = int(dt)
    arr.dev = dev                         # the tensors' GPU
    return arr


DP_ATTENTION_CAUSAL, DP_ATTENTION_LAST = 1, 2


class DPAttention(ctypes.Structure):
    """struct dp_attention of dpgrad.h."""
    _fields_ = [("dt", ctypes.c_int32), ("flags", ctypes.c_uint32)] + \
               [(f, ctypes.c_int64) for f in ("N", "Tq", "Tk", "Hq", "Hk", "D", "ldq", "ldk", "ldv", "ldo")] + \
               [("scale", ctypes.c_float), ("softcap", ctypes.c_float)] + \
               [(f, ctypes.c_void_p) for f in ("slopes", "lens", "prefix", "docs")]


def make_attention(dt, N, Tq, Tk, Hq, Hk, D, scale, flags=0, softcap=0.0, slopes=None, lens=None, prefix=None, docs=None,
                   ldq=None, ldk=None, ldv=None, ldo=None):
    """A dp_attention; ld* default to dense positions.  It keeps the tensors whose addresses it holds."""
    import torch
    a = DPAttention(dt=dt, flags=flags, N=N, Tq=Tq, Tk=Tk, Hq=Hq, Hk=Hk, D=D, scale=scale, softcap=softcap)
    a.ldq, a.ldo = [Hq * D if ld is None else ld for ld in (ldq, ldo)]
    a.ldk, a.ldv = [Hk * D if ld is None else ld for ld in (ldk, ldv)]
    i32 = torch.int32
    a.dev, p = _tensors("make_attention", ("slopes", slopes, torch.float32, Hq), ("lens", lens, i32, N),
                        ("prefix", prefix, i32, N), ("docs", docs, i32, N * Tk))
    a.slopes, a.lens, a.prefix, a.docs = p
    a.kept = (slopes, lens, prefix, docs)
    return a


class DPError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__("%s: %s" % (where, status_string(code)))


_lib = None


def lib():
    """Load libdpgrad.so (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError("libdpgrad.so is not built (%s); run `python -m paper_2109_12298_amd.build`"
                               % LIB_PATH)
        L = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(L, name)
            fn.restype = res
            fn.argtypes = args
        _lib = L
    return _lib


def status_string(code: int) -> str:
    return lib().dp_status_string(code).decode()


def dp_status_string(code: int) -> str:
    return status_string(code)


def dp_abi_version() -> int:
    return lib().dp_abi_version()


def _ptr(x):
    if x is None:
        return None
    if isinstance(x, int):
        return x
    return x.data_ptr()


def _nbytes(x) -> int:
    if x is None:
        return 0
    return x.numel() * x.element_size()


def _numel(x) -> int:
    return 0 if x is None else x.numel()


def _stream(stream):
    if stream is None:
        import torch
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def dtype_of(t) -> int:
    import torch
    if t.dtype == torch.float32:
        return DP_F32
    if t.dtype == torch.bfloat16:
        return DP_BF16
    raise TypeError("unsupported dtype %s" % t.dtype)


def _tdtype(dt):
    """The torch type of a dp_dtype (None for an unknown one, which the call itself refuses)."""
    import torch
    return torch.float32 if dt == DP_F32 else torch.bfloat16 if dt == DP_BF16 else None


def _tensors(where, *args):
    """Addresses of a call's tensor arguments (name, tensor, type, elements),
    and the GPU they are on (None where all were given as integers or None).
    Each tensor must be dense, on that one GPU, of its type (None: any) and at
    least its size: a host tensor's address, say, would fault the GPU.
    Integers pass as addresses."""
    dev, ptrs = None, []
    for name, x, dtype, numel in args:
        if x is None or x.__class__ is int:
            ptrs.append(x)
            continue
        d = x.get_device()
        if d != dev:
            if d < 0:
                raise ValueError("%s: %s is not on a GPU" % (where, name))
            if dev is not None:
                raise ValueError("%s: %s is on GPU %d, other arguments on GPU %d" % (where, name, d, dev))
            dev = d
        if dtype is not None and x.dtype is not dtype:
            raise TypeError("%s: %s is %s, not %s" % (where, name, x.dtype, dtype))
        if not x.is_contiguous():
            raise ValueError("%s: %s is not contiguous" % (where, name))
        if x.numel() < numel:
            raise ValueError("%s: %s has %d elements, %d are needed" % (where, name, x.numel(), numel))
        ptrs.append(x.data_ptr())
    return dev, ptrs


def _rows(where, dev, dtype, *args):
    """As _tensors for arrays of N samples of T positions with `ld` values from
    one position to the next, `width` of them used (name, tensor, N, T, ld,
    width).  A tensor that is not dense has to be a view [N][T][...] with those
    strides.  `dev`: the GPU of the call's other tensors, or None."""
    ptrs = []
    for name, x, N, T, ld, width in args:
        if x is None or x.__class__ is int:
            ptrs.append(x)
            continue
        d = x.get_device()
        if d != dev:
            if d < 0:
                raise ValueError("%s: %s is not on a GPU" % (where, name))
            if dev is not None:
                raise ValueError("%s: %s is on GPU %d, other arguments on GPU %d" % (where, name, d, dev))
            dev = d
        if dtype is not None and x.dtype is not dtype:
            raise TypeError("%s: %s is %s, not %s" % (where, name, x.dtype, dtype))
        need = (N * T - 1) * ld + width if N > 0 and T > 0 else 0
        if not x.is_contiguous():
            st, sh = x.stride(), x.shape
            inner = 1
            for k in range(x.dim() - 1, 1, -1):
                if sh[k] != 1 and st[k] != inner:
                    break
                inner *= sh[k]
            else:
                if x.dim() >= 3 and sh[0] >= N and sh[1] >= T and inner >= width and (N <= 1 or (st[0] == T * ld and sh[1] == T)) \
                        and (T <= 1 or st[1] == ld):
                    ptrs.append(x.data_ptr())
                    continue
            raise ValueError("%s: %s is neither contiguous nor [N][T][...] with %d values from one position to the next"
                             % (where, name, ld))
        if x.numel() < need:
            raise ValueError("%s: %s has %d elements, %d are needed" % (where, name, x.numel(), need))
        ptrs.append(x.data_ptr())
    return dev, ptrs


def _run(where, dev, fn, *args, stream):
    """The call on GPU `dev` (None: the current one), on its current stream unless the caller names one."""
    import torch
    if stream is not None and dev is not None and dev != getattr(stream, "device_index", dev):
        raise ValueError("%s: the stream is on GPU %d, the tensors on GPU %d" % (where, stream.device_index, dev))
    if dev is None or dev == torch.cuda.current_device():
        code = fn(*args, _raw_stream(dev) if stream is None and dev is not None else _stream(stream))
    else:
        with torch.cuda.device(dev):
            code = fn(*args, _stream(stream))
    if code != DP_OK:
        raise DPError(code, where)


def _raw_stream(dev: int) -> int:
    """The handle of torch's current stream on GPU dev, without the stream object where torch offers that (it takes
    0.1 us instead of 1.1, of a call's 6)."""
    import torch
    get = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return get(dev) if get is not None else torch.cuda.current_stream(dev).cuda_stream


def _check(code: int, where: str):
    if code != DP_OK:
        raise DPError(code, where)


# ---------------------------------------------------------------------------
# per-sample gradients
# ---------------------------------------------------------------------------

def dp_grad_sample_linear_workspace_bytes(N, T, d_in, d_out, dt) -> int:
    return lib().dp_grad_sample_linear_workspace_bytes(N, T, d_in, d_out, dt)


def dp_grad_sample_linear(A, B, dt, N, T, d_in, d_out, scale, gW, gb=None, sqnorm=None, status=None,
                          ws=None, stream=None):
    _check(lib().dp_grad_sample_linear(_ptr(A), _ptr(B), dt, N, T, d_in, d_out, scale, _ptr(gW), _ptr(gb),
                                       _ptr(sqnorm), _ptr(status), _ptr(ws), _nbytes(ws), _stream(stream)),
           "dp_grad_sample_linear")


def dp_grad_sample_linear_noalloc_max_bytes() -> int:
    return lib().dp_grad_sample_linear_noalloc_max_bytes()


def dp_grad_sample_linear_noalloc(A, B, dt, N, T, d_in, d_out, scale, gW, gb=None, sqnorm=None, status=None,
                                  stream=None):
    _check(lib().dp_grad_sample_linear_noalloc(_ptr(A), _ptr(B), dt, N, T, d_in, d_out, scale, _ptr(gW),
                                               _ptr(gb), _ptr(sqnorm), _ptr(status), _stream(stream)),
           "dp_grad_sample_linear_noalloc")


def dp_grad_sample_conv2d_workspace_bytes(N, Cin, H, W, Cout, kh, kw, sh, sw, ph, pw) -> int:
    return lib().dp_grad_sample_conv2d_workspace_bytes(N, Cin, H, W, Cout, kh, kw, sh, sw, ph, pw)


def dp_grad_sample_conv2d(X, GY, dt, N, Cin, H, W, Cout, Ho, Wo, kh, kw, sh, sw, ph, pw, dh, dw, groups,
                          scale, gW, gb=None, sqnorm=None, status=None, ws=None, stream=None):
    _check(lib().dp_grad_sample_conv2d(_ptr(X), _ptr(GY), dt, N, Cin, H, W, Cout, Ho, Wo, kh, kw, sh, sw, ph,
                                       pw, dh, dw, groups, scale, _ptr(gW), _ptr(gb), _ptr(sqnorm),
                                       _ptr(status), _ptr(ws), _nbytes(ws), _stream(stream)),
           "dp_grad_sample_conv2d")


DP_CONV_AUTO, DP_CONV_TILED, DP_CONV_ROWS = 0, 1, 2


def dp_conv2d_set_path(path: int) -> int:
    """Process-wide kernel choice of dp_grad_sample_conv2d; returns the previous one."""
    prev = lib().dp_conv2d_set_path(path)
    if prev < 0:
        raise ValueError("unknown conv2d path %r" % (path,))
    return prev


DP_CONV_KERNEL_SMALL, DP_CONV_KERNEL_ROWS, DP_CONV_KERNEL_TILED = 0, 1, 2


def dp_conv2d_kernel_choice(N, Cin, H, W, Cout, kh, kw, sh, sw, ph, pw) -> int:
    """The conv kernel dp_grad_sample_conv2d would run for this shape now."""
    return lib().dp_conv2d_kernel_choice(N, Cin, H, W, Cout, kh, kw, sh, sw, ph, pw)


def dp_grad_sample_embedding_workspace_bytes(N, T) -> int:
    return lib().dp_grad_sample_embedding_workspace_bytes(N, T)


def dp_grad_sample_embedding(ids, B, dt, N, T, V, D, scale, row_ptr, uniq_ids, rows, cap, sqnorm=None,
                             status=None, ws=None, stream=None):
    _check(lib().dp_grad_sample_embedding(_ptr(ids), _ptr(B), dt, N, T, V, D, scale, _ptr(row_ptr),
                                          _ptr(uniq_ids), _ptr(rows), cap, _ptr(sqnorm), _ptr(status),
                                          _ptr(ws), _nbytes(ws), _stream(stream)),
           "dp_grad_sample_embedding")


def dp_embedding_lookup(ids, E, dt, N, T, V, D, scale, Y, dt_y, status=None, stream=None):
    import torch
    dev, p = _tensors("dp_embedding_lookup", ("ids", ids, torch.int64, N * T), ("E", E, _tdtype(dt), V * D),
                      ("Y", Y, _tdtype(dt_y), N * T * D), ("status", status, torch.int32, 1))
    _run("dp_embedding_lookup", dev, lib().dp_embedding_lookup, p[0], p[1], dt, N, T, V, D, scale, p[2], dt_y, p[3],
         stream=stream)


DP_ACT_SILU, DP_ACT_GELU_TANH = 0, 1


def dp_gated_ffn_forward_workspace_bytes(M, d_in, d_ff, dt) -> int:
    return lib().dp_gated_ffn_forward_workspace_bytes(M, d_in, d_ff, dt)


def dp_gated_ffn_forward(X, Wg, Wu, dt, M, d_in, d_ff, act, H, G=None, U=None, ws=None, stream=None):
    t, k, n = _tdtype(dt), d_ff * d_in, M * d_ff
    dev, p = _tensors("dp_gated_ffn_forward", ("X", X, t, M * d_in), ("Wg", Wg, t, k), ("Wu", Wu, t, k), ("H", H, t, n),
                      ("G", G, t, n), ("U", U, t, n), ("ws", ws, None, 0))
    _run("dp_gated_ffn_forward", dev, lib().dp_gated_ffn_forward, p[0], p[1], p[2], dt, M, d_in, d_ff, act, p[3], p[4],
         p[5], p[6], _nbytes(ws), stream=stream)


def dp_gated_ffn_backward_workspace_bytes(M, d_in, d_ff, dt) -> int:
    return lib().dp_gated_ffn_backward_workspace_bytes(M, d_in, d_ff, dt)


def dp_gated_ffn_backward(dH, G, U, Wg, Wu, dt, M, d_in, d_ff, act, BG, BU, dX=None, ws=None, stream=None):
    t, k, n = _tdtype(dt), d_ff * d_in, M * d_ff
    dev, p = _tensors("dp_gated_ffn_backward", ("dH", dH, t, n), ("G", G, t, n), ("U", U, t, n), ("Wg", Wg, t, k),
                      ("Wu", Wu, t, k), ("BG", BG, t, n), ("BU", BU, t, n), ("dX", dX, t, M * d_in), ("ws", ws, None, 0))
    _run("dp_gated_ffn_backward", dev, lib().dp_gated_ffn_backward, p[0], p[1], p[2], p[3], p[4], dt, M, d_in, d_ff, act,
         p[5], p[6], p[7], p[8], _nbytes(ws), stream=stream)


DP_ROTARY_HALVES, DP_ROTARY_ADJACENT = 0, 1


def dp_rotary(X, dt, N, T, H, D, ldx, pos, sections, freq, layout, inverse, Y, ldy, stream=None):
    """sections: a list of pairs per axis."""
    import torch
    where, axes = "dp_rotary", len(sections)
    counts = (ctypes.c_int64 * max(axes, 1))(*sections)
    dev, p = _tensors(where, ("pos", pos, torch.int64, axes * N * T), ("freq", freq, torch.float64, sum(sections)))
    dev, r = _rows(where, dev, _tdtype(dt), ("X", X, N, T, ldx, H * D), ("Y", Y, N, T, ldy, H * D))
    _run(where, dev, lib().dp_rotary, r[0], dt, N, T, H, D, ldx, p[0], ctypes.addressof(counts), axes, p[1], layout,
         1 if inverse else 0, r[1], ldy, stream=stream)


def dp_attention_forward_workspace_bytes(a) -> int:
    return lib().dp_attention_forward_workspace_bytes(ctypes.addressof(a))


def _attention_tensors(where, a, lse, ws, rows):
    """rows: (name, tensor, positions, ld, heads)."""
    import torch
    dev, p = _tensors(where, ("lse", lse, torch.float32, a.N * a.Hq * a.Tq), ("ws", ws, None, 0))
    on = getattr(a, "dev", None)
    if dev is not None and on is not None and dev != on:
        raise ValueError("%s: lse or ws is on GPU %d, the masks on GPU %d" % (where, dev, on))
    dev, r = _rows(where, on if dev is None else dev, _tdtype(a.dt), *[(n, x, a.N, T, ld, H * a.D) for n, x, T, ld, H in rows])
    return dev, p, r


def dp_attention_forward(a, Q, K, V, O, lse=None, ws=None, stream=None):
    dev, p, r = _attention_tensors("dp_attention_forward", a, lse, ws,
                                   (("Q", Q, a.Tq, a.ldq, a.Hq), ("K", K, a.Tk, a.ldk, a.Hk), ("V", V, a.Tk, a.ldv, a.Hk),
                                    ("O", O, a.Tq, a.ldo, a.Hq)))
    _run("dp_attention_forward", dev, lib().dp_attention_forward, ctypes.addressof(a), r[0], r[1], r[2], r[3], p[0], p[1],
         _nbytes(ws), stream=stream)


def dp_attention_backward_workspace_bytes(a) -> int:
    return lib().dp_attention_backward_workspace_bytes(ctypes.addressof(a))


def dp_attention_backward(a, Q, K, V, O, lse, dO, dQ, dK, dV, ws=None, stream=None):
    dev, p, r = _attention_tensors("dp_attention_backward", a, lse, ws,
                                   (("Q", Q, a.Tq, a.ldq, a.Hq), ("K", K, a.Tk, a.ldk, a.Hk), ("V", V, a.Tk, a.ldv, a.Hk),
                                    ("O", O, a.Tq, a.ldo, a.Hq), ("dO", dO, a.Tq, a.ldo, a.Hq),
                                    ("dQ", dQ, a.Tq, a.ldq, a.Hq), ("dK", dK, a.Tk, a.ldk, a.Hk),
                                    ("dV", dV, a.Tk, a.ldv, a.Hk)))
    _run("dp_attention_backward", dev, lib().dp_attention_backward, ctypes.addressof(a), r[0], r[1], r[2], r[3], p[0], r[4],
         r[5], r[6], r[7], p[1], _nbytes(ws), stream=stream)


def dp_distill_loss_workspace_bytes(M, V, K, dt) -> int:
    return lib().dp_distill_loss_workspace_bytes(M, V, K, dt)


def dp_distill_loss(Z, dt, M, V, ids, logits, K, labels, alpha, tau, weight, loss, dZ=None, status=None, ws=None,
                    stream=None):
    import torch
    t, f = _tdtype(dt), torch.float32
    dev, p = _tensors("dp_distill_loss", ("Z", Z, t, M * V), ("ids", ids, torch.int64, M * K), ("logits", logits, f, M * K),
                      ("labels", labels, torch.int64, M), ("weight", weight, f, M), ("loss", loss, f, M), ("dZ", dZ, t, M * V),
                      ("status", status, torch.int32, 1), ("ws", ws, None, 0))
    _run("dp_distill_loss", dev, lib().dp_distill_loss, p[0], dt, M, V, p[1], p[2], K, p[3], alpha, tau, p[4], p[5], p[6],
         p[7], p[8], _nbytes(ws), stream=stream)


def dp_lstm_backward(gates, c, W_hh, dh_out, dh_last, N, T, H, delta, status=None, stream=None):
    _check(lib().dp_lstm_backward(_ptr(gates), _ptr(c), _ptr(W_hh), _ptr(dh_out), _ptr(dh_last), N, T, H,
                                  _ptr(delta), _ptr(status), _stream(stream)), "dp_lstm_backward")


def dp_grad_sample_layernorm_workspace_bytes(N, T, D) -> int:
    return lib().dp_grad_sample_layernorm_workspace_bytes(N, T, D)


def dp_grad_sample_layernorm(xhat, B, dt, N, T, D, scale, ggamma, gbeta, sqnorm=None, status=None, ws=None,
                             stream=None):
    _check(lib().dp_grad_sample_layernorm(_ptr(xhat), _ptr(B), dt, N, T, D, scale, _ptr(ggamma), _ptr(gbeta),
                                          _ptr(sqnorm), _ptr(status), _ptr(ws), _nbytes(ws),
                                          _stream(stream)),
           "dp_grad_sample_layernorm")


def dp_grad_sample_groupnorm_workspace_bytes(N, C, P) -> int:
    return lib().dp_grad_sample_groupnorm_workspace_bytes(N, C, P)


def dp_grad_sample_groupnorm(xhat, B, dt, N, C, P, scale, ggamma, gbeta=None, sqnorm=None, status=None, ws=None,
                             stream=None):
    _check(lib().dp_grad_sample_groupnorm(_ptr(xhat), _ptr(B), dt, N, C, P, scale, _ptr(ggamma), _ptr(gbeta),
                                          _ptr(sqnorm), _ptr(status), _ptr(ws), _nbytes(ws),
                                          _stream(stream)),
           "dp_grad_sample_groupnorm")


# ---------------------------------------------------------------------------
# norms and clipping
# ---------------------------------------------------------------------------

def dp_per_sample_norms(sqnorm, n_layers, N, norm, status=None, stream=None):
    _check(lib().dp_per_sample_norms(_ptr(sqnorm), n_layers, N, _ptr(norm), _ptr(status), _stream(stream)),
           "dp_per_sample_norms")


def dp_per_sample_norms_active(sqnorm, n_layers, N, n_active, norm, status=None, stream=None):
    _check(lib().dp_per_sample_norms_active(_ptr(sqnorm), n_layers, N, _ptr(n_active), _ptr(norm), _ptr(status),
                                            _stream(stream)), "dp_per_sample_norms_active")


def dp_sqnorm_from_grads(G, N, numel, sqnorm, status=None, stream=None):
    _check(lib().dp_sqnorm_from_grads(_ptr(G), N, numel, _ptr(sqnorm), _ptr(status), _stream(stream)),
           "dp_sqnorm_from_grads")


def dp_clip_factors(norm, N, C, c, status=None, stream=None):
    _check(lib().dp_clip_factors(_ptr(norm), N, C, _ptr(c), _ptr(status), _stream(stream)), "dp_clip_factors")


def dp_clip_accumulate_workspace_bytes(N, numel) -> int:
    return lib().dp_clip_accumulate_workspace_bytes(N, numel)


def dp_clip_accumulate(G, norm, C, N, numel, sum, c_out=None, status=None, ws=None, stream=None):
    _check(lib().dp_clip_accumulate(_ptr(G), _ptr(norm), C, N, numel, _ptr(sum), _ptr(c_out), _ptr(status),
                                    _ptr(ws), _nbytes(ws), _stream(stream)),
           "dp_clip_accumulate")


def dp_clip_accumulate_linear_workspace_bytes(N, T, d_in, d_out, dt) -> int:
    return lib().dp_clip_accumulate_linear_workspace_bytes(N, T, d_in, d_out, dt)


def dp_clip_accumulate_linear(A, B, dt, N, T, d_in, d_out, scale, norm, C, sumW, sumb=None, status=None,
                              ws=None, stream=None):
    _check(lib().dp_clip_accumulate_linear(_ptr(A), _ptr(B), dt, N, T, d_in, d_out, scale, _ptr(norm), C,
                                           _ptr(sumW), _ptr(sumb), _ptr(status), _ptr(ws), _nbytes(ws),
                                           _stream(stream)),
           "dp_clip_accumulate_linear")


def dp_clip_accumulate_linear_many_workspace_bytes(items, count, dt, N) -> int:
    return lib().dp_clip_accumulate_linear_many_workspace_bytes(ctypes.cast(items, ctypes.c_void_p), count, dt, N)


def dp_clip_accumulate_linear_many(items, count, dt, N, norm, C, status=None, ws=None, stream=None):
    _check(lib().dp_clip_accumulate_linear_many(ctypes.cast(items, ctypes.c_void_p), count, dt, N, _ptr(norm), C,
                                                _ptr(status), _ptr(ws), _nbytes(ws), _stream(stream)),
           "dp_clip_accumulate_linear_many")


def dp_ghost_norm_linear_workspace_bytes(N, T, d_in, d_out) -> int:
    return lib().dp_ghost_norm_linear_workspace_bytes(N, T, d_in, d_out)


def dp_ghost_norm_linear(A, B, dt, N, T, d_in, d_out, scale, bias, sqnorm, status=None, ws=None, stream=None):
    _check(lib().dp_ghost_norm_linear(_ptr(A), _ptr(B), dt, N, T, d_in, d_out, scale, 1 if bias else 0,
                                      _ptr(sqnorm), _ptr(status), _ptr(ws), _nbytes(ws), _stream(stream)),
           "dp_ghost_norm_linear")


def dp_ghost_norm_linear_many_workspace_bytes(items, count, N) -> int:
    return lib().dp_ghost_norm_linear_many_workspace_bytes(ctypes.cast(items, ctypes.c_void_p), count, N)


def dp_ghost_norm_linear_many(items, count, dt, N, status=None, ws=None, stream=None):
    _check(lib().dp_ghost_norm_linear_many(ctypes.cast(items, ctypes.c_void_p), count, dt, N, _ptr(status),
                                           _ptr(ws), _nbytes(ws), _stream(stream)),
           "dp_ghost_norm_linear_many")


def dp_grad_sample_layernorm_many_workspace_bytes(items, count, N, dt) -> int:
    return lib().dp_grad_sample_layernorm_many_workspace_bytes(ctypes.cast(items, ctypes.c_void_p), count, N, dt)


def dp_grad_sample_layernorm_many(items, count, dt, N, status=None, ws=None, stream=None):
    _check(lib().dp_grad_sample_layernorm_many(ctypes.cast(items, ctypes.c_void_p), count, dt, N, _ptr(status),
                                               _ptr(ws), _nbytes(ws), _stream(stream)),
           "dp_grad_sample_layernorm_many")


def dp_grad_sample_many_grouped(items, k, dt, N) -> bool:
    """Whether layer k of a dp_layer_grad array goes into the grouped launch."""
    return bool(lib().dp_grad_sample_many_grouped(ctypes.cast(ctypes.byref(items[k]), ctypes.c_void_p), dt, N))


def dp_grad_sample_many_workspace_bytes(items, count, dt, N) -> int:
    return lib().dp_grad_sample_many_workspace_bytes(ctypes.cast(items, ctypes.c_void_p), count, dt, N)


def dp_grad_sample_many(items, count, dt, N, status=None, ws=None, stream=None):
    _check(lib().dp_grad_sample_many(ctypes.cast(items, ctypes.c_void_p), count, dt, N, _ptr(status), _ptr(ws),
                                     _nbytes(ws), _stream(stream)),
           "dp_grad_sample_many")


def dp_clip_accumulate_embedding_workspace_bytes(N, V) -> int:
    return lib().dp_clip_accumulate_embedding_workspace_bytes(N, V)


def dp_clip_accumulate_embedding(row_ptr, uniq_ids, rows, cap, norm, C, N, V, D, sum, status=None, ws=None,
                                 stream=None):
    _check(lib().dp_clip_accumulate_embedding(_ptr(row_ptr), _ptr(uniq_ids), _ptr(rows), cap, _ptr(norm), C, N,
                                              V, D, _ptr(sum), _ptr(status), _ptr(ws), _nbytes(ws),
                                              _stream(stream)),
           "dp_clip_accumulate_embedding")


def dp_clip_accumulate_tokens_workspace_bytes(N, T, V, D, dt) -> int:
    return lib().dp_clip_accumulate_tokens_workspace_bytes(N, T, V, D, dt)


def dp_clip_accumulate_tokens(ids, B, dt, N, T, V, D, scale, norm, C, sum, status=None, ws=None, stream=None):
    import torch
    dev, p = _tensors("dp_clip_accumulate_tokens", ("ids", ids, torch.int64, N * T), ("B", B, _tdtype(dt), N * T * D),
                      ("norm", norm, torch.float32, N), ("sum", sum, torch.float32, V * D),
                      ("status", status, torch.int32, 1), ("ws", ws, None, 0))
    _run("dp_clip_accumulate_tokens", dev, lib().dp_clip_accumulate_tokens, p[0], p[1], dt, N, T, V, D, scale, p[2], C,
         p[3], p[4], p[5], _nbytes(ws), stream=stream)


def _grad_tensors(where, items, count):
    """Address of a dp_grad_tensor array that holds `count` of them (None: of none)."""
    if count > (0 if items is None else len(items)):
        raise ValueError("%s: %d tensors of an array of %d" % (where, count, 0 if items is None else len(items)))
    return None if items is None else ctypes.addressof(items)


def dp_clip_global_norm_many_workspace_bytes(items, count) -> int:
    return lib().dp_clip_global_norm_many_workspace_bytes(
        _grad_tensors("dp_clip_global_norm_many_workspace_bytes", items, count), count)


def dp_clip_global_norm_many(items, count, C, norm, status=None, ws=None, stream=None):
    import torch
    dev, p = _tensors("dp_clip_global_norm_many", ("norm", norm, torch.float32, 1), ("status", status, torch.int32, 1),
                      ("ws", ws, None, 0))
    where = "dp_clip_global_norm_many"
    at, on = _grad_tensors(where, items, count), getattr(items, "dev", None)
    if dev is not None and on is not None and dev != on:
        raise ValueError("%s: norm, status or ws is on GPU %d, the tensors on GPU %d" % (where, dev, on))
    _run(where, on if dev is None else dev, lib().dp_clip_global_norm_many, at, count, C, p[0], p[1], p[2], _nbytes(ws),
         stream=stream)


# ---------------------------------------------------------------------------
# grouped clip + noise
# ---------------------------------------------------------------------------

def dp_clip_noise_many_workspace_bytes(params, count, N) -> int:
    return lib().dp_clip_noise_many_workspace_bytes(ctypes.cast(params, ctypes.c_void_p), count, N)


def dp_clip_noise_many(params, count, N, norm, C, seed, step, step_dev, sigma, denom, status=None, ws=None,
                       stream=None):
    _check(lib().dp_clip_noise_many(ctypes.cast(params, ctypes.c_void_p), count, N, _ptr(norm), C, seed, step,
                                    _ptr(step_dev), sigma, denom, _ptr(status), _ptr(ws), _nbytes(ws),
                                    _stream(stream)),
           "dp_clip_noise_many")


def dp_norms_clip_noise_workspace_bytes(params, count, N) -> int:
    return lib().dp_norms_clip_noise_workspace_bytes(ctypes.cast(params, ctypes.c_void_p), count, N)


def dp_norms_clip_noise(sqnorm, n_layers, params, count, N, norm, C, seed, step, step_dev, sigma, denom,
                        status=None, ws=None, stream=None):
    _check(lib().dp_norms_clip_noise(_ptr(sqnorm), n_layers, ctypes.cast(params, ctypes.c_void_p), count, N,
                                     _ptr(norm), C, seed, step, _ptr(step_dev), sigma, denom, _ptr(status),
                                     _ptr(ws), _nbytes(ws), _stream(stream)),
           "dp_norms_clip_noise")


def dp_norms_clip_noise_sched(sqnorm, n_layers, params, count, N, norm, C, seed, step, step_dev, sigma_table,
                              denom, status=None, ws=None, stream=None, n_active=None):
    """dp_norms_clip_noise with the noise multiplier of step t read from
    sigma_table[min(t, len - 1)] (a device float tensor) on the device, and
    optionally the active batch size from n_active (a device int64)."""
    _check(lib().dp_norms_clip_noise_sched(_ptr(sqnorm), n_layers, ctypes.cast(params, ctypes.c_void_p), count, N,
                                           _ptr(norm), C, seed, step, _ptr(step_dev), _ptr(sigma_table),
                                           _numel(sigma_table), _ptr(n_active), denom, _ptr(status), _ptr(ws),
                                           _nbytes(ws), _stream(stream)),
           "dp_norms_clip_noise_sched")


def dp_step_advance(step_dev, by=1, stream=None):
    _check(lib().dp_step_advance(_ptr(step_dev), by, _stream(stream)), "dp_step_advance")


# ---------------------------------------------------------------------------
# noise
# ---------------------------------------------------------------------------

def dp_add_noise(sum, out, numel, seed, step, param_index, sigma, C, denom, status=None, stream=None):
    _check(lib().dp_add_noise(_ptr(sum), _ptr(out), numel, seed, step, param_index, sigma, C, denom,
                              _ptr(status), _stream(stream)),
           "dp_add_noise")


def dp_philox_normals(z, raw, numel, seed, step, param_index, stream=None):
    _check(lib().dp_philox_normals(_ptr(z), _ptr(raw), numel, seed, step, param_index, _stream(stream)),
           "dp_philox_normals")
