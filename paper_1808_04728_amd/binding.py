"""ctypes binding of the C ABI in include/cosmoflow.h.

Argument marshalling only: every function here has the name of its C entry
point, turns torch tensors into device pointers and the current torch stream
into a hipStream_t, calls the library and raises ``CfError`` on a non-zero
status.  All computation happens in the HIP kernels of libcosmoflow_hip.so;
if the library is missing this module raises instead of computing anything
another way.
"""
from __future__ import annotations

import ctypes
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libcosmoflow_hip.so")

CF_OK, CF_ERR_INVALID_ARG, CF_ERR_UNSUPPORTED, CF_ERR_ALIGNMENT, CF_ERR_ALIAS, \
    CF_ERR_WORKSPACE, CF_ERR_LAUNCH = range(7)
CF_F32, CF_BF16 = 0, 1
CF_PAD_SAME_TF, CF_PAD_VALID = 0, 1
CF_FUSE_POOL2 = 1
CF_FUSE_MASK = 2
FUSED_FWD, FUSED_BWD_WEIGHT, FUSED_BWD_DATA, FUSED_BWD_WEIGHT_DZ = 1, 2, 4, 8

STATUS_NAMES = {0: "CF_OK", 1: "CF_ERR_INVALID_ARG", 2: "CF_ERR_UNSUPPORTED", 3: "CF_ERR_ALIGNMENT",
                4: "CF_ERR_ALIAS", 5: "CF_ERR_WORKSPACE", 6: "CF_ERR_LAUNCH"}

# every symbol the header declares
EXPORTS = [
    "cf_version", "cf_last_error", "cf_conv3d_out_shape", "cf_conv3d_fwd", "cf_conv3d_bwd_data",
    "cf_conv3d_bwd_weight_workspace_size", "cf_conv3d_bwd_weight", "cf_bias_lrelu_fwd",
    "cf_bias_lrelu_bwd_workspace_size", "cf_bias_lrelu_bwd", "cf_avgpool3d_fwd", "cf_avgpool3d_bwd",
    "cf_conv3d_fused_supported", "cf_conv3d_mask_bytes", "cf_conv3d_fwd_fused",
    "cf_conv3d_bwd_weight_fused_workspace_size", "cf_conv3d_bwd_weight_fused", "cf_conv3d_bwd_weight_fused_dz",
    "cf_conv3d_bwd_data_fused", "cf_reduce_partials", "cf_conv3d_bwd_weight_deferred", "cf_bias_lrelu_bwd_deferred",
    "cf_conv3d_bwd_weight_fused_deferred", "cf_adam_larc_workspace_size", "cf_adam_larc_step",
    "cf_fc_fwd_workspace_size", "cf_fc_fwd", "cf_fc_bwd_data", "cf_fc_bwd_weight", "cf_mse_loss",
    "cf_fc_head_workspace_size", "cf_fc_head",
    "cf_conv3d_bwd_weight_noalloc", "cf_avgpool3d_lrelu_bwd_workspace_size", "cf_avgpool3d_lrelu_bwd",
    "cf_avgpool3d_lrelu_bwd_deferred", "cf_conv3d_bwd_fused", "cf_conv3d_bwd_fused_deferred",
    "cf_conv3d_bwd", "cf_conv3d_bwd_deferred",
    "cf_layernorm_fwd_workspace_size", "cf_layernorm_fwd", "cf_layernorm_bwd_workspace_size", "cf_layernorm_bwd",
    "cf_newton_schulz_workspace_size", "cf_newton_schulz", "cf_muon_workspace_size", "cf_muon_step",
    "cf_groupnorm_fwd_workspace_size", "cf_groupnorm_fwd", "cf_groupnorm_bwd_workspace_size", "cf_groupnorm_bwd",
    "cf_linear_fwd_workspace_size", "cf_linear_fwd", "cf_linear_bwd_data_workspace_size", "cf_linear_bwd_data",
    "cf_linear_bwd_weight_workspace_size", "cf_linear_bwd_weight", "cf_adamw_step",
]


class CfError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"{STATUS_NAMES.get(status, status)}: {msg}")
        self.status = status


class cf_conv3d_desc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in
                ("n", "d", "h", "w", "c_in", "c_out", "kd", "kh", "kw", "sd", "sh", "sw", "pad", "dtype")]


class cf_reduction(ctypes.Structure):
    _fields_ = [("part", ctypes.c_void_p), ("out", ctypes.c_void_p), ("rows", ctypes.c_int32),
                ("cols", ctypes.c_int32)]


CF_MAX_PENDING = 4


class cf_adam_larc_hparams(ctypes.Structure):
    _fields_ = [("eta0", ctypes.c_double), ("eta_min", ctypes.c_double), ("t_decay", ctypes.c_int64),
                ("beta1", ctypes.c_double), ("beta2", ctypes.c_double), ("eps_hat", ctypes.c_double),
                ("larc_coef", ctypes.c_double), ("larc_fallback", ctypes.c_double), ("larc_clip", ctypes.c_double)]


CF_ADAM_MAX_GROUPS = 128
#: the paper's hyperparameters (Section III-B); t_decay is the caller's choice
PAPER_HPARAMS = dict(eta0=2e-3, eta_min=1e-4, beta1=0.9, beta2=0.999, eps_hat=1e-8,
                     larc_coef=0.002, larc_fallback=6.25e-5, larc_clip=1.0)


def make_hparams(t_decay, **kw) -> cf_adam_larc_hparams:
    h = dict(PAPER_HPARAMS)
    h.update(kw)
    return cf_adam_larc_hparams(h["eta0"], h["eta_min"], int(t_decay), h["beta1"], h["beta2"], h["eps_hat"],
                                h["larc_coef"], h["larc_fallback"], h["larc_clip"])


class cf_matrix(ctypes.Structure):
    _fields_ = [("offset", ctypes.c_int64), ("rows", ctypes.c_int32), ("cols", ctypes.c_int32)]


class cf_ns_hparams(ctypes.Structure):
    _fields_ = [("a", ctypes.c_double), ("b", ctypes.c_double), ("c", ctypes.c_double), ("eps", ctypes.c_double),
                ("steps", ctypes.c_int32)]


class cf_muon_hparams(ctypes.Structure):
    _fields_ = [("eta0", ctypes.c_double), ("eta_min", ctypes.c_double), ("t_decay", ctypes.c_int64),
                ("mu", ctypes.c_double), ("weight_decay", ctypes.c_double), ("ns", cf_ns_hparams),
                ("nesterov", ctypes.c_int32), ("scale", ctypes.c_int32)]


CF_NS_MAX_STEPS = 32
CF_MUON_SCALE_SHAPE, CF_MUON_SCALE_RMS = 0, 1
#: the usual quintic: singular values from 1e-2 on end between 0.7 and 1.2 after five steps
NS_COEF = (3.4445, -4.7750, 2.0315)


def make_ns_hparams(steps=5, coef=NS_COEF, eps=1e-7) -> cf_ns_hparams:
    return cf_ns_hparams(*(float(x) for x in coef), float(eps), int(steps))


def make_muon_hparams(t_decay, eta0=0.02, eta_min=0.001, mu=0.95, weight_decay=0.0, steps=5, coef=NS_COEF, eps=1e-7,
                      nesterov=True, scale=CF_MUON_SCALE_SHAPE) -> cf_muon_hparams:
    return cf_muon_hparams(eta0, eta_min, int(t_decay), mu, weight_decay, make_ns_hparams(steps, coef, eps), int(nesterov),
                           int(scale))


def make_matrices(offsets, rows, cols):
    """Host array of cf_matrix: matrix l is rows[l] x cols[l] values from offsets[l] on."""
    if not len(offsets) == len(rows) == len(cols):
        raise ValueError("make_matrices: offsets, rows and cols differ in length")
    return (cf_matrix * len(offsets))(*[cf_matrix(int(o), int(r), int(c)) for o, r, c in zip(offsets, rows, cols)])


CF_ACT_NONE, CF_ACT_LRELU, CF_ACT_SILU, CF_ACT_GELU = range(4)
_ACTS = {"none": CF_ACT_NONE, "lrelu": CF_ACT_LRELU, "silu": CF_ACT_SILU, "gelu": CF_ACT_GELU}

#: values that share a scale where AdamW's moments are held in 8 bits
CF_ADAMW_BLOCK = 256


class cf_adamw_tensor(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("p", "g", "m", "v", "m_scale", "v_scale", "p16")] + [
        ("count", ctypes.c_int64), ("weight_decay", ctypes.c_float), ("g_dtype", ctypes.c_int32)]


class cf_adamw_hparams(ctypes.Structure):
    _fields_ = [("eta0", ctypes.c_double), ("eta_min", ctypes.c_double), ("t_decay", ctypes.c_int64),
                ("beta1", ctypes.c_double), ("beta2", ctypes.c_double), ("eps", ctypes.c_double),
                ("seed", ctypes.c_uint32)]


def make_adamw_hparams(t_decay, eta0=1e-3, eta_min=1e-4, beta1=0.9, beta2=0.999, eps=1e-8, seed=0) -> cf_adamw_hparams:
    return cf_adamw_hparams(eta0, eta_min, int(t_decay), beta1, beta2, eps, int(seed) & 0xFFFFFFFF)


def make_adamw_tensors(tensors):
    """Host array of cf_adamw_tensor from one dict a tensor: p (fp32), g (fp32 or bf16), m, v
    (fp32, or a byte a value with m_scale and v_scale), p16 (bf16 copy of p), weight_decay;
    all contiguous and on one device (ValueError).  The dicts' tensors have to live as long as
    the array is used."""
    out = (cf_adamw_tensor * max(len(tensors), 1))()
    device = tensors[0]["p"].device if tensors else None
    for l, (a, d) in enumerate(zip(out, tensors)):
        p = d["p"]
        n = p.numel()
        eight = d.get("m_scale") is not None
        blocks = -(-n // CF_ADAMW_BLOCK)
        for name, size, types in (("p", n, (torch.float32,)), ("g", n, (torch.float32, torch.bfloat16)),
                                  ("m", n, (torch.float8_e4m3fn, torch.uint8) if eight else (torch.float32,)),
                                  ("v", n, (torch.float8_e4m3fn, torch.uint8) if eight else (torch.float32,)),
                                  ("m_scale", blocks, (torch.float32,)), ("v_scale", blocks, (torch.float32,)),
                                  ("p16", n, (torch.bfloat16,))):
            x = d.get(name)
            if x is None:
                if name in ("p16", "m_scale", "v_scale"):
                    continue
                raise ValueError(f"tensor {l}, {name}: missing")
            if x.numel() != size or x.dtype not in types or x.device != device or not x.is_contiguous():
                raise ValueError(f"tensor {l}, {name}: {x.numel()} {x.dtype} on {x.device}, or not contiguous")
            setattr(a, name, x.data_ptr())
        a.count, a.weight_decay, a.g_dtype = n, float(d.get("weight_decay", 0.0)), dtype_code(d["g"].dtype)
    return len(tensors), out


_lib = None


def lib():
    """Load libcosmoflow_hip.so (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_1808_04728_amd.build` "
                          "(there is no fallback implementation)")
    L = ctypes.CDLL(LIB_PATH)
    vp, i32, i64, f32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t
    D = ctypes.POINTER(cf_conv3d_desc)
    sig = {
        "cf_version": ([], ctypes.c_char_p),
        "cf_last_error": ([], ctypes.c_char_p),
        "cf_conv3d_out_shape": ([D, ctypes.POINTER(i32)], ctypes.c_int),
        "cf_conv3d_fwd": ([D, vp, vp, vp, vp], ctypes.c_int),
        "cf_conv3d_bwd_data": ([D, vp, vp, vp, vp], ctypes.c_int),
        "cf_conv3d_bwd_weight_workspace_size": ([D], sz),
        "cf_conv3d_bwd_weight": ([D, vp, vp, vp, vp, sz, vp], ctypes.c_int),
        "cf_conv3d_bwd_weight_noalloc": ([D, vp, vp, vp, vp], ctypes.c_int),
        "cf_bias_lrelu_fwd": ([i64, i32, i32, vp, vp, f32, vp, vp], ctypes.c_int),
        "cf_bias_lrelu_bwd_workspace_size": ([i64, i32], sz),
        "cf_bias_lrelu_bwd": ([i64, i32, i32, vp, vp, f32, vp, vp, vp, sz, vp], ctypes.c_int),
        "cf_avgpool3d_fwd": ([i32] * 8 + [vp, vp, vp], ctypes.c_int),
        "cf_avgpool3d_bwd": ([i32] * 8 + [vp, vp, vp], ctypes.c_int),
        "cf_avgpool3d_lrelu_bwd_workspace_size": ([i32] * 5, sz),
        "cf_avgpool3d_lrelu_bwd": ([i32] * 6 + [vp, vp, f32, vp, vp, vp, sz, vp], ctypes.c_int),
        "cf_avgpool3d_lrelu_bwd_deferred": ([i32] * 6 + [vp, vp, f32, vp, vp, vp, sz, ctypes.POINTER(cf_reduction),
                                                         ctypes.POINTER(i32), vp], ctypes.c_int),
        "cf_conv3d_fused_supported": ([D, ctypes.c_uint32], i32),
        "cf_conv3d_mask_bytes": ([D], sz),
        "cf_conv3d_fwd_fused": ([D, vp, vp, vp, f32, ctypes.c_uint32, vp, vp, vp], ctypes.c_int),
        "cf_conv3d_bwd_weight_fused_workspace_size": ([D, ctypes.c_uint32], sz),
        "cf_conv3d_bwd_weight_fused": ([D, vp, vp, vp, f32, ctypes.c_uint32, vp, vp, vp, sz, vp], ctypes.c_int),
        "cf_conv3d_bwd_weight_fused_dz": ([D, vp, vp, vp, f32, ctypes.c_uint32, vp, vp, vp, vp, sz, vp],
                                          ctypes.c_int),
        "cf_conv3d_bwd_data_fused": ([D, vp, vp, vp, f32, ctypes.c_uint32, vp, vp], ctypes.c_int),
        "cf_conv3d_bwd": ([D, vp, vp, vp, vp, vp, vp, sz, vp], ctypes.c_int),
        "cf_conv3d_bwd_deferred": ([D, vp, vp, vp, vp, vp, vp, sz, ctypes.POINTER(cf_reduction),
                                    ctypes.POINTER(i32), vp], ctypes.c_int),
        "cf_conv3d_bwd_fused": ([D, vp, vp, vp, vp, f32, ctypes.c_uint32, vp, vp, vp, vp, sz, vp], ctypes.c_int),
        "cf_conv3d_bwd_fused_deferred": ([D, vp, vp, vp, vp, f32, ctypes.c_uint32, vp, vp, vp, vp, sz,
                                          ctypes.POINTER(cf_reduction), ctypes.POINTER(i32), vp], ctypes.c_int),
        "cf_reduce_partials": ([i32, ctypes.POINTER(cf_reduction), vp], ctypes.c_int),
        "cf_conv3d_bwd_weight_deferred": ([D, vp, vp, vp, vp, sz, ctypes.POINTER(cf_reduction),
                                           ctypes.POINTER(i32), vp], ctypes.c_int),
        "cf_bias_lrelu_bwd_deferred": ([i64, i32, i32, vp, vp, f32, vp, vp, vp, sz, ctypes.POINTER(cf_reduction),
                                        ctypes.POINTER(i32), vp], ctypes.c_int),
        "cf_conv3d_bwd_weight_fused_deferred": ([D, vp, vp, vp, f32, ctypes.c_uint32, vp, vp, vp, vp, sz,
                                                 ctypes.POINTER(cf_reduction), ctypes.POINTER(i32), vp],
                                                ctypes.c_int),
        "cf_layernorm_fwd_workspace_size": ([i64, i32, i32], sz),
        "cf_layernorm_fwd": ([i64, i32, i32, vp, vp, vp, f32, vp, vp, vp, vp, sz, vp], ctypes.c_int),
        "cf_layernorm_bwd_workspace_size": ([i64, i32, i32], sz),
        "cf_layernorm_bwd": ([i64, i32, i32] + [vp] * 9 + [sz, vp], ctypes.c_int),
        "cf_newton_schulz_workspace_size": ([i32, ctypes.POINTER(cf_matrix), i32], sz),
        "cf_newton_schulz": ([i32, ctypes.POINTER(cf_matrix), i32, ctypes.POINTER(cf_ns_hparams), vp, vp, vp, sz, vp],
                             ctypes.c_int),
        "cf_muon_workspace_size": ([i32, ctypes.POINTER(cf_matrix)], sz),
        "cf_muon_step": ([i32, ctypes.POINTER(cf_matrix), i64, ctypes.POINTER(cf_muon_hparams), vp, vp, vp, vp, vp, sz, vp],
                         ctypes.c_int),
        "cf_groupnorm_fwd_workspace_size": ([i32, i64, i32, i32, i32], sz),
        "cf_groupnorm_fwd": ([i32, i64, i32, i32, i32, vp, vp, vp, f32, i32, f32, vp, vp, vp, vp, sz, vp], ctypes.c_int),
        "cf_groupnorm_bwd_workspace_size": ([i32, i64, i32, i32, i32], sz),
        "cf_groupnorm_bwd": ([i32, i64, i32, i32, i32] + [vp] * 6 + [i32, f32, vp, vp, vp, vp, sz, vp], ctypes.c_int),
        "cf_linear_fwd_workspace_size": ([i32] * 4, sz),
        "cf_linear_fwd": ([i32] * 4 + [vp, vp, vp, i32, f32, vp, vp, vp, vp, sz, vp], ctypes.c_int),
        "cf_linear_bwd_data_workspace_size": ([i32] * 4, sz),
        "cf_linear_bwd_data": ([i32] * 4 + [vp, vp, vp, vp, i32, f32, vp, vp, sz, vp], ctypes.c_int),
        "cf_linear_bwd_weight_workspace_size": ([i32] * 4, sz),
        "cf_linear_bwd_weight": ([i32] * 4 + [vp, vp, vp, vp, vp, sz, vp], ctypes.c_int),
        "cf_adamw_step": ([i32, ctypes.POINTER(cf_adamw_tensor), i64, ctypes.POINTER(cf_adamw_hparams), vp], ctypes.c_int),
        "cf_adam_larc_workspace_size": ([i32, ctypes.POINTER(i64)], sz),
        "cf_adam_larc_step": ([i32, ctypes.POINTER(i64), i64, ctypes.POINTER(cf_adam_larc_hparams), vp, vp, vp, vp,
                               vp, vp, sz, vp], ctypes.c_int),
        "cf_fc_fwd_workspace_size": ([i32, i32, i32], sz),
        "cf_fc_fwd": ([i32, i32, i32, i32, vp, vp, vp, vp, sz, vp], ctypes.c_int),
        "cf_fc_bwd_data": ([i32, i32, i32, i32, vp, vp, vp, vp], ctypes.c_int),
        "cf_fc_bwd_weight": ([i32, i32, i32, i32, vp, vp, vp, vp], ctypes.c_int),
        "cf_mse_loss": ([i32, i32, i32, vp, vp, vp, vp, vp], ctypes.c_int),
        "cf_fc_head_workspace_size": ([i32, i32, ctypes.POINTER(i32)], sz),
        "cf_fc_head": ([i32, i32, ctypes.POINTER(i32), i32, vp, ctypes.POINTER(vp), ctypes.POINTER(vp), f32, vp,
                        ctypes.POINTER(vp), ctypes.POINTER(vp), ctypes.POINTER(vp), ctypes.POINTER(vp),
                        ctypes.POINTER(vp), vp, vp, sz, vp], ctypes.c_int),
    }
    for name, (args, res) in sig.items():
        f = getattr(L, name)
        f.argtypes = args
        f.restype = res
    _lib = L
    return L


def _check(status: int):
    if status != CF_OK:
        raise CfError(status, lib().cf_last_error().decode())


def _ptr(t):
    """Device pointer of a tensor, or an int/None passed through."""
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


def check_params(own, params):
    """ValueError unless params can stand in for own, the parameters of each layer (a dict of
    tensors a layer): the same layers and names, shapes, dtypes and device, contiguous and
    16-byte aligned."""
    if len(params) != len(own):
        raise ValueError(f"parameters of {len(params)} layers for {len(own)}")
    for i, (o, p) in enumerate(zip(own, params)):
        for k, t in o.items():
            x = p.get(k)
            if not isinstance(x, torch.Tensor):
                raise ValueError(f"layer {i}, {k}: not a tensor")
            if x.shape != t.shape or x.dtype != t.dtype or x.device != t.device:
                raise ValueError(f"layer {i}, {k}: {tuple(x.shape)} {x.dtype} on {x.device}, not {tuple(t.shape)} {t.dtype} on {t.device}")
            if not x.is_contiguous() or x.data_ptr() % 16:
                raise ValueError(f"layer {i}, {k}: not contiguous or not 16-byte aligned")


_raw_current = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def raw_stream(stream):
    """The hipStream_t of a torch stream, an int passed through, or (None) the
    current stream's (asked for by handle: building torch's stream object for it
    took 2.8 us of an 8 us call, this 0.2)."""
    if stream is None:
        if _raw_current is not None and torch.cuda.is_initialized():
            return _raw_current(torch._C._cuda_getDevice())
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


_stream = raw_stream


def dtype_code(dt) -> int:
    if dt in (torch.float32, "f32", CF_F32):
        return CF_F32
    if dt in (torch.bfloat16, "bf16", CF_BF16):
        return CF_BF16
    raise ValueError(f"unsupported dtype {dt}")


def act_code(act) -> int:
    """Code of an activation's name (or code)."""
    if act in _ACTS:
        return _ACTS[act]
    if act in _ACTS.values():
        return int(act)
    raise ValueError(f"unknown activation {act}")


def make_desc(n, dhw, c_in, c_out, k, stride=1, pad="same", dtype=CF_F32) -> cf_conv3d_desc:
    k3 = tuple(k) if isinstance(k, (tuple, list)) else (k,) * 3
    s3 = tuple(stride) if isinstance(stride, (tuple, list)) else (stride,) * 3
    return cf_conv3d_desc(n, *dhw, c_in, c_out, *k3, *s3,
                          CF_PAD_SAME_TF if pad == "same" else CF_PAD_VALID, dtype_code(dtype))


# ---------------------------------------------------------------------------
# entry points (same names as the C ABI)
# ---------------------------------------------------------------------------

def cf_version() -> str:
    return lib().cf_version().decode()


def cf_last_error() -> str:
    return lib().cf_last_error().decode()


def cf_conv3d_out_shape(desc):
    out = (ctypes.c_int32 * 3)()
    _check(lib().cf_conv3d_out_shape(ctypes.byref(desc), out))
    return tuple(out)


def cf_conv3d_fwd(desc, x, w, z, stream=None):
    _check(lib().cf_conv3d_fwd(ctypes.byref(desc), _ptr(x), _ptr(w), _ptr(z), _stream(stream)))


def cf_conv3d_bwd_data(desc, dz, w, dx, stream=None):
    _check(lib().cf_conv3d_bwd_data(ctypes.byref(desc), _ptr(dz), _ptr(w), _ptr(dx), _stream(stream)))


def cf_conv3d_bwd_weight_workspace_size(desc) -> int:
    return int(lib().cf_conv3d_bwd_weight_workspace_size(ctypes.byref(desc)))


def cf_conv3d_bwd_weight(desc, x, dz, dw, ws, ws_bytes=None, stream=None):
    if ws_bytes is None:
        ws_bytes = 0 if ws is None or isinstance(ws, int) else ws.numel() * ws.element_size()
    _check(lib().cf_conv3d_bwd_weight(ctypes.byref(desc), _ptr(x), _ptr(dz), _ptr(dw), _ptr(ws),
                                      ws_bytes, _stream(stream)))


def cf_conv3d_bwd_weight_noalloc(desc, x, dz, dw, stream=None):
    _check(lib().cf_conv3d_bwd_weight_noalloc(ctypes.byref(desc), _ptr(x), _ptr(dz), _ptr(dw), _stream(stream)))


def cf_bias_lrelu_fwd(nvox, c, dtype, z, bias, alpha, y, stream=None):
    _check(lib().cf_bias_lrelu_fwd(nvox, c, dtype_code(dtype), _ptr(z), _ptr(bias), alpha, _ptr(y),
                                   _stream(stream)))


def cf_bias_lrelu_bwd_workspace_size(nvox, c) -> int:
    return int(lib().cf_bias_lrelu_bwd_workspace_size(nvox, c))


def cf_bias_lrelu_bwd(nvox, c, dtype, dy, y, alpha, dz, db, ws, ws_bytes=None, stream=None):
    if ws_bytes is None:
        ws_bytes = 0 if ws is None or isinstance(ws, int) else ws.numel() * ws.element_size()
    _check(lib().cf_bias_lrelu_bwd(nvox, c, dtype_code(dtype), _ptr(dy), _ptr(y), alpha, _ptr(dz), _ptr(db),
                                   _ptr(ws), ws_bytes, _stream(stream)))


def cf_avgpool3d_fwd(n, d, h, w, c, k, s, dtype, y, p, stream=None):
    _check(lib().cf_avgpool3d_fwd(n, d, h, w, c, k, s, dtype_code(dtype), _ptr(y), _ptr(p), _stream(stream)))


def cf_avgpool3d_bwd(n, d, h, w, c, k, s, dtype, dp, dy, stream=None):
    _check(lib().cf_avgpool3d_bwd(n, d, h, w, c, k, s, dtype_code(dtype), _ptr(dp), _ptr(dy), _stream(stream)))


def cf_avgpool3d_lrelu_bwd_workspace_size(n, d, h, w, c) -> int:
    return int(lib().cf_avgpool3d_lrelu_bwd_workspace_size(n, d, h, w, c))


def cf_avgpool3d_lrelu_bwd(n, d, h, w, c, dtype, dp, mask, alpha, dz, db, ws, ws_bytes=None, stream=None):
    if ws_bytes is None:
        ws_bytes = 0 if ws is None or isinstance(ws, int) else ws.numel() * ws.element_size()
    _check(lib().cf_avgpool3d_lrelu_bwd(n, d, h, w, c, dtype_code(dtype), _ptr(dp), _ptr(mask), alpha, _ptr(dz),
                                        _ptr(db), _ptr(ws), ws_bytes, _stream(stream)))


def cf_conv3d_fused_supported(desc, flags=CF_FUSE_POOL2) -> int:
    return int(lib().cf_conv3d_fused_supported(ctypes.byref(desc), flags))


def cf_conv3d_mask_bytes(desc) -> int:
    return int(lib().cf_conv3d_mask_bytes(ctypes.byref(desc)))


def cf_conv3d_fwd_fused(desc, x, w, bias, alpha, flags, out, mask, stream=None):
    _check(lib().cf_conv3d_fwd_fused(ctypes.byref(desc), _ptr(x), _ptr(w), _ptr(bias), alpha, flags, _ptr(out),
                                     _ptr(mask), _stream(stream)))


def cf_conv3d_bwd_weight_fused_workspace_size(desc, flags=CF_FUSE_POOL2) -> int:
    return int(lib().cf_conv3d_bwd_weight_fused_workspace_size(ctypes.byref(desc), flags))


def cf_conv3d_bwd_weight_fused(desc, x, g, mask, alpha, flags, dw, db, ws, ws_bytes=None, stream=None):
    if ws_bytes is None:
        ws_bytes = 0 if ws is None or isinstance(ws, int) else ws.numel() * ws.element_size()
    _check(lib().cf_conv3d_bwd_weight_fused(ctypes.byref(desc), _ptr(x), _ptr(g), _ptr(mask), alpha, flags,
                                            _ptr(dw), _ptr(db), _ptr(ws), ws_bytes, _stream(stream)))


def cf_conv3d_bwd_weight_fused_dz(desc, x, g, mask, alpha, flags, dw, db, dz, ws, ws_bytes=None, stream=None):
    if ws_bytes is None:
        ws_bytes = 0 if ws is None or isinstance(ws, int) else ws.numel() * ws.element_size()
    _check(lib().cf_conv3d_bwd_weight_fused_dz(ctypes.byref(desc), _ptr(x), _ptr(g), _ptr(mask), alpha, flags,
                                               _ptr(dw), _ptr(db), _ptr(dz), _ptr(ws), ws_bytes, _stream(stream)))


def cf_conv3d_bwd_data_fused(desc, g, mask, w, alpha, flags, dx, stream=None):
    _check(lib().cf_conv3d_bwd_data_fused(ctypes.byref(desc), _ptr(g), _ptr(mask), _ptr(w), alpha, flags, _ptr(dx),
                                          _stream(stream)))


def cf_conv3d_bwd(desc, x, dz, w, dw, dx, ws, ws_bytes=None, stream=None):
    if ws_bytes is None:
        ws_bytes = 0 if ws is None or isinstance(ws, int) else ws.numel() * ws.element_size()
    _check(lib().cf_conv3d_bwd(ctypes.byref(desc), _ptr(x), _ptr(dz), _ptr(w), _ptr(dw), _ptr(dx), _ptr(ws),
                               ws_bytes, _stream(stream)))


def cf_conv3d_bwd_fused(desc, x, g, mask, w, alpha, flags, dw, db, dx, ws, ws_bytes=None, stream=None):
    if ws_bytes is None:
        ws_bytes = 0 if ws is None or isinstance(ws, int) else ws.numel() * ws.element_size()
    _check(lib().cf_conv3d_bwd_fused(ctypes.byref(desc), _ptr(x), _ptr(g), _ptr(mask), _ptr(w), alpha, flags,
                                     _ptr(dw), _ptr(db), _ptr(dx), _ptr(ws), ws_bytes, _stream(stream)))


# ---- deferred gradient sums --------------------------------------------------
# The _deferred calls return a list of pending cf_reduction jobs (host
# structures holding device pointers); cf_reduce_partials runs any collection
# of them.

def _pending_list(arr, n):
    return [cf_reduction(arr[i].part, arr[i].out, arr[i].rows, arr[i].cols) for i in range(n.value)]


def cf_reduce_partials(jobs, stream=None):
    n = len(jobs)
    arr = (cf_reduction * max(n, 1))(*jobs)
    _check(lib().cf_reduce_partials(n, arr, _stream(stream)))


def cf_conv3d_bwd_weight_deferred(desc, x, dz, dw, ws, ws_bytes=None, stream=None):
    if ws_bytes is None:
        ws_bytes = 0 if ws is None or isinstance(ws, int) else ws.numel() * ws.element_size()
    arr, n = (cf_reduction * CF_MAX_PENDING)(), ctypes.c_int32(0)
    _check(lib().cf_conv3d_bwd_weight_deferred(ctypes.byref(desc), _ptr(x), _ptr(dz), _ptr(dw), _ptr(ws), ws_bytes,
                                               arr, ctypes.byref(n), _stream(stream)))
    return _pending_list(arr, n)


def cf_bias_lrelu_bwd_deferred(nvox, c, dtype, dy, y, alpha, dz, db, ws, ws_bytes=None, stream=None):
    if ws_bytes is None:
        ws_bytes = 0 if ws is None or isinstance(ws, int) else ws.numel() * ws.element_size()
    arr, n = (cf_reduction * CF_MAX_PENDING)(), ctypes.c_int32(0)
    _check(lib().cf_bias_lrelu_bwd_deferred(nvox, c, dtype_code(dtype), _ptr(dy), _ptr(y), alpha, _ptr(dz), _ptr(db),
                                            _ptr(ws), ws_bytes, arr, ctypes.byref(n), _stream(stream)))
    return _pending_list(arr, n)


def cf_avgpool3d_lrelu_bwd_deferred(n, d, h, w, c, dtype, dp, mask, alpha, dz, db, ws, ws_bytes=None,
                                    stream=None):
    if ws_bytes is None:
        ws_bytes = 0 if ws is None or isinstance(ws, int) else ws.numel() * ws.element_size()
    arr, n_ = (cf_reduction * CF_MAX_PENDING)(), ctypes.c_int32(0)
    _check(lib().cf_avgpool3d_lrelu_bwd_deferred(n, d, h, w, c, dtype_code(dtype), _ptr(dp), _ptr(mask), alpha,
                                                 _ptr(dz), _ptr(db), _ptr(ws), ws_bytes, arr, ctypes.byref(n_),
                                                 _stream(stream)))
    return _pending_list(arr, n_)


def cf_conv3d_bwd_weight_fused_deferred(desc, x, g, mask, alpha, flags, dw, db, dz, ws, ws_bytes=None,
                                        stream=None):
    if ws_bytes is None:
        ws_bytes = 0 if ws is None or isinstance(ws, int) else ws.numel() * ws.element_size()
    arr, n = (cf_reduction * CF_MAX_PENDING)(), ctypes.c_int32(0)
    _check(lib().cf_conv3d_bwd_weight_fused_deferred(ctypes.byref(desc), _ptr(x), _ptr(g), _ptr(mask), alpha, flags,
                                                     _ptr(dw), _ptr(db), _ptr(dz), _ptr(ws), ws_bytes, arr,
                                                     ctypes.byref(n), _stream(stream)))
    return _pending_list(arr, n)


def cf_conv3d_bwd_deferred(desc, x, dz, w, dw, dx, ws, ws_bytes=None, stream=None):
    if ws_bytes is None:
        ws_bytes = 0 if ws is None or isinstance(ws, int) else ws.numel() * ws.element_size()
    arr, n = (cf_reduction * CF_MAX_PENDING)(), ctypes.c_int32(0)
    _check(lib().cf_conv3d_bwd_deferred(ctypes.byref(desc), _ptr(x), _ptr(dz), _ptr(w), _ptr(dw), _ptr(dx), _ptr(ws),
                                        ws_bytes, arr, ctypes.byref(n), _stream(stream)))
    return _pending_list(arr, n)


def cf_conv3d_bwd_fused_deferred(desc, x, g, mask, w, alpha, flags, dw, db, dx, ws, ws_bytes=None, stream=None):
    if ws_bytes is None:
        ws_bytes = 0 if ws is None or isinstance(ws, int) else ws.numel() * ws.element_size()
    arr, n = (cf_reduction * CF_MAX_PENDING)(), ctypes.c_int32(0)
    _check(lib().cf_conv3d_bwd_fused_deferred(ctypes.byref(desc), _ptr(x), _ptr(g), _ptr(mask), _ptr(w), alpha,
                                              flags, _ptr(dw), _ptr(db), _ptr(dx), _ptr(ws), ws_bytes, arr,
                                              ctypes.byref(n), _stream(stream)))
    return _pending_list(arr, n)


def _offsets(offsets):
    """(ngroups, ctypes int64 array); an already built pair passes through."""
    if isinstance(offsets, tuple) and len(offsets) == 2 and isinstance(offsets[1], ctypes.Array):
        return offsets
    arr = (ctypes.c_int64 * max(len(offsets), 1))(*[int(o) for o in offsets])
    return len(offsets) - 1, arr


def adam_offsets(offsets):
    """Pre-marshalled offsets for repeated cf_adam_larc_step calls."""
    return _offsets(offsets)


def cf_adam_larc_workspace_size(offsets) -> int:
    n, arr = _offsets(offsets)
    return lib().cf_adam_larc_workspace_size(n, arr)


def cf_adam_larc_step(offsets, t, hp, v, g, m, s, v16, ws, ws_bytes=None, stream=None):
    """offsets: ngroups + 1 host integers; hp: a cf_adam_larc_hparams (see make_hparams)."""
    if ws_bytes is None:
        ws_bytes = 0 if ws is None or isinstance(ws, int) else ws.numel() * ws.element_size()
    n, arr = _offsets(offsets)
    _check(lib().cf_adam_larc_step(n, arr, int(t), ctypes.byref(hp), _ptr(v), _ptr(g), _ptr(m), _ptr(s), _ptr(v16),
                                   _ptr(ws), ws_bytes, _stream(stream)))


# ---- fully-connected head and loss ---------------------------------------------

def cf_fc_fwd_workspace_size(m, k, n) -> int:
    return int(lib().cf_fc_fwd_workspace_size(m, k, n))


def cf_fc_fwd(m, k, n, dtype, x, w, z, ws, ws_bytes=None, stream=None):
    if ws_bytes is None:
        ws_bytes = 0 if ws is None or isinstance(ws, int) else ws.numel() * ws.element_size()
    _check(lib().cf_fc_fwd(m, k, n, dtype_code(dtype), _ptr(x), _ptr(w), _ptr(z), _ptr(ws), ws_bytes,
                           _stream(stream)))


def cf_fc_bwd_data(m, k, n, dtype, dz, w, dx, stream=None):
    _check(lib().cf_fc_bwd_data(m, k, n, dtype_code(dtype), _ptr(dz), _ptr(w), _ptr(dx), _stream(stream)))


def cf_fc_bwd_weight(m, k, n, dtype, x, dz, dw, stream=None):
    _check(lib().cf_fc_bwd_weight(m, k, n, dtype_code(dtype), _ptr(x), _ptr(dz), _ptr(dw), _stream(stream)))


def _i32s(v):
    return (ctypes.c_int32 * len(v))(*[int(a) for a in v])


def _ptrs(ts):
    """Host array of the device pointers of a list of tensors."""
    return (ctypes.c_void_p * max(len(ts), 1))(*[_ptr(t) for t in ts])


def cf_fc_head_workspace_size(m, dims) -> int:
    return int(lib().cf_fc_head_workspace_size(m, len(dims) - 1, _i32s(dims)))


def cf_fc_head(m, dims, dtype, x, w, b, alpha, target, y, dz, dx, dw, db, loss, ws, ws_bytes=None, stream=None):
    """Forward, loss and backward of the whole head (lists of per-layer tensors)."""
    if ws_bytes is None:
        ws_bytes = 0 if ws is None or isinstance(ws, int) else ws.numel() * ws.element_size()
    _check(lib().cf_fc_head(m, len(dims) - 1, _i32s(dims), dtype_code(dtype), _ptr(x), _ptrs(w), _ptrs(b),
                            float(alpha), _ptr(target), _ptrs(y), _ptrs(dz), _ptrs(dx), _ptrs(dw), _ptrs(db),
                            _ptr(loss), _ptr(ws), ws_bytes, _stream(stream)))


def cf_mse_loss(m, n, dtype, p, t, loss, dp, stream=None):
    _check(lib().cf_mse_loss(m, n, dtype_code(dtype), _ptr(p), _ptr(t), _ptr(loss), _ptr(dp), _stream(stream)))


# ---- layer normalisation ---------------------------------------------------------

def cf_layernorm_fwd_workspace_size(rows, c, dtype) -> int:
    return int(lib().cf_layernorm_fwd_workspace_size(rows, c, dtype_code(dtype)))


def cf_layernorm_fwd(rows, c, dtype, x, gamma, beta, eps, y, mean, rstd, ws=None, ws_bytes=None, stream=None):
    if ws_bytes is None:
        ws_bytes = 0 if ws is None or isinstance(ws, int) else ws.numel() * ws.element_size()
    _check(lib().cf_layernorm_fwd(rows, c, dtype_code(dtype), _ptr(x), _ptr(gamma), _ptr(beta), float(eps), _ptr(y),
                                  _ptr(mean), _ptr(rstd), _ptr(ws), ws_bytes, _stream(stream)))


def cf_layernorm_bwd_workspace_size(rows, c, dtype) -> int:
    return int(lib().cf_layernorm_bwd_workspace_size(rows, c, dtype_code(dtype)))


def cf_layernorm_bwd(rows, c, dtype, dy, x, gamma, mean, rstd, dx, dgamma, dbeta, ws, ws_bytes=None, stream=None):
    if ws_bytes is None:
        ws_bytes = 0 if ws is None or isinstance(ws, int) else ws.numel() * ws.element_size()
    _check(lib().cf_layernorm_bwd(rows, c, dtype_code(dtype), _ptr(dy), _ptr(x), _ptr(gamma), _ptr(mean), _ptr(rstd),
                                  _ptr(dx), _ptr(dgamma), _ptr(dbeta), _ptr(ws), ws_bytes, _stream(stream)))


# ---- orthogonalised updates --------------------------------------------------------

def cf_newton_schulz_workspace_size(mats, dtype) -> int:
    """mats: an array of cf_matrix (see make_matrices)."""
    return int(lib().cf_newton_schulz_workspace_size(len(mats), mats, dtype_code(dtype)))


def cf_newton_schulz(mats, dtype, hp, g, o, ws, ws_bytes=None, stream=None):
    """hp: a cf_ns_hparams (see make_ns_hparams)."""
    if ws_bytes is None:
        ws_bytes = 0 if ws is None or isinstance(ws, int) else ws.numel() * ws.element_size()
    _check(lib().cf_newton_schulz(len(mats), mats, dtype_code(dtype), ctypes.byref(hp), _ptr(g), _ptr(o), _ptr(ws), ws_bytes,
                                  _stream(stream)))


def cf_muon_workspace_size(mats) -> int:
    return int(lib().cf_muon_workspace_size(len(mats), mats))


def cf_muon_step(mats, t, hp, v, g, m, v16, ws, ws_bytes=None, stream=None):
    """hp: a cf_muon_hparams (see make_muon_hparams)."""
    if ws_bytes is None:
        ws_bytes = 0 if ws is None or isinstance(ws, int) else ws.numel() * ws.element_size()
    _check(lib().cf_muon_step(len(mats), mats, int(t), ctypes.byref(hp), _ptr(v), _ptr(g), _ptr(m), _ptr(v16), _ptr(ws),
                              ws_bytes, _stream(stream)))


# ---- group normalisation ---------------------------------------------------------

def _sizes32(*sizes):
    """ValueError unless each fits the 32 bits of its C argument (ctypes would pass the low ones)."""
    for s in sizes:
        if not -0x80000000 <= s < 0x80000000:
            raise ValueError(f"a size of {s}: past 32 bits")


def _ws_bytes(ws, ws_bytes):
    if ws_bytes is None:
        return 0 if ws is None or isinstance(ws, int) else ws.numel() * ws.element_size()
    return ws_bytes


def cf_groupnorm_fwd_workspace_size(n, vox, c, groups, dtype) -> int:
    _sizes32(n, c, groups)
    return int(lib().cf_groupnorm_fwd_workspace_size(n, vox, c, groups, dtype_code(dtype)))


def cf_groupnorm_fwd(n, vox, c, groups, dtype, x, gamma, beta, eps, act, alpha, y, mean, rstd, ws=None, ws_bytes=None,
                     stream=None):
    """act: "none", "lrelu", "silu" or "gelu" (or a CF_ACT_ code)."""
    _sizes32(n, c, groups)
    _check(lib().cf_groupnorm_fwd(n, vox, c, groups, dtype_code(dtype), _ptr(x), _ptr(gamma), _ptr(beta), float(eps),
                                  act_code(act), float(alpha), _ptr(y), _ptr(mean), _ptr(rstd), _ptr(ws),
                                  _ws_bytes(ws, ws_bytes), _stream(stream)))


def cf_groupnorm_bwd_workspace_size(n, vox, c, groups, dtype) -> int:
    _sizes32(n, c, groups)
    return int(lib().cf_groupnorm_bwd_workspace_size(n, vox, c, groups, dtype_code(dtype)))


def cf_groupnorm_bwd(n, vox, c, groups, dtype, dy, x, gamma, beta, mean, rstd, act, alpha, dx, dgamma, dbeta, ws,
                     ws_bytes=None, stream=None):
    _sizes32(n, c, groups)
    _check(lib().cf_groupnorm_bwd(n, vox, c, groups, dtype_code(dtype), _ptr(dy), _ptr(x), _ptr(gamma), _ptr(beta),
                                  _ptr(mean), _ptr(rstd), act_code(act), float(alpha), _ptr(dx), _ptr(dgamma),
                                  _ptr(dbeta), _ptr(ws), _ws_bytes(ws, ws_bytes), _stream(stream)))


# ---- matrix products with an epilogue ----------------------------------------------

def cf_linear_fwd_workspace_size(m, k, n, dtype) -> int:
    _sizes32(m, k, n)
    return int(lib().cf_linear_fwd_workspace_size(m, k, n, dtype_code(dtype)))


def cf_linear_fwd(m, k, n, dtype, x, w, bias, act, alpha, residual, y, z=None, ws=None, ws_bytes=None, stream=None):
    _sizes32(m, k, n)
    _check(lib().cf_linear_fwd(m, k, n, dtype_code(dtype), _ptr(x), _ptr(w), _ptr(bias), act_code(act), float(alpha),
                               _ptr(residual), _ptr(y), _ptr(z), _ptr(ws), _ws_bytes(ws, ws_bytes), _stream(stream)))


def cf_linear_bwd_data_workspace_size(m, k, n, dtype) -> int:
    _sizes32(m, k, n)
    return int(lib().cf_linear_bwd_data_workspace_size(m, k, n, dtype_code(dtype)))


def cf_linear_bwd_data(m, k, n, dtype, dz, w, residual, z, act, alpha, dx, ws=None, ws_bytes=None, stream=None):
    _sizes32(m, k, n)
    _check(lib().cf_linear_bwd_data(m, k, n, dtype_code(dtype), _ptr(dz), _ptr(w), _ptr(residual), _ptr(z), act_code(act),
                                    float(alpha), _ptr(dx), _ptr(ws), _ws_bytes(ws, ws_bytes), _stream(stream)))


def cf_linear_bwd_weight_workspace_size(m, k, n, dtype) -> int:
    _sizes32(m, k, n)
    return int(lib().cf_linear_bwd_weight_workspace_size(m, k, n, dtype_code(dtype)))


def cf_linear_bwd_weight(m, k, n, dtype, x, dz, dw, db=None, ws=None, ws_bytes=None, stream=None):
    _sizes32(m, k, n)
    _check(lib().cf_linear_bwd_weight(m, k, n, dtype_code(dtype), _ptr(x), _ptr(dz), _ptr(dw), _ptr(db), _ptr(ws),
                                      _ws_bytes(ws, ws_bytes), _stream(stream)))


# ---- AdamW -------------------------------------------------------------------------

def cf_adamw_step(tensors, t, hp, stream=None):
    """tensors: what make_adamw_tensors returns; hp: a cf_adamw_hparams (see make_adamw_hparams)."""
    n, arr = tensors
    _check(lib().cf_adamw_step(n, arr, int(t), ctypes.byref(hp), _stream(stream)))
