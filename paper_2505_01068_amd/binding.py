"""ctypes binding over libimattn.so: same names as the C ABI (include/imattn.h).

Argument marshalling only.  Torch supplies device memory and the current HIP
stream; every step of the computation runs inside the library's kernels.  There
is no fallback: a missing library or a non-zero return code raises.
"""
from __future__ import annotations

import ctypes as C
import os

import torch

IM_MAX_SEG = 8
IM_DTYPE_F32, IM_DTYPE_BF16 = 0, 1
IM_OK, IM_ERR_INVALID, IM_ERR_UNSUPPORTED, IM_ERR_WORKSPACE, IM_ERR_HIP = 0, -1, -2, -3, -4
IM_IFM_FORWARD, IM_IFM_BACKWARD, IM_IEM, IM_DENSE = 0x062, 0x08C, 0x111, 0x1FF
# the named 3 x 3 patterns of include/imattn.h (segment order t, v, a; bit i*3 + j <=> block (query i, key j) live)
NAMED_MASKS = {
    "ifm_forward": IM_IFM_FORWARD, "ifm_backward": IM_IFM_BACKWARD, "iem": IM_IEM, "dense": IM_DENSE,
    "structure1_a": 0x0A4, "structure1_b": 0x04A, "structure2_a": 0x08A, "structure2_b": 0x064,
    "structure3_a": 0x0A2, "structure3_b": 0x04C, "self_only": 0x0EE,
}

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libimattn.so")


class ImShape(C.Structure):
    _fields_ = [("batch", C.c_int32), ("n_seg", C.c_int32), ("seg_len", C.c_int32 * IM_MAX_SEG),
                ("d_model", C.c_int32), ("n_heads", C.c_int32), ("live_mask", C.c_uint64),
                ("scale", C.c_float), ("dtype", C.c_int32),
                ("cu_rows", C.c_void_p), ("total_rows", C.c_int64)]


class ImWorkItem(C.Structure):
    _fields_ = [("q_seg", C.c_int32), ("q_start", C.c_int32), ("q_rows", C.c_int32), ("n_key_seg", C.c_int32),
                ("key_seg", C.c_int32 * IM_MAX_SEG), ("pairs", C.c_int64)]


IM_MAX_AXES = 4
IM_NORM_MAX_D = 16384


class ImView(C.Structure):
    _fields_ = [("ptr", C.c_void_p), ("batch", C.c_int64), ("row", C.c_int64), ("head", C.c_int64)]


class ImRotary(C.Structure):
    _fields_ = [("batch", C.c_int32), ("rows", C.c_int32), ("n_axes", C.c_int32), ("pairs", C.c_int32 * IM_MAX_AXES),
                ("q_heads", C.c_int32), ("k_heads", C.c_int32), ("head_dim", C.c_int32), ("interleaved", C.c_int32),
                ("inverse", C.c_int32), ("dtype", C.c_int32)]


class ImCore(C.Structure):
    _fields_ = [("batch", C.c_int32), ("n_seg", C.c_int32), ("q_len", C.c_int32 * IM_MAX_SEG), ("k_len", C.c_int32 * IM_MAX_SEG),
                ("n_heads", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("live_mask", C.c_uint64),
                ("scale", C.c_float), ("cap", C.c_float), ("causal", C.c_int32), ("dtype", C.c_int32)]


class ImCoreRules(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("valid_len", "key_pad", "q_pos", "k_pos", "slope", "prefix", "q_doc", "k_doc")]


class ImAttnError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"imattn error {code}: {msg}")
        self.code = code


_lib = None


def lib():
    """Load the shared library (built in-tree by paper_2505_01068_amd/build.py); raises if absent."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise ImportError(f"{_LIB_PATH} not found: build it with `python -m paper_2505_01068_amd.build` "
                              "(there is no CPU or PyTorch fallback)")
        L = C.CDLL(_LIB_PATH)
        vp, sz = C.c_void_p, C.c_size_t
        shp = C.POINTER(ImShape)
        L.im_last_error.restype = C.c_char_p
        L.im_version.restype = C.c_char_p
        L.im_schedule_build.argtypes = [shp, C.c_int32, C.POINTER(ImWorkItem), C.c_int32, C.POINTER(C.c_int32),
                                        C.POINTER(C.c_int64)]
        L.im_attention_sizes.argtypes = [shp, C.POINTER(sz), C.POINTER(sz)]
        L.im_attention_fwd.argtypes = [shp] + [vp] * 14 + [sz, vp]
        L.im_attention_bwd.argtypes = [shp] + [vp] * 19 + [sz, vp]
        L.im_attention_fwd_noalloc.argtypes = [shp] + [vp] * 13
        L.im_noalloc_init.argtypes = []
        L.im_calibrate_mfma.argtypes = [C.c_int32, vp, C.POINTER(C.c_double), vp]
        L.im_calibrate_copy.argtypes = [vp, vp, sz, vp]
        L.gsit_layer_sizes.argtypes = [shp, C.c_int32, C.POINTER(sz)]
        L.gsit_layer_fwd.argtypes = [shp, C.c_int32] + [vp] * 17 + [C.c_float] + [vp] * 4 + [sz, vp]
        L.im_profile_enable.argtypes = [C.c_int]
        L.im_profile_get.argtypes = [C.c_int, C.POINTER(C.c_char_p), C.POINTER(C.c_double), C.POINTER(C.c_int64)]
        L.im_profile_enable.restype = C.c_int
        L.im_profile_get.restype = C.c_int
        L.gsit_layer_train_sizes.argtypes = [C.c_void_p, C.c_int32, C.POINTER(C.c_size_t), C.POINTER(C.c_size_t)]
        L.gsit_layer_fwd_train.argtypes = [C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_float, C.c_void_p, C.c_void_p,
                                           C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
        L.gsit_layer_bwd.argtypes = [C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_float, C.c_void_p, C.c_void_p,
                                     C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
        L.gsit_model_sizes.argtypes = [C.c_void_p, C.c_void_p, C.POINTER(C.c_size_t)]
        L.gsit_model_fwd.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                     C.c_size_t, C.c_void_p]
        view, i32, i64 = C.POINTER(ImView), C.c_int32, C.c_int64
        L.im_layernorm_sizes.argtypes = [i64, i32, i32, C.POINTER(sz)]
        L.im_layernorm_fwd.argtypes = [i64, i32, i32, vp, i64, vp, vp, C.c_float, vp, i64, vp, vp, vp]
        L.im_layernorm_bwd.argtypes = [i64, i32, i32, vp, i64, vp, vp, vp, vp, i64, vp, i64, vp, vp, vp, sz, vp]
        L.im_rotary_apply.argtypes = [C.POINTER(ImRotary), vp, i64, vp] + [view] * 4 + [vp]
        core, rules = C.POINTER(ImCore), C.POINTER(ImCoreRules)
        L.im_core_attention_sizes.argtypes = [core] + [C.POINTER(sz)] * 3
        L.im_core_attention_fwd.argtypes = [core, rules] + [view] * 4 + [vp, vp, vp, sz, vp]
        L.im_core_attention_bwd.argtypes = [core, rules] + [view] * 3 + [vp] + [view] * 4 + [vp, vp, sz, vp]
        for f in (L.im_layernorm_sizes, L.im_layernorm_fwd, L.im_layernorm_bwd, L.im_rotary_apply, L.im_core_attention_sizes,
                  L.im_core_attention_fwd, L.im_core_attention_bwd, L.im_schedule_build, L.im_attention_sizes, L.im_attention_fwd, L.im_attention_bwd,
                  L.im_attention_fwd_noalloc, L.im_noalloc_init, L.im_calibrate_mfma, L.im_calibrate_copy,
                  L.gsit_layer_sizes, L.gsit_layer_fwd, L.gsit_model_sizes, L.gsit_model_fwd,
                  L.gsit_layer_train_sizes, L.gsit_layer_fwd_train, L.gsit_layer_bwd):
            f.restype = C.c_int
        _lib = L
    return _lib


def _check(rc):
    if rc != 0:
        raise ImAttnError(rc, lib().im_last_error().decode())


def make_shape(batch, seg_len, d_model, n_heads, live_mask, scale, dtype, cu_rows=None, total_rows=0):
    """The problem statement.  Packed rows: cu_rows = int32 device tensor [batch * n_seg + 1] of row offsets,
    total_rows = its last entry (host int); seg_len then bounds the per-sample segment lengths.  The shape
    keeps a reference to cu_rows, whose device memory it points into."""
    s = ImShape()
    s.cu_rows, s.total_rows = (None, 0) if cu_rows is None else (cu_rows.data_ptr(), int(total_rows))
    s._cu_rows_ref = cu_rows
    s.batch, s.n_seg, s.d_model, s.n_heads = int(batch), len(seg_len), int(d_model), int(n_heads)
    for i, n in enumerate(seg_len):
        s.seg_len[i] = int(n)
    s.live_mask, s.scale = int(live_mask), float(scale)
    s.dtype = {"fp32": IM_DTYPE_F32, "bf16": IM_DTYPE_BF16, torch.float32: IM_DTYPE_F32,
               torch.bfloat16: IM_DTYPE_BF16, 0: 0, 1: 1}[dtype]
    return s


def _p(t):
    return None if t is None else C.c_void_p(t.data_ptr())


def _stream():
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


def im_schedule_build(shape, tile_rows):
    """Host-side listing of the live-block schedule: (items, n_pairs)."""
    n, pairs = C.c_int32(0), C.c_int64(0)
    _check(lib().im_schedule_build(C.byref(shape), tile_rows, None, 0, C.byref(n), C.byref(pairs)))
    items = (ImWorkItem * max(1, n.value))()
    _check(lib().im_schedule_build(C.byref(shape), tile_rows, items, n.value, C.byref(n), C.byref(pairs)))
    return [items[i] for i in range(n.value)], pairs.value


def im_attention_sizes(shape):
    a, b = C.c_size_t(0), C.c_size_t(0)
    _check(lib().im_attention_sizes(C.byref(shape), C.byref(a), C.byref(b)))
    return a.value, b.value


def gsit_layer_sizes(shape, d_ff):
    a = C.c_size_t(0)
    _check(lib().gsit_layer_sizes(C.byref(shape), int(d_ff), C.byref(a)))
    return a.value


def im_attention_fwd(shape, x, wq, wk, wv, wo, bq=None, bk=None, bv=None, bo=None, valid_len=None, key_pad=None,
                     y=None, saved=None, workspace=None):
    """y = IMAttention(x).  Tensors are CUDA(HIP) tensors; `saved`/`workspace` are uint8 buffers."""
    if y is None:
        y = torch.empty_like(x)
    wbytes = 0 if workspace is None else workspace.numel()
    _check(lib().im_attention_fwd(C.byref(shape), _p(x), _p(wq), _p(wk), _p(wv), _p(wo), _p(bq), _p(bk), _p(bv),
                                  _p(bo), _p(valid_len), _p(key_pad), _p(y), _p(saved), _p(workspace), wbytes,
                                  _stream()))
    return y


IM_NOALLOC_MAX_BYTES = 64 << 20


def im_noalloc_init():
    _check(lib().im_noalloc_init())


def im_attention_fwd_noalloc(shape, x, wq, wk, wv, wo, bq=None, bk=None, bv=None, bo=None, valid_len=None,
                             key_pad=None, y=None):
    """Inference forward on the library's built-in scratch buffer; `y` must be given (nothing is allocated)."""
    _check(lib().im_attention_fwd_noalloc(C.byref(shape), _p(x), _p(wq), _p(wk), _p(wv), _p(wo), _p(bq), _p(bk),
                                          _p(bv), _p(bo), _p(valid_len), _p(key_pad), _p(y), _stream()))
    return y


def im_attention_bwd(shape, x, wq, wk, wv, wo, saved, dy, dx, dwq, dwk, dwv, dwo, dbq=None, dbk=None, dbv=None,
                     dbo=None, valid_len=None, key_pad=None, workspace=None):
    wbytes = 0 if workspace is None else workspace.numel()
    _check(lib().im_attention_bwd(C.byref(shape), _p(x), _p(wq), _p(wk), _p(wv), _p(wo), _p(valid_len), _p(key_pad),
                                  _p(saved), _p(dy), _p(dx), _p(dwq), _p(dwk), _p(dwv), _p(dwo), _p(dbq), _p(dbk),
                                  _p(dbv), _p(dbo), _p(workspace), wbytes, _stream()))
    return dx


def gsit_layer_fwd(shape, d_ff, x, p, ln_eps=1e-5, valid_len=None, key_pad=None, y=None, workspace=None):
    """One encoder layer; `p` maps parameter names (ln1_g, ln1_b, wq, ..., w2, b2) to device tensors."""
    if y is None:
        y = torch.empty_like(x)
    wbytes = 0 if workspace is None else workspace.numel()
    g = p.get
    _check(lib().gsit_layer_fwd(C.byref(shape), int(d_ff), _p(x), _p(p["ln1_g"]), _p(p["ln1_b"]), _p(p["wq"]),
                                _p(p["wk"]), _p(p["wv"]), _p(p["wo"]), _p(g("bq")), _p(g("bk")), _p(g("bv")),
                                _p(g("bo")), _p(p["ln2_g"]), _p(p["ln2_b"]), _p(p["w1"]), _p(g("b1")), _p(p["w2"]),
                                _p(g("b2")), float(ln_eps), _p(valid_len), _p(key_pad), _p(y), _p(workspace), wbytes,
                                _stream()))
    return y


LAYER_FIELDS = ("ln1_g", "ln1_b", "wq", "wk", "wv", "wo", "bq", "bk", "bv", "bo", "ln2_g", "ln2_b", "w1", "b1", "w2", "b2")


class GsitLayerParams(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in LAYER_FIELDS]


class GsitModel(C.Structure):
    _fields_ = [("n_layers_inter", C.c_int32), ("n_layers_intra", C.c_int32), ("d_ff_inter", C.c_int32),
                ("d_ff_intra", C.c_int32), ("n_heads_intra", C.c_int32), ("n_out", C.c_int32),
                ("scale_intra", C.c_float), ("ln_eps", C.c_float),
                ("mask_fwd", C.c_uint64), ("mask_bwd", C.c_uint64), ("mask_intra", C.c_uint64),
                ("fwd_layers", C.POINTER(GsitLayerParams)), ("bwd_layers", C.POINTER(GsitLayerParams)),
                ("intra_layers", C.POINTER(GsitLayerParams)), ("wf", C.c_void_p), ("bf", C.c_void_p)]


def _layer_array(layers):
    arr = (GsitLayerParams * len(layers))()
    for i, p in enumerate(layers):
        for n in LAYER_FIELDS:
            t = p.get(n)
            setattr(arr[i], n, None if t is None else t.data_ptr())
    return arr


def make_model(model, d_ff_inter, d_ff_intra, n_heads_intra, scale_intra, ln_eps=1e-5,
               mask_fwd=0x062, mask_bwd=0x08C, mask_intra=0x111):
    """gsit_model_t from a dict of device tensors: fwd_layers / bwd_layers / intra_layers (lists of
    layer dicts as for gsit_layer_fwd), wf, bf.  The returned object keeps the arrays alive."""
    m = GsitModel()
    m._keep = (_layer_array(model["fwd_layers"]), _layer_array(model["bwd_layers"]), _layer_array(model["intra_layers"]), model)
    m.n_layers_inter, m.n_layers_intra = len(model["fwd_layers"]), len(model["intra_layers"])
    if len(model["bwd_layers"]) != m.n_layers_inter:
        raise ValueError("the two inter-modal encoders must have the same number of layers")
    m.d_ff_inter, m.d_ff_intra, m.n_heads_intra = int(d_ff_inter), int(d_ff_intra), int(n_heads_intra)
    m.n_out = int(model["wf"].shape[1])
    m.scale_intra, m.ln_eps = float(scale_intra), float(ln_eps)
    m.mask_fwd, m.mask_bwd, m.mask_intra = int(mask_fwd), int(mask_bwd), int(mask_intra)
    m.fwd_layers, m.bwd_layers, m.intra_layers = m._keep[0], m._keep[1], m._keep[2]
    m.wf = model["wf"].data_ptr()
    m.bf = None if model.get("bf") is None else model["bf"].data_ptr()
    return m


def _layer_struct(p):
    st = GsitLayerParams()
    for n in LAYER_FIELDS:
        t = p.get(n)
        setattr(st, n, None if t is None else t.data_ptr())
    return st


def gsit_layer_train_sizes(shape, d_ff):
    a, b = C.c_size_t(0), C.c_size_t(0)
    _check(lib().gsit_layer_train_sizes(C.byref(shape), int(d_ff), C.byref(a), C.byref(b)))
    return a.value, b.value


def gsit_layer_fwd_train(shape, d_ff, x, p, saved, ln_eps=1e-5, valid_len=None, key_pad=None, y=None, workspace=None):
    """Training forward of one encoder layer: y as gsit_layer_fwd, `saved` filled for gsit_layer_bwd."""
    if y is None:
        y = torch.empty_like(x)
    st = _layer_struct(p)
    _check(lib().gsit_layer_fwd_train(C.byref(shape), int(d_ff), _p(x), C.byref(st), float(ln_eps), _p(valid_len),
                                      _p(key_pad), _p(y), _p(saved), _p(workspace), workspace.numel(), _stream()))
    return y


def gsit_layer_bwd(shape, d_ff, x, p, saved, dy, grads, ln_eps=1e-5, valid_len=None, key_pad=None, dx=None, workspace=None):
    """Backward of one encoder layer.  `grads` maps parameter names to fp32 device tensors to overwrite
    (missing / None = not wanted).  Returns dx."""
    if dx is None:
        dx = torch.empty_like(x)
    st, gs = _layer_struct(p), _layer_struct(grads)
    _check(lib().gsit_layer_bwd(C.byref(shape), int(d_ff), _p(x), C.byref(st), float(ln_eps), _p(valid_len), _p(key_pad),
                                _p(saved), _p(dy), _p(dx), C.byref(gs), _p(workspace), workspace.numel(), _stream()))
    return dx


def gsit_model_sizes(shape, model):
    a = C.c_size_t(0)
    _check(lib().gsit_model_sizes(C.byref(shape), C.byref(model), C.byref(a)))
    return a.value


def gsit_model_fwd(shape, model, x, valid_len=None, key_pad=None, out=None, workspace=None):
    """out [B, n_out] = GsiT(x): two IFM encoders, feature concat, IEM encoder, last steps, final linear."""
    if out is None:
        out = torch.empty(x.shape[0], model.n_out, dtype=x.dtype, device=x.device)
    wbytes = 0 if workspace is None else workspace.numel()
    _check(lib().gsit_model_fwd(C.byref(shape), C.byref(model), _p(x), _p(valid_len), _p(key_pad), _p(out),
                                _p(workspace), wbytes, _stream()))
    return out


# ---- operators around the attention of a layer ----
# (Small calls are bound by the host: the checks below touch each tensor once and build no containers.)

_DTYPES = {torch.float32: IM_DTYPE_F32, torch.bfloat16: IM_DTYPE_BF16, "fp32": IM_DTYPE_F32, "bf16": IM_DTYPE_BF16}
_TORCH_TYPES = (torch.float32, torch.bfloat16)


def _dtype(t):
    if t not in _DTYPES:
        raise ValueError(f"dtype must be float32 or bfloat16 (got {t})")
    return _DTYPES[t]


def _device(what, x):
    """The call goes to the current device's current stream: every tensor has to live on that device.  Its index."""
    i = x.get_device()
    if i < 0 or i != torch._C._cuda_getDevice():
        raise ValueError(f"{what}: tensors must be on the current GPU, got {x.device}")
    return i


def _raw_stream(device):
    return torch._C._cuda_getCurrentRawStream(device)


def _want(what, name, t, shape, dtype, device):
    """Address of a dense tensor of that shape and type; None stays None."""
    if t is None:
        return None
    if t.dtype is not dtype or t.shape != shape or not t.is_contiguous() or t.get_device() != device:
        raise ValueError(f"{what}: {name} must be a contiguous {dtype} tensor of shape {tuple(shape)} on cuda:{device}, got {t.dtype} "
                         f"{tuple(t.shape)} with strides {t.stride()} on {t.device}")
    return t.data_ptr()


def _needed(what, name, t):
    if t is None:
        raise ValueError(f"{what}: {name} is needed")


def _bytes(what, name, t, device, need=0):
    """(address, bytes) of a uint8 buffer"""
    if t is None:
        return None, 0
    if t.dtype is not torch.uint8 or not t.is_contiguous() or t.get_device() != device:
        raise ValueError(f"{what}: {name} must be a contiguous uint8 tensor on cuda:{device}")
    if t.numel() < need:
        raise ValueError(f"{what}: {name} has {t.numel()} bytes, {need} are needed")
    return t.data_ptr(), t.numel()


def _rows(what, name, t, d, dtype, n=None):
    """(rows, distance) of a tensor [..., d] whose rows lie at one distance from each other."""
    shape, stride = t.shape, t.stride()
    if len(shape) < 1 or shape[-1] != d or t.dtype is not dtype or (d > 1 and stride[-1] != 1):
        raise ValueError(f"{what}: {name} must be a {dtype} tensor [..., {d}] with its last dimension dense, got {t.dtype} {tuple(shape)} "
                         f"with strides {stride}")
    rows, ld = 1, 0
    for i in range(len(shape) - 2, -1, -1):
        if shape[i] != 1:
            if shape[i] == 0:   # no rows: whatever the strides
                rows = 0
                break
            if rows == 1:
                ld = stride[i]
            elif stride[i] != ld * rows:
                raise ValueError(f"{what}: the rows of {name} must lie at one distance from each other, got shape {tuple(shape)} with strides {stride}")
            rows *= shape[i]
    if n is not None and rows != n:
        raise ValueError(f"{what}: {name} has {rows} rows, {n} are needed")
    return rows, ld if rows > 1 else d


def _row_stat(what, name, t, rows, device):
    if t is None:
        return None
    if t.dtype is not torch.float32 or t.numel() != rows or not t.is_contiguous() or t.get_device() != device:
        raise ValueError(f"{what}: {name} must be a contiguous float32 tensor of {rows} elements on cuda:{device}, got {t.dtype} {tuple(t.shape)} on {t.device}")
    return t.data_ptr()


def im_layernorm_sizes(rows, d, dtype):
    """Workspace bytes of im_layernorm_bwd."""
    a = C.c_size_t(0)
    _check(lib().im_layernorm_sizes(int(rows), int(d), _dtype(dtype), C.byref(a)))
    return a.value


def im_layernorm_fwd(x, gamma=None, beta=None, eps=1e-5, y=None, mean=None, rstd=None):
    """y = layer norm of x [..., d] over its last dimension, rows at one distance.  mean, rstd: fp32 tensors with one element a
    row that the backward needs, or None for inference.  y may be x."""
    what = "im_layernorm_fwd"
    dev = _device(what, x)
    if y is None:
        y = torch.empty_like(x)
    elif y.get_device() != dev:
        raise ValueError(f"{what}: y is on {y.device}, not on cuda:{dev}")
    d, dt = x.shape[-1] if x.dim() else 0, x.dtype
    rows, ldx = _rows(what, "x", x, d, dt)
    _, ldy = _rows(what, "y", y, d, dt, rows)
    _check((_lib or lib()).im_layernorm_fwd(rows, d, _dtype(dt), x.data_ptr(), ldx, _want(what, "gamma", gamma, (d,), dt, dev),
                                            _want(what, "beta", beta, (d,), dt, dev), eps, y.data_ptr(), ldy,
                                            _row_stat(what, "mean", mean, rows, dev), _row_stat(what, "rstd", rstd, rows, dev), _raw_stream(dev)))
    return y


def im_layernorm_bwd(x, gamma, mean, rstd, dy, dx=None, dgamma=None, dbeta=None, workspace=None):
    """Gradients of im_layernorm_fwd into those of dx [..., d], dgamma and dbeta (fp32 [d]) that are given.  dx may be dy."""
    what = "im_layernorm_bwd"
    dev = _device(what, x)
    if dy.get_device() != dev or (dx is not None and dx.get_device() != dev):
        raise ValueError(f"{what}: dy and dx must be on cuda:{dev}")
    d, dt = x.shape[-1] if x.dim() else 0, x.dtype
    rows, ldx = _rows(what, "x", x, d, dt)
    _, lddy = _rows(what, "dy", dy, d, dt, rows)
    lddx = _rows(what, "dx", dx, d, dt, rows)[1] if dx is not None else 0
    _needed(what, "mean", mean)
    _needed(what, "rstd", rstd)
    ws, nbytes = _bytes(what, "workspace", workspace, dev)
    f32 = torch.float32
    _check((_lib or lib()).im_layernorm_bwd(rows, d, _dtype(dt), x.data_ptr(), ldx, _want(what, "gamma", gamma, (d,), dt, dev),
                                            _row_stat(what, "mean", mean, rows, dev), _row_stat(what, "rstd", rstd, rows, dev), dy.data_ptr(), lddy,
                                            None if dx is None else dx.data_ptr(), lddx, _want(what, "dgamma", dgamma, (d,), f32, dev),
                                            _want(what, "dbeta", dbeta, (d,), f32, dev), ws, nbytes, _raw_stream(dev)))
    return dx


def _view(what, name, t, shape, dtype, device=None):
    if t is None or t.dtype is not dtype or t.shape != shape or (device is not None and t.get_device() != device):
        got = "None" if t is None else f"{t.dtype} {tuple(t.shape)} on {t.device}"
        raise ValueError(f"{what}: {name} must be a {dtype} tensor of shape {tuple(shape)} on the current GPU, got {got}")
    b, r, h, e = t.stride()
    if e != 1 and shape[3] > 1:
        raise ValueError(f"{what}: the heads of {name} must be dense, got strides {t.stride()}")
    return ImView(t.data_ptr(), b, r, h)


def im_rotary(pos, inv_freq, pairs, q, k=None, q_out=None, k_out=None, interleaved=False, inverse=False):
    """Rotary positions on q [B, T, heads, head_dim] and, if given, k [B, T, k_heads, head_dim] (any strides, dense heads).
    pos: fp32 [B, T, axes], or [T, axes] for all batch elements; pairs: rotated pairs of each axis; inv_freq: fp32
    [sum of pairs].  inverse: the gradient's rotation.  q_out / k_out may be q / k.  Returns (q_out, k_out)."""
    what = "im_rotary"
    dev = _device(what, q)
    if q.dim() != 4 or (k is not None and k.dim() != 4):
        raise ValueError(f"{what}: q and k must be [batch, rows, heads, head_dim]")
    dt, shape = q.dtype, q.shape
    batch, rows, heads, dh = shape
    if q_out is None:
        q_out = torch.empty(shape, dtype=dt, device=q.device)
    axes = len(pairs)
    if not 1 <= axes <= IM_MAX_AXES:
        raise ValueError(f"{what}: 1 to {IM_MAX_AXES} axes, got {axes}")
    _needed(what, "pos", pos)
    _needed(what, "inv_freq", inv_freq)
    shared = pos.dim() == 2
    kh = 0 if k is None else k.shape[2]
    s = ImRotary(batch, rows, axes, (C.c_int32 * IM_MAX_AXES)(*pairs), heads, kh, dh, bool(interleaved), bool(inverse), _dtype(dt))
    vk = vk_out = None
    if k is not None:
        kshape = (batch, rows, kh, dh)
        if k_out is None:
            k_out = torch.empty(kshape, dtype=dt, device=q.device)
        vk, vk_out = _view(what, "k", k, kshape, dt, dev), _view(what, "k_out", k_out, kshape, dt, dev)
    f32 = torch.float32
    _check((_lib or lib()).im_rotary_apply(s, _want(what, "pos", pos, (rows, axes) if shared else (batch, rows, axes), f32, dev),
                                           0 if shared else rows * axes, _want(what, "inv_freq", inv_freq, (sum(pairs),), f32, dev),
                                           _view(what, "q", q, shape, dt, dev), _view(what, "q_out", q_out, shape, dt, dev), vk, vk_out, _raw_stream(dev)))
    return q_out, k_out


def make_core(batch, q_len, k_len, n_heads, n_kv_heads, head_dim, live_mask, scale, dtype, cap=0.0, causal=False):
    """The problem statement of im_core_attention_*: per-segment numbers of queries and keys, heads, block pattern, cap."""
    s = ImCore()
    if len(q_len) != len(k_len) or not 1 <= len(q_len) <= IM_MAX_SEG:
        raise ValueError(f"q_len and k_len must have the same 1 to {IM_MAX_SEG} segments")
    s.batch, s.n_seg, s.n_heads, s.n_kv_heads, s.head_dim = int(batch), len(q_len), int(n_heads), int(n_kv_heads), int(head_dim)
    for i, (nq, nk) in enumerate(zip(q_len, k_len)):
        s.q_len[i], s.k_len[i] = int(nq), int(nk)
    if not 0 <= int(live_mask) < 1 << 64:
        raise ValueError(f"live_mask must have at most 64 bits, got {live_mask:#x}")
    s.live_mask, s.scale, s.cap, s.causal, s.dtype = int(live_mask), float(scale), float(cap), bool(causal), _dtype(dtype)
    return s


def im_core_attention_sizes(core):
    """(saved bytes, forward workspace bytes, backward workspace bytes)"""
    a, f, b = C.c_size_t(0), C.c_size_t(0), C.c_size_t(0)
    _check(lib().im_core_attention_sizes(C.byref(core), C.byref(a), C.byref(f), C.byref(b)))
    return a.value, f.value, b.value


def _core_shapes(core):
    """(batch, query rows, key rows, heads, bytes of `saved`)"""
    n = core.n_seg
    tq, tk = sum(core.q_len[:n]), sum(core.k_len[:n])
    rows = core.batch * core.n_heads * tq * 4
    return core.batch, tq, tk, core.n_heads, (rows * core.head_dim + 255 & ~255) + (rows + 255 & ~255)


def _core_rules(what, core, batch, tq, tk, dev, valid_len, key_pad, q_pos, k_pos, slope, prefix, q_doc, k_doc):
    i32, f32 = torch.int32, torch.float32
    return ImCoreRules(_want(what, "valid_len", valid_len, (batch, core.n_seg), i32, dev), _want(what, "key_pad", key_pad, (batch, tk), torch.uint8, dev),
                       _want(what, "q_pos", q_pos, (batch, tq), f32, dev), _want(what, "k_pos", k_pos, (batch, tk), f32, dev),
                       _want(what, "slope", slope, (core.n_heads,), f32, dev), _want(what, "prefix", prefix, (batch,), f32, dev),
                       _want(what, "q_doc", q_doc, (batch, tq), i32, dev), _want(what, "k_doc", k_doc, (batch, tk), i32, dev))


def im_core_attention_fwd(core, q, k, v, valid_len=None, key_pad=None, q_pos=None, k_pos=None, slope=None, prefix=None, q_doc=None,
                          k_doc=None, o=None, lse=None, saved=None, workspace=None):
    """o [B, Tq, heads, head_dim] = attention of q over k, v [B, Tk, kv_heads, head_dim] (any strides, dense heads) under the rules
    given; see include/imattn.h.  lse: fp32 [B, heads, Tq] or None; saved / workspace: uint8 buffers of
    im_core_attention_sizes (saved None for inference)."""
    what = "im_core_attention_fwd"
    dev = _device(what, q)
    if o is None:
        o = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    batch, tq, tk, heads, need = _core_shapes(core)
    dt = _TORCH_TYPES[core.dtype == IM_DTYPE_BF16]
    shape_q, shape_k = (batch, tq, heads, core.head_dim), (batch, tk, core.n_kv_heads, core.head_dim)
    r = _core_rules(what, core, batch, tq, tk, dev, valid_len, key_pad, q_pos, k_pos, slope, prefix, q_doc, k_doc)
    keep, _ = _bytes(what, "saved", saved, dev, need)
    ws, nbytes = _bytes(what, "workspace", workspace, dev)
    _check((_lib or lib()).im_core_attention_fwd(core, r, _view(what, "q", q, shape_q, dt, dev), _view(what, "k", k, shape_k, dt, dev),
                                                 _view(what, "v", v, shape_k, dt, dev), _view(what, "o", o, shape_q, dt, dev),
                                                 _want(what, "lse", lse, (batch, heads, tq), torch.float32, dev), keep, ws, nbytes, _raw_stream(dev)))
    return o


def im_core_attention_bwd(core, q, k, v, saved, d_o, dq, dk, dv, dslope=None, valid_len=None, key_pad=None, q_pos=None, k_pos=None,
                          slope=None, prefix=None, q_doc=None, k_doc=None, workspace=None):
    """Gradients of im_core_attention_fwd with the same arguments and its `saved`: dq, dk, dv and, if given, dslope (fp32
    [heads]) are overwritten."""
    what = "im_core_attention_bwd"
    dev = _device(what, q)
    batch, tq, tk, heads, need = _core_shapes(core)
    dt = _TORCH_TYPES[core.dtype == IM_DTYPE_BF16]
    shape_q, shape_k = (batch, tq, heads, core.head_dim), (batch, tk, core.n_kv_heads, core.head_dim)
    r = _core_rules(what, core, batch, tq, tk, dev, valid_len, key_pad, q_pos, k_pos, slope, prefix, q_doc, k_doc)
    keep, _ = _bytes(what, "saved", saved, dev, need)
    ws, nbytes = _bytes(what, "workspace", workspace, dev)
    _check((_lib or lib()).im_core_attention_bwd(core, r, _view(what, "q", q, shape_q, dt, dev), _view(what, "k", k, shape_k, dt, dev),
                                                 _view(what, "v", v, shape_k, dt, dev), keep, _view(what, "d_o", d_o, shape_q, dt, dev),
                                                 _view(what, "dq", dq, shape_q, dt, dev), _view(what, "dk", dk, shape_k, dt, dev),
                                                 _view(what, "dv", dv, shape_k, dt, dev), _want(what, "dslope", dslope, (heads,), torch.float32, dev), ws,
                                                 nbytes, _raw_stream(dev)))
    return dq, dk, dv


def im_calibrate_mfma(iters, sink):
    """Enqueue the register-resident MFMA loop; returns the flops it launched."""
    f = C.c_double(0)
    _check(lib().im_calibrate_mfma(int(iters), _p(sink), C.byref(f), _stream()))
    return f.value


def im_calibrate_copy(dst, src):
    """Enqueue a streaming device copy of src (uint8 tensor) into dst."""
    _check(lib().im_calibrate_copy(_p(dst), _p(src), src.numel() * src.element_size(), _stream()))


def im_profile_enable(on, only=None):
    """on: time every kernel family; only=<family name>: time just that one (cheaper)."""
    if only is not None:
        names = im_profile_names()
        lib().im_profile_enable(1 << (names.index(only) + 1))
    else:
        lib().im_profile_enable(1 if on else 0)


def im_profile_names():
    n = lib().im_profile_get(-1, None, None, None)
    out = []
    for i in range(n):
        name = C.c_char_p()
        lib().im_profile_get(i, C.byref(name), None, None)
        out.append(name.value.decode())
    return out


def im_profile_get():
    """{family: (total_ms, launches)} since the last im_profile_enable(True); call after a synchronize."""
    out = {}
    n = lib().im_profile_get(0, None, None, None)
    for i in range(n):
        name, ms, cnt = C.c_char_p(), C.c_double(0), C.c_int64(0)
        lib().im_profile_get(i, C.byref(name), C.byref(ms), C.byref(cnt))
        out[name.value.decode()] = (ms.value, cnt.value)
    return out
