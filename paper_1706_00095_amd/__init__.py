"""Python binding of libcg (argument marshalling only).

Every function has the name and the argument order of its C entry point in
include/cg.h.  Tensors are torch CUDA (ROCm) tensors used purely as device
memory; streams are torch.cuda.Stream objects (or None for the current
stream).  Nothing here computes: a missing or unloadable libcg.so raises.
"""
import ctypes as C
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.environ.get("CG_LIB_PATH", os.path.join(_HERE, "libcg.so"))

CG_OK, CG_EINVAL, CG_ENOSPC, CG_EUNSUPPORTED, CG_EHIP = 0, -1, -2, -3, -4
CG_PASS_FWD, CG_PASS_BWD_DATA, CG_PASS_BWD_WEIGHT = 0, 1, 2
CG_STEP_OVERLAP, CG_STEP_SERIAL, CG_STEP_JOIN, CG_STEP_TREE_SUM, CG_STEP_BF16, CG_STEP_BF16X3 = 0, 1, 2, 4, 8, 16
CG_MATH_FP32, CG_MATH_BF16, CG_MATH_BF16X3 = 0, 1, 2
CG_TYPE_FP32, CG_TYPE_BF16 = 0, 1
CG_MAX_PEERS = 64
CG_NOALLOC_SCRATCH_BYTES = 64 << 20
LAYER_KINDS = {"conv": 0, "relu": 1, "lrn": 2, "maxpool": 3, "avgpool": 4, "fc": 5, "dropout": 6,
               "concat": 7, "softmax_ce": 8}

EXPORTS = [
    "cg_conv_out_shape", "cg_conv_workspace_bytes", "cg_conv_fwd", "cg_conv_bwd_data", "cg_conv_bwd_weight", "cg_conv_bwd_weight_noalloc",
    "cg_conv_fwd_math", "cg_conv_bwd_data_math", "cg_conv_bwd_weight_math",
    "cg_grad_reduce_sgd", "cg_grad_reduce_sgd_multi", "cg_grad_reduce_sgd_tree", "cg_grad_reduce_sgd_tree_multi", "cg_net_create", "cg_net_destroy", "cg_net_param_count", "cg_net_layer_fused", "cg_net_bind",
    "cg_net_workspace_bytes", "cg_train_step", "cg_net_tensor", "cg_net_tensor_image_stride", "cg_strerror", "cg_version", "cg_last_hip_error", "cg_debug_conv_operand", "cg_debug_copy", "cg_debug_stream", "cg_debug_mfma_loop", "cg_debug_launch_count", "cg_debug_fuse_lrn_pool", "cg_debug_patch_min_tiles", "cg_debug_resident_blocks", "cg_debug_band_kernel", "cg_debug_direct_kernel",
    "cg_profile_enable", "cg_profile_count", "cg_profile_get",
    "cg_dropout_fwd", "cg_dropout_bwd", "cg_layernorm_fwd", "cg_layernorm_workspace_bytes", "cg_layernorm_bwd",
    "cg_dropout_add_layernorm_fwd", "cg_dropout_add_layernorm_bwd",
    "cg_attn_workspace_bytes", "cg_attn_fwd", "cg_attn_bwd",
]


class CgError(RuntimeError):
    def __init__(self, code, where):
        self.code = code
        super().__init__(f"{where}: {strerror(code)} (code {code})")


class cg_conv_desc(C.Structure):
    _fields_ = [(n, C.c_int) for n in
                ("N", "C", "H", "W", "M", "KH", "KW", "stride_h", "stride_w", "pad_h", "pad_w", "groups")]


class cg_sgd(C.Structure):
    _fields_ = [("lr", C.c_float), ("mu", C.c_float), ("wd", C.c_float), ("grad_scale", C.c_float)]


class cg_layer_desc(C.Structure):
    _fields_ = [("kind", C.c_int), ("n_inputs", C.c_int), ("inputs", C.c_int * 4), ("conv", cg_conv_desc),
                ("k", C.c_int), ("stride", C.c_int), ("pad", C.c_int), ("lrn_size", C.c_int),
                ("lrn_alpha", C.c_float), ("lrn_beta", C.c_float), ("lrn_kappa", C.c_float),
                ("fc_out", C.c_int), ("drop_p", C.c_float)]


class cg_drop(C.Structure):
    _fields_ = [("p", C.c_double), ("seed", C.c_uint64), ("offset", C.c_uint64)]


class cg_layernorm_desc(C.Structure):
    _fields_ = [("type", C.c_int), ("rows", C.c_int64), ("cols", C.c_int64), ("eps", C.c_float)]


class cg_attn_desc(C.Structure):
    _fields_ = [("type", C.c_int), ("B", C.c_int), ("Hq", C.c_int), ("Hkv", C.c_int), ("D", C.c_int),
                ("Tq", C.c_int64), ("Tk", C.c_int64),
                ("q_tok", C.c_int64), ("q_head", C.c_int64), ("k_tok", C.c_int64), ("k_head", C.c_int64),
                ("v_tok", C.c_int64), ("v_head", C.c_int64), ("o_tok", C.c_int64), ("o_head", C.c_int64),
                ("scale", C.c_float), ("causal", C.c_int), ("buckets", C.c_int), ("max_distance", C.c_int), ("both", C.c_int)]


class cg_profile_record(C.Structure):
    _fields_ = [("kernel", C.c_char * 64), ("pass_", C.c_char * 32), ("layer", C.c_int), ("ms", C.c_float),
                ("flops", C.c_double), ("bytes", C.c_double)]


_lib = None


def lib():
    """The loaded shared library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is missing: run `python -c 'import __graft_entry__ as g; g.build()'`")
        L = C.CDLL(LIB_PATH)
        vp, sz, ip = C.c_void_p, C.c_size_t, C.POINTER(C.c_int)
        dp = C.POINTER(cg_conv_desc)
        L.cg_conv_out_shape.argtypes = [dp, ip, ip]
        L.cg_conv_workspace_bytes.argtypes = [dp, C.c_int]
        L.cg_conv_workspace_bytes.restype = sz
        L.cg_conv_fwd.argtypes = [dp, vp, vp, vp, vp, vp, sz, vp]
        L.cg_conv_bwd_data.argtypes = [dp, vp, vp, vp, vp, sz, vp]
        L.cg_conv_bwd_weight.argtypes = [dp, vp, vp, vp, vp, vp, sz, vp]
        L.cg_conv_bwd_weight_noalloc.argtypes = [dp, vp, vp, vp, vp, vp]
        L.cg_conv_fwd_math.argtypes = [dp, vp, vp, vp, vp, vp, sz, C.c_int, vp]
        L.cg_conv_bwd_data_math.argtypes = [dp, vp, vp, vp, vp, sz, C.c_int, vp]
        L.cg_conv_bwd_weight_math.argtypes = [dp, vp, vp, vp, vp, vp, sz, C.c_int, vp]
        L.cg_grad_reduce_sgd.argtypes = [vp, vp, vp, C.POINTER(vp), C.c_int, sz, C.POINTER(cg_sgd), vp]
        L.cg_grad_reduce_sgd_multi.argtypes = [C.c_int, C.POINTER(vp), C.POINTER(vp), C.POINTER(vp),
                                               C.POINTER(C.POINTER(vp)), C.c_int, C.POINTER(sz), C.POINTER(cg_sgd), vp]
        L.cg_grad_reduce_sgd_tree.argtypes = L.cg_grad_reduce_sgd.argtypes
        L.cg_grad_reduce_sgd_tree_multi.argtypes = L.cg_grad_reduce_sgd_multi.argtypes
        L.cg_net_create.argtypes = [C.POINTER(cg_layer_desc), C.c_int, C.c_int, C.c_int, C.c_int, C.c_int,
                                    C.POINTER(vp)]
        L.cg_net_destroy.argtypes = [vp]
        L.cg_debug_copy.argtypes = [vp, vp, sz, vp]
        L.cg_debug_stream.argtypes = [vp, vp, vp, sz, C.c_int, vp]
        L.cg_debug_mfma_loop.argtypes = [vp, C.c_int, C.c_int, vp]
        L.cg_debug_launch_count.restype = C.c_ulonglong
        L.cg_net_param_count.argtypes = [vp, C.c_int]
        L.cg_net_param_count.restype = C.c_longlong
        L.cg_net_layer_fused.argtypes = [vp, C.c_int]
        L.cg_net_layer_fused.restype = C.c_int
        L.cg_net_tensor_image_stride.argtypes = [vp, C.c_int]
        L.cg_net_tensor_image_stride.restype = C.c_longlong
        L.cg_net_bind.argtypes = [vp, C.c_int, vp, vp, vp, C.POINTER(vp), C.c_int]
        L.cg_net_workspace_bytes.argtypes = [vp]
        L.cg_net_workspace_bytes.restype = sz
        L.cg_train_step.argtypes = [vp, vp, vp, C.POINTER(vp), C.POINTER(cg_sgd), vp, sz, vp, vp, vp, C.c_int]
        L.cg_net_tensor.argtypes = [vp, C.c_int, C.c_int, vp, C.POINTER(vp), C.POINTER(sz)]
        L.cg_debug_conv_operand.argtypes = [dp, C.c_int, C.c_int, C.c_uint, C.c_uint, C.c_uint,
                                            C.POINTER(C.c_longlong), ip]
        L.cg_profile_enable.argtypes = [C.c_int]
        L.cg_profile_get.argtypes = [C.c_int, C.POINTER(cg_profile_record)]
        i64, rp, np_ = C.c_int64, C.POINTER(cg_drop), C.POINTER(cg_layernorm_desc)
        L.cg_dropout_fwd.argtypes = [rp, C.c_int, i64, i64, vp, i64, vp, i64, vp, i64, vp]
        L.cg_dropout_bwd.argtypes = [rp, C.c_int, i64, i64, vp, i64, vp, i64, vp]
        L.cg_layernorm_workspace_bytes.argtypes = [np_]
        L.cg_layernorm_workspace_bytes.restype = sz
        L.cg_layernorm_fwd.argtypes = [np_, vp, i64, vp, vp, vp, i64, vp, vp, vp]
        L.cg_layernorm_bwd.argtypes = [np_, vp, i64, vp, i64, vp, vp, vp, vp, i64, vp, i64, vp, vp, vp, sz, vp]
        L.cg_dropout_add_layernorm_fwd.argtypes = [np_, rp, vp, i64, vp, i64, vp, vp, vp, i64, vp, i64, vp, vp, vp]
        L.cg_dropout_add_layernorm_bwd.argtypes = [np_, rp, vp, i64, vp, i64, vp, i64, vp, vp, vp, vp, i64, vp, i64, vp, vp, vp, sz, vp]
        ap = C.POINTER(cg_attn_desc)
        L.cg_attn_workspace_bytes.argtypes = [ap, C.c_int]
        L.cg_attn_workspace_bytes.restype = sz
        L.cg_attn_fwd.argtypes = [ap, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.cg_attn_bwd.argtypes = [ap, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.cg_strerror.argtypes = [C.c_int]
        L.cg_strerror.restype = C.c_char_p
        L.cg_version.restype = C.c_char_p
        L.cg_last_hip_error.restype = C.c_int
        _lib = L
    return _lib


def strerror(code):
    return lib().cg_strerror(code).decode()


def version():
    return lib().cg_version().decode()


def _check(rc, where):
    if rc != CG_OK:
        raise CgError(rc, where)


def _ptr(t):
    if t is None:
        return None
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.is_contiguous()):
        raise TypeError("expected a contiguous device tensor")
    return t.data_ptr()


# the handle of torch.cuda.current_stream() without an object made for it, which takes 3 us a call
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) if hasattr(torch._C, "_cuda_getDevice") else None


def _stream(s):
    if s is None:
        if _raw_stream is not None:
            return _raw_stream(torch._C._cuda_getDevice())
        s = torch.cuda.current_stream()
    return s.cuda_stream


def _ptr_array(tensors):
    arr = (C.c_void_p * max(len(tensors), 1))()
    for i, t in enumerate(tensors):
        arr[i] = _ptr(t)
    return arr


def conv_desc(N, Cin, H, W, M, KH, KW=None, stride=1, pad=0, groups=1):
    return cg_conv_desc(N, Cin, H, W, M, KH, KH if KW is None else KW, stride, stride, pad, pad, groups)


def cg_conv_out_shape(d):
    oh, ow = C.c_int(), C.c_int()
    _check(lib().cg_conv_out_shape(C.byref(d), C.byref(oh), C.byref(ow)), "cg_conv_out_shape")
    return oh.value, ow.value


def cg_conv_workspace_bytes(d, which):
    return int(lib().cg_conv_workspace_bytes(C.byref(d), which))


def _ws_args(ws):
    return (_ptr(ws), ws.numel() * ws.element_size()) if ws is not None else (None, 0)


def cg_conv_fwd(d, x, w, bias, y, ws=None, stream=None):
    _check(lib().cg_conv_fwd(C.byref(d), _ptr(x), _ptr(w), _ptr(bias), _ptr(y), *_ws_args(ws), _stream(stream)),
           "cg_conv_fwd")


def cg_conv_bwd_data(d, dy, w, dx, ws=None, stream=None):
    _check(lib().cg_conv_bwd_data(C.byref(d), _ptr(dy), _ptr(w), _ptr(dx), *_ws_args(ws), _stream(stream)),
           "cg_conv_bwd_data")


def cg_conv_bwd_weight(d, x, dy, dw, dbias, ws=None, stream=None):
    _check(lib().cg_conv_bwd_weight(C.byref(d), _ptr(x), _ptr(dy), _ptr(dw), _ptr(dbias), *_ws_args(ws),
                                    _stream(stream)), "cg_conv_bwd_weight")


def cg_conv_fwd_math(d, x, w, bias, y, ws, math, stream=None):
    _check(lib().cg_conv_fwd_math(C.byref(d), _ptr(x), _ptr(w), _ptr(bias), _ptr(y), *_ws_args(ws), math, _stream(stream)),
           "cg_conv_fwd_math")


def cg_conv_bwd_data_math(d, dy, w, dx, ws, math, stream=None):
    _check(lib().cg_conv_bwd_data_math(C.byref(d), _ptr(dy), _ptr(w), _ptr(dx), *_ws_args(ws), math, _stream(stream)),
           "cg_conv_bwd_data_math")


def cg_conv_bwd_weight_math(d, x, dy, dw, dbias, ws, math, stream=None):
    _check(lib().cg_conv_bwd_weight_math(C.byref(d), _ptr(x), _ptr(dy), _ptr(dw), _ptr(dbias), *_ws_args(ws), math,
                                         _stream(stream)), "cg_conv_bwd_weight_math")


def cg_conv_bwd_weight_noalloc(d, x, dy, dw, dbias, stream=None):
    _check(lib().cg_conv_bwd_weight_noalloc(C.byref(d), _ptr(x), _ptr(dy), _ptr(dw), _ptr(dbias), _stream(stream)),
           "cg_conv_bwd_weight_noalloc")


def _reduce_sgd(name, w, v, g_local, g_peers, n, sgd, stream):
    K = len(g_peers)
    _check(getattr(lib(), name)(_ptr(w), _ptr(v), _ptr(g_local), _ptr_array(g_peers), K, n, C.byref(sgd),
                                _stream(stream)), name)


def cg_grad_reduce_sgd(w, v, g_local, g_peers, n, sgd, stream=None):
    """g_peers: sequence of K device tensors; sgd: cg_sgd."""
    _reduce_sgd("cg_grad_reduce_sgd", w, v, g_local, g_peers, n, sgd, stream)


def cg_grad_reduce_sgd_tree(w, v, g_local, g_peers, n, sgd, stream=None):
    """The same arguments; the sum is taken in binomial-tree association."""
    _reduce_sgd("cg_grad_reduce_sgd_tree", w, v, g_local, g_peers, n, sgd, stream)


def cg_grad_reduce_sgd_tree_multi(ws, vs, gs, peers, ns, sgd, stream=None):
    """cg_grad_reduce_sgd_multi's arguments; the sums are taken in binomial-tree association."""
    cg_grad_reduce_sgd_multi(ws, vs, gs, peers, ns, sgd, stream, _name="cg_grad_reduce_sgd_tree_multi")


def cg_grad_reduce_sgd_multi(ws, vs, gs, peers, ns, sgd, stream=None, _name="cg_grad_reduce_sgd_multi"):
    """One launch for several buckets: ws, vs, gs sequences of device tensors, peers a sequence of
    sequences of K device tensors each, ns the element counts."""
    nb = len(ws)
    K = len(peers[0]) if nb else 0
    assert all(len(p) == K for p in peers)
    rows = [_ptr_array(p) for p in peers]
    table = (C.POINTER(C.c_void_p) * max(nb, 1))()
    for i, r in enumerate(rows):
        table[i] = C.cast(r, C.POINTER(C.c_void_p))
    counts = (C.c_size_t * max(nb, 1))(*ns)
    _check(getattr(lib(), _name)(nb, _ptr_array(ws), _ptr_array(vs), _ptr_array(gs), table, K, counts,
                                 C.byref(sgd), _stream(stream)), _name)


# ---- the operators of an attention sublayer ----

_TYPES = {torch.float32: CG_TYPE_FP32, torch.bfloat16: CG_TYPE_BF16}


def drop(p, seed, offset=0):
    """The numbers that say which elements a dropout drops: the same for a layer's forward and backward pass."""
    return cg_drop(p, seed & 0xFFFFFFFFFFFFFFFF, offset & 0xFFFFFFFFFFFFFFFF)


def _type_of(t):
    code = _TYPES.get(t.dtype)
    if code is None:
        raise TypeError(f"expected a tensor of torch.float32 or torch.bfloat16, got {t.dtype}")
    return code


def _shape_of_rows(t):
    """(rows, columns) of a tensor of any number of dimensions: the last one is a row's."""
    if t.dim() < 1:
        raise ValueError("expected a tensor of rows")
    cols = t.shape[-1]
    return (t.shape[0] if t.dim() == 2 else t.numel() // cols if cols else 0), cols


def _row_args(t, like, what):
    """(pointer, elements from a row to the next) of a tensor of `like`'s shape and type; its rows may lie in wider ones."""
    if t is None:
        return None, 0
    if t is not like and t.shape != like.shape:
        raise ValueError(f"{what}: expected the shape {tuple(like.shape)}, got {tuple(t.shape)}")
    if t.dtype is not like.dtype or not t.is_cuda:
        raise TypeError(f"{what}: expected a device tensor of {like.dtype}")
    steps = t.stride()
    if len(steps) == 2:
        rows, cols = t.shape
        if steps[1] != 1 and cols > 1:
            raise ValueError(f"{what}: the elements of a row have to lie next to each other")
        return t.data_ptr(), (steps[0] if rows > 1 else cols)
    if not t.is_contiguous():
        raise ValueError(f"{what}: tensors of other than two dimensions have to be contiguous")
    return t.data_ptr(), t.shape[-1]


def _weights(t, n, what):
    if t is None:
        return None
    if t.numel() != n or t.dtype is not torch.float32 or not t.is_contiguous() or not t.is_cuda:
        raise TypeError(f"{what}: expected a contiguous device tensor of {n} float32")
    return t.data_ptr()


def cg_dropout_fwd(drop, x, add, y, stream=None):
    """y = drop(x) + add (None: nothing is added)."""
    _check(lib().cg_dropout_fwd(drop, _type_of(x), *_shape_of_rows(x), *_row_args(x, x, "x"), *_row_args(add, x, "add"),
                                *_row_args(y, x, "y"), _stream(stream)), "cg_dropout_fwd")


def cg_dropout_bwd(drop, dy, dx, stream=None):
    _check(lib().cg_dropout_bwd(drop, _type_of(dy), *_shape_of_rows(dy), *_row_args(dy, dy, "dy"), *_row_args(dx, dy, "dx"),
                                _stream(stream)), "cg_dropout_bwd")


def layernorm_desc(x, eps=1e-5):
    """Descriptor for tensors of x's type and shape."""
    return cg_layernorm_desc(_type_of(x), *_shape_of_rows(x), eps)


def cg_layernorm_workspace_bytes(d):
    return int(lib().cg_layernorm_workspace_bytes(d))


def _norm_tensor(d, x, what):
    rows, cols = d.rows, d.cols
    if _TYPES.get(x.dtype) != d.type or (x.shape != (rows, cols) and _shape_of_rows(x) != (rows, cols)):
        raise ValueError(f"{what}: not of the descriptor's type and shape")


def cg_layernorm_fwd(d, x, gamma, beta, y, mean=None, rstd=None, stream=None):
    _norm_tensor(d, x, "x")
    n, r = d.cols, d.rows
    _check(lib().cg_layernorm_fwd(d, *_row_args(x, x, "x"), _weights(gamma, n, "gamma"), _weights(beta, n, "beta"), *_row_args(y, x, "y"),
                                  _weights(mean, r, "mean"), _weights(rstd, r, "rstd"), _stream(stream)), "cg_layernorm_fwd")


def cg_layernorm_bwd(d, dy, x, gamma, mean, rstd, dsum, dx, dgamma, dbeta, ws, stream=None):
    _norm_tensor(d, x, "x")
    n, r = d.cols, d.rows
    _check(lib().cg_layernorm_bwd(d, *_row_args(dy, x, "dy"), *_row_args(x, x, "x"), _weights(gamma, n, "gamma"), _weights(mean, r, "mean"),
                                  _weights(rstd, r, "rstd"), *_row_args(dsum, x, "dsum"), *_row_args(dx, x, "dx"), _weights(dgamma, n, "dgamma"),
                                  _weights(dbeta, n, "dbeta"), *_ws_args(ws), _stream(stream)), "cg_layernorm_bwd")


def cg_dropout_add_layernorm_fwd(d, drop, branch, x, gamma, beta, total, y, mean=None, rstd=None, stream=None):
    """total = x + drop(branch); y = layer norm of total."""
    _norm_tensor(d, x, "x")
    n, r = d.cols, d.rows
    _check(lib().cg_dropout_add_layernorm_fwd(d, drop, *_row_args(branch, x, "branch"), *_row_args(x, x, "x"), _weights(gamma, n, "gamma"),
                                              _weights(beta, n, "beta"), *_row_args(total, x, "total"), *_row_args(y, x, "y"),
                                              _weights(mean, r, "mean"), _weights(rstd, r, "rstd"), _stream(stream)),
           "cg_dropout_add_layernorm_fwd")


def cg_dropout_add_layernorm_bwd(d, drop, dy, dsum, total, gamma, mean, rstd, dx, dbranch, dgamma, dbeta, ws, stream=None):
    _norm_tensor(d, total, "total")
    n, r = d.cols, d.rows
    _check(lib().cg_dropout_add_layernorm_bwd(d, drop, *_row_args(dy, total, "dy"), *_row_args(dsum, total, "dsum"), *_row_args(total, total, "total"),
                                              _weights(gamma, n, "gamma"), _weights(mean, r, "mean"), _weights(rstd, r, "rstd"),
                                              *_row_args(dx, total, "dx"), *_row_args(dbranch, total, "dbranch"), _weights(dgamma, n, "dgamma"),
                                              _weights(dbeta, n, "dbeta"), *_ws_args(ws), _stream(stream)), "cg_dropout_add_layernorm_bwd")


def attn_desc(q, k, v, o, B, scale, causal=False, buckets=0, max_distance=0, both=False):
    """Descriptor of attention over B packed sequences: q, o [Tq][Hq][D], k, v [Tk][Hkv][D], of any token and head strides."""
    if q.dim() != 3 or k.dim() != 3 or k.shape != v.shape or q.shape != o.shape:
        raise ValueError("expected q and o of one shape [tokens][heads][D], k and v of another with the same D")
    Tq, Hq, D = q.shape
    Tk, Hkv, Dk = k.shape
    (qt, qh, q1), (kt, kh, k1), (vt, vh, v1), (ot, oh, o1) = q.stride(), k.stride(), v.stride(), o.stride()
    if D != Dk:
        raise ValueError("expected q and o of one shape [tokens][heads][D], k and v of another with the same D")
    dtype = q.dtype
    if k.dtype is not dtype or v.dtype is not dtype or o.dtype is not dtype:
        raise TypeError("q, k, v and o have to be of one type")
    if not (q1 == k1 == v1 == o1 == 1) and D > 1:
        raise ValueError("the elements of a head have to lie next to each other")
    return cg_attn_desc(_type_of(q), B, Hq, Hkv, D, Tq, Tk, qt, qh, kt, kh, vt, vh, ot, oh, scale, causal, buckets, max_distance, both)


def cg_attn_workspace_bytes(d, which):
    return int(lib().cg_attn_workspace_bytes(d, which))


_DTYPES = {code: dtype for dtype, code in _TYPES.items()}


def _heads(dtype, shape, steps, t, what):
    """The pointer of a tensor [T][H][D] with the descriptor's type, shape and strides."""
    if t is None:
        return None
    if t.dtype is not dtype or not t.is_cuda:
        raise TypeError(f"{what}: expected a device tensor of the descriptor's type")
    if t.shape != shape or (t.stride() != steps and t.numel() > 0 and any(n > 1 and a != b for n, a, b in zip(shape, t.stride(), steps))):
        raise ValueError(f"{what}: not of the descriptor's shape and strides")
    return t.data_ptr()


def _lengths(t, d, what):
    if t is None:
        return None
    if not t.is_cuda or t.dtype is not torch.int32 or not t.is_contiguous() or t.numel() != d.B + 1:
        raise TypeError(f"{what}: expected a contiguous device tensor of {d.B + 1} int32")
    return t.data_ptr()


def cg_attn_fwd(d, q, k, v, cu_q, cu_k, bias, o, lse, o_rest=None, ws=None, stream=None):
    t, of_q, of_k = _DTYPES.get(d.type), (d.Tq, d.Hq, d.D), (d.Tk, d.Hkv, d.D)
    o_steps = (d.o_tok, d.o_head, 1)
    _check(lib().cg_attn_fwd(d, _heads(t, of_q, (d.q_tok, d.q_head, 1), q, "q"), _heads(t, of_k, (d.k_tok, d.k_head, 1), k, "k"),
                             _heads(t, of_k, (d.v_tok, d.v_head, 1), v, "v"), _lengths(cu_q, d, "cu_q"), _lengths(cu_k, d, "cu_k"),
                             _weights(bias, d.Hq * d.buckets, "bias"), _heads(t, of_q, o_steps, o, "o"), _weights(lse, d.Hq * d.Tq, "lse"),
                             _heads(t, of_q, o_steps, o_rest, "o_rest"), *_ws_args(ws), _stream(stream)), "cg_attn_fwd")


def cg_attn_bwd(d, d_o, q, k, v, cu_q, cu_k, bias, o, o_rest, lse, dq, dk, dv, dbias, ws, stream=None):
    t, of_q, of_k, n = _DTYPES.get(d.type), (d.Tq, d.Hq, d.D), (d.Tk, d.Hkv, d.D), d.Hq * d.buckets
    q_steps, k_steps, v_steps, o_steps = (d.q_tok, d.q_head, 1), (d.k_tok, d.k_head, 1), (d.v_tok, d.v_head, 1), (d.o_tok, d.o_head, 1)
    _check(lib().cg_attn_bwd(d, _heads(t, of_q, o_steps, d_o, "d_o"), _heads(t, of_q, q_steps, q, "q"), _heads(t, of_k, k_steps, k, "k"),
                             _heads(t, of_k, v_steps, v, "v"), _lengths(cu_q, d, "cu_q"), _lengths(cu_k, d, "cu_k"), _weights(bias, n, "bias"),
                             _heads(t, of_q, o_steps, o, "o"), _heads(t, of_q, o_steps, o_rest, "o_rest"), _weights(lse, d.Hq * d.Tq, "lse"),
                             _heads(t, of_q, q_steps, dq, "dq"), _heads(t, of_k, k_steps, dk, "dk"), _heads(t, of_k, v_steps, dv, "dv"),
                             _weights(dbias, n, "dbias"), *_ws_args(ws), _stream(stream)), "cg_attn_bwd")


def cg_debug_patch_min_tiles(tiles):
    _check(lib().cg_debug_patch_min_tiles(int(tiles)), "cg_debug_patch_min_tiles")


def cg_debug_resident_blocks(blocks):
    _check(lib().cg_debug_resident_blocks(int(blocks)), "cg_debug_resident_blocks")


def cg_debug_direct_kernel(on):
    _check(lib().cg_debug_direct_kernel(int(bool(on))), "cg_debug_direct_kernel")


def cg_debug_band_kernel(on):
    _check(lib().cg_debug_band_kernel(int(bool(on))), "cg_debug_band_kernel")


def cg_debug_copy(dst, src, nbytes, stream=None):
    _check(lib().cg_debug_copy(_ptr(dst), _ptr(src), nbytes, _stream(stream)), "cg_debug_copy")


def cg_debug_fuse_lrn_pool(mode):
    _check(lib().cg_debug_fuse_lrn_pool(int(mode)), "cg_debug_fuse_lrn_pool")


def cg_debug_launch_count():
    return int(lib().cg_debug_launch_count())


def cg_debug_stream(dst, src, src2, nbytes, mode, stream=None):
    _check(lib().cg_debug_stream(_ptr(dst), _ptr(src), _ptr(src2), nbytes, mode, _stream(stream)), "cg_debug_stream")


def cg_debug_mfma_loop(out, blocks, iters, stream=None):
    _check(lib().cg_debug_mfma_loop(_ptr(out), blocks, iters, _stream(stream)), "cg_debug_mfma_loop")


def cg_debug_conv_operand(d, which_pass, operand, row, k, group):
    """(element offset in floats, valid) -- host-side evaluation, launches nothing."""
    off, ok = C.c_longlong(), C.c_int()
    _check(lib().cg_debug_conv_operand(C.byref(d), which_pass, operand, row, k, group, C.byref(off), C.byref(ok)),
           "cg_debug_conv_operand")
    return off.value, bool(ok.value)


def cg_profile_enable(on):
    _check(lib().cg_profile_enable(1 if on else 0), "cg_profile_enable")


def cg_profile_count():
    return int(lib().cg_profile_count())


def cg_profile_get(i):
    r = cg_profile_record()
    _check(lib().cg_profile_get(i, C.byref(r)), "cg_profile_get")
    return dict(kernel=r.kernel.decode(), pass_=r.pass_.decode(), layer=r.layer, ms=float(r.ms),
                flops=float(r.flops), bytes=float(r.bytes))


def layer_descs(layers):
    """cg_layer_desc array from the plain-dict layer list used throughout the tests."""
    arr = (cg_layer_desc * len(layers))()
    for i, ly in enumerate(layers):
        d = arr[i]
        d.kind = LAYER_KINDS[ly["kind"]]
        d.n_inputs = len(ly["inputs"])
        for k, s in enumerate(ly["inputs"]):
            d.inputs[k] = s
        if ly["kind"] == "conv":
            d.conv = cg_conv_desc(0, 0, 0, 0, ly["M"], ly["k"], ly["k"], ly["stride"], ly["stride"], ly["pad"],
                                  ly["pad"], ly["groups"])
        elif ly["kind"] == "maxpool":
            d.k, d.stride, d.pad = ly["k"], ly["stride"], ly["pad"]
        elif ly["kind"] == "lrn":
            d.lrn_size, d.lrn_alpha, d.lrn_beta, d.lrn_kappa = ly["size"], ly["alpha"], ly["beta"], ly["kappa"]
        elif ly["kind"] == "fc":
            d.fc_out = ly["out"]
        elif ly["kind"] == "dropout":
            d.drop_p = ly["p"]
    return arr


class Net:
    """Owner of a cg_net handle (cg_net_create / cg_net_destroy)."""

    def __init__(self, layers, B, in_shape):
        self.layers = layers
        self.B = B
        self.handle = C.c_void_p()
        descs = layer_descs(layers)
        _check(lib().cg_net_create(descs, len(layers), B, *in_shape, C.byref(self.handle)), "cg_net_create")
        self._keep = []

    def close(self):
        if self.handle:
            lib().cg_net_destroy(self.handle)
            self.handle = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def cg_net_param_count(net, layer):
    n = lib().cg_net_param_count(net.handle, layer)
    if n < 0:
        raise CgError(int(n), "cg_net_param_count")
    return int(n)


def cg_net_layer_fused(net, layer):
    r = lib().cg_net_layer_fused(net.handle, layer)
    if r < 0:
        raise CgError(int(r), "cg_net_layer_fused")
    return int(r)


def cg_net_bind(net, layer, w, v, g_local, g_peers):
    net._keep.append((w, v, g_local, list(g_peers)))
    _check(lib().cg_net_bind(net.handle, layer, _ptr(w), _ptr(v), _ptr(g_local), _ptr_array(g_peers), len(g_peers)),
           "cg_net_bind")


def cg_net_workspace_bytes(net):
    return int(lib().cg_net_workspace_bytes(net.handle))


def cg_train_step(net, x, labels, dropout_masks, sgd, ws, compute_stream, update_stream, loss_dev, flags=0):
    """dropout_masks: {layer index: uint8 device tensor} or None."""
    L = len(net.layers)
    marr = None
    if dropout_masks:
        marr = (C.c_void_p * L)()
        for i, t in dropout_masks.items():
            marr[i] = _ptr(t)
    _check(lib().cg_train_step(net.handle, _ptr(x), _ptr(labels), marr, C.byref(sgd), *_ws_args(ws),
                               _stream(compute_stream), update_stream.cuda_stream if update_stream is not None else None,
                               _ptr(loss_dev), flags), "cg_train_step")


def cg_net_tensor(net, layer, which, ws):
    """A float32 view (torch tensor sharing the workspace memory) of a layer's output or gradient."""
    p, n = C.c_void_p(), C.c_size_t()
    _check(lib().cg_net_tensor(net.handle, layer, which, _ptr(ws), C.byref(p), C.byref(n)), "cg_net_tensor")
    off = (p.value - ws.data_ptr()) // 4
    flat = ws.view(torch.float32)[off:off + n.value]
    if which == 0:
        stride = int(lib().cg_net_tensor_image_stride(net.handle, layer))
        per_image = n.value - (net.B - 1) * stride
        if per_image != stride:       # a channel slice of a wider tensor: gathered into a dense copy
            return torch.as_strided(flat, (net.B, per_image), (stride, 1)).reshape(-1)
    return flat
