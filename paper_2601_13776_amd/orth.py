"""Thin ctypes binding of liborth (include/orth.h).

Argument marshalling only: every step of the path runs in the HIP library.
Functions keep the C names.  Tensors are torch tensors on the GPU; the
library runs on torch's current stream.  If liborth.so is missing the first
call raises: there is no fallback implementation.
"""

import ctypes
import os

import torch

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "liborth.so")
_lib = None

ORTH_OK, ORTH_EINVAL, ORTH_EUNSUPPORTED, ORTH_EWORKSPACE, ORTH_EHIP = range(5)
ORTH_F32, ORTH_BF16 = 0, 1
ORTH_COMPUTE_F32, ORTH_COMPUTE_BF16 = 0, 1
ORTH_PRESCALE_NONE, ORTH_PRESCALE_FROBENIUS, ORTH_PRESCALE_SPECTRAL = 0, 1, 2
ORTH_CHECK_GRAM, ORTH_CHECK_CONV, ORTH_CHECK_CONV_ADJOINT = 0, 1, 2
ORTH_NOALLOC_SCRATCH_BYTES = 64 << 20   # the allocation-free entry point's device scratch per GPU

EXPORTED = [
    "orth_orthogonalize_workspace_size", "orth_orthogonalize_batched", "orth_orthogonalize_batched_noalloc",
    "orth_orthogonalize_vjp_workspace_size", "orth_orthogonalize_vjp_batched",
    "orth_orthogonalize_save_workspace_size", "orth_orthogonalize_save_batched", "orth_aoc_param_shapes",
    "orth_build_conv_kernels_workspace_size", "orth_build_conv_kernels_batched", "orth_build_conv_kernel",
    "orth_build_conv_kernels_vjp_workspace_size", "orth_build_conv_kernels_vjp_batched",
    "orth_build_conv_kernels_save_workspace_size", "orth_build_conv_kernels_save_batched",
    "orth_build_conv_kernels_vjp_saved_batched", "orth_conv_apply",
    "orth_exp_map_workspace_size", "orth_exp_map_batched", "orth_conv_exp_workspace_size", "orth_conv_exp_batched",
    "orth_linear_apply", "orth_linear_grad_weight_workspace_size", "orth_linear_grad_weight",
    "orth_linear_xent_workspace_size", "orth_linear_xent", "orth_linear_xent_vjp_workspace_size",
    "orth_linear_xent_vjp", "orth_grad_norm_workspace_size", "orth_grad_norm_batched", "orth_grad_clip_batched",
    "orth_check_workspace_size", "orth_check_norm", "orth_status_string", "orth_last_error",
    "orth_version", "orth_timing_enable", "orth_timing_filter", "orth_timing_reset", "orth_timing_read",
    "orth_timing_span", "orth_timing_names",
]


class OrthError(RuntimeError):
    def __init__(self, code, where):
        self.code = code
        msg = lib().orth_last_error().decode()
        super().__init__(f"{where}: {lib().orth_status_string(code).decode()} ({msg})")


class orth_mat(ctypes.Structure):
    _fields_ = [("in_", ctypes.c_void_p), ("out", ctypes.c_void_p), ("rows", ctypes.c_int32),
                ("cols", ctypes.c_int32), ("ld_in", ctypes.c_int64), ("ld_out", ctypes.c_int64)]


class orth_bjorck_opts(ctypes.Structure):
    _fields_ = [("iters", ctypes.c_int32), ("beta", ctypes.c_float), ("prescale", ctypes.c_int32),
                ("in_dtype", ctypes.c_int32), ("out_dtype", ctypes.c_int32), ("compute", ctypes.c_int32),
                ("power_iters", ctypes.c_int32), ("u", ctypes.c_void_p), ("tile", ctypes.c_int32),
                ("saved", ctypes.c_int32)]


class orth_vjp_mat(ctypes.Structure):
    _fields_ = [("w", ctypes.c_void_p), ("grad_out", ctypes.c_void_p), ("grad_in", ctypes.c_void_p),
                ("rows", ctypes.c_int32), ("cols", ctypes.c_int32), ("ld_w", ctypes.c_int64),
                ("ld_grad_out", ctypes.c_int64), ("ld_grad_in", ctypes.c_int64)]


class orth_exp_opts(ctypes.Structure):
    _fields_ = [("terms", ctypes.c_int32), ("power_iters", ctypes.c_int32), ("u", ctypes.c_void_p),
                ("in_dtype", ctypes.c_int32), ("out_dtype", ctypes.c_int32)]


class orth_conv_exp_desc(ctypes.Structure):
    _fields_ = [("channels", ctypes.c_int32), ("k", ctypes.c_int32), ("terms", ctypes.c_int32),
                ("scale", ctypes.c_float), ("kernel", ctypes.c_void_p), ("out", ctypes.c_void_p)]


class orth_conv_geom(ctypes.Structure):
    _fields_ = [("cin", ctypes.c_int32), ("cout", ctypes.c_int32), ("k", ctypes.c_int32),
                ("stride", ctypes.c_int32), ("dilation", ctypes.c_int32), ("groups", ctypes.c_int32)]


class orth_conv_desc(ctypes.Structure):
    _fields_ = [("geom", orth_conv_geom), ("rko", ctypes.c_void_p), ("proj", ctypes.c_void_p),
                ("kernel", ctypes.c_void_p)]


class orth_conv_vjp_desc(ctypes.Structure):
    _fields_ = [("geom", orth_conv_geom), ("rko", ctypes.c_void_p), ("proj", ctypes.c_void_p),
                ("grad_kernel", ctypes.c_void_p), ("grad_rko", ctypes.c_void_p), ("grad_proj", ctypes.c_void_p)]


class orth_conv_apply_args(ctypes.Structure):
    _fields_ = [("geom", orth_conv_geom), ("kernel", ctypes.c_void_p), ("kernel_dtype", ctypes.c_int32),
                ("transposed", ctypes.c_int32), ("x", ctypes.c_void_p), ("y", ctypes.c_void_p),
                ("batch", ctypes.c_int32), ("height", ctypes.c_int32), ("width", ctypes.c_int32)]


class orth_check_args(ctypes.Structure):
    _fields_ = [("mode", ctypes.c_int32), ("mats", ctypes.POINTER(orth_mat)), ("n_mats", ctypes.c_int32),
                ("mat_dtype", ctypes.c_int32), ("kernel", ctypes.c_void_p), ("kernel_dtype", ctypes.c_int32),
                ("geom", orth_conv_geom), ("x", ctypes.c_void_p), ("batch", ctypes.c_int32),
                ("height", ctypes.c_int32), ("width", ctypes.c_int32)]


class orth_linear_args(ctypes.Structure):
    _fields_ = [("x", ctypes.c_void_p), ("w", ctypes.c_void_p), ("y", ctypes.c_void_p), ("offsets", ctypes.c_void_p),
                ("rows", ctypes.c_int32), ("groups", ctypes.c_int32), ("in_features", ctypes.c_int32),
                ("out_features", ctypes.c_int32), ("ld_x", ctypes.c_int64), ("ld_w", ctypes.c_int64),
                ("stride_w", ctypes.c_int64), ("ld_y", ctypes.c_int64), ("dtype", ctypes.c_int32),
                ("grad_dtype", ctypes.c_int32), ("transposed", ctypes.c_int32)]


class orth_linear_xent_args(ctypes.Structure):
    _fields_ = [("x", ctypes.c_void_p), ("w", ctypes.c_void_p), ("targets", ctypes.c_void_p),
                ("rows", ctypes.c_int32), ("features", ctypes.c_int32), ("classes", ctypes.c_int32),
                ("ld_x", ctypes.c_int64), ("ld_w", ctypes.c_int64), ("scale", ctypes.c_float),
                ("dtype", ctypes.c_int32), ("piece", ctypes.c_int32)]


class orth_grad(ctypes.Structure):
    _fields_ = [("grad", ctypes.c_void_p), ("out", ctypes.c_void_p), ("rows", ctypes.c_int32),
                ("cols", ctypes.c_int32), ("ld_grad", ctypes.c_int64), ("ld_out", ctypes.c_int64),
                ("dtype", ctypes.c_int32)]


class orth_clip_opts(ctypes.Structure):
    _fields_ = [("max_norm", ctypes.c_float), ("eps", ctypes.c_float), ("norm_given", ctypes.c_int32)]


def lib():
    """Load liborth.so (once)."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise RuntimeError(f"{_LIB_PATH} is missing: build it with `python -m paper_2601_13776_amd.build`")
        L = ctypes.CDLL(_LIB_PATH)
        vp, i32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
        P = ctypes.POINTER
        L.orth_orthogonalize_workspace_size.argtypes = [P(orth_mat), i32, P(orth_bjorck_opts), P(sz)]
        L.orth_orthogonalize_batched.argtypes = [P(orth_mat), i32, P(orth_bjorck_opts), vp, sz, vp, vp]
        L.orth_orthogonalize_batched_noalloc.argtypes = [P(orth_mat), i32, P(orth_bjorck_opts), vp, vp]
        L.orth_orthogonalize_vjp_workspace_size.argtypes = [P(orth_vjp_mat), i32, P(orth_bjorck_opts), P(sz)]
        L.orth_orthogonalize_vjp_batched.argtypes = [P(orth_vjp_mat), i32, P(orth_bjorck_opts), vp, sz, vp, vp]
        L.orth_orthogonalize_save_workspace_size.argtypes = [P(orth_mat), i32, P(orth_bjorck_opts), P(sz)]
        L.orth_orthogonalize_save_batched.argtypes = [P(orth_mat), i32, P(orth_bjorck_opts), vp, sz, vp, vp]
        L.orth_aoc_param_shapes.argtypes = [P(orth_conv_geom)] + [P(i32)] * 5
        L.orth_build_conv_kernels_workspace_size.argtypes = [P(orth_conv_desc), i32, i32, P(sz)]
        L.orth_build_conv_kernels_batched.argtypes = [P(orth_conv_desc), i32, i32, vp, sz, vp]
        L.orth_build_conv_kernel.argtypes = [vp, vp, i32, i32, i32, i32, i32, i32, i32, vp, vp, sz, vp]
        L.orth_build_conv_kernels_vjp_workspace_size.argtypes = [P(orth_conv_vjp_desc), i32, i32, P(sz)]
        L.orth_build_conv_kernels_vjp_batched.argtypes = [P(orth_conv_vjp_desc), i32, i32, vp, sz, vp]
        L.orth_build_conv_kernels_save_workspace_size.argtypes = [P(orth_conv_desc), i32, i32, P(sz)]
        L.orth_build_conv_kernels_save_batched.argtypes = [P(orth_conv_desc), i32, i32, vp, sz, vp]
        L.orth_build_conv_kernels_vjp_saved_batched.argtypes = [P(orth_conv_vjp_desc), i32, i32, vp, sz, vp]
        L.orth_conv_apply.argtypes = [P(orth_conv_apply_args), vp]
        L.orth_exp_map_workspace_size.argtypes = [P(orth_mat), i32, P(orth_exp_opts), P(sz)]
        L.orth_exp_map_batched.argtypes = [P(orth_mat), i32, P(orth_exp_opts), vp, sz, vp, vp]
        L.orth_conv_exp_workspace_size.argtypes = [P(orth_conv_exp_desc), i32, i32, P(sz)]
        L.orth_conv_exp_batched.argtypes = [P(orth_conv_exp_desc), i32, i32, vp, sz, vp]
        L.orth_linear_apply.argtypes = [P(orth_linear_args), vp]
        L.orth_linear_grad_weight_workspace_size.argtypes = [P(orth_linear_args), P(sz)]
        L.orth_linear_grad_weight.argtypes = [P(orth_linear_args), vp, sz, vp]
        L.orth_linear_xent_workspace_size.argtypes = [P(orth_linear_xent_args), P(sz)]
        L.orth_linear_xent.argtypes = [P(orth_linear_xent_args), vp, vp, vp, sz, vp]
        L.orth_linear_xent_vjp_workspace_size.argtypes = [P(orth_linear_xent_args), P(sz)]
        L.orth_linear_xent_vjp.argtypes = [P(orth_linear_xent_args), vp, vp, vp, ctypes.c_int64, vp, ctypes.c_int64,
                                           vp, sz, vp]
        L.orth_grad_norm_workspace_size.argtypes = [P(orth_grad), i32, P(sz)]
        L.orth_grad_norm_batched.argtypes = [P(orth_grad), i32, vp, vp, sz, vp]
        L.orth_grad_clip_batched.argtypes = [P(orth_grad), i32, P(orth_clip_opts), vp, vp, sz, vp]
        L.orth_check_workspace_size.argtypes = [P(orth_check_args), P(sz)]
        L.orth_check_norm.argtypes = [P(orth_check_args), vp, vp, sz, vp]
        L.orth_status_string.argtypes = [ctypes.c_int]
        L.orth_status_string.restype = ctypes.c_char_p
        L.orth_last_error.restype = ctypes.c_char_p
        L.orth_timing_enable.argtypes = [i32]
        L.orth_timing_read.argtypes = [ctypes.c_char_p, P(ctypes.c_double), P(ctypes.c_int64)]
        L.orth_timing_filter.argtypes = [ctypes.c_char_p]
        L.orth_timing_span.argtypes = [ctypes.c_char_p, P(ctypes.c_double), P(ctypes.c_int64)]
        L.orth_timing_names.argtypes = [ctypes.c_char_p, sz]
        for name in EXPORTED:
            if name not in ("orth_status_string", "orth_last_error"):
                getattr(L, name).restype = ctypes.c_int
        _lib = L
    return _lib


def _check(rc, where):
    if rc != ORTH_OK:
        raise OrthError(rc, where)


def _dtype_code(t):
    if t.dtype == torch.float32:
        return ORTH_F32
    if t.dtype == torch.bfloat16:
        return ORTH_BF16
    raise TypeError(f"unsupported dtype {t.dtype}")


def _stream(stream):
    if stream is None:
        return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    return ctypes.c_void_p(stream.cuda_stream if hasattr(stream, "cuda_stream") else stream)


def _ld(t):
    if t.dim() != 2 or t.stride(1) != 1:
        raise ValueError("matrices must be 2-D with unit column stride")
    return t.stride(0)


def _workspace(nbytes, device, workspace):
    if nbytes == 0:
        return None, 0
    if workspace is not None and workspace.numel() * workspace.element_size() >= nbytes:
        return workspace, workspace.numel() * workspace.element_size()
    ws = torch.empty(nbytes, dtype=torch.uint8, device=device)
    return ws, nbytes


def _mats(ins, outs):
    arr = (orth_mat * len(ins))()
    for i, (a, b) in enumerate(zip(ins, outs)):
        if a.shape != b.shape:
            raise ValueError("input and output shapes differ")
        arr[i] = orth_mat(a.data_ptr(), b.data_ptr(), a.shape[0], a.shape[1], _ld(a), _ld(b))
    return arr


def _opts(ins, outs, iters, beta, prescale, compute, power_iters=1, u=None, tile=0, saved=0, need_u=True):
    in_dt = _dtype_code(ins[0]) if ins else ORTH_F32
    out_dt = _dtype_code(outs[0]) if outs else ORTH_F32
    for a, b in zip(ins, outs):
        if _dtype_code(a) != in_dt or _dtype_code(b) != out_dt:
            raise TypeError("all inputs (and all outputs) must share one dtype")
    pres = {"frobenius": ORTH_PRESCALE_FROBENIUS, "none": ORTH_PRESCALE_NONE,
            "spectral": ORTH_PRESCALE_SPECTRAL}[prescale]
    comp = {"f32": ORTH_COMPUTE_F32, "bf16": ORTH_COMPUTE_BF16}[compute]
    uptr = None
    if pres == ORTH_PRESCALE_SPECTRAL and ins and (need_u or u is not None):
        need = sum(min(t.shape[0], t.shape[1]) for t in ins)
        if u is None or u.dtype != torch.float32 or not u.is_contiguous() or u.numel() < need:
            raise ValueError(f"spectral pre-scaling needs u: a contiguous float32 tensor of {need} values "
                             "(min(rows, cols) per matrix, packed in batch order)")
        uptr = u.data_ptr()
    return orth_bjorck_opts(iters, beta, pres, in_dt, out_dt, comp, power_iters, uptr, tile, saved)


def orth_orthogonalize_workspace_size(ins, iters, beta=0.5, prescale="frobenius", compute="f32", outs=None,
                                      power_iters=1, u=None, tile=0):
    outs = ins if outs is None else outs
    mats = _mats(ins, outs)
    opts = _opts(ins, outs, iters, beta, prescale, compute, power_iters, u, tile)
    n = ctypes.c_size_t()
    _check(lib().orth_orthogonalize_workspace_size(mats, len(ins), ctypes.byref(opts), ctypes.byref(n)),
           "orth_orthogonalize_workspace_size")
    return n.value


def orth_orthogonalize_batched(ins, outs, iters, beta=0.5, prescale="frobenius", compute="f32", status=None,
                               workspace=None, stream=None, power_iters=1, u=None, tile=0):
    """Björck-orthogonalize every ins[i] into outs[i] (see include/orth.h).
    prescale="spectral" takes power_iters and u, the packed float32 cached
    vectors (min(rows, cols) per matrix), updated in place.  tile (0, 128
    or 256) is the bf16 tile edge of matrices with min(rows, cols) >= 1024
    (0: chosen by occupancy).
    Returns the workspace tensor so that callers can reuse it."""
    mats = _mats(ins, outs)
    opts = _opts(ins, outs, iters, beta, prescale, compute, power_iters, u, tile)
    n = ctypes.c_size_t()
    _check(lib().orth_orthogonalize_workspace_size(mats, len(ins), ctypes.byref(opts), ctypes.byref(n)),
           "orth_orthogonalize_workspace_size")
    device = ins[0].device if ins else torch.device("cuda")
    ws, nbytes = _workspace(n.value, device, workspace)
    if status is not None and (status.dtype != torch.int32 or status.numel() < len(ins)):
        raise ValueError("status must be an int32 tensor with one slot per matrix")
    rc = lib().orth_orthogonalize_batched(mats, len(ins), ctypes.byref(opts),
                                          ws.data_ptr() if ws is not None else None, nbytes,
                                          status.data_ptr() if status is not None else None, _stream(stream))
    _check(rc, "orth_orthogonalize_batched")
    return ws


def orth_orthogonalize_batched_noalloc(ins, outs, iters, beta=0.5, prescale="frobenius", compute="f32",
                                       status=None, stream=None, power_iters=1, u=None, tile=0):
    """orth_orthogonalize_batched without a workspace: the library's own
    device scratch (ORTH_NOALLOC_SCRATCH_BYTES per GPU) holds the iterates,
    so neither the library nor this binding allocates anything.  Calls on
    one GPU share the scratch and must not overlap."""
    mats = _mats(ins, outs)
    opts = _opts(ins, outs, iters, beta, prescale, compute, power_iters, u, tile)
    if status is not None and (status.dtype != torch.int32 or status.numel() < len(ins)):
        raise ValueError("status must be an int32 tensor with one slot per matrix")
    rc = lib().orth_orthogonalize_batched_noalloc(mats, len(ins), ctypes.byref(opts),
                                                  status.data_ptr() if status is not None else None,
                                                  _stream(stream))
    _check(rc, "orth_orthogonalize_batched_noalloc")


def _vjp_mats(ws, gouts, gins):
    arr = (orth_vjp_mat * len(ws))()
    for i, (w, go, gi) in enumerate(zip(ws, gouts, gins)):
        if not (w.shape == go.shape == gi.shape):
            raise ValueError("w, grad_out and grad_in shapes differ")
        arr[i] = orth_vjp_mat(w.data_ptr(), go.data_ptr(), gi.data_ptr(), w.shape[0], w.shape[1], _ld(w), _ld(go),
                              _ld(gi))
    return arr


def orth_orthogonalize_vjp_batched(ws, grads_out, grads_in, iters, beta=0.5, prescale="frobenius", compute="f32",
                                   status=None, workspace=None, stream=None, tile=0, saved=False, power_iters=1,
                                   u=None):
    """dL/dW into grads_in[i] for L depending on ws[i] through
    orth_orthogonalize_batched with the same options, given grads_out[i] =
    dL/d(output) (see include/orth.h).  grads_in share the dtype of ws,
    grads_out that of the forward outputs.  saved=True takes the forward
    iterates from `workspace`, which orth_orthogonalize_save_batched filled
    for the same ws and options.  prescale="spectral": u holds the cached
    vectors as the differentiated forward found them (read only; not needed
    with saved=True).  Returns the workspace tensor."""
    if saved and workspace is None:
        raise ValueError("saved=True needs the workspace of orth_orthogonalize_save_batched")
    if len(ws) != len(grads_out) or len(ws) != len(grads_in):
        raise ValueError("ws, grads_out and grads_in must have the same length")
    for w, gi in zip(ws, grads_in):
        if w.dtype != gi.dtype:
            raise TypeError("grads_in must have the dtype of ws")
    mats = _vjp_mats(ws, grads_out, grads_in)
    opts = _opts(ws, grads_out, iters, beta, prescale, compute, power_iters, u, tile=tile, saved=1 if saved else 0,
                 need_u=not saved)
    n = ctypes.c_size_t()
    _check(lib().orth_orthogonalize_vjp_workspace_size(mats, len(ws), ctypes.byref(opts), ctypes.byref(n)),
           "orth_orthogonalize_vjp_workspace_size")
    device = ws[0].device if ws else torch.device("cuda")
    wsp, nbytes = _workspace(n.value, device, workspace)
    if status is not None and (status.dtype != torch.int32 or status.numel() < len(ws)):
        raise ValueError("status must be an int32 tensor with one slot per matrix")
    rc = lib().orth_orthogonalize_vjp_batched(mats, len(ws), ctypes.byref(opts),
                                              wsp.data_ptr() if wsp is not None else None, nbytes,
                                              status.data_ptr() if status is not None else None, _stream(stream))
    _check(rc, "orth_orthogonalize_vjp_batched")
    return wsp


def orth_orthogonalize_save_batched(ins, outs, iters, beta=0.5, prescale="frobenius", compute="f32", status=None,
                                    workspace=None, stream=None, tile=0, power_iters=1, u=None):
    """orth_orthogonalize_batched that also keeps, in the returned workspace,
    the forward iterates that orth_orthogonalize_vjp_batched(..., saved=True,
    workspace=<it>) reuses (see include/orth.h).  outs must not be ins."""
    mats = _mats(ins, outs)
    opts = _opts(ins, outs, iters, beta, prescale, compute, power_iters, u, tile=tile)
    n = ctypes.c_size_t()
    _check(lib().orth_orthogonalize_save_workspace_size(mats, len(ins), ctypes.byref(opts), ctypes.byref(n)),
           "orth_orthogonalize_save_workspace_size")
    device = ins[0].device if ins else torch.device("cuda")
    ws, nbytes = _workspace(n.value, device, workspace)
    if status is not None and (status.dtype != torch.int32 or status.numel() < len(ins)):
        raise ValueError("status must be an int32 tensor with one slot per matrix")
    rc = lib().orth_orthogonalize_save_batched(mats, len(ins), ctypes.byref(opts),
                                               ws.data_ptr() if ws is not None else None, nbytes,
                                               status.data_ptr() if status is not None else None, _stream(stream))
    _check(rc, "orth_orthogonalize_save_batched")
    return ws


def orth_orthogonalize_vjp_workspace_size(ws, iters, beta=0.5, prescale="frobenius", compute="f32",
                                          grads_out=None, tile=0, power_iters=1):
    grads_out = ws if grads_out is None else grads_out
    mats = _vjp_mats(ws, grads_out, ws)
    opts = _opts(ws, grads_out, iters, beta, prescale, compute, power_iters, tile=tile, need_u=False)
    n = ctypes.c_size_t()
    _check(lib().orth_orthogonalize_vjp_workspace_size(mats, len(ws), ctypes.byref(opts), ctypes.byref(n)),
           "orth_orthogonalize_vjp_workspace_size")
    return n.value


def orth_aoc_param_shapes(cin, cout, k, stride=1, dilation=1, groups=1):
    g = orth_conv_geom(cin, cout, k, stride, dilation, groups)
    out = [ctypes.c_int32() for _ in range(5)]
    _check(lib().orth_aoc_param_shapes(ctypes.byref(g), *[ctypes.byref(o) for o in out]), "orth_aoc_param_shapes")
    return tuple(o.value for o in out)


def _conv_descs(layers):
    arr = (orth_conv_desc * len(layers))()
    for i, L in enumerate(layers):
        geom = orth_conv_geom(*L["geom"])
        proj = L.get("proj")
        arr[i] = orth_conv_desc(geom, L["rko"].data_ptr(), proj.data_ptr() if proj is not None else None,
                                L["kernel"].data_ptr())
    return arr


def orth_build_conv_kernels_batched(layers, workspace=None, stream=None):
    """layers: list of dicts with geom=(cin, cout, k, stride, dilation, groups),
    rko, proj (or None) and kernel tensors (contiguous, one dtype)."""
    if not layers:
        return None
    dt = _dtype_code(layers[0]["kernel"])
    for L in layers:
        for key in ("rko", "proj", "kernel"):
            t = L.get(key)
            if t is not None and (not t.is_contiguous() or _dtype_code(t) != dt):
                raise ValueError(f"{key} must be contiguous and of the kernel's dtype")
    descs = _conv_descs(layers)
    n = ctypes.c_size_t()
    _check(lib().orth_build_conv_kernels_workspace_size(descs, len(layers), dt, ctypes.byref(n)),
           "orth_build_conv_kernels_workspace_size")
    ws, nbytes = _workspace(n.value, layers[0]["kernel"].device, workspace)
    rc = lib().orth_build_conv_kernels_batched(descs, len(layers), dt, ws.data_ptr() if ws is not None else None,
                                               nbytes, _stream(stream))
    _check(rc, "orth_build_conv_kernels_batched")
    return ws


def orth_build_conv_kernel(rko, proj, cin, cout, k, stride, dilation, groups, kernel_out, workspace=None,
                           stream=None):
    return orth_build_conv_kernels_batched(
        [dict(geom=(cin, cout, k, stride, dilation, groups), rko=rko, proj=proj, kernel=kernel_out)],
        workspace, stream)


def orth_build_conv_kernels_vjp_batched(layers, workspace=None, stream=None, saved=False):
    """layers: list of dicts with geom, rko, proj (or None), grad_kernel,
    grad_rko and grad_proj (or None) tensors (contiguous, one dtype).
    Writes dL/d rko and dL/d proj given dL/d kernel.  saved=True skips the
    forward recomputation: `workspace` holds what
    orth_build_conv_kernels_save_batched left for the same layers."""
    if not layers:
        return None
    if saved and workspace is None:
        raise ValueError("saved=True needs the workspace of orth_build_conv_kernels_save_batched")
    dt = _dtype_code(layers[0]["grad_kernel"])
    arr = (orth_conv_vjp_desc * len(layers))()
    for i, L in enumerate(layers):
        for key in ("rko", "proj", "grad_kernel", "grad_rko", "grad_proj"):
            t = L.get(key)
            if t is not None and (not t.is_contiguous() or _dtype_code(t) != dt):
                raise ValueError(f"{key} must be contiguous and of one dtype")
        ptr = lambda key: L[key].data_ptr() if L.get(key) is not None else None
        arr[i] = orth_conv_vjp_desc(orth_conv_geom(*L["geom"]), ptr("rko"), ptr("proj"), ptr("grad_kernel"),
                                    ptr("grad_rko"), ptr("grad_proj"))
    n = ctypes.c_size_t()
    _check(lib().orth_build_conv_kernels_vjp_workspace_size(arr, len(layers), dt, ctypes.byref(n)),
           "orth_build_conv_kernels_vjp_workspace_size")
    ws, nbytes = _workspace(n.value, layers[0]["grad_kernel"].device, workspace)
    fn = lib().orth_build_conv_kernels_vjp_saved_batched if saved else lib().orth_build_conv_kernels_vjp_batched
    rc = fn(arr, len(layers), dt, ws.data_ptr() if ws is not None else None, nbytes, _stream(stream))
    _check(rc, "orth_build_conv_kernels_vjp_batched")
    return ws


def orth_build_conv_kernels_save_batched(layers, workspace=None, stream=None):
    """orth_build_conv_kernels_batched that also keeps, in the returned
    (composition-VJP) workspace, what orth_build_conv_kernels_vjp_batched(...,
    saved=True, workspace=<it>) reuses.  layers as for
    orth_build_conv_kernels_batched."""
    if not layers:
        return None
    dt = _dtype_code(layers[0]["kernel"])
    for L in layers:
        for key in ("rko", "proj", "kernel"):
            t = L.get(key)
            if t is not None and (not t.is_contiguous() or _dtype_code(t) != dt):
                raise ValueError(f"{key} must be contiguous and of the kernel's dtype")
    descs = _conv_descs(layers)
    n = ctypes.c_size_t()
    _check(lib().orth_build_conv_kernels_save_workspace_size(descs, len(layers), dt, ctypes.byref(n)),
           "orth_build_conv_kernels_save_workspace_size")
    ws, nbytes = _workspace(n.value, layers[0]["kernel"].device, workspace)
    rc = lib().orth_build_conv_kernels_save_batched(descs, len(layers), dt, ws.data_ptr() if ws is not None else None,
                                                    nbytes, _stream(stream))
    _check(rc, "orth_build_conv_kernels_save_batched")
    return ws


def orth_conv_apply(kernel, geom, x, transposed=False, stream=None):
    """Circular conv (or its transpose) of the float32 NCHW batch x with the
    explicit kernel; returns the new output tensor."""
    if x.dtype != torch.float32 or not x.is_contiguous() or not kernel.is_contiguous():
        raise ValueError("x must be contiguous float32 and the kernel contiguous")
    cin, cout, k, s, d, g = geom
    b = x.shape[0]
    if transposed:
        h, w = x.shape[2] * s, x.shape[3] * s
        y = torch.empty(b, cin, h, w, dtype=torch.float32, device=x.device)
    else:
        h, w = x.shape[2], x.shape[3]
        y = torch.empty(b, cout, h // s, w // s, dtype=torch.float32, device=x.device)
    args = orth_conv_apply_args(orth_conv_geom(*geom), kernel.data_ptr(), _dtype_code(kernel), int(transposed),
                                x.data_ptr(), y.data_ptr(), b, h, w)
    _check(lib().orth_conv_apply(ctypes.byref(args), _stream(stream)), "orth_conv_apply")
    return y


def orth_exp_map_batched(ins, outs, terms, u, power_iters=1, status=None, workspace=None, stream=None):
    """What = exp(A / sigma), A = W - W^T, for every square ins[i] into
    outs[i] (see include/orth.h); u: packed float32 cached vectors (C per
    matrix), updated in place.  Returns the workspace tensor."""
    if not ins:
        return None
    mats = _mats(ins, outs)
    in_dt, out_dt = _dtype_code(ins[0]), _dtype_code(outs[0])
    for a, b in zip(ins, outs):
        if _dtype_code(a) != in_dt or _dtype_code(b) != out_dt:
            raise TypeError("all inputs (and all outputs) must share one dtype")
    need = sum(t.shape[0] for t in ins)
    if u.dtype != torch.float32 or not u.is_contiguous() or u.numel() < need:
        raise ValueError(f"u must be a contiguous float32 tensor of {need} values")
    opts = orth_exp_opts(terms, power_iters, u.data_ptr(), in_dt, out_dt)
    n = ctypes.c_size_t()
    _check(lib().orth_exp_map_workspace_size(mats, len(ins), ctypes.byref(opts), ctypes.byref(n)),
           "orth_exp_map_workspace_size")
    ws, nbytes = _workspace(n.value, ins[0].device, workspace)
    if status is not None and (status.dtype != torch.int32 or status.numel() < len(ins)):
        raise ValueError("status must be an int32 tensor with one slot per matrix")
    rc = lib().orth_exp_map_batched(mats, len(ins), ctypes.byref(opts), ws.data_ptr() if ws is not None else None,
                                    nbytes, status.data_ptr() if status is not None else None, _stream(stream))
    _check(rc, "orth_exp_map_batched")
    return ws


def orth_conv_exp_batched(layers, workspace=None, stream=None):
    """layers: dicts with kernel (c x c x k x k), out (c x c x S x S,
    S = terms (k - 1) + 1), terms and scale; contiguous, one dtype."""
    if not layers:
        return None
    dt = _dtype_code(layers[0]["kernel"])
    arr = (orth_conv_exp_desc * len(layers))()
    for i, L in enumerate(layers):
        kern, out = L["kernel"], L["out"]
        if not kern.is_contiguous() or not out.is_contiguous() or _dtype_code(kern) != dt or _dtype_code(out) != dt:
            raise ValueError("kernel and out must be contiguous and of one dtype")
        c, k = kern.shape[0], kern.shape[2]
        arr[i] = orth_conv_exp_desc(c, k, L["terms"], float(L.get("scale", 1.0)), kern.data_ptr(), out.data_ptr())
    n = ctypes.c_size_t()
    _check(lib().orth_conv_exp_workspace_size(arr, len(layers), dt, ctypes.byref(n)), "orth_conv_exp_workspace_size")
    ws, nbytes = _workspace(n.value, layers[0]["kernel"].device, workspace)
    rc = lib().orth_conv_exp_batched(arr, len(layers), dt, ws.data_ptr() if ws is not None else None, nbytes,
                                     _stream(stream))
    _check(rc, "orth_conv_exp_batched")
    return ws


# ---- rows grouped by matrix, the head's loss, gradient clipping -----------
# These run on the device that holds their tensors, whichever is current, and
# what they allocate belongs to the stream they run on.
def _on_device(call, stream, *tensors, workspace=None):
    """call(raw stream) with the tensors' device, and the stream if one is
    given, made current; every tensor must be on that device (None: not
    there), the workspace too."""
    index = tensors[0].get_device()
    if workspace is not None:
        if not workspace.is_contiguous():
            raise ValueError("workspace must be contiguous")
        tensors += (workspace,)
    for t in tensors:
        if t is not None and t.get_device() != index:
            raise ValueError("all tensors must be on one device")
    if index < 0:
        raise ValueError("tensors must be on the GPU")
    if stream is not None:
        if not hasattr(stream, "cuda_stream"):
            stream = torch.cuda.ExternalStream(stream, device=index)
        with torch.cuda.device(index), torch.cuda.stream(stream):
            return call(stream.cuda_stream)
    if torch.cuda.current_device() == index:
        return call(_raw_stream(index))
    with torch.cuda.device(index):
        return call(_raw_stream(index))


_MOST = 2 ** 31 - 1


def _extents(*sizes):
    """The library's sizes are 32 bits."""
    if max(sizes) > _MOST:
        raise ValueError("a size does not fit 32 bits")


def _raw_stream(index):
    # (torch.cuda.current_stream makes an object first: 2.5 us of a call)
    return torch._C._cuda_getCurrentRawStream(index)


def _rows_ld(t, what):
    """Leading dimension of a rows x columns tensor."""
    if t.dim() != 2 or (t.stride(1) != 1 and t.shape[1] > 1):
        raise ValueError(f"{what} must be 2-D with unit column stride")
    return t.stride(0) if t.shape[0] > 1 else max(t.stride(0), t.shape[1], 1)


def _stack_ld(w, what):
    """(groups, rows, cols, ld, group stride) of a matrix or a stack of them."""
    if w.dim() == 2:
        return 1, w.shape[0], w.shape[1], _rows_ld(w, what), 0
    if w.dim() != 3 or (w.stride(2) != 1 and w.shape[2] > 1):
        raise ValueError(f"{what} must be a matrix or a stack of matrices with unit column stride")
    g, r, c = w.shape
    ld = w.stride(1) if r > 1 else max(w.stride(1), c, 1)
    return g, r, c, ld, w.stride(0)


def _offsets_ptr(offsets, groups):
    if offsets is None:
        if groups != 1:
            raise ValueError("several matrices need offsets")
        return None
    if offsets.dtype != torch.int32 or not offsets.is_contiguous() or offsets.numel() != groups + 1:
        raise ValueError("offsets must be a contiguous int32 tensor of groups + 1 row numbers")
    return offsets.data_ptr()


def orth_linear_apply(x, w, offsets=None, transposed=False, out=None, stream=None):
    """y_r = W_g x_r (transposed: W_g^T x_r) for every row r of group g: x is
    rows x in_features, w a matrix or a stack of matrices (groups x
    out_features x in_features), offsets the groups + 1 row numbers on the
    GPU (int32; None with one matrix: every row).  Rows of no group keep what
    `out` holds (a new output: nothing defined).  Returns the output."""
    groups, n_out, n_in, ld_w, stride_w = _stack_ld(w, "w")
    cx, cy = (n_out, n_in) if transposed else (n_in, n_out)
    if x.dim() != 2 or x.shape[1] != cx:
        raise ValueError(f"x must be rows x {cx}")
    if out is not None and out.shape != (x.shape[0], cy):
        raise ValueError(f"out must be {x.shape[0]} x {cy}")
    if w.dtype != x.dtype or (out is not None and out.dtype != x.dtype):
        raise TypeError("x, w and out must share one dtype")
    dt = _dtype_code(x)
    _extents(x.shape[0], groups, n_in, n_out)

    def call(s):
        y = torch.empty(x.shape[0], cy, dtype=x.dtype, device=x.device) if out is None else out
        args = orth_linear_args(x.data_ptr(), w.data_ptr(), y.data_ptr(), _offsets_ptr(offsets, groups), x.shape[0],
                                groups, n_in, n_out, _rows_ld(x, "x"), ld_w, stride_w, _rows_ld(y, "out"), dt, dt,
                                1 if transposed else 0)
        _check(lib().orth_linear_apply(ctypes.byref(args), s), "orth_linear_apply")
        return y

    return _on_device(call, stream, x, w, out, offsets)


def orth_linear_grad_weight(grad_y, x, offsets=None, out=None, dtype=None, workspace=None, stream=None):
    """dL/dW_g = sum over group g's rows of grad_y_r x_r^T (zeros for a group
    without rows) into `out`, a matrix or a stack of them, float32 or
    bfloat16; without it into a new stack in `dtype` (default: that of x; one
    matrix, not a stack, if offsets is None).  Returns it."""
    if x.dim() != 2 or grad_y.dim() != 2 or x.shape[0] != grad_y.shape[0]:
        raise ValueError("grad_y and x must be 2-D with the same rows")
    if x.dtype != grad_y.dtype:
        raise TypeError("grad_y and x must share one dtype")
    n_out, n_in = grad_y.shape[1], x.shape[1]
    _extents(x.shape[0], n_in, n_out)

    def call(s):
        gw = out
        if gw is None:
            shape = (n_out, n_in) if offsets is None else (offsets.numel() - 1, n_out, n_in)
            gw = torch.empty(shape, dtype=dtype or x.dtype, device=x.device)
        g, r, c, ld_w, stride_w = _stack_ld(gw, "out")
        if (r, c) != (n_out, n_in):
            raise ValueError(f"out must hold {n_out} x {n_in} matrices")
        args = ctypes.byref(orth_linear_args(
            x.data_ptr(), gw.data_ptr(), grad_y.data_ptr(), _offsets_ptr(offsets, g), x.shape[0], g, n_in, n_out,
            _rows_ld(x, "x"), ld_w, stride_w, _rows_ld(grad_y, "grad_y"), _dtype_code(x), _dtype_code(gw), 0))
        n = ctypes.c_size_t()
        _check(lib().orth_linear_grad_weight_workspace_size(args, ctypes.byref(n)),
               "orth_linear_grad_weight_workspace_size")
        ws, nbytes = _workspace(n.value, x.device, workspace)
        _check(lib().orth_linear_grad_weight(args, ws.data_ptr() if ws is not None else None, nbytes, s),
               "orth_linear_grad_weight")
        return gw

    return _on_device(call, stream, x, grad_y, out, offsets, workspace=workspace)


def _xent_args(x, w, targets, scale, piece):
    if x.dim() != 2 or w.dim() != 2 or x.shape[1] != w.shape[1]:
        raise ValueError("x must be rows x features and w classes x features")
    if x.dtype != w.dtype:
        raise TypeError("x and w must share one dtype")
    if targets.dtype != torch.int64 or targets.shape != (x.shape[0],) or not targets.is_contiguous():
        raise ValueError("targets must be a contiguous int64 tensor of one class per row")
    _extents(*x.shape, w.shape[0])
    return orth_linear_xent_args(x.data_ptr(), w.data_ptr(), targets.data_ptr(), x.shape[0], x.shape[1], w.shape[0],
                                 _rows_ld(x, "x"), _rows_ld(w, "w"), scale, _dtype_code(x), piece)


def orth_linear_xent(x, w, targets, scale=1.0, workspace=None, stream=None):
    """(loss, lse) of the logits scale * x w^T, float32 per row: lse the log of
    the sum of their exponentials, loss = lse - the target's logit, 0 for a
    row whose target is no class."""
    args = ctypes.byref(_xent_args(x, w, targets, scale, 0))

    def call(s):
        loss = torch.empty(x.shape[0], dtype=torch.float32, device=x.device)
        lse = torch.empty_like(loss)
        n = ctypes.c_size_t()
        _check(lib().orth_linear_xent_workspace_size(args, ctypes.byref(n)), "orth_linear_xent_workspace_size")
        ws, nbytes = _workspace(n.value, x.device, workspace)
        _check(lib().orth_linear_xent(args, loss.data_ptr(), lse.data_ptr(), ws.data_ptr() if ws is not None else None,
                                      nbytes, s), "orth_linear_xent")
        return loss, lse

    return _on_device(call, stream, x, w, targets, workspace=workspace)


def orth_linear_xent_vjp(x, w, targets, lse, grad_loss, scale=1.0, grad_x=None, grad_w=None, want=(True, True),
                         piece=0, workspace=None, stream=None):
    """(grad_x, grad_w) given grad_loss = dL/d(loss of each row) (float32) and
    the lse that orth_linear_xent gave; want says which are computed (the
    other is None).  piece: classes per piece (0: chosen)."""
    args = ctypes.byref(_xent_args(x, w, targets, scale, piece))
    for t, what in ((lse, "lse"), (grad_loss, "grad_loss")):
        if t.dtype != torch.float32 or t.shape != (x.shape[0],) or not t.is_contiguous():
            raise ValueError(f"{what} must be a contiguous float32 tensor of one value per row")
    given = (grad_x if want[0] else None, grad_w if want[1] else None)

    def call(s):
        grads, place = [], []
        for t, like, wanted, what in ((given[0], x, want[0], "grad_x"), (given[1], w, want[1], "grad_w")):
            if wanted and t is None:
                t = torch.empty(like.shape, dtype=like.dtype, device=like.device)
            if t is not None and (t.shape != like.shape or t.dtype != like.dtype):
                raise ValueError(f"{what} must have the shape and dtype of what it is the gradient of")
            grads.append(t)
            place += [t.data_ptr(), _rows_ld(t, what)] if t is not None else [None, 0]
        n = ctypes.c_size_t()
        _check(lib().orth_linear_xent_vjp_workspace_size(args, ctypes.byref(n)), "orth_linear_xent_vjp_workspace_size")
        ws, nbytes = _workspace(n.value, x.device, workspace)
        _check(lib().orth_linear_xent_vjp(args, lse.data_ptr(), grad_loss.data_ptr(), *place,
                                          ws.data_ptr() if ws is not None else None, nbytes, s),
               "orth_linear_xent_vjp")
        return tuple(grads)

    return _on_device(call, stream, x, w, targets, lse, grad_loss, *given, workspace=workspace)


class orth_grad_list:
    """Descriptors of a list of gradients (and of the tensors that take the
    clipped ones; default: in place), for orth_grad_norm_batched and
    orth_grad_clip_batched.  Tensors of up to two dimensions with unit column
    stride, or contiguous ones of any; float32 and bfloat16 may be mixed.  A
    program that keeps its gradients' buffers keeps this list with them: its
    descriptors are made once (8 us a tensor).  The list holds the tensors'
    memory, and every call looks whether each tensor is still where it was (50
    ns each) and makes the descriptors again where one is not, its .data
    replaced or resized past its storage.  A tensor that changes its shape where
    it is needs refresh()."""

    def __init__(self, grads, outs=None):
        outs = grads if outs is None else outs
        if len(grads) != len(outs):
            raise ValueError("grads and outs must have the same length")
        if not grads:
            raise ValueError("the list must hold at least one tensor")
        self.tensors = (list(grads), list(outs))
        self._every = [*grads, *(o for g, o in zip(grads, outs) if o is not g)]
        self.refresh()

    def _current(self):
        if list(map(torch.Tensor.data_ptr, self._every)) != self._at:
            self.refresh()
        return self

    def refresh(self):
        """Makes the descriptors again from the tensors as they are now."""
        grads, outs = self.tensors
        self._at = None   # (nothing is taken for read if this raises)
        self.device = grads[0].device
        if any(t.device != self.device for t in (*grads, *outs)) or self.device.type != "cuda":
            raise ValueError("all tensors must be on one GPU")
        # (what the descriptors point to stays allocated while they do)
        self._memory = list(map(torch.Tensor.untyped_storage, self._every))
        descs = []
        for g, o in zip(grads, outs):
            if g.shape != o.shape or g.dtype != o.dtype:
                raise ValueError("a gradient and its output must have one shape and dtype")
            for g2, o2 in self._matrices(g, o):
                _extents(*g2.shape)
                descs.append(orth_grad(g2.data_ptr(), o2.data_ptr(), g2.shape[0], g2.shape[1],
                                       _rows_ld(g2, "gradients"), _rows_ld(o2, "outputs"), _dtype_code(g)))
        self.array = (orth_grad * len(descs))(*descs)
        n = ctypes.c_size_t()
        _check(lib().orth_grad_norm_workspace_size(self.array, len(descs), ctypes.byref(n)),
               "orth_grad_norm_workspace_size")
        self.workspace_bytes = n.value
        self._at = list(map(torch.Tensor.data_ptr, self._every))

    @staticmethod
    def _matrices(g, o):
        """The pair as matrices: contiguous ones as rows of up to 2^30 values."""
        if g.is_contiguous() and o.is_contiguous():
            most = 1 << 30
            g, o = g.view(-1), o.view(-1)
            return [(g[i:i + most].view(1, -1), o[i:i + most].view(1, -1)) for i in range(0, max(g.numel(), 1), most)]
        if g.dim() > 2:
            raise ValueError("gradients of more than two dimensions must be contiguous")
        for t in (g, o):   # (a view, as above, says so by itself)
            last = t.storage_offset() + sum((n - 1) * k for n, k in zip(t.shape, t.stride()))
            if t.numel() and (last + 1) * t.element_size() > t.untyped_storage().nbytes():
                raise RuntimeError("a gradient's storage does not hold it")
        return [(g, o) if g.dim() == 2 else (g.unsqueeze(1), o.unsqueeze(1))]


def _as_list(grads):
    return grads._current() if isinstance(grads, orth_grad_list) else orth_grad_list(grads)


def _norm_call(fn, where, lst, norm, workspace, stream, *opts):
    if norm is not None and (norm.dtype != torch.float32 or norm.numel() != 1):
        raise ValueError("norm must be a float32 tensor of one value")

    def call(s):
        n = torch.empty(1, dtype=torch.float32, device=lst.device) if norm is None else norm
        ws, nbytes = _workspace(lst.workspace_bytes, lst.device, workspace)
        _check(fn(lst.array, len(lst.array), *opts, n.data_ptr(), ws.data_ptr(), nbytes, s), where)
        return n

    return _on_device(call, stream, lst.tensors[0][0], norm, workspace=workspace)


def orth_grad_norm_batched(grads, norm=None, workspace=None, stream=None):
    """The norm of all gradients together, as a float32 tensor of one value.
    grads: tensors or an orth_grad_list."""
    return _norm_call(lib().orth_grad_norm_batched, "orth_grad_norm_batched", _as_list(grads), norm, workspace, stream)


def orth_grad_clip_batched(grads, max_norm, eps=1e-6, norm=None, norm_given=False, workspace=None, stream=None):
    """Every gradient times min(1, max_norm / (norm + eps)), norm the norm of
    them all together (norm_given: the value that `norm` holds).  grads:
    tensors, clipped in place, or an orth_grad_list.  Returns the norm."""
    if norm_given and norm is None:
        raise ValueError("norm_given needs norm")
    opts = orth_clip_opts(max_norm, eps, 1 if norm_given else 0)
    return _norm_call(lib().orth_grad_clip_batched, "orth_grad_clip_batched", _as_list(grads), norm, workspace, stream,
                      ctypes.byref(opts))


def _check_call(args, out, workspace, stream):
    n = ctypes.c_size_t()
    _check(lib().orth_check_workspace_size(ctypes.byref(args), ctypes.byref(n)), "orth_check_workspace_size")
    ws, nbytes = _workspace(n.value, out.device, workspace)
    rc = lib().orth_check_norm(ctypes.byref(args), out.data_ptr(), ws.data_ptr() if ws is not None else None,
                               nbytes, _stream(stream))
    _check(rc, "orth_check_norm")


def orth_check_norm_gram(mats, workspace=None, stream=None):
    """max |G - I| per matrix (G the smaller Gram matrix), as a float32 tensor."""
    arr = _mats(mats, mats)
    out = torch.empty(len(mats), dtype=torch.float32, device=mats[0].device)
    args = orth_check_args()
    args.mode = ORTH_CHECK_GRAM
    args.mats = ctypes.cast(arr, ctypes.POINTER(orth_mat))
    args.n_mats = len(mats)
    args.mat_dtype = _dtype_code(mats[0])
    _check_call(args, out, workspace, stream)
    return out


def orth_check_norm_conv(kernel, geom, x, adjoint=False, workspace=None, stream=None):
    """||conv_circ(K, x_b)|| / ||x_b|| per sample (or the adjoint's ratio)."""
    if x.dtype != torch.float32 or not x.is_contiguous() or not kernel.is_contiguous():
        raise ValueError("x must be contiguous float32 and the kernel contiguous")
    out = torch.empty(x.shape[0], dtype=torch.float32, device=x.device)
    args = orth_check_args()
    args.mode = ORTH_CHECK_CONV_ADJOINT if adjoint else ORTH_CHECK_CONV
    args.kernel = kernel.data_ptr()
    args.kernel_dtype = _dtype_code(kernel)
    args.geom = orth_conv_geom(*geom)
    args.x = x.data_ptr()
    args.batch, args.height, args.width = x.shape[0], x.shape[2], x.shape[3]
    _check_call(args, out, workspace, stream)
    return out


def orth_timing_enable(on=True):
    _check(lib().orth_timing_enable(1 if on else 0), "orth_timing_enable")


def orth_timing_filter(*prefixes):
    """Time only launches whose kernel names start with one of the prefixes
    (none: every launch)."""
    _check(lib().orth_timing_filter(";".join(prefixes).encode()), "orth_timing_filter")


def orth_timing_reset():
    _check(lib().orth_timing_reset(), "orth_timing_reset")


def orth_timing_read(name):
    ms, n = ctypes.c_double(), ctypes.c_int64()
    _check(lib().orth_timing_read(name.encode(), ctypes.byref(ms), ctypes.byref(n)), "orth_timing_read")
    return ms.value, n.value


def orth_timing_span(*prefixes):
    """Wall-clock ms covered by the launches whose names start with any of
    the prefixes (overlapping launches count once), and their number."""
    ms, n = ctypes.c_double(), ctypes.c_int64()
    _check(lib().orth_timing_span(";".join(prefixes).encode(), ctypes.byref(ms), ctypes.byref(n)),
           "orth_timing_span")
    return ms.value, n.value


def orth_timing_names():
    buf = ctypes.create_string_buffer(4096)
    _check(lib().orth_timing_names(buf, 4096), "orth_timing_names")
    return [s for s in buf.value.decode().split(";") if s]
