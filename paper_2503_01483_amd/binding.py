"""ctypes binding of libkurtail.so; same names as the C entry points."""
import ctypes
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libkurtail.so")
_lib = None

KT_F32, KT_BF16 = 0, 1
KT_OP_LOSS_GRAD, KT_OP_CAYLEY, KT_OP_FAKEQUANT, KT_OP_POOLED_LOSS_GRAD, KT_OP_QUANT_METRICS = 0, 1, 2, 3, 4
KT_OP_FUSE_ROTATION, KT_OP_SENSITIVITY, KT_OP_LOSS_GRAD_RECOMPUTE, KT_OP_POOLED_LOSS_GRAD_RECOMPUTE = 5, 6, 7, 8
KT_Q_NONE, KT_Q_INT4, KT_Q_INT8, KT_Q_E4M3 = 0, 1, 2, 3
KT_KV_BF16, KT_KV_U8, KT_KV_U4 = 0, 1, 2

EXPORTS = ("kt_version", "kt_last_error", "kt_workspace_bytes", "kt_kurtosis_loss_grad",
           "kt_pooled_kurtosis_loss_grad", "kt_cayley_step", "kt_cayley_adam_step", "kt_rotate_fakequant_int4", "kt_rotate_quant_metrics", "kt_hadamard_rows", "kt_fuse_rotation", "kt_quant_sensitivity", "kt_profile_enable", "kt_profile_read",
           "kt_profile_reset", "kt_cayley_step_static", "kt_build_id", "kt_add_rmsnorm_quant", "kt_kv_cache_bytes", "kt_kv_append",
           "kt_kv_gather", "kt_paged_attention", "kt_paged_attention_bytes", "kt_tree_attention", "kt_attention_mass", "kt_kv_select",
           "kt_kv_compact")


class _CacheDesc(ctypes.Structure):
    """kt_kv_cache"""
    _fields_ = [("data", ctypes.c_void_p), ("n_pages", ctypes.c_int64), ("page_size", ctypes.c_int64),
                ("n_heads", ctypes.c_int64), ("head_dim", ctypes.c_int64), ("format", ctypes.c_int32)]


class KtError(RuntimeError):
    def __init__(self, status, text):
        super().__init__(f"kt status {status}: {text}")
        self.status = status


def lib_path():
    return _LIB_PATH


def lib():
    """Load the library.  It is built first when no built library is present, and rebuilt when the one present
    was compiled from other sources than those in csrc/ now (it carries an id of its sources): a stale library
    is never loaded silently."""
    global _lib
    if _lib is not None:
        return _lib
    from .build import build_library, source_id
    if not os.path.exists(_LIB_PATH):
        build_library()
    L = ctypes.CDLL(_LIB_PATH)
    want = source_id()
    try:
        L.kt_build_id.restype = ctypes.c_char_p
        have = L.kt_build_id().decode()
    except AttributeError:
        have = "(none)"
    if have != want:
        import warnings
        warnings.warn(f"libkurtail.so was built from other sources (id {have}, csrc/ now {want}): rebuilding")
        tmp = _LIB_PATH + ".stale"
        os.replace(_LIB_PATH, tmp)     # the mapped file stays valid; the new one gets a fresh inode
        build_library()
        os.remove(tmp)
        L = ctypes.CDLL(_LIB_PATH)
        L.kt_build_id.restype = ctypes.c_char_p
        if L.kt_build_id().decode() != want:
            raise RuntimeError("libkurtail.so does not match its sources after a rebuild")
    vp, i64, f32, sz = ctypes.c_void_p, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t
    i32 = ctypes.c_int32
    L.kt_version.restype = i32
    L.kt_version.argtypes = []
    L.kt_last_error.restype = ctypes.c_char_p
    L.kt_last_error.argtypes = []
    L.kt_workspace_bytes.restype = sz
    L.kt_workspace_bytes.argtypes = [i32, i64, i64, i64, i32]
    L.kt_kurtosis_loss_grad.restype = i32
    L.kt_kurtosis_loss_grad.argtypes = [vp, i64, vp, i64, i64, i64, i64, i32, i32, f32,
                                        vp, vp, vp, vp, sz, vp]
    L.kt_pooled_kurtosis_loss_grad.restype = i32
    L.kt_pooled_kurtosis_loss_grad.argtypes = [vp, i64, vp, i64, i64, i64, i64, i32, i32, f32, f32, vp, vp, vp,
                                               vp, sz, vp]
    L.kt_rotate_quant_metrics.restype = i32
    L.kt_rotate_quant_metrics.argtypes = [vp, i64, vp, i64, i64, i64, i64, i32, i32, f32, vp, vp, vp, vp, vp, vp,
                                          vp, sz, vp]
    L.kt_hadamard_rows.restype = i32
    L.kt_hadamard_rows.argtypes = [vp, i64, vp, i64, vp, i64, i64, i32, vp]
    L.kt_fuse_rotation.restype = i32
    L.kt_fuse_rotation.argtypes = [vp, i64, vp, i64, vp, i64, i64, i64, i32, vp, sz, vp]
    L.kt_quant_sensitivity.restype = i32
    L.kt_quant_sensitivity.argtypes = [vp, i64, i32, vp, i32, vp, vp, vp, sz, vp]
    L.kt_cayley_step.restype = i32
    L.kt_cayley_step.argtypes = [vp, vp, vp, i64, i64, f32, vp, vp, vp, sz, vp]
    L.kt_cayley_step_static.restype = i32
    L.kt_cayley_step_static.argtypes = [vp, vp, vp, i64, i64, f32, vp, vp, vp]
    L.kt_cayley_adam_step.restype = i32
    L.kt_cayley_adam_step.argtypes = [vp, vp, vp, vp, i64, vp, i64, i64, f32, f32, f32, f32, f32, vp, vp, vp,
                                      vp, sz, vp]
    L.kt_rotate_fakequant_int4.restype = i32
    L.kt_rotate_fakequant_int4.argtypes = [vp, i64, vp, i64, i64, i64, i64, i32, i32, f32,
                                           vp, vp, vp, vp, vp, sz, vp]
    cache = ctypes.POINTER(_CacheDesc)
    L.kt_add_rmsnorm_quant.restype = i32
    L.kt_add_rmsnorm_quant.argtypes = [vp, i64, vp, i64, vp, i64, i64, i32, i32, f32, f32, i32, vp, i64, vp, i64, vp, i64, vp, vp]
    L.kt_kv_cache_bytes.restype = sz
    L.kt_kv_cache_bytes.argtypes = [cache]
    L.kt_kv_append.restype = i32
    L.kt_kv_append.argtypes = [cache, vp, i64, vp, i64, vp, i64, i64, i64, i32, vp, vp, vp, i64, i64, i32, i32, vp, i64, vp]
    L.kt_kv_gather.restype = i32
    L.kt_kv_gather.argtypes = [cache, vp, i64, vp, i64, vp, i64, i32, vp]
    L.kt_paged_attention_bytes.restype = sz
    L.kt_paged_attention_bytes.argtypes = [i64, i64, i64, i64]
    L.kt_paged_attention.restype = i32
    L.kt_paged_attention.argtypes = [cache, vp, i64, i32, vp, vp, vp, i64, i64, i64, i64, i64, vp, i64, f32, vp, i64, vp, vp, sz, vp]
    L.kt_profile_enable.restype = i32
    L.kt_tree_attention.argtypes = [cache, vp, i64, i32, vp, vp, vp, i64, i64, i64, i64, i64, vp, i64, vp, i64, f32, vp, i64, vp, vp, sz, vp]
    L.kt_tree_attention.restype = i32
    L.kt_attention_mass.argtypes = [cache, vp, i64, i32, vp, vp, vp, i64, i64, i64, i64, i64, f32, vp, f32, vp, vp]
    L.kt_attention_mass.restype = i32
    L.kt_kv_select.argtypes = [cache, vp, vp, vp, i64, i64, vp, i64, i64, vp, i64, vp, vp]
    L.kt_kv_select.restype = i32
    L.kt_kv_compact.argtypes = [cache, vp, i64, i64, vp, i64, i32, vp, vp, vp, i64, vp, vp]
    L.kt_kv_compact.restype = i32
    L.kt_profile_enable.argtypes = [i32]
    L.kt_profile_read.restype = i32
    L.kt_profile_read.argtypes = [i32, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(i32)]
    L.kt_profile_reset.restype = i32
    L.kt_profile_reset.argtypes = []
    _lib = L
    return L


def kt_version():
    return int(lib().kt_version())


def kt_last_error():
    return lib().kt_last_error().decode()


def kt_workspace_bytes(op, batch, n, d, x_dtype):
    return int(lib().kt_workspace_bytes(op, batch, n, d, x_dtype))


def _ptr(t):
    return None if t is None else t.data_ptr()


def _dtype_code(t):
    if t.dtype == torch.bfloat16:
        return KT_BF16
    if t.dtype == torch.float32:
        return KT_F32
    raise TypeError(f"unsupported dtype {t.dtype}")


def _stream(stream, dev=None):
    """Handle of a stream (a stream, a handle, or None: the current one), of device `dev` where the current device is known."""
    if stream is None:
        # torch.cuda.current_stream().cuda_stream without the stream object (of a call of 8 us it took 1.5)
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device() if dev is None else dev)
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else stream


def _check(status):
    if status != 0:
        raise KtError(status, kt_last_error())


def _new(make, stream, *args, **kwargs):
    """What a call makes for a kernel on `stream` (a stream, its handle, or None: the current one), made on that stream: it is filled in front
    of the kernel, and its memory, once freed, is given to nobody who does not wait for the kernel."""
    if stream is None:
        return make(*args, **kwargs)
    with torch.cuda.stream(stream if hasattr(stream, "cuda_stream") else torch.cuda.ExternalStream(stream)):
        return make(*args, **kwargs)


class Workspace:
    """A caller-owned scratch buffer (torch uint8 tensor) that grows on demand."""

    def __init__(self, device="cuda"):
        self.device = device
        self.buf = None

    def get(self, nbytes):
        if self.buf is None or self.buf.numel() < nbytes:
            self.buf = None
            self.buf = torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=self.device)
        return self.buf


def _xr_dims(X, R):
    if X.dim() == 2:
        X = X.unsqueeze(0)
    if R.dim() == 2:
        R = R.unsqueeze(0)
    batch, n, d = X.shape
    assert R.shape == (batch, d, d), (X.shape, R.shape)
    assert X.stride(2) == 1 and R.stride(2) == 1
    assert batch == 1 or (X.stride(0) == n * X.stride(1) and R.stride(0) == d * R.stride(1))
    return X, R, batch, n, d


def kt_kurtosis_loss_grad(X, R, *, kappa_target=0.0, loss=None, row_kurt=None, dR=None,
                          workspace=None, stream=None, recompute=False):
    """loss [batch] fp32 (returned), optional row_kurt [batch][n] and dR [batch][d][d] outputs.
    recompute=True hands the library only the smaller workspace, with which it recomputes Y for the
    backward pass instead of keeping it (same result)."""
    X, R, batch, n, d = _xr_dims(X, R)
    if loss is None:
        loss = _new(torch.empty, stream, batch, dtype=torch.float32, device=X.device)
    xdt = _dtype_code(X)
    need = kt_workspace_bytes(KT_OP_LOSS_GRAD_RECOMPUTE if recompute else KT_OP_LOSS_GRAD, batch, n, d, xdt)
    ws = _new((workspace or Workspace(X.device)).get, stream, need)
    _check(lib().kt_kurtosis_loss_grad(_ptr(X), X.stride(1), _ptr(R), R.stride(1), batch, n, d, xdt,
                                       _dtype_code(R), float(kappa_target), _ptr(loss),
                                       _ptr(row_kurt), _ptr(dR), _ptr(ws), need if recompute else ws.numel(),
                                       _stream(stream)))
    return loss


def kt_pooled_kurtosis_loss_grad(X, R, *, kappa_target=1.8, rms_eps=0.0, loss=None, kappa=None, dR=None,
                                 workspace=None, stream=None, recompute=False):
    """Paper-literal pooled loss [batch] fp32 (returned), optional kappa [batch] and dR outputs.
    recompute: as for kt_kurtosis_loss_grad."""
    X, R, batch, n, d = _xr_dims(X, R)
    if loss is None:
        loss = _new(torch.empty, stream, batch, dtype=torch.float32, device=X.device)
    xdt = _dtype_code(X)
    need = kt_workspace_bytes(KT_OP_POOLED_LOSS_GRAD_RECOMPUTE if recompute else KT_OP_POOLED_LOSS_GRAD,
                              batch, n, d, xdt)
    ws = _new((workspace or Workspace(X.device)).get, stream, need)
    _check(lib().kt_pooled_kurtosis_loss_grad(_ptr(X), X.stride(1), _ptr(R), R.stride(1), batch, n, d, xdt,
                                              _dtype_code(R), float(kappa_target), float(rms_eps), _ptr(loss),
                                              _ptr(kappa), _ptr(dR), _ptr(ws), need if recompute else ws.numel(),
                                              _stream(stream)))
    return loss


def kt_cayley_step(R, dR, lr, *, R_lowp=None, ortho_err=None, info=None, workspace=None, stream=None):
    """In-place Cayley step on R [batch][d][d] fp32."""
    Rv = R if R.dim() == 3 else R.unsqueeze(0)
    batch, d, _ = Rv.shape
    assert Rv.is_contiguous() and dR.is_contiguous() and dR.numel() == Rv.numel()
    assert R.dtype == torch.float32 and dR.dtype == torch.float32
    need = kt_workspace_bytes(KT_OP_CAYLEY, batch, 0, d, KT_F32)
    ws = _new((workspace or Workspace(R.device)).get, stream, need)
    _check(lib().kt_cayley_step(_ptr(Rv), _ptr(dR), _ptr(R_lowp), batch, d, float(lr), _ptr(ortho_err),
                                _ptr(info), _ptr(ws), ws.numel(), _stream(stream)))
    return R


def kt_cayley_step_static(R, dR, lr, *, R_lowp=None, ortho_err=None, info=None, stream=None):
    """kt_cayley_step on the library's own static device scratch: no workspace, no allocation (small sizes)."""
    Rv = R if R.dim() == 3 else R.unsqueeze(0)
    batch, d, _ = Rv.shape
    assert Rv.is_contiguous() and dR.is_contiguous() and dR.numel() == Rv.numel()
    assert R.dtype == torch.float32 and dR.dtype == torch.float32
    _check(lib().kt_cayley_step_static(_ptr(Rv), _ptr(dR), _ptr(R_lowp), batch, d, float(lr), _ptr(ortho_err),
                                       _ptr(info), _stream(stream)))
    return R


def kt_cayley_adam_step(R, dR, M, v, step, lr, *, beta1=0.9, beta2=0.99, eps=1e-8, q=0.5, R_lowp=None,
                        ortho_err=None, info=None, scalars=None, workspace=None, stream=None):
    """In-place Cayley Adam step on R [batch][d][d] fp32 with state M [batch][d][d], v [batch]."""
    Rv = R if R.dim() == 3 else R.unsqueeze(0)
    batch, d, _ = Rv.shape
    assert Rv.is_contiguous() and dR.is_contiguous() and M.is_contiguous() and v.is_contiguous()
    assert dR.numel() == Rv.numel() and M.numel() == Rv.numel() and v.numel() == batch
    assert R.dtype == dR.dtype == M.dtype == v.dtype == torch.float32
    need = kt_workspace_bytes(KT_OP_CAYLEY, batch, 0, d, KT_F32)
    ws = _new((workspace or Workspace(R.device)).get, stream, need)
    _check(lib().kt_cayley_adam_step(_ptr(Rv), _ptr(dR), _ptr(M), _ptr(v), int(step), _ptr(R_lowp), batch, d,
                                     float(lr), float(beta1), float(beta2), float(eps), float(q),
                                     _ptr(ortho_err), _ptr(info), _ptr(scalars), _ptr(ws), ws.numel(),
                                     _stream(stream)))
    return R


def kt_rotate_fakequant_int4(X, R, *, clip_ratio=1.0, scales_in=None, scales_out=None, codes=None,
                             err=None, workspace=None, stream=None):
    X, R, batch, n, d = _xr_dims(X, R)
    xdt = _dtype_code(X)
    need = kt_workspace_bytes(KT_OP_FAKEQUANT, batch, n, d, xdt)
    ws = _new((workspace or Workspace(X.device)).get, stream, need)
    _check(lib().kt_rotate_fakequant_int4(_ptr(X), X.stride(1), _ptr(R), R.stride(1), batch, n, d, xdt,
                                          _dtype_code(R), float(clip_ratio), _ptr(scales_in),
                                          _ptr(scales_out), _ptr(codes), _ptr(err), _ptr(ws),
                                          ws.numel(), _stream(stream)))


def kt_rotate_quant_metrics(X, R, *, quantile=0.98, Y=None, amax=None, threshold=None, err_sym=None,
                            err_asym=None, success=None, workspace=None, stream=None):
    X, R, batch, n, d = _xr_dims(X, R)
    xdt = _dtype_code(X)
    need = kt_workspace_bytes(KT_OP_QUANT_METRICS, batch, n, d, xdt)
    ws = _new((workspace or Workspace(X.device)).get, stream, need)
    _check(lib().kt_rotate_quant_metrics(_ptr(X), X.stride(1), _ptr(R), R.stride(1), batch, n, d, xdt,
                                         _dtype_code(R), float(quantile), _ptr(Y), _ptr(amax), _ptr(threshold),
                                         _ptr(err_sym), _ptr(err_asym), _ptr(success), _ptr(ws), ws.numel(),
                                         _stream(stream)))


def kt_hadamard_rows(X, *, signs=None, out=None, stream=None):
    """Y = (X * signs) H_d / sqrt(d) on the rows of X [n][d] (fp32 or bf16); returns Y (out or new)."""
    assert X.dim() == 2 and X.stride(1) == 1
    n, d = X.shape
    Y = _new(torch.empty_like, stream, X) if out is None else out
    assert Y.shape == X.shape and Y.dtype == X.dtype and Y.stride(1) == 1
    if signs is not None:
        assert signs.dtype == torch.int8 and signs.numel() == d and signs.is_contiguous()
    _check(lib().kt_hadamard_rows(_ptr(X), X.stride(0), _ptr(Y), Y.stride(0), _ptr(signs), n, d, _dtype_code(X),
                                  _stream(stream)))
    return Y


def kt_fuse_rotation(W, R, side, *, out=None, workspace=None, stream=None):
    """side 0: W [k][d] -> W R;  side 1: W [d][k] -> R^T W  (fp32)."""
    d = R.shape[-1]
    k = W.shape[0] if side == 0 else W.shape[1]
    assert W.dtype == R.dtype == torch.float32 and W.stride(1) == 1 and R.stride(-1) == 1 and R.dim() == 2
    out = _new(torch.empty_like, stream, W) if out is None else out
    need = kt_workspace_bytes(KT_OP_FUSE_ROTATION, 1, k, d, KT_F32)
    ws = _new((workspace or Workspace(W.device)).get, stream, need)
    _check(lib().kt_fuse_rotation(_ptr(W), W.stride(0), _ptr(R), R.stride(0), _ptr(out), out.stride(0), k, d,
                                  int(side), _ptr(ws), ws.numel(), _stream(stream)))
    return out


def kt_quant_sensitivity(Y, alphas, *, bits=4, workspace=None, stream=None):
    """Returns (out [2] = {s_opt, MSE(s_opt)}, gamma [len(alphas)]) as device tensors."""
    assert Y.dtype == torch.float32 and Y.is_contiguous() and alphas.dtype == torch.float32
    out = _new(torch.empty, stream, 2, dtype=torch.float32, device=Y.device)
    gamma = _new(torch.empty, stream, alphas.numel(), dtype=torch.float32, device=Y.device)
    need = kt_workspace_bytes(KT_OP_SENSITIVITY, 1, 1, 128, KT_F32)
    ws = _new((workspace or Workspace(Y.device)).get, stream, need)
    _check(lib().kt_quant_sensitivity(_ptr(Y), Y.numel(), int(bits), _ptr(alphas), alphas.numel(), _ptr(out),
                                      _ptr(gamma), _ptr(ws), ws.numel(), _stream(stream)))
    return out, gamma


def _device(t, name):
    """The current device, which `t` has to be on (a kernel is launched there)."""
    dev = t.get_device()
    if dev < 0 or dev != torch._C._cuda_getDevice():     # (torch.cuda.current_device(), which first asks whether there is a device: a tensor is on one)
        raise ValueError(f"{name} is on {t.device}: operands have to be on the current device")
    return dev


def _refuse(name, t, dev, dtype, what):
    raise ValueError(f"{name}: {dtype} {what} on cuda:{dev} needed, got {t.dtype} {tuple(t.shape)}, strides {t.stride()}, on {t.device}")


def _index(t, name, dev, dtype, shape):
    """Address of a contiguous tensor of that type and shape."""
    if t.get_device() != dev or t.dtype is not dtype or t.shape != shape or not t.is_contiguous():
        _refuse(name, t, dev, dtype, f"of shape {tuple(shape)}, contiguous,")
    return t.data_ptr()


def _rows(t, name, dev, dtype, shape):
    """Leading dimension of a tensor of shape [n, width] with contiguous rows."""
    if t.get_device() != dev or t.dtype is not dtype or t.shape != shape:
        _refuse(name, t, dev, dtype, f"of shape {tuple(shape)}")
    ld, one = t.stride()
    n, width = shape
    if (one != 1 and width > 1) or (ld < width and n > 1):
        _refuse(name, t, dev, dtype, "with contiguous rows")
    return ld if ld > width else width


def _heads(t, name, dev, dtype, n, heads, head_dim):
    """Leading dimension of [n, heads, head_dim] (or [n, heads * head_dim]) rows with their heads next to each other."""
    if t.dim() != 3:
        return _rows(t, name, dev, dtype, (n, heads * head_dim))
    if t.get_device() != dev or t.dtype is not dtype or t.shape != (n, heads, head_dim):
        _refuse(name, t, dev, dtype, f"of shape {(n, heads, head_dim)}")
    ld, of_head, one = t.stride()
    width = heads * head_dim
    if one != 1 or (of_head != head_dim and heads > 1) or (ld < width and n > 1):
        _refuse(name, t, dev, dtype, "with contiguous rows of heads")
    return ld if ld > width else width


_CODE_TYPES = {KT_Q_INT4: (torch.int8,), KT_Q_INT8: (torch.int8,), KT_Q_E4M3: (torch.float8_e4m3fn, torch.uint8)}


def kt_add_rmsnorm_quant(X, *, res=None, gain=None, eps=1e-6, clip_ratio=1.0, format=KT_Q_INT8, res_out=None, Y=None,
                         codes=None, scales=None, stream=None):
    """Norm of the rows of X (+ res) [n][d] and their codes.  Writes the outputs that are given; returns (codes, scales)."""
    dev, dtype, shape = _device(X, "X"), X.dtype, X.shape
    if len(shape) != 2:
        raise ValueError(f"X: [n, d] needed, got {tuple(shape)}")
    n, d = shape
    xdt = gdt = _dtype_code(X)
    ldx = _rows(X, "X", dev, dtype, shape)
    ldres = ldro = ldy = ldc = 0
    pres = pgain = pro = py = pc = ps = None
    if res is not None:
        ldres, pres = _rows(res, "res", dev, dtype, shape), res.data_ptr()
    if gain is not None:
        gdt, pgain = _dtype_code(gain), _index(gain, "gain", dev, gain.dtype, (d,))
    if res_out is not None:
        ldro, pro = _rows(res_out, "res_out", dev, dtype, shape), res_out.data_ptr()
    if Y is not None:
        ldy, py = _rows(Y, "Y", dev, dtype, shape), Y.data_ptr()
    if codes is not None:
        if codes.dtype not in _CODE_TYPES.get(format, ()):
            raise TypeError(f"codes of type {codes.dtype} do not fit format {format}")
        ldc, pc = _rows(codes, "codes", dev, codes.dtype, shape), codes.data_ptr()
    if scales is not None:
        ps = _index(scales, "scales", dev, torch.float32, (n,))
    _check(lib().kt_add_rmsnorm_quant(X.data_ptr(), ldx, pres, ldres, pgain, n, d, xdt, gdt, eps, clip_ratio, format, pro, ldro, py, ldy,
                                      pc, ldc, ps, _stream(stream)))
    return codes, scales


class KVCache:
    """A paged key / value cache: its shape, which does not change, and `data`, a uint8 tensor of as many bytes (allocated here unless
    given; another one can be put in its place)."""

    def __init__(self, n_pages, page_size, n_heads, head_dim, format, *, data=None, device="cuda"):
        self.desc = _CacheDesc(None, n_pages, page_size, n_heads, head_dim, format)
        self.ref = ctypes.byref(self.desc)
        self.nbytes = lib().kt_kv_cache_bytes(self.ref)
        if self.nbytes == 0:
            raise KtError(2, kt_last_error() or "bad cache sizes")
        self._mass_shape = (self.n_pages, self.n_heads, self.page_size)
        self.data = torch.empty(self.nbytes, dtype=torch.uint8, device=device) if data is None else data

    # the sizes that a call checks its operands against are those that the kernels go by
    n_pages, page_size, n_heads, head_dim, format = (property(lambda self, name=name: getattr(self.desc, name))
                                                     for name in ("n_pages", "page_size", "n_heads", "head_dim", "format"))

    @property
    def data(self):
        return self._data

    @data.setter
    def data(self, data):
        if data.dtype != torch.uint8 or not data.is_contiguous() or data.numel() != self.nbytes:
            raise ValueError(f"data: {self.nbytes} contiguous bytes (uint8) needed, got {data.dtype} {tuple(data.shape)}")
        self._data = data

    def _on(self, dev):
        """The descriptor for a call on device `dev`, with the address that the data has now."""
        data = self._data
        if data.get_device() != dev or data.numel() != self.nbytes or not data.is_contiguous():
            _refuse("cache", data, dev, torch.uint8, f"of {self.nbytes} bytes, contiguous,")
        self.desc.data = data.data_ptr()
        return self.ref


def kt_kv_append(cache, K, V, slots, *, Q=None, positions=None, rope=None, interleaved=False, hadamard=False, Q_out=None,
                 stream=None):
    """Rotated, quantised K and V [n][heads][head_dim] into `slots` [n] of the cache; returns the rotated queries (Q_out, or new ones, 0 for
    tokens that are passed over)."""
    dev, dtype, n = _device(K, "K"), K.dtype, K.shape[0]
    dt, hd, heads, ref = _dtype_code(K), cache.head_dim, cache.n_heads, cache._on(dev)
    ldk, ldv = _heads(K, "K", dev, dtype, n, heads, hd), _heads(V, "V", dev, dtype, n, heads, hd)
    pslots = _index(slots, "slots", dev, torch.int64, (n,))
    hq = ldq = ldqo = n_pos = rot = 0
    pq = pqo = ppos = prope = None
    if Q is not None:
        if Q_out is None:
            Q_out = _new(torch.zeros, stream, Q.shape, dtype=Q.dtype, device=Q.device)     # (rows of tokens that are passed over are not written)
        hq = Q.numel() // (n * hd) if n else 0
        ldq, ldqo = _heads(Q, "Q", dev, dtype, n, hq, hd), _heads(Q_out, "Q_out", dev, dtype, n, hq, hd)
        pq, pqo = Q.data_ptr(), Q_out.data_ptr()
    elif Q_out is not None:
        raise ValueError("Q_out without Q")
    if rope is not None:
        if positions is None or rope.dim() != 2:
            raise ValueError("rope: [n_pos, rot_dim] needed, and positions with it")
        ppos, prope = _index(positions, "positions", dev, torch.int32, (n,)), _index(rope, "rope", dev, torch.float32, rope.shape)
        n_pos, rot = rope.shape
    _check(lib().kt_kv_append(ref, pq, ldq, K.data_ptr(), ldk, V.data_ptr(), ldv, n, hq, dt, pslots, ppos, prope, n_pos, rot,
                              bool(interleaved), bool(hadamard), pqo, ldqo, _stream(stream)))
    return Q_out


def kt_kv_gather(cache, slots, *, K=None, V=None, dtype=torch.bfloat16, stream=None):
    """The values held in `slots` [n]: (K, V) [n][heads][head_dim], those given or, if neither is, new ones of `dtype` (zeros for slots
    outside the cache)."""
    dev, n, heads, hd = _device(slots, "slots"), slots.shape[0], cache.n_heads, cache.head_dim
    if K is None and V is None:
        K, V = (_new(torch.zeros, stream, n, heads, hd, dtype=dtype, device=slots.device) for _ in range(2))
    ref = cache._on(dev)
    pslots = _index(slots, "slots", dev, torch.int64, (n,))
    first = K if K is not None else V
    ldk = ldv = 0
    pk = pv = None
    if K is not None:
        ldk, pk = _heads(K, "K", dev, first.dtype, n, heads, hd), K.data_ptr()
    if V is not None:
        ldv, pv = _heads(V, "V", dev, first.dtype, n, heads, hd), V.data_ptr()
    _check(lib().kt_kv_gather(ref, pslots, n, pk, ldk, pv, ldv, _dtype_code(first), _stream(stream)))
    return K, V


def kt_paged_attention(Q, cache, pages, lens, *, q_starts=None, max_q=None, prefix_pages=None, prefix_len=0, scale=None, out=None,
                       lse=None, workspace=None, stream=None):
    """Attention of Q [n_tokens][heads][head_dim] over the cache; returns out (given or new).  scale: 1 / sqrt(head_dim).
    max_q: a bound on the queries of a sequence (rows of a longer one can be left as they were); without one, all of Q's."""
    return _attention(Q, cache, pages, lens, None, q_starts, max_q, prefix_pages, prefix_len, scale, out, lse, workspace, stream)


def kt_tree_attention(Q, cache, pages, lens, tree, *, q_starts=None, max_q=None, prefix_pages=None, prefix_len=0, scale=None, out=None,
                      lse=None, workspace=None, stream=None):
    """kt_paged_attention where a query sees, of its sequence's queries, those whose bit is set in its row of `tree` [n_tokens][words] int64
    (query d: bit d % 64 of word d / 64).  max_q: without one, all of Q's, for which the words need bits; a sequence with more queries than a bound that is
    given has wrong rows (queries behind the last bit are seen by none)."""
    if tree.dim() != 2:
        raise ValueError(f"tree: [n_tokens, words] needed, got {tuple(tree.shape)}")
    if max_q is None and q_starts is not None and Q.shape[0] > 64 * tree.shape[1]:
        raise ValueError(f"max_q: needed where Q has more rows ({Q.shape[0]}) than words of tree have bits ({64 * tree.shape[1]})")
    return _attention(Q, cache, pages, lens, tree, q_starts, max_q, prefix_pages, prefix_len, scale, out, lse, workspace, stream)


def _queries(Q, cache, dev):
    """Sizes of Q [n_tokens][heads][head_dim], its leading dimension."""
    if Q.dim() != 3:
        raise ValueError(f"Q: [n_tokens, heads, head_dim] needed, got {tuple(Q.shape)}")
    n, hq, hd = Q.shape
    if hd != cache.head_dim:
        raise ValueError(f"Q: heads of {hd} features, {cache.head_dim} in the cache")
    return n, hq, hd, _heads(Q, "Q", dev, Q.dtype, n, hq, hd)


def _table(pages, name, dev, n_seq):
    """Address and width of a table of pages."""
    if pages.dim() != 2:
        raise ValueError(f"{name}: [{n_seq}, pages of a sequence] needed, got {tuple(pages.shape)}")
    return _index(pages, name, dev, torch.int32, (n_seq, pages.shape[1])), pages.shape[1]


def _attention(Q, cache, pages, lens, tree, q_starts, max_q, prefix_pages, prefix_len, scale, out, lse, workspace, stream):
    dev, dtype = _device(Q, "Q"), Q.dtype
    n, hq, hd, ldq = _queries(Q, cache, dev)
    if out is None:     # (rows in no sequence are not written)
        out = _new(torch.empty if q_starts is None else torch.zeros, stream, n, hq, hd, dtype=dtype, device=Q.device)
    ws = workspace if workspace is not None else Workspace(Q.device)
    ref = cache._on(dev)
    n_seq = lens.shape[0]
    if max_q is None:
        max_q = 1 if q_starts is None else n
    ldo = _heads(out, "out", dev, dtype, n, hq, hd)
    plens = _index(lens, "lens", dev, torch.int32, (n_seq,))
    ppages, ldp = _table(pages, "pages", dev, n_seq)
    pstarts = pprefix = plse = None
    if q_starts is not None:
        pstarts = _index(q_starts, "q_starts", dev, torch.int32, (n_seq + 1,))
    if prefix_len:
        if prefix_pages is None or prefix_pages.dim() != 1 or prefix_pages.shape[0] * cache.page_size < prefix_len:
            raise ValueError("prefix_pages: one dimension of pages for prefix_len tokens needed")
        pprefix = _index(prefix_pages, "prefix_pages", dev, torch.int32, prefix_pages.shape)
    if lse is not None:
        plse = _index(lse, "lse", dev, torch.float32, (n, hq))
    masks = () if tree is None else (_index(tree, "tree", dev, torch.int64, (n, tree.shape[1])), tree.shape[1])
    L = lib()
    buf = _new(ws.get, stream, L.kt_paged_attention_bytes(n, hq, hd, prefix_len))
    if buf.get_device() != dev:
        raise ValueError(f"workspace is on {buf.device}: operands have to be on the current device")
    call = L.kt_paged_attention if tree is None else L.kt_tree_attention
    _check(call(ref, Q.data_ptr(), ldq, _dtype_code(Q), pstarts, plens, ppages, ldp, n_seq, n, max_q, hq, *masks, pprefix, prefix_len,
                hd ** -0.5 if scale is None else scale, out.data_ptr(), ldo, plse, buf.data_ptr(), buf.numel(), _stream(stream, dev)))
    return out


def _mass(mass, cache, dev):
    return _index(mass, "mass", dev, torch.float32, cache._mass_shape)


def kt_attention_mass(Q, cache, pages, lens, lse, mass, *, q_starts=None, max_q=None, scale=None, decay=1.0, stream=None):
    """Adds to `mass` [n_pages][heads][page_size] fp32 the attention weight that the cache's tokens receive from Q [n_tokens][heads][head_dim], whose
    lse [n_tokens][heads] attention has written, after a product of what is there with `decay`; returns mass.  Tokens of pages that sequences begin with together
    get that of the first of them."""
    dev = _device(Q, "Q")
    n, hq, hd, ldq = _queries(Q, cache, dev)
    ref = cache._on(dev)
    n_seq = lens.shape[0]
    if max_q is None:
        max_q = 1 if q_starts is None else n
    plens = _index(lens, "lens", dev, torch.int32, (n_seq,))
    ppages, ldp = _table(pages, "pages", dev, n_seq)
    pstarts = None if q_starts is None else _index(q_starts, "q_starts", dev, torch.int32, (n_seq + 1,))
    _check(lib().kt_attention_mass(ref, Q.data_ptr(), ldq, _dtype_code(Q), pstarts, plens, ppages, ldp, n_seq, n, max_q, hq,
                                   hd ** -0.5 if scale is None else scale, _index(lse, "lse", dev, torch.float32, (n, hq)), decay,
                                   _mass(mass, cache, dev), _stream(stream, dev)))
    return mass


def kt_kv_select(cache, mass, pages, lens, keep, *, sink=0, recent=0, kept=None, n_kept=None, stream=None):
    """The tokens of every sequence and head that stay: (kept [n_seq][heads][most] int32, n_kept [n_seq] int32), those given or new ones.
    keep: tokens of each sequence [n_seq] int32 (kept is needed then), or a number for all of them."""
    dev, n_seq = _device(mass, "mass"), lens.shape[0]
    plens = _index(lens, "lens", dev, torch.int32, (n_seq,))
    ppages, ldp = _table(pages, "pages", dev, n_seq)
    pmass = _mass(mass, cache, dev)
    if not isinstance(keep, torch.Tensor):
        most = min(int(keep), ldp * cache.page_size)
        if most < 1:
            raise ValueError(f"keep: a positive number needed, got {keep}")
        keep = _new(torch.full, stream, (n_seq,), most, dtype=torch.int32, device=mass.device)
        if kept is None:
            kept = _new(torch.zeros, stream, n_seq, cache.n_heads, most, dtype=torch.int32, device=mass.device)
    if kept is None or kept.dim() != 3:
        raise ValueError("kept: [n_seq, heads, most tokens to keep] needed")
    if n_kept is None:
        n_kept = _new(torch.empty, stream, n_seq, dtype=torch.int32, device=mass.device)
    _check(lib().kt_kv_select(cache.ref, pmass, plens, ppages, ldp, n_seq, _index(keep, "keep", dev, torch.int32, (n_seq,)), sink, recent,
                              _index(kept, "kept", dev, torch.int32, (n_seq, cache._mass_shape[1], kept.shape[2])), kept.shape[2],
                              _index(n_kept, "n_kept", dev, torch.int32, (n_seq,)), _stream(stream, dev)))
    return kept, n_kept


def kt_kv_compact(cache, pages, src, count, *, first=None, to_pages=None, mass=None, stream=None):
    """Token src[j] of every sequence becomes its token first + j (first [n_seq] int32: 0 without), j < count [n_seq] int32, in place or in to_pages.
    src: [n_seq][most] int32, or [n_seq][heads][most] with a list for each head."""
    dev, n_seq = _device(pages, "pages"), count.shape[0]
    ref = cache._on(dev)
    ppages, ldp = _table(pages, "pages", dev, n_seq)
    if src.dim() not in (2, 3):
        raise ValueError(f"src: [n_seq, tokens] or [n_seq, heads, tokens] needed, got {tuple(src.shape)}")
    lds, per_head = src.shape[-1], src.dim() == 3
    psrc = _index(src, "src", dev, torch.int32, (n_seq, cache._mass_shape[1], lds) if per_head else (n_seq, lds))
    pto, ldt = (None, 0) if to_pages is None else _table(to_pages, "to_pages", dev, n_seq)
    _check(lib().kt_kv_compact(ref, ppages, ldp, n_seq, psrc, lds, per_head, _index(count, "count", dev, torch.int32, (n_seq,)),
                               None if first is None else _index(first, "first", dev, torch.int32, (n_seq,)), pto, ldt,
                               None if mass is None else _mass(mass, cache, dev), _stream(stream, dev)))


def kt_profile_enable(max_records):
    _check(lib().kt_profile_enable(int(max_records)))


def kt_profile_reset():
    _check(lib().kt_profile_reset())


def kt_profile_read(kernel_id):
    """(total_ms, launches) of the bracketed launches with this id since the last reset."""
    tot, cnt = ctypes.c_double(0.0), ctypes.c_int32(0)
    _check(lib().kt_profile_read(int(kernel_id), ctypes.byref(tot), ctypes.byref(cnt)))
    return tot.value, cnt.value
