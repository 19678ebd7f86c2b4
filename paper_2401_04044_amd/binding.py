"""ctypes binding: same names as the C ABI, argument marshalling only."""
import contextlib
import ctypes
import os

import torch

ACT_GELU, ACT_SWIGLU = 0, 1
F32, BF16 = 0, 1
REM_NONE, REM_DENSE, REM_LOWRANK, REM_INT4, REM_W3H8 = 0, 1, 2, 3, 4
SCORE_SUMSQ, SCORE_MEAN_L2, SCORE_ACT_ONLY = 0, 1, 2
SCORE_REUSE_TILED = 0x100
WS_SCORE, WS_SELECT, WS_BUILD, WS_FORWARD, WS_FACTORIZE, WS_STACK = 0, 1, 2, 3, 4, 5
WS_DENSE_FORWARD, WS_DENSE_BACKWARD, WS_DENSE_STACK, WS_GRAD_NORM = 6, 7, 8, 9
GRAD_F32, GRAD_ACCUMULATE = 1, 2
E_NONFINITE = -7

_HERE = os.path.dirname(os.path.abspath(__file__))


def lib_path() -> str:
    return os.path.join(_HERE, "libffsplit.so")


class FFSplitError(RuntimeError):
    def __init__(self, code, where):
        self.code = code
        super().__init__(f"{where}: {status_string(code)} ({code})")


class Epilogue(ctypes.Structure):
    _fields_ = [("b1_packed", ctypes.c_void_p), ("b2", ctypes.c_void_p), ("residual", ctypes.c_void_p),
                ("y_f32", ctypes.c_int32)]


class Desc(ctypes.Structure):
    _fields_ = [("d_model", ctypes.c_int32), ("d_ff", ctypes.c_int32), ("act", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("k", ctypes.c_int32), ("rem_kind", ctypes.c_int32),
                ("rank", ctypes.c_int32), ("group", ctypes.c_int32)]


def _load():
    path = lib_path()
    if not os.path.exists(path):
        raise ImportError(f"{path} is missing: build it first (python -c 'import __graft_entry__ as g; g.build()')")
    L = ctypes.CDLL(path)
    vp, i32, i64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
    dp = ctypes.POINTER(Desc)
    L.ffsplit_status_string.restype = ctypes.c_char_p
    L.ffsplit_status_string.argtypes = [ctypes.c_int]
    L.ffsplit_workspace_bytes.restype = sz
    L.ffsplit_workspace_bytes.argtypes = [dp, i32, i64]
    L.ffsplit_split_bytes.restype = sz
    L.ffsplit_split_bytes.argtypes = [dp]
    L.ffsplit_score_neurons.restype = ctypes.c_int
    L.ffsplit_score_neurons.argtypes = [dp, vp, i64, vp, vp, vp, vp, ctypes.POINTER(i64), vp, i32, vp, sz, vp]
    L.ffsplit_select_heavy.restype = ctypes.c_int
    L.ffsplit_select_heavy.argtypes = [vp, i32, i32, vp, vp, vp, vp, sz, vp]
    L.ffsplit_select_heavy_static.restype = ctypes.c_int
    L.ffsplit_select_heavy_static.argtypes = [vp, i32, i32, vp, vp, vp, vp]
    L.ffsplit_build_split.restype = ctypes.c_int
    L.ffsplit_build_split.argtypes = [dp, vp, vp, vp, vp, ctypes.POINTER(vp), vp, vp, sz, vp]
    L.ffsplit_forward.restype = ctypes.c_int
    L.ffsplit_forward.argtypes = [dp, vp, vp, i64, vp, vp, vp, vp, sz, vp]
    L.ffsplit_forward_ex.restype = ctypes.c_int
    L.ffsplit_forward_ex.argtypes = [dp, vp, vp, i64, vp, vp, vp, ctypes.POINTER(Epilogue), vp, sz, vp]
    L.ffsplit_neuron_bias_floats.restype = sz
    L.ffsplit_neuron_bias_floats.argtypes = [dp]
    L.ffsplit_pack_neuron_bias.restype = ctypes.c_int
    L.ffsplit_pack_neuron_bias.argtypes = [dp, vp, vp, vp, vp, sz, vp]
    L.ffsplit_token_rmsnorm.restype = ctypes.c_int
    L.ffsplit_token_rmsnorm.argtypes = [vp, i64, i32, ctypes.c_float, i32, vp, vp]
    L.ffsplit_stack_forward.restype = ctypes.c_int
    L.ffsplit_stack_forward.argtypes = [dp, i32, ctypes.POINTER(vp), ctypes.POINTER(vp), ctypes.POINTER(vp), vp, i64,
                                        ctypes.c_float, vp, sz, vp]
    L.ffsplit_probe_mfma.restype = ctypes.c_int
    L.ffsplit_probe_mfma.argtypes = [i32, i32, vp, ctypes.POINTER(ctypes.c_double), vp]
    L.ffsplit_probe_stream_read.restype = ctypes.c_int
    L.ffsplit_probe_stream_read.argtypes = [vp, sz, i32, vp, vp]
    L.ffsplit_factorize_remainder.restype = ctypes.c_int
    L.ffsplit_factorize_remainder.argtypes = [dp, vp, vp, vp, vp, ctypes.c_uint32, ctypes.POINTER(vp), vp, sz, vp]
    vpp, f32 = ctypes.POINTER(vp), ctypes.c_float
    L.ffsplit_dense_kept_bytes.restype = sz
    L.ffsplit_dense_kept_bytes.argtypes = [dp, i64]
    L.ffsplit_dense_forward.restype = ctypes.c_int
    L.ffsplit_dense_forward.argtypes = [dp, vp, i64, vp, vp, vp, vp, vp, i32, vp, vp, sz, vp]
    L.ffsplit_dense_backward.restype = ctypes.c_int
    L.ffsplit_dense_backward.argtypes = [dp, vp, i64, vp, vp, vp, vp, vp, vp, vp, vp, vp, i32, vp, sz, vp]
    L.ffsplit_token_rmsnorm_backward.restype = ctypes.c_int
    L.ffsplit_token_rmsnorm_backward.argtypes = [vp, vp, i64, i32, f32, i32, vp, vp, vp, vp]
    L.ffsplit_grad_norm.restype = ctypes.c_int
    L.ffsplit_grad_norm.argtypes = [i32, vpp, ctypes.POINTER(i64), ctypes.POINTER(i32), vp, vp, vp, sz, vp]
    L.ffsplit_grad_clip.restype = ctypes.c_int
    L.ffsplit_grad_clip.argtypes = [i32, vpp, ctypes.POINTER(i64), ctypes.POINTER(i32), vp, f32, vpp, vp]
    L.ffsplit_dense_stack_kept_bytes.restype = sz
    L.ffsplit_dense_stack_kept_bytes.argtypes = [dp, i32, i64]
    L.ffsplit_dense_stack_forward.restype = ctypes.c_int
    L.ffsplit_dense_stack_forward.argtypes = [dp, i32, vpp, vpp, vpp, vp, i64, f32, vp, vp, sz, vp]
    L.ffsplit_dense_stack_backward.restype = ctypes.c_int
    L.ffsplit_dense_stack_backward.argtypes = [dp, i32, vpp, vpp, vpp, vp, vp, i64, f32, vpp, vpp, vpp, i32, f32, vp, vp,
                                               vp, sz, vp]
    L.ffsplit_split_export.restype = ctypes.c_int
    L.ffsplit_split_export.argtypes = [dp, vp, i32, vp, vp, vp]
    return L


lib = _load()


def status_string(code: int) -> str:
    return lib.ffsplit_status_string(int(code)).decode()


def make_desc(d_model, d_ff, act="gelu", dtype="bf16", k=0, rem_kind="none", rank=0, group=0) -> Desc:
    acts = {"gelu": ACT_GELU, "swiglu": ACT_SWIGLU}
    dts = {"f32": F32, "bf16": BF16}
    rems = {"none": REM_NONE, "dense": REM_DENSE, "lowrank": REM_LOWRANK, "int4": REM_INT4, "w3h8": REM_W3H8}
    return Desc(d_model, d_ff, acts.get(act, act), dts.get(dtype, dtype), k, rems.get(rem_kind, rem_kind),
                rank, group)


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream():
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


def _check(code, where):
    if code != 0:
        raise FFSplitError(code, where)


def workspace_bytes(desc: Desc, call_id: int, T: int = 0) -> int:
    return int(lib.ffsplit_workspace_bytes(ctypes.byref(desc), call_id, T))


def split_bytes(desc: Desc) -> int:
    return int(lib.ffsplit_split_bytes(ctypes.byref(desc)))


def _ws(nbytes, workspace, device):
    if workspace is not None:
        return workspace
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)


def score_neurons(desc, X, W1, Wg, W2, acc, T_total, scores=None, score_kind=SCORE_SUMSQ, workspace=None):
    """One calibration batch.  Returns the updated token count."""
    T = 0 if X is None else X.shape[0]
    ws = _ws(workspace_bytes(desc, WS_SCORE, T), workspace, acc.device)
    tt = ctypes.c_int64(int(T_total))
    rc = lib.ffsplit_score_neurons(ctypes.byref(desc), _ptr(X), T, _ptr(W1), _ptr(Wg), _ptr(W2), _ptr(acc),
                                   ctypes.byref(tt), _ptr(scores), score_kind, _ptr(ws), ws.numel(), _stream())
    _check(rc, "ffsplit_score_neurons")
    return tt.value


def select_heavy(scores, k, want_perm=False, workspace=None):
    """Returns (idx [k] int32, perm [d_ff] int32 or None, nan_flag [1] int32), all on the device."""
    d_ff = scores.numel()
    dev = scores.device
    idx = torch.empty(max(k, 1), dtype=torch.int32, device=dev)[:k]
    perm = torch.empty(d_ff, dtype=torch.int32, device=dev) if want_perm else None
    flag = torch.empty(1, dtype=torch.int32, device=dev)   # (every call writes it)
    ws = _ws(int(lib.ffsplit_workspace_bytes(ctypes.byref(make_desc(8, d_ff)), WS_SELECT, 0)), workspace, dev)
    rc = lib.ffsplit_select_heavy(_ptr(scores), d_ff, k, _ptr(idx) if k > 0 else None, _ptr(perm), _ptr(flag),
                                  _ptr(ws), ws.numel(), _stream())
    _check(rc, "ffsplit_select_heavy")
    return idx, perm, flag


SELECT_STATIC_MAX_DFF = 65536


def select_heavy_static(scores, k, idx, perm=None, flag=None):
    """ffsplit_select_heavy_static: every buffer is the caller's, nothing is allocated here."""
    rc = lib.ffsplit_select_heavy_static(_ptr(scores), scores.numel(), k, _ptr(idx) if k > 0 else None, _ptr(perm),
                                         _ptr(flag), _stream())
    _check(rc, "ffsplit_select_heavy_static")


def build_split(desc, W1, Wg, W2, idx, factors=None, split=None, workspace=None):
    """factors: dict with P1, Q1, Pg, Qg, P2, Q2 (device tensors or None).  Returns the packed split."""
    dev = W1.device
    nbytes = split_bytes(desc)
    if nbytes == 0:
        _check(-2, "ffsplit_split_bytes")
    if split is None:
        split = torch.empty(nbytes, dtype=torch.uint8, device=dev)
    ws = _ws(workspace_bytes(desc, WS_BUILD, 0), workspace, dev)
    fac = None
    if factors is not None:
        arr = (ctypes.c_void_p * 6)()
        for i, nm in enumerate(("P1", "Q1", "Pg", "Qg", "P2", "Q2")):
            t = factors.get(nm)
            arr[i] = None if t is None else t.data_ptr()
        fac = arr
    rc = lib.ffsplit_build_split(ctypes.byref(desc), _ptr(W1), _ptr(Wg), _ptr(W2),
                                 _ptr(idx) if idx is not None and idx.numel() > 0 else None, fac, _ptr(split),
                                 _ptr(ws), ws.numel(), _stream())
    _check(rc, "ffsplit_build_split")
    return split


def factorize_remainder(desc, W1, Wg, W2, idx, seed=0, workspace=None):
    """Rank-r factors of the remainder on the device: dict P1, Q1, Pg, Qg, P2, Q2 (device tensors)."""
    dev = W1.device
    d, m, r = desc.d_model, desc.d_ff - desc.k, desc.rank
    glu = Wg is not None
    shapes = {"P1": (d, r), "Q1": (r, m), "Pg": (d, r), "Qg": (r, m), "P2": (m, r), "Q2": (r, d)}
    out = {nm: (torch.empty(sh, dtype=W1.dtype, device=dev) if (glu or nm not in ("Pg", "Qg")) else None)
           for nm, sh in shapes.items()}
    arr = (ctypes.c_void_p * 6)()
    for i, nm in enumerate(("P1", "Q1", "Pg", "Qg", "P2", "Q2")):
        arr[i] = None if out[nm] is None else out[nm].data_ptr()
    ws = _ws(workspace_bytes(desc, WS_FACTORIZE, 0), workspace, dev)
    rc = lib.ffsplit_factorize_remainder(ctypes.byref(desc), _ptr(W1), _ptr(Wg), _ptr(W2),
                                         _ptr(idx) if idx is not None and idx.numel() > 0 else None,
                                         ctypes.c_uint32(seed), arr, _ptr(ws), ws.numel(), _stream())
    _check(rc, "ffsplit_factorize_remainder")
    return out


def forward(desc, split, X, Y=None, want_parts=False, workspace=None):
    """Returns Y, or (Y, Y_heavy, Y_rem) with want_parts."""
    T = X.shape[0]
    if Y is None:
        Y = torch.empty((T, desc.d_model), dtype=X.dtype, device=X.device)
    Yh = torch.empty_like(Y) if want_parts else None
    Yr = torch.empty_like(Y) if want_parts else None
    ws = _ws(workspace_bytes(desc, WS_FORWARD, T), workspace, X.device)
    rc = lib.ffsplit_forward(ctypes.byref(desc), _ptr(split), _ptr(X), T, _ptr(Y), _ptr(Yh), _ptr(Yr), _ptr(ws),
                             ws.numel(), _stream())
    _check(rc, "ffsplit_forward")
    return (Y, Yh, Yr) if want_parts else Y


def forward_ex(desc, split, X, Y=None, b1_packed=None, b2=None, residual=None, y_f32=False, want_parts=False,
               workspace=None):
    """ffsplit_forward_ex: Y = [residual +] FFN_split(X) [+ b2], neuron biases in packed order.
    Returns Y, or (Y, Y_heavy, Y_rem) with want_parts."""
    T = X.shape[0]
    if Y is None:
        Y = torch.empty((T, desc.d_model), dtype=torch.float32 if y_f32 else X.dtype, device=X.device)
    Yh = torch.empty((T, desc.d_model), dtype=X.dtype, device=X.device) if want_parts else None
    Yr = torch.empty((T, desc.d_model), dtype=X.dtype, device=X.device) if want_parts else None
    ws = _ws(workspace_bytes(desc, WS_FORWARD, T), workspace, X.device)
    e = Epilogue(None if b1_packed is None else b1_packed.data_ptr(), None if b2 is None else b2.data_ptr(),
                 None if residual is None else residual.data_ptr(), 1 if y_f32 else 0)
    rc = lib.ffsplit_forward_ex(ctypes.byref(desc), _ptr(split), _ptr(X), T, _ptr(Y), _ptr(Yh), _ptr(Yr),
                                ctypes.byref(e), _ptr(ws), ws.numel(), _stream())
    _check(rc, "ffsplit_forward_ex")
    return (Y, Yh, Yr) if want_parts else Y


def pack_neuron_bias(desc, b1, idx, workspace=None):
    """b1 [d_ff] in the layer's dtype -> fp32 vector in the packed split's neuron order."""
    n = int(lib.ffsplit_neuron_bias_floats(ctypes.byref(desc)))
    out = torch.empty(max(n, 1), dtype=torch.float32, device=b1.device)
    ws = _ws(workspace_bytes(desc, WS_BUILD, 0), workspace, b1.device)
    rc = lib.ffsplit_pack_neuron_bias(ctypes.byref(desc), _ptr(b1), _ptr(idx) if idx is not None and idx.numel() > 0
                                      else None, _ptr(out), _ptr(ws), ws.numel(), _stream())
    _check(rc, "ffsplit_pack_neuron_bias")
    return out


def token_rmsnorm(x, dtype=BF16, eps=1e-6, out=None):
    """n(x) = x / sqrt(mean(x^2) + eps) per token; x fp32 [T, d]."""
    T, d = x.shape
    if out is None:
        out = torch.empty((T, d), dtype=torch.bfloat16 if dtype == BF16 else torch.float32, device=x.device)
    rc = lib.ffsplit_token_rmsnorm(_ptr(x), T, d, ctypes.c_float(eps), dtype, _ptr(out), _stream())
    _check(rc, "ffsplit_token_rmsnorm")
    return out


def stack_forward(desc, splits, x, b1_packed=None, b2=None, eps=1e-6, workspace=None):
    """x <- x + FFN_split_l(n(x)) [+ b2_l] for every layer, in place on the fp32 stream x [T, d]."""
    n, T = len(splits), x.shape[0]

    def arr(ts):
        if ts is None:
            return None
        a = (ctypes.c_void_p * n)()
        for i, t in enumerate(ts):
            a[i] = None if t is None else t.data_ptr()
        return a

    ws = _ws(workspace_bytes(desc, WS_STACK, T), workspace, x.device)
    rc = lib.ffsplit_stack_forward(ctypes.byref(desc), n, arr(splits), arr(b1_packed), arr(b2), _ptr(x), T,
                                   ctypes.c_float(eps), _ptr(ws), ws.numel(), _stream())
    _check(rc, "ffsplit_stack_forward")
    return x


_DTYPES = {F32: torch.float32, BF16: torch.bfloat16}


def _take(t, what, shape, dtype, device):
    """A tensor argument of the training calls: they take plain row-major matrices, so that a view with
    strides, another type or another device is an error here and not a wrong result there."""
    if t is None:
        return None
    if t.dtype is not dtype and t.dtype != dtype:
        raise TypeError(f"{what}: {t.dtype}, wanted {dtype}")
    if shape is not None and t.shape != shape:
        raise ValueError(f"{what}: shape {tuple(t.shape)}, wanted {tuple(shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{what}: not contiguous")
    if t.device != device:
        raise ValueError(f"{what}: on {t.device}, wanted {device}")
    return t


def _no_graph(**tensors):
    """The calls are not recorded by autograd: a graph that leads into one would end there unnoticed, and a write into a
    tensor of a graph would not be noticed either.  (Weights may be parameters: their gradients are dense_backward's.)"""
    if torch.is_grad_enabled():
        for what, t in tensors.items():
            if t is not None and t.requires_grad:
                raise ValueError(f"{what}: requires grad, but the call is not recorded: detach it and take its gradient from the "
                                 "backward call")


_HERE_ALREADY = contextlib.nullcontext()


def _raw_stream(device):
    """The current stream of a device, without the stream object that _stream() makes (5 us of a 10 us call)."""
    return torch._C._cuda_getCurrentRawStream(device.index)



def _on(device):
    """The device of the tensors made current, for the stream, the scratch and the launches."""
    if device.type != "cuda":
        raise ValueError(f"tensors on {device}, wanted a GPU")
    return _HERE_ALREADY if torch.cuda.current_device() == device.index else torch.cuda.device(device)


def _take_layer(desc, W1, Wg, W2, device, what=""):
    dt, d, f = _DTYPES[desc.dtype], desc.d_model, desc.d_ff
    _take(W1, "W1" + what, (d, f), dt, device)
    _take(Wg, "Wg" + what, (d, f), dt, device)
    _take(W2, "W2" + what, (f, d), dt, device)


def _scratch(nbytes, workspace, device):
    if workspace is not None:
        return _take(workspace, "workspace", None, torch.uint8, device)
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)


def _ptrs(ts):
    if ts is None:
        return None
    a = (ctypes.c_void_p * max(len(ts), 1))()
    for i, t in enumerate(ts):
        a[i] = None if t is None else t.data_ptr()
    return a


def dense_kept_bytes(desc, T):
    return int(lib.ffsplit_dense_kept_bytes(ctypes.byref(desc), T))


def dense_forward(desc, X, W1, Wg, W2, Y=None, residual=None, y_f32=False, want_saved=False, saved=None, workspace=None):
    """The uncompressed layer on plain weights: Y = [residual +] act(X W1, X Wg) W2.  Returns Y, or (Y, saved)
    with want_saved or a buffer for it: what dense_backward needs.  Not recorded by autograd (dense_backward gives the
    gradients): X, residual and Y that require grad are refused while it records, weights may be parameters."""
    _no_graph(X=X, residual=residual, Y=Y)
    T, dev, dt = X.shape[0], X.device, _DTYPES[desc.dtype]
    _take(X, "X", (T, desc.d_model), dt, dev)
    _take_layer(desc, W1, Wg, W2, dev)
    y_dt = torch.float32 if y_f32 else dt
    if Y is None:
        Y = torch.empty((T, desc.d_model), dtype=y_dt, device=dev)
    _take(Y, "Y", (T, desc.d_model), y_dt, dev)
    _take(residual, "residual", (T, desc.d_model), torch.float32, dev)
    keep = want_saved or saved is not None
    if keep:
        need = dense_kept_bytes(desc, T)
        if saved is None:
            saved = torch.empty(max(need, 256), dtype=torch.uint8, device=dev)
        _take_kept(saved, need, dev)
    with _on(dev):
        ws = _scratch(workspace_bytes(desc, WS_DENSE_FORWARD, T), workspace, dev)
        rc = lib.ffsplit_dense_forward(ctypes.byref(desc), _ptr(X), T, _ptr(W1), _ptr(Wg), _ptr(W2), _ptr(Y), _ptr(residual),
                                       1 if y_f32 else 0, _ptr(saved) if keep else None, _ptr(ws), ws.numel(), _raw_stream(dev))
    _check(rc, "ffsplit_dense_forward")
    return (Y, saved) if keep else Y


def _take_kept(saved, need, device):
    _take(saved, "saved", None, torch.uint8, device)
    if saved.numel() < need:
        raise ValueError(f"saved: {saved.numel()} bytes, wanted {need}")


def _grad_flags(accumulate, grad_f32):
    return (GRAD_ACCUMULATE if accumulate else 0) | (GRAD_F32 if grad_f32 else 0)


def _grads_for(desc, grads, accumulate, grad_f32, device, what=""):
    """The gradients' buffers of one layer: given ones (a dict; a missing or None entry is not computed), or new."""
    names = ("W1", "Wg", "W2") if desc.act == ACT_SWIGLU else ("W1", "W2")
    dt = torch.float32 if grad_f32 else _DTYPES[desc.dtype]
    shapes = {"W1": (desc.d_model, desc.d_ff), "Wg": (desc.d_model, desc.d_ff), "W2": (desc.d_ff, desc.d_model)}
    if grads is None:
        if accumulate:
            raise ValueError("accumulate: the gradients to add to are wanted")
        return {k: torch.empty(shapes[k], dtype=dt, device=device) if k in names else None for k in shapes}
    for k, g in grads.items():
        if k not in shapes or (g is not None and k not in names):
            raise ValueError(f"no gradient {k!r} of this layer")
        _take(g, f"gradient of {k}{what}", shapes[k], dt, device)
    return {k: grads.get(k) for k in shapes}


def _grads_apart(written, others):
    """A gradient's buffer is written once, and while the call still reads the other tensors."""
    spans = sorted([(t.data_ptr(), t.nbytes, 1) for t in written] + [(t.data_ptr(), t.nbytes, 0) for t in others])
    end = end_written = 0       # of what begins further in front
    for at, n, is_written in spans:
        if at < (end if is_written else end_written):
            raise ValueError("gradients: a buffer that overlaps another tensor of the call")
        end = max(end, at + n)
        if is_written:
            end_written = max(end_written, at + n)


def dense_backward(desc, X, W1, Wg, W2, saved, dY, dX=None, want_dx=True, grads=None, accumulate=False, grad_f32=False,
                   workspace=None):
    """Backward pass of dense_forward.  Returns (dX or None, {"W1", "Wg", "W2": gradients or None})."""
    T, dev, dt = X.shape[0], X.device, _DTYPES[desc.dtype]
    _take(X, "X", (T, desc.d_model), dt, dev)
    _take_layer(desc, W1, Wg, W2, dev)
    _take(dY, "dY", (T, desc.d_model), dt, dev)
    _take_kept(saved, dense_kept_bytes(desc, T), dev)
    mine = [] if dX is None else [dX]
    if dX is None and want_dx:
        dX = torch.empty((T, desc.d_model), dtype=dt, device=dev)
    _take(dX, "dX", (T, desc.d_model), dt, dev)
    if dX is not None and T and dX.data_ptr() in (dY.data_ptr(), X.data_ptr()):
        raise ValueError("dX: the buffer of dY or X, which the weights' gradients read behind it")
    g = _grads_for(desc, grads, accumulate, grad_f32, dev)
    if grads is not None:
        mine += [t for t in g.values() if t is not None]
    if mine and T:
        _grads_apart(mine, [t for t in (dY, X, W1, Wg, W2, saved) if t is not None])
    with _on(dev):
        ws = _scratch(workspace_bytes(desc, WS_DENSE_BACKWARD, T), workspace, dev)
        rc = lib.ffsplit_dense_backward(ctypes.byref(desc), _ptr(X), T, _ptr(W1), _ptr(Wg), _ptr(W2), _ptr(saved), _ptr(dY),
                                        _ptr(dX), _ptr(g["W1"]), _ptr(g["Wg"]), _ptr(g["W2"]),
                                        _grad_flags(accumulate, grad_f32), _ptr(ws), ws.numel(), _raw_stream(dev))
    _check(rc, "ffsplit_dense_backward")
    return dX, g


def token_rmsnorm_backward(x, dn, eps=1e-6, residual=None, dx=None, want_cast=False):
    """Gradient of x behind token_rmsnorm: dx = [residual +] r dn - x r^3 mean(x dn), fp32 [T, d] (residual may
    be dx).  Returns dx, or (dx, dx in dn's type) with want_cast."""
    shape, dev = x.shape, x.device
    T, d = shape
    _take(x, "x", None, torch.float32, dev)
    bf16 = dn.dtype == torch.bfloat16
    _take(dn, "dn", shape, torch.bfloat16 if bf16 else torch.float32, dev)
    _take(residual, "residual", shape, torch.float32, dev)
    if dx is None:
        dx = torch.empty_like(x)
    else:
        _take(dx, "dx", shape, torch.float32, dev)
    cast = torch.empty_like(dn) if want_cast else None
    with _on(dev):
        rc = lib.ffsplit_token_rmsnorm_backward(x.data_ptr(), dn.data_ptr(), T, d, eps, BF16 if bf16 else F32, _ptr(residual),
                                                dx.data_ptr(), _ptr(cast), _raw_stream(dev))
    _check(rc, "ffsplit_token_rmsnorm_backward")
    return (dx, cast) if want_cast else dx


class _GradList:
    """The host arrays that describe a list of gradients."""

    def __init__(self, grads):
        n = self.n = len(grads)
        self.device = dev = grads[0].device if n else torch.device("cuda", torch.cuda.current_device())
        ptrs, counts, dtypes = [], [], []
        for g in grads:
            dt = g.dtype
            if dt != torch.float32 and dt != torch.bfloat16:
                raise TypeError(f"gradients: {dt}, wanted torch.float32 or torch.bfloat16")
            if not g.is_contiguous() or g.device != dev:
                raise ValueError(f"gradients: contiguous tensors on one device are wanted ({dev})")
            ptrs.append(g.data_ptr())
            counts.append(g.numel())
            dtypes.append(F32 if dt == torch.float32 else BF16)
        self._at = ptrs if 0 not in counts else [p if c else 0 for p, c in zip(ptrs, counts)]   # 0: nothing there
        self.ptrs, self.counts = (ctypes.c_void_p * max(n, 1))(*ptrs), (ctypes.c_int64 * max(n, 1))(*counts)
        self.dtypes = (ctypes.c_int32 * max(n, 1))(*dtypes)

    def out_ptrs(self, grads, out):
        if out is None:
            self._apart(self._at)
            return self.ptrs
        if len(out) != self.n:
            raise ValueError(f"out: {len(out)} tensors for {self.n} gradients")
        ptrs = []
        for g, o in zip(grads, out):
            if o.dtype != g.dtype or o.shape != g.shape or not o.is_contiguous() or o.device != self.device:
                raise ValueError("out: tensors like the gradients are wanted, contiguous and on their device")
            ptrs.append(o.data_ptr())
        at = ptrs if self._at.count(0) == 0 else [p if q else 0 for p, q in zip(ptrs, self._at)]
        there = self._apart(at)
        if not there.isdisjoint(self._at) and any(p != q and p in there for p, q in zip(self._at, at) if p):
            raise ValueError("out: the buffer of another gradient, which is still read")
        return (ctypes.c_void_p * max(self.n, 1))(*ptrs)

    def _apart(self, at):
        there = set(at)
        if len(there) + max(at.count(0) - 1, 0) != len(at):
            raise ValueError("gradients: a tensor that is written is listed twice")
        there.discard(0)
        return there

    def norm(self, norm, flag, workspace):
        dev = self.device
        norm = torch.empty(1, dtype=torch.float32, device=dev) if norm is None else _take(norm, "norm", (1,), torch.float32, dev)
        flag = torch.empty(1, dtype=torch.int32, device=dev) if flag is None else _take(flag, "flag", (1,), torch.int32, dev)
        ws = _scratch(lib.ffsplit_workspace_bytes(None, WS_GRAD_NORM, self.n), workspace, dev)
        _check(lib.ffsplit_grad_norm(self.n, self.ptrs, self.counts, self.dtypes, norm.data_ptr(), flag.data_ptr(), ws.data_ptr(),
                                     ws.numel(), _raw_stream(dev)), "ffsplit_grad_norm")
        return norm, flag

    def clip(self, norm, max_norm, out_ptrs):
        dev = self.device
        _check(lib.ffsplit_grad_clip(self.n, self.ptrs, self.counts, self.dtypes, norm.data_ptr(), max_norm, out_ptrs,
                                     _raw_stream(dev)), "ffsplit_grad_clip")


def grad_norm(grads, norm=None, flag=None, workspace=None):
    """Norm over all elements of all tensors.  Returns (norm [1] fp32, flag [1] int32), on the device; the flag is
    E_NONFINITE if the norm is not finite, else 0."""
    g = _GradList(grads)
    with _on(g.device):
        return g.norm(norm, flag, workspace)


def grad_clip(grads, norm, max_norm, out=None):
    """out = grads * min(1, max_norm / norm), in place without `out`; unchanged where the norm (on the device) is
    not finite.  Returns the list of clipped gradients."""
    g = _GradList(grads)
    to = g.out_ptrs(grads, out)
    _take(norm, "norm", (1,), torch.float32, g.device)
    with _on(g.device):
        g.clip(norm, max_norm, to)
    return grads if out is None else out


def clip_grad_norm(grads, max_norm, out=None, workspace=None):
    """grad_norm, then grad_clip.  Returns (norm, flag, clipped gradients)."""
    g = _GradList(grads)
    to = g.out_ptrs(grads, out)
    with _on(g.device):
        norm, flag = g.norm(None, None, workspace)
        g.clip(norm, max_norm, to)
    return norm, flag, grads if out is None else out


def _stack_args(desc, layers, device):
    for l, W in enumerate(layers):
        _take_layer(desc, W["W1"], W.get("Wg"), W["W2"], device, f" of layer {l}")
    gated = desc.act == ACT_SWIGLU
    return (_ptrs([W["W1"] for W in layers]), _ptrs([W.get("Wg") for W in layers]) if gated else None,
            _ptrs([W["W2"] for W in layers]))


def dense_stack_forward(desc, layers, x, eps=1e-6, want_saved=False, saved=None, workspace=None):
    """x <- x + FFN_l(n(x)) for every layer (dicts W1, Wg, W2), in place on the fp32 stream x [T, d].  Returns x, or
    what dense_stack_backward needs with want_saved or a buffer for it.  Not recorded by autograd, as dense_forward."""
    _no_graph(x=x)
    n, T, dev = len(layers), x.shape[0], x.device
    _take(x, "x", (T, desc.d_model), torch.float32, dev)
    keep = want_saved or saved is not None
    if keep:
        need = int(lib.ffsplit_dense_stack_kept_bytes(ctypes.byref(desc), n, T))
        if saved is None:
            saved = torch.empty(max(need, 256), dtype=torch.uint8, device=dev)
        _take_kept(saved, need, dev)
    W1, Wg, W2 = _stack_args(desc, layers, dev)
    with _on(dev):
        ws = _scratch(workspace_bytes(desc, WS_DENSE_STACK, T), workspace, dev)
        rc = lib.ffsplit_dense_stack_forward(ctypes.byref(desc), n, W1, Wg, W2, _ptr(x), T, ctypes.c_float(eps),
                                             _ptr(saved) if keep else None, _ptr(ws), ws.numel(), _raw_stream(dev))
    _check(rc, "ffsplit_dense_stack_forward")
    return saved if keep else x


def dense_stack_backward(desc, layers, saved, dx, eps=1e-6, grads=None, accumulate=False, grad_f32=False, max_norm=0.0,
                         workspace=None, want_norm=True):
    """Backward pass of dense_stack_forward, in place on the stream's gradient dx [T, d].  Returns (gradients: a dict
    W1, Wg, W2 per layer; their norm [1]; its flag [1]); with max_norm > 0 the gradients are clipped.  grads: dicts of
    buffers, one for every weight.  Without want_norm (all but the last of accumulated micro-batches) the gradients are
    not read again, and norm and flag are None."""
    n, T, dev = len(layers), dx.shape[0], dx.device
    _take(dx, "dx", (T, desc.d_model), torch.float32, dev)
    _take_kept(saved, int(lib.ffsplit_dense_stack_kept_bytes(ctypes.byref(desc), n, T)), dev)
    if grads is not None and len(grads) != n:
        raise ValueError(f"gradients of {len(grads)} layers for {n}")
    g = [_grads_for(desc, grads[l] if grads is not None else None, accumulate, grad_f32, dev, f" of layer {l}")
         for l in range(n)]
    written = [t.data_ptr() for q in g for t in q.values() if t is not None]
    if len(set(written)) != len(written):
        raise ValueError("gradients: a buffer is listed twice")
    if grads is not None:
        _grads_apart([t for q in g for t in q.values() if t is not None],
                     [W[k] for W in layers for k in ("W1", "Wg", "W2") if W.get(k) is not None] + [saved, dx])
    if max_norm > 0 and not want_norm:
        raise ValueError("max_norm: clipping needs the norm")
    W1, Wg, W2 = _stack_args(desc, layers, dev)
    gated = desc.act == ACT_SWIGLU
    with _on(dev):
        norm = torch.empty(1, dtype=torch.float32, device=dev) if want_norm else None
        flag = torch.empty(1, dtype=torch.int32, device=dev) if want_norm else None
        need = max(workspace_bytes(desc, WS_DENSE_STACK, T), int(lib.ffsplit_workspace_bytes(None, WS_GRAD_NORM, 3 * n)))
        ws = _scratch(need, workspace, dev)
        rc = lib.ffsplit_dense_stack_backward(ctypes.byref(desc), n, W1, Wg, W2, _ptr(saved), _ptr(dx), T,
                                              ctypes.c_float(eps), _ptrs([q["W1"] for q in g]),
                                              _ptrs([q["Wg"] for q in g]) if gated else None, _ptrs([q["W2"] for q in g]),
                                              _grad_flags(accumulate, grad_f32), ctypes.c_float(max_norm), _ptr(norm),
                                              _ptr(flag), _ptr(ws), ws.numel(), _raw_stream(dev))
    _check(rc, "ffsplit_dense_stack_backward")
    return g, norm, flag


def probe_mfma(workgroups, iters, scratch):
    """Enqueue the pure matrix-core loop; returns its flop count."""
    fl = ctypes.c_double(0.0)
    _check(lib.ffsplit_probe_mfma(workgroups, iters, _ptr(scratch), ctypes.byref(fl), _stream()), "ffsplit_probe_mfma")
    return fl.value


def probe_stream_read(buf, workgroups, scratch):
    """Enqueue one streaming read of buf (a uint8 tensor whose size is a multiple of 16)."""
    _check(lib.ffsplit_probe_stream_read(_ptr(buf), buf.numel() * buf.element_size(), workgroups, _ptr(scratch), _stream()),
           "ffsplit_probe_stream_read")


def split_export(desc, split, what):
    """Test hook of the quantised kinds: (q int8 [n, d_model], scale bits uint16 as int16 tensor
    [n, d_model/group]); what 0..2 = remainder W1 / Wg / W2 (n = m), 3..5 = heavy (W3H8 only, n = k)."""
    n = desc.k if what >= 3 else desc.d_ff - desc.k
    q = torch.empty((n, desc.d_model), dtype=torch.int8, device=split.device)
    s = torch.empty((n, desc.d_model // desc.group), dtype=torch.int16, device=split.device)
    rc = lib.ffsplit_split_export(ctypes.byref(desc), _ptr(split), what, _ptr(q), _ptr(s), _stream())
    _check(rc, "ffsplit_split_export")
    return q, s
