"""Layers and losses of all learners at once: ctypes binding of include/psgd_layers.h, argument marshalling only.

What produces the gradients G of `psgd.mix_step`.  Activations are [n, t, c] device tensors (t tokens of each of n learners), parameters are
views of the rows of an [n, d] tensor like X, gradients of parameters are written into views of the rows of another, like G:

    w = X.as_strided((n, out, inn), (X.stride(0), inn, 1), offset)      # learner i's matrix lies in row i
    layers.linear(x, w, y, bias=X[:, b0:b1], act="gelu", z=z)
    layers.linear_grad(dy, x, w, dx=dx, dw=dw, db=db, act="gelu", z=z)

Matrices have the type of the activations: in bf16 w and b are views of a bf16 copy of X, made after each step (`Xb.copy_(X)`), and dw and db of a bf16 G.
A single model is n = 1.  Every operand has unit stride along its last dimension and any strides along the others (0 shares an input between
learners); outputs are the caller's tensors.  Work is enqueued on `stream` (None: torch's current stream).  A workspace that a call needs is
taken from torch's allocator on that stream, or is the caller's `workspace` (a contiguous uint8 tensor of at least the bytes that the
function's *_workspace says).  There is no fallback: what the library refuses raises `psgd.PsgdError`, a tensor that is not what a call
takes raises ValueError.

Calls that are plainly in order take the short way of the _call extension, as psgd.py's do.
"""
import ctypes

from . import psgd

F32, BF16, I32 = 0, 1, 2
ACTS = {"none": 0, "relu": 1, "gelu": 2, "silu": 3}
MAX_TOP, MAX_SLOTS = 64, 1024

EXPORTS = ("psgd_layer_norm", "psgd_layer_norm_grad", "psgd_layer_norm_grad_workspace", "psgd_linear", "psgd_linear_workspace",
           "psgd_linear_grad", "psgd_linear_grad_workspace", "psgd_token_logprobs", "psgd_distill")


class View(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("learner", ctypes.c_int64), ("row", ctypes.c_int64), ("type", ctypes.c_int32)]


_lib = None
_types = None
_ext = None              # the extension, once bound to the library's functions


def load():
    """The library of psgd.load() with these functions' signatures declared."""
    global _lib
    lib = psgd.load()
    if _lib is lib:
        return lib
    view, vp, i32, i64, f32, size = ctypes.POINTER(View), ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t
    shape3, shape4, work = [i32, i64, i64], [i32, i64, i64, i64], [vp, size]
    signatures = {
        "psgd_layer_norm": (i32, [view] * 4 + [vp, vp] + shape3 + [f32, vp]),
        "psgd_layer_norm_grad": (i32, [view] * 3 + [vp, vp] + [view] * 4 + shape3 + work + [vp]),
        "psgd_layer_norm_grad_workspace": (size, shape3),
        "psgd_linear": (i32, [view] * 6 + [i32] + shape4 + work + [vp]),
        "psgd_linear_workspace": (size, [view] * 2 + shape4),
        "psgd_linear_grad": (i32, [view] * 7 + [i32] + shape4 + work + [vp]),
        "psgd_linear_grad_workspace": (size, [view] * 6 + [i32] + shape4),
        "psgd_token_logprobs": (i32, [view] * 2 + [vp] * 4 + [i32] + shape3 + [vp]),
        "psgd_distill": (i32, [view] * 3 + [vp, vp, view, f32, i32] + shape3 + [vp]),
    }
    for name, (res, args) in signatures.items():
        fn = getattr(lib, name)
        fn.restype, fn.argtypes = res, args
    _lib = lib
    _bind()
    return lib


def _bind():
    """Hand the extension, if psgd.py has it, the addresses of the loaded library's functions."""
    global _ext
    _ext = None
    if psgd._call is not None and hasattr(psgd._call, "bind_layers"):
        psgd._call.bind_layers(*(ctypes.cast(getattr(_lib, name), ctypes.c_void_p).value for name in EXPORTS))
        _ext = psgd._call


def _short(name, *args):
    """Whether the short way has made the call."""
    if _ext is None or _lib is not psgd._lib:
        if _lib is None or psgd._call is None or not hasattr(psgd._call, "bind_layers"):
            return False
        load()                   # psgd may have loaded the library again
        if _ext is None:
            _bind()
    return psgd._answered(getattr(_ext, name)(*args))


def _view(what, t, shape):
    """The operand `t` of the given shape (None: any size) as the library takes it.  No tensor: no operand."""
    global _types
    if t is None:
        return None
    import torch
    if _types is None:
        _types = {torch.float32: F32, torch.bfloat16: BF16, torch.int32: I32}
    if not isinstance(t, torch.Tensor):
        raise ValueError("%s must be a tensor" % what)
    got, strides = tuple(t.shape), t.stride()
    if len(got) != len(shape) or any(w is not None and g != w for g, w in zip(got, shape)):
        raise ValueError("%s must be of shape %s, not %s" % (what, list(shape), list(got)))
    kind = _types.get(t.dtype)
    if kind is None:
        raise ValueError("%s must be float32, bfloat16 or int32" % what)
    if got[-1] > 1 and strides[-1] != 1:
        raise ValueError("%s must have unit stride along its last dimension" % what)
    return View(t.data_ptr(), strides[0] if got[0] > 1 else 0, strides[1] if len(got) == 3 and got[1] > 1 else 0, kind)


def _vector(what, t, numel, dtype):
    """The address of a contiguous tensor of `numel` elements (None: NULL)."""
    if t is None:
        return None
    import torch
    if not isinstance(t, torch.Tensor) or t.dtype != dtype or t.numel() != numel or not t.is_contiguous():
        raise ValueError("%s must be a contiguous %s tensor of %d elements" % (what, dtype, numel))
    return t.data_ptr()


def _shape(what, t, dims):
    import torch
    if not isinstance(t, torch.Tensor) or t.dim() != dims:
        raise ValueError("%s must be a tensor of %d dimensions" % (what, dims))
    return tuple(t.shape)


def _workspace(given, need, stream):
    """(tensor to keep until the call has returned, its address, its bytes)."""
    import torch
    if given is not None:
        if not isinstance(given, torch.Tensor) or given.dtype != torch.uint8 or not given.is_contiguous():
            raise ValueError("workspace must be a contiguous uint8 tensor")
        psgd._on_current_device(given)
        return given, given.data_ptr(), given.numel()
    if not need:
        return None, None, 0
    if stream is None:
        room = torch.empty(need, dtype=torch.uint8, device="cuda")
    else:
        with torch.cuda.stream(stream):
            room = torch.empty(need, dtype=torch.uint8, device="cuda")
    return room, room.data_ptr(), need


def layer_norm(x, gain, bias, y, eps=1e-5, mean=None, rstd=None, stream=None):
    """Enqueue y = (x - m) r gain + bias over the last dimension; m and r to mean and rstd ([n, t] float32, both or neither).
    x, y [n, t, c] of one type (y may be x), gain and bias [n, c] of one type (bias may be None)."""
    if _short("layer_norm", x, gain, bias, y, eps, mean, rstd, stream):
        return
    import torch
    n, t, c = _shape("x", x, 3)
    vx, vg, vb, vy = _view("x", x, (n, t, c)), _view("gain", gain, (n, c)), _view("bias", bias, (n, c)), _view("y", y, (n, t, c))
    pm, pr = _vector("mean", mean, n * t, torch.float32), _vector("rstd", rstd, n * t, torch.float32)
    psgd._on_current_device(x, gain, bias, y, mean, rstd)
    psgd._check(load().psgd_layer_norm(vx, vg, vb, vy, pm, pr, n, t, c, float(eps), psgd._stream_handle(stream)))


def layer_norm_grad_workspace(n, t, c):
    return load().psgd_layer_norm_grad_workspace(n, t, c)


def layer_norm_grad(dy, x, gain, mean, rstd, dx, dgain=None, dbias=None, add=None, workspace=None, stream=None):
    """Enqueue the backward pass of layer_norm: dx (plus `add`, the gradient that reaches x by another way), dgain and dbias from dy.
    dx may be dy or add; dgain and dbias [n, c] are float32 or bfloat16 alike, whatever x and gain are."""
    if workspace is None and _short("layer_norm_grad", dy, x, gain, mean, rstd, dx, dgain, dbias, add, stream):
        return
    import torch
    n, t, c = _shape("x", x, 3)
    vdy, vx, vg = _view("dy", dy, (n, t, c)), _view("x", x, (n, t, c)), _view("gain", gain, (n, c))
    pm, pr = _vector("mean", mean, n * t, torch.float32), _vector("rstd", rstd, n * t, torch.float32)
    va, vdx = _view("add", add, (n, t, c)), _view("dx", dx, (n, t, c))
    vdg, vdb = _view("dgain", dgain, (n, c)), _view("dbias", dbias, (n, c))
    psgd._on_current_device(dy, x, gain, mean, rstd, dx, dgain, dbias, add)
    lib = load()
    need = lib.psgd_layer_norm_grad_workspace(n, t, c) if vdg or vdb else 0
    room, pw, bw = _workspace(workspace, need, stream)
    psgd._check(lib.psgd_layer_norm_grad(vdy, vx, vg, pm, pr, va, vdx, vdg, vdb, n, t, c, pw, bw, psgd._stream_handle(stream)))


def _act(act):
    if act not in ACTS:
        raise ValueError("act must be one of %s" % ", ".join(ACTS))
    return ACTS[act]


def linear(x, w, y, bias=None, act="none", residual=None, z=None, workspace=None, stream=None):
    """Enqueue z = x w' + bias, y = act(z) + residual for every learner: x [n, t, in], w [n, out, in], bias [n, out], y, residual and z
    [n, t, out], all of one type.  z is written where it is given (linear_grad wants it unless act is "none"); residual may be y."""
    a = _act(act)
    if workspace is None and _short("linear", x, w, y, bias, a, residual, z, stream):
        return
    n, t, i = _shape("x", x, 3)
    o = _shape("w", w, 3)[1]
    vx, vw, vb = _view("x", x, (n, t, i)), _view("w", w, (n, o, i)), _view("bias", bias, (n, o))
    vr, vy, vz = _view("residual", residual, (n, t, o)), _view("y", y, (n, t, o)), _view("z", z, (n, t, o))
    psgd._on_current_device(x, w, bias, residual, y, z)
    lib = load()
    room, pw, bw = _workspace(workspace, lib.psgd_linear_workspace(vx, vw, n, t, i, o), stream)
    psgd._check(lib.psgd_linear(vx, vw, vb, vr, vy, vz, a, n, t, i, o, pw, bw, psgd._stream_handle(stream)))


def linear_grad(dy, x, w, dx=None, dw=None, db=None, act="none", z=None, workspace=None, stream=None):
    """Enqueue the backward pass of linear: with dz = dy act'(z), dx = dz w, dw = dz' x, db = sum_t dz, each where it is given."""
    a = _act(act)
    if workspace is None and _short("linear_grad", dy, x, w, dx, dw, db, a, z, stream):
        return
    n, t, i = _shape("x", x, 3)
    o = _shape("w", w, 3)[1]
    vdy, vz, vx, vw = _view("dy", dy, (n, t, o)), _view("z", z, (n, t, o)), _view("x", x, (n, t, i)), _view("w", w, (n, o, i))
    vdx, vdw, vdb = _view("dx", dx, (n, t, i)), _view("dw", dw, (n, o, i)), _view("db", db, (n, o))
    psgd._on_current_device(dy, z, x, w, dx, dw, db)
    lib = load()
    room, pw, bw = _workspace(workspace, lib.psgd_linear_grad_workspace(vdy, vx, vw, vdx, vdw, vdb, a, n, t, i, o), stream)
    psgd._check(lib.psgd_linear_grad(vdy, vz, vx, vw, vdx, vdw, vdb, a, n, t, i, o, pw, bw, psgd._stream_handle(stream)))


def token_logprobs(logits, tokens, logp, entropy=None, top_logp=None, top_idx=None, stream=None):
    """Enqueue log softmax(logits) at `tokens` ([n, t] int32; negative: none given, 0) into logp, each row's entropy, and the k largest log
    probabilities with their columns ([n, t, k] float32 and int32, largest first, equal ones by column)."""
    if _short("token_logprobs", logits, tokens, logp, entropy, top_logp, top_idx, stream):
        return
    import torch
    n, t, v = _shape("logits", logits, 3)
    vl = _view("logits", logits, (n, t, v))
    if _shape("tokens", tokens, 2) != (n, t) or tokens.dtype != torch.int32:
        raise ValueError("tokens must be int32 of shape [%d, %d]" % (n, t))
    vt = View(tokens.data_ptr(), tokens.stride(0) if n > 1 else 0, tokens.stride(1) if t > 1 else 0, I32)
    if (top_logp is None) != (top_idx is None):
        raise ValueError("top_logp and top_idx go together")
    k = _shape("top_idx", top_idx, 3)[2] if top_idx is not None else 0
    pl, pe = _vector("logp", logp, n * t, torch.float32), _vector("entropy", entropy, n * t, torch.float32)
    ptl, pti = _vector("top_logp", top_logp, n * t * k, torch.float32), _vector("top_idx", top_idx, n * t * k, torch.int32)
    psgd._on_current_device(logits, tokens, logp, entropy, top_logp, top_idx)
    psgd._check(load().psgd_token_logprobs(vl, vt, pl, pe, ptl, pti, k, n, t, v, psgd._stream_handle(stream)))


def distill(logits, top_idx, top_logit, loss, tau=1.0, weight=None, dlogits=None, stream=None):
    """Enqueue the distillation loss of every row against a teacher's k top logits, weight tau^2 KL(p || q), into loss ([n, t] float32), and
    where `dlogits` is given the gradient of the logits (it may be `logits`).  top_idx [n, t, k] int32 (negative: no slot), top_logit
    [n, t, k] float32 (logits or log probabilities), weight [n, t] float32 or None."""
    if _short("distill", logits, top_idx, top_logit, loss, tau, weight, dlogits, stream):
        return
    import torch
    n, t, v = _shape("logits", logits, 3)
    k = _shape("top_idx", top_idx, 3)[2]
    vl, vi, vt = _view("logits", logits, (n, t, v)), _view("top_idx", top_idx, (n, t, k)), _view("top_logit", top_logit, (n, t, k))
    vg = _view("dlogits", dlogits, (n, t, v))
    pw, po = _vector("weight", weight, n * t, torch.float32), _vector("loss", loss, n * t, torch.float32)
    psgd._on_current_device(logits, top_idx, top_logit, loss, weight, dlogits)
    psgd._check(load().psgd_distill(vl, vi, vt, pw, po, vg, float(tau), k, n, t, v, psgd._stream_handle(stream)))
