"""Layer norm, linear layers and 8-bit activation copies for PyTorch on MI355X.

The forward and backward passes of a transformer's feed-forward block on the
library's kernels (the training operators of include/mfac.h), for models trained
with the optimizer of this package. Its window of gradients takes most of a
card's memory; with ``copy8=True`` a layer keeps what its backward pass needs
as 8-bit copies, about half of the bytes of 16-bit activations.

Three levels:

* ``layer_norm_forward``, ``layer_norm_backward``, ``linear_forward``,
  ``linear_backward``, ``act_backward``, ``pack8``, ``unpack8``: the passes
  themselves, on tensors and ``Packed8`` copies;
* ``layer_norm``, ``linear``, ``feed_forward``: the same with autograd;
* ``LayerNorm``, ``Linear``, ``FeedForward``: modules.

Data is float32, bfloat16 or float16 on one CUDA device; leading dimensions are
rows, the last one needs unit stride (others are copied first). Layer norm's
parameters and biases are float32 or of the data's type. In the autograd
functions a float32 weight may come with 16-bit data: it is rounded for the
products at every call, and its gradient comes back in float32 (a weight that is
used again and again without training is better handed over in 16 bits). Where
gradients are off, or no input needs one, nothing is kept. Calls run on the current
stream of the data's device, with workspaces from torch's allocator.
"""

import torch
from torch.autograd.function import once_differentiable

from . import _binding as B
from ._binding import MfacError, load  # noqa: F401

_TYPES = {torch.float32: B.MFAC_F32, torch.bfloat16: B.MFAC_BF16, torch.float16: B.MFAC_F16}
ACTIVATIONS = {"none": B.MFAC_ACT_NONE, "relu": B.MFAC_ACT_RELU, "gelu": B.MFAC_ACT_GELU,
               "gelu_tanh": B.MFAC_ACT_GELU_TANH, "silu": B.MFAC_ACT_SILU}
GROUP = 32


class Packed8:
    """The 8-bit copy of a matrix: ``q`` (rows x cols int8), ``s`` (rows x ceil(cols / 32)
    uint8). Row r, column c stands for q[r, c] * 2 ** (s[r, c // 32] - 127), and for NaN
    where s is 255."""

    def __init__(self, q, s):
        if q.dtype != torch.int8 or s.dtype != torch.uint8 or q.dim() != 2 or s.dim() != 2:
            raise ValueError("Packed8: q is a 2-d int8 tensor and s a 2-d uint8 tensor")
        if s.shape != (q.shape[0], -(-q.shape[1] // GROUP)) or s.device != q.device:
            raise ValueError("Packed8: s has one byte for each 32 columns of q, on its device")
        if (q.shape[1] > 1 and q.stride(1) != 1) or (q.shape[0] > 1 and q.stride(0) < q.shape[1]):
            raise ValueError("Packed8: q's rows have unit stride and do not overlap")
        self.q, self.s = q, s if s.is_contiguous() else s.contiguous()

    @staticmethod
    def empty(rows, cols, device):
        """Room for a copy; rows of q lie a multiple of 32 bytes apart."""
        groups = -(-cols // GROUP)
        q = torch.empty((rows, groups * GROUP), dtype=torch.int8, device=device)
        p = Packed8.__new__(Packed8)   # nothing to check
        p.q = q if cols == groups * GROUP else q[:, :cols]
        p.s = torch.empty((rows, groups), dtype=torch.uint8, device=device)
        return p

    @property
    def shape(self):
        return self.q.shape

    @property
    def device(self):
        return self.q.device

    @property
    def nbytes(self):
        return self.q.shape[0] * (self._ld() + self.s.shape[1])

    def _ld(self):
        return max(self.q.stride(0), self.q.shape[1])

    def _args(self):
        return self.q.data_ptr(), self._ld(), self.s.data_ptr()


_NO_COPY = (None, 0, None)


# ---------------------------------------------------------------- marshalling
def _type(t, what):
    try:
        return _TYPES[t.dtype]
    except KeyError:
        raise ValueError(f"{what}: float32, bfloat16 or float16, not {t.dtype}") from None


def _rows(t, what):
    """t as a matrix of rows with unit stride (a copy where it has none)."""
    if t.dim() == 2 and t.is_cuda:   # most calls: nothing to do
        (rows, cols), (ld, unit) = t.shape, t.stride()
        if unit == 1 and ld >= cols > 0:
            return t
    if not t.is_cuda:
        raise ValueError(f"{what}: a CUDA tensor, not one on {t.device}")
    if t.dim() == 0 or t.shape[-1] == 0:
        raise ValueError(f"{what}: at least one dimension, the last of size 1 or more")
    if t.dim() != 2:
        t = t.reshape(-1, t.shape[-1])
    if (t.shape[1] > 1 and t.stride(1) != 1) or (t.shape[0] > 1 and t.stride(0) < t.shape[1]):
        t = t.contiguous()
    return t


def _ld(t):
    return max(t.stride(0), t.shape[1])


def _mat(t):
    return (None, 0) if t is None else (t.data_ptr(), _ld(t))


def _ptr(t):
    return None if t is None else t.data_ptr()


def _same(what, t, like, shape):
    if t.dtype is not like.dtype or t.shape != shape or t.device != like.device:
        raise ValueError(f"{what}: {tuple(shape)} {like.dtype} on {like.device}, not {tuple(t.shape)} {t.dtype} on "
                         f"{t.device}")


def _param(what, p, data, n):
    """A parameter vector of n values in float32 or the data's type."""
    d = p.dtype
    if (d is not torch.float32 and d is not data.dtype) or p.shape != (n,) or p.device != data.device:
        raise ValueError(f"{what}: {n} values in float32 or {data.dtype} on {data.device}, not {tuple(p.shape)} "
                         f"{p.dtype} on {p.device}")
    return p.contiguous()


def _weight(w):
    if w.dim() != 2:
        raise ValueError(f"linear: weight is a matrix (cout x cin), not {tuple(w.shape)}")
    return _rows(w, "linear: weight")


def _act(name):
    try:
        return ACTIVATIONS[name]
    except KeyError:
        raise ValueError(f"act: one of {', '.join(ACTIVATIONS)}, not {name!r}") from None


# torch.cuda.current_device and current_stream without the objects they build (2 us a call)
_device, _raw_stream = torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream
_functions = {}


def _function(name):
    fn = _functions.get(name)
    if fn is None:
        fn = _functions[name] = getattr(load(), name)
    return fn


def _call(name, device, *args):
    """The C call of this name on the current stream of `device`."""
    index = device.index
    if index == _device():
        status = _function(name)(*args, _raw_stream(index))
    else:
        with torch.cuda.device(device):
            status = _function(name)(*args, torch.cuda.current_stream(device).cuda_stream)
    if status != B.MFAC_OK:
        raise MfacError(name, status)


def _like(t):
    """Room for a result of t's shape and type, its rows contiguous."""
    return torch.empty_like(t, memory_format=torch.contiguous_format)


def _workspace(nbytes, device):
    """(pointer, bytes, the tensor that holds them)"""
    if nbytes == 0:
        return None, 0, None
    w = torch.empty((nbytes,), dtype=torch.uint8, device=device)
    return w.data_ptr(), nbytes, w


# ---------------------------------------------------------------- 8-bit copies
def pack8(x):
    """The 8-bit copy of x (leading dimensions are rows)."""
    x = _rows(x, "pack8")
    p = Packed8.empty(x.shape[0], x.shape[1], x.device)
    _call("mfac_pack8", x.device, _type(x, "pack8"), *x.shape, *_mat(x), *p._args())
    return p


def unpack8(p, dtype=torch.float32):
    """The values a copy stands for (rows x cols) in float32, bfloat16 or float16."""
    y = torch.empty(p.shape, dtype=dtype, device=p.device)
    if y.shape[1] == 0:
        return y
    _call("mfac_unpack8", p.device, _type(y, "unpack8"), *p.shape, *p._args(), *_mat(y))
    return y


# ---------------------------------------------------------------- layer norm
def layer_norm_forward(x, weight=None, bias=None, eps=1e-5, pack=False):
    """(y, mean, rstd) over the last dimension; with ``pack`` (y, the 8-bit copy of
    (x - mean) * rstd, rstd). mean and rstd are float32, one for each row."""
    x2 = _rows(x, "layer_norm: x")
    rows, cols = x2.shape
    w, b, wt = _norm_params(weight, bias, x2)
    y = _like(x)
    rstd = torch.empty((rows,), dtype=torch.float32, device=x.device)
    mean = None if pack else torch.empty_like(rstd)
    p = Packed8.empty(rows, cols, x.device) if pack else None
    _call("mfac_layer_norm", x.device, _type(x2, "layer_norm: x"), wt, rows, cols, *_mat(x2), _ptr(w), _ptr(b),
          float(eps), y.data_ptr(), cols, _ptr(mean), rstd.data_ptr(), *(p._args() if pack else _NO_COPY))
    return (y, p, rstd) if pack else (y, mean, rstd)


def _norm_params(weight, bias, x):
    w = None if weight is None else _param("layer_norm: weight", weight, x, x.shape[1])
    b = None if bias is None else _param("layer_norm: bias", bias, x, x.shape[1])
    if w is not None and b is not None and w.dtype != b.dtype:
        raise ValueError("layer_norm: weight and bias of one type")
    like = w if w is not None else b
    return w, b, _TYPES[torch.float32 if like is None else like.dtype]


def layer_norm_backward(dy, x, mean, rstd, weight=None, add=None, params=True):
    """(dx, dweight, dbias) from what the forward pass took or kept: x and mean, or the
    8-bit copy (a Packed8 as x, mean None). ``add`` (like dy) is added to dx. The
    parameters' gradients have the weight's type (float32 without one), and are
    None with ``params=False``."""
    dy2 = _rows(dy, "layer_norm: dy")
    rows, cols = dy2.shape
    w, _, wt = _norm_params(weight, None, dy2)
    if isinstance(x, Packed8):
        if x.shape != dy2.shape or x.device != dy2.device or mean is not None:
            raise ValueError("layer_norm: an 8-bit copy of dy's shape, and no mean")
        xm, packed = (None, 0), x._args()
    else:
        x2 = _rows(x, "layer_norm: x")
        _same("layer_norm: x", x2, dy2, dy2.shape)
        xm, packed = _mat(x2), _NO_COPY
    for what, t in (("mean", mean), ("rstd", rstd)):
        if t is not None and (t.dtype != torch.float32 or t.numel() != rows or not t.is_contiguous()
                              or t.device != dy2.device):
            raise ValueError(f"layer_norm: {what} is a contiguous float32 tensor, one value for each row")
    if rstd is None or (mean is None and not isinstance(x, Packed8)):
        raise ValueError("layer_norm: needs mean (without an 8-bit copy) and rstd")
    if add is not None:
        add = _rows(add, "layer_norm: add")
        _same("layer_norm: add", add, dy2, dy2.shape)
    dx = _like(dy)
    dw = db = None
    ws = (None, 0, None)
    if params:
        # one allocation for both, whose storage they share
        grads = torch.empty((2, cols), dtype=torch.float32 if w is None else w.dtype, device=dy.device)
        dw, db = grads.unbind(0)
        ws = _workspace(_function("mfac_layer_norm_bwd_workspace_bytes")(rows, cols), dy.device)
    _call("mfac_layer_norm_bwd", dy.device, _type(dy2, "layer_norm: dy"), wt, rows, cols, *_mat(dy2), *xm, _ptr(mean),
          rstd.data_ptr(), *packed, _ptr(w), *_mat(add), dx.data_ptr(), cols, _ptr(dw), _ptr(db), ws[0], ws[1])
    return dx, dw, db


# ---------------------------------------------------------------- linear layers
def linear_forward(x, weight, bias=None, act="none", residual=None, keep=None):
    """y = act(x weight^T + bias) + residual. ``keep``: also return the pre-activation for
    the backward pass, "z" as a tensor or "pack8" as its 8-bit copy."""
    a = _act(act)
    x2 = _rows(x, "linear: x")
    rows, cin = x2.shape
    w = _weight(weight)
    cout = w.shape[0]
    _same("linear: weight", w, x2, (cout, cin))
    b = None if bias is None else _param("linear: bias", bias, x2, cout)
    if keep not in (None, "z", "pack8"):
        raise ValueError(f"linear: keep is None, 'z' or 'pack8', not {keep!r}")
    shape = x.shape[:-1] + (cout,)
    if residual is not None:
        residual = _rows(residual, "linear: residual")
        _same("linear: residual", residual, x2, (rows, cout))
    y = x.new_empty(shape)
    z = x.new_empty(shape) if keep == "z" else None
    p = Packed8.empty(rows, cout, x.device) if keep == "pack8" else None
    t = _type(x2, "linear: x")
    xm, wm = _mat(x2), _mat(w)
    ws = _workspace(_function("mfac_linear_workspace_bytes")(t, rows, cin, cout, *xm, *wm), x.device)
    _call("mfac_linear", x.device, t, t if b is None else _TYPES[b.dtype], a, rows, cin, cout, *xm, *wm, _ptr(b),
          *_mat(residual), y.data_ptr(), cout, _ptr(z), cout, *(_NO_COPY if p is None else p._args()), ws[0], ws[1])
    return y if keep is None else (y, z if keep == "z" else p)


def act_backward(dy, z=None, act="none", want_a=False, want_db=True):
    """(dz, a, db): dz = dy act'(z) in dy's type, a = act(z) (``want_a``, else None), db the
    column sums of dy act'(z) in float32 (``want_db``, else None). z is a tensor or a
    Packed8; with act "none" there is no z, and dz is dy."""
    code = _act(act)
    dy2 = _rows(dy, "act: dy")
    rows, cols = dy2.shape
    if (z is None) != (code == B.MFAC_ACT_NONE) or (want_a and z is None):
        raise ValueError("act: z goes with an activation")
    zm, packed = (None, 0), _NO_COPY
    if isinstance(z, Packed8):
        if z.shape != dy2.shape or z.device != dy2.device:
            raise ValueError("act: an 8-bit copy of dy's shape")
        packed = z._args()
    elif z is not None:
        z = _rows(z, "act: z")
        _same("act: z", z, dy2, dy2.shape)
        zm = _mat(z)
    dz = dy if z is None else _like(dy)
    a = _like(dy) if want_a else None
    db = torch.empty(cols, dtype=torch.float32, device=dy.device) if want_db else None
    if z is None and not want_db:
        return dz, None, None
    ws = _workspace(_function("mfac_act_bwd_workspace_bytes")(rows, cols) if want_db else 0, dy.device)
    _call("mfac_act_bwd", dy.device, _type(dy2, "act: dy"), code, rows, cols, *_mat(dy2), *zm, *packed,
          None if z is None else dz.data_ptr(), cols, _ptr(a), cols, _ptr(db), ws[0], ws[1])
    return dz, a, db


def linear_backward_input(dz, weight, add=None):
    """dx = dz weight + add."""
    dz2 = _rows(dz, "linear: dz")
    rows, cout = dz2.shape
    w = _weight(weight)
    cin = w.shape[1]
    _same("linear: weight", w, dz2, (cout, cin))
    if add is not None:
        add = _rows(add, "linear: add")
        _same("linear: add", add, dz2, (rows, cin))
    dx = dz.new_empty(dz.shape[:-1] + (cin,))
    t = _type(dz2, "linear: dz")
    zm, wm = _mat(dz2), _mat(w)
    ws = _workspace(_function("mfac_linear_bwd_input_workspace_bytes")(t, rows, cin, cout, *zm, *wm), dz.device)
    _call("mfac_linear_bwd_input", dz.device, t, rows, cin, cout, *zm, *wm, *_mat(add), dx.data_ptr(), cin, ws[0],
          ws[1])
    return dx


def linear_backward_weight(dz, x, affine=None, db=None, grad_dtype=None):
    """dW = dz^T x (cout x cin) in ``grad_dtype`` (float32 or dz's type, the default). x is a
    tensor or a Packed8. ``affine`` = (gamma, beta), float32: the layer's input was
    gamma * x + beta; db, the column sums of dz in float32, is then needed."""
    dz2 = _rows(dz, "linear: dz")
    rows, cout = dz2.shape
    xm, packed = (None, 0), _NO_COPY
    if isinstance(x, Packed8):
        packed = x._args()
    else:
        x = _rows(x, "linear: x")
        _same("linear: x", x, dz2, (rows, x.shape[1]))
        xm = _mat(x)
    if x.shape[0] != rows or x.device != dz2.device:
        raise ValueError("linear: x and dz have the same rows, on one device")
    cin = x.shape[1]
    grad_dtype = dz.dtype if grad_dtype is None else grad_dtype
    if grad_dtype not in (torch.float32, dz.dtype):
        raise ValueError(f"linear: grad_dtype is float32 or {dz.dtype}")
    gamma = beta = None
    if affine is not None:
        gamma, beta = (_param("linear: affine", v.float(), dz2, cin) for v in affine)
        if db is None or db.dtype != torch.float32:
            raise ValueError("linear: affine needs db, the column sums of dz in float32")
        db = _param("linear: db", db, dz2, cout)
    dw = torch.empty((cout, cin), dtype=grad_dtype, device=dz.device)
    t = _type(dz2, "linear: dz")
    zm = _mat(dz2)
    ws = _workspace(_function("mfac_linear_bwd_weight_workspace_bytes")(t, rows, cin, cout, *zm, *xm), dz.device)
    _call("mfac_linear_bwd_weight", dz.device, t, _TYPES[grad_dtype], rows, cin, cout, *zm, *xm, *packed, _ptr(gamma),
          _ptr(beta), _ptr(db) if affine is not None else None, dw.data_ptr(), cin, ws[0], ws[1])
    return dw


def linear_backward(dy, x, weight, z=None, act="none", affine=None, grad_dtype=None, need=(True, True, True)):
    """(dx, dweight, dbias) of y = act(x weight^T + bias) from dy, the layer's input x and the
    pre-activation z (tensors or Packed8; z only with an activation). ``affine``: see
    linear_backward_weight; dx is then the gradient of gamma * x + beta. dbias is float32.
    ``need``: which of the three to form; the others are None."""
    need_x, need_w, need_b = need
    if not (need_x or need_w or need_b):   # z may be absent then
        return None, None, None
    dz, _, db = act_backward(dy, z, act, want_db=need_b or (need_w and affine is not None))
    dx = linear_backward_input(dz, weight) if need_x else None
    dw = linear_backward_weight(dz, x, affine, db, grad_dtype) if need_w else None
    return dx, dw, db if need_b else None


# ---------------------------------------------------------------- autograd
def _keep(ctx, **values):
    """Saves tensors and copies for the backward pass, None among them."""
    ctx.names, tensors = [], []
    for name, v in values.items():
        if isinstance(v, Packed8):
            ctx.names.append((name, 2))
            tensors += [v.q, v.s]
        else:
            ctx.names.append((name, 1))
            tensors.append(v)
    ctx.save_for_backward(*tensors)


def _kept(ctx):
    got, it = {}, iter(ctx.saved_tensors)
    for name, n in ctx.names:
        got[name] = next(it) if n == 1 else Packed8(next(it), next(it))
    return got


def _to(t, dtype):
    return None if t is None else t.to(dtype)


def _grad_dtype(param, data):
    """The type that a weight's gradient is formed in: its own, or float32 where the data has neither."""
    return param if param == data.dtype else torch.float32


# `grad`, the last argument of each: torch.is_grad_enabled() where it was called. Within forward it is always
# off, and needs_input_grad says what the inputs ask for whether it is on or not.
class _LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, eps, copy8, grad):
        if not (grad and any(ctx.needs_input_grad)):
            return layer_norm_forward(x, weight, bias, eps)[0]
        y, kept, rstd = layer_norm_forward(x, weight, bias, eps, pack=copy8)
        ctx.types = tuple(None if p is None else p.dtype for p in (weight, bias))
        if copy8:
            _keep(ctx, x=kept, mean=None, rstd=rstd, w=weight)
        else:
            _keep(ctx, x=x, mean=kept, rstd=rstd, w=weight)
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        k = _kept(ctx)
        need = ctx.needs_input_grad
        dx, dw, db = layer_norm_backward(dy, k["x"], k["mean"], k["rstd"], k["w"], params=need[1] or need[2])
        return (dx, _to(dw, ctx.types[0]) if need[1] else None, _to(db, ctx.types[1]) if need[2] else None, None, None,
                None)


class _Linear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, act, residual, copy8, grad):
        w = weight.to(x.dtype)
        need = [grad and n for n in ctx.needs_input_grad[:3]]
        keep = None if act == "none" or not any(need) else "pack8" if copy8 else "z"
        out = linear_forward(x, w, bias, act, residual, keep)
        y, z = (out, None) if keep is None else out
        ctx.act, ctx.wdtype, ctx.bdtype = act, weight.dtype, None if bias is None else bias.dtype
        ctx.rshape = None if residual is None else residual.shape   # its rows may lie in other dimensions than y's
        _keep(ctx, x=(pack8(x) if copy8 else x) if need[1] else None, w=w if need[0] else None, z=z)
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        k = _kept(ctx)
        need = ctx.needs_input_grad
        dx, dw, db = linear_backward(dy, k["x"], k["w"], k["z"], ctx.act, grad_dtype=_grad_dtype(ctx.wdtype, dy),
                                     need=need[:3])
        dres = dy.reshape(ctx.rshape) if need[4] else None
        return dx, _to(dw, ctx.wdtype), _to(db, ctx.bdtype), None, dres, None, None


class _FeedForward(torch.autograd.Function):
    """y = x + act(LN(x) W1^T + b1) W2^T + b2. Kept with copy8: the 8-bit copies of the
    normalised x, which serves both layer norm's backward pass and W1's gradient, and of
    the pre-activation, from which act(z) is formed again for W2's gradient."""

    @staticmethod
    def forward(ctx, x, lw, lb, w1, b1, w2, b2, act, eps, copy8, grad):
        c1, c2 = w1.to(x.dtype), w2.to(x.dtype)
        if not (grad and any(ctx.needs_input_grad)):
            a = linear_forward(layer_norm_forward(x, lw, lb, eps)[0], c1, b1, act)
            return linear_forward(a, c2, b2, residual=x)
        need = ctx.needs_input_grad
        norm, hidden = any(need[:3]), any(need[:5])   # whether a gradient passes through the norm, or through act
        pack = copy8 and (norm or need[3])
        h, kept, rstd = layer_norm_forward(x, lw, lb, eps, pack=pack)
        keep = None if not (hidden or need[5]) else "pack8" if copy8 else "z"
        out = linear_forward(h, c1, b1, act, keep=keep)
        a, z = (out, None) if keep is None else out
        y = linear_forward(a, c2, b2, residual=x)
        ctx.act, ctx.copy8, ctx.types = act, copy8, tuple(p.dtype for p in (lw, lb, w1, b1, w2, b2))
        _keep(ctx, x=kept if pack else x if norm else None, mean=kept if norm and not pack else None,
              rstd=rstd if norm else None, h=h if need[3] and not copy8 else None, z=z, lw=lw if norm or pack else None,
              lb=lb if pack else None, c1=c1 if norm else None, c2=c2 if hidden else None)
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        k = _kept(ctx)
        t, z = ctx.types, k["z"]
        nx, nlw, nlb, nw1, nb1, nw2, nb2 = ctx.needs_input_grad[:7]
        norm, hidden = nx or nlw or nlb, nx or nlw or nlb or nw1 or nb1
        dx = dlw = dlb = dw1 = db1 = dw2 = db2 = None
        if nb2:
            _, _, db2 = act_backward(dy)
        if hidden or nw2:
            # where w2 alone asks for act(z), any tensor of its shape will do for the gradient that is not looked at
            da = linear_backward_input(dy, k["c2"]) if hidden else unpack8(z, dy.dtype) if ctx.copy8 else z
            dz, a, db1 = act_backward(da, z, ctx.act, want_a=nw2, want_db=nb1 or (nw1 and ctx.copy8))
            if nw2:
                dw2 = linear_backward_weight(dy, a, grad_dtype=_grad_dtype(t[4], dy))
            del a, da
        if nw1:
            if ctx.copy8:
                dw1 = linear_backward_weight(dz, k["x"], (k["lw"], k["lb"]), db1, _grad_dtype(t[2], dy))
            else:
                dw1 = linear_backward_weight(dz, k["h"], grad_dtype=_grad_dtype(t[2], dy))
        if norm:
            dh = linear_backward_input(dz, k["c1"])
            dx, dlw, dlb = layer_norm_backward(dh, k["x"], k["mean"], k["rstd"], k["lw"], add=dy, params=nlw or nlb)
        return (dx, _to(dlw, t[0]), _to(dlb, t[1]), _to(dw1, t[2]), _to(db1, t[3]), _to(dw2, t[4]), _to(db2, t[5]),
                None, None, None, None)


def layer_norm(x, weight=None, bias=None, eps=1e-5, copy8=False):
    """Layer norm over the last dimension, differentiable. copy8: keep the normalised x in
    8 bits for the backward pass instead of x."""
    return _LayerNorm.apply(x, weight, bias, eps, copy8, torch.is_grad_enabled())


def linear(x, weight, bias=None, act="none", residual=None, copy8=False):
    """act(x weight^T + bias) + residual, differentiable. copy8: keep x and the
    pre-activation in 8 bits for the backward pass."""
    _act(act)
    return _Linear.apply(x, weight, bias, act, residual, copy8, torch.is_grad_enabled())


def feed_forward(x, ln_weight, ln_bias, w1, b1, w2, b2, act="gelu", eps=1e-5, copy8=False):
    """x + act(layer_norm(x) w1^T + b1) w2^T + b2, differentiable. copy8: what the backward
    pass needs is kept in 8 bits."""
    if _act(act) == B.MFAC_ACT_NONE:
        raise ValueError("feed_forward: needs an activation")
    if any(p is None for p in (ln_weight, ln_bias, w1, b1, w2, b2)):
        raise ValueError("feed_forward: needs its six parameters")
    return _FeedForward.apply(x, ln_weight, ln_bias, w1, b1, w2, b2, act, eps, copy8, torch.is_grad_enabled())


# ---------------------------------------------------------------- modules
class LayerNorm(torch.nn.Module):
    """Layer norm over the last dimension, of size `dim`."""

    def __init__(self, dim, eps=1e-5, copy8=False, device=None):
        super().__init__()
        self.eps, self.copy8 = eps, copy8
        self.weight = torch.nn.Parameter(torch.ones(dim, device=device))
        self.bias = torch.nn.Parameter(torch.zeros(dim, device=device))

    def forward(self, x):
        return layer_norm(x, self.weight, self.bias, self.eps, self.copy8)


class Linear(torch.nn.Module):
    """act(x W^T + b) + residual; weights uniform within 1 / sqrt(cin)."""

    def __init__(self, cin, cout, bias=True, act="none", copy8=False, device=None):
        super().__init__()
        _act(act)
        self.act, self.copy8 = act, copy8
        r = cin ** -0.5
        self.weight = torch.nn.Parameter(torch.empty(cout, cin, device=device).uniform_(-r, r))
        self.bias = torch.nn.Parameter(torch.empty(cout, device=device).uniform_(-r, r)) if bias else None

    def forward(self, x, residual=None):
        return linear(x, self.weight, self.bias, self.act, residual, self.copy8)


class FeedForward(torch.nn.Module):
    """A transformer's feed-forward block with its norm and skip connection:
    x + act(LN(x) W1^T + b1) W2^T + b2."""

    def __init__(self, dim, hidden, act="gelu", eps=1e-5, copy8=False, device=None):
        super().__init__()
        self.norm = LayerNorm(dim, eps, device=device)
        self.up = Linear(dim, hidden, act=act, device=device)
        self.down = Linear(hidden, dim, device=device)
        self.copy8 = copy8

    def forward(self, x):
        return feed_forward(x, self.norm.weight, self.norm.bias, self.up.weight, self.up.bias, self.down.weight,
                            self.down.bias, self.up.act, self.norm.eps, self.copy8)
