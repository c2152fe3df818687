"""Norms, linear and gated layers, dropout and 8-bit activation copies for PyTorch on MI355X.

The forward and backward passes of a transformer's feed-forward block on the
library's kernels (the training operators of include/mfac.h), for models trained
with the optimizer of this package. Its window of gradients takes most of a
card's memory; with ``copy8=True`` a layer keeps what its backward pass needs
as 8-bit copies, about half of the bytes of 16-bit activations.

Three levels:

* ``layer_norm_forward``, ``layer_norm_backward``, ``linear_forward``,
  ``linear_backward``, ``act_backward``, ``pack8``, ``unpack8``,
  ``gated_linear_forward``, ``gated_linear_backward``,
  ``gated_feed_forward_backward``, ``residual_norm_forward``,
  ``residual_norm_backward``, ``dropout_forward``: the passes themselves, on
  tensors and ``Packed8`` copies;
* ``layer_norm``, ``rms_norm``, ``residual_norm``, ``linear``, ``gated_linear``,
  ``feed_forward``, ``gated_feed_forward``, ``dropout``: the same with autograd;
* ``LayerNorm``, ``RMSNorm``, ``Linear``, ``GatedLinear``, ``FeedForward``,
  ``GatedFeedForward``, ``GatedStack``, ``Dropout``: modules.

Dropout's masks come from a counter-based generator (include/mfac.h) and are never
stored. Where they start, ``at``, is a tensor of two int64 on the device: by default
drawn with torch's generator of the device, so that torch's seed, activation
checkpointing and captured graphs work as with torch's own dropout.

Data is float32, bfloat16 or float16 on one CUDA device; leading dimensions are
rows, the last one needs unit stride (others are copied first). Layer norm's
parameters and biases are float32 or of the data's type. In the autograd
functions a float32 weight may come with 16-bit data: it is rounded for the
products at every call, and its gradient comes back in float32 (a weight that is
used again and again without training is better handed over in 16 bits). Where
gradients are off, or no input needs one, nothing is kept. Calls run on the current
stream of the data's device, with workspaces from torch's allocator.
"""

from typing import NamedTuple, Optional

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


# ---------------------------------------------------------------- gated layers
def _gate_weight(weight, bias, x2):
    w = _weight(weight)
    n, cin = w.shape[0] // 2, x2.shape[1]
    if w.shape[0] % 2 or n == 0:
        raise ValueError(f"gated_linear: weight has the gate's rows and as many of the other projection, not {tuple(w.shape)}")
    _same("gated_linear: weight", w, x2, (2 * n, cin))
    return w, n, None if bias is None else _param("gated_linear: bias", bias, x2, 2 * n)


def gated_linear_forward(x, weight, bias=None, act="silu", keep=None):
    """y = act(x Wg^T + bg) * (x Wu^T + bu) for weight = [Wg; Wu], one matrix of 2 hidden rows, and
    bias = [bg, bu]. ``keep``: also return the pair of pre-activations (gate, other) for the
    backward pass, "z" as tensors (the halves of one) or "pack8" as their 8-bit copies."""
    a = _act(act)
    x2 = _rows(x, "gated_linear: x")
    w, n, b = _gate_weight(weight, bias, x2)
    rows, cin = x2.shape
    if keep not in (None, "z", "pack8"):
        raise ValueError(f"gated_linear: keep is None, 'z' or 'pack8', not {keep!r}")
    y = x.new_empty(x.shape[:-1] + (n,))
    zg = zu = None
    zm, packed = (None, None, 0), (None, None, None, None, 0)
    if keep == "z":
        z = x.new_empty(x.shape[:-1] + (2 * n,))
        zg, zu = z[..., :n], z[..., n:]
        zm = z.data_ptr(), z.data_ptr() + n * z.element_size(), 2 * n
    elif keep == "pack8":
        zg, zu = (Packed8.empty(rows, n, x.device) for _ in range(2))
        packed = zg.q.data_ptr(), zg.s.data_ptr(), zu.q.data_ptr(), zu.s.data_ptr(), zg._ld()
    t = _type(x2, "gated_linear: x")
    xm, wm = _mat(x2), _mat(w)
    ws = _workspace(_function("mfac_gated_linear_workspace_bytes")(t, rows, cin, n, *xm, *wm), x.device)
    _call("mfac_gated_linear", x.device, t, t if b is None else _TYPES[b.dtype], a, rows, cin, n, *xm, *wm, _ptr(b),
          y.data_ptr(), n, *zm, *packed, ws[0], ws[1])
    return y if keep is None else (y, (zg, zu))


def _gate_pair(z, rows, n, like):
    """The arguments of the pre-activations z = (gate, other), and what holds them."""
    try:
        zg, zu = z
    except (TypeError, ValueError):
        raise ValueError("gated: z is the pair (gate, other) of pre-activations") from None
    if isinstance(zg, Packed8) and isinstance(zu, Packed8):
        for v in (zg, zu):
            if v.shape != (rows, n) or v.device != like.device:
                raise ValueError("gated: 8-bit copies of rows x hidden values")
        if rows > 1 and zg._ld() != zu._ld():
            raise ValueError("gated: 8-bit copies whose rows lie equally far apart")
        return (None, None, 0), (zg.q.data_ptr(), zg.s.data_ptr(), zu.q.data_ptr(), zu.s.data_ptr(), zg._ld()), (zg, zu)
    if isinstance(zg, Packed8) or isinstance(zu, Packed8):
        raise ValueError("gated: both pre-activations as tensors, or both as 8-bit copies")
    zg, zu = (_rows(v, "gated: z") for v in (zg, zu))
    for v in (zg, zu):
        _same("gated: z", v, like, (rows, n))
    if rows > 1 and _ld(zg) != _ld(zu):
        zg, zu = zg.contiguous(), zu.contiguous()
    return (zg.data_ptr(), zu.data_ptr(), _ld(zg)), (None, None, None, None, 0), (zg, zu)


def _gate_width(z):
    try:
        return z[0].shape[-1]
    except (TypeError, AttributeError, IndexError):
        raise ValueError("gated: z is the pair (gate, other) of pre-activations") from None


def _gated_backward(dy, x, w1, w2, z, act, affine, grad_dtype, need, behind=True):
    """(dx, dw1, db1, dw2), of a gated layer, or of it and the layer w2 `behind` it (w2 None: dw2 alone is wanted)."""
    code = _act(act)
    dy2 = _rows(dy, "gated: dy")
    rows = dy2.shape[0]
    need_x, need_w1, need_b1, need_w2 = need
    if not any(need):
        return None, None, None, None
    w2m, cout = (None, 0), 0
    n = dy2.shape[1]
    if behind:
        cout = n
        if w2 is not None:
            w2 = _weight(w2)
            n = w2.shape[1]
            _same("gated: w2", w2, dy2, (cout, n))
            w2m = _mat(w2)
        elif need_x or need_w1 or need_b1:
            raise ValueError("gated: only dw2 is formed without w2")
        else:
            n = _gate_width(z)
    zm, packed_z, held = _gate_pair(z, rows, n, dy2)
    xm, packed, cin, gamma, beta, w1m = (None, 0), _NO_COPY, 1, None, None, (None, 0)
    if need_x:
        w1 = _weight(w1)
        cin = w1.shape[1]
        _same("gated: w1", w1, dy2, (2 * n, cin))
        w1m = _mat(w1)
    if need_w1:
        if isinstance(x, Packed8):
            packed = x._args()
        else:
            x = _rows(x, "gated: x")
            _same("gated: x", x, dy2, (rows, x.shape[1]))
            xm = _mat(x)
        if x.shape[0] != rows or x.device != dy2.device or (need_x and x.shape[1] != cin):
            raise ValueError("gated: x has the rows of dy and the columns of w1, on dy's device")
        cin = x.shape[1]
        if affine is not None:
            gamma, beta = (None if v is None else _param("gated: affine", v.float(), dy2, cin) for v in affine)
            if gamma is None:
                raise ValueError("gated: affine is (gamma, beta or None)")
    grad_dtype = dy.dtype if grad_dtype is None else grad_dtype
    if grad_dtype not in (torch.float32, dy.dtype):
        raise ValueError(f"gated: grad_dtype is float32 or {dy.dtype}")
    dx = dy.new_empty(dy.shape[:-1] + (cin,)) if need_x else None
    dw1 = torch.empty((2 * n, cin), dtype=grad_dtype, device=dy.device) if need_w1 else None
    db1 = torch.empty(2 * n, dtype=torch.float32, device=dy.device) if need_b1 else None
    dw2 = torch.empty((cout, n), dtype=grad_dtype, device=dy.device) if need_w2 else None
    t, gt = _type(dy2, "gated: dy"), _TYPES[grad_dtype]
    wanted = need_x | need_w1 << 1 | need_b1 << 2 | need_w2 << 3 | (beta is not None) << 4
    ym = _mat(dy2)
    ws = _workspace(_function("mfac_gated_bwd_workspace_bytes")(t, gt, rows, cin, n, cout, *ym, *w2m, *xm, *w1m, wanted),
                    dy.device)
    _call("mfac_gated_bwd", dy.device, t, gt, code, rows, cin, n, cout, *ym, *w2m, *xm, *packed, _ptr(gamma), _ptr(beta),
          *w1m, *zm, *packed_z, _ptr(dx), cin, _ptr(dw1), cin, _ptr(db1), _ptr(dw2), n, ws[0], ws[1])
    return dx, dw1, db1, dw2


def gated_linear_backward(dy, x, weight, z, act="silu", affine=None, grad_dtype=None, need=(True, True, True)):
    """(dx, dweight, dbias) of y = act(zg) * zu, [zg, zu] = x weight^T + bias, from dy, the input x and the pre-activations z
    (a pair of tensors or of Packed8). ``affine``, ``grad_dtype``: see gated_feed_forward_backward. ``need``: which of the
    three to form; the others are None."""
    return _gated_backward(dy, x, weight, None, z, act, affine, grad_dtype, (*map(bool, need), False), behind=False)[:3]


def gated_feed_forward_backward(dy, x, w1, w2, z, act="silu", affine=None, grad_dtype=None, need=(True,) * 5):
    """(dx, dw1, db1, dw2, db2) of y = (act(zg) * zu) w2^T + b2, [zg, zu] = x w1^T + b1, from dy, the input x and the
    pre-activations z (a pair of tensors or of Packed8). ``affine`` = (gamma, beta or None), float32: the input was
    gamma * x + beta; dx is then the gradient of that. dw1 and dw2 are of ``grad_dtype`` (float32 or dy's type, the default);
    in float32 of 16-bit data they are those of dz and act(zg) * zu in two parts each, which doubles their products: rounded to
    one, these would leave them off by 2e-3. db1 and db2 are float32. ``need``: which of the five to form; the others are
    None. w2 may be None where neither dx, dw1 nor db1 is."""
    need_x, need_w1, need_b1, need_w2, need_b2 = map(bool, need)
    dx, dw1, db1, dw2 = _gated_backward(dy, x, w1, w2, z, act, affine, grad_dtype, (need_x, need_w1, need_b1, need_w2))
    return dx, dw1, db1, dw2, act_backward(dy)[2] if need_b2 else None


# ---------------------------------------------------------------- between two blocks
KINDS = {"rms": 0, "layer": B.MFAC_NORM_LAYER}


class ResidualNorm(NamedTuple):
    """s, h, and what the backward pass takes: the norms' (mean, rstd), one float32 for each row (mean None for rms norm),
    and the 8-bit copy of N_pre's xhat. None for what there is not."""
    s: Optional[torch.Tensor]
    h: Optional[torch.Tensor]
    post: Optional[tuple]
    pre: Optional[tuple]
    copy: Optional[Packed8]


class ResidualNormGrads(NamedTuple):
    """Gradients; dpost and dpre are (dweight, dbias)."""
    dy: Optional[torch.Tensor]
    dresidual: Optional[torch.Tensor]
    dgate: Optional[torch.Tensor]
    dpost: tuple
    dpre: tuple


def dropout_at(device):
    """Where a mask starts: seed and offset, drawn with torch's generator of the device."""
    return torch.empty(2, dtype=torch.int64, device=device).random_()


def _drop(p, at, data):
    p = float(p)
    if not 0 <= p <= 1:
        raise ValueError(f"dropout: p between 0 and 1, not {p}")
    if at is not None and (at.dtype != torch.int64 or at.shape != (2,) or at.device != data.device or not at.is_contiguous()):
        raise ValueError(f"dropout: at is two int64 on {data.device}")
    if p > 0 and at is None:
        raise ValueError("dropout: needs at, where the mask starts")
    return p, _ptr(at) if p > 0 else None


def dropout_forward(x, p, at):
    """x where the mask of (p, at) keeps a value, times 65536 / (65536 - T), T = floor(65536 p + 0.5); 0 elsewhere. The
    mask depends on the row (leading dimensions are rows) and the column; the gradient of x is the same of dy."""
    x2 = _rows(x, "dropout: x")
    p, ptr = _drop(p, at, x2)
    y = _like(x)
    if p == 0:
        return y.copy_(x)
    _call("mfac_dropout", x.device, _type(x2, "dropout: x"), *x2.shape, *_mat(x2), p, ptr, y.data_ptr(), x2.shape[1])
    return y


def _pair(norm):
    """(weight, bias) of a norm, None twice where there is none."""
    if norm is None:
        return None, None
    try:
        w, b = norm
    except (TypeError, ValueError):
        raise ValueError("residual_norm: a norm is None or a pair (weight, bias)") from None
    return w, b


def _between(y, post, pre, gate, kind):
    """(norms, type code of the parameters, post w, post b, pre w, pre b, gate, gates) for rows like y."""
    layer = KINDS.get(kind)
    if layer is None:
        raise ValueError(f"residual_norm: kind is one of {', '.join(KINDS)}, not {kind!r}")
    if y.shape[1] > 1 << 15:
        raise ValueError(f"residual_norm: at most 32768 columns, not {y.shape[1]}")
    norms, w1, b1, w2, b2, gv, gm = 0, None, None, None, None, None, None

    def vector(v, like):
        v = _param("residual_norm: parameters", v, y, y.shape[1])
        if like is not None and v.dtype is not like:
            raise ValueError("residual_norm: parameters of one type")
        return v, v.dtype

    found = None
    for i, norm in ((0, post), (1, pre)):
        if norm is None:
            continue
        w, b = _pair(norm)
        if w is not None:
            w, found = vector(w, found)
        if b is not None:
            if not layer:
                raise ValueError("residual_norm: rms norm has no bias")
            b, found = vector(b, found)
        if i == 0:
            w1, b1, norms = w, b, B.MFAC_NORM_POST
        else:
            w2, b2, norms = w, b, norms | B.MFAC_NORM_PRE
    if gate is not None:
        if gate.dim() == 1:
            gv, found = vector(gate, found)
        else:
            gm = _rows(gate, "residual_norm: gate")
            _same("residual_norm: gate", gm, y, y.shape)
    return norms | layer if norms else 0, _TYPES[found or torch.float32], w1, b1, w2, b2, gv, gm


def residual_norm_forward(y, residual=None, post=None, pre=None, gate=None, scale=1.0, p=0.0, at=None, kind="rms", eps=1e-6,
                          pack=False, stats=True):
    """What lies between two blocks of a network with a residual stream, as a ResidualNorm:

        n = N_post(y), s = scale * residual + gate * dropout(n), h = N_pre(s)

    over the last dimension. ``post`` and ``pre`` are None (no norm; n = y, no h) or (weight, bias), either None; ``kind``
    "rms" (no biases) or "layer" for both. ``gate``: one value for each channel, or a tensor like y. ``p`` and ``at``: see
    dropout_forward. ``pack``: also the 8-bit copy of N_pre's xhat. ``stats=False``: no statistics. With pre alone h is y's
    norm, and s is y itself."""
    y2 = _rows(y, "residual_norm: y")
    rows, cols = y2.shape
    norms, wt, w1, b1, w2, b2, gv, gm = _between(y2, post, pre, gate, kind)
    p, ptr = _drop(p, at, y2) if p != 0 or at is not None else (0.0, None)
    if residual is not None:
        residual = _rows(residual, "residual_norm: residual")
        _same("residual_norm: residual", residual, y2, y2.shape)
    if pack and pre is None:
        raise ValueError("residual_norm: the 8-bit copy is of pre's xhat")
    plain = residual is None and post is None and gate is None and p == 0
    if plain and pre is None:
        return ResidualNorm(y, None, None, None, None)
    s = None if plain else _like(y)
    h = None if pre is None else _like(y)
    m1 = r1 = m2 = r2 = None
    if stats:
        layer, device = kind == "layer", y.device
        if post is not None:
            r1 = torch.empty(rows, dtype=torch.float32, device=device)
            m1 = torch.empty_like(r1) if layer else None
        if pre is not None:
            r2 = torch.empty(rows, dtype=torch.float32, device=device)
            m2 = torch.empty_like(r2) if layer else None
    copy = Packed8.empty(rows, cols, y.device) if pack else None
    q = _NO_COPY if copy is None else copy._args()
    _call("mfac_residual_norm", y.device, _type(y2, "residual_norm: y"), wt, norms, rows, cols, *_mat(y2), _ptr(w1),
          _ptr(b1), _ptr(gv), *_mat(gm), *_mat(residual), float(scale), p, ptr, _ptr(w2), _ptr(b2), float(eps), _ptr(s),
          cols, _ptr(h), cols, _ptr(m1), _ptr(r1), _ptr(m2), _ptr(r2), *q)
    return ResidualNorm(y if plain else s, h, None if r1 is None else (m1, r1), None if r2 is None else (m2, r2), copy)


def residual_norm_backward(ds, dh, y, s, post_stats=None, pre_stats=None, post=None, pre=None, gate=None, scale=1.0, p=0.0,
                           at=None, kind="rms", need=(True, True, True, True)):
    """The gradients of residual_norm_forward as ResidualNormGrads, from ds, the gradient that reaches s by its other uses
    (None: none), dh, that of h, and what the forward pass took and returned: y (None where neither post nor the gate's
    gradient needs it), s or the 8-bit copy of N_pre's xhat (a Packed8 as s), the statistics. ``need``: which of dy,
    dresidual, dgate and the parameters' gradients to form; the others are None. dresidual is dy itself where they are equal."""
    if (dh is None) != (pre is None) or (ds is None and dh is None):
        raise ValueError("residual_norm: dh goes with pre, and without it ds is needed")
    like = ds if ds is not None else dh
    d2 = _rows(like, "residual_norm: ds, dh")
    rows, cols = d2.shape
    norms, wt, w1, b1, w2, b2, gv, gm = _between(d2, post, pre, gate, kind)
    p, ptr = _drop(p, at, d2)
    layer = kind == "layer"
    need_y, need_r, need_gate, need_params = need
    need_gate = need_gate and gate is not None

    shape, dtype, device = d2.shape, d2.dtype, d2.device

    def rows_of(t, what):
        t = _rows(t, what)
        if t.dtype is not dtype or t.shape != shape or t.device != device:
            raise ValueError(f"residual_norm: {what}: {tuple(shape)} {dtype} on {device}, not {tuple(t.shape)} {t.dtype} on "
                             f"{t.device}")
        return t

    def stats_of(stats, on, what, mean_needed):
        mean, rstd = (None, None) if not on else stats if stats is not None else (None, None)
        for t in (mean, rstd):
            if t is not None and (t.dtype != torch.float32 or t.numel() != rows or not t.is_contiguous()
                                  or t.device != device):
                raise ValueError(f"residual_norm: {what} statistics are contiguous float32 tensors, one value for each row")
        if on and (rstd is None or (mean_needed and mean is None)):
            raise ValueError(f"residual_norm: needs {what} statistics")
        return mean if mean_needed else None, rstd

    if dh is not None:
        dh = rows_of(dh, "dh")
    if ds is not None:
        ds = rows_of(ds, "ds")
    needs_y = post is not None or need_gate
    if needs_y and y is None:
        raise ValueError("residual_norm: post and the gate's gradient need y")
    y = rows_of(y, "y") if needs_y else None
    sm, packed = (None, 0), _NO_COPY
    if pre is not None:
        if isinstance(s, Packed8):
            if s.shape != d2.shape or s.device != d2.device:
                raise ValueError("residual_norm: an 8-bit copy of dh's shape")
            packed = s._args()
        elif s is None:
            raise ValueError("residual_norm: pre needs s or the 8-bit copy")
        else:
            s = rows_of(s, "s")
            sm = _mat(s)
    m1, r1 = stats_of(post_stats, post is not None, "post", layer and post is not None)
    m2, r2 = stats_of(pre_stats, pre is not None, "pre", layer and pre is not None and not isinstance(s, Packed8))

    same = post is None and gate is None and p == 0 and float(scale) == 1
    dy = _like(like) if need_y or (same and need_r) else None
    dr = dy if same else _like(like) if need_r else None
    wanted = [v is not None and need_params for v in (w1, b1, w2, b2)] + [gv is not None and need_gate]
    t = _type(d2, "residual_norm: ds, dh")
    grads, ws = [None] * 5, (None, 0, None)
    if any(wanted):
        of = next(v.dtype for v in (w1, b1, w2, b2, gv) if v is not None)
        parts = iter(torch.empty((sum(wanted), cols), dtype=of, device=device).unbind(0))
        grads = [next(parts) if on else None for on in wanted]
        ws = _workspace(_function("mfac_residual_norm_bwd_workspace_bytes")(t, norms, rows, cols), like.device)
    dg = _like(gate) if gm is not None and need_gate else None
    _call("mfac_residual_norm_bwd", like.device, t, wt, norms, rows, cols, *_mat(ds),
          *_mat(dh), *_mat(y), _ptr(m1), _ptr(r1), *sm, *packed, _ptr(m2), _ptr(r2), _ptr(w1), _ptr(b1), _ptr(gv),
          *_mat(gm), float(scale), p, ptr, _ptr(w2), _ptr(dy), cols, None if same else _ptr(dr), cols, _ptr(dg), cols,
          _ptr(grads[0]), _ptr(grads[1]), _ptr(grads[4]), _ptr(grads[2]), _ptr(grads[3]), ws[0], ws[1])
    return ResidualNormGrads(dy if need_y else None, dr if need_r else None, grads[4] if gm is None else dg,
                             (grads[0], grads[1]), (grads[2], grads[3]))


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


class _GatedLinear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, act, copy8, grad):
        w = weight.to(x.dtype)
        need = [grad and n for n in ctx.needs_input_grad[:3]]
        if not any(need):
            return gated_linear_forward(x, w, bias, act)
        y, (zg, zu) = gated_linear_forward(x, w, bias, act, "pack8" if copy8 else "z")
        ctx.act, ctx.wdtype, ctx.bdtype = act, weight.dtype, None if bias is None else bias.dtype
        _keep(ctx, x=(pack8(x) if copy8 else x) if need[1] else None, w=w if need[0] else None, zg=zg, zu=zu)
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        k = _kept(ctx)
        dx, dw, db = gated_linear_backward(dy, k["x"], k["w"], (k["zg"], k["zu"]), ctx.act,
                                           grad_dtype=_grad_dtype(ctx.wdtype, dy), need=ctx.needs_input_grad[:3])
        return dx, _to(dw, ctx.wdtype), _to(db, ctx.bdtype), None, None, None


class _GatedFeedForward(torch.autograd.Function):
    """y = (act(zg) * zu) W2^T + b2, [zg, zu] = x W1^T + b1. act(zg) * zu is formed again in the backward pass. q and s: the
    8-bit copy that the norm before the block keeps, of which x is gamma times that plus beta; kept for dW1 in place of a copy
    of x."""

    @staticmethod
    def forward(ctx, x, w1, b1, w2, b2, act, copy8, grad, q, s, gamma, beta):
        c1, c2 = w1.to(x.dtype), w2.to(x.dtype)
        need = [grad and n for n in ctx.needs_input_grad[:5]]
        inner = any(need[:3])   # whether a gradient passes through the gate
        if not (inner or need[3]):
            ctx.types = tuple(None if p is None else p.dtype for p in (w1, b1, w2, b2))
            _keep(ctx, x=None, zg=None, zu=None, c1=None, c2=None, gamma=None, beta=None)
            return linear_forward(gated_linear_forward(x, c1, b1, act), c2, b2)
        a, (zg, zu) = gated_linear_forward(x, c1, b1, act, "pack8" if copy8 else "z")
        y = linear_forward(a, c2, b2)
        ctx.act, ctx.types = act, tuple(None if p is None else p.dtype for p in (w1, b1, w2, b2))
        shared = q is not None and need[1]
        kept = None if not need[1] else Packed8(q, s) if shared else pack8(x) if copy8 else x
        _keep(ctx, x=kept, zg=zg, zu=zu, c1=c1 if need[0] else None, c2=c2 if inner else None, gamma=gamma if shared else None,
              beta=beta if shared else None)
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        k = _kept(ctx)
        t = ctx.types
        need = ctx.needs_input_grad[:5]
        if not any(need[:4]):
            return (None, None, None, None, _to(act_backward(dy)[2], t[3])) + (None,) * 7
        # in float32 where either weight has neither its own type nor the data's
        grad = dy.dtype if t[0] == t[2] == dy.dtype else torch.float32
        dx, dw1, db1, dw2, db2 = gated_feed_forward_backward(dy, k["x"], k["c1"], k["c2"], (k["zg"], k["zu"]), ctx.act,
                                                             None if k["gamma"] is None else (k["gamma"], k["beta"]), grad, need)
        return (dx, _to(dw1, t[0]), _to(db1, t[1]), _to(dw2, t[2]), _to(db2, t[3])) + (None,) * 7


class _Residual(torch.autograd.Function):
    @staticmethod
    def forward(ctx, y, residual, w1, b1, w2, b2, gate, post, pre, scale, p, at, kind, eps, copy8, grad):
        """(s, h, the kept copy of N_pre's xhat as two tensors), s None where it is y."""
        ctx.set_materialize_grads(False)
        need = [grad and n for n in ctx.needs_input_grad[:7]]
        train = any(need)
        o = residual_norm_forward(y, residual, (w1, b1) if post else None, (w2, b2) if pre else None, gate, scale, p, at, kind,
                                  eps, pack=copy8 and pre and train, stats=train)
        plain = o.s is y
        if train:
            ctx.options = post, pre, scale, p, kind
            ctx.rshape = None if residual is None else residual.shape   # its rows may lie in other dimensions than y's
            m1, r1 = o.post if post else (None, None)
            m2, r2 = o.pre if pre else (None, None)
            _keep(ctx, y=y if post or need[6] else None, s=o.copy if o.copy is not None else o.s if pre else None, m1=m1, r1=r1,
                  m2=m2, r2=r2, w1=w1, b1=b1, w2=w2, b2=b2, gate=gate, at=at if p > 0 else None)
        copy = (None, None) if o.copy is None else (o.copy.q, o.copy.s)
        ctx.mark_non_differentiable(*(t for t in copy if t is not None))
        return (None if plain else o.s, o.h, *copy)

    @staticmethod
    @once_differentiable
    def backward(ctx, ds, dh, *of_copy):
        post, pre, scale, p, kind = ctx.options
        if ds is None and dh is None:
            return (None,) * 16
        k = _kept(ctx)
        need = ctx.needs_input_grad[:7]
        used = dh is not None   # s alone may have been used
        g = residual_norm_backward(ds, dh, k["y"], k["s"], (k["m1"], k["r1"]), (k["m2"], k["r2"]),
                                   (k["w1"], k["b1"]) if post else None, (k["w2"], k["b2"]) if used else None, k["gate"],
                                   scale, p, k["at"], kind, need=(need[0], need[1], need[6], any(need[2:6])))
        dr = None if g.dresidual is None else g.dresidual.reshape(ctx.rshape)
        params = [v if n else None for v, n in zip((*g.dpost, *g.dpre), need[2:6])]
        return (g.dy, dr, *params, g.dgate if need[6] else None) + (None,) * 9


class _Dropout(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, p, at):
        ctx.p = p
        ctx.save_for_backward(at)
        return dropout_forward(x, p, at)

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        return dropout_forward(dy, ctx.p, *ctx.saved_tensors), None, None


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


def gated_linear(x, weight, bias=None, act="silu", copy8=False):
    """act(x Wg^T + bg) * (x Wu^T + bu), differentiable, for weight = [Wg; Wu] (2 hidden x cin) and bias = [bg, bu].
    copy8: keep x and the pre-activations in 8 bits for the backward pass."""
    _act(act)
    return _GatedLinear.apply(x, weight, bias, act, copy8, torch.is_grad_enabled())


def gated_feed_forward(x, w1, w2, b1=None, b2=None, act="silu", copy8=False):
    """gated_linear(x, w1, b1, act) w2^T + b2, differentiable. copy8: what the backward pass needs is kept in 8 bits."""
    _act(act)
    return _GatedFeedForward.apply(x, w1, b1, w2, b2, act, copy8, torch.is_grad_enabled(), None, None, None, None)


def residual_norm(y, residual=None, post=None, pre=None, gate=None, scale=1.0, p=0.0, at=None, kind="rms", eps=1e-6,
                  copy8=False):
    """(s, h) of residual_norm_forward, differentiable; h is None without pre, and s is y where nothing lies between.
    ``at`` is drawn where p > 0 and none is given. copy8: keep N_pre's xhat in 8 bits for the backward pass instead of s."""
    return _residual_norm(y, residual, post, pre, gate, scale, p, at, kind, eps, copy8)[:2]


def _residual_norm(y, residual=None, post=None, pre=None, gate=None, scale=1.0, p=0.0, at=None, kind="rms", eps=1e-6,
                   copy8=False):
    """(s, h, and the kept copy of N_pre's xhat as two tensors, or None twice)"""
    if post is None and pre is None and gate is None and residual is None and p == 0:
        return y, None, None, None
    of_post, of_pre = _pair(post), _pair(pre)
    if p > 0 and at is None:
        at = dropout_at(y.device)
    s, *rest = _Residual.apply(y, residual, *of_post, *of_pre, gate, post is not None, pre is not None, scale, p, at, kind, eps,
                               copy8, torch.is_grad_enabled())
    return (y if s is None else s, *rest)


def rms_norm(x, weight=None, eps=1e-6, copy8=False):
    """x / sqrt(mean(x^2) + eps) * weight over the last dimension, differentiable. copy8: keep the normalised x in 8 bits
    for the backward pass instead of x."""
    return residual_norm(x, pre=(weight, None), eps=eps, copy8=copy8)[1]


def dropout(x, p=0.5, training=True, at=None):
    """Dropout, differentiable: see dropout_forward. ``at`` is drawn where none is given."""
    if not training or p == 0:
        return x
    at = dropout_at(x.device) if at is None else at
    return _Dropout.apply(x, p, at)


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


class RMSNorm(torch.nn.Module):
    """RMS norm over the last dimension, of size `dim`."""

    def __init__(self, dim, eps=1e-6, copy8=False, device=None):
        super().__init__()
        self.eps, self.copy8 = eps, copy8
        self.weight = torch.nn.Parameter(torch.ones(dim, device=device))

    def forward(self, x):
        return rms_norm(x, self.weight, self.eps, self.copy8)


class GatedLinear(torch.nn.Module):
    """act(x Wg^T + bg) * (x Wu^T + bu); weight = [Wg; Wu], uniform within 1 / sqrt(cin)."""

    def __init__(self, cin, hidden, bias=False, act="silu", copy8=False, device=None):
        super().__init__()
        _act(act)
        self.act, self.copy8 = act, copy8
        r = cin ** -0.5
        self.weight = torch.nn.Parameter(torch.empty(2 * hidden, cin, device=device).uniform_(-r, r))
        self.bias = torch.nn.Parameter(torch.empty(2 * hidden, device=device).uniform_(-r, r)) if bias else None

    def forward(self, x):
        return gated_linear(x, self.weight, self.bias, self.act, self.copy8)


class Dropout(torch.nn.Module):
    """Dropout whose mask is not stored, in training mode."""

    def __init__(self, p=0.5):
        super().__init__()
        if not 0 <= p <= 1:
            raise ValueError(f"dropout: p between 0 and 1, not {p}")
        self.p = p

    def forward(self, x, at=None):
        return dropout(x, self.p, self.training, at)


class GatedFeedForward(torch.nn.Module):
    """A gated feed-forward block with its norms and skip connection:
    scale * x + gate * dropout(N_post(FF(N_pre(x)))), FF(h) = (act(h Wg^T) * (h Wu^T)) W2^T.

    kind: "rms" or "layer"; post_norm: whether there is a norm after the block; gate: the first value of a learned gate for
    each channel, or None for none; p: dropout's, in training mode."""

    def __init__(self, dim, hidden, act="silu", kind="rms", eps=1e-6, post_norm=False, gate=None, scale=1.0, p=0.0, bias=False,
                 copy8=False, device=None):
        super().__init__()
        if kind not in KINDS or not 0 <= p <= 1:
            raise ValueError(f"GatedFeedForward: kind is one of {', '.join(KINDS)}, and p between 0 and 1")
        self.kind, self.eps, self.scale, self.p, self.copy8 = kind, eps, scale, p, copy8

        def norm():
            return RMSNorm(dim, eps, device=device) if kind == "rms" else LayerNorm(dim, eps, device=device)

        self.norm, self.post = norm(), norm() if post_norm else None
        self.up = GatedLinear(dim, hidden, bias, act, device=device)
        self.down = Linear(hidden, dim, bias, device=device)
        self.gate = None if gate is None else torch.nn.Parameter(torch.full((dim,), float(gate), device=device))

    def inner(self, h, copy=None):
        """The block without its norms and skip connection. copy: what self.norm kept of h, (q, s) or None (see join)."""
        q, s, gamma, beta = None, None, None, None
        if self.copy8 and copy is not None:
            (q, s), (gamma, beta) = copy, (None if v is None else v.detach() for v in _norm_of(self.norm))
        return _GatedFeedForward.apply(h, self.up.weight, self.up.bias, self.down.weight, self.down.bias, self.up.act, self.copy8,
                                       torch.is_grad_enabled(), q, s, gamma, beta)

    def join(self, y, x, pre=None, want_copy=False):
        """(s, h): the stream after the block, and its norm `pre` (the next block's; None: no h). want_copy: also the 8-bit copy
        that the norm keeps of h's xhat, (q, s), or None where it keeps none: the next block's `inner` shares it."""
        s, h, *copy = _residual_norm(y, x, _norm_of(self.post), _norm_of(pre), self.gate, self.scale,
                                     self.p if self.training else 0.0, kind=self.kind, eps=self.eps, copy8=self.copy8)
        return (s, h, copy if copy[0] is not None else None) if want_copy else (s, h)

    def first(self, x):
        """(h, copy): the norm before the block, of x, and what it keeps of it, as in join."""
        _, h, *copy = _residual_norm(x, pre=_norm_of(self.norm), kind=self.kind, eps=self.eps, copy8=self.copy8)
        return h, copy if copy[0] is not None else None

    def forward(self, x):
        h, copy = self.first(x)
        return self.join(self.inner(h) if copy is None else self.inner(h, copy), x)[0]


def _norm_of(module):
    return None if module is None else (module.weight, getattr(module, "bias", None))


class GatedStack(torch.nn.Module):
    """`depth` GatedFeedForward blocks and a last norm. The norms after a block and before the next, with what lies between
    them, are one pass over the rows."""

    def __init__(self, dim, hidden, depth, kind="rms", eps=1e-6, device=None, **block):
        super().__init__()
        if depth < 1:
            raise ValueError("GatedStack: at least one block")
        self.blocks = torch.nn.ModuleList([GatedFeedForward(dim, hidden, kind=kind, eps=eps, device=device, **block)
                                           for _ in range(depth)])
        self.norm = RMSNorm(dim, eps, device=device) if kind == "rms" else LayerNorm(dim, eps, device=device)

    def forward(self, x):
        h, copy = self.blocks[0].first(x)
        for block, norm in zip(self.blocks, [b.norm for b in self.blocks[1:]] + [self.norm]):
            y = block.inner(h) if copy is None else block.inner(h, copy)
            x, h, *kept = block.join(y, x, norm, want_copy=True) if block.copy8 else block.join(y, x, norm)
            copy = kept[0] if kept else None
        return h
