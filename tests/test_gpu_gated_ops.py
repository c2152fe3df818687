"""Gated layers, what lies between two blocks, and dropout against their definitions in 64 bits."""

import pytest
import torch

from gated_ref import (drop_factor, gate_slopes64, gated64, residual64, residual_back64, rounded)
from gpu_common import require_gpu, say
from train_ref import E32, TINY, U, act64, growth, off, unpack64

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
ACTS = ["none", "relu", "gelu", "gelu_tanh", "silu"]


@pytest.fixture(scope="module")
def dev():
    return require_gpu()


def rand(dev, seed, *shape, dtype=F32, scale=1.0, at=0.0, pad=0):
    """Normal values around `at` in dtype; rows `pad` elements further apart than they are long."""
    g = torch.Generator(device=dev).manual_seed(seed)
    x = (at + scale * torch.randn(*shape, generator=g, device=dev)).to(dtype)
    if not pad:
        return x
    wide = torch.full((*shape[:-1], shape[-1] + pad), float("nan"), dtype=dtype, device=dev)
    wide[..., :shape[-1]] = x
    return wide[..., :shape[-1]]


def holds(got, want, bound, what):
    o = off(got, want, bound)
    assert o <= 1, (what, o)


def copy_holds(p, want, err, what):
    """The copy of values that are off by err: half a step, and a step no larger than they need."""
    step = torch.exp2(p.s.double() - 127)
    holds(unpack64(p.q, p.s), want, step.repeat_interleave(32, 1)[:, :want.shape[1]] / 2 + err, what)
    most = torch.nn.functional.pad(want.abs() + err, (0, -want.shape[1] % 32)).view(want.shape[0], -1, 32).amax(2)
    assert (step <= torch.clamp(2 * most / 127, min=2.0 ** -126)).all(), what


# ---------------------------------------------------------------- dropout
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 7), (3, 8), (5, 100), (257, 1000), (2, 70000), (70000, 3)])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_dropout(dev, dtype, rows, cols):
    from paper_2107_03356_amd import nn
    say("dropout", dtype, rows, cols)
    for pad in (0, 3):
        x = rand(dev, 1, rows, cols, dtype=dtype, pad=pad)
        for p, at in ((0.1, (5, 6)), (0.5, (-1, -2)), (1.0, (3, 1 << 62)), (2.0 ** -18, (1 << 40, 1 << 33))):
            f = drop_factor(rows, cols, p, at).to(dev)
            y = nn.dropout_forward(x, p, torch.tensor(at, device=dev))
            want = x.double() * f
            holds(y, want, (U[dtype] + 2 * E32) * want.abs() + TINY[dtype], (p, at))
            assert torch.equal(y == 0, (f == 0) | (x == 0))


def test_dropout_of_what_is_not_finite(dev):
    from paper_2107_03356_amd import nn
    say("dropout not finite")
    at = torch.tensor([9, 9], device=dev)
    f = drop_factor(4, 64, 0.5, (9, 9)).to(dev)
    for bad in (float("nan"), float("inf")):
        y = nn.dropout_forward(torch.full((4, 64), bad, device=dev), 0.5, at)
        assert (y[f == 0] == 0).all() and not torch.isfinite(y[f != 0]).any()


def test_dropout_in_place_and_gradient(dev):
    from paper_2107_03356_amd import _binding as B
    from paper_2107_03356_amd import nn
    say("dropout in place")
    at = torch.tensor([21, 22], device=dev)
    x = rand(dev, 1, 50, 333)
    want = nn.dropout_forward(x, 0.3, at)
    same = x.clone()
    assert B.mfac_dropout(B.MFAC_F32, 50, 333, same.data_ptr(), 333, 0.3, at.data_ptr(), same.data_ptr(), 333,
                          torch.cuda.current_stream().cuda_stream) == B.MFAC_OK
    assert torch.equal(same, want)
    leaf, dy = x.clone().requires_grad_(), rand(dev, 2, 50, 333)
    y = nn.dropout(leaf, 0.3, at=at)
    y.backward(dy)
    assert torch.equal(y, want) and torch.equal(leaf.grad, nn.dropout_forward(dy, 0.3, at))
    assert nn.dropout(x, 0.3, training=False) is x and nn.dropout(x, 0.0) is x
    module = nn.Dropout(0.3)
    torch.manual_seed(5)
    a, b = module(x), module(x)
    torch.manual_seed(5)
    assert torch.equal(module(x), a) and not torch.equal(a, b)
    assert module.eval()(x) is x


# ---------------------------------------------------------------- gated layers
# (rows, cin, hidden) of every kernel: few rows with 8, 16 and 32 columns a work-group; tiles of 64, 128 and 256, whole
# and with edges, in one and in more parts of K; and sizes that nothing divides
FORWARD = [(1, 64, 1), (1, 2048, 300), (5, 40, 33), (16, 1000, 3000), (3, 520, 5001), (17, 64, 40), (40, 1000, 77), (40, 4104, 96),
           (300, 520, 261), (1003, 264, 523), (301, 4104, 261), (1101, 4104, 515), (2051, 200, 1027), (3001, 520, 1539)]


def test_forward_sizes_run_every_kernel(dev):
    from paper_2107_03356_amd import _binding as B
    from gated_cases import gated_plan
    seen = {gated_plan("bf16", False, *size)[:2] for size in FORWARD if size[0] > 16}
    assert {t for t, _ in seen} == {64, 128, 256} and any(s > 1 for _, s in seen), seen
    assert gated_plan("bf16", False, 16, 1000, 3000)[0] == 0
    assert B.mfac_gated_plan(3, 0, 1, 1, 1, None) == B.MFAC_EINVAL


def forward_reference(x, w, b):
    n = w.shape[0] // 2
    z = x.double() @ w.double().t()
    e = E32 * growth(x.shape[1]) * (x.double().abs() @ w.double().abs().t())
    if b is not None:
        z, e = z + b.double(), e + 2 * E32 * (z + b.double()).abs() + 2 * E32 * b.double().abs()
    return (z[:, :n], z[:, n:]), (e[:, :n], e[:, n:])


@pytest.mark.parametrize("rows,cin,hid", FORWARD)
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_gated_forward(dev, dtype, rows, cin, hid):
    from paper_2107_03356_amd import nn
    say("gated forward", dtype, rows, cin, hid)
    tiny = TINY[dtype]
    for pad, bias in ((0, False), (5, True)):
        x = rand(dev, 1, rows, cin, dtype=dtype, pad=pad)
        w = rand(dev, 2, 2 * hid, cin, dtype=dtype, scale=cin ** -0.5, pad=pad)
        b = rand(dev, 3, 2 * hid, scale=0.5) if bias else None
        z, e = forward_reference(x, w, b)
        for act in ACTS if rows < 400 else ACTS[2:]:
            y64, ye = gated64(act, *z, *e)
            y = nn.gated_linear_forward(x, w, b, act)
            holds(y, y64, rounded(y64, ye, dtype, tiny), act)
        yz, kept = nn.gated_linear_forward(x, w, b, act, keep="z")
        y8, copies = nn.gated_linear_forward(x, w, b, act, keep="pack8")
        assert torch.equal(yz, y) and torch.equal(y8, y)
        for i in range(2):
            holds(kept[i], z[i], rounded(z[i], e[i], dtype, tiny), "z")
            copy_holds(copies[i], z[i], e[i], "copy")
    if b is not None and dtype != F32:
        y64, ye = gated64(act, *forward_reference(x, w, b.to(dtype))[0], *e)
        holds(nn.gated_linear_forward(x, w, b.to(dtype), act), y64, rounded(y64, ye, dtype, tiny), "bias of the data's type")


def halves(dev, n, dtype):
    """Weights [I; 0] and [0; I], by which dx is the gate's half of dz, or the other one."""
    eye = torch.eye(n, device=dev, dtype=dtype)
    return torch.cat([eye, 0 * eye]), torch.cat([0 * eye, eye])


@pytest.mark.parametrize("rows,hid", [(1, 1), (3, 40), (70, 515), (2000, 33), (9, 2050), (3000, 1030)])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("act", ACTS)
def test_gated_linear_backward_through_the_gate(dev, act, dtype, rows, hid):
    from paper_2107_03356_amd import nn
    say("gated backward through the gate", act, dtype, rows, hid)
    tiny = TINY[dtype]
    da = rand(dev, 1, rows, hid, dtype=dtype, pad=1)
    pair = rand(dev, 2, rows, 2 * hid, dtype=dtype, scale=2.0)
    zg, zu = pair[:, :hid], pair[:, hid:]
    packs = nn.pack8(zg), nn.pack8(zu)
    for z in ((zg, zu), packs):
        g64, u64 = ((unpack64(v.q, v.s) for v in z) if z is packs else (zg.double(), zu.double()))
        dg, du, _ = gate_slopes64(act, g64, u64, da.double(), 0 * g64)
        for w, (v, e) in zip(halves(dev, hid, dtype), (dg, du)):
            dx, none, db = nn.gated_linear_backward(da, None, w, z, act, need=(True, False, True))
            # one product with 1, others with 0: exact in 16 bits, of three parts in fp32 to two roundings
            holds(dx, v, rounded(v, e + 2 * E32 * v.abs() * (dtype == F32), dtype, tiny), "dz")
            assert none is None
        v, e = torch.cat([dg[0], du[0]], 1), torch.cat([dg[1], du[1]], 1)
        holds(db, v.sum(0), E32 * (rows / 4 + 60) * v.abs().sum(0) + e.sum(0) + 1e-30, "db")
        again = nn.gated_linear_backward(da, None, w, z, act, need=(True, False, False))
        assert torch.equal(again[0], dx) and again[2] is None


# (rows, hidden, cout)
HIDDEN = [(1, 33, 40), (20, 128, 64), (20, 100, 64), (300, 256, 520), (1003, 523, 264), (1003, 576, 264), (301, 320, 4104),
          (301, 261, 4104), (1101, 1088, 4104), (2051, 1024, 200), (3001, 3008, 264), (3001, 3077, 264)]


def test_hidden_sizes_run_every_kernel(dev):
    from gated_cases import gated_plan
    seen = {gated_plan("bf16", True, r, c, h)[:2] for r, h, c in HIDDEN}
    assert {t for t, _ in seen} == {64, 128, 256} and any(s > 1 for _, s in seen), seen
    # where parts of K are joined, dz and a are formed there, whatever the hidden size (test_gated_feed_forward_backward)
    for dtype in ("f32", "bf16"):
        assert all(gated_plan(dtype, True, r, c, h)[1] > 1 for r, c, h in ((260, 2056, 261), (70, 2056, 320)))


@pytest.mark.parametrize("rows,hid,cout", HIDDEN)
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_gated_backward_behind_the_next_layer(dev, dtype, rows, hid, cout):
    """dz where da = dy w2, formed in that product (no db; parts of K joined, or 16-bit data and hidden a multiple of 64) or
    from a stored da."""
    from paper_2107_03356_amd import nn
    say("gated backward behind the next layer", dtype, rows, hid, cout)
    tiny = TINY[dtype]
    weights = halves(dev, hid, dtype)
    for pad in (0, 3):
        dy = rand(dev, 1, rows, cout, dtype=dtype, pad=pad)
        w = rand(dev, 2, cout, hid, dtype=dtype, scale=cout ** -0.5, pad=pad)
        da = dy.double() @ w.double()
        ed = E32 * growth(cout) * (dy.double().abs() @ w.double().abs())
        z = rand(dev, 3, rows, hid, dtype=dtype, pad=pad), rand(dev, 4, rows, hid, dtype=dtype, pad=pad)
        packs = tuple(nn.pack8(v) for v in z)
        for act in ACTS if rows < 400 else ACTS[2:]:
            for pair in (z, packs) if act in ("silu", "gelu") else (z,):
                g64, u64 = (unpack64(v.q, v.s) for v in pair) if pair is packs else (v.double() for v in pair)
                dg, du, _ = gate_slopes64(act, g64, u64, da, ed)
                for w1, (v, e) in zip(weights, (dg, du)):
                    bound = rounded(v, e + 2 * E32 * v.abs() * (dtype == F32), dtype, tiny)
                    dx = nn.gated_feed_forward_backward(dy, None, w1, w, pair, act, need=(True, False, False, False, False))[0]
                    holds(dx, v, bound, (act, "dz"))
        dx, _, db, _, _ = nn.gated_feed_forward_backward(dy, None, w1, w, pair, act, need=(True, False, True, False, False))
        holds(dx, v, bound, "dz beside db")
        v, e = torch.cat([dg[0], du[0]], 1), torch.cat([dg[1], du[1]], 1)
        holds(db, v.sum(0), E32 * (rows / 4 + 60) * v.abs().sum(0) + e.sum(0) + 1e-30, "db")


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("rows,hid", [(1, 64), (40, 64), (70, 100), (130, 1028)])
def test_gated_activation_formed_again(dev, dtype, rows, hid):
    """With dy the identity, dw2 is act(zg) zu itself: rounded to the data's type, or in two parts for a gradient in fp32."""
    from paper_2107_03356_amd import nn
    say("gated activation formed again", dtype, rows, hid)
    dy, w2 = torch.eye(rows, dtype=dtype, device=dev), rand(dev, 1, rows, hid, dtype=dtype)
    z = rand(dev, 2, rows, hid, dtype=dtype, scale=2.0), rand(dev, 3, rows, hid, dtype=dtype)
    for act in ACTS:
        _, _, (a, e) = gate_slopes64(act, z[0].double(), z[1].double(), w2.double(), 0 * w2.double())
        for grad in (F32, dtype):
            got = nn.gated_feed_forward_backward(dy, None, None, w2, z, act, grad_dtype=grad, need=(False, False, False, True, False))
            step = U[dtype] if grad == dtype else U[dtype] ** 2 + 2 * E32
            holds(got[3], a, 1.02 * step * a.abs() + 1.01 * e + 2 * E32 * a.abs() + TINY[dtype], (act, grad))
            assert got[0] is got[1] is got[2] is got[4] is None


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,dim,hid", [(1, 64, 96), (130, 72, 200), (700, 264, 515), (260, 2056, 261), (70, 2056, 320)])
def test_gated_feed_forward_backward(dev, dtype, rows, dim, hid):
    """Against the formulas, with dz and a counted as the call rounds them: to the data's type for dx and for gradients
    of that type, in two parts for gradients in float32."""
    from paper_2107_03356_amd import nn
    say("gated feed forward backward", dtype, rows, dim, hid)
    tiny = TINY[dtype]
    dy, x = rand(dev, 1, rows, dim, dtype=dtype), rand(dev, 2, rows, dim, dtype=dtype)
    w1 = rand(dev, 3, 2 * hid, dim, dtype=dtype, scale=dim ** -0.5)
    w2 = rand(dev, 4, dim, hid, dtype=dtype, scale=hid ** -0.5)
    pair = rand(dev, 5, rows, 2 * hid, dtype=dtype)
    packs = nn.pack8(pair[:, :hid].contiguous()), nn.pack8(pair[:, hid:].contiguous())
    xp, gamma, beta = nn.pack8(x), rand(dev, 6, dim, at=1, scale=0.2), rand(dev, 7, dim)
    da = dy.double() @ w2.double()
    ed = E32 * growth(dim) * (dy.double().abs() @ w2.double().abs())
    dm = dy.double().abs()
    for z, kept, affine in (((pair[:, :hid], pair[:, hid:]), x, None), (packs, xp, (gamma, None)), (packs, xp, (gamma, beta))):
        g64, u64 = (unpack64(v.q, v.s) for v in z) if z is packs else (v.double() for v in z)
        b64 = beta.double() if affine is not None and affine[1] is not None else torch.zeros_like(gamma).double()
        x64 = x.double() if affine is None else unpack64(xp.q, xp.s) * gamma.double() + b64
        x_size = x64.abs() if affine is None else unpack64(xp.q, xp.s).abs() * gamma.double().abs() + b64.abs()
        (dg, eg), (du, eu), (a, ea) = gate_slopes64("silu", g64, u64, da, ed)
        dz, e = torch.cat([dg, du], 1), torch.cat([eg, eu], 1)
        for grad in (F32, dtype):
            step = U[dtype] if grad == dtype else U[dtype] ** 2 + E32
            ez, eb = (1.02 * step * v.abs() + 1.01 * err + tiny for v, err in ((dz, e), (a, ea)))
            for need in ((True, True, False, True, False), (True,) * 5):
                got = nn.gated_feed_forward_backward(dy, kept, w1, w2, z, affine=affine, grad_dtype=grad, need=need)
                dx, once = dz @ w1.double(), U[dtype] * dz.abs() + 1.01 * e + tiny
                holds(got[0], dx, rounded(dx, (once + E32 * growth(2 * hid) * dz.abs()) @ w1.double().abs(), dtype, tiny), "dx")
                # products over the rows (twice as many of two parts), the affine part's roundings and db's sum
                units = E32 * (2 * growth(rows) + 1 + (0 if affine is None else growth(rows) + rows / 4 + 60))
                dw1 = dz.t() @ x64
                holds(got[1], dw1, rounded(dw1, (ez + units * dz.abs()).t() @ x_size, grad, 1e-30 + TINY[grad]), "dw1")
                dw2 = dy.double().t() @ a
                holds(got[3], dw2, rounded(dw2, dm.t() @ (eb + units * a.abs()), grad, 1e-30 + TINY[grad]), "dw2")
                if need[2]:
                    holds(got[2], dz.sum(0), e.sum(0) * 1.01 + E32 * (rows / 4 + 60) * dz.abs().sum(0) + 1e-30, "db1")
                    holds(got[4], dy.double().sum(0), E32 * (rows / 4 + 60) * dm.sum(0) + 1e-30, "db2")
                else:
                    assert got[2] is None and got[4] is None


@pytest.mark.parametrize("size", [1.0, 2.0 ** -9, 2.0 ** -16])
@pytest.mark.parametrize("rows,hid", [(1, 64), (130, 515), (333, 192), (1300, 64)])
def test_fp16_gradients_as_small_as_they_come(dev, rows, hid, size):
    """With x the identity, dw1 is dz transposed, from two fp16 parts: the second is stored times 2^11, where a step of
    fp16 is at least 2^-24, so the two are within 2^-36 of a value, however small."""
    from paper_2107_03356_amd import nn
    say("fp16 gradients as small as they come", rows, hid, size)
    dim, x = 40, torch.eye(rows, dtype=F16, device=dev)
    z = rand(dev, 2, rows, hid, dtype=F16), rand(dev, 3, rows, hid, dtype=F16)
    dy, w2 = (rand(dev, 4, rows, dim) * size).to(F16), rand(dev, 5, dim, hid, dtype=F16, scale=dim ** -0.5)
    w1, mine = rand(dev, 6, 2 * hid, rows, dtype=F16), (rand(dev, 7, rows, hid) * size).to(F16)
    zero = torch.zeros(rows, hid, dtype=torch.float64, device=dev)
    da, ed = dy.double() @ w2.double(), E32 * growth(dim) * (dy.double().abs() @ w2.double().abs())
    for d, err, got in (
            (da, ed, nn.gated_feed_forward_backward(dy, x, w1, w2, z, grad_dtype=F32, need=(False, True, False, True, False))[1]),
            (mine.double(), zero, nn.gated_linear_backward(mine, x, w1, z, grad_dtype=F32, need=(False, True, False))[1])):
        (dg, eg), (du, eu), _ = gate_slopes64("silu", z[0].double(), z[1].double(), d, err)
        dz, e = torch.cat([dg, du], 1), torch.cat([eg, eu], 1)
        # a product with 1 and sums with 0 are exact; the two parts' sum is rounded once, joined parts of K once more
        holds(got, dz.t(), (1.02 * U[F16] ** 2 * dz.abs() + 1.01 * e + 2.0 ** -36 + 2 * E32 * dz.abs()).t(), (rows, hid, size))


# ---------------------------------------------------------------- between two blocks
SIZES = [(1, 1), (3, 7), (5, 64), (77, 512), (33, 513), (9, 1000), (6, 1025), (7, 2048), (4, 4093), (5, 8192), (3, 8193), (4, 9000),
         (2, 32768), (1500, 40)]
COMBOS = [(post, pre, gate, p) for post, pre in ((0, 0), (1, 0), (0, 1), (1, 1)) for gate in ("none", "vector", "rows")
          for p in (0.0, 0.25)]


@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_residual_norm(dev, kind, dtype, rows, cols):
    from paper_2107_03356_amd import nn
    say("residual norm", kind, dtype, rows, cols)
    eps, at, tiny, pad = 1e-5, (77, -3), TINY[dtype], cols % 4
    t = lambda seed, **kw: rand(dev, seed, rows, cols, dtype=dtype, pad=pad, **kw)   # noqa: E731
    y, r, full = t(1, scale=2.0, at=0.3), t(2, at=-0.5), t(3, scale=0.2, at=0.6)
    wt = F32 if rows % 2 else dtype
    w1, w2, gv = (rand(dev, s, cols, dtype=wt, at=1, scale=0.2) for s in (4, 5, 6))
    b1, b2 = (rand(dev, s, cols, dtype=wt, scale=0.3) if kind == "layer" else None for s in (7, 8))
    zero = torch.zeros(cols, dtype=torch.float64, device=dev)
    wide = lambda w, b: (w.double(), zero if b is None else b.double())   # noqa: E731
    ds, dh = t(9), t(10)
    mask = drop_factor(rows, cols, 0.25, at).to(dev)
    for n, (post, pre, gate, p) in enumerate(COMBOS):
        res, scale = (r, 0.7) if n % 3 else (None, 1.0)
        what = (post, pre, gate, p, scale)
        g = {"none": None, "vector": gv, "rows": full}[gate]
        g64 = torch.ones((), dtype=torch.float64, device=dev) if g is None else g.double()
        f = mask if p else torch.ones_like(mask)
        kw = dict(post=(w1, b1) if post else None, pre=(w2, b2) if pre else None, gate=g, scale=scale, p=p,
                  at=torch.tensor(at, device=dev) if p else None, kind=kind)
        one, two = (wide(w1, b1) if post else None), (wide(w2, b2) if pre else None)
        want = residual64(y.double(), None if res is None else res.double(), one, two, g64, scale, f, kind, eps)
        o = nn.residual_norm_forward(y, res, eps=eps, pack=bool(pre), **kw)
        if o.s is not y:
            holds(o.s, want["s"][0], rounded(*want["s"], dtype, tiny), (what, "s"))
        if pre:
            holds(o.h, want["h"][0], rounded(*want["h"], dtype, tiny), (what, "h"))
            copy_holds(o.copy, *want["xhat"], (what, "copy"))
            plain = nn.residual_norm_forward(y, res, eps=eps, stats=False, **kw)
            assert plain.pre is None and torch.equal(plain.h, o.h) and torch.equal(plain.s, o.s)
        # the backward pass, from what the forward pass gave
        none = torch.zeros((), dtype=torch.float64, device=dev)
        column = lambda st, on, i: none if not on or st[i] is None else st[i].double()[:, None]   # noqa: E731
        stats = [column(o.post, post, 0), column(o.post, post, 1), column(o.pre, pre, 0), column(o.pre, pre, 1)]
        for copy in (False, True) if pre else (False,):
            for d in (ds, None) if pre else (ds,):
                back = residual_back64(None if d is None else d.double(), dh.double() if pre else None, y.double(), o.s.double(),
                                       stats, one, two, g64, gate == "rows", scale, f, kind,
                                       unpack64(o.copy.q, o.copy.s) if copy else None)
                got = nn.residual_norm_backward(d, dh if pre else None, y, o.copy if copy else o.s, o.post, o.pre, **kw)
                holds(got.dy, back["dy"][0], rounded(*back["dy"], dtype, tiny), (what, "dy"))
                holds(got.dresidual, back["dr"][0], rounded(*back["dr"], dtype, tiny), (what, "dresidual"))
                pairs = [("dpost_w", got.dpost[0], post), ("dpost_b", got.dpost[1], post and kind == "layer"),
                         ("dpre_w", got.dpre[0], pre), ("dpre_b", got.dpre[1], pre and kind == "layer"),
                         ("dgate", got.dgate, g is not None)]
                for name, value, on in pairs:
                    assert (value is not None) == bool(on), (what, name)
                    if on:
                        holds(value, back[name][0], rounded(*back[name], value.dtype, TINY[value.dtype]), (what, name))


def test_residual_norm_in_place(dev):
    """s over y or the residual, dy and dresidual over ds and dh, as the header allows."""
    from paper_2107_03356_amd import _binding as B
    from paper_2107_03356_amd import nn
    say("residual in place")
    for rows, cols in ((300, 100), (700, 1000), (40, 9000)):
        y, r, ds, dh = (rand(dev, s, rows, cols, dtype=BF16) for s in (1, 2, 3, 4))
        w1, w2 = rand(dev, 5, cols, at=1), rand(dev, 6, cols, at=1)
        o = nn.residual_norm_forward(y, r, post=(w1, None), pre=(w2, None))
        g = nn.residual_norm_backward(ds, dh, y, o.s, o.post, o.pre, post=(w1, None), pre=(w2, None))
        st = torch.cuda.current_stream().cuda_stream
        for s_at in ("y", "r"):
            t = {"y": y.clone(), "r": r.clone()}
            h = torch.empty_like(y)
            assert B.mfac_residual_norm(
                B.MFAC_BF16, B.MFAC_F32, B.MFAC_NORM_POST | B.MFAC_NORM_PRE, rows, cols, t["y"].data_ptr(), cols, w1.data_ptr(),
                None, None, None, 0, t["r"].data_ptr(), cols, 1.0, 0.0, None, w2.data_ptr(), None, 1e-6, t[s_at].data_ptr(),
                cols, h.data_ptr(), cols, None, None, None, None, None, 0, None, st) == B.MFAC_OK
            assert torch.equal(t[s_at], o.s) and torch.equal(h, o.h)
        a, b = ds.clone(), dh.clone()
        assert B.mfac_residual_norm_bwd(
            B.MFAC_BF16, B.MFAC_F32, B.MFAC_NORM_POST | B.MFAC_NORM_PRE, rows, cols, a.data_ptr(), cols, b.data_ptr(), cols,
            y.data_ptr(), cols, None, o.post[1].data_ptr(), o.s.data_ptr(), cols, None, 0, None, None, o.pre[1].data_ptr(),
            w1.data_ptr(), None, None, None, 0, 1.0, 0.0, None, w2.data_ptr(), b.data_ptr(), cols, a.data_ptr(), cols, None, 0,
            None, None, None, None, None, None, 0, st) == B.MFAC_OK
        assert torch.equal(b, g.dy) and torch.equal(a, g.dresidual)


def test_rows_past_the_last_and_padding_stay(dev):
    """Nothing is written behind the rows or in their padding."""
    from paper_2107_03356_amd import _binding as B
    say("padding stays")
    st = torch.cuda.current_stream().cuda_stream
    for rows, cols in ((5, 100), (3, 1000), (2, 9001)):
        ld = cols + 7
        y, r = rand(dev, 1, rows, ld), rand(dev, 2, rows, ld)
        out = torch.full((2, rows + 1, ld), 7.0, device=dev)
        assert B.mfac_residual_norm(B.MFAC_F32, B.MFAC_F32, B.MFAC_NORM_PRE, rows, cols, y.data_ptr(), ld, None, None, None, None,
                                    0, r.data_ptr(), ld, 1.0, 0.0, None, None, None, 1e-6, out[0].data_ptr(), ld,
                                    out[1].data_ptr(), ld, None, None, None, None, None, 0, None, st) == B.MFAC_OK
        assert (out[:, rows] == 7).all() and (out[:, :, cols:] == 7).all() and (out[:, :rows, :cols] != 7).any(1).any()
        x, w = rand(dev, 3, rows, 64), rand(dev, 4, 2 * cols, 64)
        z = torch.full((rows + 1, 2 * cols + 7), 7.0, device=dev)
        out = torch.full((rows + 1, ld), 7.0, device=dev)
        need = B.mfac_gated_linear_workspace_bytes(B.MFAC_F32, rows, 64, cols, x.data_ptr(), 64, w.data_ptr(), 64)
        ws = torch.empty(max(need, 1), dtype=torch.uint8, device=dev)
        assert B.mfac_gated_linear(B.MFAC_F32, B.MFAC_F32, B.MFAC_ACT_SILU, rows, 64, cols, x.data_ptr(), 64, w.data_ptr(), 64,
                                   None, out.data_ptr(), ld, z.data_ptr(), z.data_ptr() + 4 * cols, 2 * cols + 7, None, None, None,
                                   None, 0, ws.data_ptr(), need, st) == B.MFAC_OK
        assert (out[rows] == 7).all() and (out[:, cols:] == 7).all() and (z[rows] == 7).all() and (z[:, 2 * cols:] == 7).all()


def test_rows_that_are_not_finite_stay_alone(dev):
    from paper_2107_03356_amd import nn
    say("rows that are not finite")
    for cols in (200, 3000, 9000):
        y, r, w = rand(dev, 1, 6, cols), rand(dev, 2, 6, cols), rand(dev, 3, cols, at=1)
        clean = nn.residual_norm_forward(y, r, post=(w, None), pre=(w, None))
        y[1, 5], y[4, 0] = float("nan"), float("inf")
        o = nn.residual_norm_forward(y, r, post=(w, None), pre=(w, None))
        for a, b in ((o.s, clean.s), (o.h, clean.h)):
            assert torch.equal(a[[0, 2, 3, 5]], b[[0, 2, 3, 5]]) and torch.isnan(a[1]).all()
        # zero rows have a norm of zero
        o = nn.residual_norm_forward(0 * r, pre=(w, None))
        assert (o.h == 0).all()


def test_values_that_are_dropped_take_no_part(dev):
    """Without a norm after the block, a NaN or an infinity of y that the mask drops comes into nothing, the gate's gradient
    among it."""
    from paper_2107_03356_amd import nn
    say("dropped values")
    for cols in (200, 9000):
        at = torch.tensor([3, 4], device=dev)
        f = drop_factor(40, cols, 0.5, (3, 4)).to(dev)
        clean, r, ds = rand(dev, 1, 40, cols), rand(dev, 2, 40, cols), rand(dev, 3, 40, cols)
        clean[f == 0] = 0
        bad = torch.where((f == 0) & (clean == 0), torch.tensor(float("nan"), device=dev), clean)
        bad[7] = torch.where(f[7] == 0, torch.tensor(float("inf"), device=dev), clean[7])
        for gate in (rand(dev, 4, cols), rand(dev, 5, 40, cols)):
            runs = []
            for y in (clean, bad):
                s = nn.residual_norm_forward(y, r, gate=gate, p=0.5, at=at).s
                g = nn.residual_norm_backward(ds, None, y, s, gate=gate, p=0.5, at=at)
                runs.append((s, g.dy, g.dresidual, g.dgate))
            assert all(torch.equal(u, v) and torch.isfinite(u).all() for u, v in zip(*runs))


@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_norms_without_parameters(dev, kind):
    """A norm without weight and bias is that of ones and zeros."""
    from paper_2107_03356_amd import nn
    say("no parameters", kind)
    for cols in (5, 300, 9000):
        y, r, ds, dh = (rand(dev, s, 20, cols) for s in (1, 2, 3, 4))
        one, zero = torch.ones(cols, device=dev), torch.zeros(cols, device=dev) if kind == "layer" else None
        runs = []
        for norm in ((None, None), (one, zero)):
            o = nn.residual_norm_forward(y, r, post=norm, pre=norm, kind=kind)
            g = nn.residual_norm_backward(ds, dh, y, o.s, o.post, o.pre, post=norm, pre=norm, kind=kind)
            runs.append((o.s, o.h, g.dy, g.dresidual))
            assert (g.dpost[0] is None) == (g.dpre[0] is None) == (norm[0] is None)
            assert (g.dpost[1] is None) == (g.dpre[1] is None) == (norm[1] is None)
        assert all(torch.equal(u, v) for u, v in zip(*runs))


def test_no_rows(dev):
    from paper_2107_03356_amd import nn
    say("no rows")
    x, w = torch.zeros(0, 64, device=dev), rand(dev, 1, 80, 64).requires_grad_()
    y = nn.gated_linear(x, w)
    assert y.shape == (0, 40)
    y.sum().backward()
    assert (w.grad == 0).all()
    v = rand(dev, 2, 64).requires_grad_()
    s, h = nn.residual_norm(x, x, pre=(v, None), post=(v, None), p=0.5)
    h.sum().backward()
    assert s.shape == h.shape == (0, 64) and (v.grad == 0).all()
    assert nn.dropout(x, 0.5).shape == (0, 64)
