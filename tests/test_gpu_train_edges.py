"""The training operators where arguments, values and sizes are out of the ordinary."""

import pytest
import torch

from gpu_common import require_gpu, say
from train_cases import PRODUCTS, layer, runs
from train_ref import E32, TINY, U, act64, act_error, growth, off, pack64, unpack64  # noqa: F401

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def dev():
    return require_gpu()


def rand(dev, seed, *shape, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g, dtype=torch.float64) * scale).to(dev)


def holds(got, want, bound, what):
    o = off(got, want, bound)
    assert o <= 1, (what, o)


# ---------------------------------------------------------------- arguments
def test_weight_gradient_with_db_of_any_stride(dev):
    from paper_2107_03356_amd import nn
    say("db strides")
    dz, p = rand(dev, 1, 50, 40).to(BF16), nn.pack8(rand(dev, 2, 50, 64).to(BF16))
    g, b = rand(dev, 3, 64).to(F32), rand(dev, 4, 64).to(F32)
    _, _, db = nn.act_backward(dz)
    wide = torch.full((40, 3), float("nan"), device=dev)
    wide[:, 1] = db
    want = nn.linear_backward_weight(dz, p, (g, b), db)
    assert torch.equal(nn.linear_backward_weight(dz, p, (g, b), wide[:, 1]), want)
    for bad in (db.cpu(), db.double(), db[:39], None):
        with pytest.raises(ValueError):
            nn.linear_backward_weight(dz, p, (g, b), bad)


# ---------------------------------------------------------------- values
ENDS = [0.0, 1e-30, -1e-30, 5.0, -5.0, 30.0, -30.0, 300.0, -300.0, 1e4, -1e4, 1e15, -1e15, 1e19, -1e19, 1e20, -1e20, 3e38, -3e38,
        float("inf")]


def end_values(dev, act):
    """Pre-activations far out, and the infinities that the activation's definition has values for."""
    z = torch.tensor(ENDS + [float("-inf") if act == "relu" else 0.0] + [1.0] * 11, dtype=F32, device=dev)
    return z, act64(act, z.double())


def end_bound(z, a):
    z = z.clamp(-1e39, 1e39)   # infinities have no size of their own
    return act_error(z) * torch.clamp(a.abs() * 1e9, max=1.0) + 1e-30 + E32 * a.abs()


# one token, a tile of the products, and a long sum in parts
@pytest.mark.parametrize("rows,cin", [(3, 64), (40, 64), (40, 8192)])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("act", ["relu", "gelu", "gelu_tanh", "silu"])
def test_activations_far_out_and_at_infinity(dev, act, dtype, rows, cin):
    from paper_2107_03356_amd import nn
    say("activations far out", act, dtype, rows, cin)
    z, (a64, _) = end_values(dev, act)
    x, w = torch.zeros(rows, cin, dtype=dtype, device=dev), rand(dev, 1, z.numel(), cin).to(dtype)
    y = nn.linear_forward(x, w, z, act)   # 0 + z
    want = a64.to(dtype).double().expand(rows, -1)
    bound = end_bound(z.double(), torch.nan_to_num(a64, posinf=0.0)) + U[dtype] * torch.nan_to_num(a64.abs(), posinf=0.0)
    holds(y, want, bound.expand(rows, -1), "y")
    same = torch.isinf(want)
    assert torch.equal(y.double()[same], want[same])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("act", ["relu", "gelu", "gelu_tanh", "silu"])
def test_slopes_far_out(dev, act, dtype):
    """Far out a slope is 0 or 1, however large z * z is; act(z) as the forward pass gives it, +inf at +inf."""
    from paper_2107_03356_amd import nn
    say("slopes far out", act, dtype)
    z, _ = end_values(dev, act)
    z = z.to(dtype)[None]
    a64, s64 = act64(act, z.double())
    dz, a, _ = nn.act_backward(torch.ones_like(z), z, act, want_a=True)
    at = torch.isfinite(z)
    holds(dz[at], s64[at], act_error(z.double()[at]).clamp(max=1e-6) + U[dtype] * s64[at].abs(), "slope")
    a64 = a64.to(dtype).double()
    holds(a, a64, end_bound(z.double(), torch.nan_to_num(a64, posinf=0.0)) + U[dtype] * torch.nan_to_num(a64.abs(), posinf=0.0), "a")


# ---------------------------------------------------------------- which gradients
@pytest.mark.parametrize("act", ["none", "gelu"])
@pytest.mark.parametrize("copy8", [False, True])
def test_linear_whose_residual_alone_needs_a_gradient(dev, act, copy8):
    from paper_2107_03356_amd import nn
    say("residual alone", act, copy8)
    x, w, b = rand(dev, 1, 20, 64).to(BF16), rand(dev, 2, 48, 64).to(BF16), rand(dev, 3, 48).to(F32)
    r = rand(dev, 4, 20, 48).to(BF16).requires_grad_()
    dy = rand(dev, 5, 20, 48).to(BF16)
    nn.linear(x, w, b, act=act, residual=r, copy8=copy8).backward(dy)
    assert torch.equal(r.grad, dy)


def test_gradient_of_a_residual_of_other_dimensions(dev):
    """A residual whose rows lie in other leading dimensions than y's gets its gradient in its own shape."""
    from paper_2107_03356_amd import nn
    say("residual dimensions")
    x, w = rand(dev, 1, 4, 10, 64).to(BF16), rand(dev, 2, 48, 64).to(BF16)
    dy = rand(dev, 5, 4, 10, 48).to(BF16)
    for shape in ((40, 48), (2, 20, 48), (4, 10, 48)):
        r = rand(dev, 4, *shape).to(BF16).requires_grad_()
        y = nn.linear(x, w, residual=r)
        assert y.shape == dy.shape
        y.backward(dy)
        assert torch.equal(r.grad, dy.view(shape))


@pytest.mark.parametrize("copy8", [False, True])
def test_inference_gives_the_same_and_keeps_nothing(dev, copy8):
    from paper_2107_03356_amd import nn
    say("inference", copy8)
    torch.manual_seed(2)
    rows, dim, hid = 2048, 128, 4096
    block, lin = nn.FeedForward(dim, hid, copy8=copy8, device=dev), nn.Linear(dim, hid, act="silu", copy8=copy8, device=dev)
    norm = nn.LayerNorm(dim, copy8=copy8, device=dev)
    x = rand(dev, 1, rows, dim).to(BF16)
    trained = [m(x).detach() for m in (block, lin, norm)]
    kept = []
    with torch.no_grad(), torch.autograd.graph.saved_tensors_hooks(lambda t: kept.append(t) or t, lambda t: t):
        assert all(torch.equal(m(x), t) for m, t in zip((block, lin, norm), trained))
    assert not kept

    def by_hand(x):
        c1, c2 = block.up.weight.to(BF16), block.down.weight.to(BF16)
        a = nn.linear_forward(nn.layer_norm_forward(x, block.norm.weight, block.norm.bias)[0], c1, block.up.bias, "gelu")
        return nn.linear_forward(a, c2, block.down.bias, residual=x)

    peaks = []
    for f in (by_hand, block):   # z or its copy, rows x hid, would come on top
        torch.cuda.synchronize()
        torch.cuda.reset_peak_memory_stats()
        before = torch.cuda.memory_allocated()
        with torch.no_grad():
            f(x)
        peaks.append(torch.cuda.max_memory_allocated() - before)
    assert peaks[1] <= peaks[0], peaks


@pytest.mark.parametrize("copy8", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_block_gradients_one_by_one_are_those_of_all(dev, dtype, copy8):
    from paper_2107_03356_amd import nn
    say("block gradients one by one", dtype, copy8)
    dy = rand(dev, 9, 4, 50, 72).to(dtype)

    def gradients(needed):
        t = [rand(dev, 1, 4, 50, 72).to(dtype), 1 + 0.2 * rand(dev, 2, 72).to(F32), rand(dev, 3, 72).to(F32),
             rand(dev, 4, 200, 72, scale=0.1).to(F32), rand(dev, 5, 200).to(F32), rand(dev, 6, 72, 200, scale=0.1).to(F32),
             rand(dev, 7, 72).to(F32)]
        for i in needed:
            t[i].requires_grad_()
        nn.feed_forward(*t, act="gelu_tanh", copy8=copy8).backward(dy)
        assert [v.grad is not None for v in t] == [i in needed for i in range(7)]
        return {i: t[i].grad for i in needed}

    every = gradients(range(7))
    for needed in [[i] for i in range(7)] + [[1, 2], [3, 5], [0, 4, 6]]:
        for i, g in gradients(needed).items():
            assert torch.equal(g, every[i]), (needed, i)


def test_fp32_products_of_the_largest_values(dev):
    """Finite fp32 values near the largest have finite products, whichever kernel forms them."""
    from paper_2107_03356_amd import nn
    say("largest fp32 values")
    big = torch.finfo(F32).max
    for rows in (5, 40):
        x, w = rand(dev, 1, rows, 72).to(F32), (rand(dev, 2, 24, 72) * 2.0 ** -30).to(F32)
        x[2, 7], x[3, 0], x[4, 71] = big, -big, 3.395e38
        z64 = x.double() @ w.double().t()
        bound = E32 * (growth(72) + 1) * (x.double().abs() @ w.double().abs().t())
        holds(nn.linear_forward(x, w), z64, bound, "y")
        # as the gradient that both products of the backward pass take
        dx = nn.linear_backward_input(x, w.t().contiguous())
        holds(dx, z64, bound, "dx")
        t = rand(dev, 3, rows, 24).to(F32) * 2.0 ** -30
        dw = nn.linear_backward_weight(x, t)
        holds(dw, x.double().t() @ t.double(), E32 * (growth(rows) + 1) * (x.double().abs().t() @ t.double().abs()), "dw")


def test_fp32_infinities_spoil_their_row_only(dev):
    """An infinite fp32 value: what the definition gives up to 16 rows; from three bf16 parts its products are not
    finite. Other rows stay as they are."""
    from paper_2107_03356_amd import nn
    say("fp32 infinities")
    w = rand(dev, 2, 24, 72).to(F32)
    for rows in (16, 17):
        x = rand(dev, 1, rows, 72).to(F32)
        clean = nn.linear_forward(x, w)
        x[2, 7] = float("inf")
        y = nn.linear_forward(x, w)
        assert torch.equal(y[:2], clean[:2]) and torch.equal(y[3:], clean[3:])
        assert not torch.isfinite(y[2]).any()
        if rows <= 16:
            assert torch.equal(y[2].double(), (x.double() @ w.double().t())[2])


def test_fp32_products_of_single_values(dev):
    """One product a sum: off by what the three left out come to, 2^-24 (1 + 2^-10) of it, and by the additions' cuts, a
    unit of 2^-23 for the last and 2^-8 of one for those before."""
    from paper_2107_03356_amd import nn
    say("single products")
    x = 1 + torch.rand(600, 1, generator=torch.Generator().manual_seed(1)).to(dev)
    x[0] = 1.0038986
    want = x.double() @ x.double().t()
    holds(nn.linear_forward(x, x), want, E32 * (1 + 2.0 ** -10 + 2 * (1 + 5 * 2.0 ** -8)) * want, "y")


# ---------------------------------------------------------------- every kernel of the large products, with every epilogue
TYPE = {"f32": F32, "bf16": BF16, "f16": F16}
KERNELS = [(t, size, want) for size, want, types in PRODUCTS for t in types]


def matrix(dev, seed, dtype, *shape, scale=1.0):
    g = torch.Generator(device=dev).manual_seed(seed)
    return (torch.randn(*shape, generator=g, device=dev) * scale).to(dtype)


@pytest.mark.parametrize("t,size,want", KERNELS)
def test_forward_product_of_each_kernel(dev, t, size, want):
    from paper_2107_03356_amd import _binding as B
    from paper_2107_03356_amd import nn
    say("forward product", t, size, want)
    dtype = TYPE[t]
    rows, cin, cout = layer(B.MFAC_PRODUCT_FORWARD, *size)
    assert runs(t, t, B.MFAC_PRODUCT_FORWARD, size, want)
    x, w = matrix(dev, 1, dtype, rows, cin), matrix(dev, 2, dtype, cout, cin, scale=cin ** -0.5)
    b, res = matrix(dev, 3, F32, cout, scale=0.5), matrix(dev, 4, dtype, rows, cout)
    z64 = x.double() @ w.double().t() + b.double()
    ze = E32 * (growth(cin) * (x.double().abs() @ w.double().abs().t()) + 2 * b.double().abs())
    tiny = TINY[dtype]
    for act in ("none", "relu", "gelu", "gelu_tanh", "silu"):
        a64, _ = act64(act, z64)
        err = 1.2 * ze + (act_error(z64) if act != "none" else 0)
        holds(nn.linear_forward(x, w, b, act), a64, U[dtype] * a64.abs() + err + tiny, act)
    a64 += res.double()
    bound = U[dtype] * a64.abs() + err + E32 * a64.abs() + tiny
    y = nn.linear_forward(x, w, b, act, residual=res)
    holds(y, a64, bound, "y + res")
    yz, z = nn.linear_forward(x, w, b, act, residual=res, keep="z")
    assert torch.equal(yz, y)
    holds(z, z64, U[dtype] * z64.abs() + ze + tiny, "z")
    y8, p = nn.linear_forward(x, w, b, act, residual=res, keep="pack8")
    assert torch.equal(y8, y)
    step = torch.exp2(p.s.double() - 127)
    holds(nn.unpack8(p), z64, step.repeat_interleave(32, 1)[:, :cout] / 2 + ze, "copy of z")
    most = torch.nn.functional.pad(z64.abs() + ze, (0, -cout % 32)).view(rows, -1, 32).amax(2)
    assert (step <= torch.clamp(2 * most / 127, min=2.0 ** -126)).all()
    z64 -= b.double()
    holds(nn.linear_forward(x, w), z64, U[dtype] * z64.abs() + ze + tiny, "no bias")


@pytest.mark.parametrize("t,size,want", KERNELS)
def test_input_product_of_each_kernel(dev, t, size, want):
    from paper_2107_03356_amd import _binding as B
    from paper_2107_03356_amd import nn
    say("input product", t, size, want)
    dtype = TYPE[t]
    rows, cin, cout = layer(B.MFAC_PRODUCT_INPUT, *size)
    assert runs(t, t, B.MFAC_PRODUCT_INPUT, size, want)
    dz, w = matrix(dev, 5, dtype, rows, cout), matrix(dev, 6, dtype, cout, cin, scale=cout ** -0.5)
    add = matrix(dev, 7, dtype, rows, cin)
    want64 = dz.double() @ w.double()
    err = E32 * growth(cout) * (dz.double().abs() @ w.double().abs()) + TINY[dtype]
    holds(nn.linear_backward_input(dz, w), want64, U[dtype] * want64.abs() + err, "dx")
    want64 += add.double()
    holds(nn.linear_backward_input(dz, w, add=add), want64, (U[dtype] + E32) * want64.abs() + err, "dx + add")


@pytest.mark.parametrize("t,size,want", KERNELS)
def test_weight_product_of_each_kernel(dev, t, size, want):
    from paper_2107_03356_amd import _binding as B
    from paper_2107_03356_amd import nn
    say("weight product", t, size, want)
    dtype = TYPE[t]
    rows, cin, cout = layer(B.MFAC_PRODUCT_WEIGHT, *size)
    dz, x = matrix(dev, 8, dtype, rows, cout), matrix(dev, 9, dtype, rows, cin)
    gamma, beta = 1 + matrix(dev, 10, F32, cin, scale=0.2), matrix(dev, 11, F32, cin, scale=0.3)
    d, dm = dz.double(), dz.double().abs()
    want64 = d.t() @ x.double()
    err = E32 * growth(rows) * (dm.t() @ x.double().abs())
    gtypes = [("f32", F32)] + ([(t, dtype)] if t != "f32" else [])
    for g, gtype in gtypes:
        assert runs(t, g, B.MFAC_PRODUCT_WEIGHT, size, want)
        holds(nn.linear_backward_weight(dz, x, grad_dtype=gtype), want64, U[gtype] * want64.abs() + err + TINY[gtype], "dw")
    p = nn.pack8(x)
    xq = unpack64(p.q, p.s)
    _, _, db = nn.act_backward(dz)
    want64 = d.t() @ (xq * gamma.double() + beta.double())
    # products, the affine part's three roundings, and db's own sum
    err = E32 * 2 * growth(rows) * (dm.t() @ (xq.abs() * gamma.double().abs() + beta.double().abs()))
    for g, gtype in gtypes:
        got = nn.linear_backward_weight(dz, p, (gamma, beta), db, gtype)
        holds(got, want64, U[gtype] * want64.abs() + err + TINY[gtype], "dw from the copy")


def test_gelu_keeps_its_digits_in_the_tail(dev):
    """z Phi(z) for negative z is a product of small numbers: its error is relative to itself. By z^2 / 2 of the
    exponential's argument, which has three roundings (1.5 z^2 units of 2^-24, 2 taken), and about ten roundings of the
    rest, which the polynomial's terms of both signs and the reciprocal's slope raise to 40."""
    from paper_2107_03356_amd import nn
    say("gelu tail")
    z = torch.linspace(-9, 9, 4001, dtype=F32, device=dev)
    a64, s64 = act64("gelu", z.double())
    unit = E32 * (40 + 2 * z.double().square())
    for rows in (1, 40):
        y = nn.linear_forward(torch.zeros(rows, 64, device=dev), rand(dev, 1, 4001, 64).to(F32), z, "gelu")
        holds(y, a64.expand(rows, -1), (unit * a64.abs() + TINY[F32]).expand(rows, -1), "act")
    dz, a, _ = nn.act_backward(torch.ones(1, 4001, device=dev), z[None], "gelu", want_a=True)
    holds(a[0], a64, unit * a64.abs() + TINY[F32], "a")
    zd = z.double()
    density = zd.abs() * torch.exp(-zd * zd / 2) / (2 * torch.pi) ** 0.5
    holds(dz[0], s64, unit * (density + (s64 - zd.sign() * density).abs()) + TINY[F32], "slope")
