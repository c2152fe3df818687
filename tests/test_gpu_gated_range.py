"""Gradients in float32 of fp16 gated layers whose dz or act(zg) zu is past fp16's range, against 64 bits."""

import math

import pytest
import torch

from gated_ref import gate_slopes64, rounded
from gpu_common import require_gpu, say
from test_gpu_gated_ops import holds, rand
from train_ref import E32, TINY, U, growth, unpack64

pytestmark = pytest.mark.gpu

F32, F16 = torch.float32, torch.float16


@pytest.fixture(scope="module")
def dev():
    return require_gpu()


def cut(bound):
    """What two fp16 parts leave of a value: 2^-36, or more by the power of two that takes the bound below 2^15."""
    return 2.0 ** (max(0, math.frexp(bound)[1] - 15) - 36)


def most(*tensors):
    return max(t.double().abs().max().item() for t in tensors)


@pytest.mark.parametrize("size", [1.0, 2.0 ** 6, 2.0 ** 12])
@pytest.mark.parametrize("rows,hid", [(1, 64), (130, 515), (333, 192), (1300, 64)])
def test_fp16_gradients_as_large_as_they_come(dev, rows, hid, size):
    """With x the identity, dw1 is dz transposed, from two parts whose factors are taken out in the sums: 2^-22 of a value and
    what a step of the second part cuts (2^-36 times the factor). dx = dz w1, small enough for fp16, from the first part."""
    from paper_2107_03356_amd import nn
    say("fp16 gradients as large as they come", rows, hid, size)
    dim, x = 40, torch.eye(rows, dtype=F16, device=dev)
    pair = rand(dev, 2, rows, hid, dtype=F16, scale=8.0), rand(dev, 3, rows, hid, dtype=F16, scale=8.0)
    copies = tuple(nn.pack8(v) for v in pair)
    dy, w2 = (rand(dev, 4, rows, dim) * size).to(F16), rand(dev, 5, dim, hid, dtype=F16, scale=4.0)
    w1 = rand(dev, 6, 2 * hid, rows, dtype=F16, scale=2.0 ** -10 / size)
    mine = (rand(dev, 7, rows, hid) * 4 * size).clamp(-6e4, 6e4).to(F16)
    zero = torch.zeros(rows, hid, dtype=torch.float64, device=dev)
    da, ed = dy.double() @ w2.double(), E32 * growth(dim) * (dy.double().abs() @ w2.double().abs())
    for z in (pair, copies):
        g64, u64 = (unpack64(v.q, v.s) for v in z) if z is copies else (v.double() for v in z)
        # an 8-bit copy's values are counted as 127 steps, twice the largest at most
        bound = 1.13 * most(g64, u64) * (2 if z is copies else 1)
        runs = []
        for need_b in (False, True):
            got = nn.gated_feed_forward_backward(dy, x, w1, w2, z, grad_dtype=F32, need=(True, True, need_b, True, False))
            runs.append((da, ed, bound * dim * most(dy) * most(w2), *got[:3]))
        runs.append((mine.double(), zero, bound * most(mine),
                     *nn.gated_linear_backward(mine, x, w1, z, grad_dtype=F32, need=(True, True, True))))
        for d, err, b, dx, dw1, db in runs:
            (dg, eg), (du, eu), _ = gate_slopes64("silu", g64, u64, d, err)
            dz, e = torch.cat([dg, du], 1), torch.cat([eg, eu], 1)
            holds(dw1, dz.t(), (1.02 * U[F16] ** 2 * dz.abs() + 1.01 * e + cut(b) + 2 * E32 * dz.abs()).t(), "dw1")
            want = dz @ w1.double()
            once = U[F16] * dz.abs() + 1.01 * e + cut(b) * 2.0 ** 11
            holds(dx, want, rounded(want, (once + E32 * growth(2 * hid) * dz.abs()) @ w1.double().abs(), F16, TINY[F16]), "dx")
            if db is not None:
                holds(db, dz.sum(0), e.sum(0) * 1.01 + E32 * (rows / 4 + 60) * dz.abs().sum(0) + 1e-30, "db")
    assert size < 2.0 ** 12 or most(da) > 65504 / 4   # dz is past fp16's range: a pre-activation above 4 is among them


@pytest.mark.parametrize("rows,hid", [(1, 64), (40, 64), (130, 100)])
def test_fp16_activation_as_large_as_it_comes(dev, rows, hid):
    """With dy the identity, dw2 is act(zg) zu, up to the square of fp16's largest value."""
    from paper_2107_03356_amd import nn
    say("fp16 activation as large as it comes", rows, hid)
    dy, w2 = torch.eye(rows, dtype=F16, device=dev), rand(dev, 1, rows, hid, dtype=F16)
    z = rand(dev, 2, rows, hid, dtype=F16, scale=4000.0), rand(dev, 3, rows, hid, dtype=F16, scale=4000.0)
    for act in ("none", "gelu", "silu"):
        _, _, (a, e) = gate_slopes64(act, z[0].double(), z[1].double(), w2.double(), 0 * w2.double())
        x, w1 = rand(dev, 4, rows, 24, dtype=F16), rand(dev, 5, 2 * hid, 24, dtype=F16)
        for need in ((False, False, False, True, False), (False, True, False, True, False)):
            got = nn.gated_feed_forward_backward(dy, x, w1, w2, z, act, grad_dtype=F32, need=need)[3]
            holds(got, a, 1.02 * U[F16] ** 2 * a.abs() + 1.01 * e + cut(most(z[0]) * most(z[1])) + 2 * E32 * a.abs(), (act, need))
    assert a.abs().max() > 65504


@pytest.mark.parametrize("row", [0, 1000, 20011, 39999])
def test_one_large_value_is_found_in_any_row(dev, row):
    """x picks one row of dz, whose pre-activation alone is large."""
    from paper_2107_03356_amd import nn
    say("one large value", row)
    rows, dim, hid = 40000, 40, 64
    x = torch.zeros(rows, 8, dtype=F16, device=dev)
    x[row, 3] = 1
    dy, w2 = rand(dev, 1, rows, dim, dtype=F16), rand(dev, 2, dim, hid, dtype=F16, scale=2.0)
    zg, zu = rand(dev, 3, rows, hid, dtype=F16), rand(dev, 4, rows, hid, dtype=F16)
    zu[row, 5] = 6e4
    for z in ((zg, zu), (nn.pack8(zg), nn.pack8(zu))):
        got = nn.gated_feed_forward_backward(dy, x, None, w2, z, "none", grad_dtype=F32, need=(False, True, False, True, False))[1]
        u = zu if z[1] is zu else nn.unpack8(z[1])
        da = dy[row].double() @ w2.double()
        want = da * u[row].double()
        err = E32 * growth(dim) * (dy[row].double().abs() @ w2.double().abs()) * u[row].double().abs()
        b = 1.13 * most(zg, zu) * 2 * dim * most(dy) * most(w2)
        holds(got[:hid, 3], want, 1.02 * U[F16] ** 2 * want.abs() + 1.01 * err + cut(b) + 6 * E32 * want.abs(), row)
        assert want.abs().max() > 65504


def test_an_infinity_stays_where_it_belongs(dev):
    """An infinite weight makes its own channel's gradients infinite or NaN, and takes no digits from the others'."""
    from paper_2107_03356_amd import nn
    say("fp16 infinite weight")
    rows, dim, hid = 70, 48, 128
    dy, x = rand(dev, 1, rows, dim, dtype=F16), rand(dev, 2, rows, dim, dtype=F16)
    w1, w2 = rand(dev, 3, 2 * hid, dim, dtype=F16), rand(dev, 4, dim, hid, dtype=F16)
    z = rand(dev, 5, rows, hid, dtype=F16), rand(dev, 6, rows, hid, dtype=F16)
    args = dict(grad_dtype=F32, need=(False, True, False, True, False))
    clean = nn.gated_feed_forward_backward(dy, x, w1, w2, z, **args)
    w2[3, 17] = float("inf")
    got = nn.gated_feed_forward_backward(dy, x, w1, w2, z, **args)
    others = [i for i in range(2 * hid) if i % hid != 17]
    assert torch.equal(got[1][others], clean[1][others]) and torch.equal(got[3], clean[3])
    assert not torch.isfinite(got[1][[17, 17 + hid]]).any()


@pytest.mark.parametrize("rows,dim,hid", [(1, 64, 96), (130, 72, 200), (700, 264, 515), (260, 2056, 261), (70, 2056, 320), (3000, 264, 515)])
def test_gated_feed_forward_backward_of_fp16(dev, rows, dim, hid):
    """The whole backward pass in fp16, against the formulas with dz and a counted as the call rounds them."""
    from test_gpu_gated_ops import test_gated_feed_forward_backward as of_type
    of_type(dev, F16, rows, dim, hid)


def test_captured_factors_follow_their_inputs(dev):
    """A captured pass takes the factors anew at each replay, from small inputs and from large ones."""
    from paper_2107_03356_amd import nn
    say("captured factors")
    rows, dim, hid = 300, 72, 192
    x, dy = (torch.empty(rows, dim, dtype=F16, device=dev) for _ in range(2))
    w1, w2 = rand(dev, 1, 2 * hid, dim, dtype=F16, scale=2.0 ** -12), rand(dev, 2, dim, hid, dtype=F16)
    z = tuple(torch.empty(rows, hid, dtype=F16, device=dev) for _ in range(2))

    def fill(turn):
        for i, t in enumerate((x, dy, *z)):
            t.copy_(rand(dev, 10 * turn + i, *t.shape, scale=(1.0, 200.0, 2.0 ** -9, 1000.0)[turn]))

    def run():
        return nn.gated_feed_forward_backward(dy, x, w1, w2, z, grad_dtype=F32, need=(True, True, False, True, False))

    fill(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = run()
    for turn in (1, 2, 3, 0, 3):
        fill(turn)
        graph.replay()
        torch.cuda.synchronize()
        got, want = [held[i].clone() for i in (0, 1, 3)], run()
        assert all(torch.equal(a, want[i]) for a, i in zip(got, (0, 1, 3)))
        # dx is of fp16: with values of 1000 its standard deviation is 8.5e3 * 1e3 * 0.6 * 2^-12 * sqrt(384) = 2.4e4
        assert torch.isfinite(got[1]).all() and torch.isfinite(got[2]).all()
