"""Layer norm on the GPU, forward and backward, against its definition in 64 bits, with
the bounds of ops_reference (counted roundings)."""
import pytest
import torch

from paper_2110_02861_amd import bq, nn
from tests import ops_reference as ref
from tests.gpu_helpers import needs_gpu, say

pytestmark = [pytest.mark.gpu, needs_gpu]

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
TYPES = [(F32, F32), (F16, F16), (BF16, BF16), (F16, F32), (BF16, F32)]
EPS = 1e-5


def normal(shape, seed, std=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.empty(shape, device="cuda").normal_(0.0, std, generator=g)


def inputs(rows, cols, xt, wt, seed=0, offset=0.25):
    x = normal((rows, cols), seed) + offset
    x[:, cols // 2] *= 20.0
    return (x.to(xt), (1 + normal((cols,), seed + 1, 0.1)).to(wt),
            normal((cols,), seed + 2, 0.05).to(wt), normal((rows, cols), seed + 3, 0.01).to(xt))


def check_all(x, w, b, dy, wt, stats=None, eps=EPS):
    """Forward and backward of the matrix x through bq, against 64 bits."""
    y, mean, rstd = bq.bq_layer_norm_forward(x, w, b, eps, stats=True)
    yr, xh, mr, rr = ref.layer_norm(x, w, b, eps)
    n = x.shape[1]
    ref.check(y, yr, ref.forward_bound(yr, xh, w, x.dtype, n), "y")
    plain = bq.bq_layer_norm_forward(x, w, b, eps)
    assert torch.equal(plain, y)
    dx, dw, db = bq.bq_layer_norm_backward(dy, x, w, mean, rstd, param_dtype=None if w is not None
                                           else wt)
    want = ref.layer_norm_grads(dy, xh, rr, w)
    bounds = ref.backward_bounds(dy, xh, mr, rr, w, *want, x.dtype, wt)
    for got, r, e, what in zip((dx, dw, db), want, bounds, ("dx", "dw", "db")):
        assert got.dtype == (x.dtype if what == "dx" else wt)
        ref.check(got, r, e, what)
    return y, dx, dw, db


@pytest.mark.parametrize("types", TYPES, ids=str)
@pytest.mark.parametrize("cols", [1, 2, 7, 63, 64, 257, 512, 1001, 1024, 1600, 2048, 2051, 4100,
                                  8192, 16385, 33000])
def test_sizes(cols, types):
    xt, wt = types
    for rows in (1, 5, 700 if cols < 5000 else 67):
        say("layer norm", rows, cols, types)
        check_all(*inputs(rows, cols, xt, wt, seed=cols), wt)


@pytest.mark.parametrize("rows", [0, 1, 3, 4, 511, 513, 2049, 20011])
def test_rows(rows):
    say("layer norm rows", rows)
    x, w, b, dy = inputs(rows, 96, BF16, F32)
    y, dx, dw, db = check_all(x, w, b, dy, F32)
    if rows == 0:
        assert not dw.any() and not db.any()


@pytest.mark.parametrize("cols", [300, 5000, 40000])
def test_without_parameters(cols):
    x, w, b, dy = inputs(9, cols, F16, F32)
    say("layer norm without parameters", cols)
    check_all(x, None, None, dy, F32)
    check_all(x, None, None, dy, F16)
    check_all(x, w, None, dy, F32)
    y = bq.bq_layer_norm_forward(x, None, b, EPS)
    yr, xh, _, _ = ref.layer_norm(x, None, b, EPS)
    ref.check(y, yr, ref.forward_bound(yr, xh, None, F16, cols), "y")


@pytest.mark.parametrize("xt", [F32, BF16])
@pytest.mark.parametrize("cols", [100, 1601, 3000])
def test_strided_and_unaligned_rows(cols, xt):
    wide = normal((37, cols + 13), 5).to(xt)
    wide_dy = normal((37, cols + 5), 6, 0.01).to(xt)
    buf = normal((2 * cols + 2,), 7)
    w, b = (1 + buf[1:cols + 1]).contiguous(), buf[cols + 1:2 * cols + 1]
    for off in (0, 1, 3):
        say("layer norm strided", cols, xt, off)
        x, dy = wide[:, off:off + cols], wide_dy[:, off:off + cols]
        a = check_all(x, w, b, dy, F32)
        c = check_all(x.contiguous(), w, b, dy.contiguous(), F32)
        for s, t in zip(a, c):
            assert torch.equal(s, t)
    one = wide[:1, :cols].expand(21, cols)  # a row stride of zero
    check_all(one, w, b, normal((21, cols), 9, 0.01).to(xt), F32)


@pytest.mark.parametrize("cols", [512, 6000, 50000])
def test_far_from_zero(cols):
    """A mean 10^4 times the spread costs nothing in the forward pass: the mean's rounding
    is taken out again."""
    x, w, b, dy = inputs(11, cols, F32, F32, offset=1e4)
    say("layer norm far from zero", cols)
    check_all(x, w, b, dy, F32)


def test_constant_rows_and_eps():
    x = torch.full((3, 1000), 7.25, device="cuda")
    b = normal((1000,), 1)
    say("layer norm constant rows")
    assert torch.equal(bq.bq_layer_norm_forward(x, None, b, EPS), b.expand(3, 1000))
    # eps 0 and no variance: 0 / 0, as the formula has it
    assert bq.bq_layer_norm_forward(x, None, b, 0.0).isnan().all()
    x, w, b, dy = inputs(5, 300, F32, F32)
    check_all(x, w, b, dy, F32, eps=0.0)
    check_all(x * 1e-4, w, b, dy, F32, eps=1e-3)


@pytest.mark.parametrize("xt", [F32, BF16])
@pytest.mark.parametrize("rows,cols", [(600, 16384), (600, 16392), (250, 70003)])
def test_workspace_of_long_rows(rows, cols, xt):
    """A workspace of the size asked for is enough, and nothing behind it is written."""
    x, w, b, dy = inputs(rows, cols, xt, F32)
    _, mean, rstd = bq.bq_layer_norm_forward(x, w, b, EPS, stats=True)
    need = bq.lib().bq_layer_norm_workspace_bytes(rows, cols)
    ws = torch.full((need + 4096,), 77, dtype=torch.uint8, device="cuda")
    say("layer norm workspace", rows, cols, xt)
    got = bq.bq_layer_norm_backward(dy, x, w, mean, rstd, workspace=ws[:need])
    assert bool((ws[need:] == 77).all())
    _, xh, mr, rr = ref.layer_norm(x, w, b, EPS)
    want = ref.layer_norm_grads(dy, xh, rr, w)
    for g, r, e, what in zip(got, want, ref.backward_bounds(dy, xh, mr, rr, w, *want, xt, F32),
                             ("dx", "dw", "db")):
        ref.check(g, r, e, what)


@pytest.mark.parametrize("xt", [F32, BF16])
def test_gradients_of_large_constant_rows(xt):
    """Rows of 2^120, whose mean is exact: the mean times rstd is above fp32's largest value,
    xh is 0."""
    x = torch.full((5, 32), 2.0 ** 120, device="cuda", dtype=xt)
    w, dy = 1 + normal((32,), 1, 0.1), normal((5, 32), 2, 0.01).to(xt)
    _, mean, rstd = bq.bq_layer_norm_forward(x, w, None, EPS, stats=True)
    say("layer norm large constant rows", xt)
    got = bq.bq_layer_norm_backward(dy, x, w, mean, rstd)
    _, xh, mr, rr = ref.layer_norm(x, w, None, EPS)
    assert not xh.any() and torch.equal(mean.double(), mr[:, 0])
    want = ref.layer_norm_grads(dy, xh, rr, w)
    # the saved mean is exact, and takes no part in the bounds
    bounds = ref.backward_bounds(dy, xh, torch.zeros_like(mr), rr, w, *want, xt, F32)
    for g, r, e, what in zip(got, want, bounds, ("dx", "dw", "db")):
        ref.check(g, r, e, what)


@pytest.mark.parametrize("cols", [200, 3000, 40000])
def test_rows_that_are_not_finite_stay_apart(cols):
    x, w, b, dy = inputs(6, cols, F32, F32)
    say("layer norm not finite", cols)
    good = bq.bq_layer_norm_forward(x, w, b, EPS)
    x[1, 3], x[4, cols - 1] = float("nan"), float("inf")
    y = bq.bq_layer_norm_forward(x, w, b, EPS)
    assert y[1].isnan().all() and y[4].isnan().all()
    for r in (0, 2, 3, 5):
        assert torch.equal(y[r], good[r])


def test_what_is_not_asked_for():
    x, w, b, dy = inputs(50, 700, BF16, F32)
    say("layer norm parts")
    _, mean, rstd = bq.bq_layer_norm_forward(x, w, b, EPS, stats=True)
    dx, dw, db = bq.bq_layer_norm_backward(dy, x, w, mean, rstd)
    only, none, none2 = bq.bq_layer_norm_backward(dy, x, w, mean, rstd, need_params=False)
    assert torch.equal(only, dx) and none is None and none2 is None
    none, dw2, db2 = bq.bq_layer_norm_backward(dy, x, w, mean, rstd, need_dx=False)
    assert none is None and torch.equal(dw, dw2) and torch.equal(db, db2)


def test_same_bits_and_other_streams():
    x, w, b, dy = inputs(3000, 1600, BF16, F32)
    _, mean, rstd = bq.bq_layer_norm_forward(x, w, b, EPS, stats=True)
    first = bq.bq_layer_norm_backward(dy, x, w, mean, rstd)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    say("layer norm on a side stream")
    y = bq.bq_layer_norm_forward(x, w, b, EPS, stream=side)
    again = bq.bq_layer_norm_backward(dy, x, w, mean, rstd, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(y, bq.bq_layer_norm_forward(x, w, b, EPS))
    for s, t in zip(first, again):
        assert torch.equal(s, t)


@pytest.mark.parametrize("types", TYPES, ids=str)
def test_autograd(types):
    xt, wt = types
    x, w, b, dy = inputs(60, 333, xt, wt)
    say("layer norm autograd", types)
    x3 = x.view(4, 15, 333).requires_grad_()
    layer = nn.LayerNorm(333, device="cuda", dtype=wt)
    with torch.no_grad():
        layer.weight.copy_(w)
        layer.bias.copy_(b)
    y = layer(x3)
    assert y.shape == x3.shape and y.dtype == xt
    y.backward(dy.view(4, 15, 333))
    yr, xh, mr, rr = ref.layer_norm(x, w, b, EPS)
    ref.check(y.view(60, 333), yr, ref.forward_bound(yr, xh, w, xt, 333), "y")
    want = ref.layer_norm_grads(dy, xh, rr, w)
    bounds = ref.backward_bounds(dy, xh, mr, rr, w, *want, xt, wt)
    for got, r, e in zip((x3.grad.view(60, 333), layer.weight.grad, layer.bias.grad), want, bounds):
        ref.check(got, r, e, "gradient")
    # orders other than the packed one, and a gradient that is one value for all
    t = x.view(4, 15, 333).transpose(0, 1).detach().requires_grad_()
    out = nn.layer_norm(t, w, b, EPS)
    assert torch.equal(out.transpose(0, 1).reshape(60, 333), y.detach().view(60, 333))
    out.sum().backward()
    assert t.grad.shape == t.shape
    with torch.no_grad():
        assert torch.equal(nn.layer_norm(x, w, b, EPS), y.view(60, 333))


def test_gradient_against_differences():
    """<grad, v> against the central difference of the 64-bit layer norm along v: with
    h = 1e-4 its error is h^2 times a third derivative, below 1e-6 here; the gradient's own
    is that of fp32 sums over 40 x 50 terms, below 1e-5 of the terms' magnitudes."""
    x, w, b, _ = inputs(40, 50, F32, F32)
    c = normal((40, 50), 9)
    leaves = [t.clone().requires_grad_() for t in (x, w, b)]
    say("layer norm differences")
    grads = torch.autograd.grad((nn.layer_norm(*leaves, EPS) * c).sum(), leaves)
    for i, (leaf, g) in enumerate(zip((x, w, b), grads)):
        v = normal(leaf.shape, 20 + i)
        h = 1e-4

        def f(s):
            args = [t.double() for t in (x, w, b)]
            args[i] = args[i] + s * v.double()
            return (ref.layer_norm(*args, EPS)[0] * c.double()).sum()
        diff = float((f(h) - f(-h)) / (2 * h))
        terms = float((g.double() * v.double()).abs().sum())
        assert abs(float((g.double() * v.double()).sum()) - diff) <= 1e-5 * terms + 1e-5
