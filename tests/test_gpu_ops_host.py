"""The native half of nn's functions and of the clipping against the Python code that it
stands in for: the same bits, the same errors, and who handles what."""
import pytest
import torch

from paper_2110_02861_amd import bq, nn, optim
from tests.gpu_helpers import needs_gpu, say

pytestmark = [pytest.mark.gpu, needs_gpu]

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


class _Sub(torch.Tensor):
    pass


def normal(shape, seed, std=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.empty(shape, device="cuda").normal_(0.0, std, generator=g)


@pytest.fixture
def handled(monkeypatch):
    """Names of the native functions that handled a call, in order."""
    module, names = bq.host(), []

    class Recorder:
        def __getattr__(self, name):
            f = getattr(module, name)

            def call(*args):
                r = f(*args)
                if r is not None:
                    names.append(name)
                return r
            return call
    monkeypatch.setattr(bq, "_host_module", Recorder())
    return names


def python_only(monkeypatch):
    monkeypatch.setattr(bq, "_host_module", bq._PythonOnly())


def layer_norm_case(xt, wt):
    x, w, b = normal((3, 7, 90), 1).to(xt), normal((90,), 2).to(wt), normal((90,), 3).to(wt)
    return nn.layer_norm, (x, w, b), (0, 1, 2), {"eps": 1e-4}


def embedding_case(wt, yt):
    ids = torch.tensor([[3, 0, 3], [8, 1, 3]], device="cuda")
    return nn.embedding, (ids, normal((9, 40), 1).to(wt)), (1,), dict(padding_idx=-1, scale=3.0,
                                                                      out_dtype=yt)


def stable_case(wt, yt):
    ids = torch.tensor([[3, 0, 3], [8, 1, 3]], device="cuda", dtype=torch.int32)
    return (nn.stable_embedding,
            (ids, normal((9, 40), 1).to(wt), normal((40,), 2).to(wt), normal((40,), 3).to(wt)),
            (1, 2, 3), dict(eps=1e-4, padding_idx=8, out_dtype=yt))


CASES = {"layer_norm f32": layer_norm_case(F32, F32), "layer_norm bf16 f32": layer_norm_case(BF16, F32),
         "embedding": embedding_case(F32, BF16), "embedding f16": embedding_case(F16, None),
         "stable": stable_case(F32, F16), "stable bf16": stable_case(BF16, None)} \
    if torch.cuda.is_available() else {}
NAMES = ["layer_norm f32", "layer_norm bf16 f32", "embedding", "embedding f16", "stable",
         "stable bf16"]


def outcome(fn, args, grads, kw, which=None):
    """The result and the gradients of the wanted arguments."""
    which = grads if which is None else which
    leaves = [a.detach().clone().requires_grad_(i in which) if i in grads else a
              for i, a in enumerate(args)]
    y = fn(*leaves, **kw)
    assert y.requires_grad == bool(which)
    dy = torch.linspace(-1, 1, y.numel(), device="cuda").view(y.shape).to(y.dtype)
    return [y.detach()] + list(torch.autograd.grad(y, [leaves[i] for i in which], dy)
                               if which else ())


@pytest.mark.parametrize("name", NAMES)
def test_native_and_python_agree(name, monkeypatch, handled):
    fn, args, grads, kw = CASES[name]
    say("native and python", name)
    sets = [None, (), grads[:1], grads[-1:], grads[1:]]
    native = [outcome(fn, args, grads, kw, s) for s in sets]
    assert len(handled) == len(sets)
    with torch.no_grad():
        plain = fn(*args, **kw)
    python_only(monkeypatch)
    for s, want in zip(sets, native):
        got = outcome(fn, args, grads, kw, s)
        assert len(got) == len(want)
        for a, b in zip(got, want):
            assert a.dtype == b.dtype and torch.equal(a, b)
    assert torch.equal(plain, native[0][0])


@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("name", NAMES)
def test_second_derivatives_raise(name, native, monkeypatch):
    fn, args, grads, kw = CASES[name]
    say("second derivative", name, native)
    if not native:
        python_only(monkeypatch)
    leaves = [a.clone().requires_grad_(i in grads) if i in grads else a
              for i, a in enumerate(args)]
    want = [leaves[i] for i in grads]
    y = fn(*leaves, **kw)
    # a first derivative with a graph is a first derivative
    first = torch.autograd.grad(y.float().square().sum(), want, create_graph=True)
    with pytest.raises(RuntimeError, match="differentiate twice"):
        first[0].float().sum().backward()


@pytest.mark.parametrize("name", NAMES)
def test_changed_inputs_are_noticed(name):
    """A leaf that the backward pass reads, changed in between by torch."""
    fn, args, grads, kw = CASES[name]
    if name.startswith("embedding"):
        args[0].add_(0)
        leaves = [args[0].clone(), args[1].clone().requires_grad_()]
        at = 0
    else:
        leaves = [a.clone().requires_grad_() if i in grads else a for i, a in enumerate(args)]
        at = 1
    say("changed inputs", name)
    y = fn(*leaves, **kw)
    with torch.no_grad():
        leaves[at].add_(0)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.float().sum().backward()


@pytest.mark.parametrize("native", [True, False])
def test_errors(native, monkeypatch):
    if not native:
        python_only(monkeypatch)
    x, w = normal((4, 8), 1), normal((8,), 2)
    ids, table = torch.tensor([1, 2], device="cuda"), normal((10, 8), 3)
    say("errors", native)
    for bad in (lambda: nn.layer_norm(x.double()), lambda: nn.layer_norm(x, w.half()),
                lambda: nn.layer_norm(x, w, w.half()), lambda: nn.embedding(ids.float(), table),
                lambda: nn.embedding(ids, table.half(), out_dtype=F32),
                lambda: nn.embedding(ids, table, out_dtype=torch.float64),
                lambda: nn.stable_embedding(ids, table, w.half()),
                lambda: nn.layer_norm(x, w.cpu()), lambda: nn.embedding(ids.cpu(), table)):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: nn.layer_norm(x, w[:7]), lambda: nn.embedding(ids, table, padding_idx=10),
                lambda: nn.embedding(ids, table, padding_idx=-11), lambda: nn.embedding(ids, w),
                lambda: nn.stable_embedding(ids, table, w[:5]),
                lambda: nn.layer_norm(x[:, :0]), lambda: nn.embedding(ids, table.t())):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: nn.layer_norm(x, w, eps=-1.0), lambda: nn.layer_norm(x, w, eps=float("nan")),
                lambda: nn.embedding(ids, table, scale=float("inf")),
                lambda: nn.stable_embedding(ids, table, eps=-1.0)):
        with pytest.raises(bq.BQError):
            bad()


def test_what_is_left_to_python(handled):
    x, w = normal((4, 8), 1), normal((8,), 2)
    ids, table = torch.tensor([1, 2], device="cuda"), normal((10, 8), 3)
    say("left to python")
    want = nn.layer_norm(x, w)
    assert handled.pop() == "layer_norm"
    assert torch.equal(nn.layer_norm(x.t().contiguous().t(), w), want)
    assert handled.pop() == "layer_norm"  # of the packed copy
    assert torch.equal(nn.layer_norm(x.as_subclass(_Sub), w), want)
    assert nn.layer_norm(x[:0], w).shape == (0, 8)
    assert nn.embedding(ids[:0], table).shape == (0, 8)
    assert handled == []
    assert torch.equal(nn.layer_norm(normal((4, 30), 9)[:, 3:11], w),
                       nn.layer_norm(normal((4, 30), 9)[:, 3:11].contiguous(), w))


@pytest.mark.parametrize("native", [True, False])
def test_clip_agrees(native, monkeypatch, handled):
    say("clip native", native)
    if not native:
        python_only(monkeypatch)
    shared = normal((50,), 7)
    params = []
    for i, (dtype, shape) in enumerate(((F32, (30, 40)), (F16, (7,)), (BF16, (5, 6, 7)), (F32, (50,)),
                                        (F32, (50,)))):
        p = torch.nn.Parameter(normal(shape, i))
        p.grad_dtype = None
        p.grad = shared if shape == (50,) else normal(shape, i + 20).to(dtype)
        params.append(p)
    params[0].grad = normal((40, 30), 5).t()
    params.append(torch.nn.Parameter(normal((3,), 9)))
    before = [None if p.grad is None else p.grad.clone() for p in params]
    versions = [p.grad._version for p in params[:-1]]
    want = torch.cat([g.double().reshape(-1) for g in before[:4]]).norm()
    norm = optim.clip_grad_norm_((p for p in params), 0.25)
    assert (handled == ["clip"]) == native
    assert abs(float(norm) - float(want)) <= 1e-7 * float(want)
    c = 0.25 / (float(want) + 1e-6)
    for p, b in zip(params[:4], before):  # the shared one once
        tol = 3 * 2.0 ** -24 if b.dtype == F32 else torch.finfo(b.dtype).eps
        assert bool(((p.grad.double() - b.double() * c).abs()
                     <= tol * c * b.double().abs() + 1e-7).all())
    assert all(p.grad._version > v for p, v in zip(params[:-1], versions))
    with pytest.raises(ValueError):
        optim.clip_grad_norm_(params, 1.0, norm_type=1.0)
    params[0].grad = normal((30, 40), 6)
    other = torch.nn.Parameter(normal((1200,), 4))
    other.grad = params[0].grad.view(1200)
    kept = other.grad.clone()
    with pytest.raises(ValueError, match="same place"):
        optim.clip_grad_norm_([params[0], other], 1.0)
    assert torch.equal(kept, other.grad)
    params[0].grad = normal((30, 80), 3)[:, ::2]
    with pytest.raises(ValueError):
        optim.clip_grad_norm_(params, 1.0)


@pytest.mark.parametrize("native", [True, False])
def test_views_with_a_pending_negation(native, monkeypatch):
    """Such views (the imaginary part of a conjugate is one) hold the values that they are
    the negatives of."""
    say("negated views", native)
    if not native:
        python_only(monkeypatch)
    x, w, dy = normal((6, 40), 1), normal((40,), 2), normal((6, 40), 3)
    table, ids = normal((10, 40), 4), torch.tensor([1, 2, 9, 1, 0, 1], device="cuda")
    nx, ndy = torch._neg_view(x), torch._neg_view(dy)
    assert nx.is_neg() and nx.is_contiguous()
    assert torch.equal(nn.layer_norm(nx, w), nn.layer_norm(-x, w))
    for run, leaf in ((lambda t: nn.layer_norm(t, w), x), (lambda t: nn.embedding(ids, t), table),
                      (lambda t: nn.stable_embedding(ids, t), table)):
        leaf = leaf.clone().requires_grad_()
        a, = torch.autograd.grad(run(leaf), leaf, ndy)
        b, = torch.autograd.grad(run(leaf), leaf, -dy)
        assert torch.equal(a, b)
    for bad in (lambda: bq.bq_layer_norm_forward(nx), lambda: nn.layer_norm(x, torch._neg_view(w)),
                lambda: nn.embedding(ids, torch._neg_view(table)), lambda: bq.bq_grad_norm([nx])):
        with pytest.raises(TypeError, match="negation"):
            bad()
