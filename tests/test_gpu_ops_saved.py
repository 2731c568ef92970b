"""Saved tensors that hooks hand back in another form than they were given: another order of
memory gives the same gradients, anything else is refused before a kernel reads it."""
import pytest
import torch

from paper_2110_02861_amd import bq, nn
from tests.gpu_helpers import needs_gpu, say

pytestmark = [pytest.mark.gpu, needs_gpu]


def normal(shape, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.empty(shape, device="cuda").normal_(generator=g)


def case(name):
    """(function, its differentiable arguments, number of saved tensors)"""
    ids = torch.tensor([[3, 0, 3], [8, 1, 3]], device="cuda")
    x, w, b, table = normal((5, 6, 40), 1), normal((40,), 2), normal((40,), 3), normal((9, 40), 4)
    return {"layer_norm": (lambda *a: nn.layer_norm(*a), (x, w, b), 4),
            "embedding": (lambda t: nn.embedding(ids, t), (table,), 1),
            "stable_embedding": (lambda *a: nn.stable_embedding(ids, *a), (table, w, b), 3)}[name]


def other_order(t):
    """The same values, with the first axis (of a vector: every second place) the fastest."""
    if t.dim() == 1:
        return torch.stack([t, t], 1)[:, 0]
    return t.transpose(0, -1).contiguous().transpose(0, -1)


@pytest.fixture(params=[True, False], ids=["native", "python"])
def half(request, monkeypatch):
    if not request.param:
        monkeypatch.setattr(bq, "_host_module", bq._PythonOnly())


def gradients(name, change=None, at=None):
    """With change on the at-th tensor that is unpacked (on all for None)."""
    fn, args, _ = case(name)
    leaves = [a.detach().requires_grad_() for a in args]
    count = [0]

    def unpack(t):
        count[0] += 1
        return change(t) if change and at in (None, count[0] - 1) else t
    with torch.autograd.graph.saved_tensors_hooks(lambda t: t.detach(), unpack):
        y = fn(*leaves)
    dy = normal(y.shape, 9)
    return torch.autograd.grad(y, leaves, dy), count[0]


@pytest.mark.parametrize("name", ["layer_norm", "embedding", "stable_embedding"])
def test_other_orders_of_memory(name, half):
    say("saved tensors in another order", name)
    want, saved = gradients(name)
    assert saved == case(name)[2]
    got, _ = gradients(name, other_order)
    for a, b in zip(got, want):
        assert torch.equal(a, b)


CHANGES = {"on the host": lambda t: t.cpu(), "another type": lambda t: t.double(),
           "fewer": lambda t: t[:1], "more": lambda t: torch.cat([t, t]),
           "sparse": lambda t: t.to_sparse()}


@pytest.mark.parametrize("change", CHANGES)
@pytest.mark.parametrize("name", ["layer_norm", "embedding", "stable_embedding"])
def test_other_tensors_are_refused(name, change, half):
    for at in range(case(name)[2]):
        say("saved tensor changed", name, change, at)
        with pytest.raises((RuntimeError, TypeError, ValueError)):
            gradients(name, CHANGES[change], at)
    torch.cuda.synchronize()
    gradients(name)
