"""The refusal of forward-mode tangents on the GPU, where the native half would otherwise make
the call, and in the Python half."""
import pytest
import torch
import torch.autograd.forward_ad as fwd

from paper_2110_02861_amd import optim
from tests.gpu_helpers import needs_gpu, say
from tests.test_gpu_ops_tracing import NAMES, case, half, normal  # noqa: F401

pytestmark = [pytest.mark.gpu, needs_gpu]


@pytest.mark.parametrize("name", NAMES)
def test_forward_mode_is_refused(name, half):
    fn, args = case(name)
    say("forward mode", name)
    want = fn(*args)
    with fwd.dual_level():
        for i in range(len(args)):
            for grads in (False, True):
                if grads and name.startswith("bq"):
                    continue
                dual = [fwd.make_dual(a.detach().requires_grad_(grads), torch.ones_like(a))
                        if i == j else a for j, a in enumerate(args)]
                with pytest.raises(NotImplementedError, match="forward-mode"):
                    fn(*dual)
                with torch.no_grad(), pytest.raises(NotImplementedError, match="forward-mode"):
                    fn(*dual)
        assert torch.equal(fn(*args), want)  # none of the arguments is a dual tensor
    with torch.inference_mode():
        assert torch.equal(fn(*args), want)


@pytest.mark.parametrize("name", NAMES[:3])
def test_a_dual_gradient_is_refused(name, half):
    """Forward over reverse: the tangent of what comes into the backward pass."""
    fn, args = case(name)
    say("dual gradient", name)
    leaves = [a.detach().requires_grad_() for a in args]
    with fwd.dual_level():
        y = fn(*leaves)
        dy = fwd.make_dual(torch.ones_like(y), torch.ones_like(y))
        with pytest.raises(NotImplementedError, match="forward-mode"):
            torch.autograd.grad(y, leaves, dy, retain_graph=True)
        assert torch.autograd.grad(y, leaves, torch.ones_like(y))[0].shape == args[0].shape


def test_clipping_is_refused_and_changes_nothing(half):
    g = normal((50,), 5)
    kept = g.clone()
    p = torch.nn.Parameter(torch.zeros_like(g))
    say("clip of dual gradients")
    with fwd.dual_level():
        p.grad = fwd.make_dual(g, torch.ones_like(g))
        for call in (lambda: optim.clip_grad_norm_([p], 0.1), lambda: optim.grad_norm([p])):
            with pytest.raises(NotImplementedError, match="forward-mode"):
                call()
        p.grad = None
    assert torch.equal(g, kept)
