"""Python code that runs while the native half saves tensors: its exceptions end the call,
which is not made a second time.  Activation checkpointing depends on it."""
import pytest
import torch
from torch.utils.checkpoint import checkpoint

from paper_2110_02861_amd import bq, nn
from tests.gpu_helpers import needs_gpu, say
from tests.test_gpu_ops_saved import case, half, normal  # noqa: F401

pytestmark = [pytest.mark.gpu, needs_gpu]

NAMES = ["layer_norm", "embedding", "stable_embedding"]


@pytest.mark.parametrize("reentrant", [False, True])
@pytest.mark.parametrize("name", NAMES)
def test_checkpointed(name, reentrant, half):
    """The operator is the segment's last: recomputing stops in the middle of its saving."""
    fn, args, _ = case(name)
    say("checkpointed", name, reentrant)
    results = []
    for run in (lambda f, *a: f(*a), lambda f, *a: checkpoint(f, *a, use_reentrant=reentrant)):
        leaves = [a.detach().requires_grad_() for a in args]
        y = run(lambda t, *rest: fn(t * 2.0, *rest), *leaves)
        y.backward(normal(y.shape, 9))
        results.append([y.detach()] + [t.grad for t in leaves])
    for a, b in zip(*results):
        assert torch.equal(a, b)


@pytest.mark.parametrize("name", NAMES)
def test_an_exception_while_saving(name, half):
    fn, args, saved = case(name)
    say("exception while saving", name)
    leaves = [a.detach().requires_grad_() for a in args]
    for at in range(saved):
        seen = []

        def pack(t):
            seen.append(t.shape)
            if len(seen) == at + 1:
                raise KeyError("enough")
            return t
        with torch.autograd.graph.saved_tensors_hooks(pack, lambda t: t):
            with pytest.raises(KeyError, match="enough"):
                fn(*leaves)
        assert len(seen) == at + 1
    assert torch.equal(fn(*leaves), fn(*args))
