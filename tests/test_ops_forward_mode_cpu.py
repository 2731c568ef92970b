"""The operators around the optimizer step refuse tensors with a forward-mode tangent, before
anything else is looked at: the refusals show on CPU tensors too."""
import pytest
import torch
import torch.autograd.forward_ad as fwd

from tests.test_ops_tracing_cpu import CALLS


@pytest.mark.parametrize("name", CALLS)
def test_forward_mode_is_refused(name):
    """The result of a dual tensor would have no tangent."""
    fn, args = CALLS[name]
    with fwd.dual_level():
        for i in range(len(args)):
            dual = [fwd.make_dual(a, torch.ones_like(a)) if i == j else a
                    for j, a in enumerate(args)]
            with pytest.raises(NotImplementedError, match="forward-mode"):
                fn(*dual)
            with torch.no_grad(), pytest.raises(NotImplementedError, match="forward-mode"):
                fn(*dual)
        with pytest.raises(TypeError):  # no dual tensor among the arguments
            fn(*args)
