"""The operators around the optimizer step refuse to be traced, before anything else is
looked at: the refusals show on CPU tensors too."""
import pytest
import torch
from torch.fx.experimental.proxy_tensor import make_fx

from paper_2110_02861_amd import bq, nn, optim

X, W = torch.randn(4, 8), torch.randn(8)
TABLE, IDS = torch.randn(10, 8), torch.tensor([1, 2, 9, 1])


def param(g):
    p = torch.nn.Parameter(torch.zeros_like(g))
    p.grad = g
    return p


CALLS = {
    "layer_norm": (lambda x, w: nn.layer_norm(x, w, w), (X, W)),
    "LayerNorm": (lambda x: nn.LayerNorm(8)(x), (X,)),
    "embedding": (lambda t: nn.embedding(IDS, t), (TABLE,)),
    "stable_embedding": (lambda t, w: nn.stable_embedding(IDS, t, w), (TABLE, W)),
    "bq layer norm": (lambda x, w: bq.bq_layer_norm_forward(x, w), (X, W)),
    "bq layer norm backward": (lambda x: bq.bq_layer_norm_backward(x, x, None, x, x), (X,)),
    "bq embedding": (lambda t: bq.bq_embedding_forward(t, IDS), (TABLE,)),
    "bq embedding backward": (lambda x: bq.bq_embedding_backward(x, IDS, 10), (X,)),
    "bq stable embedding": (lambda t: bq.bq_stable_embedding_forward(t, IDS), (TABLE,)),
    "bq stable embedding backward":
        (lambda x, t: bq.bq_stable_embedding_backward(x, IDS, t), (X, TABLE)),
    "bq norm": (lambda x: bq.bq_grad_norm([x]), (X,)),
    "bq clip": (lambda x: bq.bq_clip_grad_norm([x], 1.0), (X,)),
    "clip": (lambda x: optim.clip_grad_norm_([param(x)], 1.0), (X,)),
}


@pytest.mark.parametrize("name", CALLS)
def test_tracing_is_refused(name):
    """A trace would hold the allocation of the result and not the kernel that fills it."""
    fn, args = CALLS[name]
    with pytest.raises(NotImplementedError, match="traced"):
        torch.jit.trace(fn, args, check_trace=False)
    for pre_dispatch in (False, True):
        with pytest.raises(NotImplementedError, match="traced"):
            make_fx(fn, tracing_mode="real", pre_dispatch=pre_dispatch)(*args)
    with pytest.raises(TypeError):  # eager, it is the device that is wrong
        fn(*args)


def test_traced_modules_and_empty_lists_are_refused():
    for m in (nn.Embedding(10, 8), nn.StableEmbedding(10, 8, fused=True)):
        with pytest.raises(NotImplementedError, match="traced"):
            torch.jit.trace(m, (IDS,))
    with pytest.raises(NotImplementedError, match="traced"):
        torch.jit.trace(lambda x: x + bq.bq_grad_norm([]), (X,))
    # the plain stable embedding is made of torch's operations
    m = nn.StableEmbedding(10, 8)
    assert torch.equal(torch.jit.trace(m, (IDS,))(IDS), m(IDS))
