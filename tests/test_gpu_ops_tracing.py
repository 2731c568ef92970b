"""The refusal of tracing on the GPU, where the native half would otherwise make the call,
and in the Python half."""
import pytest
import torch
from torch.fx.experimental.proxy_tensor import make_fx

from paper_2110_02861_amd import bq, nn, optim
from tests.gpu_helpers import needs_gpu, say

pytestmark = [pytest.mark.gpu, needs_gpu]


def normal(shape, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.empty(shape, device="cuda").normal_(generator=g)


def case(name):
    """(function, differentiable arguments)"""
    ids = torch.tensor([[3, 0, 3], [8, 1, 3]], device="cuda")
    x, w, b, table = normal((6, 40), 1), normal((40,), 2), normal((40,), 3), normal((9, 40), 4)
    return {"layer_norm": (lambda *a: nn.layer_norm(*a), (x, w, b)),
            "embedding": (lambda t: nn.embedding(ids, t), (table,)),
            "stable_embedding": (lambda *a: nn.stable_embedding(ids, *a), (table, w, b)),
            "bq layer norm": (lambda *a: bq.bq_layer_norm_forward(*a), (x, w, b)),
            "bq embedding": (lambda t: bq.bq_embedding_forward(t, ids), (table,)),
            "bq stable embedding":
                (lambda t, *a: bq.bq_stable_embedding_forward(t, ids, *a), (table, w, b))}[name]


NAMES = ["layer_norm", "embedding", "stable_embedding", "bq layer norm", "bq embedding",
         "bq stable embedding"]


@pytest.fixture(params=[True, False], ids=["native", "python"])
def half(request, monkeypatch):
    if not request.param:
        monkeypatch.setattr(bq, "_host_module", bq._PythonOnly())


@pytest.mark.parametrize("name", NAMES)
def test_tracing_is_refused(name, half):
    fn, args = case(name)
    say("tracing", name)
    for grads in (False, True):
        args = tuple(a.detach().requires_grad_(grads) for a in args)
        with pytest.raises(NotImplementedError, match="traced"):
            torch.jit.trace(fn, args, check_trace=False)
    args = tuple(a.detach() for a in args)
    for pre_dispatch in (False, True):
        with pytest.raises(NotImplementedError, match="traced"):
            make_fx(fn, tracing_mode="real", pre_dispatch=pre_dispatch)(*args)
    assert torch.equal(fn(*args), fn(*args))


def test_clipping_is_refused_and_changes_nothing(half):
    g = normal((50,), 5)
    kept = g.clone()
    p = torch.nn.Parameter(torch.zeros_like(g))
    p.grad = g
    say("clip traced")
    with pytest.raises(NotImplementedError, match="traced"):
        torch.jit.trace(lambda x: x + optim.clip_grad_norm_([p], 0.1), (kept,), check_trace=False)
    assert torch.equal(g, kept)
