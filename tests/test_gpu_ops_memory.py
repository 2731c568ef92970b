"""Tensors whose storage has been emptied, as sharded training does with parameters that it
does not need for a while: refused, not taken for parameters that were left out."""
import pytest
import torch

from paper_2110_02861_amd import bq, nn, optim
from tests.gpu_helpers import needs_gpu, say

pytestmark = [pytest.mark.gpu, needs_gpu]


def normal(shape, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.empty(shape, device="cuda").normal_(generator=g)


@pytest.fixture(params=[True, False], ids=["native", "python"])
def half(request, monkeypatch):
    if not request.param:
        monkeypatch.setattr(bq, "_host_module", bq._PythonOnly())


def empty(t):
    t.untyped_storage().resize_(0)
    return t


def test_emptied_arguments(half):
    say("emptied arguments")
    ids = torch.tensor([1, 2], device="cuda")
    x, w, table = normal((4, 8), 1), normal((8,), 2), normal((10, 8), 3)
    gone, gone_table, gone_x = empty(normal((8,), 4)), empty(normal((10, 8), 5)), \
        empty(normal((4, 8), 6))
    part = normal((20,), 7)[4:12]  # a view that does not start at the storage's start
    empty(part)
    assert gone.shape == (8,) and part.shape == (8,)
    for v in (gone, part):
        for call in (lambda: nn.layer_norm(x, v), lambda: nn.layer_norm(x, w, v),
                     lambda: nn.layer_norm(x, None, v), lambda: nn.stable_embedding(ids, table, v),
                     lambda: nn.stable_embedding(ids, table, w, v),
                     lambda: bq.bq_layer_norm_forward(x, v),
                     lambda: bq.bq_layer_norm_forward(x, w, out=gone_x),
                     lambda: bq.bq_grad_norm([x, v]), lambda: bq.bq_clip_grad_norm([v], 1.0)):
            with pytest.raises(ValueError, match="memory"):
                call()
    for call in (lambda: nn.layer_norm(gone_x, w), lambda: nn.embedding(ids, gone_table),
                 lambda: nn.stable_embedding(ids, gone_table),
                 lambda: nn.embedding(empty(torch.tensor([1, 2], device="cuda")), table)):
        with pytest.raises(ValueError, match="memory"):
            call()
    p = torch.nn.Parameter(normal((8,), 8))
    p.grad = gone
    with pytest.raises(ValueError, match="memory"):
        optim.clip_grad_norm_([p], 1.0)


@pytest.mark.parametrize("which", ["x", "weight", "table", "norm_weight", "ids"])
def test_emptied_before_the_backward_pass(which, half):
    say("emptied before the backward pass", which)
    t = dict(x=normal((4, 8), 1), weight=normal((8,), 2), table=normal((10, 8), 3),
             norm_weight=normal((8,), 4), ids=torch.tensor([1, 2], device="cuda"))
    leaves = {k: v.requires_grad_() if k != "ids" else v for k, v in t.items()}
    if which in ("x", "weight"):
        y = nn.layer_norm(leaves["x"], leaves["weight"])
    else:
        y = nn.stable_embedding(leaves["ids"], leaves["table"], leaves["norm_weight"])
    empty(t[which])
    with pytest.raises((RuntimeError, ValueError), match="memory"):
        y.backward(torch.ones_like(y))


@pytest.mark.filterwarnings("ignore:Accessing the data pointer")
def test_tensors_without_memory_of_their_own(half):
    """Fake tensors, and those that a transform wraps, have a null address."""
    from torch._subclasses.fake_tensor import FakeTensorMode
    say("tensors without memory")
    x, w, table = normal((4, 8), 1), normal((8,), 2), normal((10, 8), 3)
    ids = torch.tensor([1, 2], device="cuda")
    fake = FakeTensorMode().from_tensor(w)
    calls = (lambda v: nn.layer_norm(x, v), lambda v: nn.layer_norm(x, w, v),
             lambda v: bq.bq_layer_norm_forward(x, None, v),
             lambda v: nn.stable_embedding(ids, table, v),
             lambda v: nn.stable_embedding(ids, table, w, v))
    for call in calls:
        with pytest.raises(ValueError, match="memory"):
            call(fake)
        with pytest.raises(ValueError, match="memory"):
            torch.func.functionalize(call)(w)
    with FakeTensorMode() as mode, pytest.raises(ValueError, match="memory"):
        nn.layer_norm(mode.from_tensor(x))
