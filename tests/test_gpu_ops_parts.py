"""Operators without a weight, without a bias, or without either, through autograd: the native
half makes the call, and both halves agree with 64 bits."""
import pytest
import torch

from paper_2110_02861_amd import bq, nn
from tests import ops_reference as ref
from tests.gpu_helpers import needs_gpu, say
from tests.test_gpu_ops_host import handled  # noqa: F401

pytestmark = [pytest.mark.gpu, needs_gpu]

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
EPS = 1e-5


def normal(shape, seed, std=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.empty(shape, device="cuda").normal_(0.0, std, generator=g)


PARTS = [(False, False), (True, False), (False, True), (True, True)]


@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("types", [(F32, F32), (BF16, F32), (F16, F16)], ids=str)
@pytest.mark.parametrize("weight,bias", PARTS)
def test_layer_norm(weight, bias, types, native, monkeypatch, handled):
    xt, wt = types
    if not native:
        monkeypatch.setattr(bq, "_host_module", bq._PythonOnly())
    say("layer norm parts", weight, bias, types, native)
    x, dy = normal((23, 90), 1).to(xt), normal((23, 90), 4, 0.01).to(xt)
    w = (1 + normal((90,), 2, 0.1)).to(wt) if weight else None
    b = normal((90,), 3).to(wt) if bias else None
    yr, xh, mr, rr = ref.layer_norm(x, w, b, EPS)
    want = ref.layer_norm_grads(dy, xh, rr, w)
    # the parameters' type is x's where there are none
    bounds = ref.backward_bounds(dy, xh, mr, rr, w, *want, xt, wt if weight or bias else xt)
    given = [0] + [1] * weight + [2] * bias
    sets = [some for some in (given, given[:1], given[1:], given[-1:]) if some]
    for some in sets:
        args = [None if t is None else t.detach().requires_grad_(i in some)
                for i, t in enumerate((x, w, b))]
        y = nn.layer_norm(*args, EPS)
        ref.check(y, yr, ref.forward_bound(yr, xh, w, xt, 90), "y")
        y.backward(dy)
        for i, t in enumerate(args):
            if i in some:
                ref.check(t.grad, want[i], bounds[i], f"gradient {i}")
            else:
                assert t is None or t.grad is None
    assert handled == ["layer_norm"] * len(sets) * native


@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("weight,bias", PARTS)
def test_stable_embedding(weight, bias, native, monkeypatch, handled):
    if not native:
        monkeypatch.setattr(bq, "_host_module", bq._PythonOnly())
    say("stable embedding parts", weight, bias, native)
    table, dy = normal((30, 90), 1, 0.05), normal((200, 90), 4, 0.01)
    ids = torch.randint(0, 30, (200,), device="cuda", generator=torch.Generator("cuda").manual_seed(5))
    w = 1 + normal((90,), 2, 0.1) if weight else None
    b = normal((90,), 3) if bias else None
    d, dw, db = bq.bq_stable_embedding_backward(dy, ids, table, w, EPS)  # held against 64 bits
    want = dict(enumerate((d, dw, db)))                                  # in test_gpu_embedding
    given = [0] + [1] * weight + [2] * bias
    sets = [some for some in (given, given[:1], given[1:], given[-1:]) if some]
    for some in sets:
        args = [None if t is None else t.detach().requires_grad_(i in some)
                for i, t in enumerate((table, w, b))]
        y = nn.stable_embedding(ids, *args, EPS)
        assert torch.equal(y, bq.bq_stable_embedding_forward(table, ids, w, b, EPS))
        y.backward(dy)
        for i, t in enumerate(args):
            if i in some:
                assert torch.equal(t.grad, want[i])
            else:
                assert t is None or t.grad is None
    assert handled == ["stable_embedding"] * 2 * len(sets) * native


def test_modules_without_a_bias_are_native(handled):
    say("modules without a bias")
    x = normal((5, 40), 1)
    for kw in (dict(bias=False), dict(elementwise_affine=False), {}):
        m = nn.LayerNorm(40, device="cuda", **kw)
        m(x.clone().requires_grad_()).sum().backward()
    assert handled == ["layer_norm"] * 3
