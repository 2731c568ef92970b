"""The fused stable embedding around a layer norm that has to be called, on the GPU."""
import pytest
import torch

from paper_2110_02861_amd import nn
from tests import ops_reference as ref
from tests.gpu_helpers import needs_gpu, say
from tests.test_gpu_embedding import F16, F32, normal, word_ids

pytestmark = [pytest.mark.gpu, needs_gpu]


@pytest.mark.parametrize("out", [None, F16])
def test_hooks_on_the_norm(out):
    """They run, and what they leave unchanged is as it was to rounding: y within the sum of
    both forms' bounds, the gradients within 2e-5 of the largest value."""
    say("stable embedding with hooks", out)
    torch.manual_seed(0)
    emb = nn.StableEmbedding(400, 80, padding_idx=3, device="cuda", fused=True, out_dtype=out)
    ids = word_ids(600, 400, 1).view(20, 30)
    dy = normal((20, 30, 80), 2, 0.01).to(out or F32)

    def run():
        for p in emb.parameters():
            p.grad = None
        y = emb(ids)
        y.backward(dy)
        return [y.detach()] + [p.grad for p in emb.parameters()]
    want = run()
    seen = []
    handles = [emb.norm.register_forward_hook(lambda m, i, o: seen.append("forward")),
               emb.norm.register_forward_pre_hook(lambda m, i: seen.append("before")),
               emb.norm.register_full_backward_hook(lambda m, i, o: seen.append("backward"))]
    got = run()
    assert seen == ["before", "forward", "backward"]
    for h in handles:
        h.remove()
    with torch.no_grad():
        rows = emb.weight[ids.view(-1)]
        yr, xh, _, _ = ref.layer_norm(rows, emb.norm.weight, emb.norm.bias, emb.norm.eps)
        bound = ref.forward_bound(yr, xh, emb.norm.weight, out or F32, 80)
        for y in (got[0], want[0]):
            assert y.dtype == (out or F32)
            ref.check(y.view(-1, 80), yr, bound, "y")
    for a, b in zip(got[1:], want[1:]):
        assert float((a - b).abs().max()) <= 2e-5 * float(b.abs().max())
    again = run()
    assert seen == ["before", "forward", "backward"]
    for a, b in zip(again, want):
        assert torch.equal(a, b)
