"""torch.compile runs the operators between its graphs: the same bits as without it."""
import pytest
import torch

from paper_2110_02861_amd import nn
from tests.gpu_helpers import needs_gpu, say

pytestmark = [pytest.mark.gpu, needs_gpu]


class Model(torch.nn.Module):
    def __init__(self):
        super().__init__()
        self.words = nn.StableEmbedding(50, 64, fused=True, device="cuda")
        self.scaled = nn.Embedding(50, 64, scale=8.0, device="cuda")
        self.norm = nn.LayerNorm(64, device="cuda")

    def forward(self, ids):
        return self.norm(torch.tanh(self.words(ids)) + self.scaled(ids))


@pytest.mark.filterwarnings("ignore")
@pytest.mark.parametrize("backend", ["eager", "aot_eager"])
def test_compiled(backend):
    say("compiled", backend)
    torch.manual_seed(0)
    m = Model()
    ids = torch.randint(0, 50, (6, 7), device="cuda")
    dy = torch.randn((6, 7, 64), device="cuda")

    def run(f):
        for p in m.parameters():
            p.grad = None
        y = f(ids)
        y.backward(dy)
        return [y.detach()] + [p.grad for p in m.parameters()]
    want = run(m)
    try:
        compiled = torch.compile(m, backend=backend)
        for _ in range(2):
            for a, b in zip(run(compiled), want):
                assert torch.equal(a, b)
    finally:
        torch._dynamo.reset()
