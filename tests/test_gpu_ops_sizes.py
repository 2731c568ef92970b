"""The stable embedding's backward pass in a workspace of exactly the size asked for: small
tables, where the partial sums' rows are as many as the table's."""
import pytest
import torch

from paper_2110_02861_amd import bq
from tests.gpu_helpers import needs_gpu, say
from tests.test_gpu_embedding import BF16, EPS, F32, check_stable, normal, stable_inputs, word_ids

pytestmark = [pytest.mark.gpu, needs_gpu]


@pytest.mark.parametrize("wt", [F32, BF16])
@pytest.mark.parametrize("num,dim", [(1, 48), (3, 16384), (97, 300), (97, 9000), (513, 1000),
                                     (1023, 1600), (1025, 1600), (2047, 200), (9000, 64)])
def test_workspace_of_small_tables(num, dim, wt):
    w, lw, lb = stable_inputs(num, dim, wt)
    ids = word_ids(300, num, 1)
    dy = normal((300, dim), 2, 0.01).to(wt)
    need = bq.lib().bq_stable_embedding_workspace_bytes(300, num, dim)
    ws = torch.full((need + 8192,), 77, dtype=torch.uint8, device="cuda")
    say("stable embedding workspace", num, dim, wt)
    check_stable(w, ids, lw, lb, wt, dy)
    want = bq.bq_stable_embedding_backward(dy, ids, w, lw, EPS)
    got = bq.bq_stable_embedding_backward(dy, ids, w, lw, EPS, workspace=ws[:need])
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    assert bool((ws[need:] == 77).all())
