"""Parts of long gradients against 64 bits: sums over spans of chunks where waves and
workgroups hold a row, and rows that are cut into slabs of columns."""
import pytest
import torch

from tests.gpu_helpers import needs_gpu, say
from tests.test_gpu_embedding import (BF16, F16, F32, check_lookup, check_stable, normal,
                                      stable_inputs, word_ids)

pytestmark = [pytest.mark.gpu, needs_gpu]


@pytest.mark.parametrize("types", [(F32, F32), (BF16, BF16), (F32, F16)], ids=str)
@pytest.mark.parametrize("dim", [333, 1024, 1601, 2051, 3001, 5000, 9001])
def test_spans(dim, types):
    """33,001 tokens on 40 rows: the frequent ones hold several whole spans of 1024 tokens,
    with chunks and tokens on both sides."""
    wt, yt = types
    w, lw, lb = stable_inputs(40, dim, wt)
    ids = word_ids(33001, 40, dim)
    say("embedding spans", dim, types)
    check_lookup(w, ids, yt, 1.5, padding=1)
    check_stable(w, ids, lw, lb, yt, padding=1)


@pytest.mark.parametrize("dim,types", [(9001, (F32, F32)), (20001, (F32, F32)),
                                       (20001, (F32, BF16)), (20001, (BF16, BF16)),
                                       (33000, (F16, F16))], ids=str)
def test_slabs(dim, types):
    """A row with several whole chunks, others with a few tokens, some without."""
    wt, yt = types
    w = normal((23, dim), 1).to(wt)
    ids = torch.cat([torch.full((150,), 5, device="cuda"), word_ids(200, 23, 1)])
    ids = ids[torch.randperm(350, generator=torch.Generator().manual_seed(1)).cuda()]
    say("embedding slabs", dim, types)
    check_lookup(w, ids, yt, 2.5)
    check_lookup(w, ids, yt, 1.0, padding=5)
