"""Embedding lookup with scaling, its gradient by sorted tokens, and the stable embedding
on the GPU, against their definitions in 64 bits with the bounds of ops_reference."""
import math

import pytest
import torch

from paper_2110_02861_amd import bq, nn
from tests import ops_reference as ref
from tests.gpu_helpers import needs_gpu, say

pytestmark = [pytest.mark.gpu, needs_gpu]

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
TYPES = [(F32, F32), (F16, F16), (BF16, BF16), (F32, F16), (F32, BF16)]
EPS = 1e-5


def normal(shape, seed, std=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.empty(shape, device="cuda").normal_(0.0, std, generator=g)


def uniform_ids(count, num, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(0, num, (count,), device="cuda", generator=g)


def word_ids(count, num, seed):
    """Frequencies that fall with the rank."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    u = torch.rand(count, dtype=torch.float64, device="cuda", generator=g)
    return (torch.exp(u * math.log(num + 1)) - 1).long().clamp_(0, num - 1)


def check_lookup(w, ids, yt, scale, dy=None, padding=None):
    num, dim = w.shape
    y = bq.bq_embedding_forward(w, ids, scale, yt)
    # one product in fp32, one rounding to the type
    want = (w.float()[ids.long()] * scale).to(yt)
    assert torch.equal(y, want)
    if dy is None:
        dy = normal((*ids.shape, dim), 3, 0.01).to(yt)
    d = bq.bq_embedding_backward(dy, ids, num, padding, scale, w.dtype)
    check_lookup_grad(d, dy, ids, num, w.dtype, scale, padding)
    return d


def check_lookup_grad(d, dy, ids, num, wt, scale, padding):
    s, a, count = ref.row_sums(dy, ids, num)
    want = s * scale
    bound = (ref.sum_error(a, count) * abs(scale) + (2 * ref.U + ref.HALF[wt]) * want.abs() +
             ref.TINY[wt])
    if padding is not None:
        want[padding] = 0.0
    assert d.dtype == wt
    ref.check(d, want, bound, "dweight")
    assert not d[count == 0].any()
    if padding is not None:
        assert not d[padding].any()


@pytest.mark.parametrize("types", TYPES, ids=str)
@pytest.mark.parametrize("dim", [1, 3, 64, 255, 300, 1024, 1600, 2051, 5000])
def test_dims(dim, types):
    wt, yt = types
    w = normal((61, dim), 1).to(wt)
    for count in (1, 7, 300):
        say("embedding", dim, types, count)
        check_lookup(w, uniform_ids(count, 61, dim), yt, 1.0)
        check_lookup(w, word_ids(count, 61, dim), yt, 5.5, padding=0)


@pytest.mark.parametrize("num", [1, 2, 255, 256, 257, 1023, 50257, 65536, 300007, 1 << 20])
def test_table_sizes(num):
    w = normal((num, 12), 1)
    say("embedding rows", num)
    check_lookup(w, uniform_ids(5000, num, 1), F32, 1.0)
    check_lookup(w, word_ids(5000, num, 2).int(), BF16, 1.0, padding=num - 1)
    ends = torch.tensor([0, num - 1, 0, num - 1, num // 2], device="cuda")
    check_lookup(w, ends, F32, 2.0)


@pytest.mark.parametrize("count", [1, 63, 64, 65, 127, 128, 4095, 4096, 4097, 8192, 70001])
def test_token_counts(count):
    w = normal((700, 40), 1)
    say("embedding tokens", count)
    check_lookup(w, word_ids(count, 700, count), F32, 1.0)
    check_lookup(w, word_ids(count, 700, count), F16, 1.0)


@pytest.mark.parametrize("count", [64, 1000, 20000])
def test_one_row_for_all_tokens(count):
    """Every token the same: whole chunks, at their borders and between."""
    w = normal((300, 130), 1)
    for row in (0, 150, 299):
        say("embedding one row", count, row)
        ids = torch.full((count,), row, device="cuda")
        check_lookup(w, ids, F32, 1.0)
        ids[count // 2] = 151
        check_lookup(w, ids, BF16, 3.0)
        check_lookup(w, ids, F32, 1.0, padding=row)


@pytest.mark.parametrize("count", [32767, 32768, 50001])
def test_thousands_of_tokens_in_a_row(count):
    """Rows of a few whole spans of chunks, with chunks and tokens on both sides of them."""
    w = normal((40, 70), 1)
    say("embedding spans", count)
    check_lookup(w, word_ids(count, 40, 1), F32, 1.0)
    check_lookup(w, word_ids(count, 40, 2), BF16, 1.0, padding=1)
    ids = torch.full((count,), 20, device="cuda")
    ids[::5000] = 3
    check_lookup(w, ids, F32, 1.0)
    check_lookup(w, ids, F32, 1.0, padding=20)
    check_stable(w, ids, None, None, F32, padding=20)


def test_a_million_tokens():
    say("embedding a million tokens")
    w = normal((50257, 8), 1)
    check_lookup(w, word_ids((1 << 20) + 13, 50257, 1), F32, 1.0)


def test_ids_outside_of_the_table():
    """They read nothing, give rows of NaN and no gradient, and leave the others alone."""
    w = normal((100, 70), 1)
    ids = torch.tensor([5, -1, 99, 100, 5, 1 << 40, -(1 << 40), 0], device="cuda")
    bad = (ids < 0) | (ids >= 100)
    say("embedding ids outside")
    for i, b in ((ids, bad), (ids[:5].int(), bad[:5])):
        y = bq.bq_embedding_forward(w, i, 2.0)
        z = bq.bq_stable_embedding_forward(w, i, None, None, EPS)
        assert y[b].isnan().all() and z[b].isnan().all()
        assert torch.equal(y[~b], w[i[~b].long()] * 2.0) and not z[~b].isnan().any()
        dy = normal((i.numel(), 70), 2)
        check_lookup_grad(bq.bq_embedding_backward(dy, i, 100, None, 2.0), dy, i, 100, F32, 2.0, None)
        check_stable(w, i, None, None, F32, dy, forward=False)
    none = torch.full((200,), 100, device="cuda")
    assert not bq.bq_embedding_backward(normal((200, 70), 2), none, 100).any()


def test_no_tokens():
    w, ids = normal((30, 20), 1), torch.zeros((0,), dtype=torch.int64, device="cuda")
    say("embedding no tokens")
    assert bq.bq_embedding_forward(w, ids).shape == (0, 20)
    d = bq.bq_embedding_backward(torch.zeros((0, 20), device="cuda"), ids, 30)
    assert d.shape == (30, 20) and not d.any()
    d, dw, db = bq.bq_stable_embedding_backward(torch.zeros((0, 20), device="cuda"), ids, w)
    assert not d.any() and not dw.any() and not db.any()


def test_gradients_that_are_not_finite_stay_in_their_row():
    w = normal((10, 33), 1)
    ids = torch.tensor([1, 2, 3, 2, 1], device="cuda")
    dy = normal((5, 33), 2)
    dy[3, 4] = float("inf")
    say("embedding not finite")
    d = bq.bq_embedding_backward(dy, ids, 10)
    assert d[2, 4].isinf() and d.isinf().sum() == 1 and not d.isnan().any()
    # a padding row and ids outside of the table take no part at all
    dy[:] = float("nan")
    assert not bq.bq_embedding_backward(dy, torch.full((5,), 4, device="cuda"), 10, 4).any()


# ---------------------------------------------------------------------------
# stable embedding
# ---------------------------------------------------------------------------

def check_stable(w, ids, lw, lb, yt, dy=None, padding=None, forward=True):
    num, dim = w.shape
    keep = ((ids >= 0) & (ids < num)).reshape(-1)
    rows = w[ids.reshape(-1)[keep].long()]
    if forward:
        y = bq.bq_stable_embedding_forward(w, ids, lw, lb, EPS, yt)
        yr, xh, _, _ = ref.layer_norm(rows, lw, lb, EPS)
        ref.check(y.view(-1, dim), yr, ref.forward_bound(yr, xh, lw, yt, dim), "y")
    if dy is None:
        dy = normal((*ids.shape, dim), 4, 0.01).to(yt)
    d, dw, db = bq.bq_stable_embedding_backward(dy, ids, w, lw, EPS, padding)
    # the definition: the layer norm's gradient of every token, summed by row
    s, a, count = ref.row_sums(dy, ids, num)
    used = count > 0
    _, xh, mr, rr = ref.layer_norm(w, lw, lb, EPS)
    g, dwr, dbr = ref.layer_norm_grads(s[used], xh[used], rr[used], lw)
    want = torch.zeros_like(s)
    want[used] = g
    se = ref.sum_error(a, count)[used]
    de, dwe, dbe = ref.backward_bounds(s[used], xh[used], mr[used], rr[used], lw, g, dwr, dbr,
                                       w.dtype, w.dtype, dy_error=se)
    bound = torch.zeros_like(s)
    bound[used] = de
    if padding is not None:
        want[padding] = 0.0
        assert not d[padding].any()
    ref.check(d, want, bound, "dweight")
    ref.check(dw, dwr, dwe, "dnorm_weight")
    ref.check(db, dbr, dbe, "dnorm_bias")


def stable_inputs(num, dim, wt, seed=0):
    return (normal((num, dim), seed, 0.05).to(wt), (1 + normal((dim,), seed + 1, 0.1)).to(wt),
            normal((dim,), seed + 2, 0.05).to(wt))


@pytest.mark.parametrize("types", TYPES, ids=str)
@pytest.mark.parametrize("dim", [2, 5, 64, 256, 300, 1000, 1600, 2051, 5000, 9000, 16384])
def test_stable_dims(dim, types):
    wt, yt = types
    w, lw, lb = stable_inputs(97, dim, wt)
    for count in (1, 50, 400 if dim < 3000 else 90):
        say("stable embedding", dim, types, count)
        check_stable(w, word_ids(count, 97, dim), lw, lb, yt)
    check_stable(w, word_ids(200, 97, dim), lw, lb, yt, padding=0)


@pytest.mark.parametrize("num,count", [(1, 500), (5000, 3), (50257, 4097), (70001, 30000)])
def test_stable_tables(num, count):
    w, lw, lb = stable_inputs(num, 48, F32)
    say("stable embedding table", num, count)
    check_stable(w, word_ids(count, num, 1).int(), lw, lb, F32, padding=num - 1)
    check_stable(w, uniform_ids(count, num, 2), None, None, BF16)


def test_stable_same_as_its_parts_and_only_what_is_asked_for():
    w, lw, lb = stable_inputs(200, 96, F32)
    ids = word_ids(999, 200, 1).view(27, 37)
    say("stable embedding parts")
    y = bq.bq_stable_embedding_forward(w, ids, lw, lb, EPS)
    # both kernels normalize a row alike
    assert torch.equal(y, bq.bq_layer_norm_forward(bq.bq_embedding_forward(w, ids), lw, lb, EPS))
    dy = normal((27, 37, 96), 5)
    d, dw, db = bq.bq_stable_embedding_backward(dy, ids, w, lw, EPS)
    alone, none, none2 = bq.bq_stable_embedding_backward(dy, ids, w, lw, EPS, need_norm=False)
    assert torch.equal(d, alone) and none is None and none2 is None


# ---------------------------------------------------------------------------
# gradients through torch, streams, repeats
# ---------------------------------------------------------------------------

def test_same_bits_and_other_streams():
    w, lw, lb = stable_inputs(3000, 200, F32)
    ids = word_ids(20000, 3000, 1)
    dy = normal((20000, 200), 5)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    say("embedding side stream")
    first = [bq.bq_embedding_backward(dy, ids, 3000),
             *bq.bq_stable_embedding_backward(dy, ids, w, lw, EPS)]
    again = [bq.bq_embedding_backward(dy, ids, 3000, stream=side),
             *bq.bq_stable_embedding_backward(dy, ids, w, lw, EPS, stream=side)]
    y = bq.bq_stable_embedding_forward(w, ids, lw, lb, EPS, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    for s, t in zip(first, again):
        assert torch.equal(s, t)
    assert torch.equal(y, bq.bq_stable_embedding_forward(w, ids, lw, lb, EPS))


def test_embedding_module():
    say("embedding module")
    emb = nn.Embedding(50, 24, padding_idx=-1, scale=4.0, out_dtype=BF16, device="cuda")
    ids = word_ids(90, 50, 1).view(9, 10)
    y = emb(ids)
    assert y.dtype == BF16 and y.shape == (9, 10, 24)
    dy = normal((9, 10, 24), 3).to(BF16)
    y.backward(dy)
    check_lookup_grad(emb.weight.grad, dy, ids, 50, F32, 4.0, 49)
    # transposed ids; a gradient that is one value for all
    emb.weight.grad = None
    emb(ids.t()).sum().backward()
    check_lookup_grad(emb.weight.grad, torch.ones((90, 24), device="cuda"), ids, 50, F32, 4.0, 49)


@pytest.mark.parametrize("out", [F32, F16])
def test_stable_module_against_plain(out):
    """fused=True and plain torch, the same parameters: both within their bounds of 64 bits."""
    torch.manual_seed(0)
    say("stable module", out)
    fused = nn.StableEmbedding(400, 80, padding_idx=3, device="cuda", fused=True, out_dtype=out)
    ids = word_ids(600, 400, 1).view(20, 30)
    y = fused(ids)
    assert y.dtype == out
    dy = normal((20, 30, 80), 2, 0.01).to(out)
    y.backward(dy)
    with torch.no_grad():
        check_stable(fused.weight, ids, fused.norm.weight, fused.norm.bias, out, dy, padding=3)
    plain = nn.StableEmbedding(400, 80, padding_idx=3, device="cuda")
    assert plain.state_dict().keys() == fused.state_dict().keys()
    plain.load_state_dict(fused.state_dict())
    plain(ids).backward(dy.float())
    for p, q in zip(plain.parameters(), fused.parameters()):
        scale = float(p.grad.abs().max())
        assert float((p.grad - q.grad).abs().max()) <= 2e-5 * scale


def test_stable_gradient_against_differences():
    """As the layer norm's: the central difference of the 64-bit form along a direction."""
    w, lw, lb = stable_inputs(30, 40, F32)
    w = w * 20
    ids = word_ids(100, 30, 1)
    c = normal((100, 40), 9)
    leaves = [t.clone().requires_grad_() for t in (w, lw, lb)]
    say("stable differences")
    grads = torch.autograd.grad((nn.stable_embedding(ids, *leaves, EPS) * c).sum(), leaves)
    for i, g in enumerate(grads):
        v = normal(g.shape, 20 + i)
        h = 1e-4

        def f(s):
            args = [t.double() for t in (w, lw, lb)]
            args[i] = args[i] + s * v.double()
            return (ref.layer_norm(args[0][ids], args[1], args[2], EPS)[0] * c.double()).sum()
        diff = float((f(h) - f(-h)) / (2 * h))
        terms = float((g.double() * v.double()).abs().sum())
        assert abs(float((g.double() * v.double()).sum()) - diff) <= 1e-5 * terms + 1e-5
