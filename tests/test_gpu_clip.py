"""The norm of a list of gradients, and clipping, on the GPU."""
import math

import pytest
import torch

from paper_2110_02861_amd import bq, optim
from tests import ops_reference as ref
from tests.gpu_helpers import needs_gpu, say

pytestmark = [pytest.mark.gpu, needs_gpu]

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
INF = float("inf")


def normal(n, seed, std=1e-2, dtype=F32):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.empty(n, device="cuda").normal_(0.0, std, generator=g).to(dtype)


def grads_of(sizes, dtypes, seed=0):
    return [normal(n, seed + i, dtype=dtypes[i % len(dtypes)]) for i, n in enumerate(sizes)]


def norm64(grads, kind):
    if not any(g.numel() for g in grads):
        return 0.0
    flat = torch.cat([g.double().reshape(-1) for g in grads])
    return float(flat.norm()) if kind == 2 else float(flat.abs().max())


def check_clip(grads, max_norm, kind=2.0):
    """Norm: fp64 sums, one rounding (U), and the reference's own (1e-12).  Clipped values: the
    coefficient is rounded once, the product once in fp32 and once in the type."""
    before = [g.clone() for g in grads]
    want = norm64(grads, kind)
    norm = bq.bq_clip_grad_norm(grads, max_norm, kind)
    assert norm.shape == () and norm.dtype == F32
    assert abs(float(norm) - want) <= ref.U * 1.01 * want
    c = min(1.0, max_norm / (want + 1e-6))
    for g, b in zip(grads, before):
        if c == 1.0:
            assert torch.equal(g, b)
        else:
            r = b.double() * c
            ref.check(g, r, (2.01 * ref.U + ref.HALF[g.dtype]) * r.abs() + ref.TINY[g.dtype] * 1.01,
                      "clipped")
    return norm


@pytest.mark.parametrize("kind", [2.0, INF])
@pytest.mark.parametrize("dtypes", [(F32,), (F16,), (BF16,), (F16, F32, BF16)], ids=str)
@pytest.mark.parametrize("sizes", [(1,), (3, 0, 5), (4096,), (4097, 8191, 8192, 8193, 1),
                                   (1 << 20, 77), (30_000_001,)], ids=str)
def test_lists(sizes, dtypes, kind):
    say("clip", sizes, dtypes, kind)
    grads = grads_of(sizes, dtypes)
    n = norm64(grads, kind)
    assert abs(float(bq.bq_grad_norm(grads, kind)) - n) <= ref.U * 1.01 * n
    check_clip(grads, 2 * n + 1.0, kind)
    check_clip(grads, 0.1 * n, kind)
    check_clip(grads, 0.0, kind)


@pytest.mark.parametrize("count", [179, 180, 181, 580, 1000])
def test_many_tensors(count):
    """More tensors than one launch carries, and more partial sums than a clip launch adds."""
    say("clip many", count)
    sizes = [(7919 * i) % 60000 + (i % 5) for i in range(count)]
    grads = grads_of(sizes, (F16, F32, BF16))
    check_clip(grads, 0.5 * norm64(grads, 2))


def test_many_partial_sums():
    say("clip many partial sums")
    grads = grads_of([100_000] * 600, (F32,))
    check_clip(grads, 0.5 * norm64(grads, 2))
    check_clip(grads, 0.5 * norm64(grads, INF), INF)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_unaligned_views_leave_their_neighbours(dtype):
    flat = normal(200_000, 1, dtype=dtype)
    keep = flat.clone()
    spans = [(1, 4099), (5000, 5001), (5003, 13197), (13200, 199_999)]
    say("clip views", dtype)
    check_clip([flat[a:b] for a, b in spans], 0.01)
    inside = torch.zeros(200_000, dtype=torch.bool, device="cuda")
    for a, b in spans:
        inside[a:b] = True
    assert torch.equal(flat[~inside], keep[~inside])


def test_orders_of_memory():
    """A transposed or channels-last gradient fills one range; a strided one does not."""
    a = normal(600, 1).view(20, 30).t()
    b = normal(2 * 3 * 4 * 5, 2).view(2, 3, 4, 5).to(memory_format=torch.channels_last)
    say("clip orders")
    check_clip([a, b], 0.01)
    with pytest.raises(ValueError):
        bq.bq_grad_norm([normal(100, 1)[::2]])
    with pytest.raises(ValueError):
        bq.bq_grad_norm([normal(10, 1).expand(4, 10)])


def test_large_and_small_values():
    """Squares that fp32 cannot hold, at both ends."""
    say("clip range")
    for scale in (1e30, 1e-30):
        check_clip([normal(5000, 1, scale), normal(300, 2, scale)], 1.0)


def test_not_finite():
    say("clip not finite")
    for bad in (INF, -INF, float("nan")):
        for kind in (2.0, INF):
            g = [normal(9000, 1), normal(100, 2)]
            g[0][8999] = bad
            want = torch.nn.utils.get_total_norm([t.clone() for t in g], kind)
            norm = bq.bq_clip_grad_norm(g, 1.0, kind)
            assert torch.equal(norm, want) or (norm.isnan() and want.isnan())
            if norm.isnan():
                assert g[0].isnan().all() and g[1].isnan().all()
            else:  # c = 0
                assert g[0][8999].isnan() and not g[0][:8999].any() and not g[1].any()


def test_empty_list():
    say("clip empty")
    for grads in ([], [torch.zeros(0, device="cuda")]):
        assert float(bq.bq_grad_norm(grads)) == 0.0
        assert float(bq.bq_clip_grad_norm(grads, 1.0)) == 0.0


def test_beyond_2_31_elements():
    say("clip 2^31")
    n = (1 << 31) + 5000
    g = torch.full((n,), 1e-3, dtype=F16, device="cuda")
    g[-1] = 2.0
    v = float(g[0])
    want = math.sqrt(v * v * (n - 1) + 4.0)
    norm = bq.bq_clip_grad_norm([g], 0.5 * want)
    assert abs(float(norm) - want) <= ref.U * 1.01 * want
    assert float(g[-1]) == 1.0 and float(g[0]) == float(g[-2]) == float(g[1 << 31])
    assert abs(float(g[0]) - 0.5 * v) <= 0.5 * v * ref.HALF[F16] + ref.TINY[F16]


def test_same_bits_streams_and_parameters():
    say("clip parameters")
    params = [torch.nn.Parameter(normal(n, n)) for n in (1000, 33, 70000)]
    unused = torch.nn.Parameter(normal(5, 5))
    for p in params:
        p.grad = normal(p.numel(), p.numel() + 1)
    copies = [p.grad.clone() for p in params]
    version = params[0].grad._version
    norm = optim.clip_grad_norm_(iter(params + [unused, params[0]]), 0.5)
    assert params[0].grad._version > version
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    again = bq.bq_clip_grad_norm(copies, 0.5, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(norm, again)
    for p, c in zip(params, copies):
        assert torch.equal(p.grad, c)
    want = torch.nn.utils.get_total_norm([p.grad.double() for p in params])
    assert abs(float(optim.grad_norm(params)) - float(want)) <= 1e-6 * float(want)
    opt = optim.Adam8bit(params + [unused])
    half = 0.5 * float(want)
    opt.clip_grad_norm_(half)
    assert abs(float(optim.grad_norm(params)) - half) <= 1e-5 * half
    params[1].grad[3] = INF
    kept = [p.grad.clone() for p in params]
    with pytest.raises(RuntimeError):
        optim.clip_grad_norm_(params, 1.0, error_if_nonfinite=True)
    for p, c in zip(params, kept):
        assert torch.equal(p.grad, c)
