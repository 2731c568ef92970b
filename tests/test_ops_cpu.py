"""Refusals of the operators around the optimizer step, without a GPU: every call below
carries at least one invalid argument, or is one that launches nothing, so none reaches the
HIP runtime; the addresses are never dereferenced."""
import ctypes

import pytest
import torch

from paper_2110_02861_amd import bq, nn, optim

A = 0x10000
ODD = 0x10001
F, H, B = bq.BQ_F32, bq.BQ_F16, bq.BQ_BF16
NULL, SIZE, DTYPE, ALIGN, ARG, ENUM, OK = (bq.BQ_ERR_NULL, bq.BQ_ERR_SIZE, bq.BQ_ERR_DTYPE,
                                           bq.BQ_ERR_ALIGN, bq.BQ_ERR_ARG, bq.BQ_ERR_ENUM, bq.BQ_OK)
NAN, INF = float("nan"), float("inf")


def call(fn, defaults, **change):
    args = dict(defaults)
    assert set(change) <= set(args)
    args.update(change)
    return getattr(bq.lib(), fn)(*args.values())


LN = dict(dtype=F, pdtype=F, x=A, rows=4, cols=8, stride=8, w=A, b=A, eps=1e-5, y=A, mean=A,
          rstd=A, stream=None)


@pytest.mark.parametrize("change,want", [
    (dict(dtype=3), DTYPE), (dict(dtype=-1), DTYPE), (dict(pdtype=H), DTYPE),
    (dict(dtype=H, pdtype=B), DTYPE), (dict(rows=-1), SIZE), (dict(cols=0), SIZE),
    (dict(cols=-5), SIZE), (dict(cols=1 << 31), SIZE), (dict(rows=1 << 41), SIZE),
    (dict(rows=1 << 40, cols=1 << 30), SIZE), (dict(stride=-1), SIZE),
    (dict(rows=1 << 30, stride=1 << 40), SIZE), (dict(eps=-1e-5), ARG), (dict(eps=NAN), ARG),
    (dict(eps=INF), ARG), (dict(x=None), NULL), (dict(y=None), NULL), (dict(mean=None), NULL),
    (dict(rstd=None), NULL), (dict(x=A + 2), ALIGN), (dict(dtype=H, x=ODD), ALIGN),
    (dict(w=ODD), ALIGN), (dict(b=A + 2), ALIGN), (dict(mean=A + 2), ALIGN), (dict(y=ODD), ALIGN),
    (dict(rows=0, x=None, y=None), OK)])
def test_layer_norm_forward(change, want):
    assert call("bq_layer_norm_forward", LN, **change) == want


LNB = dict(dtype=F, pdtype=F, dy=A, dys=8, x=A, xs=8, rows=4, cols=8, w=A, mean=A, rstd=A, dx=A,
           dw=A, db=A, ws=A, stream=None)


@pytest.mark.parametrize("change,want", [
    (dict(dtype=7), DTYPE), (dict(dtype=B, pdtype=H), DTYPE), (dict(rows=-1), SIZE),
    (dict(cols=0), SIZE), (dict(dys=-1), SIZE), (dict(xs=-1), SIZE), (dict(dy=None), NULL),
    (dict(x=None), NULL), (dict(mean=None), NULL), (dict(rstd=None), NULL), (dict(ws=None), NULL),
    (dict(ws=A + 8), ALIGN), (dict(dx=A + 2), ALIGN), (dict(dw=A + 2), ALIGN),
    (dict(dy=ODD), ALIGN), (dict(dx=None, dw=None, db=None), OK),
    (dict(rows=0, dw=None, db=None, ws=None), OK)])
def test_layer_norm_backward(change, want):
    assert call("bq_layer_norm_backward", LNB, **change) == want


EMB = dict(dtype=F, out=F, w=A, num=100, dim=8, ids=A, bits=64, count=4, scale=1.0, y=A,
           stream=None)


@pytest.mark.parametrize("change,want", [
    (dict(dtype=3), DTYPE), (dict(dtype=H), DTYPE), (dict(dtype=H, out=B), DTYPE),
    (dict(bits=16), DTYPE), (dict(bits=0), DTYPE), (dict(num=0), SIZE),
    (dict(num=(1 << 31) - 1), SIZE), (dict(dim=0), SIZE), (dict(dim=(1 << 24) + 1), SIZE),
    (dict(count=-1), SIZE), (dict(count=1 << 31), SIZE), (dict(scale=NAN), ARG),
    (dict(scale=INF), ARG), (dict(w=None), NULL), (dict(ids=None), NULL), (dict(y=None), NULL),
    (dict(ids=A + 4), ALIGN), (dict(bits=32, ids=A + 2), ALIGN), (dict(w=A + 2), ALIGN),
    (dict(y=ODD), ALIGN), (dict(count=0, w=None, ids=None, y=None), OK)])
def test_embedding_forward(change, want):
    assert call("bq_embedding_forward", EMB, **change) == want


EMBB = dict(dtype=F, out=F, dy=A, ids=A, bits=64, count=4, num=100, dim=8, padding=-1, scale=1.0,
            dw=A, ws=A, stream=None)


@pytest.mark.parametrize("change,want", [
    (dict(dtype=H, out=F), DTYPE), (dict(bits=8), DTYPE), (dict(num=0), SIZE),
    (dict(count=1 << 31), SIZE), (dict(padding=-2), ARG), (dict(padding=100), ARG),
    (dict(scale=NAN), ARG), (dict(dy=None), NULL), (dict(ids=None), NULL), (dict(dw=None), NULL),
    (dict(ws=None), NULL), (dict(count=0, ws=None), NULL), (dict(ws=A + 8), ALIGN),
    (dict(dy=ODD), ALIGN), (dict(dw=ODD), ALIGN)])
def test_embedding_backward(change, want):
    assert call("bq_embedding_backward", EMBB, **change) == want


SE = dict(dtype=F, out=F, w=A, num=100, dim=8, ids=A, bits=64, count=4, nw=A, nb=A, eps=1e-5, y=A,
          stream=None)
SEB = dict(dtype=F, out=F, dy=A, ids=A, bits=64, count=4, w=A, num=100, dim=8, padding=-1, nw=A,
           eps=1e-5, dw=A, dnw=A, dnb=A, ws=A, stream=None)


@pytest.mark.parametrize("change,want", [
    (dict(dtype=B, out=F), DTYPE), (dict(dim=16385), SIZE), (dict(eps=-1.0), ARG),
    (dict(eps=NAN), ARG), (dict(w=None), NULL), (dict(y=None), NULL), (dict(nw=A + 2), ALIGN),
    (dict(nb=ODD), ALIGN), (dict(count=0, y=None), OK)])
def test_stable_embedding_forward(change, want):
    assert call("bq_stable_embedding_forward", SE, **change) == want


@pytest.mark.parametrize("change,want", [
    (dict(dtype=B, out=F), DTYPE), (dict(dim=16385), SIZE), (dict(eps=INF), ARG),
    (dict(padding=100), ARG), (dict(padding=-2), ARG), (dict(w=None), NULL), (dict(dw=None), NULL),
    (dict(dy=None), NULL), (dict(ws=None), NULL), (dict(count=0, ws=None), NULL),
    (dict(dnw=A + 2), ALIGN), (dict(dnb=ODD), ALIGN), (dict(ws=A + 4), ALIGN)])
def test_stable_embedding_backward(change, want):
    assert call("bq_stable_embedding_backward", SEB, **change) == want


def grads(*rows):
    arr = (bq.bq_grad * max(1, len(rows)))()
    for i, r in enumerate(rows):
        arr[i].data, arr[i].numel, arr[i].dtype = r
    return arr


GOOD = (A, 10, F)


@pytest.mark.parametrize("rows,n,kind,ws,norm,want", [
    ([GOOD], 1, 2, A, A, ENUM), ([GOOD], -1, 0, A, A, SIZE), (None, 1, 0, A, A, NULL),
    ([GOOD], 1, 0, None, A, NULL), ([GOOD], 1, 0, A, None, NULL), ([GOOD], 1, 0, A + 4, A, ALIGN),
    ([GOOD], 1, 0, A, A + 2, ALIGN), ([GOOD, (A, 10, 3)], 2, 0, A, A, DTYPE),
    ([(A, -1, F)], 1, 1, A, A, SIZE), ([(A, 1 << 41, F)], 1, 0, A, A, SIZE),
    ([(A, 1 << 40, F)] * 5, 5, 0, A, A, SIZE), ([(None, 10, F)], 1, 0, A, A, NULL),
    ([(A + 2, 10, F)], 1, 0, A, A, ALIGN), ([(ODD, 10, B)], 1, 0, A, A, ALIGN)])
def test_grad_norm(rows, n, kind, ws, norm, want):
    arr = None if rows is None else grads(*rows)
    assert bq.lib().bq_grad_norm(arr, n, kind, ws, norm, None) == want
    assert bq.lib().bq_clip_grad_norm(arr, n, kind, 1.0, ws, norm, None) == want


def test_clip_limit():
    for bad in (-1.0, NAN):
        assert bq.lib().bq_clip_grad_norm(grads(GOOD), 1, 0, bad, A, A, None) == ARG
        with pytest.raises(ValueError):
            optim.clip_grad_norm_([], bad)
    with pytest.raises(ValueError):
        bq.bq_grad_norm([], norm_type=3)


def test_workspace_sizes():
    lib = bq.lib()
    assert lib.bq_layer_norm_workspace_bytes(10, 0) == 0
    assert lib.bq_layer_norm_workspace_bytes(-1, 8) == 0
    assert lib.bq_layer_norm_workspace_bytes(10, 8) >= 2 * 8 * 4
    # rows above 16384 elements: fewer partial rows the longer they are
    assert lib.bq_layer_norm_workspace_bytes(4096, 1 << 20) == 4 * 2 * (1 << 20) * 4
    assert lib.bq_layer_norm_workspace_bytes(3, 1 << 20) == 3 * 2 * (1 << 20) * 4
    assert lib.bq_layer_norm_workspace_bytes(1 << 20, 1 << 27) == 2 * (1 << 27) * 4
    assert lib.bq_embedding_workspace_bytes(1 << 31, 10, 8) == 0
    assert lib.bq_embedding_workspace_bytes(10, 0, 8) == 0
    assert lib.bq_stable_embedding_workspace_bytes(10, 10, 16385) == 0
    assert lib.bq_embedding_workspace_bytes(100, 10, 8) >= 100 * 8
    assert lib.bq_embedding_workspace_bytes(0, 10, 8) >= 0
    assert lib.bq_stable_embedding_workspace_bytes(0, 10, 8) >= 2 * 8 * 4
    assert lib.bq_grad_norm_workspace_bytes(-1) == 0
    assert lib.bq_grad_norm_workspace_bytes(0) == 8
    assert lib.bq_grad_norm_workspace_bytes((1 << 31) - 1) > (1 << 31) // 180 * 8
    # more than 4 GiB: the sizes are 64-bit
    assert lib.bq_embedding_workspace_bytes((1 << 31) - 1, 50257, 4096) > 1 << 36
    assert ctypes.sizeof(bq.bq_grad) == 24


def test_cpu_tensors_raise():
    x, w = torch.randn(4, 8), torch.randn(8)
    table, ids = torch.randn(10, 8), torch.tensor([1, 2])
    for fn in (lambda: bq.bq_layer_norm_forward(x, w, w), lambda: nn.layer_norm(x, w, w),
               lambda: nn.LayerNorm(8)(x), lambda: bq.bq_embedding_forward(table, ids),
               lambda: nn.embedding(ids, table), lambda: nn.Embedding(10, 8)(ids),
               lambda: nn.stable_embedding(ids, table),
               lambda: nn.StableEmbedding(10, 8, fused=True)(ids),
               lambda: bq.bq_embedding_backward(x, ids, 10), lambda: bq.bq_grad_norm([x]),
               lambda: bq.bq_clip_grad_norm([x], 1.0)):
        with pytest.raises(TypeError):
            fn()
    p = torch.nn.Parameter(x)
    p.grad = x.clone()
    with pytest.raises(TypeError):
        optim.clip_grad_norm_([p], 1.0)
    with pytest.raises(TypeError):
        optim.Adam8bit([p]).clip_grad_norm_(1.0)


def test_modules():
    with pytest.raises(ValueError):
        nn.LayerNorm((4, 8))
    with pytest.raises(ValueError):
        nn.Embedding(10, 8, scale=INF)
    for kw in (dict(fused=True, max_norm=1.0), dict(fused=True, scale_grad_by_freq=True),
               dict(out_dtype=torch.float16)):
        with pytest.raises(ValueError):
            nn.StableEmbedding(10, 8, **kw)
    assert nn.LayerNorm(8).state_dict().keys() == torch.nn.LayerNorm(8).state_dict().keys()
    # a module saved before `fused` existed runs in plain torch
    emb = nn.StableEmbedding(10, 8)
    del emb.fused, emb.out_dtype
    assert emb(torch.tensor([1, 2])).shape == (2, 8)
