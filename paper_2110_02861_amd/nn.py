"""Layers for models that the 8-bit optimizers train: the stable embedding layer of
Section 3.3, and the layer norm and embedding that it is made of, in HIP kernels.

``layer_norm``, ``embedding`` and ``stable_embedding`` are functions with gradients over
libbq's kernels (``bq.bq_layer_norm_forward`` and its kin), ``LayerNorm`` and ``Embedding``
the modules, with the parameters, names and initial values of torch's.  They take GPU
tensors in fp32, fp16 or bf16 and raise for others: there is no CPU fallback.  Gradients
are of first order, and the same bits every time.  Tracing (``torch.jit.trace``,
``make_fx``) and tensors with a forward-mode tangent raise.  A training step is captured into a graph
like one of torch's own layers: backward passes on a side stream, and no graph of an
eager pass over the same leaves still alive.  ``StableEmbedding`` runs in plain torch
unless it is built with ``fused=True``.

The stable embedding: a word embedding initialized with Xavier-uniform values whose output goes
through a layer norm (add position embeddings after it).  Its weight carries
the attribute ``bq_32bit_state = True``, which makes every 8-bit optimizer of
``paper_2110_02861_amd.optim`` keep that weight's optimizer states in 32 bit
(the paper keeps only this layer's states in 32 bit); the weight and its
gradient keep their own dtype.
"""
from __future__ import annotations

import math

import torch
import torch.nn.functional as F
from torch.autograd.function import once_differentiable

from . import bq


def _device_of(t, name):
    """A context in which t's device is the current one."""
    bq._eager()
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a GPU torch tensor (libbq runs on the GPU only)")
    return torch.cuda.device(t.get_device())


def _wants_grad(*tensors):
    return torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in tensors)


def _packed_rows(x):
    """x as the kernels take it: packed, or a matrix of packed rows."""
    x = x.resolve_neg()
    if x.is_contiguous() or (x.dim() == 2 and x.stride(1) == 1):
        return x
    return x.contiguous()


def _packed(t):
    return None if t is None else t.resolve_neg().contiguous()


class _LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, eps):
        with _device_of(x, "x"):
            y, mean, rstd = bq.bq_layer_norm_forward(x, weight, bias, eps, stats=True)
        ctx.save_for_backward(x, weight, mean, rstd)
        ctx.param_dtype = None if bias is None else bias.dtype
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        x, weight, mean, rstd = ctx.saved_tensors
        need_x, need_w, need_b, _ = ctx.needs_input_grad
        with _device_of(dy, "dy"):
            # (hooks on saved tensors may hand them back in another order of memory)
            dx, dw, db = bq.bq_layer_norm_backward(
                _packed_rows(dy), _packed_rows(x), _packed(weight), _packed(mean), _packed(rstd),
                need_dx=need_x, need_params=need_w or need_b, param_dtype=ctx.param_dtype)
        return dx, dw if need_w else None, db if need_b else None, None


def layer_norm(x, weight=None, bias=None, eps: float = 1e-5):
    """The layer norm of x over its last dimension: (x - mean) / sqrt(var + eps) * weight +
    bias.  x in fp32, fp16 or bf16; weight and bias of that type or fp32, each may be
    None.  Statistics and sums are fp32."""
    y = bq.host().layer_norm(x, weight, bias, eps, True)
    if y is not None:
        return y
    bq._no_tangent(x, weight, bias)
    with _device_of(x, "x"):
        x = _packed_rows(x)
        if _wants_grad(x, weight, bias):
            return _LayerNorm.apply(x, weight, bias, eps)
        return bq.bq_layer_norm_forward(x, weight, bias, eps)


class _Embedding(torch.autograd.Function):
    @staticmethod
    def forward(ctx, ids, weight, padding_idx, scale, out_dtype):
        with _device_of(weight, "weight"):
            y = bq.bq_embedding_forward(weight, ids, scale, out_dtype)
        ctx.save_for_backward(ids)
        ctx.call = (weight.size(0), padding_idx, scale, weight.dtype)
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        ids, = ctx.saved_tensors
        with _device_of(dy, "dy"):
            dw = bq.bq_embedding_backward(_packed(dy), _packed(ids), *ctx.call)
        return None, dw, None, None, None


def embedding(ids, weight, padding_idx=None, scale: float = 1.0, out_dtype=None):
    """scale * weight[ids], with a dense gradient of weight (zero for the row padding_idx)
    that is summed by sorted ids, in fp32 and in one order.  ids: int64 or int32, any
    shape; out_dtype: weight's type, or any of the three where weight is fp32.  An id
    outside of the table gives a row of NaN and no gradient."""
    y = bq.host().embedding(ids, weight, padding_idx, scale, out_dtype, True)
    if y is not None:
        return y
    bq._no_tangent(weight)
    with _device_of(weight, "weight"):
        bq._padding(padding_idx, weight.size(0))
        ids = ids.contiguous()
        if _wants_grad(weight):
            return _Embedding.apply(ids, weight, padding_idx, scale, out_dtype)
        return bq.bq_embedding_forward(weight, ids, scale, out_dtype)


class _StableEmbedding(torch.autograd.Function):
    @staticmethod
    def forward(ctx, ids, weight, norm_weight, norm_bias, eps, padding_idx, out_dtype):
        with _device_of(weight, "weight"):
            y = bq.bq_stable_embedding_forward(weight, ids, norm_weight, norm_bias, eps,
                                               out_dtype)
        ctx.save_for_backward(ids, weight, norm_weight)
        ctx.call = (eps, padding_idx)
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        ids, weight, norm_weight = ctx.saved_tensors
        need = ctx.needs_input_grad
        with _device_of(dy, "dy"):
            dweight, dw, db = bq.bq_stable_embedding_backward(
                _packed(dy), _packed(ids), _packed(weight), _packed(norm_weight), *ctx.call,
                need_norm=need[2] or need[3])
        return (None, dweight if need[1] else None, dw if need[2] else None,
                db if need[3] else None, None, None, None)


def stable_embedding(ids, weight, norm_weight=None, norm_bias=None, eps: float = 1e-5,
                     padding_idx=None, out_dtype=None):
    """layer_norm(weight[ids], norm_weight, norm_bias, eps) as one operator: the looked-up
    rows are never in memory, and the backward pass takes the layer norm's gradient once
    per distinct id.  All parameters have weight's type; rows of up to
    bq.BQ_STABLE_EMBEDDING_MAX_DIM elements.  The other arguments as ``embedding``."""
    y = bq.host().stable_embedding(ids, weight, norm_weight, norm_bias, eps, padding_idx,
                                   out_dtype, True)
    if y is not None:
        return y
    bq._no_tangent(weight, norm_weight, norm_bias)
    with _device_of(weight, "weight"):
        bq._padding(padding_idx, weight.size(0))
        ids = ids.contiguous()
        if _wants_grad(weight, norm_weight, norm_bias):
            return _StableEmbedding.apply(ids, weight, norm_weight, norm_bias, eps, padding_idx,
                                          out_dtype)
        return bq.bq_stable_embedding_forward(weight, ids, norm_weight, norm_bias, eps, out_dtype)


def _table_sizes(embeddings):
    if embeddings.dim() != 2:
        raise ValueError("embeddings must be a matrix")
    return embeddings.shape


class LayerNorm(torch.nn.LayerNorm):
    """torch.nn.LayerNorm over the last dimension, through ``layer_norm``: its parameters may
    be fp32 with inputs in fp16 or bf16."""

    def __init__(self, normalized_shape, eps: float = 1e-5, elementwise_affine: bool = True,
                 bias: bool = True, device=None, dtype=None):
        super().__init__(normalized_shape, eps, elementwise_affine, bias, device, dtype)
        if len(self.normalized_shape) != 1:
            raise ValueError("the HIP layer norm normalizes the last dimension only")

    def forward(self, input: torch.Tensor) -> torch.Tensor:
        if input.dim() == 0 or input.size(-1) != self.normalized_shape[0]:
            raise ValueError(f"expected a last dimension of {self.normalized_shape[0]}")
        return layer_norm(input, self.weight, self.bias, self.eps)


class Embedding(torch.nn.Embedding):
    """torch.nn.Embedding through ``embedding``: the rows times ``scale`` (e.g. sqrt of the
    dimension), in ``out_dtype``."""

    def __init__(self, num_embeddings: int, embedding_dim: int, padding_idx=None,
                 scale: float = 1.0, out_dtype=None, device=None, dtype=None, *, _weight=None,
                 _freeze: bool = False):
        if not math.isfinite(scale):
            raise ValueError(f"invalid scale {scale}")
        super().__init__(num_embeddings, embedding_dim, padding_idx, _weight=_weight,
                         _freeze=_freeze, device=device, dtype=dtype)
        self.scale = float(scale)
        self.out_dtype = out_dtype

    @classmethod
    def from_pretrained(cls, embeddings, freeze: bool = True, padding_idx=None, *,
                        scale: float = 1.0, out_dtype=None):
        """A module around the table embeddings, which gets no gradient if freeze."""
        return cls(*_table_sizes(embeddings), padding_idx, scale, out_dtype, _weight=embeddings,
                   _freeze=freeze)

    def forward(self, input: torch.Tensor) -> torch.Tensor:
        return embedding(input, self.weight, self.padding_idx, self.scale, self.out_dtype)


def _called(norm):
    """Whether a layer norm's module has to be called for what it does (a class made for its
    parametrized weight has torch's forward)."""
    forward = getattr(type(norm), "forward", None)
    return forward not in (torch.nn.LayerNorm.forward, LayerNorm.forward) or bool(
        "forward" in norm.__dict__ or norm._forward_hooks or norm._forward_pre_hooks or
        norm._backward_hooks or norm._backward_pre_hooks)


class StableEmbedding(torch.nn.Embedding):
    """fused=True runs lookup and layer norm as one HIP operator (``stable_embedding``), with
    results that differ from plain torch's by rounding; out_dtype is its result's type.  The
    operator does not call the module ``norm``: where that has hooks, or another forward than
    a layer norm's, the two run apart."""

    fused, out_dtype = False, None  # of modules saved before there was a choice

    def __init__(self, num_embeddings: int, embedding_dim: int, padding_idx=None,
                 max_norm=None, norm_type: float = 2.0, scale_grad_by_freq: bool = False,
                 sparse: bool = False, device=None, dtype=None, fused: bool = False,
                 out_dtype=None, *, _weight=None, _freeze: bool = False):
        if sparse:
            raise ValueError("the 8-bit optimizers take dense gradients only")
        if fused and (max_norm is not None or scale_grad_by_freq):
            raise ValueError("the fused stable embedding has no max_norm or scale_grad_by_freq")
        if out_dtype is not None and not fused:
            raise ValueError("out_dtype needs fused=True")
        super().__init__(num_embeddings, embedding_dim, padding_idx, max_norm, norm_type,
                         scale_grad_by_freq, sparse=False, _weight=_weight, _freeze=_freeze,
                         device=device, dtype=dtype)
        if _weight is not None:
            device, dtype = _weight.device, _weight.dtype
        self.norm = torch.nn.LayerNorm(embedding_dim, device=device, dtype=dtype)
        self.weight.bq_32bit_state = True
        self.fused = bool(fused)
        self.out_dtype = out_dtype

    @classmethod
    def from_pretrained(cls, embeddings, freeze: bool = True, padding_idx=None, max_norm=None,
                        norm_type: float = 2.0, scale_grad_by_freq: bool = False,
                        sparse: bool = False, *, fused: bool = False, out_dtype=None):
        """A module around the table embeddings, which gets no gradient if freeze, with a layer
        norm of its own."""
        return cls(*_table_sizes(embeddings), padding_idx, max_norm, norm_type, scale_grad_by_freq,
                   sparse, fused=fused, out_dtype=out_dtype, _weight=embeddings, _freeze=freeze)

    def reset_parameters(self) -> None:
        torch.nn.init.xavier_uniform_(self.weight)
        self._fill_padding_idx_with_zero()

    def forward(self, input: torch.Tensor) -> torch.Tensor:
        if self.fused:
            if _called(self.norm):
                y = self.norm(embedding(input, self.weight, self.padding_idx))
                return y if self.out_dtype is None else y.to(self.out_dtype)
            return stable_embedding(input, self.weight, self.norm.weight, self.norm.bias,
                                    self.norm.eps, self.padding_idx, self.out_dtype)
        emb = F.embedding(input, self.weight, self.padding_idx, self.max_norm, self.norm_type,
                          self.scale_grad_by_freq, self.sparse)
        return self.norm(emb)
