"""nn's modules on the CPU: tables taken over from elsewhere, and a layer norm with hooks
inside of the fused stable embedding."""
import pytest
import torch
import torch.nn.functional as F

from paper_2110_02861_amd import nn


def test_embedding_from_pretrained():
    table = torch.randn(7, 5)
    emb = nn.Embedding.from_pretrained(table)
    assert type(emb) is nn.Embedding and emb.weight.data_ptr() == table.data_ptr()
    assert (emb.num_embeddings, emb.embedding_dim, emb.padding_idx) == (7, 5, None)
    assert not emb.weight.requires_grad and emb.scale == 1.0 and emb.out_dtype is None
    emb = nn.Embedding.from_pretrained(table, freeze=False, padding_idx=-1, scale=2.0,
                                       out_dtype=torch.float16)
    assert emb.weight.requires_grad and emb.padding_idx == 6
    assert emb.scale == 2.0 and emb.out_dtype == torch.float16
    assert torch.equal(emb.weight, table)  # the padding row as it was given
    with pytest.raises(TypeError):  # of torch's arguments, those that this module lacks
        nn.Embedding.from_pretrained(table, max_norm=1.0)
    with pytest.raises(ValueError):
        nn.Embedding.from_pretrained(table[0])


def test_stable_embedding_from_pretrained():
    table = torch.randn(7, 5, dtype=torch.float64)
    ids = torch.tensor([1, 6, 1])
    emb = nn.StableEmbedding.from_pretrained(table, padding_idx=2)
    assert type(emb) is nn.StableEmbedding and not emb.fused and emb.padding_idx == 2
    assert emb.weight.data_ptr() == table.data_ptr() and not emb.weight.requires_grad
    assert emb.weight.bq_32bit_state is True
    assert emb.norm.weight.dtype == torch.float64 and emb.norm.weight.requires_grad
    assert torch.equal(emb(ids), F.layer_norm(table[ids], (5,)))
    emb = nn.StableEmbedding.from_pretrained(table.float(), freeze=False, fused=True,
                                             out_dtype=torch.float16)
    assert emb.fused and emb.out_dtype == torch.float16 and emb.weight.requires_grad
    with pytest.raises(ValueError):
        nn.StableEmbedding.from_pretrained(table, sparse=True)
    with pytest.raises(ValueError):
        nn.StableEmbedding.from_pretrained(table, fused=True, max_norm=1.0)

def hooks(module):
    """Ways to be called when the module is, each with its handle."""
    yield module.register_forward_hook(lambda m, i, o: o + 1.0)
    yield module.register_forward_pre_hook(lambda m, i: (i[0] * 2.0,))
    yield module.register_full_backward_hook(lambda m, gi, go: None)
    yield module.register_full_backward_pre_hook(lambda m, go: None)


def test_fused_stable_embedding_calls_a_norm_that_has_hooks(monkeypatch):
    """The two layers run apart then, the lookup by its own operator (torch's here)."""
    emb = nn.StableEmbedding(10, 8, padding_idx=1, fused=True, out_dtype=torch.float16)
    plain = nn.StableEmbedding(10, 8, padding_idx=1)
    plain.load_state_dict(emb.state_dict())
    ids = torch.tensor([1, 2, 9])
    fused = object()
    monkeypatch.setattr(nn, "stable_embedding", lambda *a: fused)
    monkeypatch.setattr(nn, "embedding",
                        lambda i, w, padding_idx: F.embedding(i, w, padding_idx))
    assert emb(ids) is fused
    for h, g in zip(hooks(emb.norm), hooks(plain.norm)):
        assert torch.equal(emb(ids), plain(ids).half())
        h.remove()
        g.remove()
        assert emb(ids) is fused

    class Other(torch.nn.LayerNorm):
        def forward(self, x):
            return super().forward(x) * 3.0
    emb.norm = Other(8)
    assert torch.equal(emb(ids), (F.layer_norm(F.embedding(ids, emb.weight), (8,)) * 3.0).half())


def test_fused_stable_embedding_around_a_parametrized_norm(monkeypatch):
    """The operator takes the parametrized weight; a module whose forward was replaced is
    called."""
    emb = nn.StableEmbedding(10, 8, fused=True)
    seen = []
    monkeypatch.setattr(nn, "stable_embedding", lambda *a: seen.append(a[2].detach()))
    monkeypatch.setattr(nn, "embedding",
                        lambda i, w, padding_idx: F.embedding(i, w, padding_idx))

    class Double(torch.nn.Module):
        def forward(self, w):
            return w * 2.0
    torch.nn.utils.parametrize.register_parametrization(emb.norm, "weight", Double())
    emb(torch.tensor([1]))
    assert torch.equal(seen[0], torch.full((8,), 2.0))
    emb.norm.forward = lambda x: x + 1.0
    ids = torch.tensor([1, 4])
    assert torch.equal(emb(ids), emb.weight[ids] + 1.0) and len(seen) == 1
