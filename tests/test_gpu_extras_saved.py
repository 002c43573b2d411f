"""What the backward passes of attention with a bias, dropout and lengths, of the dense bias and of dropout are handed: saved tensors that a
hook changes, inputs changed in place, gradients that are not plain numbers."""
import numpy as np
import pytest
import torch

from test_gpu_extras import _inputs, _rng, _table, sp  # noqa: F401  (sp: the module's fixture)
from test_gpu_parity import _pattern_from_mask

pytestmark = pytest.mark.gpu
BLOCK, NB, B, H = 32, 2, 2, 2
L = BLOCK * NB


def _calls(sp):
    """Each operator as (function of its leaves, leaves, gradient of its output): the attention, the same through the sub-layer, the dense bias, dropout."""
    pat = _pattern_from_mask(sp, np.ones((NB, NB), dtype=np.uint8), BLOCK)
    q, k, v, do = _inputs(B, H, L, torch.bfloat16, 1)
    table, buckets = _table(32, H, torch.bfloat16, 2), sp.relative_buckets(L + 5, device="cuda")
    kw = dict(lengths=torch.tensor([L, L - 7], dtype=torch.int32, device="cuda"), rng=_rng())
    torch.manual_seed(3)
    mha = sp.SparseMHA(64 * H, H, device="cuda", dtype=torch.bfloat16, buckets=buckets, attn_dropout=0.1)
    E, dE = torch.randn(2, B, L, 64 * H, device="cuda", dtype=torch.bfloat16)
    dbias = torch.randn(H, L, L, device="cuda").to(torch.bfloat16)
    leaf = lambda t: t.detach().clone().requires_grad_(True)
    return {"attention": (lambda *a: sp.sparse_attention(*a[:3], pat, bias=a[3], buckets=buckets, dropout=0.1, **kw), [leaf(t) for t in (q, k, v, table)], do,
                          buckets.map),
            "heads": (lambda x, t: sp.binding._native().heads_attention_with(   # as the sub-layer calls it, on the heads where the projection has them
                x, H, pat.row_ptr, pat.col_idx, pat.col_ptr, pat.row_idx, pat.bsr_pos, pat.nnzb, BLOCK, False, t, buckets.map[5:-5], kw["lengths"], 0.1,
                kw["rng"], 0), [leaf(torch.randn(B, L, 192 * H, device="cuda").to(torch.bfloat16)), leaf(table)], dE, buckets.map),
            "sub-layer": (lambda *a: mha(a[0], pat, **kw), [leaf(E), *mha.parameters()], dE, mha.bucket_map),
            "dense bias": (lambda t: sp.relative_bias(t, buckets, L, L), [leaf(table)], dbias, buckets.map),
            "dropout": (lambda x, r: sp.dropout_add(x, r, 0.1, kw["rng"]), [leaf(q), leaf(k)], do, None)}


OPERATORS = ["attention", "heads", "sub-layer", "dense bias", "dropout"]


# On the host, of another type, a lazy negative, of another shape and, where it has several dimensions, as many elements.
CHANGES = {"host": lambda t: t.cpu(), "type": lambda t: t.to(torch.float64 if t.is_floating_point() else torch.int16),
           "lazy": torch._neg_view, "shape": lambda t: t.transpose(t.dim() // 2 - 1, t.dim() // 2).contiguous() if t.dim() > 1 else t[:-1].clone()}


def _refused_when_changed(f, leaves, g, change, error=ValueError):
    """The backward pass, with one kind of saved tensor after the other changed."""
    kinds = set()
    note = lambda t: kinds.add((t.dtype, t.shape)) or t
    with torch.autograd.graph.saved_tensors_hooks(note, lambda t: t):
        f(*leaves)
    for kind in kinds:
        with torch.autograd.graph.saved_tensors_hooks(lambda t: t, lambda t: change(t) if (t.dtype, t.shape) == kind else t):
            out = f(*leaves)
            with pytest.raises(error):
                torch.autograd.grad(out, leaves, g)
    return kinds


@pytest.mark.parametrize("change", CHANGES)
@pytest.mark.parametrize("name", ["attention", "heads"])
def test_saved_tensors_of_the_attention(sp, name, change):
    f, leaves, g, _ = _calls(sp)[name]
    shapes = {tuple(s) for _, s in _refused_when_changed(f, leaves, g, CHANGES[change])}
    assert {tuple(leaves[0].shape), tuple(g.shape), (32, H), (B,)} < shapes   # Q, K and V; O; the table; the lengths; and what the forward left


@pytest.mark.parametrize("change", CHANGES)
def test_saved_tensors_of_dropout(sp, change):
    f, leaves, g, _ = _calls(sp)["dropout"]
    assert _refused_when_changed(f, leaves, g, CHANGES[change]) == {(torch.int64, (2,))}   # seed and offset


@pytest.mark.parametrize("name", OPERATORS)
def test_gradients_with_a_tangent_are_refused(sp, name):
    f, leaves, g, _ = _calls(sp)[name]
    out = f(*leaves)
    with torch.autograd.forward_ad.dual_level(), pytest.raises(NotImplementedError):
        torch.autograd.grad(out, leaves, torch.autograd.forward_ad.make_dual(g, torch.ones_like(g)))


@pytest.mark.parametrize("name", ["attention", "heads", "dense bias", "dropout"])   # (the sub-layer's projection writes them out)
def test_gradients_that_are_lazy_negatives(sp, name):
    f, leaves, g, _ = _calls(sp)[name]
    out = f(*leaves)
    want = torch.autograd.grad(out, leaves, -g, retain_graph=True)
    got = torch.autograd.grad(out, leaves, torch._neg_view(g))
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("name", OPERATORS)
def test_gradients_in_a_batch_are_refused(sp, name):
    f, leaves, g, _ = _calls(sp)[name]
    with pytest.raises(NotImplementedError):
        torch.autograd.grad(f(*leaves), leaves, torch.stack([g, g]), is_grads_batched=True)


@pytest.mark.parametrize("name", ["attention", "heads", "dense bias"])
def test_a_map_changed_in_place_is_seen(sp, name):
    f, leaves, g, bucket_map = _calls(sp)[name]
    out = f(*leaves)
    torch.autograd.grad(out, leaves, g, retain_graph=True)
    bucket_map[0] = 1   # of a distance that these sequences do not have: the counter is the whole map's
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        torch.autograd.grad(out, leaves, g)
    torch.autograd.grad(f(*leaves), leaves, g)


def test_a_map_made_in_inference_mode(sp):
    pat = _pattern_from_mask(sp, np.ones((NB, NB), dtype=np.uint8), BLOCK)
    q, k, v, do = _inputs(B, H, L, torch.bfloat16, 1)
    table = _table(32, H, torch.bfloat16, 2).requires_grad_(True)
    with torch.inference_mode():
        made_there = sp.relative_buckets(L, device="cuda")
    maps = made_there, sp.relative_buckets(L, device="cuda")
    a, b = [torch.autograd.grad(sp.sparse_attention(q, k, v, pat, bias=table, buckets=m), table, do)[0] for m in maps]
    assert torch.equal(a, b)
    dbias = torch.randn(H, L, L, device="cuda").to(torch.bfloat16)
    a, b = [torch.autograd.grad(sp.relative_bias(table, m, L, L), table, dbias)[0] for m in maps]
    assert torch.equal(a, b)


def test_a_sub_layers_map_written_between_two_passes(sp):
    """As DistributedDataParallel does with a module's buffers, before a backward pass through both."""
    f, leaves, g, bucket_map = _calls(sp)["sub-layer"]
    want = torch.autograd.grad(f(*leaves), leaves, g)
    first = f(*leaves)
    bucket_map.copy_(bucket_map.clone())
    second = f(*leaves)
    got = torch.autograd.grad([first, second], leaves, [g, torch.zeros_like(g)])
    assert all(torch.equal(a, b) for a, b in zip(got, want))
