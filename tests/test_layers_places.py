"""Where the layers may write: groups' gradients that would share memory are refused (host code only, no kernel is launched), and those
that lie apart in any order are right (on the GPU)."""
import numpy as np
import pytest
import torch

from oracle import layers as ol
from paper_1902_01064_amd import hop, layers
from test_layers_refusals import A, BAD, grad, grads, ints, residual


# 2 groups of 8 x 8: behind each other from 64 floats on, side by side within a row of 16
@pytest.mark.parametrize("over", [dict(dw_stride=0), dict(dw_stride=1), dict(dw_stride=7), dict(dw_stride=8), dict(dw_stride=63), dict(dw_stride=-63),
                                  dict(dw_stride=70, lddw=9), dict(dw_stride=7, lddw=16), dict(dw_stride=9, lddw=16), dict(dw_stride=8, lddw=23, G=3),
                                  dict(n=1, dw_stride=7), dict(n=1, dw_stride=0)])
def test_products_gradients_that_share_memory(over):
    assert layers.load().hop_product_grad(grad(**over), A, 1 << 30, 0) == BAD
    assert layers.load().hop_product_grad_scratch_bytes(grad(**over)) == 0


@pytest.mark.parametrize("rows", [(0, 2), (5, 3)])
def test_products_gradients_that_share_memory_by_index(rows):
    at, keep = ints(*rows)                                 # two of 8 columns side by side in 24, with another between them: not in 23
    assert layers.load().hop_product_grad(grad(index=at, dw_stride=8, lddw=23), A, 1 << 30, 0) == BAD
    assert layers.load().hop_product_grad(grad(index=at, dw_stride=31, n=2, lddw=24), A, 1 << 30, 0) == BAD


@pytest.mark.parametrize("over", [dict(dpost_s=0), dict(dpost_s=7), dict(dpost_s=-7), dict(dpre_s=0), dict(dpre_s=-1), dict(dpost_s=7, dpre_s=7)])
def test_vectors_gradients_that_share_memory(over):
    assert layers.load().hop_residual_grad(residual(), grads(**over), A, 1 << 30, 0) == BAD
    at, keep = ints(4, 1)
    assert layers.load().hop_residual_grad(residual(), grads(index=at, **over), A, 1 << 30, 0) == BAD
    gated = residual(kind=1, gate=A, gate_s=8)
    assert layers.load().hop_residual_grad(gated, grads(dpost=0, dpre=0, dgate=A, dgate_s=7), A, 1 << 30, 0) == BAD


@pytest.mark.parametrize("over", [dict(dpost_s=0), dict(dpre_s=3)])
def test_one_group_has_no_distance(over):
    """The scratch that a call names tells that its arguments were taken."""
    assert layers.load().hop_residual_grad_scratch_bytes(residual(G=1), grads(**over)) > 0
    assert layers.load().hop_residual_grad_scratch_bytes(residual(), grads(**over)) == 0
    assert layers.load().hop_residual_grad_scratch_bytes(residual(), grads(dpost_s=-8, dpre_s=9)) > 0


@pytest.mark.gpu
def test_expanded_gradients_are_refused():
    dev = "cuda:0"
    x, rb = torch.ones(4, 8, device=dev), torch.tensor([0, 1, 4], dtype=torch.int32, device=dev)
    vec = torch.ones(2, 8, device=dev)
    for fn in (lambda: layers.product_grad(x, x, rb, out=torch.empty(1, 8, 8, device=dev).expand(2, 8, 8)),
               lambda: layers.residual_grad(x, None, None, x, rb, post=vec, dpost=torch.empty(1, 8, device=dev).expand(2, 8))):
        with pytest.raises(hop.HopError) as e:
            fn()
        assert e.value.code == hop.HOP_ERR_INVALID_ARG


@pytest.mark.gpu
@pytest.mark.parametrize("way", ["behind", "side by side", "columns of a matrix", "picked", "one row each"])
def test_gradients_that_lie_apart(way):
    dev, G, n, k = "cuda:0", 3, 6, 10
    counts = [5, 0, 4]
    begin = np.array([0, 5, 5, 9], dtype=np.int32)
    rng = np.random.default_rng(1)
    if way == "one row each":
        n = 1
    dy, x = (rng.integers(-8, 9, (sum(counts), c)).astype(np.float32) for c in (n, k))          # products and sums of these are exact
    index = [4, 0, 2] if way == "picked" else None
    M = 5 if index else G
    flat = torch.full((M * n * k + 40,), 7.0, device=dev)
    part = flat[:M * n * k]
    out = {"behind": lambda: part.view(M, n, k), "side by side": lambda: part.view(n, M, k).transpose(0, 1),
           "columns of a matrix": lambda: part.view(n, M * k).unflatten(1, (M, k)).transpose(0, 1), "picked": lambda: part.view(n, M, k).transpose(0, 1),
           "one row each": lambda: part.view(M, 1, k)}[way]()
    got = layers.product_grad(torch.from_numpy(dy).to(dev), torch.from_numpy(x).to(dev), torch.from_numpy(begin).to(dev), out=out, index=index)
    want = ol.product_grad(dy.astype(np.float64), x.astype(np.float64), begin)
    assert np.array_equal(got[index or list(range(G))].double().cpu().numpy(), want)
    got[index or list(range(G))] = 7.0
    assert (flat == 7.0).all()
