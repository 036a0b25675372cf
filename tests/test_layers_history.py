"""The layers beside torch's own differentiation: a tensor whose gradient would be lost is refused, and a tensor written in place is known to be."""
import pytest
import torch

from paper_1902_01064_amd import layers

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
G, T, K, N = 2, 6, 8, 16


def args():
    torch.manual_seed(1)
    return dict(x=torch.randn(T, K, device=DEV), b=torch.randn(T, K, device=DEV), z=torch.randn(T, K, device=DEV), dy=torch.randn(T, N, device=DEV),
                w=torch.randn(G, N, K, device=DEV), post=torch.rand(G, K, device=DEV), pre=torch.rand(G, K, device=DEV), gate=torch.rand(G, K, device=DEV))


def calls(a, rb):
    drop = layers.Drop(0.5, 1)
    how = dict(row_begin=rb, post=a["post"], next_norm="rms", pre=a["pre"])
    return {
        "product": (("x", "w"), lambda **o: layers.product(a["x"], a["w"], rb, **o), dict(out=(T, N))),
        "transposed": (("dy", "w"), lambda **o: layers.product(a["dy"], a["w"], rb, transposed=True, **o), dict(out=(T, K))),
        "product_grad": (("x", "dy"), lambda **o: layers.product_grad(a["dy"], a["x"], rb, **o), dict(out=(G, N, K))),
        "dropout": (("x",), lambda **o: layers.dropout(a["x"], drop, **o), dict(out=(T, K))),
        "norm": (("x", "pre"), lambda **o: layers.norm(a["x"], a["pre"], rb, **o), dict(out=(T, K))),
        "norm_grad": (("b", "x", "pre"), lambda **o: layers.norm_grad(a["b"], a["x"], a["pre"], rb, **o), dict(dx=(T, K), dpre=(G, K))),
        "residual": (("x", "b", "post", "gate", "pre"), lambda **o: layers.residual(a["x"], a["b"], gate=a["gate"], drop=drop, **how, **o),
                     dict(out=(T, K), out_next=(T, K))),
        "logits": (("x", "b", "z"), lambda **o: layers.residual(a["x"], a["b"], gate_logits=a["z"], **how, **o), dict(out=(T, K), out_next=(T, K))),
        "residual_grad": (("x", "z", "b", "post", "gate", "pre"), lambda **o: layers.residual_grad(a["x"], a["z"], a["x"], a["b"], gate=a["gate"], **how, **o),
                          dict(dx=(T, K), db=(T, K), dpost=(G, K), dpre=(G, K), dgate=(G, K))),
        "logits' gradient": (("x", "z", "b"), lambda **o: layers.residual_grad(a["x"], None, a["x"], a["b"], gate_logits=a["z"], **how, **o),
                             dict(dx=(T, K), db=(T, K), dlogits=(T, K), dpost=(G, K))),
    }


def test_a_gradient_that_would_be_lost_is_refused():
    rb = torch.tensor([0, 2, T], dtype=torch.int32, device=DEV)
    names = list(calls(args(), rb))
    for name in names:
        inputs, _, outs = calls(args(), rb)[name]
        for which in inputs:
            a = args()
            a[which].requires_grad_(True)
            call = calls(a, rb)[name][1]
            with pytest.raises(ValueError, match="requires a gradient"):
                call()
            with torch.no_grad():
                call()
            a[which] = a[which].detach()
            calls(a, rb)[name][1]()
        for which in outs:
            given = {k: torch.zeros(s, device=DEV) for k, s in outs.items()}
            call = calls(args(), rb)[name][1]
            given[which].requires_grad_(True)
            with pytest.raises(ValueError, match="requires a gradient"):
                call(**given)
            with torch.no_grad():
                call(**given)


def test_what_a_call_writes_counts_as_changed():
    rb = torch.tensor([0, 2, T], dtype=torch.int32, device=DEV)
    a = args()
    for name, (inputs, call, outs) in calls(a, rb).items():
        given = {k: torch.zeros(s, device=DEV) for k, s in outs.items()}
        before = {k: t._version for k, t in given.items()}
        read = {k: a[k]._version for k in inputs}
        call(**given)
        assert all(given[k]._version > v for k, v in before.items()), name
        assert all(a[k]._version == v for k, v in read.items()), name
    leaf = torch.ones(T, K, device=DEV, requires_grad=True)
    kept = torch.ones(T, K, device=DEV)
    loss = (leaf * kept).sum()                             # keeps `kept` for its gradient
    layers.dropout(kept, layers.Drop(0.5, 1), out=kept)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()
    with torch.inference_mode():
        layers.dropout(a["x"], layers.Drop(0.5, 1), out=torch.zeros(T, K, device=DEV))
