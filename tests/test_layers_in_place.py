"""hop_residual whose y is x or b: the same bits as with a y of its own; another distance between rows is refused."""
import pytest
import torch

from paper_1902_01064_amd import hop, layers
from test_layers_refusals import A, BAD, residual

DEV = "cuda:0"


# y at the address of x, or of b, with rows 8 apart there and 9 (or the other way round) here; x, b, y of their own otherwise
@pytest.mark.parametrize("x,ldx,b,ldb,ldy", [(A, 8, A + 4096, 8, 9), (A, 9, A + 4096, 8, 8), (A + 4096, 8, A, 8, 9), (A + 4096, 9, A, 9, 8), (A, 8, A, 9, 8),
                                             (A, 9, A, 8, 8)])
def test_another_distance_is_refused(x, ldx, b, ldb, ldy):
    assert layers.load().hop_residual(residual(b=b, ldb=ldb), x, ldx, A, ldy, A + 8192, 8, 0) == BAD


# one workgroup width after the other, rows of whole pieces of eight columns and others, pieces of several rows, over 8192 columns
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", [(1, 5), (7, 8), (4000, 64), (3000, 77), (900, 1000), (700, 1003), (300, 2504), (300, 5001), (5, 8192), (40, 8195),
                                       (600, 9000), (20, 16384), (9, 16390), (7, 20003)])
@pytest.mark.parametrize("norm,gate,p", [("rms", None, 0.0), (None, "vector", 0.3), ("centred", "element", 0.3), (None, None, 0.0)])
def test_in_place(dtype, rows, cols, norm, gate, p):
    g = torch.Generator(device=DEV).manual_seed(rows + cols)
    wide = [torch.randn(rows, cols + 8, generator=g, device=DEV).to(dtype) for _ in range(3)]
    x, b, z = (t[:, :cols] for t in wide)
    table = torch.tensor([0, rows // 3, rows], dtype=torch.int32, device=DEV)
    vec = torch.rand(2, cols, generator=g, device=DEV) + 0.5
    how = dict(row_begin=table, norm=norm, post=vec, gate=vec if gate == "vector" else None, gate_logits=z if gate == "element" else None, scale=0.7,
               drop=layers.Drop(p, 3) if p else None, next_norm="rms", pre=vec)
    y, h = layers.residual(x, b, **how)
    for at in (0, 1):
        mine = [wide[0].clone(), wide[1].clone()]
        xs, bs = (t[:, :cols] for t in mine)
        got, next_h = layers.residual(xs, bs, out=(xs, bs)[at], **how)
        assert torch.equal(got, y) and torch.equal(next_h, h)
        assert torch.equal(mine[at][:, cols:], wide[at][:, cols:]) and torch.equal(mine[1 - at], wide[1 - at])


@pytest.mark.gpu
def test_another_distance_is_refused_from_tensors():
    flat = torch.zeros(400, device=DEV)
    x, y = flat[:40].view(5, 8), flat[:50].view(5, 10)[:, :8]
    for a, b in ((x, torch.zeros(5, 8, device=DEV)), (torch.zeros(5, 8, device=DEV), x)):
        with pytest.raises(hop.HopError) as e:
            layers.residual(a, b, out=y)
        assert e.value.code == hop.HOP_ERR_INVALID_ARG
    one, _ = layers.residual(x[:1], torch.ones(1, 8, device=DEV), norm=None, out=y[:1])          # a single row has no distance
    assert (one == 1).all()
