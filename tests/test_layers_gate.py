"""The logistic gate of hop_residual and its gradient over the whole range of its argument, in 32 bits.

With x = 0, b = 1, scale 1 and no norm the result is the gate itself, and with dy = 1 the gradient of the logits is s (1 - s).
Tolerance, u = 2^-24: the power of two and the reciprocal are right to a unit in the last place (2 u each), the correction of the power's
argument, its product and the sum are rounded (u each): 7 u of s.  s (1 - s) moves by |1 - 2 s| times that, and its difference and three products
are rounded: 4 u.  What is below the smallest normal number may be zero."""
import numpy as np
import pytest
import torch

from paper_1902_01064_amd import layers

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
U, TINY = 2.0 ** -24, 2.0 ** -126


@pytest.mark.parametrize("cols", [1024, 1003, 9000])
def test_gate_of_any_size(cols):
    r = np.random.default_rng(cols)
    z = np.concatenate([r.uniform(-88, 88, 60 * cols), r.uniform(-104, -80, 4 * cols), r.standard_normal(6 * cols), 10.0 ** r.uniform(-30, 2, 2 * cols),
                        -(10.0 ** r.uniform(-30, 38, 2 * cols)), np.zeros(cols)]).astype(np.float32).reshape(-1, cols)
    z64 = z.astype(np.float64)
    small = np.exp(-np.abs(z64))
    s = np.where(z64 < 0, small, 1.0) / (1.0 + small)
    rest = np.where(z64 < 0, 1.0, small) / (1.0 + small)   # 1 - s
    logits = torch.from_numpy(z).to(DEV)
    one, zero = torch.ones_like(logits), torch.zeros_like(logits)
    y, _ = layers.residual(zero, one, norm=None, gate_logits=logits)
    off = np.abs(y.double().cpu().numpy() - s)
    assert (off <= 7 * U * s + TINY).all(), (float((off / (s + TINY)).max() / U), z[off > 7 * U * s + TINY][:3])
    g = layers.residual_grad(one, None, None, one, norm=None, gate_logits=logits)
    assert torch.equal(g.db, y)                            # db = dy s
    off = np.abs(g.dlogits.double().cpu().numpy() - s * rest)
    assert (off <= 7 * U * s * np.abs(1 - 2 * s) + 4 * U * s * rest + 2 * TINY).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_gate_of_no_number(dtype):
    z = torch.tensor([[float("inf"), float("-inf"), float("nan"), 3.3e38, -3.3e38, 0.0, -0.0, 1e-40]], device=DEV).to(dtype)
    one, zero = torch.ones_like(z), torch.zeros_like(z)
    y, _ = layers.residual(zero, one, norm=None, gate_logits=z)
    assert y[0].tolist()[:2] == [1, 0] and torch.isnan(y[0, 2]) and y[0].tolist()[3:] == [1, 0, 0.5, 0.5, 0.5]
    g = layers.residual_grad(one, None, None, one, norm=None, gate_logits=z).dlogits
    assert g[0].tolist()[:2] == [0, 0] and torch.isnan(g[0, 2]) and g[0].tolist()[3:] == [0, 0, 0.25, 0.25, 0.25]
