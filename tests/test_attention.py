"""Attention's kernels, and those of the norm and rotation of queries and keys, against their 64-bit statement (oracle/attention.py), on the GPU.

Tolerances, element by element, come from oracle/attention.py with u = 2^-24 and, where rows are bfloat16, weights rounded by half a step of 2^-8;
results in bfloat16 are rounded once more: 2^-8 of the result and of the first error's neighbour.  The gradient may take sum do o from o as it was written, or before
its rounding: the bounds of what follows from it count the difference of the two, as it is.
"""
import numpy as np
import pytest
import torch

from oracle import attention as oa
from paper_1902_01064_amd import attention
from test_layers import DEV, U, begin_of, close, holes, laid_out, rounded, table

pytestmark = pytest.mark.gpu


def scattered(r, rows, cols, dtype, odd, loud=1.0):
    t, t64 = rounded(loud * r.standard_normal((rows, cols)), dtype)
    return (laid_out(t, 3, 1) if odd else laid_out(t, 8, 0)), t64


def check(dtype, nq, nk, hq, hk, D, causal, scale=None, odd=False, loud=1.0, grad=True):
    """One forward and backward pass on packed sequences, everything between and around them left as it was."""
    r = np.random.default_rng(sum(nq) * 7 + sum(nk) + hq * 1000 + D)
    qb, kb = begin_of(nq), begin_of(nk)
    Tq, Tk = sum(nq), sum(nk)
    q, q64 = scattered(r, Tq, hq * D, dtype, odd, loud)
    k, k64 = scattered(r, Tk, hk * D, dtype, odd)
    v, v64 = scattered(r, Tk, hk * D, dtype, odd)
    do, do64 = scattered(r, Tq, hq * D, dtype, odd)
    o, unharmed = holes(Tq, hq * D, dtype, 3 if odd else 8, 1 if odd else 0)
    how = dict(q_heads=hq, k_heads=hk, q_begin=table(qb), k_begin=table(kb), causal=causal, scale=scale)
    _, lse = attention.attention(q, k, v, out=o, **how)
    scale = D ** -0.5 if scale is None else scale
    rest = (hq, hk, qb, kb, causal, scale)
    want, want_lse = oa.attention(q64, k64, v64, *rest)
    rounding = 2.0 ** -8 if dtype == "bf16" else 0.0
    o64, lse64 = o.double().cpu().numpy(), lse.double().cpu().numpy()
    bounds = oa.attention_bounds(do64, want, want_lse, q64, k64, v64, *rest, U, rounding)
    close(o, want, bounds[0], dtype, "o")
    empty = np.isneginf(want_lse)
    assert np.array_equal(np.isneginf(lse64), empty)
    close(torch.from_numpy(np.where(empty, 0, lse64)), np.where(empty, 0, want_lse), np.where(empty, 0, bounds[1]), "f32", "lse")
    assert unharmed()
    if not grad:
        return
    # the gradient from o and lse as they were written
    outs = [holes(rows, heads * D, dtype, 3 if odd else 8, 1 if odd else 0) for rows, heads in ((Tq, hq), (Tk, hk), (Tk, hk))]
    for t, _ in outs:
        t.fill_(float("nan"))
    attention.attention_grad(do, o, lse, q, k, v, dq=outs[0][0], dk=outs[1][0], dv=outs[2][0], **how)
    wants = oa.attention_grad(do64, o64, lse64, q64, k64, v64, *rest)
    bounds = oa.attention_bounds(do64, o64, lse64, q64, k64, v64, *rest, U, rounding, want)[2:]
    for (t, fine), w, b, name in zip(outs, wants, bounds, ("dq", "dk", "dv")):
        close(t, w, b, dtype, name)
        assert fine(), name


LENGTHS = {"one": ([1], [1]), "odd": ([77], [77]), "tile": ([128], [128]), "several": ([64, 0, 1, 200, 33], [64, 0, 1, 200, 33]), "ones": ([1] * 9, [1] * 9),
           "more keys": ([5, 1, 40], [70, 300, 129]), "fewer keys": ([40, 150, 3, 7], [7, 90, 0, 8]), "tokens": ([1] * 5, [513, 1, 0, 64, 65]),
           "none": ([0], [40]), "nothing to see": ([3], [0]), "long": ([300], [700])}


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lengths", list(LENGTHS))
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("heads", [(1, 1, 64), (4, 2, 128), (6, 2, 72), (3, 1, 33), (5, 5, 16)])
def test_attention_and_its_gradients(dtype, lengths, causal, heads):
    nq, nk = LENGTHS[lengths]
    hq, hk, D = heads
    check(dtype, nq, nk, hq, hk, D, causal, odd=D % 8 != 0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [1, 7, 8, 20, 40, 65, 96, 100, 127])
def test_columns_of_a_head(dtype, D):
    check(dtype, [70, 3], [70, 3], 2, 1, D, True)
    check(dtype, [9], [130], 2, 1, D, False, odd=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("group", [1, 2, 3, 7, 8, 32, 33])
def test_heads_of_a_group(dtype, group):
    check(dtype, [50, 2], [50, 2], 2 * group, 2, 64, True)
    check(dtype, [1, 1, 1], [300, 20, 65], 2 * group, 2, 64, True, odd=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_loud_scores_move_the_maximum(dtype):
    check(dtype, [150], [150], 2, 1, 64, True, loud=20.0)
    check(dtype, [40], [400], 2, 2, 128, False, scale=2.0)
    check(dtype, [40], [400], 2, 2, 128, True, scale=1e-6)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("nq,nk,hq,hk,D", [([2], [2600], 2, 1, 128), ([1, 1], [3000, 700], 8, 2, 64), ([600], [1200], 2, 2, 64), ([1300], [70], 4, 1, 64), ([1, 1, 1], [900, 0, 1500], 1, 1, 72)])
def test_long_contractions_cut_in_parts(dtype, nq, nk, hq, hk, D):
    check(dtype, nq, nk, hq, hk, D, False)
    check(dtype, nq, nk, hq, hk, D, True)


ROTATIONS = [(128, 128, False), (64, 64, False), (16, 16, False), (8, 8, False), (128, 64, False), (90, 46, False), (90, 46, True), (128, 128, True), (7, 6, True), (1, 0, False), (33, 2, False), (72, 72, False),
             (2, 2, False), (120, 0, True)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D,rotary,adjacent", ROTATIONS)
@pytest.mark.parametrize("norm", ["rms", "centred", None])
@pytest.mark.parametrize("heads,counts", [((1, 1), [1]), ((5, 2), [3, 0, 40, 1]), ((0, 3), [70]), ((4, 0), [0, 9]), ((33, 3), [2, 2])])
def test_rotation_and_its_gradients(dtype, D, rotary, adjacent, norm, heads, counts):
    hq, hk = heads
    T, G = sum(counts), len(counts)
    r = np.random.default_rng(D * 100 + rotary + T + hq)
    odd = (D + hq) % 2 == 1
    begin = begin_of(counts)
    x, x64 = scattered(r, T, (hq + hk) * D, dtype, odd)
    dy, dy64 = scattered(r, T, (hq + hk) * D, dtype, not odd)
    wq, wq64 = rounded(1 + 0.3 * r.standard_normal((G, D)), "f32")
    wk, wk64 = rounded(1 + 0.3 * r.standard_normal((G, D)), "f32")
    pos = r.integers(0, 2000000, T).astype(np.int32)
    how = dict(q_heads=hq, k_heads=hk, q_weight=wq, k_weight=wk, row_begin=table(begin), positions=torch.from_numpy(pos).to(DEV), rotary=rotary, adjacent=adjacent,
               base=500.0, norm=norm, eps=1e-3)
    rest = (hq, hk, wq64, wk64, begin, pos, rotary, adjacent, 500.0, norm, float(np.float32(1e-3)))
    y, unharmed = holes(T, (hq + hk) * D, dtype, 3 if odd else 8, 1 if odd else 0)
    attention.rotate(x, out=y, **how)
    bounds = oa.rotate_bounds(dy64, x64, *rest, U)
    close(y, oa.rotate(x64, *rest), bounds[0], dtype, "y")
    assert unharmed()
    dx, unharmed = holes(T, (hq + hk) * D, dtype, 3 if odd else 8, 1 if odd else 0)
    _, dwq, dwk = attention.rotate_grad(dy, x, dx=dx, **how)
    wants = oa.rotate_grad(dy64, x64, *rest)
    close(dx, wants[0], bounds[1], dtype, "dx")
    close(dwq, wants[1], bounds[2], "f32", "dq_weight")
    close(dwk, wants[2], bounds[3], "f32", "dk_weight")
    assert unharmed()
