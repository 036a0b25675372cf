"""The layers' kernels against their 64-bit statement (oracle/layers.py), on the GPU.

Tolerances, element by element, u = 2^-24:
  products    a sum of K products in fp32, in any order: (K + 3) u times the sum of the products' magnitudes; results in bfloat16
              are rounded once more: 2^-9 of the result, and of the first error's neighbour (2^-8 in all)
  norms       every statistic is a tree of at most 32 additions a level deep, every element at most 16 operations behind it: 64 u
              times the magnitudes that meet in it (a centred element: of the row's mean magnitude too)
  sums over a group's rows: (rows + 128) u times the magnitudes of the terms
"""
import itertools

import numpy as np
import pytest
import torch

from oracle import layers as ol
from paper_1902_01064_amd import hop, layers

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
U = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def begin_of(counts):
    return np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)


def table(begin):
    return torch.from_numpy(begin).to(DEV)


def rounded(a, dtype):
    """Values of a type as (torch on the GPU, numpy in 64 bits)."""
    t = torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(DT[dtype]).to(DEV)
    return t, t.double().cpu().numpy()


def laid_out(t, pad, offset):
    """The same matrix with rows `pad` elements further apart, starting `offset` elements into its memory; NaN all around."""
    rows, cols = t.shape
    flat = torch.full((offset + rows * (cols + pad) + 64,), float("nan"), dtype=t.dtype, device=t.device)
    v = flat[offset:offset + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    v.copy_(t)
    return v


def holes(rows, cols, dtype, pad, offset):
    """An output with marks around it, and a check that nothing but it was written."""
    flat = torch.full((offset + rows * (cols + pad) + 64,), 7.0, dtype=DT[dtype], device=DEV)
    v = flat[offset:offset + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]

    def unharmed():
        keep = v.clone()
        v.fill_(7.0)
        ok = bool((flat == 7.0).all())
        v.copy_(keep)
        return ok
    return v, unharmed


def close(got, want, tol, dtype, what):
    got = got.double().cpu().numpy()
    tol = tol + (2.0 ** -8 * (np.abs(want) + tol) if dtype == "bf16" else 0.0) + 1e-37
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (what, int(bad.sum()), np.argwhere(bad)[:3].tolist(), got[bad][:3], want[bad][:3], np.broadcast_to(tol, want.shape)[bad][:3])


# ------------------------------------------------------------------------------------------- products ----
COUNTS = {"one": [1], "single": [200], "none at all": [0], "holes": [0, 3, 0, 0, 65, 1, 0], "even": [64, 64, 64], "ones": [1] * 9, "skew": [300, 1, 0, 17, 2],
          "many": [(g * 7) % 5 for g in range(150)], "long": [700, 513]}
SIZES = [(1, 1), (7, 5), (64, 64), (33, 130), (256, 192), (200, 72), (520, 264), (777, 129)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("counts", list(COUNTS))
@pytest.mark.parametrize("size", SIZES)
def test_product_and_its_gradients(dtype, counts, size):
    n = COUNTS[counts]
    K, N = size
    r = np.random.default_rng(K * 1000 + N + len(n))
    T, G, begin = sum(n), len(n), begin_of(n)
    odd = (K + N) % 2 == 1                       # unaligned addresses and distances
    x, x64 = rounded(r.standard_normal((T, K)), dtype)
    dy, dy64 = rounded(r.standard_normal((T, N)), dtype)
    w, w64 = rounded(r.standard_normal((G, N, K)), dtype)
    if odd:
        x, dy = laid_out(x, 3, 1), laid_out(dy, 5, 3)
    y, unharmed = holes(T, N, dtype, 3 if odd else 8, 1 if odd else 0)
    layers.product(x, w, table(begin), out=y)
    close(y, ol.product(x64, w64, begin), (K + 3) * U * ol.product(np.abs(x64), np.abs(w64), begin), dtype, "y")
    assert unharmed()
    dx = layers.product(dy, w, table(begin), transposed=True)
    close(dx, ol.product(dy64, w64, begin, True), (N + 3) * U * ol.product(np.abs(dy64), np.abs(w64), begin, True), dtype, "dx")
    dw, unharmed = holes(G * N, K, "f32", 1 if odd else 4, 3 if odd else 0)
    dw3 = dw.unflatten(0, (G, N))
    dw3.fill_(float("nan"))
    layers.product_grad(dy, x, table(begin), out=dw3)
    longest = max(n)
    close(dw3, ol.product_grad(dy64, x64, begin), (longest + 3) * U * ol.product_grad(np.abs(dy64), np.abs(x64), begin), "f32", "dw")
    assert unharmed()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,K,N", [(1, 4100, 1040), (3, 8192, 515), (5000, 64, 48), (3001, 130, 70), (640, 1024, 1024), (9, 72, 6000), (1100, 512, 768)])
def test_one_group_long_in_one_direction(dtype, T, K, N):
    r = np.random.default_rng(T + K + N)
    x, x64 = rounded(r.standard_normal((T, K)), dtype)
    dy, dy64 = rounded(r.standard_normal((T, N)), dtype)
    w, w64 = rounded(r.standard_normal((1, N, K)), dtype)
    begin = np.array([0, T], dtype=np.int32)
    close(layers.product(x, w), ol.product(x64, w64, begin), (K + 3) * U * ol.product(np.abs(x64), np.abs(w64), begin), dtype, "y")
    close(layers.product(dy, w, transposed=True), ol.product(dy64, w64, begin, True), (N + 3) * U * ol.product(np.abs(dy64), np.abs(w64), begin, True),
          dtype, "dx")
    close(layers.product_grad(dy, x), ol.product_grad(dy64, x64, begin), (T + 3) * U * ol.product_grad(np.abs(dy64), np.abs(x64), begin), "f32", "dw")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("K,N,per", [(64, 96, 3), (256, 256, 40), (129, 77, 40), (512, 512, 200)])
def test_a_groups_bad_rows_stay_with_it(dtype, K, N, per):
    """Infinities and NaN in one group's rows and weights do not reach another's results."""
    r = np.random.default_rng(K)
    G, begin = 3, begin_of([per, per + 1, per])
    T = int(begin[-1])
    x, x64 = rounded(r.standard_normal((T, K)), dtype)
    dy, _ = rounded(r.standard_normal((T, N)), dtype)
    w, w64 = rounded(r.standard_normal((G, N, K)), dtype)
    want = [layers.product(x, w, table(begin)), layers.product(dy, w, table(begin), transposed=True), layers.product_grad(dy, x, table(begin))]
    mid = slice(int(begin[1]), int(begin[2]))
    x[mid], dy[mid], w[1] = float("nan"), float("inf"), float("-inf")
    got = [layers.product(x, w, table(begin)), layers.product(dy, w, table(begin), transposed=True), layers.product_grad(dy, x, table(begin))]
    for a, b in zip(want[:2], got[:2]):
        assert torch.equal(a[:mid.start], b[:mid.start]) and torch.equal(a[mid.stop:], b[mid.stop:])
        assert not torch.isfinite(b[mid]).any()
    assert torch.equal(want[2][0], got[2][0]) and torch.equal(want[2][2], got[2][2]) and not torch.isfinite(got[2][1]).any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_infinities_large_and_tiny_values(dtype):
    """An infinity, the largest values and very small ones come out as the formula has them."""
    K, N, T = 96, 64, 40
    r = np.random.default_rng(3)
    x, _ = rounded(r.standard_normal((T, K)), dtype)
    w, _ = rounded(r.standard_normal((1, N, K)), dtype)
    w[0, 5] = 0.0
    w[0, 5, 7] = 1.0
    x[0, 7], x[1, 7], x[2, 7], x[3, 7] = float("inf"), float("-inf"), 3.0e38, 1e-30
    x[4, 7] = float("nan")
    y = layers.product(x, w).float().cpu().numpy()
    assert np.isnan(y[4]).all()
    for row, v in ((0, np.inf), (1, -np.inf)):
        assert y[row, 5] == v and not np.isfinite(y[row]).any()
    for row in (2, 3):
        assert abs(y[row, 5] / float(x[row, 7]) - 1) < 2.0 ** -8 and np.isfinite(y[row, 5])
    assert np.isfinite(y[5:]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_parameters_in_a_lattice_of_replicas(dtype):
    """Weights and gradients as views of [workers x slots, stride] arenas, rows chosen by index; other rows are not touched."""
    K, N, G, rows = 72, 40, 3, 10
    r = np.random.default_rng(1)
    begin, index = begin_of([5, 20, 9]), [7, 2, 4]
    T, stride = int(begin[-1]), 3 + N * K + 64
    arena = torch.from_numpy(r.standard_normal((rows, stride)).astype(np.float32)).to(DT[dtype]).to(DEV)
    w = arena[:, 3:3 + N * K].unflatten(1, (N, K))
    w64 = w[index].double().cpu().numpy()
    x, x64 = rounded(r.standard_normal((T, K)), dtype)
    dy, dy64 = rounded(r.standard_normal((T, N)), dtype)
    close(layers.product(x, w, table(begin), index=index), ol.product(x64, w64, begin), (K + 3) * U * ol.product(np.abs(x64), np.abs(w64), begin),
          dtype, "y")
    close(layers.product(dy, w, table(begin), index=index, transposed=True), ol.product(dy64, w64, begin, True),
          (N + 3) * U * ol.product(np.abs(dy64), np.abs(w64), begin, True), dtype, "dx")
    flat = torch.full((rows, stride), 7.0, device=DEV)
    dw = flat[:, 5:5 + N * K].unflatten(1, (N, K))
    layers.product_grad(dy, x, table(begin), out=dw, index=index)
    close(dw[index], ol.product_grad(dy64, x64, begin), 23 * U * ol.product_grad(np.abs(dy64), np.abs(x64), begin), "f32", "dw")
    dw[index] = 7.0
    assert (flat == 7.0).all()


# -------------------------------------------------------------------------------------------- dropout ----
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols,pad,offset,p", [(1, 1, 0, 0, 0.5), (3, 7, 0, 0, 0.1), (64, 1023, 1, 1, 0.5), (5, 4096, 8, 0, 0.9), (130, 72, 3, 3, 0.25),
                                                    (2, 70000, 0, 0, 0.3), (4, 64, 0, 0, 0.0), (4, 64, 0, 0, 1.0), (70001, 9, 0, 0, 0.5)])
def test_dropout(dtype, rows, cols, pad, offset, p):
    r = np.random.default_rng(rows)
    x, x64 = rounded(r.standard_normal((rows, cols)), dtype)
    drop = layers.Drop(p, 11, 2, 30, 4, (1 << 40) + 5)
    y, unharmed = holes(rows, cols, dtype, pad, offset)
    layers.dropout(laid_out(x, pad, offset), drop, out=y)
    m = ol.mask(drop, rows, cols)
    close(y, x64 * m, 2 * U * np.abs(x64 * m), dtype, "y")          # the factor and the product, rounded
    assert (y.cpu().numpy() if dtype == "f32" else y.float().cpu().numpy())[m == 0].any() == False  # noqa: E712
    assert unharmed()


def test_dropout_drops_what_is_no_number_and_works_in_place():
    drop = layers.Drop(0.5, 1)
    m = ol.mask(drop, 8, 100)
    for v in (float("nan"), float("inf")):
        x = torch.full((8, 100), v, device=DEV)
        y = layers.dropout(x, drop, out=x).cpu().numpy()
        assert (y[m == 0] == 0).all() and not np.isfinite(y[m != 0]).any()
    negative = layers.Drop(0.5, -1, -1, -2, -3)                        # numbers below zero are as good as others
    y = layers.dropout(torch.ones(8, 100, device=DEV), negative).cpu().numpy()
    assert np.array_equal(y, ol.mask(negative, 8, 100).astype(np.float32))


# ------------------------------------------------------------------------------- norms around a block ----
def magnitude_of_norm(v64, how, eps):
    """What an error of 1 unit in the row's values amounts to behind the norm: |n|, and for a centred row the mean's share."""
    n, r = ol.normed(v64, how, eps)
    return n, r, np.abs(n) + (r * np.abs(v64).mean(1, keepdims=True) if how == "centred" else 0.0)


def through_magnitude(a, n, nm, r, how):
    m = np.abs(a).mean(1, keepdims=True)
    return r * (np.abs(a) + m + nm * np.abs(a * n).mean(1, keepdims=True) + np.abs(n) * (np.abs(a) * nm).mean(1, keepdims=True))


def residual_case(dtype, counts, cols, norm, next_norm, gate, post, pre, p, seed, pad=0, offset=0):
    r = np.random.default_rng(seed)
    begin = begin_of(counts)
    T, G = int(begin[-1]), len(counts)

    def rows(v):
        t, v64 = rounded(v, dtype)
        return (laid_out(t, pad, offset) if pad or offset else t), v64

    def vector(mean, dev):
        return rounded(mean + dev * r.standard_normal((G, cols)), "f32")
    x, b, z, dy, dh, y = (rows(a + s * r.standard_normal((T, cols))) for a, s in ((0, 1), (0.3, 0.7), (0, 1), (0, 1), (0, 1), (0.2, 1.5)))
    none = (None, None)
    post, pre = vector(1, 0.2) if post else none, vector(1, 0.2) if pre and next_norm else none
    gamma = vector(0.5, 0.2) if gate == "vector" else none
    if gate != "element":
        z = none
    drop = layers.Drop(p, 5, 1, 2, 3, 17) if p else None
    return begin, x, b, z, dy, dh, y, post, pre, gamma, drop


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("norm,next_norm,gate,p", [(None, None, None, 0.0), ("rms", None, None, 0.3), ("rms", "rms", "vector", 0.0), ("rms", "rms", "element", 0.1),
                                                   ("centred", "centred", None, 0.5), ("centred", "rms", "vector", 0.2), (None, "centred", "element", 0.0)])
@pytest.mark.parametrize("cols,counts", [(1, [3]), (7, [2, 0, 5]), (64, [1]), (200, [9, 1, 0, 30]), (513, [4, 4]), (1024, [40]), (1500, [1, 2]), (3001, [5, 3]),
                                         (5000, [2, 0, 1]), (9000, [3]), (20000, [2, 1]), (256, [600, 700])])
def test_residual_and_its_gradients(dtype, norm, next_norm, gate, p, cols, counts):
    pad, offset = (3, 1) if cols % 2 else (8, 0)
    with_vectors = cols % 3 != 0
    begin, x, b, z, dy, dh, y, post, pre, gamma, drop = residual_case(dtype, counts, cols, norm, next_norm, gate, with_vectors, with_vectors, p,
                                                                      cols + len(counts), pad, offset)
    eps = 1e-3
    how = dict(row_begin=table(begin), norm=norm, post=post[0], gate=gamma[0], gate_logits=z[0], scale=0.7, drop=drop, next_norm=next_norm,
               pre=pre[0], eps=eps)
    how64 = dict(norm=norm, post=post[1], gate=gamma[1], logits=z[1], scale=0.7, drop=drop, next_norm=next_norm, pre=pre[1], eps=eps)
    T = int(begin[-1])
    out, unharmed = holes(T, cols, dtype, pad, offset)
    out_next, unharmed_next = holes(T, cols, dtype, pad, offset) if next_norm else (None, None)
    got_y, got_h = layers.residual(x[0], b[0], out=out, out_next=out_next, **how)
    y64, h64 = ol.residual(x[1], b[1], begin, **how64)
    # magnitudes: the branch's elements with their row's mean where centred
    n, rb, nm = magnitude_of_norm(b[1], norm, eps) if norm else (b[1], 1.0, np.abs(b[1]))
    post_rows = ol.spread(post[1], begin) if post[1] is not None else 1.0
    pre_rows = ol.spread(pre[1], begin) if pre[1] is not None else 1.0
    s = ol.spread(gamma[1], begin) if gate == "vector" else 1 / (1 + np.exp(-z[1])) if gate == "element" else 1.0
    m = ol.mask(drop, T, cols) if drop else 1.0
    branch = 0.7 * nm * np.abs(post_rows * s) * m
    ymag = np.abs(x[1]) + branch
    close(got_y, y64, 64 * U * ymag, dtype, "y")
    assert unharmed()
    if next_norm:
        hn, ry, hm = magnitude_of_norm(y64, next_norm, eps)
        tol = 64 * U * (hm + ry * ymag + np.abs(hn) * (np.abs(hn) * ry * ymag).mean(1, keepdims=True) + ry * ymag.mean(1, keepdims=True))
        close(got_h, h64, tol * np.abs(pre_rows), dtype, "h")
        assert unharmed_next()
    else:
        assert got_h is None
    # gradients; y as stored is an input
    back = layers.residual_grad(dy[0], dh[0] if next_norm else None, y[0], b[0], **how)
    want = ol.residual_grad(dy[1], dh[1] if next_norm else None, y[1], b[1], begin, **how64)
    emag = np.abs(dy[1])
    longest = max(counts)
    if next_norm:
        n2, r2, nm2 = magnitude_of_norm(y[1], next_norm, eps)
        emag = emag + through_magnitude(dh[1] * pre_rows, n2, nm2, r2, next_norm)
    close(back.dx, want["dx"], 64 * U * emag, dtype, "dx")
    fmag = 0.7 * emag * m
    qmag = fmag * np.abs(s)

    def sums(v):
        return np.stack([v[r].sum(0) for _, r in ol.groups(begin)])
    if pre[1] is not None:
        close(back.dpre, want["dpre"], (longest + 128) * U * sums(np.abs(dh[1]) * nm2), "f32", "dpre")
    if gate == "vector":
        close(back.dgate, want["dgate"], (longest + 128) * U * sums(fmag * nm * np.abs(post_rows)), "f32", "dgate")
    if gate == "element":
        close(back.dlogits, want["dlogits"], 64 * U * fmag * nm * np.abs(post_rows) * s, dtype, "dlogits")
    if post[1] is not None:
        close(back.dpost, want["dpost"], (longest + 128) * U * sums(qmag * nm), "f32", "dpost")
    amag = qmag * np.abs(post_rows)
    if norm:
        amag = through_magnitude(amag, n, nm, rb, norm)
    close(back.db, want["db"], 64 * U * amag, dtype, "db")
    assert [v is None for v in back] == [False, False, post[1] is None, pre[1] is None, gate != "vector", gate != "element"]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("how", ["rms", "centred"])
def test_norm_by_itself(dtype, how):
    begin, x, _, _, dy, dh, _, _, pre, _, _ = residual_case(dtype, [3, 0, 6], 300, None, how, None, False, True, 0.0, 9)
    h = layers.norm(x[0], pre[0], table(begin), norm=how, eps=1e-3)
    _, want = ol.residual(x[1], None, begin, next_norm=how, pre=pre[1], eps=1e-3)
    n, r, nm = magnitude_of_norm(x[1], how, 1e-3)
    pre_rows = ol.spread(pre[1], begin)
    close(h, want, 64 * U * nm * np.abs(pre_rows), dtype, "h")
    for with_dy in (False, True):
        dx, dpre = layers.norm_grad(dh[0], x[0], pre[0], table(begin), norm=how, eps=1e-3, dy=dy[0] if with_dy else None)
        want = ol.residual_grad(dy[1] if with_dy else None, dh[1], x[1], None, begin, next_norm=how, pre=pre[1], eps=1e-3)
        mag = through_magnitude(dh[1] * pre_rows, n, nm, r, how) + (np.abs(dy[1]) if with_dy else 0)
        close(dx, want["dx"], 64 * U * mag, dtype, "dx")
        close(dpre, want["dpre"], 134 * U * np.stack([(np.abs(dh[1]) * nm)[r].sum(0) for _, r in ol.groups(begin)]), "f32", "dpre")


def test_residual_parameters_and_gradients_in_a_lattice():
    cols, index, grad_index = 130, [4, 1, 6], [2, 0, 1]
    begin, x, b, _, dy, dh, y, post, pre, gamma, drop = residual_case("f32", [5, 2, 40], cols, "rms", "rms", "vector", True, True, 0.2, 3)
    arena = torch.randn(8, 3 * cols + 5, device=DEV)
    grads = torch.full((3, 3 * cols + 5), 7.0, device=DEV)
    part = [slice(1 + i * cols, 1 + (i + 1) * cols) for i in range(3)]
    for s, v in zip(part, (post, pre, gamma)):
        arena[index, s] = v[0]
    how = dict(row_begin=table(begin), norm="rms", scale=0.7, drop=drop, next_norm="rms", eps=1e-3)
    apart = dict(how, post=post[0], pre=pre[0], gate=gamma[0])
    there = dict(how, post=arena[:, part[0]], pre=arena[:, part[1]], gate=arena[:, part[2]], index=index)
    for a, c in zip(layers.residual(x[0], b[0], **apart), layers.residual(x[0], b[0], **there)):
        assert torch.equal(a, c)
    a = layers.residual_grad(dy[0], dh[0], y[0], b[0], **apart)
    c = layers.residual_grad(dy[0], dh[0], y[0], b[0], **there, dpost=grads[:, part[0]], dpre=grads[:, part[1]], dgate=grads[:, part[2]],
                             grad_index=grad_index)
    assert torch.equal(a.dx, c.dx) and torch.equal(a.db, c.db)
    for s, v in zip(part, (a.dpost, a.dpre, a.dgate)):
        assert torch.equal(v, grads[grad_index, s])
        grads[:, s] = 7.0
    assert (grads == 7.0).all()


def test_no_rows_gradients_are_zero():
    none = torch.zeros(3, dtype=torch.int32, device=DEV)
    empty = torch.empty(0, 40, device=DEV)
    vec = torch.ones(2, 40, device=DEV)
    g = layers.residual_grad(empty, empty, empty, empty, row_begin=none, post=vec, gate=vec, next_norm="rms", pre=vec)
    for v in (g.dpost, g.dpre, g.dgate):
        assert v.shape == (2, 40) and (v == 0).all()
    assert layers.dropout(empty, layers.Drop(0.5, 1)).shape == (0, 40)
    assert layers.product(empty, torch.ones(2, 7, 40, device=DEV), none).shape == (0, 7)
    dw = layers.product_grad(torch.empty(0, 7, device=DEV), empty, none)
    assert dw.shape == (2, 7, 40) and (dw == 0).all()
    y, h = layers.residual(empty, empty, row_begin=none, post=vec, next_norm="rms")
    assert y.shape == h.shape == (0, 40)


def test_dropped_places_take_nothing_from_a_gradient_that_is_no_number():
    cols, drop = 96, layers.Drop(0.5, 4)
    m = ol.mask(drop, 6, cols)
    x, b = torch.randn(6, cols, device=DEV), torch.randn(6, cols, device=DEV)
    dy = torch.where(torch.from_numpy(m).to(DEV) == 0, float("nan"), 1.0).float()
    g = layers.residual_grad(dy, None, None, b, norm=None, drop=drop)
    assert np.array_equal(g.db.cpu().numpy(), m.astype(np.float32))
    b[torch.from_numpy(m).to(DEV) == 0] = float("inf")
    y, _ = layers.residual(x, b, norm=None, drop=drop)
    assert torch.isfinite(y).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cols", [8, 256, 1032, 4104, 6000])
def test_any_alignment_gives_the_same_rows(dtype, cols):
    """The same values at addresses and distances that are multiples of 16, 8, 4 and 2 bytes; rows of whole pieces of eight columns go
    another way than others, sums in the same order."""
    begin, x, b, z, dy, dh, y, post, pre, _, drop = residual_case(dtype, [5, 0, 30], cols, "rms", "centred", "element", True, True, 0.25, cols)
    how = dict(row_begin=table(begin), norm="rms", post=post[0], scale=0.7, drop=drop, next_norm="centred", pre=pre[0], eps=1e-3)

    def run(at, pad):
        def moved(t):
            return laid_out(t, pad, at)
        out, _ = holes(35, cols, dtype, pad, at)
        layers.residual(moved(x[0]), moved(b[0]), gate_logits=moved(z[0]), out=out, **how)
        g = layers.residual_grad(moved(dy[0]), moved(dh[0]), moved(y[0]), moved(b[0]), gate_logits=moved(z[0]), **how)
        return [out.clone(), *[t for t in g if t is not None], layers.dropout(moved(x[0]), drop)]
    want = run(0, 0)
    for at, pad in ((8, 8), (4, 4), (2, 2), (1, 0), (0, 1), (3, 5)):
        for a, c in zip(want, run(at, pad)):
            assert torch.allclose(a.float(), c.float(), rtol=2.0 ** -7 if dtype == "bf16" else 1e-5, atol=1e-5), (at, pad)


# --------------------------------------------------------------------- streams, graphs, the same bits ----
def everything(x, b, w, w2, vec, rb, drop):
    h = layers.norm(x, vec, rb)
    u = layers.dropout(layers.product(h, w, rb), drop)
    v = layers.product(u, w2, rb)
    y, h2 = layers.residual(x, v, rb, post=vec, gate=vec, drop=drop, next_norm="centred", pre=vec)
    g = layers.residual_grad(b, h, y, v, rb, post=vec, gate=vec, drop=drop, next_norm="centred", pre=vec)
    du = layers.dropout(layers.product(g.db, w2, rb, transposed=True), drop)
    return [h, u, v, y, h2, *[t for t in g if t is not None], du, layers.product_grad(g.db, u, rb), layers.product_grad(du, h, rb)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("counts,cols,hidden", [([3, 1, 0, 2], 96, 200), ([200, 90, 222], 256, 512)])
def test_streams_graphs_and_repeats_give_the_same_bits(dtype, counts, cols, hidden):
    torch.manual_seed(1)
    begin = begin_of(counts)
    T, G, rb, dt = int(begin[-1]), len(counts), table(begin), DT[dtype]
    args = [torch.randn(T, cols, device=DEV).to(dt), torch.randn(T, cols, device=DEV).to(dt), torch.randn(G, hidden, cols, device=DEV).to(dt),
            torch.randn(G, cols, hidden, device=DEV).to(dt), torch.randn(G, cols, device=DEV), rb, layers.Drop(0.2, 3)]
    want = [t.clone() for t in everything(*args)]
    assert all(torch.isfinite(t).all() for t in want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = everything(*args)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = everything(*args)
    for _ in range(3):
        for t in got:
            t.zero_()
        (torch.randn(1000, device=DEV) * 2).sum().item()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, got))


def test_refusals_of_the_tensor_calls():
    x, w = torch.zeros(4, 8, device=DEV), torch.zeros(2, 6, 8, device=DEV)
    rb = torch.tensor([0, 1, 4], dtype=torch.int32, device=DEV)
    ok = layers.product(x, w, rb)
    assert ok.shape == (4, 6)
    for fn in (lambda: layers.product(x.cpu(), w, rb), lambda: layers.product(x, w.cpu(), rb), lambda: layers.product(x, w, rb.cpu()),
               lambda: layers.product(x, w, rb.long()), lambda: layers.product(x, w), lambda: layers.product(x, w[0], rb),
               lambda: layers.product(x, w, rb, index=[0]), lambda: layers.product(x, w, rb, index=[0, 2]), lambda: layers.product(x, w, rb, index=[0, -1]),
               lambda: layers.product(x.t(), w, rb), lambda: layers.product(x[:, :7], w, rb), lambda: layers.product(x[:1].expand(4, 8), w, rb),
               lambda: layers.product(x, w.transpose(1, 2), rb, transposed=True), lambda: layers.product(x, w, rb, out=torch.zeros(4, 5, device=DEV)),
               lambda: layers.product_grad(x, x[:3], rb), lambda: layers.product_grad(x, x, rb, index=[0, 1]),
               lambda: layers.residual(x, None), lambda: layers.residual(x, x[:2]), lambda: layers.residual(x, x, post=torch.zeros(2, 8, device=DEV)),
               lambda: layers.residual(x, x, norm="other"), lambda: layers.residual_grad(None, None, x, x), lambda: layers.residual_grad(None, x, None, x),
               lambda: layers.residual(x, x, rb, gate=torch.zeros(2, 8, device=DEV), gate_logits=x),
               lambda: layers.residual_grad(x, None, None, x, dpost=torch.zeros(1, 8, device=DEV))):
        with pytest.raises(ValueError):
            fn()
    for fn in (lambda: layers.product(x.half(), w, rb), lambda: layers.product(x.double(), w, rb), lambda: layers.dropout(x.int(), layers.Drop(0.1, 1)),
               lambda: layers.residual(x, x.bfloat16()), lambda: layers.product(x, w, rb, out=torch.zeros(4, 6, device=DEV).bfloat16())):
        with pytest.raises(TypeError):
            fn()
    for fn in (lambda: layers.dropout(x, layers.Drop(1.5, 1)), lambda: layers.residual(x, x, eps=-1.0), lambda: layers.residual(x, x, scale=float("inf")),
               lambda: layers.norm(torch.zeros(2, layers.HOP_MAX_NORM_COLS + 1, device=DEV))):
        with pytest.raises(hop.HopError) as e:
            fn()
        assert e.value.code == hop.HOP_ERR_INVALID_ARG
