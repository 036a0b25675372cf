"""The 64-bit statement of the layers: its generator against the published known answers, its gradients against differences."""
import itertools

import numpy as np
import pytest

from oracle import layers as ol


def test_philox_known_answers():
    # the vectors that Salmon et al. publish with the generator (philox4x32, 10 rounds)
    for counter, key, want in (
            ((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
            ((0xFFFFFFFF,) * 4, (0xFFFFFFFF,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
            ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0), (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1))):
        assert tuple(int(w) for w in ol.philox4x32([np.array(c) for c in counter], key)) == want


def test_mask_probability_rows_and_pieces():
    m = ol.mask((0.25, 7, 1, 2, 3, 0), 400, 1003)
    kept, n = (m != 0).sum(), m.size
    assert abs(kept - 0.75 * n) < 5 * np.sqrt(n * 0.75 * 0.25)          # five standard deviations
    assert set(np.unique(m)) == {0.0, 4.0 / 3.0}
    assert np.array_equal(m[100:], ol.mask((0.25, 7, 1, 2, 3, 100), 300, 1003))         # a batch in two pieces
    assert np.array_equal(m[:, :500], ol.mask((0.25, 7, 1, 2, 3, 0), 400, 500))         # a column's draw is its own
    for other in ((0.25, 8, 1, 2, 3, 0), (0.25, 7, 0, 2, 3, 0), (0.25, 7, 1, 1, 3, 0), (0.25, 7, 1, 2, 4, 0), (0.25, 7, 1, 2, 3, 1 << 32)):
        assert 0.5 < ((m != 0) == (ol.mask(other, 400, 1003) != 0)).mean() < 0.75       # 0.625 expected of independent masks
    assert (ol.mask((1.0, 7, 1, 2, 3, 0), 4, 40) == 0).all() and (ol.mask((0.0, 7, 1, 2, 3, 0), 4, 40) == 1).all()


@pytest.mark.parametrize("norm,next_norm,gate,dropped", [c for c in itertools.product((None, "rms", "centred"), (None, "rms", "centred"),
                                                                                     (None, "vector", "element"), (False, True))])
def test_residual_gradients_against_differences(norm, next_norm, gate, dropped):
    r = np.random.default_rng(5)
    begin, d = np.array([0, 2, 2, 5]), 7
    x, b, z = (r.standard_normal((5, d)) for _ in range(3))
    post, pre, vec = (1 + 0.3 * r.standard_normal((3, d)) for _ in range(3))
    dy, dh = r.standard_normal((5, d)), r.standard_normal((5, d)) if next_norm else None
    how = dict(norm=norm, scale=0.7, drop=(0.4, 3, 0, 0, 0, 0) if dropped else None, next_norm=next_norm, eps=1e-3)

    def value(x, b, post, pre, vec, z):
        y, h = ol.residual(x, b, begin, post=post, gate=vec if gate == "vector" else None, logits=z if gate == "element" else None,
                           pre=pre if next_norm else None, **how)
        return (y * dy).sum() + (0.0 if h is None else (h * dh).sum())
    args = dict(x=x, b=b, post=post, pre=pre, vec=vec, z=z)
    y, _ = ol.residual(x, b, begin, post=post, gate=vec if gate == "vector" else None, logits=z if gate == "element" else None,
                       pre=pre if next_norm else None, **how)
    got = ol.residual_grad(dy, dh, y, b, begin, post=post, gate=vec if gate == "vector" else None, logits=z if gate == "element" else None,
                           pre=pre if next_norm else None, **how)
    names = dict(x="dx", b="db", post="dpost", pre="dpre", vec="dgate", z="dlogits")
    checked = 0
    for name, key in names.items():
        if key not in got:
            continue
        want = np.zeros_like(args[name])
        for i in np.ndindex(want.shape):
            for s in (1e-5, -1e-5):
                a = {k: v.copy() for k, v in args.items()}
                a[name][i] += s
                want[i] += value(**a) / (2 * s)
        # central differences: third derivatives of order 10 times 1e-10, and 1e-15 of a value of order 10 over 1e-5
        assert np.abs(got[key] - want).max() < 1e-7 * (1 + np.abs(want).max()), key
        checked += 1
    assert checked == 3 + (next_norm is not None) + (gate is not None)


def test_product_gradients_against_differences():
    r = np.random.default_rng(6)
    begin = np.array([0, 3, 3, 4])
    x, w, dy = r.standard_normal((4, 5)), r.standard_normal((3, 6, 5)), r.standard_normal((4, 6))

    def value(x, w):
        return (ol.product(x, w, begin) * dy).sum()
    dx, dw = ol.product(dy, w, begin, transposed=True), ol.product_grad(dy, x, begin)
    for i in np.ndindex(x.shape):
        e = np.zeros_like(x)
        e[i] = 1e-5
        assert abs((value(x + e, w) - value(x - e, w)) / 2e-5 - dx[i]) < 1e-8
    for i in np.ndindex(w.shape):
        e = np.zeros_like(w)
        e[i] = 1e-5
        assert abs((value(x, w + e) - value(x, w - e)) / 2e-5 - dw[i]) < 1e-8
    assert (dw[1] == 0).all()
