"""The 64-bit statement of attention and of the rotation: against sums by hand, its gradients against differences."""
import numpy as np
import pytest

from oracle import attention as oa


def difference(f, x, direction, h=1e-6):
    return (f(x + h * direction) - f(x - h * direction)) / (2 * h)


def test_attention_by_hand():
    q, k, v = np.array([[1.0], [2.0]]), np.array([[0.5], [-1.0], [3.0]]), np.array([[1.0], [2.0], [4.0]])
    o, lse = oa.attention(q, k, v, 1, 1, [0, 2], [0, 3], True, 1.0)
    first = np.exp([0.5, -1.0])                  # the first of two queries sees two of three keys
    last = np.exp([1.0, -2.0, 6.0])
    assert np.allclose(o[:, 0], [(first @ v[:2, 0]) / first.sum(), (last @ v[:, 0]) / last.sum()])
    assert np.allclose(lse[0], np.log([first.sum(), last.sum()]))
    o, lse = oa.attention(np.ones((3, 1)), k[:1], v[:1], 1, 1, [0, 3], [0, 1], True, 1.0)
    assert o[:, 0].tolist() == [0.0, 0.0, 1.0] and np.isneginf(lse[0, :2]).all()


@pytest.mark.parametrize("causal", [False, True])
def test_attention_gradients_against_differences(causal):
    r = np.random.default_rng(3)
    qb, kb, hq, hk, D = [0, 3, 3, 7], [0, 2, 4, 10], 4, 2, 5
    q, k, v = r.standard_normal((7, hq * D)), r.standard_normal((10, hk * D)), r.standard_normal((10, hk * D))
    do = r.standard_normal(q.shape)
    how = (hq, hk, qb, kb, causal, 0.6)
    o, lse = oa.attention(q, k, v, *how)
    grads = oa.attention_grad(do, o, lse, q, k, v, *how)
    for i, g in enumerate(grads):
        for _ in range(4):
            args = [q, k, v]
            d = r.standard_normal(args[i].shape)
            want = difference(lambda t: (oa.attention(*(args[:i] + [t] + args[i + 1:]), *how)[0] * do).sum(), args[i], d)
            assert abs((g * d).sum() - want) < 1e-7 * (1 + abs(want))


@pytest.mark.parametrize("norm", [None, "rms", "centred"])
@pytest.mark.parametrize("adjacent", [False, True])
def test_rotation_gradients_against_differences(norm, adjacent):
    r = np.random.default_rng(4)
    hq, hk, D, rotary, begin = 3, 2, 9, 6, [0, 2, 2, 5]
    x, dy = r.standard_normal((5, (hq + hk) * D)), r.standard_normal((5, (hq + hk) * D))
    wq, wk = 1 + 0.3 * r.standard_normal((3, D)), 1 + 0.3 * r.standard_normal((3, D))
    pos = np.array([0, 1, 70000, 3, 4])
    rest = (begin, pos, rotary, adjacent, 100.0, norm, 1e-3)
    grads = oa.rotate_grad(dy, x, hq, hk, wq, wk, *rest)
    for i, g in enumerate(grads):
        args = [x, wq, wk]
        d = r.standard_normal(args[i].shape)

        def f(t):
            a = args[:i] + [t] + args[i + 1:]
            return (oa.rotate(a[0], hq, hk, a[1], a[2], *rest) * dy).sum()
        assert abs((g * d).sum() - difference(f, args[i], d)) < 1e-7


def test_rotation_turns_pairs_and_keeps_lengths():
    x = np.arange(1.0, 9.0)[None]
    y = oa.rotate(x, 1, 0, None, None, [0, 1], [3], 4, False, 10000.0, None, 0.0)
    a = np.array([3.0, 0.03])
    assert np.allclose(y[0, :2], x[0, :2] * np.cos(a) - x[0, 2:4] * np.sin(a)) and np.allclose(y[0, 4:], x[0, 4:])
    z = oa.rotate(x, 1, 0, None, None, [0, 1], [3], 4, True, 10000.0, None, 0.0)
    assert np.allclose(z[0, :4:2] ** 2 + z[0, 1:4:2] ** 2, x[0, :4:2] ** 2 + x[0, 1:4:2] ** 2)
    assert np.allclose(z[0, 1], x[0, 1] * np.cos(3.0) + x[0, 0] * np.sin(3.0))
