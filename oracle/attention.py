"""Attention over packed sequences, and the norm and rotation of its queries and keys, in 64 bits (oracle side).

TEST INFRASTRUCTURE ONLY - see oracle/__init__.py.  Written from the formulas, sequence by sequence and head by head:

    attention  s_ij = scale q_i k_j over the keys j that query i sees, p = softmax_j(s), o_i = sum_j p_ij v_j, lse_i = log sum_j exp s_ij
               causal: i of nq queries sees j <= i + nk - nq of nk keys; who sees nothing has o = 0, lse = -infinity
    rotate     n = norm(x_h), t = n w, (y_c, y_c') = (t_c cos a - t_c' sin a, t_c' cos a + t_c sin a), a = position base^(-2 i / rotary)
Each also says how much meets in a result, for bounds on what rounding may do to it.
"""
import numpy as np


def _heads(x, h, cols):
    return x[:, h * cols:(h + 1) * cols]


def seen(nq, nk, causal):
    i, j = np.arange(nq)[:, None], np.arange(nk)[None, :]
    return j <= i + nk - nq if causal else np.ones((nq, nk), bool)


def each(q_begin, k_begin, q_heads, k_heads):
    """(rows of queries, rows of keys, query head, key head) of every sequence and head."""
    for s in range(len(q_begin) - 1):
        for h in range(q_heads):
            yield slice(int(q_begin[s]), int(q_begin[s + 1])), slice(int(k_begin[s]), int(k_begin[s + 1])), h, h // (q_heads // k_heads)


def attention(q, k, v, q_heads, k_heads, q_begin, k_begin, causal, scale):
    D = q.shape[1] // q_heads
    o, lse = np.zeros_like(q), np.full((q_heads, q.shape[0]), -np.inf)
    for rq, rk, h, hk in each(q_begin, k_begin, q_heads, k_heads):
        see = seen(rq.stop - rq.start, rk.stop - rk.start, causal)
        a, b, c = _heads(q[rq], h, D), _heads(k[rk], hk, D), _heads(v[rk], hk, D)
        for i in np.flatnonzero(see.any(1)):
            s = scale * (b[see[i]] @ a[i])
            m = s.max()
            e = np.exp(s - m)
            lse[h, rq.start + i] = m + np.log(e.sum())
            o[rq.start + i, h * D:(h + 1) * D] = (e / e.sum()) @ c[see[i]]
    return o, lse


def attention_grad(do, o, lse, q, k, v, q_heads, k_heads, q_begin, k_begin, causal, scale):
    """Gradients from o and lse as they are given."""
    D = q.shape[1] // q_heads
    dq, dk, dv = np.zeros_like(q), np.zeros_like(k), np.zeros_like(v)
    for rq, rk, h, hk in each(q_begin, k_begin, q_heads, k_heads):
        p, ds = _weights(do, o, lse, q, k, v, rq, rk, h, hk, D, causal, scale)
        dq[rq, h * D:(h + 1) * D] += scale * ds @ _heads(k[rk], hk, D)
        dk[rk, hk * D:(hk + 1) * D] += scale * ds.T @ _heads(q[rq], h, D)
        dv[rk, hk * D:(hk + 1) * D] += p.T @ _heads(do[rq], h, D)
    return dq, dk, dv


def _weights(do, o, lse, q, k, v, rq, rk, h, hk, D, causal, scale):
    see = seen(rq.stop - rq.start, rk.stop - rk.start, causal)
    s = scale * _heads(q[rq], h, D) @ _heads(k[rk], hk, D).T
    level = np.where(np.isfinite(lse[h, rq]), lse[h, rq], 0.0)[:, None]
    p = np.where(see, np.exp(np.where(see, s - level, 0.0)), 0.0)
    g = _heads(do[rq], h, D)
    return p, p * (g @ _heads(v[rk], hk, D).T - (g * _heads(o[rq], h, D)).sum(1)[:, None])


def attention_bounds(do, o, lse, q, k, v, q_heads, k_heads, q_begin, k_begin, causal, scale, u, r, exact_o=None):
    """How far sums in a precision of u (half a step) with weights rounded by r may be off: (o, lse, dq, dk, dv), before results are rounded.
    exact_o: sum_c do_ic o_ic may as well be that of this o, which differs from o by its rounding; so ds may be off by p times the difference of the two sums.

    A score is a sum of D products, scaled and shifted: off by e = (D + 8) u scale sum |q k| + 4 u (|s| + |lse|), which is how far its exponential is off
    relatively, with 4 u more for the exponential itself.  The rest is sums of n products: (n + 3) u times the magnitudes that meet."""
    D = q.shape[1] // q_heads
    eo, el, eq, ek, ev = np.zeros_like(q), np.zeros_like(lse), np.zeros_like(q), np.zeros_like(k), np.zeros_like(v)
    for rq, rk, h, hk in each(q_begin, k_begin, q_heads, k_heads):
        nq, nk = rq.stop - rq.start, rk.stop - rk.start
        if not nq or not nk:
            continue
        p, ds = _weights(do, o, lse, q, k, v, rq, rk, h, hk, D, causal, scale)
        a, b, c, g = (np.abs(_heads(t[rows], i, D)) for t, rows, i in ((q, rq, h), (k, rk, hk), (v, rk, hk), (do, rq, h)))
        level = np.abs(np.where(np.isfinite(lse[h, rq]), lse[h, rq], 0.0))[:, None]
        e = (D + 8) * u * scale * (a @ b.T) + 4 * u * (scale * np.abs(_heads(q[rq], h, D) @ _heads(k[rk], hk, D).T) + level) + 4 * u
        e = np.where(p > 0, e, 0.0)
        row = (p * e).sum(1, keepdims=True)               # of the softmax's sum, relatively
        at = slice(h * D, (h + 1) * D), slice(hk * D, (hk + 1) * D)
        eo[rq, at[0]] += (p * (e + row + (nk + 6) * u + r)) @ c
        el[h, rq] += (row + (nk + 6) * u)[:, 0] + 4 * u * level[:, 0]
        meet = g @ c.T + (g * np.abs(_heads(o[rq], h, D))).sum(1)[:, None]
        es = p * (e * meet + (D + 6) * u * meet)
        if exact_o is not None:
            es = es + p * np.abs((_heads(do[rq], h, D) * _heads(o[rq] - exact_o[rq], h, D)).sum(1))[:, None]
        eq[rq, at[0]] += scale * (es + np.abs(ds) * ((nk + 6) * u + r)) @ b
        ek[rk, at[1]] += scale * (es + np.abs(ds) * ((nq * (q_heads // k_heads) + 6) * u + r)).T @ a
        ev[rk, at[1]] += (p * (e + (nq * (q_heads // k_heads) + 6) * u + r)).T @ g
    return eo, el, eq, ek, ev


def angles(positions, rotary, base):
    return np.asarray(positions, dtype=np.float64)[:, None] * np.float64(base) ** (-2.0 * np.arange(rotary // 2) / rotary)


def _pairs(rotary, adjacent):
    i = np.arange(rotary // 2)
    return (2 * i, 2 * i + 1) if adjacent else (i, i + rotary // 2)


def turned(t, angle, adjacent):
    """t: rows x heads x columns; angle: rows x pairs."""
    y = t.copy()
    a, b = _pairs(2 * angle.shape[1], adjacent)
    cos, sin = np.cos(angle)[:, None], np.sin(angle)[:, None]
    y[..., a] = t[..., a] * cos - t[..., b] * sin
    y[..., b] = t[..., b] * cos + t[..., a] * sin
    return y


def normed(x, norm, eps):
    """(norm(x), its factor) over the last axis."""
    if norm is None:
        return x, np.ones(x.shape[:-1] + (1,))
    if norm == "centred":
        x = x - x.mean(-1, keepdims=True)
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    return x * r, r


def _weight_of_rows(q_weight, k_weight, q_heads, k_heads, begin, cols):
    """rows x heads x columns of the weights."""
    n = int(begin[-1])
    w = np.ones((n, q_heads + k_heads, cols))
    for g in range(len(begin) - 1):
        rows = slice(int(begin[g]), int(begin[g + 1]))
        if q_weight is not None:
            w[rows, :q_heads] = q_weight[g]
        if k_weight is not None:
            w[rows, q_heads:] = k_weight[g]
    return w


def rotate(x, q_heads, k_heads, q_weight, k_weight, begin, positions, rotary, adjacent, base, norm, eps):
    D = x.shape[1] // (q_heads + k_heads)
    n, _ = normed(x.reshape(x.shape[0], -1, D), norm, eps)
    return turned(n * _weight_of_rows(q_weight, k_weight, q_heads, k_heads, begin, D), angles(positions, rotary, base), adjacent).reshape(x.shape)


def rotate_grad(dy, x, q_heads, k_heads, q_weight, k_weight, begin, positions, rotary, adjacent, base, norm, eps):
    """(dx, dq_weight, dk_weight); a weight's gradient also where there is no weight."""
    D = x.shape[1] // (q_heads + k_heads)
    n, r = normed(x.reshape(x.shape[0], -1, D), norm, eps)
    u = turned(dy.reshape(n.shape), -angles(positions, rotary, base), adjacent)
    dw = np.stack([(u * n)[int(begin[g]):int(begin[g + 1])].sum(0) for g in range(len(begin) - 1)])
    a = u * _weight_of_rows(q_weight, k_weight, q_heads, k_heads, begin, D)
    if norm is not None:
        a = a - n * (a * n).mean(-1, keepdims=True)
        if norm == "centred":
            a = a - a.mean(-1, keepdims=True)
    return (a * r).reshape(x.shape), dw[:, :q_heads].sum(1), dw[:, q_heads:].sum(1)


def rotate_bounds(dy, x, q_heads, k_heads, q_weight, k_weight, begin, positions, rotary, adjacent, base, norm, eps, u):
    """How far sums and operations in a precision of u (half a step) may be off: (y, dx, dq_weight, dk_weight), before results are rounded.

    Statistics of D columns: (D + 8) u of what meets.  Sines and cosines: 8 u each, absolutely (half a turn rounded to 32 bits, and two steps of the function)."""
    D, H = x.shape[1] // (q_heads + k_heads), q_heads + k_heads
    shape = (x.shape[0], H, D)
    x3 = x.reshape(shape)
    n, r = normed(x3, norm, eps)
    w = np.abs(_weight_of_rows(q_weight, k_weight, q_heads, k_heads, begin, D))
    en = (D + 8) * u * (np.abs(n) + (np.abs(x3).mean(-1, keepdims=True) * r if norm == "centred" else 0.0)) if norm else 0.0 * n

    def met(t):                              # of a column and its other one
        y = np.abs(t).copy()
        a, b = _pairs(rotary, adjacent)
        y[..., a] = y[..., b] = np.abs(t[..., a]) + np.abs(t[..., b])
        return y

    ey = met(w * (en + 12 * u * np.abs(n)))
    du = met(dy.reshape(shape))
    U = np.abs(turned(dy.reshape(shape), -angles(positions, rotary, base), adjacent))
    eu = 12 * u * du
    parts = eu * (np.abs(n) + en) + U * en
    counts = np.diff(np.asarray(begin, dtype=np.int64))
    dw = np.stack([(parts + (counts[g] * H + 40) * u * U * np.abs(n))[int(begin[g]):int(begin[g + 1])].sum(0) for g in range(len(begin) - 1)])
    a, ea = U * w, eu * w + 2 * u * U * w
    if norm:
        mean = lambda t: t.mean(-1, keepdims=True)  # noqa: E731
        an, ean = mean(a * np.abs(n)), mean(ea * np.abs(n) + a * en)
        ea = ea + np.abs(n) * (ean + (D + 8) * u * an) + en * an
        a = a + np.abs(n) * an
        if norm == "centred":
            ea = ea + mean(ea) + (D + 8) * u * mean(a)
            a = a + mean(a)
    dx = r * (ea + (D + 12) * u * a)
    return ey.reshape(x.shape), dx.reshape(x.shape), dw[:, :q_heads].sum(1), dw[:, q_heads:].sum(1)
