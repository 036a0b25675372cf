"""Layers of a residual block on grouped rows in 64 bits (oracle side).

TEST INFRASTRUCTURE ONLY - see oracle/__init__.py.  Written from the formulas: rows r of group g are begin[g] <= r < begin[g + 1].

    product        y[r] = w_g x[r]                      gradient to w: sum over the group's rows of dy[r] x[r]^T
    norm           rms: v / sqrt(mean v^2 + eps)        centred: (v - mean v) / sqrt(mean (v - mean v)^2 + eps)
    residual       y = x + scale * mask * gate * norm(b) * post,  h = next_norm(y) * pre
"""
import numpy as np

from . import rng

STREAM_DROPOUT = 8
_LO = np.uint64(0xFFFFFFFF)


def philox4x32(counter, key, rounds=10):
    """Philox4x32 of Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3" (2011).
    counter: four arrays of 32-bit words; returns four."""
    c = [np.asarray(w, dtype=np.uint64) for w in counter]
    k0, k1 = key
    s = np.uint64(32)
    for _ in range(rounds):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> s) ^ c[1] ^ np.uint64(k0), b & _LO, (a >> s) ^ c[3] ^ np.uint64(k1), a & _LO]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return c


def threshold(p):
    return int(np.floor(float(np.float32(p)) * 65536.0 + 0.5))


def mask(drop, rows, cols):
    """0 where (row, column) is dropped, else the factor of what is kept.  drop: (p, seed, worker, iter, site, first_row)."""
    p, seed, worker, it, site, first = drop
    key = rng.mix(seed, STREAM_DROPOUT, worker, it, site)
    blocks = -(-cols // 8)
    row = np.repeat(np.arange(rows, dtype=np.uint64) + np.uint64(first), blocks)
    words = philox4x32((np.tile(np.arange(blocks, dtype=np.uint64), rows), row & _LO, row >> np.uint64(32), np.zeros_like(row)),
                       (key & 0xFFFFFFFF, key >> 32))
    draws = np.stack([h for w in words for h in (w & np.uint64(0xFFFF), w >> np.uint64(16))], axis=1).reshape(rows, blocks * 8)[:, :cols]
    t = threshold(p)
    return (draws >= t) * (65536.0 / (65536 - t) if t < 65536 else 0.0)


def groups(begin):
    return [(g, slice(int(begin[g]), int(begin[g + 1]))) for g in range(len(begin) - 1)]


def product(x, w, begin, transposed=False):
    y = np.zeros((x.shape[0], w.shape[2 if transposed else 1]))
    for g, r in groups(begin):
        y[r] = x[r] @ (w[g] if transposed else w[g].T)
    return y


def product_grad(dy, x, begin):
    return np.stack([dy[r].T @ x[r] for _, r in groups(begin)])


def spread(v, begin):
    """A group's vector for each of its rows."""
    return np.repeat(v, np.diff(begin), axis=0)


def normed(v, how, eps):
    """(norm(v), its factor)"""
    if how == "centred":
        v = v - v.mean(1, keepdims=True)
    r = 1.0 / np.sqrt((v * v).mean(1, keepdims=True) + eps)
    return v * r, r


def through(a, n, r, how):
    m = a.mean(1, keepdims=True) if how == "centred" else 0.0
    return r * (a - m - n * (a * n).mean(1, keepdims=True))


def _parts(b, begin, norm, post, gate, logits, eps):
    n, r = normed(b, norm, eps) if norm else (b, None)
    t = n * spread(post, begin) if post is not None else n
    s = spread(gate, begin) if gate is not None else 1 / (1 + np.exp(-logits)) if logits is not None else np.ones_like(b)
    return n, r, t, s


def residual(x, b, begin, norm="rms", post=None, gate=None, logits=None, scale=1.0, drop=None, next_norm=None, pre=None, eps=1e-5):
    y = x
    if b is not None:
        _, _, t, s = _parts(b, begin, norm, post, gate, logits, eps)
        m = 1.0 if drop is None else mask(drop, *x.shape)
        y = x + scale * np.where(m != 0, t * s, 0.0) * m
    if next_norm is None:
        return y, None
    return y, normed(y, next_norm, eps)[0] * (1.0 if pre is None else spread(pre, begin))


def residual_grad(dy, dh, y, b, begin, norm="rms", post=None, gate=None, logits=None, scale=1.0, drop=None, next_norm=None, pre=None, eps=1e-5):
    """{dx, db, dpost, dpre, dgate, dlogits}: those that exist."""
    out = {}

    def sums(v):
        return np.stack([v[r].sum(0) for _, r in groups(begin)])
    e = np.zeros_like(dh if dy is None else dy) if dy is None else dy
    if dh is not None:
        n, r = normed(y, next_norm, eps)
        a = dh if pre is None else dh * spread(pre, begin)
        if pre is not None:
            out["dpre"] = sums(dh * n)
        e = e + through(a, n, r, next_norm)
    out["dx"] = e
    if b is None:
        return out
    n, r, t, s = _parts(b, begin, norm, post, gate, logits, eps)
    m = 1.0 if drop is None else mask(drop, *b.shape)
    f = scale * np.where(m != 0, e, 0.0) * m
    if gate is not None:
        out["dgate"] = sums(f * t)
    if logits is not None:
        out["dlogits"] = f * t * s * (1 - s)
    q = f * s
    if post is not None:
        out["dpost"] = sums(q * n)
        q = q * spread(post, begin)
    out["db"] = through(q, n, r, norm) if norm else q
    return out
