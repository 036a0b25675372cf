"""The layers of a residual block on all replicas at once, as cases that can be timed and compared.

    listed()            the cases by name
    draw(rng)           one more case of the same ranges
    prepare(case, seed) inputs, weights and row tables: what a program has in hand before the call
    run(state)          one pass through an operator: plain torch in 32 bits, or with `own` the framework's kernels
    exact(case, seed)   the same outputs in 64 bits, written apart from the plain form
    work(case)          bytes and operations the pass cannot do without

Kinds of case
    product  rows grouped by worker or expert times their group's weights; with `train` also the gradients to rows and weights
    norm     y = x + scale * dropout(gate * norm(b) * post), h = norm(y) * pre; with `train` the gradients of all of them,
             for another micro-batch whose y the forward pass has stored
    dropout  of a tensor, and of its gradient with the same key
"""
import math
import random

import numpy as np
import torch

own = False

DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
SEED = 190201064                    # of the dropout keys: the framework's default
EPS = 1e-5
M32, M64 = (1 << 32) - 1, (1 << 64) - 1


# ------------------------------------------------------------------------------------------- the cases ----
def _product(**over):
    c = dict(kind="product", dtype="bf16", G=16, rows=2048, K=1024, N=1024, spread="even", lattice=False, train=False)
    c.update(over)
    return c


def _norm(**over):
    c = dict(kind="norm", dtype="bf16", G=1, rows=1024, cols=4096, spread="even", lattice=False, train=False, norm="rms",
             post=True, pre=True, gate="vector", scale=1.0, p=0.0)
    c.update(over)
    return c


def _dropout(**over):
    c = dict(kind="dropout", dtype="bf16", rows=1024, cols=4096, pad=0, p=0.1)
    c.update(over)
    return c


def listed():
    return [
        # ---- products
        # one token on its way through its 8 experts, while an answer is being written: the smallest call there is
        _product(name="product-token-bf16", G=8, rows=8),
        # two tokens for each of 64 experts: all weights are read for very few rows
        _product(name="product-decode-bf16", G=64, rows=128, K=2048, N=4096),
        # a long prompt over 32 experts, popular ones with many times the rows of others: matrix rate
        _product(name="product-prompt-bf16", G=32, rows=16384, K=4096, N=4096, spread="skewed"),
        # a training step of 16 experts in bf16, gradients of the weights in 32 bits; an odd number of rows
        _product(name="product-train-bf16", rows=8191, K=2048, N=4096, spread="skewed", train=True),
        # a wave of 16 workers with a minibatch of 128 each, weights read out of the 32-bit replicas in their rings
        _product(name="product-workers-f32", dtype="f32", rows=2048, K=1024, N=4096, lattice=True, train=True),
        # no size a multiple of anything: 5 workers of a layer of 777 inputs and 1290 outputs
        _product(name="product-odd-f32", dtype="f32", G=5, rows=1003, K=777, N=1290, spread="skewed", lattice=True, train=True),
        # ---- norms around a block
        # 8 sequences, one token each: latency
        _norm(name="norm-token-bf16", rows=8),
        # a training step's residual stream, 16384 tokens: bytes
        _norm(name="norm-train-bf16", rows=16384, train=True, scale=0.5, p=0.1),
        # 64 workers with 128 rows each and norms of their own in their replicas; a gate for every element
        _norm(name="norm-workers-f32", dtype="f32", G=64, rows=8192, cols=1024, lattice=True, train=True, gate="element", p=0.2),
        # odd sizes, centred norms, no gate
        _norm(name="norm-odd-bf16", G=7, rows=777, cols=5001, spread="skewed", norm="centred", gate="none", train=True, p=0.5),
        # ---- dropout by itself
        # the hidden units of one worker's minibatch of 64, rows not aligned
        _dropout(name="dropout-small-f32", dtype="f32", rows=64, cols=1023, p=0.5),
        # the hidden units of 8192 tokens, 8192 wide
        _dropout(name="dropout-large-bf16", rows=8192, cols=8192),
    ]


def _size(rng, lo, hi):
    """Spread over the logarithm; one in three is odd, the others multiples of the largest power of two that changes them little."""
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    v = min(max(v, lo), hi)
    if rng.random() < 1 / 3:
        return min(hi, v | 1)
    step = 1 << max(0, v.bit_length() - 3)
    return max(lo, min(hi, (v + step // 2) // step * step))


def _cost(c):
    """Seconds, order of magnitude only: keeps drawn cases below the dearest listed one."""
    w = work(c)
    return w["bytes"] / 4e12 + w["flops"] / (6e14 if c["dtype"] == "bf16" else 1e14)


def draw(rng):
    what = rng.choice(["product", "product", "product-train", "norm", "norm-train", "norm-train", "dropout"])
    dtype, spread = rng.choice(["bf16", "f32"]), rng.choice(["even", "skewed"])
    if what.startswith("product"):
        c = _product(dtype=dtype, spread=spread, G=_size(rng, 1, 64), rows=_size(rng, 1, 16384), K=_size(rng, 64, 8192),
                     N=_size(rng, 64, 8192), train=what.endswith("train"), lattice=dtype == "f32" and rng.random() < 0.5)
    elif what.startswith("norm"):
        c = _norm(dtype=dtype, spread=spread, G=rng.choice([1, _size(rng, 1, 64)]), rows=_size(rng, 1, 16384),
                  cols=_size(rng, 64, 16384), norm=rng.choice(["rms", "centred"]), gate=rng.choice(["none", "vector", "element"]),
                  p=rng.choice([0.0, 0.1, 0.5]), post=rng.random() < 0.8, pre=rng.random() < 0.8,
                  scale=rng.choice([1.0, 0.5]), train=what.endswith("train"), lattice=rng.random() < 0.3)
    else:
        c = _dropout(dtype=dtype, rows=_size(rng, 1, 16384), cols=_size(rng, 64, 16384), pad=rng.choice([0, 0, 8, 3]),
                     p=rng.choice([0.1, 0.2, 0.5]))
    most = max(_cost(x) for x in listed() if x["kind"] == c["kind"])
    while _cost(c) > most and c["rows"] > 1:
        c["rows"] = (c["rows"] + 1) // 2
    for side in ("K", "N", "G"):
        while side in c and _cost(c) > most and c[side] > 64:
            c[side] = (c[side] + 1) // 2
    return c


def work(c):
    e = 2 if c["dtype"] == "bf16" else 4
    if c["kind"] == "product":
        T, K, N, G = c["rows"], c["K"], c["N"], min(c["G"], c["rows"])
        b, f = e * (T * K + G * N * K + T * N), 2.0 * T * N * K
        if c["train"]:                      # dx = dy W, dW = dy^T x: reads dy, W, x, writes dx and dW in 32 bits
            b += e * (T * N + G * N * K + T * K + T * K) + 4 * c["G"] * N * K
            f *= 3
        return {"bytes": float(b), "flops": f}
    n = c["rows"] * c["cols"]
    if c["kind"] == "dropout":
        return {"bytes": 4.0 * n * e, "flops": 2.0 * n}
    streams = 3 + c["pre"] + (c["gate"] == "element")
    vectors = c["post"] + c["pre"] + (c["gate"] == "vector")
    b, f = streams * n * e + 4 * vectors * c["G"] * c["cols"], 12.0 * n
    if c["train"]:                          # reads dy, dh, b, (z, y); writes dx, db, (dz) and the parameters' gradients
        b += (4 + 2 * c["pre"] + 2 * (c["gate"] == "element")) * n * e + 8 * vectors * c["G"] * c["cols"]
        f *= 3
    return {"bytes": float(b), "flops": f}


# --------------------------------------------------------------------------------------- what is in hand ----
def _counts(c, seed):
    """Rows of each group: near equal, or Zipf-like in a random order, where small groups may have none."""
    r, G, T = random.Random(seed * 7919 + 11), c["G"], c["rows"]
    if c["spread"] == "even":
        n = [T // G + (g < T % G) for g in range(G)]
        for g in range(0, G - 1, 2):
            d = r.randint(-(n[g] // 4), n[g + 1] // 4)
            n[g], n[g + 1] = n[g] + d, n[g + 1] - d
        r.shuffle(n)
        return n
    p = [1.0 / (g + 1) for g in range(G)]
    r.shuffle(p)
    cut = [0.0]
    for v in p:
        cut.append(cut[-1] + v)
    at = [int(T * v / cut[-1]) for v in cut[:-1]] + [T]
    return [at[g + 1] - at[g] for g in range(G)]


def _groups(c, seed, state):
    counts = _counts(c, seed)
    begin = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    state["counts"], state["row_begin"] = counts, torch.from_numpy(begin).to(DEV)


def _replicas(c, seed, parts, state, g):
    """The groups' parameters: views [groups, ...] of stacked tensors, or of the flat replicas [workers x ring slots, stride] with the
    row of each group's current version in `index`.  parts: (name, shape, mean, deviation)."""
    state["index"] = None
    if not c["lattice"]:
        for name, shape, mean, dev in parts:
            dt = TYPES[c["dtype"]] if name == "w" else torch.float32
            state[name] = (torch.randn((c["G"],) + shape, device=DEV, generator=g) * dev + mean).to(dt)
        return
    d = sum(math.prod(shape) for _, shape, _, _ in parts)
    stride, slots = (d + 63) // 64 * 64 + 64, 2
    arena = torch.empty(c["G"] * slots, stride, device=DEV)
    arena.normal_(generator=g)
    r = random.Random(seed * 31 + 7)
    state["index"] = [i * slots + r.randrange(slots) for i in range(c["G"])]
    at = 0
    for name, shape, mean, dev in parts:
        n = math.prod(shape)
        arena[:, at:at + n].mul_(dev).add_(mean)
        state[name] = arena[:, at:at + n].unflatten(1, shape)
        at += n


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    dt = TYPES[c["dtype"]]

    def normal(*shape):
        return torch.randn(shape, device=DEV, generator=g)

    s = {"case": c}
    if c["kind"] == "product":
        _groups(c, seed, s)
        T, K, N = c["rows"], c["K"], c["N"]
        s["x"] = normal(T, K).to(dt)
        _replicas(c, seed, [("w", (N, K), 0.0, K ** -0.5)], s, g)
        if c["train"]:
            s["dy"] = normal(T, N).to(dt)
    elif c["kind"] == "norm":
        _groups(c, seed, s)
        T, d = c["rows"], c["cols"]
        loud = 1 + 7 * (torch.rand(d, device=DEV, generator=g) < 0.01)          # a residual stream has a few loud columns
        s["x"] = (normal(T, d) * loud).to(dt)
        s["b"] = (normal(T, d) * 0.5 + 0.1).to(dt)
        parts = [("post", (d,), 1.0, 0.1)] * c["post"] + [("pre", (d,), 1.0, 0.1)] * c["pre"]
        parts += [("gamma", (d,), 0.5, 0.2)] * (c["gate"] == "vector")
        s.update(post=None, pre=None, gamma=None, z=None, index=None)
        if parts:
            _replicas(c, seed, parts, s, g)
        if c["gate"] == "element":
            s["z"] = normal(T, d).to(dt)
        s["key"] = (SEED, seed % 1000, seed % 77, 3)                            # seed, worker, iteration, layer
        if c["train"]:
            s["y"] = (normal(T, d) * loud).to(dt)                               # as an earlier forward pass stored it
            s["dy"] = normal(T, d).to(dt)
            s["dh"] = normal(T, d).to(dt) if c["pre"] else None
    else:
        T, d, pad = c["rows"], c["cols"], c["pad"]
        s["x"] = torch.relu(normal(T, d + pad)).to(dt)[:, :d]
        s["dy"] = normal(T, d + pad).to(dt)[:, :d]
        s["key"] = (SEED, seed % 1000, seed % 77, 5)
    return s


# ----------------------------------------------------------------------------------------- the plain form ----
def _sm64(z):
    z = (z + 0x9E3779B97F4A7C15) & M64
    z = ((z ^ (z >> 30)) * 0xBF58476D1CE4E5B9) & M64
    z = ((z ^ (z >> 27)) * 0x94D049BB133111EB) & M64
    return z ^ (z >> 31)


def _fold(seed, worker, iteration, site):
    """Key of a mask: SplitMix64's output function over (seed, stream of the dropout, worker, iteration, site)."""
    return _sm64(_sm64(_sm64(_sm64(_sm64(seed) ^ 8) ^ worker) ^ iteration) ^ site)


def _keep(key, rows, cols, p):
    """Philox4x32-10 on 64-bit integers: counter (column / 8, row, 0, 0), eight 16-bit draws of a counter; and the factor of what is kept."""
    k = _fold(*key)
    k0, k1 = k & M32, k >> 32
    blocks = (cols + 7) // 8
    c0 = torch.arange(blocks, device=DEV).expand(rows, blocks)
    c1 = torch.arange(rows, device=DEV)[:, None].expand(rows, blocks)
    c2 = c3 = torch.zeros((), dtype=torch.int64, device=DEV)
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((b >> 32) & M32) ^ c1 ^ k0, b & M32, ((a >> 32) & M32) ^ c3 ^ k1, a & M32
        k0, k1 = (k0 + 0x9E3779B9) & M32, (k1 + 0xBB67AE85) & M32
    words = torch.stack([c0, c1, c2, c3], dim=-1)
    draws = torch.stack([words & 0xFFFF, words >> 16], dim=-1).reshape(rows, blocks * 8)[:, :cols]
    t = int(p * 65536 + 0.5)
    return draws >= t, 65536.0 / (65536 - t) if t < 65536 else 0.0


def _drop(v, key, p):
    if p == 0:
        return v
    keep, factor = _keep(key, v.shape[0], v.shape[1], p)
    return torch.where(keep, v * factor, torch.zeros((), device=DEV))


def _rows_of(vector, s):
    """A group's vector for each of its rows."""
    v = vector if s["index"] is None else vector[s["index"]]
    return v[0] if v.shape[0] == 1 else v.repeat_interleave(torch.tensor(s["counts"], device=DEV), 0)


def _sums(v, s):
    return torch.stack([part.sum(0) for part in v.split(s["counts"])])


def _normed(v, how):
    if how == "centred":
        v = v - v.mean(1, keepdim=True)
    r = torch.rsqrt((v * v).mean(1, keepdim=True) + EPS)
    return v * r, r


def _normed_back(a, n, r, how):
    a = a - n * (a * n).mean(1, keepdim=True)
    return r * (a - a.mean(1, keepdim=True) if how == "centred" else a)


def _plain_product(s):
    c, dt = s["case"], s["x"].dtype
    x = s["x"].float().split(s["counts"])
    w = [s["w"][i] for i in (s["index"] or range(c["G"]))]
    out = {"y": torch.cat([xg @ wg.float().t() for xg, wg in zip(x, w)]).to(dt)}
    if c["train"]:
        dy = s["dy"].float().split(s["counts"])
        out["dx"] = torch.cat([dg @ wg.float() for dg, wg in zip(dy, w)]).to(dt)
        out["dw"] = torch.stack([dg.t() @ xg for dg, xg in zip(dy, x)])
    return out


def _plain_norm(s):
    c, dt, how = s["case"], s["x"].dtype, s["case"]["norm"]
    post, pre, gamma = [None if s[k] is None else _rows_of(s[k], s) for k in ("post", "pre", "gamma")]
    gate = gamma if gamma is not None else None if s["z"] is None else torch.sigmoid(s["z"].float())
    b, r = _normed(s["b"].float(), how) if c["post"] else (s["b"].float(), None)
    t = b * post if c["post"] else b
    y = s["x"].float() + c["scale"] * _drop(t if gate is None else t * gate, s["key"], c["p"])
    out = {"y": y.to(dt)}
    if c["pre"]:
        out["h"] = (_normed(y, how)[0] * pre).to(dt)
    if c["train"]:
        e = s["dy"].float()
        if c["pre"]:
            dh = s["dh"].float()
            n, ry = _normed(s["y"].float(), how)
            e = e + _normed_back(dh * pre, n, ry, how)
            out["dpre"] = _sums(dh * n, s)
        f = c["scale"] * _drop(e, s["key"], c["p"])
        if c["gate"] == "vector":
            out["dgamma"] = _sums(f * t, s)
        if c["gate"] == "element":
            out["dz"] = (f * t * gate * (1 - gate)).to(dt)
        q = f if gate is None else f * gate
        if c["post"]:
            out["dpost"] = _sums(q * b, s)
            q = _normed_back(q * post, b, r, how)
        out["dx"], out["db"] = e.to(dt), q.to(dt)
    return out


def _plain_dropout(s):
    c, dt = s["case"], s["x"].dtype
    return {"y": _drop(s["x"].float(), s["key"], c["p"]).to(dt), "dx": _drop(s["dy"].float(), s["key"], c["p"]).to(dt)}


def run(state):
    s, c = state, state["case"]
    if not own:
        return {"product": _plain_product, "norm": _plain_norm, "dropout": _plain_dropout}[c["kind"]](s)
    from paper_1902_01064_amd import layers
    if c["kind"] == "product":
        out = {"y": layers.product(s["x"], s["w"], s["row_begin"], index=s["index"])}
        if c["train"]:
            out["dx"] = layers.product(s["dy"], s["w"], s["row_begin"], index=s["index"], transposed=True)
            out["dw"] = layers.product_grad(s["dy"], s["x"], s["row_begin"])
        return out
    drop = layers.Drop(c["p"], *s["key"]) if c["p"] else None
    if c["kind"] == "dropout":
        return {"y": layers.dropout(s["x"], drop), "dx": layers.dropout(s["dy"], drop)}
    how = dict(row_begin=s["row_begin"], index=s["index"], norm=c["norm"] if c["post"] else None, post=s["post"],
               gate=s["gamma"], gate_logits=s["z"], scale=c["scale"], drop=drop,
               next_norm=c["norm"] if c["pre"] else None, pre=s["pre"], eps=EPS)
    out = {}
    out["y"], h = layers.residual(s["x"], s["b"], **how)
    if c["pre"]:
        out["h"] = h
    if c["train"]:
        back = layers.residual_grad(s["dy"], s["dh"], s["y"], s["b"], **how)
        out["dx"], out["db"] = back.dx, back.db
        for name, grad in (("dpost", back.dpost), ("dpre", back.dpre), ("dgamma", back.dgate), ("dz", back.dlogits)):
            if grad is not None:
                out[name] = grad
    return out


# ------------------------------------------------------------------------------------------ in 64 bits ----
def _mask64(key, rows, cols, p):
    """The same generator on numpy's unsigned words, row block by row block: 0 or the factor of what is kept."""
    z = key[0]
    for i, word in enumerate((8,) + tuple(key[1:])):
        z = _sm64(z if i == 0 else z) ^ word
    z = _sm64(z)
    t = int(p * 65536 + 0.5)
    out = np.zeros((rows, cols), dtype=np.float32)
    blocks = -(-cols // 8)
    lo = np.uint64(M32)
    for at in range(0, rows, 1024):
        n = min(1024, rows - at)
        c = [np.tile(np.arange(blocks, dtype=np.uint64), n), np.repeat(np.arange(at, at + n, dtype=np.uint64), blocks),
             np.zeros(n * blocks, np.uint64), np.zeros(n * blocks, np.uint64)]
        key0, key1 = z & M32, z >> 32
        for _ in range(10):
            a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
            c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(key0), b & lo, (a >> np.uint64(32)) ^ c[3] ^ np.uint64(key1), a & lo]
            key0, key1 = (key0 + 0x9E3779B9) & M32, (key1 + 0xBB67AE85) & M32
        words = np.stack([w.astype(np.uint32) for w in c], axis=1)
        halves = words.view(np.uint16).reshape(n, blocks * 8)[:, :cols]         # low half first
        out[at:at + n] = halves >= t
    return torch.from_numpy(out).to(DEV).double() * (65536.0 / (65536 - t))


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["kind"] == "product":
        x, out, at = s["x"].double(), {}, 0
        dy = s["dy"].double() if c["train"] else None
        y = torch.zeros(c["rows"], c["N"], dtype=torch.float64, device=DEV)
        dx, dw = torch.zeros_like(x), torch.zeros(c["G"], c["N"], c["K"], dtype=torch.float64, device=DEV) if c["train"] else None
        for g, n in enumerate(s["counts"]):
            w = s["w"][g if s["index"] is None else s["index"][g]].double()
            y[at:at + n] = torch.matmul(x[at:at + n], w.T)
            if c["train"]:
                dx[at:at + n] = torch.matmul(dy[at:at + n], w)
                dw[g] = torch.matmul(dy[at:at + n].T, x[at:at + n])
            at += n
        out["y"] = y
        if c["train"]:
            out.update(dx=dx, dw=dw)
        return out
    if c["kind"] == "dropout":
        m = _mask64(s["key"], c["rows"], c["cols"], c["p"])
        return {"y": s["x"].double() * m, "dx": s["dy"].double() * m}
    # norms: the forward pass by its definition, the gradients by torch's own differentiation of it
    group = np.repeat(np.arange(c["G"]), s["counts"])
    row = torch.from_numpy(group).to(DEV)
    mask = _mask64(s["key"], c["rows"], c["cols"], c["p"]) if c["p"] else None
    leaf = {}
    for name in ("post", "pre", "gamma"):
        if s[name] is not None:
            v = s[name] if s["index"] is None else s[name][torch.tensor(s["index"], device=DEV)]
            leaf[name] = v.double().requires_grad_(c["train"])
    for name in ("x", "b", "z"):
        if s[name] is not None:
            leaf[name] = s[name].double().requires_grad_(c["train"])

    def norm(v):
        if c["norm"] == "centred":
            v = v - v.sum(1, keepdim=True) / c["cols"]
        return v / torch.sqrt(v.square().sum(1, keepdim=True) / c["cols"] + EPS)

    branch = norm(leaf["b"]) * leaf["post"][row] if c["post"] else leaf["b"]
    if "gamma" in leaf:
        branch = branch * leaf["gamma"][row]
    if "z" in leaf:
        branch = branch / (1 + torch.exp(-leaf["z"]))
    branch = branch * c["scale"] if mask is None else branch * mask * c["scale"]
    y = leaf["x"] + branch
    out = {"y": y.detach()}
    if c["pre"]:
        out["h"] = (norm(y) * leaf["pre"][row]).detach()
    if c["train"]:
        e = s["dy"].double()
        if c["pre"]:
            kept = s["y"].double().requires_grad_(True)
            back = torch.autograd.grad(norm(kept) * leaf["pre"][row], [kept, leaf["pre"]], s["dh"].double())
            e, out["dpre"] = e + back[0], back[1]
        names = [n for n in ("x", "b", "z", "post", "gamma") if n in leaf]
        grads = dict(zip(names, torch.autograd.grad(y, [leaf[n] for n in names], e)))
        out.update(("d" + n, g) for n, g in grads.items())
    return out
