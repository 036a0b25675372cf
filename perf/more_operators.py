"""Attention over the replicas' packed sequences, and the norm and rotation of its queries and keys, as cases that can be timed and compared.

    listed()            the cases by name
    draw(rng)           one more case of the same ranges
    prepare(case, seed) inputs, weights and tables: what a program has in hand before the call
    run(state)          one pass through an operator: plain torch in 32 bits, or with `own` the framework's kernels
    exact(case, seed)   the same outputs in 64 bits, written apart from the plain form
    work(case)          bytes and operations the pass cannot do without

Kinds of case
    rotate  norm of every head of queries and keys times a weight, then the rotation of its columns by the row's position; with `train`
            also the gradients to rows and weights
    attend  softmax attention of packed sequences with grouped heads; queries are the last rows of their sequence's keys where causal;
            with `train` also the gradients to queries, keys and values
"""
import math
import random

import numpy as np
import torch

own = False

DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-5


# ------------------------------------------------------------------------------------------- the cases ----
def _rotate(**over):
    c = dict(kind="rotate", dtype="bf16", G=1, S=8, rows=1024, q_heads=32, k_heads=8, cols=128, rotary=128, adjacent=False, norm="rms",
             base=10000.0, far=False, spread="even", lattice=False, pad=0, train=False)
    c.update(over)
    return c


def _attend(**over):
    """q_rows of 0: the queries' rows are the keys'.  pad: columns between the end of a row and the next one."""
    c = dict(kind="attend", dtype="bf16", S=4, q_rows=0, k_rows=4096, q_heads=32, k_heads=8, cols=128, causal=True, spread="even", pad=0, train=False)
    c.update(over)
    return c


def listed():
    return [
        # ---- norm and rotation of queries and keys
        # 8 sequences, one token each, far into their texts: latency
        _rotate(name="rotate-token-bf16", rows=8, far=True),
        # a training step of 16384 tokens: bytes
        _rotate(name="rotate-train-bf16", rows=16384, train=True),
        # 64 workers with 128 rows each, weights read out of the 32-bit replicas in their rings
        _rotate(name="rotate-workers-f32", dtype="f32", G=64, S=256, rows=8192, q_heads=8, k_heads=8, cols=64, rotary=64, lattice=True, train=True),
        # odd sizes: neighbouring columns are the pairs, some columns do not turn, centred norms, rows not aligned
        _rotate(name="rotate-odd-bf16", G=7, S=19, rows=1777, q_heads=6, k_heads=3, cols=90, rotary=46, adjacent=True, norm="centred", base=500.0, spread="skewed",
                pad=3, train=True),
        # ---- attention
        # 4 sequences of about 500 tokens, the next token of each: latency
        _attend(name="attend-token-bf16", q_rows=4, k_rows=2048, q_heads=16, k_heads=4, cols=64),
        # 16 sequences of about 16384 tokens, the next token of each: the keys' and values' bytes
        _attend(name="attend-decode-bf16", S=16, q_rows=16, k_rows=262144),
        # 512 new tokens of 2 long sequences that have 8192 tokens each
        _attend(name="attend-more-bf16", S=2, q_rows=512, k_rows=16384),
        # packed prompts of very different lengths: matrix rate
        _attend(name="attend-prompt-bf16", k_rows=8192, spread="skewed"),
        # a training step over sequences of 1024 to 4096 tokens
        _attend(name="attend-train-bf16", S=6, k_rows=12288, q_heads=16, k_heads=2, train=True),
        # a wave of 16 workers with 2 sequences of about 128 tokens each, in 32 bits
        _attend(name="attend-workers-f32", dtype="f32", S=32, k_rows=4096, q_heads=8, k_heads=8, cols=64, train=True),
        # odd sizes: uneven lengths, heads of 72 columns, groups of 3 heads, rows not aligned, every key seen
        _attend(name="attend-odd-bf16", S=29, k_rows=3001, q_heads=6, k_heads=2, cols=72, causal=False, spread="skewed", pad=3, train=True),
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


def _scores(c):
    """Elements of the plain form's padded scores."""
    return c["S"] * c["q_heads"] * max(_lengths(c, "q")) * max(_lengths(c, "k"))


def draw(rng):
    what = rng.choice(["rotate", "rotate-train", "attend", "attend", "attend-train", "attend-train", "token"])
    dtype, spread = rng.choice(["bf16", "bf16", "f32"]), rng.choice(["even", "skewed"])
    if what.startswith("rotate"):
        cols = rng.choice([64, 128, 2 * _size(rng, 8, 64)])
        c = _rotate(dtype=dtype, spread=spread, G=rng.choice([1, _size(rng, 1, 64)]), S=_size(rng, 1, 256), rows=_size(rng, 1, 16384), q_heads=_size(rng, 1, 32),
                    k_heads=_size(rng, 1, 8), cols=cols, rotary=rng.choice([cols, cols, 2 * _size(rng, 1, cols // 2)]), adjacent=rng.random() < 0.3,
                    norm=rng.choice(["rms", "rms", "centred"]), base=rng.choice([10000.0, 500000.0]), far=rng.random() < 0.3, lattice=rng.random() < 0.4,
                    pad=rng.choice([0, 0, 8, 3]), train=what.endswith("train"))
    else:
        k_heads, group = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 3, 4, 8])
        c = _attend(dtype=dtype, spread=spread, S=_size(rng, 1, 32), k_rows=_size(rng, 1, 12288), q_heads=k_heads * group, k_heads=k_heads,
                    cols=rng.choice([64, 128, _size(rng, 16, 128)]), causal=rng.random() < 0.75, pad=rng.choice([0, 0, 8, 3]), train=what.endswith("train"))
        if what == "token":
            c.update(k_rows=_size(rng, 64, 262144), causal=True)
            c["q_rows"] = c["S"]
        elif rng.random() < 0.3:
            c["q_rows"] = _size(rng, 1, max(1, c["k_rows"] // 2))
        if c["train"]:                      # where all rows see one key or none, gradients are nothing but rounding
            c["k_rows"] = max(c["k_rows"], 16 * c["S"])
    same = [x for x in listed() if x["kind"] == c["kind"]]
    most = max(_cost(x) for x in same)
    room = max(_scores(x) for x in same) if c["kind"] == "attend" else 0
    while _cost(c) > most or (room and _scores(c) > room):
        for rows in ("rows", "k_rows", "q_rows"):
            if c.get(rows, 0) > 1:
                c[rows] = (c[rows] + 1) // 2
    return c


def work(c):
    e = 2 if c["dtype"] == "bf16" else 4
    if c["kind"] == "rotate":
        n = c["rows"] * (c["q_heads"] + c["k_heads"]) * c["cols"]
        w = 8 * c["G"] * c["cols"]
        b, f = 2 * n * e + w, 10.0 * n
        if c["train"]:                      # reads x, dy, writes dx and the weights' gradients
            b, f = b + 3 * n * e + 2 * w, 3 * f
        return {"bytes": float(b), "flops": f}
    pairs = 0
    for nq, nk in zip(_lengths(c, "q"), _lengths(c, "k")):
        if not c["causal"]:
            pairs += nq * nk
        else:                               # the last query sees all keys, each one before it one fewer
            seen = min(nq, nk)
            pairs += seen * nk - seen * (seen - 1) // 2
    D, Tq, Tk = c["cols"], sum(_lengths(c, "q")), sum(_lengths(c, "k"))
    q, kv = Tq * c["q_heads"] * D * e, Tk * c["k_heads"] * D * e
    b, f = 2 * q + 2 * kv + 4 * Tq * c["q_heads"], 4.0 * pairs * c["q_heads"] * D
    if c["train"]:                          # reads q, k, v, o, their sums' logarithms and do, writes dq, dk, dv
        b, f = b + 4 * q + 4 * kv + 4 * Tq * c["q_heads"], f + 10.0 * pairs * c["q_heads"] * D
    return {"bytes": float(b), "flops": f}


# --------------------------------------------------------------------------------------- what is in hand ----
def _cut(total, parts, spread, salt):
    """Rows of each part: near equal, or Zipf-like in a random order, where small parts may have none.  The case's, not the seed's."""
    r = random.Random(total * 7919 + parts * 31 + salt)
    if spread == "even":
        n = [total // parts + (g < total % parts) for g in range(parts)]
        for g in range(0, parts - 1, 2):
            d = r.randint(-(n[g] // 4), n[g + 1] // 4)
            n[g], n[g + 1] = n[g] + d, n[g + 1] - d
        r.shuffle(n)
        return n
    p = [1.0 / (g + 1) for g in range(parts)]
    r.shuffle(p)
    cut = [0.0]
    for v in p:
        cut.append(cut[-1] + v)
    at = [int(total * v / cut[-1]) for v in cut[:-1]] + [total]
    return [at[g + 1] - at[g] for g in range(parts)]


def _lengths(c, side):
    """Rows of each sequence among the queries or the keys.  New tokens of sequences with more keys are spread evenly, one each if they are as many."""
    if side == "k" or not c["q_rows"]:
        return _cut(c["k_rows"], c["S"], c["spread"], 3)
    n, S = c["q_rows"], c["S"]
    return [n // S + (g < n % S) for g in range(S)]


def _table(lengths):
    return torch.from_numpy(np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)).to(DEV)


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    dt = TYPES[c["dtype"]]

    def normal(rows, cols, pad=0, by=1.0):
        return (torch.randn((rows, cols + pad), device=DEV, generator=g) * by).to(dt)[:, :cols]

    s = {"case": c}
    if c["kind"] == "attend":
        D, nq, nk = c["cols"], _lengths(c, "q"), _lengths(c, "k")
        Tq, Tk, Hq, Hk = sum(nq), sum(nk), c["q_heads"], c["k_heads"]
        if c["q_rows"]:                     # keys and values are a cache's
            s["q"] = normal(Tq, Hq * D, c["pad"], 1.5)
            s["k"], s["v"] = normal(Tk, Hk * D, c["pad"]), normal(Tk, Hk * D, c["pad"])
        else:                               # columns of one product's result
            qkv = normal(Tk, (Hq + 2 * Hk) * D, c["pad"])
            s["q"], s["k"], s["v"] = qkv[:, :Hq * D], qkv[:, Hq * D:(Hq + Hk) * D], qkv[:, (Hq + Hk) * D:]
            s["q"].mul_(1.5)
        s["q_begin"], s["k_begin"] = _table(nq), _table(nk)
        s["Lq"], s["Lk"] = max(nq), max(nk)
        if c["train"]:
            s["do"] = normal(Tq, Hq * D)
        return s
    rows, heads, D, G = c["rows"], c["q_heads"] + c["k_heads"], c["cols"], c["G"]
    s["x"] = normal(rows, heads * D, c["pad"], 2.0) + torch.tensor(0.1, device=DEV, dtype=dt)
    if c["pad"]:                            # the sum above is contiguous again
        wide = torch.zeros((rows, heads * D + c["pad"]), device=DEV, dtype=dt)
        wide[:, :heads * D] = s["x"]
        s["x"] = wide[:, :heads * D]
    counts = _cut(rows, G, c["spread"], 1)
    s["counts"], s["row_begin"] = counts, _table(counts)
    lengths = _cut(rows, c["S"], c["spread"], 2)
    begin = _table(lengths)
    row = torch.arange(rows, device=DEV)
    which = torch.searchsorted(begin[1:].long(), row, right=True)
    far = torch.randint(0, 1000000, (c["S"],), device=DEV, generator=g) if c["far"] else torch.zeros(c["S"], dtype=torch.int64, device=DEV)
    s["positions"] = (row - begin[:-1].long()[which] + far[which]).to(torch.int32)
    s["index"], M, stride = None, G, 2 * D
    if c["lattice"]:
        slots, stride = 2, (2 * D + 63) // 64 * 64 + 64
        M, r = G * slots, random.Random(seed * 31 + 7)
        s["index"] = [i * slots + r.randrange(slots) for i in range(G)]
    arena = 1.0 + 0.1 * torch.randn((M, stride), device=DEV, generator=g)
    s["q_weight"], s["k_weight"] = arena[:, :D], arena[:, D:2 * D]
    if c["train"]:
        s["dy"] = normal(rows, heads * D)
    return s


# ----------------------------------------------------------------------------------------- the plain form ----
def _padded(x, begin, L, heads):
    """[S, L, heads, cols] in 32 bits, zeros behind a sequence's end, and which rows there are."""
    begin = begin.long()
    place = torch.arange(L, device=DEV)
    live = place < (begin[1:] - begin[:-1])[:, None]
    at = (begin[:-1, None] + place).clamp(max=x.shape[0] - 1)
    rows = x[at].float() * live[..., None]
    return rows.unflatten(2, (heads, -1)), live


def _packed(x, begin, rows):
    """The rows [S, L, ...] that there are, one behind the other."""
    row = torch.arange(rows, device=DEV)
    which = torch.searchsorted(begin[1:].long(), row, right=True)
    return x[which, row - begin.long()[which]]


def _heads_first(x, k_heads):
    """[S, L, heads, cols] -> [S, k_heads, L * group, cols]: the heads of a group behind each other."""
    S, L, H, D = x.shape
    return x.view(S, L, k_heads, H // k_heads, D).transpose(1, 2).reshape(S, k_heads, L * (H // k_heads), D)


def _rows_first(x, L):
    """Back again, as [S, L, heads * cols]."""
    S, Hk, n, D = x.shape
    return x.view(S, Hk, L, n // L, D).transpose(1, 2).reshape(S, L, Hk * (n // L) * D)


def _plain_attend(s):
    c, dt = s["case"], s["q"].dtype
    Hq, Hk, D = c["q_heads"], c["k_heads"], c["cols"]
    q, live_q = _padded(s["q"], s["q_begin"], s["Lq"], Hq)
    k, live_k = _padded(s["k"], s["k_begin"], s["Lk"], Hk)
    v, _ = _padded(s["v"], s["k_begin"], s["Lk"], Hk)
    q, k, v = _heads_first(q, Hk), _heads_first(k, Hk), _heads_first(v, Hk)
    seen = live_q[:, :, None] & live_k[:, None, :]
    if c["causal"]:
        nq, nk = live_q.sum(1), live_k.sum(1)
        last = torch.arange(s["Lq"], device=DEV) + (nk - nq)[:, None]
        seen = seen & (torch.arange(s["Lk"], device=DEV) <= last[:, :, None])
    seen = seen.repeat_interleave(Hq // Hk, 1)[:, None]
    scale = D ** -0.5
    p = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(scale).masked_fill_(~seen, -math.inf)
    top = p.amax(3, keepdim=True).clamp(min=-3e38)
    p = p.sub_(top).exp_()
    total = p.sum(3, keepdim=True)
    p = p.div_(total.clamp(min=1e-38))
    o = torch.matmul(p, v)
    lse = torch.where(total > 0, top + total.log(), -math.inf)
    rows = s["q"].shape[0]
    out = {"o": _packed(_rows_first(o, s["Lq"]), s["q_begin"], rows).to(dt), "lse": _packed(_rows_first(lse, s["Lq"]), s["q_begin"], rows).t().contiguous()}
    if c["train"]:
        do = _heads_first(_padded(s["do"], s["q_begin"], s["Lq"], Hq)[0], Hk)
        dv = torch.matmul(p.transpose(2, 3).contiguous(), do)
        ds = torch.matmul(do, v.transpose(2, 3).contiguous()).sub_((do * o).sum(3, keepdim=True)).mul_(p).mul_(scale)
        dq, dk = torch.matmul(ds, k), torch.matmul(ds.transpose(2, 3).contiguous(), q)
        out["dq"] = _packed(_rows_first(dq, s["Lq"]), s["q_begin"], rows).to(dt)
        out["dk"] = _packed(_rows_first(dk, s["Lk"]), s["k_begin"], s["k"].shape[0]).to(dt)
        out["dv"] = _packed(_rows_first(dv, s["Lk"]), s["k_begin"], s["v"].shape[0]).to(dt)
    return out


def _turned(t, cos, sin, c):
    """The first `rotary` columns of every head [rows, heads, cols] turned by the row's angles."""
    R = c["rotary"]
    cos, sin = cos[:, None], sin[:, None]
    a, b = (t[..., 0:R:2], t[..., 1:R:2]) if c["adjacent"] else (t[..., :R // 2], t[..., R // 2:R])
    a, b = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([a, b], 3).flatten(2) if c["adjacent"] else torch.cat([a, b], 2)
    return torch.cat([turned, t[..., R:]], 2)


def _plain_rotate(s):
    c, dt, D, Hq = s["case"], s["x"].dtype, s["case"]["cols"], s["case"]["q_heads"]
    x = s["x"].float().unflatten(1, (-1, D))
    mean = x.mean(2, keepdim=True) if c["norm"] == "centred" else 0.0
    r = torch.rsqrt((x - mean).square().mean(2, keepdim=True) + EPS)
    n = (x - mean) * r
    which = slice(None) if s["index"] is None else s["index"]
    counts = torch.tensor(s["counts"], device=DEV)
    wq, wk = (s[w][which].repeat_interleave(counts, 0)[:, None].expand(-1, h, -1) for w, h in (("q_weight", Hq), ("k_weight", c["k_heads"])))
    w = torch.cat([wq, wk], 1)
    i = torch.arange(c["rotary"] // 2, device=DEV, dtype=torch.float64)
    angle = s["positions"].double()[:, None] * c["base"] ** (-2 * i / c["rotary"])
    cos, sin = angle.cos().float(), angle.sin().float()
    out = {"y": _turned(n * w, cos, sin, c).flatten(1).to(dt)}
    if c["train"]:
        u = _turned(s["dy"].float().unflatten(1, (-1, D)), cos, -sin, c)
        dw = torch.stack([part.sum(0) for part in (u * n).split(s["counts"])])
        out["dq_weight"], out["dk_weight"] = dw[:, :Hq].sum(1), dw[:, Hq:].sum(1)
        u = u * w
        u = u - n * (u * n).mean(2, keepdim=True)
        if c["norm"] == "centred":
            u = u - u.mean(2, keepdim=True)
        out["dx"] = (u * r).flatten(1).to(dt)
    return out


def run(state):
    s, c = state, state["case"]
    if not own:
        return _plain_attend(s) if c["kind"] == "attend" else _plain_rotate(s)
    from paper_1902_01064_amd import attention
    if c["kind"] == "attend":
        how = dict(q_heads=c["q_heads"], k_heads=c["k_heads"], q_begin=s["q_begin"], k_begin=s["k_begin"], causal=c["causal"])
        o, lse = attention.attention(s["q"], s["k"], s["v"], **how)
        out = {"o": o, "lse": lse}
        if c["train"]:
            out["dq"], out["dk"], out["dv"] = attention.attention_grad(s["do"], o, lse, s["q"], s["k"], s["v"], **how)
        return out
    how = dict(q_heads=c["q_heads"], k_heads=c["k_heads"], q_weight=s["q_weight"], k_weight=s["k_weight"], row_begin=s["row_begin"], index=s["index"],
               positions=s["positions"], rotary=c["rotary"], adjacent=c["adjacent"], base=c["base"], norm=c["norm"], eps=EPS)
    out = {"y": attention.rotate(s["x"], **how)}
    if c["train"]:
        out["dx"], out["dq_weight"], out["dk_weight"] = attention.rotate_grad(s["dy"], s["x"], **how)
    return out


# ------------------------------------------------------------------------------------------ in 64 bits ----
def exact(case, seed):
    c, s = case, prepare(case, seed)
    D, Hq, Hk, f64 = c["cols"], c["q_heads"], c["k_heads"], torch.float64
    if c["kind"] == "attend":               # sequence by sequence and head by head, the gradients by torch's own differentiation
        Tq, Tk = s["q"].shape[0], s["k"].shape[0]
        out = {"o": torch.zeros(Tq, Hq * D, dtype=f64, device=DEV), "lse": torch.full((Hq, Tq), -math.inf, dtype=f64, device=DEV)}
        if c["train"]:
            out.update(dq=torch.zeros(Tq, Hq * D, dtype=f64, device=DEV), dk=torch.zeros(Tk, Hk * D, dtype=f64, device=DEV),
                       dv=torch.zeros(Tk, Hk * D, dtype=f64, device=DEV))
        q0 = k0 = 0
        for nq, nk in zip(_lengths(c, "q"), _lengths(c, "k")):
            rows_q, rows_k = slice(q0, q0 + nq), slice(k0, k0 + nk)
            q0, k0 = q0 + nq, k0 + nk
            if not nq or not nk:
                continue
            hidden = torch.ones(nq, nk, dtype=torch.bool, device=DEV).triu(nk - nq + 1) if c["causal"] else None
            blind = max(0, nq - nk) if c["causal"] else 0
            for h in range(Hq):
                at, at_k = slice(h * D, h * D + D), slice(h // (Hq // Hk) * D, h // (Hq // Hk) * D + D)
                leaves = [s["q"][rows_q, at].double(), s["k"][rows_k, at_k].double(), s["v"][rows_k, at_k].double()]
                q, k, v = [t.requires_grad_(c["train"]) for t in leaves]
                score = (q @ k.T)[blind:] / math.sqrt(D)
                if hidden is not None:
                    score = score.masked_fill(hidden[blind:], -math.inf)
                lse = torch.logsumexp(score, 1)
                o = torch.exp(score - lse[:, None]) @ v
                out["o"][rows_q, at][blind:], out["lse"][h, rows_q][blind:] = o.detach(), lse.detach()
                if c["train"]:
                    grads = torch.autograd.grad(o, [q, k, v], s["do"][rows_q, at].double()[blind:])
                    out["dq"][rows_q, at] += grads[0]
                    out["dk"][rows_k, at_k] += grads[1]
                    out["dv"][rows_k, at_k] += grads[2]
        return out
    # the rotation as a product of complex numbers, the gradients by torch's own differentiation
    R, rows = c["rotary"], c["rows"]
    x = s["x"].double().requires_grad_(c["train"])
    ws = []
    for name in ("q_weight", "k_weight"):
        w = s[name] if s["index"] is None else s[name][torch.tensor(s["index"], device=DEV)]
        ws.append(w.double().requires_grad_(c["train"]))
    group = torch.from_numpy(np.repeat(np.arange(c["G"]), s["counts"])).to(DEV)
    heads = x.view(rows, Hq + Hk, D)
    if c["norm"] == "centred":
        heads = heads - heads.sum(2, keepdim=True) / D
    heads = heads / torch.sqrt(heads.square().sum(2, keepdim=True) / D + EPS)
    t = torch.cat([heads[:, :Hq] * ws[0][group][:, None], heads[:, Hq:] * ws[1][group][:, None]], 1)
    speed = torch.exp(torch.arange(R // 2, device=DEV, dtype=f64) * (-2.0 / R * math.log(c["base"])))
    turn = torch.polar(torch.ones((), dtype=f64, device=DEV), s["positions"].to(f64)[:, None] * speed)[:, None]
    if c["adjacent"]:
        z = torch.view_as_complex(t[..., :R].reshape(rows, Hq + Hk, R // 2, 2)) * turn
        turned = torch.view_as_real(z).flatten(2)
    else:
        z = torch.complex(t[..., :R // 2], t[..., R // 2:R]) * turn
        turned = torch.cat([z.real, z.imag], 2)
    y = torch.cat([turned, t[..., R:]], 2).flatten(1)
    out = {"y": y.detach()}
    if c["train"]:
        out["dx"], out["dq_weight"], out["dk_weight"] = torch.autograd.grad(y, [x] + ws, s["dy"].double())
    return out
