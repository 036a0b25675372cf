"""Forms of the rotation and of attention that programs use: no norm and no weights, one kind's weights only, positions from many sequences, a cache with room to grow."""
import numpy as np
import pytest
import torch

from oracle import attention as oa
from paper_1902_01064_amd import attention
from test_attention import scattered
from test_layers import DEV, U, begin_of, close, holes, rounded, table

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D,rotary,adjacent", [(128, 128, False), (64, 64, False), (64, 64, True), (90, 46, False), (33, 0, False)])
@pytest.mark.parametrize("norm", [None, "rms", "centred"])
@pytest.mark.parametrize("with_q,with_k", [(False, False), (True, False), (False, True)])
def test_rotation_without_weights(dtype, D, rotary, adjacent, norm, with_q, with_k):
    hq, hk, counts = 3, 2, [4, 0, 13]
    T, begin = sum(counts), begin_of(counts)
    r = np.random.default_rng(D + rotary)
    x, x64 = scattered(r, T, (hq + hk) * D, dtype, D % 8 != 0)
    dy, dy64 = scattered(r, T, (hq + hk) * D, dtype, D % 8 != 0)
    wq, wq64 = rounded(1 + 0.3 * r.standard_normal((3, D)), "f32")
    wk, wk64 = rounded(1 + 0.3 * r.standard_normal((3, D)), "f32")
    if not with_q:
        wq = wq64 = None
    if not with_k:
        wk = wk64 = None
    pos = r.integers(0, 100000, T).astype(np.int32)
    how = dict(q_heads=hq, k_heads=hk, q_weight=wq, k_weight=wk, row_begin=table(begin), positions=torch.from_numpy(pos).to(DEV), rotary=rotary, adjacent=adjacent, norm=norm)
    rest = (hq, hk, wq64, wk64, begin, pos, rotary, adjacent, 10000.0, norm, float(np.float32(1e-5)))
    bounds = oa.rotate_bounds(dy64, x64, *rest, U)
    close(attention.rotate(x, **how), oa.rotate(x64, *rest), bounds[0], dtype, "y")
    wants = oa.rotate_grad(dy64, x64, *rest)
    dx, dwq, dwk = attention.rotate_grad(dy, x, **how)
    close(dx, wants[0], bounds[1], dtype, "dx")
    assert (dwq is None) == (not with_q) and (dwk is None) == (not with_k)
    if with_q:
        close(dwq, wants[1], bounds[2], "f32", "dq_weight")
    if with_k:
        close(dwk, wants[2], bounds[3], "f32", "dk_weight")


@pytest.mark.parametrize("S", [1, 63, 64, 65, 128, 129, 300, 4096])
def test_positions_from_many_sequences(S):
    """Rows count from the beginning of their sequence, of which some have none; those in front of the first and behind the last one from the nearest beginning in front."""
    r = np.random.default_rng(S)
    n = r.integers(0, 7, S)
    n[-1] = 2
    before, behind, D = 3, 5, 16
    seq = before + begin_of(n)
    T = int(seq[-1]) + behind
    pos = np.concatenate([np.arange(before), *[np.arange(v) for v in n[:-1]], np.arange(n[-1] + behind)])
    x, x64 = rounded(r.standard_normal((T, 2 * D)), "f32")
    dy, dy64 = rounded(r.standard_normal((T, 2 * D)), "f32")
    how = dict(q_heads=1, k_heads=1, seq_begin=table(seq), norm=None)
    rest = (1, 1, None, None, [0, T], pos, D, False, 10000.0, None, 0.0)
    bounds = oa.rotate_bounds(dy64, x64, *rest, U)
    close(attention.rotate(x, **how), oa.rotate(x64, *rest), bounds[0], "f32", "y")
    close(attention.rotate_grad(dy, x, **how)[0], oa.rotate_grad(dy64, x64, *rest)[0], bounds[1], "f32", "dx")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hq,hk,D", [(8, 2, 64), (4, 4, 128), (3, 1, 40)])
@pytest.mark.parametrize("new", [1, 40])
def test_a_cache_with_room_to_grow(dtype, hq, hk, D, new):
    """Room behind a sequence's keys is a sequence without queries: nothing in it is read, no row of a result belongs to it."""
    keys, room = [700, 40, 130, 2000], 2048
    nk = [v for n in keys for v in (n, room - n)]
    nq = [new, 0] * len(keys)
    qb, kb = begin_of(nq), begin_of(nk)
    r = np.random.default_rng(D)
    q, q64 = scattered(r, sum(nq), hq * D, dtype, False)
    k, k64 = scattered(r, sum(nk), hk * D, dtype, False)
    v, v64 = scattered(r, sum(nk), hk * D, dtype, False)
    rest = (hq, hk, qb, kb, True, D ** -0.5)
    want, lse = oa.attention(q64, k64, v64, *rest)
    bounds = oa.attention_bounds(np.zeros_like(want), want, lse, q64, k64, v64, *rest, U, 2.0 ** -8 if dtype == "bf16" else 0.0)
    for i, n in enumerate(keys):
        for t in (k, v):
            t[i * room + n:(i + 1) * room] = float("nan")
    o, unharmed = holes(sum(nq), hq * D, dtype, 0, 0)
    _, got = attention.attention(q, k, v, hq, hk, table(qb), table(kb), out=o)
    close(o, want, bounds[0], dtype, "o")
    close(got, lse, bounds[1], "f32", "lse")
    assert unharmed()
