"""Infinities in values that some rows see and others of the same tile do not: a row that sees one has it in its result, as in the 64-bit statement, wherever the row lies."""
import numpy as np
import pytest
import torch

from oracle import attention as oa
from paper_1902_01064_amd import attention
from test_attention import scattered
from test_layers import U, begin_of, close, table

pytestmark = pytest.mark.gpu
INF = float("inf")


def check(dtype, nq, nk, hq, hk, D, odd, places):
    """places: (key's row, column, value), the column one of all heads'."""
    r = np.random.default_rng(sum(nk) + D)
    qb, kb = begin_of(nq), begin_of(nk)
    q, q64 = scattered(r, sum(nq), hq * D, dtype, odd)
    k, k64 = scattered(r, sum(nk), hk * D, dtype, odd)
    v, v64 = scattered(r, sum(nk), hk * D, dtype, odd)
    rest = (hq, hk, qb, kb, True, D ** -0.5)
    # bounds of what stays finite: those of the values without the infinities, which it does not see
    want, lse = oa.attention(q64, k64, v64, *rest)
    bound, bound_lse = oa.attention_bounds(np.zeros_like(want), want, lse, q64, k64, v64, *rest, U, 2.0 ** -8 if dtype == "bf16" else 0.0)[:2]
    for row, column, value in places:
        v[row, column] = v64[row, column] = value
    with np.errstate(invalid="ignore"):
        want, lse = oa.attention(q64, k64, v64, *rest)
    o, got_lse = attention.attention(q, k, v, q_heads=hq, k_heads=hk, q_begin=table(qb), k_begin=table(kb))
    got = o.double().cpu().numpy()
    there = ~np.isfinite(want)
    assert np.array_equal(got[there], want[there], equal_nan=True) and np.isfinite(got[~there]).all()
    assert np.isposinf(want).any() and np.isneginf(want).any()
    close(torch.from_numpy(np.where(there, 0.0, got)), np.where(there, 0.0, want), bound, dtype, "o")
    close(got_lse, lse, bound_lse, "f32", "lse")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hq,hk,D", [(2, 2, 64), (6, 2, 128), (3, 1, 33)])
@pytest.mark.parametrize("n", [50, 300])
def test_on_the_diagonal_and_behind_it(dtype, hq, hk, D, n):
    """In the first tile that a row's pass takes, in the one on the diagonal and between; of both signs in one column the result is NaN."""
    places = [(3, 1, INF), (10, D // 2, -INF), (n // 2, 5, INF), (n // 2 + 1, 5, -INF), (n - 4, 7, -INF), (n - 2, hk * D - 1, INF)]
    check(dtype, [n], [n], hq, hk, D, D % 8 != 0, places)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [64, 128, 33])
def test_few_tokens(dtype, D):
    """Three new tokens of each sequence: the last two see what the first one does not."""
    n = [1500, 90, 3]
    end = np.cumsum(n)
    check(dtype, [3, 3, 3], n, 4, 2, D, D % 8 != 0, [(end[0] - 2, 1, INF), (end[0] - 1, 2, -INF), (end[1] - 2, 3, -INF), (end[2] - 2, D + 1, INF), (40, 4, INF)])
