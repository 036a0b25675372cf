"""Products at sizes that, between them, take every way the library has (tiles of each size, fed by the memory unit or through registers,
whole or in parts of the contraction, few rows), against torch in 64 bits; the tolerances are those of test_layers.py."""
import pytest
import torch

from paper_1902_01064_amd import layers
from test_layers import DEV, DT, U, begin_of, laid_out, table

pytestmark = pytest.mark.gpu

# rows, groups, columns of the rows, columns of the result
SIZES = [(1, 1, 4104, 72), (16, 16, 520, 520), (16, 16, 1032, 520), (20, 1, 2056, 2056), (20, 1, 4104, 2056), (33, 2, 520, 4104), (33, 5, 1032, 2056),
         (33, 16, 1032, 520), (60, 2, 1032, 4104), (60, 40, 264, 520), (60, 40, 1032, 264), (60, 40, 2056, 72), (515, 1, 64, 72), (515, 1, 520, 520),
         (515, 16, 64, 2056), (515, 16, 520, 264), (1100, 1, 64, 72), (1100, 16, 520, 72), (1100, 40, 136, 264), (1100, 40, 520, 264),
         (1100, 40, 1032, 72), (2100, 1, 520, 72), (2100, 5, 64, 72), (2100, 2, 1032, 72), (2100, 40, 64, 264), (2100, 40, 1032, 264), (4100, 2, 1032, 72),
         (4100, 16, 64, 2056), (9000, 1, 64, 264), (9000, 2, 136, 2056), (9000, 16, 4104, 72), (9000, 40, 64, 2056), (9000, 40, 4104, 264)]


def counts_of(T, G):
    """Uneven, some empty where there are many."""
    n = [(g * 37 + 11) % 23 + (g % 5 != 3) for g in range(G)]
    cut = [0]
    for v in n:
        cut.append(cut[-1] + v)
    at = [T * v // cut[-1] for v in cut]
    return [at[g + 1] - at[g] for g in range(G)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("aligned", [True, False])
@pytest.mark.parametrize("size", SIZES)
def test_every_way(dtype, aligned, size):
    T, G, K, N = size
    counts = counts_of(T, G)
    assert sum(counts) == T
    rb = table(begin_of(counts))
    g = torch.Generator(device=DEV).manual_seed(T + K + N)
    x, dy, w = (torch.randn(s, device=DEV, generator=g).to(DT[dtype]) for s in ((T, K), (T, N), (G, N, K)))
    x64, dy64, w64 = x.double(), dy.double(), w.double()
    if not aligned:
        x, dy = laid_out(x, 3, 1), laid_out(dy, 5, 3)
    y, dx, dw = layers.product(x, w, rb), layers.product(dy, w, rb, transposed=True), layers.product_grad(dy, x, rb)
    round_to = 2.0 ** -8 if dtype == "bf16" else 0.0
    at = 0
    for i, n in enumerate(counts):
        r = slice(at, at + n)
        at += n
        for got, a, b, terms, rounding in ((y[r], x64[r], w64[i].T, K, round_to), (dx[r], dy64[r], w64[i], N, round_to), (dw[i], dy64[r].T, x64[r], n, 0.0)):
            want = torch.matmul(a, b)
            tol = (terms + 3) * U * torch.matmul(a.abs(), b.abs())
            tol = tol + rounding * (want.abs() + tol) + 1e-37
            assert bool(((got.double() - want).abs() <= tol).all()), (i, n, terms)
