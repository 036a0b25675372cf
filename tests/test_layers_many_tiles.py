"""Products of more tiles than a launch has room for: they go in several, and the limits of a call are refused."""
import pytest
import torch

from paper_1902_01064_amd import layers
from test_layers_refusals import A, BAD, grad, product

DEV = "cuda:0"


def test_results_of_over_2_to_the_40_elements_are_refused():
    n, rows = 1 << 21, 1 << 19
    lib = layers.load()
    for t in (0, 1):
        assert lib.hop_product(product(rows=rows + 1, n=n, ldy=n, ldw=n, t=t), A, 1 << 30, 0) == BAD
        assert lib.hop_product_scratch_bytes(product(rows=rows + 1, n=n, ldy=n, ldw=n, t=t)) == 0
    big = dict(G=257, n=n, lddy=n, k=1 << 11, ldx=1 << 11, lddw=1 << 11, dw_stride=1 << 32)
    assert lib.hop_product_grad(grad(**big), A, 1 << 30, 0) == BAD


def rows_of(G, rows):
    """A row for each group but the second, which has none; what is left goes to the last."""
    begin = torch.arange(G + 1, dtype=torch.int32)
    begin[2:] -= 1
    begin[-1] = rows
    return begin.to(DEV)


# columns of one row each: 4096 groups x 1025 to 16392 tiles of 128 columns (64 and 256 columns wide ones come to half and twice as many; a launch
# holds 4194304), the widest with more than 2^32 threads.  A product of two 16-bit numbers is exact in 32 bits, so is a sum of up to two here.
@pytest.mark.gpu
@pytest.mark.parametrize("cols", [131136, 524352, (1 << 21) - 64])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_products_of_many_groups(cols, dtype):
    G = T = 4096
    g = torch.Generator(device=DEV).manual_seed(cols)
    begin = rows_of(G, T)
    group = torch.repeat_interleave(torch.arange(G, device=DEV), begin.diff())
    x = torch.randint(-8, 9, (T, 1), device=DEV, generator=g).to(dtype)
    w = torch.randint(-8, 9, (1, cols), device=DEV, generator=g).to(dtype)
    print("products of", T, "rows and", cols, "columns", dtype, flush=True)
    y = layers.product(x, w[:, :, None].expand(G, cols, 1), begin)
    for at in range(0, T, 512):
        assert torch.equal(y[at:at + 512], x[at:at + 512] * w)
    del y
    y = layers.product(x, w[:, None, :].expand(G, 1, cols), begin, transposed=True)
    for at in range(0, T, 512):
        assert torch.equal(y[at:at + 512], x[at:at + 512] * w)
    dw = layers.product_grad(x, y, begin)
    assert (dw[1] == 0).all()
    terms = x.float() * x.float()
    factor = torch.zeros(G, 1, device=DEV).index_add_(0, group, terms)
    for at in range(0, G, 512):
        assert torch.equal(dw[at:at + 512, 0], factor[at:at + 512] * w.float())
    del y, dw
    torch.cuda.empty_cache()
