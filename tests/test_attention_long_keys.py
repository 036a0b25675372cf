"""A few queries on long keys whose rows are not aligned, against the 64-bit statement: many stages to a wavefront, last tiles of every size, heads that end inside of a chunk."""
import pytest

from test_attention import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [33, 64, 65, 100, 127, 128])
@pytest.mark.parametrize("nq,nk", [([1], [5000]), ([9], [2049]), ([2, 1, 3], [500, 1, 3001])])
def test_few_queries_on_long_keys(dtype, D, nq, nk):
    check(dtype, nq, nk, 2, 1, D, True, odd=True, grad=False)
    check(dtype, nq, nk, 3, 3, D, False, odd=True, grad=False)
