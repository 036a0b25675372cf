"""Rows as far apart as a call takes: the last rows of a tile are nearly 2^31 bytes behind the first one.  The same bits as with rows one behind the other."""
import pytest
import torch

from paper_1902_01064_amd import attention
from test_attention_use import made
from test_layers import DEV

pytestmark = pytest.mark.gpu
FAR = 1 << 22


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,hq,hk,D", [(300, 1, 1, 128), (200, 6, 2, 64), (8, 32, 1, 128)])
def test_rows_far_apart(dtype, rows, hq, hk, D):
    widths = dict(q=hq, k=hk, v=hk, do=hq, o=hq, dq=hq, dk=hk, dv=hk)
    wide = torch.empty((rows, FAR), dtype=torch.float32 if dtype == "f32" else torch.bfloat16, device=DEV)
    near = {name: made(i, rows, h * D, dtype) for i, (name, h) in enumerate(widths.items())}
    far, column = {}, FAR                                   # the last columns of the rows
    for name, h in widths.items():
        column -= h * D
        far[name] = wide[:, column:column + h * D]
        far[name].copy_(near[name])
    for t in (near, far):
        t["lse"] = attention.attention(t["q"], t["k"], t["v"], hq, hk, out=t["o"])[1]
        attention.attention_grad(t["do"], t["o"], t["lse"], t["q"], t["k"], t["v"], hq, hk, dq=t["dq"], dk=t["dk"], dv=t["dv"])
    for name in ("o", "lse", "dq", "dk", "dv"):
        assert torch.equal(near[name], far[name]), name
