"""hop_residual and its gradient on many rows of over 8192 columns, where a workgroup holds two or four times eight columns a thread: pieces of
several rows, groups that end inside one, and none.  The comparison is test_layers.py's."""
import pytest

import test_layers as tl

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("norm,next_norm,gate,p", [("rms", "rms", "vector", 0.2), ("centred", "centred", "element", 0.0), ("rms", None, None, 0.3)])
@pytest.mark.parametrize("cols,counts", [(8200, [500, 0, 130]), (9001, [70, 3]), (16384, [210]), (20002, [65, 0, 1]), (32768, [9, 30])])
def test_wide_rows(dtype, norm, next_norm, gate, p, cols, counts):
    tl.test_residual_and_its_gradients(dtype, norm, next_norm, gate, p, cols, counts)
