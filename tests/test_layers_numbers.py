"""Arguments of the tensor calls that used to be ignored, or to raise what no caller expects."""
import pytest
import torch

from paper_1902_01064_amd import layers

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def test_a_place_for_a_result_that_there_is_not():
    x = torch.ones(4, 8, device=DEV)
    with pytest.raises(ValueError, match="out_next"):
        layers.residual(x, x, out_next=torch.empty(4, 8, device=DEV))
