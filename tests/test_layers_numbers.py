"""Arguments of the tensor calls that used to be ignored, or to raise what no caller expects."""
import pytest
import torch

from paper_1902_01064_amd import hop, layers

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def test_a_place_for_a_result_that_there_is_not():
    x = torch.ones(4, 8, device=DEV)
    with pytest.raises(ValueError, match="out_next"):
        layers.residual(x, x, out_next=torch.empty(4, 8, device=DEV))


@pytest.mark.parametrize("over", [dict(worker=1 << 31), dict(worker=-(1 << 31) - 1), dict(iter=1 << 40), dict(site=1 << 31), dict(first_row=1 << 63),
                                  dict(worker=0.5), dict(p="half")])
def test_numbers_that_a_draw_has_no_room_for(over):
    x = torch.ones(4, 8, device=DEV)
    drop = layers.Drop(0.5, 1)._replace(**over)
    for fn in (lambda: layers.dropout(x, drop), lambda: layers.residual(x, x, drop=drop), lambda: layers.residual_grad(x, None, None, x, drop=drop)):
        with pytest.raises(ValueError):
            fn()


@pytest.mark.parametrize("over", [dict(scale="one"), dict(eps=None)])
def test_what_is_no_number(over):
    x = torch.ones(4, 8, device=DEV)
    for fn in (lambda: layers.residual(x, x, **over), lambda: layers.residual_grad(x, None, None, x, **over)):
        with pytest.raises(ValueError):
            fn()


@pytest.mark.parametrize("over", [dict(scale=1e39), dict(eps=1e39), dict(drop=layers.Drop(1e39, 1))])
def test_numbers_of_over_32_bits(over):
    """Infinite for the library, which refuses them."""
    x = torch.ones(4, 8, device=DEV)
    for fn in (lambda: layers.residual(x, x, **over), lambda: layers.residual_grad(x, None, None, x, **over)):
        with pytest.raises(hop.HopError) as e:
            fn()
        assert e.value.code == hop.HOP_ERR_INVALID_ARG
