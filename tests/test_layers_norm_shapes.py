"""A residual of another shape than x is refused, also where it has as many rows: they would be added in another order."""
import pytest

from paper_2505_23725_b200 import layers
from test_decoder_operators_host import Owner, rand


@pytest.mark.parametrize("x,residual", [((2, 3, 8), (3, 2, 8)), ((2, 3, 8), (6, 8)), ((4, 8), (1, 8)), ((4, 8), (8,))])
def test_residual_of_another_shape(x, residual):
    with pytest.raises(ValueError, match="residual must have the shape of x"):
        layers.layer_norm(Owner(), rand(*x), residual=rand(*residual))


def test_residual_of_the_same_shape():
    y, h = layers.layer_norm(Owner(), rand(2, 3, 8), residual=rand(2, 3, 8))
    assert y.shape == h.shape == (2, 3, 8)
