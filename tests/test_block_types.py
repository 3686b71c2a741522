"""What a tensor that has to be like another is refused with: TypeError for another type, ValueError
for another shape, as for the other arguments."""

import pytest
import torch

from paper_2601_17654_amd import binding as b

x = torch.zeros(2, 8)


@pytest.mark.parametrize("bad", [None, [1.0], 3, x.double(), x.half()])
def test_type(bad):
    with pytest.raises(TypeError, match="residual must be a tensor of torch.float32"):
        b._like(bad, x, "residual", "x")


@pytest.mark.parametrize("bad", [x[0], x[:1], x.reshape(4, 4), x[:0]])
def test_shape(bad):
    with pytest.raises(ValueError, match="residual must be like x"):
        b._like(bad, x, "residual", "x")


def test_taken():
    b._like(x.clone(), x, "residual", "x")
