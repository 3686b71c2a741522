"""Held values that a graph is recorded of: their values, their product and a linear layer's held weight have no
gradient, and say so rather than leave the graph."""

import pytest
import torch

from paper_2601_17654_amd import binding as b


def held(track):
    q = torch.ones(4, 8).to(torch.float8_e4m3fn)
    return b.Scaled(q.requires_grad_(track), torch.zeros(1, 128, dtype=torch.uint8))


CALLS = {"values": lambda h, o: b.scaled_values(h), "matmul a": lambda h, o: b.scaled_matmul(h, o),
         "matmul b": lambda h, o: b.scaled_matmul(o, h),
         "linear": lambda h, o: b.scaled_linear(torch.ones(4, 8), h)}


@pytest.mark.parametrize("call", CALLS)
def test_refused(call):
    with pytest.raises(ValueError, match="has no gradient"):
        CALLS[call](held(True), held(False))
    # else the next thing is said, here that the tensors are not on the device
    with torch.no_grad(), pytest.raises(ValueError, match="on the current device"):
        CALLS[call](held(True), held(False))
    with pytest.raises(ValueError, match="on the current device"):
        CALLS[call](held(False), held(False))
