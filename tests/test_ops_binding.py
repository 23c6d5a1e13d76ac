"""What the binding of the second part of libbart (paper_2410_23244_amd.ops)
checks by itself, without a GPU: the tensors are stand-ins that have a shape
and strides and no memory."""
from __future__ import annotations

from types import SimpleNamespace

import pytest
import torch

from paper_2410_23244_amd import ops
from paper_2410_23244_amd.bart import BartError


def _scores(n, c):
    return SimpleNamespace(shape=(n, c), dtype=torch.float16, is_cuda=True, dim=lambda: 2,
                           stride=lambda d: (c, 1)[d], data_ptr=lambda: 1 << 20, device="cuda:0")


@pytest.mark.parametrize("c", [0, 2 ** 30 + 1, 2 ** 31 + 5, 2 ** 32, 2 ** 32 + 5])
def test_numbers_of_classes_that_the_library_does_not_take(c):
    """A count that its 32-bit field would cut down to a valid one among them."""
    with pytest.raises(BartError):
        ops._rows(_scores(3, c), None, None, 1.0)


@pytest.mark.parametrize("c", [1, 7, 2 ** 30])
def test_numbers_of_classes_arrive_whole(c):
    r = ops._rows(_scores(3, c), None, None, 1.0)
    assert (r.n, r.n_class, r.ld) == (3, c, c)
