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


def _t(shape, strides):
    return torch.empty_strided(shape, strides)


@pytest.mark.parametrize("shape,strides", [
    ((), ()), ((0,), (1,)), ((0, 5), (5, 1)), ((5, 0), (1, 1)), ((5, 0, 3), (3, 3, 1)), ((1,), (9,)),
    ((3, 4), (4, 1)), ((3, 4), (1, 3)), ((3, 1, 4), (4, 77, 1)), ((2, 3, 5, 7), (105, 1, 21, 3))])
def test_dense_tensors(shape, strides):
    assert ops._dense(_t(shape, strides))


@pytest.mark.parametrize("shape,strides", [((3,), (2,)), ((3, 4), (5, 1)), ((3, 4), (0, 1)),
                                           ((2, 2), (1, 1))])
def test_tensors_with_gaps_or_shared_elements(shape, strides):
    assert not ops._dense(_t(shape, strides))


def test_layouts_are_compared_where_they_matter():
    """The stride of a dimension of size 1, or of an empty tensor, says nothing."""
    same = ops._same_layout
    assert same(_t((8, 3, 1, 1), (3, 1, 1, 1)), _t((8, 3, 1, 1), (3, 1, 3, 3)))
    assert same(_t((1, 6), (1, 1)), _t((1, 6), (6, 1)))
    assert same(_t((5, 0), (1, 1)), _t((5, 0), (7, 1)))
    assert not same(_t((3, 4), (4, 1)), _t((3, 4), (1, 3)))
    assert not same(_t((4, 3), (3, 1)), _t((3, 4), (4, 1)))
    assert not same(_t((5, 0), (1, 1)), _t((0, 5), (1, 1)))


def test_a_gradient_alone_needs_what_was_kept():
    with pytest.raises(BartError):
        ops.logprob_grad(_scores(3, 7), None, None, None)
