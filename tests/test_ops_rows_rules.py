"""Rows of class scores where several of the header's rules meet, against the
plain implementation in 64 bits of tests/test_ops_rows.py."""
from __future__ import annotations

import math

import pytest
import torch

from tests.test_ops_rows import check, make

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    from paper_2410_23244_amd import ops

    return ops


@pytest.mark.parametrize("C", [6, 50, 700, 9_000, 70_000])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_labels_past_the_last_class_without_a_weight(ops, C, dtype):
    """Such a label spoils the gradient through its weight alone: without one the
    row's gradient is that of the entropy, or 0."""
    x, label, w, h = make(8, C, dtype, seed=53, ignored=0.0)
    label[:6] = torch.tensor([C, C + 7, C, C, C, 2 ** 40])
    w[0] = w[1] = w[2] = 0.0
    w[3] = -0.0
    h[1] = h[3] = 0.0
    x[2, C // 2] = math.nan                              # h is not 0: NaN all the same
    x[3, 0] = math.nan                                   # nothing is asked of it: 0
    check(ops, x, label, k=2, w=w, h=h)
    check(ops, x, label, k=2, w=w)
