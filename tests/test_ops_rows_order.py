"""Alternatives of rows whose large scores lie where a threshold from columns of
a row says nothing about them, against a sort.  The scores above any such
threshold come in the order in which a list of them is worst cut down."""
from __future__ import annotations

import math

import pytest
import torch

from tests.test_ops_rows import check

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    from paper_2410_23244_amd import ops

    return ops


def _rows(C, dtype, k, order, seed=0):
    """The classes are 64 (k > 40: 256) columns of 16 bytes; all large scores lie in
    k - 1 of them, rising or falling with the class, or in no order."""
    V = 4 if dtype == torch.float32 else 8
    columns = 64 if k <= 40 else 256
    ld = (C + 7) // 8 * 8
    g = torch.Generator(device="cuda").manual_seed(seed + C + k)
    buf = torch.empty((4, ld), device="cuda").normal_(generator=g)
    j = torch.arange(ld, device="cuda")
    hot = (j // V) % columns < k - 1
    at = j if order == "rising" else ld - j if order == "falling" else \
        torch.randperm(ld, device="cuda", generator=g)
    big = 20.0 + 40.0 * at.float() / ld
    buf[:3] = torch.where(hot, big, buf[:3])
    buf[1] = torch.where(hot, big.floor(), buf[1])       # runs of equal scores
    buf[2] = torch.where(hot & (j % 3 != 0), -big, buf[2])
    buf[3, C // 2] = math.nan                            # no alternatives at all
    return buf.to(dtype)[:, :C]


@pytest.mark.parametrize("order", ["rising", "falling", "mixed"])
@pytest.mark.parametrize("k", [2, 20, 41, 64])
@pytest.mark.parametrize("C", [1_000, 4_096, 9_000, 40_001, 140_001, 1_048_577])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_large_scores_in_fewer_than_k_columns(ops, dtype, C, k, order):
    check(ops, _rows(C, dtype, k, order), None, k=k)


@pytest.mark.parametrize("k", [20, 64])
@pytest.mark.parametrize("n,C", [(70, 100_001), (300, 33_001)])
def test_rows_that_are_not_split(ops, n, C, k):
    x = _rows(C, torch.bfloat16, k, "rising")[:1].expand(n, C).contiguous()
    r = ops.logprob(x, k=k, entropy=True)
    want = x[0].float().sort(descending=True, stable=True)[1][:k].int()
    assert (r.top_class == want).all()
