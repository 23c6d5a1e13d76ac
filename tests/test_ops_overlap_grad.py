"""Where a gradient may lie beside the scores it is taken of (bart_ops.h)."""
from __future__ import annotations

import os

import pytest
import torch

from paper_2410_23244_amd import bart, ops

P = 1 << 24


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(bart.LIB_PATH):
        pytest.skip("libbart.so not built")
    return ops.lib()


def _taken(L, n, C, ld, at, ld_grad):
    """Whether the library takes a gradient `at` elements from the scores: a valid call
    over these few long rows needs a workspace, an invalid one none."""
    r = ops.Rows(P, n, ld, C, ops.BART_F32, P // 2, 1, None, 0, 1.0)
    g = ops.RowsGrad(P // 4, 1, None, 0, P + 4 * at, ld_grad)
    o = ops.RowsOut(P // 8, None, None, 0, None, None)
    return L.bart_logprob_workspace_bytes(r, o, g) > 0


C = 200_000


@pytest.mark.parametrize("at", [C, -C, C + 500_000, -C - 500_000, 7 * 500_000, 1_500_000,
                                500_000 - C, -1_500_000])
def test_rows_that_lie_between_each_other(L, at):
    """Equal strides, each row of the gradient in a gap between rows of scores."""
    r = at % 500_000
    assert C <= r <= 500_000 - C or abs(at) >= 3 * 500_000
    assert _taken(L, 3, C, 500_000, at, 500_000)


@pytest.mark.parametrize("at,ld_grad", [(1, 500_000), (-1, 500_000), (C - 1, 500_000),
                                        (1 - C, 500_000), (300_001, 500_000), (500_000, 500_000),
                                        (-500_000, 500_000), (500_000 - C + 1, 500_000),
                                        (C, 500_001), (C, 400_000), (-C, 600_000)])
def test_rows_that_share_places(L, at, ld_grad):
    assert not _taken(L, 3, C, 500_000, at, ld_grad)


@pytest.mark.parametrize("at", [C, -C, 0])
def test_one_row(L, at):
    assert _taken(L, 1, C, 0, at, C)


@pytest.mark.gpu
@pytest.mark.parametrize("n,C", [(40, 10), (9, 1_000), (7, 5_001), (5, 40_001), (3, 70_001)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
@pytest.mark.parametrize("first", [True, False])
def test_gradients_beside_their_scores(n, C, dtype, first):
    """Scores and gradient as the two halves of one buffer's rows."""
    g = torch.Generator(device="cuda").manual_seed(C)
    buf = torch.empty(n, 2 * C + 3, device="cuda").normal_(generator=g).to(dtype)
    a, b = buf[:, :C], buf[:, C + 3:]
    x, out = (a, b) if first else (b, a)
    label = torch.randint(0, C, (n,), device="cuda", generator=g)
    w = torch.randn(n, device="cuda", generator=g)
    want = ops.logprob(x.contiguous(), label, grad_logp=w, norm=True)
    before, gap = x.clone(), buf[:, C:C + 3].clone()
    ops.logprob(x, label, grad_logp=w, grad_out=out)
    near = dict(rtol=1e-5, atol=1e-6) if dtype == torch.float32 else dict(rtol=2e-3, atol=1e-6)
    torch.testing.assert_close(out, want.grad, **near)
    assert torch.equal(x, before) and torch.equal(buf[:, C:C + 3], gap)
    out.fill_(0)
    ops.logprob_grad(x, label, want.norm, w, grad_out=out)
    torch.testing.assert_close(out, want.grad, **near)
    assert torch.equal(x, before) and torch.equal(buf[:, C:C + 3], gap)
