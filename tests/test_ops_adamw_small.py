"""AdamW steps whose second moments lie below the normal range of f32
(paper_2410_23244_amd.ops.AdamW with 32-bit states) against the formulas in 64
bits."""
from __future__ import annotations

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
LEAST = 2.0 ** -149                        # the spacing of f32 below 2^-126
B1, B2, LR = 0.9, 0.999, 1e-2


@pytest.fixture(scope="module")
def ops():
    from paper_2410_23244_amd import ops

    return ops


@pytest.mark.parametrize("pdt,gdt", [(torch.float32, torch.float32),
                                     (torch.bfloat16, torch.float32)])
@pytest.mark.parametrize("n", [1, 4_099, 9_000])
@pytest.mark.parametrize("every", [1, 7])
def test_tiny_second_moments(ops, pdt, gdt, n, every):
    """Gradients of 1e-21 to 1e-16, every one of them or one in seven beside ordinary
    ones, and an eps far below their roots.  v is a sum of two products, each
    rounded by half a spacing besides 6 u of itself; the root halves that share,
    and the update passes a root, a reciprocal, two sums and three products."""
    rng = np.random.default_rng([2410, 23244, 61, n])
    g = np.where(np.arange(n) % every == 0, 10.0 ** rng.uniform(-21, -16, n),
                 1e-2 * rng.normal(size=n)).astype(np.float32)
    grad = torch.from_numpy(g).cuda().to(gdt)
    g64 = grad.double().cpu().numpy()
    p = torch.zeros(n, dtype=pdt, device="cuda")
    master = [torch.zeros(n, device="cuda")] if pdt != torch.float32 else None
    eps = 1e-36
    opt = ops.AdamW([p], [grad], lr=LR, betas=(B1, B2), eps=eps, masters=master)
    w, m, v = np.zeros(n), np.zeros(n), np.zeros(n)
    e_w, e_v = np.zeros(n), np.zeros(n)
    for t in range(1, 4):
        opt.step()
        m = B1 * m + (1 - B1) * g64
        v = B2 * v + (1 - B2) * g64 ** 2
        e_v += 6 * U * v + 2 * LEAST
        root = np.sqrt(v / (1 - B2 ** t))
        up = LR / (1 - B1 ** t) * m / (root + eps)
        w = w - up
        # relative: of v halved by the root where v is larger than its error
        rel = np.where(v > 4 * e_v, e_v / np.where(v > 0, v, 1.0), np.inf)
        e_w += np.abs(up) * (rel + 24 * U) + 4 * U * np.abs(w)
        got = (master[0] if master else p).double().cpu().numpy()
        ok = np.isfinite(e_w)
        assert (np.abs(got - w) <= e_w)[ok].all(), (t, np.abs(got - w)[ok].max())
        assert np.isfinite(got).all()
        assert (np.abs(opt.state[0]["v"].double().cpu().numpy() - v) <= e_v).all()
    assert n < 100 or (ok & (v < 2.0 ** -126)).sum() > n / (3 * every)   # tiny ones among them


@pytest.mark.parametrize("bits", [32, 8])
def test_empty_tensors_and_dimensions_of_size_one(ops, bits):
    """A 1 x 1 convolution's weights and their gradients are of one layout whatever
    the strides of the two last dimensions say; a tensor without elements is dense."""
    def conv(x):
        return torch.as_strided(x.clone(), (8, 3, 1, 1), (3, 1, 3, 3))

    w, g = torch.randn(24, device="cuda"), torch.randn(24, device="cuda")
    a = [torch.as_strided(w.clone(), (8, 3, 1, 1), (3, 1, 1, 1)), torch.empty(5, 0, device="cuda")]
    b = [w.clone()]
    ops.AdamW(a, [conv(g), torch.empty(5, 0, device="cuda")], state_bits=bits).step()
    ops.AdamW(b, [g], state_bits=bits).step()
    assert torch.equal(a[0].reshape(-1), b[0]) and not torch.equal(b[0], w)


@pytest.mark.parametrize("kw", [dict(grad_scale=1e39), dict(grad_scale=-1e300), dict(lr=1e39)])
def test_rates_that_32_bits_do_not_hold(ops, kw):
    """Infinite there, such a factor makes NaN of every gradient of 0."""
    from paper_2410_23244_amd.bart import BartError

    p, g = torch.ones(5, device="cuda"), torch.zeros(5, device="cuda")
    opt = ops.AdamW([p], [g])
    with pytest.raises(BartError):
        opt.step(**kw)
    assert opt.steps == 0
    opt.step(grad_scale=3e38)
    assert (p == 1).all()
