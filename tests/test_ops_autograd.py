"""What torch's automatic differentiation sees of the operators: tensors that
they write in place count as modified, and gradients are handed to it by
backward()."""
from __future__ import annotations

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    from paper_2410_23244_amd import ops

    return ops


@pytest.mark.parametrize("dtype,masters", [(torch.float32, None), (torch.bfloat16, "new")])
def test_a_step_modifies_weights(ops, dtype, masters):
    w = torch.randn(50, device="cuda", dtype=dtype, requires_grad=True)
    opt = ops.AdamW([w, w.detach().clone()], [torch.ones_like(w.detach())] * 2, masters=masters)
    out = (w * w).sum()                                  # keeps w for its backward
    seen = [t for t in opt.params + opt.masters if t is not None]
    before = [t._version for t in seen]
    opt.step()
    assert all(t._version > v for t, v in zip(seen, before))
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        out.backward()


def test_gradients_in_place_modify_the_scores(ops):
    x = torch.randn(20, 30, device="cuda")
    label = torch.arange(20, device="cuda")
    one = torch.ones((), device="cuda")
    w = torch.randn(20, 30, device="cuda", requires_grad=True)
    out = (w * x).sum()                                  # keeps x
    r = ops.logprob(x, label, norm=True)
    version = x._version
    ops.logprob(x, label, grad_logp=one)
    assert x._version == version
    ops.logprob(x, label, grad_logp=one, grad_out=x)
    assert x._version > version
    version = x._version
    ops.logprob_grad(x, label, r.norm, one, grad_out=x)
    assert x._version > version
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        out.backward()


def test_tensors_made_in_inference_mode(ops):
    """Such tensors have no version."""
    with torch.inference_mode():
        p, g = torch.ones(9, device="cuda"), torch.ones(9, device="cuda")
        x = torch.randn(3, 9, device="cuda")
    ops.AdamW([p], [g]).step()
    assert (p < 1).all()
    label = torch.arange(3, device="cuda")
    r = ops.logprob(x, label, grad_logp=torch.ones((), device="cuda"), grad_out=x)
    assert r.grad.data_ptr() == x.data_ptr()


def test_gradients_go_on_by_backward(ops):
    """A layer's weights by scores.backward(r.grad), against torch's own loss: 4000
    terms of f32, and a product of matrices."""
    a = torch.randn(4000, 8, device="cuda")
    label = torch.randint(0, 5, (4000,), device="cuda")
    w = torch.randn(5, 8, device="cuda", requires_grad=True)
    scores = a @ w.t()
    r = ops.logprob(scores, label, grad_logp=torch.tensor(-1 / 4000, device="cuda"))
    assert not r.logp.requires_grad and not r.grad.requires_grad
    scores.backward(r.grad)
    v = w.detach().double().cpu().requires_grad_()
    torch.nn.functional.cross_entropy(a.double().cpu() @ v.t(), label.cpu()).backward()
    torch.testing.assert_close(w.grad.double().cpu(), v.grad, rtol=1e-5, atol=1e-6)
