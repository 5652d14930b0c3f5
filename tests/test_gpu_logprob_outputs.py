"""The differentiable log probabilities' outputs changed in place, as a loss does
that leaves out padding: gradients as of the same change out of place."""
import pytest
import torch

from paper_2401_04829_amd import answers as A
from tests.gpu_util import require_gpu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [1, 70])
@pytest.mark.parametrize("kind", ["logits", "hidden"])
def test_outputs_can_be_changed_in_place(kind, rows):
    dev = require_gpu()
    print("in place", kind, rows, flush=True)
    gen = torch.Generator(dev).manual_seed(rows)
    h, w = (torch.randn((n, 32), generator=gen, device=dev) for n in (rows, 300))
    t = torch.randint(0, 300, (rows,), generator=gen, device=dev)
    pad = torch.arange(rows, device=dev) % 3 == 2

    def outputs(x):
        return A.differentiable_logprobs(x @ w.t(), t) if kind == "logits" else A.differentiable_linear_logprobs(x, w, t)

    def padded(logp, ent):
        return logp.masked_fill_(pad, 0.0).mul_(2.0)
    a, b, c = (h.clone().requires_grad_() for _ in range(3))
    padded(*outputs(a)).sum().backward()
    (2.0 * outputs(b)[0].masked_fill(pad, 0.0)).sum().backward()
    assert torch.equal(a.grad, b.grad)
    logp, ent = outputs(c)
    logp[0] = 0.0
    (logp.sum() + 0.1 * ent.sum()).backward()                # the entropy's is not touched by it
    assert bool(c.grad.isfinite().all()) and float(c.grad.abs().max()) > 0
    logp, ent = outputs(h.clone().requires_grad_())
    ent.zero_()                                              # the gradient reads the entropy: autograd says so
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        logp.sum().backward()
