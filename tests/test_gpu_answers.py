"""The operators of token models together: the example's Shapley values
against the oracle's least squares on values from a float64 model, efficiency,
and the gradient through autograd."""
import math
import os
import sys

import numpy as np
import pytest
import torch

from oracle import sampler, wls
from paper_2401_04829_amd import answers as A
from tests.gpu_util import require_gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import answer_tokens  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    return require_gpu()


def _turn(x, cos, sin):
    a, b = x.chunk(2, -1)
    return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)


def _values64(model, tokens, instruction, masks, answer):
    """The coalitions' values in float64 on the CPU, with no cache and no code of the library."""
    d = torch.float64
    W = [{k: v.cpu().to(d) for k, v in b.items()} for b in model.blocks]
    embed, head, cos, sin = (x.cpu().to(d) for x in (model.embed, model.head, model.cos, model.sin))
    H, K, D = model.heads, model.kv_heads, model.dim

    def norm(x):
        return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6)

    def attend(q, k, v, seen):                                    # [n, H, D], [m, H, D], [n, m]
        s = (torch.einsum("nhd,mhd->hnm", q, k) / math.sqrt(D)).masked_fill(~seen[None], -math.inf)
        return torch.einsum("hnm,mhd->nhd", torch.softmax(s, -1), v)

    def mlp(x, a, w):
        x = x + a.flatten(1) @ w["out"]
        up, gate = (norm(x) @ w["up"]).chunk(2, 1)
        return x + (torch.nn.functional.silu(up) * gate) @ w["down"]
    t = tokens.cpu()
    n = t.numel() - 1
    causal = torch.tril(torch.ones((n, n), dtype=torch.bool))
    x, prompt = embed[t[:n]], []
    for w in W:
        q, k, v = (norm(x) @ w["qkv"]).view(n, -1, D).split([H, K, K], 1)
        q, k = (_turn(y, cos[:n, None], sin[:n, None]) for y in (q, k))
        k, v = k.repeat_interleave(H // K, 1), v.repeat_interleave(H // K, 1)
        prompt.append((k, v))
        x = mlp(x, attend(q, k, v, causal), w)
    rows = masks.shape[0]
    seen = torch.cat([torch.ones((rows, instruction), dtype=torch.bool), masks], 1)
    x = embed[t[n]].expand(rows, -1)
    for w, (k, v) in zip(W, prompt):
        q, k1, v1 = (norm(x) @ w["qkv"]).view(rows, -1, D).split([H, K, K], 1)
        q, k1 = (_turn(y, cos[n], sin[n]) for y in (q, k1))
        k1, v1 = k1.repeat_interleave(H // K, 1), v1.repeat_interleave(H // K, 1)
        s = torch.cat([torch.einsum("nhd,mhd->nhm", q, k).masked_fill(~seen[:, None], -math.inf),
                       (q * k1).sum(-1, keepdim=True)], 2) / math.sqrt(D)
        p = torch.softmax(s, -1)
        x = mlp(x, torch.einsum("nhm,mhd->nhd", p[..., :-1], v) + p[..., -1:] * v1, w)
    return torch.log_softmax(norm(x) @ head, 1)[:, answer]


@pytest.mark.parametrize("tokens,samples", [(40, 600), (150, 1000)])
def test_answer_explanation_against_float64(dev, tokens, samples):
    """In float32 a value is a chain of some 40 sums of at most 1,000 terms and
    functions of slope near 1, so within 1e-4 of float64's; phi within 1e-3 of
    its largest, as for the graph models."""
    print("answer", tokens, samples, flush=True)
    model = answer_tokens.Decoder(dtype=torch.float32, device=dev)
    t = torch.randint(0, 1000, (tokens,), generator=torch.Generator(dev).manual_seed(3), device=dev)
    e, answer, full = answer_tokens.explain(model, t, samples=samples, batch=256)
    M = tokens - 1 - 4
    pl = sampler.plan(M, samples)
    masks, w = sampler.sample(pl, 7, 0)
    np.testing.assert_array_equal(e.masks.cpu().numpy().view(np.uint64), sampler.pack(masks))
    both = np.concatenate([masks.astype(bool), np.zeros((1, M), bool), np.ones((1, M), bool)])
    y = _values64(model, t, 4, torch.from_numpy(both), int(answer)).numpy()
    scale = np.abs(y[-2:]).max()
    assert np.abs(e.y.cpu().numpy() - y[:-2]).max() <= 1e-4 * scale
    assert np.abs(e.f_empty_full.cpu().numpy() - y[-2:]).max() <= 1e-4 * scale
    assert abs(float(full.top_logprob[0, 0]) - y[-1]) <= 1e-4 * scale
    assert int(e.info) == 0
    phi = wls.kernel_shap(masks, w, y[:-2], y[-2], y[-1])
    assert np.abs(e.phi.cpu().numpy() - phi).max() <= 1e-3 * np.abs(phi).max()
    assert abs(float(e.phi.double().sum()) - (float(e.f_empty_full[1]) - float(e.f_empty_full[0]))) <= 1e-4 * scale


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_answer_explanation_in_16_bits(dev, dtype):
    """Sampled masks over a shared prompt in a 16-bit model: the efficiency
    axiom holds of whatever values the model has."""
    model = answer_tokens.Decoder(dtype=dtype, device=dev, dim=64, layers=1)
    t = torch.randint(0, 1000, (90,), generator=torch.Generator(dev).manual_seed(4), device=dev)
    e, _, full = answer_tokens.explain(model, t, samples=1000, batch=512)
    assert int(e.info) == 0 and bool(e.y.isfinite().all())
    d = float(e.f_empty_full[1] - e.f_empty_full[0])
    assert abs(float(e.phi.double().sum()) - d) <= 1e-4 * float(e.f_empty_full.abs().max())
    assert float(full.top_logprob[0, 0]) == float(full.top_logprob.max())


def test_explainer_checks_its_values(dev):
    with pytest.raises(ValueError):
        A.AnswerExplainer(lambda masks, m: masks.float(), dev).explain(10, 100, 1)
    with pytest.raises(ValueError):
        A.AnswerExplainer(None, dev, batch=1)


def test_gradient_through_autograd(dev):
    """Against torch's own log_softmax in float64."""
    gen = torch.Generator(dev).manual_seed(5)
    x = torch.randn((7, 301), generator=gen, device=dev, requires_grad=True)
    t = torch.randint(0, 301, (7,), generator=gen, device=dev)
    lp, ent = A.differentiable_logprobs(x, t)
    (2 * lp.sum() - 0.3 * (ent * torch.arange(7, device=dev)).sum()).backward()
    y = x.detach().double().requires_grad_()
    logp = torch.log_softmax(y, 1)
    e = -(logp.exp() * logp).sum(1)
    (2 * logp.gather(1, t[:, None]).sum() - 0.3 * (e * torch.arange(7, device=dev)).sum()).backward()
    assert float((x.grad.double() - y.grad).abs().max()) <= 2.0 ** -20 * 8 * 4


def test_last_batch_ends_with_the_empty_and_the_full_coalition(dev):
    """Whatever the number of rows leaves over; and the batches do not change what comes out."""
    want = None
    for batch in (16384, 2, 3, 17, 33, 100):
        parts = []

        def value(masks, m):
            parts.append(masks)
            return masks[:, 0].float()
        e = A.AnswerExplainer(value, dev, batch=batch).explain(10, 98, 1)
        assert all(p.shape[0] <= batch for p in parts)
        assert parts[-1].shape[0] >= 2 and parts[-1][-2:, 0].tolist() == [0, 1023]
        got = torch.cat(parts), e.y, e.f_empty_full, e.phi
        want = got if want is None else want
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert {(got[0].shape[0]) % b == 1 for b in (2, 3, 17, 33, 100)} == {False, True}
