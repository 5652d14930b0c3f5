"""How exact the gradients of log probabilities from hidden states are, against
float64, row by row: beside the rounding of the results to their type there is
room only for what fp32 sums leave.

The root mean square of a row's errors is at most 1.3 times that of rounding
the exact row (256 elements and more: their mean square is off by a tenth at
most) and, beside that, of `rest` times the terms' sizes s |w| (s^T |h|), s_j =
|g| (1[j = t] + p_j) + |g_H| p_j (|log p_j| + H) (not |d_j|: a relative error of
p_j is one of these parts of d_j, however much 1 - p_j or log p_j + H cancel).
rest, with u the type's half unit, D the width and n the terms of a sum:
  - d in two parts of a 16-bit type: u^2;
  - a logit's sum of D products: 2^-24 sqrt(D) of the products' root sum of
    squares (errors of additions are as often up as down), which enters p
    directly and by lse, so twice;
  - an exponential, its argument, the difference in d: 2^-24 16;
  - the sum over n terms: 2^-24 sqrt(n).
"""
import math

import pytest
import torch

from paper_2401_04829_amd import answers as A
from tests.gpu_util import require_gpu

HALF = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}


def inputs(device, dtype, rows, vocab, width, common, seed=1):
    """Hidden states and weights of which `common` is in all rows of either, tokens and incoming gradients."""
    gen = torch.Generator(device).manual_seed(seed + rows + 7 * vocab + 13 * width)
    h = torch.randn((rows, width), generator=gen, device=device)
    h = (h + 4 * common * torch.randn(width, generator=gen, device=device)).to(dtype)
    w = 2 / math.sqrt(width) * torch.randn((vocab, width), generator=gen, device=device)
    w = (w + common * torch.randn(width, generator=gen, device=device)).to(dtype)
    t = torch.randint(0, vocab, (rows,), generator=gen, device=device)
    t[::5] = -1
    gl, ge = (torch.randn(rows, generator=gen, device=device) for _ in range(2))
    return h, w, t, gl, 0.3 * ge


def exact(h, w, t, gl, ge, part=512):
    """Gradients in float64 with their terms' sizes and the logits' root sums of squares, some rows at a time."""
    w64, w2 = w.double(), w.double().square()
    gl = gl.double() * (t >= 0)
    dh, dh_size, dw, dw_size, root = [], [], 0.0, 0.0, 0.0
    for b in range(0, h.shape[0], part):
        rows = slice(b, b + part)
        x = h[rows].double()
        logp = torch.log_softmax(x @ w64.t(), 1)
        p = logp.exp()
        ent = -(p * logp).sum(1, keepdim=True)
        d = -p * (gl[rows, None] + ge[rows, None].double() * (logp + ent))
        at = torch.arange(x.shape[0], device=h.device)
        d[at, t[rows].clamp(min=0)] += gl[rows]
        s = p * (gl[rows, None].abs() + ge[rows, None].abs().double() * (logp.abs() + ent))
        s[at, t[rows].clamp(min=0)] += gl[rows].abs()
        root = max(root, float((x.square() @ w2.t()).max().sqrt()))
        dh.append(d @ w64)
        dh_size.append(s @ w64.abs())
        dw = dw + d.t() @ x
        dw_size = dw_size + s.t() @ x.abs()
    return torch.cat(dh), torch.cat(dh_size), dw, dw_size, root


def rms(x):
    return x.square().mean(1).sqrt()


def excess(got, want, size, dtype, width, terms, root):
    """The largest of the rows' errors, by what is allowed."""
    u = HALF[dtype]
    rest = (u * u if dtype != torch.float32 else 0.0) + 2.0 ** -24 * (2 * math.sqrt(width) * root + 16 + math.sqrt(terms))
    rounded = rms(want.to(dtype).double() - want)
    allowed = ((1.3 * rounded).square() + (rest * rms(size)).square()).sqrt().clamp(min=1e-300)   # (rows of zeros)
    return float((rms(got.double() - want) / allowed).max())


def check(got, ref, dtype, width):
    dh, dh_size, dw, dw_size, root = ref
    assert excess(got[0], dh, dh_size, dtype, width, dw.shape[0], root) <= 1
    assert excess(got[1], dw, dw_size, dtype, width, dh.shape[0], root) <= 1


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("common", [0.0, 0.1, 0.5])
@pytest.mark.parametrize("rows,vocab,width", [(100, 2000, 256), (128, 2000, 256), (129, 2000, 256), (256, 2000, 256),
                                              (300, 5000, 512), (1030, 3001, 260), (3000, 65, 256), (1500, 4001, 301)])
def test_16_bit_gradients_are_rounded_once(rows, vocab, width, common, dtype):
    """Weights (and hidden states) that share a vector cancel in the gradients'
    sums, and what d's rounding took from each term would not."""
    dev = require_gpu()
    print("rounded once", dtype, rows, vocab, width, common, flush=True)
    h, w, t, gl, ge = inputs(dev, dtype, rows, vocab, width, common)
    r = A.linear_logprobs(h, w, t)
    got = A.linear_logprobs_backward(h, w, t, r.maximum, r.log_sum, r.entropy, gl, ge)
    check(got, exact(h, w, t, gl, ge), dtype, width)
    lone = A.linear_logprobs_backward(h, w, t, r.maximum, r.log_sum, None, gl, None)
    check(lone, exact(h, w, t, gl, torch.zeros_like(ge)), dtype, width)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("common", [0.0, 0.5])
def test_the_check_tells_one_part_from_two(dtype, common):
    """The check above, on gradients made in torch with d rounded once and in two parts."""
    h, w, t, gl, ge = inputs("cpu", dtype, 129, 2000, 256, common)
    ref = exact(h, w, t, gl, ge)
    x = h.float() @ w.float().t()
    logp = torch.log_softmax(x, 1)
    p = logp.exp()
    ent = -(p * logp).sum(1, keepdim=True)
    gl = gl * (t >= 0)
    d = -p * (gl[:, None] + ge[:, None] * (logp + ent))
    d[torch.arange(129), t.clamp(min=0)] += gl
    scale = 2.0 ** 12 if dtype == torch.float16 else 1.0       # as large as fp16 holds, so that none of it is lost
    first = (d * scale).to(dtype).float()
    second = (d * scale - first).to(dtype).float()
    two = (first + second) / scale
    check(((two @ w.float()).to(dtype), (two.t() @ h.float()).to(dtype)), ref, dtype, 256)
    with pytest.raises(AssertionError):
        one = first / scale
        check(((one @ w.float()).to(dtype), (one.t() @ h.float()).to(dtype)), ref, dtype, 256)
