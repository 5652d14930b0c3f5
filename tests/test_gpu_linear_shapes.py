"""Log probabilities from hidden states and their gradient against float64 at
sizes that reach every shape of the kernels' tiles, segments of the vocabulary
and several pieces of it (tests/test_linear_shapes.py says which).

Values, with D the width and root the largest root of a logit's sum of squared
products: a logit's error is that of as many additions as often up as down, at
most four times 2^-24 sqrt(D) root where 10^8 of them are looked at (their own is
a quarter of that: sqrt(D / 12) roundings of partial sums that grow up to root);
a log of a sum has 64 roundings of 2^-24 in its exponentials, parts and logarithm,
and each value its own.  An entropy's are those by (log V + 2), which its
derivative by the logits, p (log p + H), is at most in all.  Gradients: as
test_gpu_linear_precision.py derives.
"""
import math

import pytest
import torch

from paper_2401_04829_amd import answers as A
from tests import linear_shapes as S
from tests.gpu_util import require_gpu
from tests.test_gpu_linear_precision import check, exact, inputs, rms

pytestmark = pytest.mark.gpu


def _types(element):
    return [torch.float32] if element == 4 else [torch.float16, torch.bfloat16]


def _values(h, w, t, part=512):
    """Log probabilities, entropies and lse in float64, some rows at a time."""
    w64, out = w.double(), []
    for b in range(0, h.shape[0], part):
        x = h[b:b + part].double() @ w64.t()
        logp = torch.log_softmax(x, 1)
        out.append(torch.stack([logp.gather(1, t[b:b + part, None].clamp(min=0))[:, 0] * (t[b:b + part] >= 0),
                                -(logp.exp() * logp).sum(1), torch.logsumexp(x, 1)]))
    return torch.cat(out, 1)


@pytest.mark.parametrize("dtype,rows,vocab,width", [(d, *s[1:]) for s in S.SIZES for d in _types(s[0])])
def test_every_shape(dtype, rows, vocab, width):
    dev = require_gpu()
    print("shapes", dtype, rows, vocab, width, flush=True)
    h, w, t, gl, ge = inputs(dev, dtype, rows, vocab, width, 0.1)
    t[1::7] = vocab - 1 - torch.arange(rows, device=dev)[1::7] % min(vocab, 600)   # in the last tiles too
    r = A.linear_logprobs(h, w, t)
    ref = exact(h, w, t, gl, ge)
    logit = 2.0 ** -24 * (4 * math.sqrt(width) * ref[4] + 64)
    for got, want, by in zip((r.logprob, r.entropy, r.lse), _values(h, w, t), (1, math.log(vocab) + 2, 1)):
        assert bool(((got.double() - want).abs() <= by * logit + 2.0 ** -22 * want.abs()).all())
    got = A.linear_logprobs_backward(h, w, t, r.maximum, r.log_sum, r.entropy, gl, ge)
    check(got, ref, dtype, width)
    again = A.linear_logprobs_backward(h, w, t, r.maximum, r.log_sum, r.entropy, gl, ge)
    assert all(torch.equal(a, b) for a, b in zip(got, again))


def test_long_sums_in_fp32():
    """Partial sums of n terms of like size grow as sqrt(k), and an addition is off by
    0.7 2^-24 / sqrt(3) of its sum (a half unit at most, by where in its binade the
    sum lies): 0.4 2^-24 sqrt(n / 2), 0.29 2^-24 sqrt(n) of the sum in one chain, and
    in eight chains 0.10.  The logits are exact (elements are multiples of 1/2 and
    1/16), so that a term is off by its row's log of a sum, its exponential and its
    argument of up to 16, 8 2^-24: sqrt(10^2 + 8^2) = 13 of the 15.6 2^-24 that 0.16
    2^-24 sqrt(n) is at 9,531 rows, where one chain would have 28."""
    dev = require_gpu()
    _, rows, vocab, width = S.LONG_SUM
    gen = torch.Generator(dev).manual_seed(rows)
    h = torch.randint(-2, 3, (rows, width), generator=gen, device=dev) / 2.0
    w = torch.randint(-4, 5, (vocab, width), generator=gen, device=dev) / 16.0
    gl = torch.randn(rows, generator=gen, device=dev)
    t = torch.zeros(rows, dtype=torch.int64, device=dev)      # token 0 stands out, no term of the others
    r = A.linear_logprobs(h, w, t)
    got = A.linear_logprobs_backward(h, w, t, r.maximum, r.log_sum, r.entropy, gl, None, of_hidden=False)[1][1:]
    want = exact(h, w, t, gl, torch.zeros_like(gl))[2][1:]
    off = float((rms(got.double() - want) / rms(want)).square().mean().sqrt())
    print("long sums", off * 2.0 ** 24, math.sqrt(rows), flush=True)
    assert off <= 2.0 ** -24 * 0.16 * math.sqrt(rows)
