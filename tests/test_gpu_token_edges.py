"""Inputs at the edges of the token operators' ranges, against plain
implementations in float64."""
import math

import pytest
import torch

from paper_2401_04829_amd import answers as A
from tests.gpu_util import require_gpu

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.float16, torch.bfloat16]


@pytest.fixture(scope="module")
def dev():
    return require_gpu()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab,top", [(1, 1), (2, 2), (41, 41), (64, 64), (65, 64), (200, 64), (257, 64), (5001, 64)])
def test_alternatives_of_rows_with_nan_are_tokens(dev, dtype, vocab, top):
    """NaN at token 0, at the last token, everywhere: the alternatives are
    different tokens of the vocabulary, however many are asked for."""
    print("nan", dtype, vocab, top, flush=True)
    x = torch.randn((4, vocab), generator=torch.Generator(dev).manual_seed(vocab), device=dev).to(dtype)
    x[0, 0] = math.nan
    x[1, -1] = math.nan
    x[2] = math.nan
    x[3], x[3, 0] = -math.inf, math.nan
    r = A.token_logprobs(x, torch.zeros(4, dtype=torch.int64, device=dev), top)
    for ids in r.top_id.tolist():
        assert all(0 <= i < vocab for i in ids) and len(set(ids)) == top, ids
    assert bool(r.top_logprob.isnan().all()) and bool(r.lse.isnan().all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,share,shared,own", [(1, 1, 0, 2048), (3, 5, 0, 700), (1, 4, 2048, 0), (260, 20, 0, 1100),
                                                   (64, 4, 2048, 0), (33, 1, 900, 20), (5, 2, 900, 20), (1, 1, 200, 33)])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_small_weights_are_not_lost(dev, dtype, dim, rows, share, shared, own):
    """The first of n keys has score 0 and value 0, the others score -25.5
    (in powers of two) and value 1,024, so that only small weights give the
    output, o = 1024 w / (1 + w) with w = (n - 1) 2^-25.5.  In fp16 a weight
    times 2^14 is a normal number and off by 2^-11 relative, in bf16 by 2^-8;
    the exponent is off by 2^-19, sums by (n + 32) 2^-24; then one rounding.
    The lse is within 2^-22 of log(1 + w) by a sum of (n + 32) additions."""
    print("small weights", dtype, dim, rows, share, shared, own, flush=True)
    page, kv, n = 16, 2, shared + own
    per_s, per_o = -(-shared // page), -(-own // page)
    k = torch.zeros((per_s + rows * per_o, page, kv, dim), dtype=dtype, device=dev)
    v = torch.full_like(k, 1024.0)
    k[..., 0] = -25.5
    first = torch.zeros(1, dtype=torch.int64, device=dev) if shared else per_o * torch.arange(rows, device=dev)
    k[first, 0, :, 0] = 0.0
    v[first, 0] = 0.0
    cache = A.PagedCache(k, v)
    q = torch.zeros((rows, kv * share, dim), dtype=dtype, device=dev)
    q[..., 0] = 1.0
    i32 = dict(dtype=torch.int32, device=dev)
    a = {}
    if own:
        a = dict(table=per_s + torch.arange(rows * per_o, **i32).view(rows, per_o), lengths=torch.full((rows,), own, **i32))
    if shared:
        a |= dict(shared_table=torch.arange(per_s, **i32)[None], shared_lengths=torch.full((1,), shared, **i32))
    out, lse = A.attend(cache, q, scale=math.log(2.0), return_lse=True, **a)
    w = (n - 1) * 2.0 ** -25.5
    want = 1024 * w / (1 + w)
    u = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}[dtype]
    tol = want * (2 * u + 2.0 ** -18 + (n + 32) * 2.0 ** -24)
    assert float((out.double() - want).abs().max()) <= tol
    assert float((lse.double() - math.log1p(w)).abs().max()) <= 2.0 ** -22 + (n + 32) * 2.0 ** -24


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("offset", [0.0, -300.0, 20000.0])
@pytest.mark.parametrize("rows,vocab", [(5, 41), (3, 301), (2, 1000), (3, 5001), (2, 70001), (4100, 3001)])
def test_gradient_of_logits_far_from_zero(dev, dtype, offset, rows, vocab):
    """Through autograd, against the gradient from log_softmax in float64.  log
    p is (x - max) - log s, off by 2^-23 (|log p| + 1) and by log s, whose sum
    has at most 64 + vocab / 1024 fp32 additions in a row and exponentials off by
    2^-22 of (1 + their average distance from the maximum, under log(vocab) + 2);
    p by as much relative, the entropy by that times log(vocab) + 2.  Nothing of
    it grows with the logits' offset."""
    print("far", dtype, offset, rows, vocab, flush=True)
    gen = torch.Generator(dev).manual_seed(vocab)
    x = (2 * torch.randn((rows, vocab), generator=gen, device=dev) + offset).to(dtype).requires_grad_()
    t = torch.randint(0, vocab, (rows,), generator=gen, device=dev)
    gl, ge = (torch.randn(rows, generator=gen, device=dev) for _ in range(2))
    logp, entropy = A.differentiable_logprobs(x, t)
    ((logp * gl).sum() + (entropy * ge).sum()).backward()
    y = x.detach().double()
    lp = torch.log_softmax(y, 1)
    p, ent = lp.exp(), -(lp.exp() * lp).sum(1, keepdim=True)
    a, b = gl.double()[:, None], ge.double()[:, None]
    hit = torch.arange(vocab, device=dev) == t[:, None]
    want = a * (hit.double() - p) - b * p * (lp + ent)
    lg = math.log(vocab) + 2
    off = 2.0 ** -23 * (lp.abs() + 1) + 2.0 ** -24 * (64 + vocab / 1024 + 4 * lg)
    u = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}[dtype]
    tol = u * want.abs() + 2 * off * p * (a.abs() + b.abs() * (lp.abs() + ent + 1)) + off * p * b.abs() * lg \
        + 2.0 ** -23 * (a.abs() * hit + p * (a.abs() + b.abs() * (lp.abs() + ent))) + 2.0 ** -25 * (dtype == torch.float16) + 1e-37
    d = (x.grad.double() - want).abs()
    assert bool((d <= tol).all()), float((d / tol).max())


def test_maximum_and_log_sum(dev):
    """The largest logit itself; -inf and 0 of a row of nothing; NaN where a row has one; for every length of rows."""
    for vocab in (1, 41, 200, 1000, 3001, 131072):
        x = torch.randn((7, vocab), generator=torch.Generator(dev).manual_seed(vocab), device=dev) + 1000
        x[1] = -math.inf
        x[2, 0] = math.nan
        x[3, vocab // 2] = math.inf
        x[5] = math.nan
        x[6], x[6, -1] = -math.inf, math.nan
        m, s = torch.full((2, 7), 7.0, device=dev).unbind(0)
        r = A.token_logprobs(x, torch.zeros(7, dtype=torch.int64, device=dev), min(vocab, 3), maximum=m, log_sum=s)
        assert torch.equal(m[[0, 1, 4]], x[[0, 1, 4]].amax(1)) and float(s[1]) == 0 and bool(s[[2, 3, 5, 6]].isnan().all())
        want = torch.log(torch.exp(x.double() - x.double().amax(1, keepdim=True)).sum(1))
        assert float((s.double() - want)[[0, 4]].abs().max()) <= 2.0 ** -23 * (64 + vocab / 1024 + 4 * (math.log(vocab) + 2))
        assert torch.equal(r.lse[[0, 1, 4]], (m + s)[[0, 1, 4]])
        one = torch.ones(7, device=dev)
        g = A.token_logprobs_backward(x, None, None, r.entropy, None, one, maximum=m, log_sum=s)
        assert bool((g[1] == 0).all()) and bool(g[[2, 3, 5, 6]].isnan().all())


def test_one_logit_far_above_the_longest_row(dev):
    """2^30 equal logits and one 2^101 above them: its probability is 1, entropy and log probability 0."""
    x = torch.zeros((1, 2 ** 30), dtype=torch.bfloat16, device=dev)
    for at in (0, 5, 2 ** 29 + 77, 2 ** 30 - 1):
        x[0, at] = 2.0 ** 101
        r = A.token_logprobs(x, torch.tensor([at], device=dev), 2)
        assert float(r.entropy) == 0 and float(r.logprob) == 0 and int(r.rank) == 0 and int(r.top_id[0, 0]) == at
        r = A.token_logprobs(x)
        assert float(r.entropy) == 0 and float(r.lse) == 2.0 ** 101
        x[0, at] = 0
    r = A.token_logprobs(x)
    assert abs(float(r.entropy) - 30 * math.log(2.0)) < 2.0 ** -18


def test_as_many_rows_as_a_launch_takes(dev):
    """2^28 - 16 short rows, 2^32 - 256 threads: the last ones as by themselves; 2^28 are refused."""
    rows, vocab = 2 ** 28 - 16, 3
    x = torch.empty((rows + 16, vocab), dtype=torch.bfloat16, device=dev)
    x.normal_(generator=torch.Generator(dev).manual_seed(1))
    t = torch.arange(rows + 16, device=dev) % vocab
    with pytest.raises(RuntimeError, match="workgroups"):
        A.token_logprobs(x, t, 1)
    r = A.token_logprobs(x[:rows], t[:rows], 1)
    for b in (0, 2 ** 27 + 5, rows - 40):
        want = A.token_logprobs(x[b:b + 40], t[b:b + 40].contiguous(), 1)
        assert all(torch.equal(p[b:min(b + 40, rows)], q[:rows - b]) for p, q in zip(r, want))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows", [3, 70])
def test_a_scale_of_almost_nothing(dev, dtype, rows):
    """All scores are 0 in fp32, also those scaled down to it: the output is the mean of what a row sees."""
    print("no scale", dtype, rows, flush=True)
    gen = torch.Generator(dev).manual_seed(rows)
    v = torch.randn((4, 16, 1, 64), generator=gen, device=dev).to(dtype)
    cache = A.PagedCache(torch.randn((4, 16, 1, 64), generator=gen, device=dev).to(dtype), v)
    q = torch.randn((rows, 2, 64), generator=gen, device=dev).to(dtype)
    i32 = dict(dtype=torch.int32, device=dev)
    keep = torch.rand((rows, 50), generator=gen, device=dev) < 0.5
    keep[:, 0] = True
    bits = (torch.nn.functional.pad(keep, (0, 14)).long() << torch.arange(64, device=dev)).sum(1, keepdim=True)
    out, lse = A.attend(cache, q, shared_table=torch.arange(4, **i32)[None], shared_lengths=torch.full((1,), 50, **i32),
                        masks=bits, num_players=50, scale=1e-50, return_lse=True)
    n = keep.sum(1, keepdim=True).double()
    want = (keep.double() @ v.view(64, 64)[:50].double() / n)[:, None]
    u = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}[dtype]
    assert float((out.double() - want).abs().max()) <= (u + 82 * 2.0 ** -24) * float(v.abs().max())
    assert float((lse.double() - torch.log(n)).abs().max()) <= 2.0 ** -20
