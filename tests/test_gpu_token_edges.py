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
