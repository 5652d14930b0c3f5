"""attention_weights of rows whose lse is far out or not finite: what such a row
does not see is as if the row gave nothing (lse -inf), bit for bit."""
import math

import pytest
import torch

from paper_2401_04829_amd import answers as A
from tests.gpu_util import require_gpu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows", [3, 90])                    # by the kernels of few and of many queries
@pytest.mark.parametrize("far", [1e8, 3e9, 1e10, -1e10, -3e10, 1e20, -1e20, 3e38, -3e38, math.inf, math.nan])
def test_rows_far_out_leave_what_they_do_not_see(rows, dtype, far):
    dev = require_gpu()
    print("far", rows, dtype, far, flush=True)
    gen = torch.Generator(dev).manual_seed(rows)
    heads, dim, tokens, page = 4, 64, 150, 16
    cache = A.PagedCache(*torch.randn((2, 10, page, 2, dim), generator=gen, device=dev).to(dtype).unbind(0))
    q = torch.randn((rows, heads, dim), generator=gen, device=dev).to(dtype)
    table = torch.randperm(10, generator=gen, device=dev).to(torch.int32)[None]
    lengths = torch.full((rows,), tokens - 20, dtype=torch.int32, device=dev)
    keep = torch.rand((rows, 130), generator=gen, device=dev) < 0.5
    keep[1, 40:] = False                                     # of the row far out: the first ones
    words = torch.zeros((rows, 192), dtype=torch.int64, device=dev)
    words[:, :130] = keep
    masks = (words.view(rows, 3, 64) << torch.arange(64, device=dev)).sum(2)
    _, lse = A.attend(cache, q, shared_table=table, shared_lengths=lengths[:1], masks=masks, num_players=130,
                      return_lse=True)
    got = []
    for value in (far, -math.inf):
        lse[1] = value
        weights = torch.arange(160, device=dev, dtype=torch.float32)[None] / 7
        A.attention_weights(cache, q, lse, table, lengths, weights, masks=masks, num_players=130)
        got.append(weights[0])
    hidden = torch.ones(160, dtype=torch.bool, device=dev)
    hidden[:130] = ~keep[1]
    assert torch.equal(got[0][hidden], got[1][hidden])
    assert torch.equal(got[0][130:], torch.arange(130, 160, device=dev, dtype=torch.float32) / 7)
