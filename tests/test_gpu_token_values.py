"""That every value of attention's context reaches the output, in its place.

Element d of the values is 0 but for the keys of every D-th block of eight
(key j with j // 8 % D == d), so that an output element is the sum of few
values and its tolerance small beside any of them.

Tolerance of an element, with u the type's half unit, c = sum_j p_j |v_j| of
that element, ds the error of a score: the weights are off by 4 ds + (n + 32)
2^-24 (see the float64 tests of attention), 16-bit ones by u more (fp16 below
2^-28 of the largest by 2^-39 absolute), the output is rounded once (fp16 below
2^-14, where its spacing is 2^-24, by 2^-25 absolute):
    max(u |out|, 2^-25 in fp16) + (4 ds + (n + 32) 2^-24 + u + n 2^-39) c.
That it is narrow enough is part of the test: results without the values of 32
keys on end are outside for every row, with those of two neighbouring keys
exchanged (which changes little where their weights are alike) for most."""
import math

import pytest
import torch

from paper_2401_04829_amd import answers as A
from tests.gpu_util import require_gpu
from tests.test_gpu_tokens import HALF, TYPES, _gen, _pack, _pages

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    return require_gpu()


def _context(cache, b, table, lengths, shared, shared_len, keep, first):
    """Pages and slots of the positions that row b sees."""
    page, place = cache.page_size, []
    if shared is not None:
        at = torch.arange(shared_len, device=cache.device)
        place.append((shared[0].long()[at // page], at % page))
    if table is not None:
        at = torch.arange(int(lengths[b]), device=cache.device)
        place.append((table[b].long()[at // page], at % page))
    p, s = (torch.cat(x) for x in zip(*place))
    seen = torch.ones(p.numel(), dtype=torch.bool, device=cache.device)
    if keep is not None:
        seen[first:first + keep.shape[1]] = keep[b]
    return p[seen], s[seen]


def _check(cache, q, out, rows, context):
    """`rows` of the output against float64."""
    kv, dim, u = cache.kv_heads, cache.head_dim, HALF[q.dtype]
    share = q.shape[1] // kv
    missing = exchanged = 0
    for b in rows:
        p, s = context(b)
        n = p.numel()
        if n == 0:
            assert bool((out[b] == 0).all())
            continue
        k, val = cache.k[p, s].double(), cache.v[p, s].double()                  # [n, kv, dim]
        x = q[b].double().view(kv, share, dim)
        scores = torch.einsum("hsd,nhd->hsn", x, k) / math.sqrt(dim)
        ds = torch.einsum("hsd,nhd->hsn", x.abs(), k.abs()).amax() / math.sqrt(dim) * (dim + 8) * 2.0 ** -24
        w = torch.softmax(scores, 2)
        want, c = (torch.einsum("hsn,nhd->hsd", w, y) for y in (val, val.abs()))
        small = 0.0 if q.dtype == torch.float32 else u + n * 2.0 ** -39
        last = (u * want.abs()).clamp(min=2.0 ** -25 if q.dtype == torch.float16 else 0.0)
        tol = last + (4 * ds + (n + 32) * 2.0 ** -24 + small) * c + 1e-30

        def off(x):
            return ((x - want).abs() > tol).any()
        got = out[b].double().view(kv, share, dim)
        assert not off(got), float(((got - want).abs() / tol).max())
        if n >= 64:
            less = val.clone()
            less[n // 2:n // 2 + 32] = 0
            missing += int(off(torch.einsum("hsn,nhd->hsd", w, less)))
            other = val.clone()
            other[n // 2], other[n // 2 + 1] = val[n // 2 + 1], val[n // 2]
            exchanged += int(off(torch.einsum("hsn,nhd->hsd", w, other)))
        else:
            missing, exchanged = missing + 1, exchanged + 1
    seen = sum(context(b)[0].numel() > 0 for b in rows)
    assert missing == seen and exchanged > seen // 2, (missing, exchanged, seen)


def _values(gen, dev, dtype, place, pages, page, kv, dim):
    """Keys, and values that are 0 but for one block of eight positions in `dim`; place: [pages, page] position or -1."""
    k, v = (torch.randn((pages, page, kv, dim), generator=gen, device=dev).to(dtype) for _ in range(2))
    block = place // 8 % dim
    only = block[:, :, None] == torch.arange(dim, device=dev)
    return k, v * only[:, :, None]


def _positions(table, page, pages, start=0):
    at = torch.zeros((pages, page), dtype=torch.int64, device=table.device)
    index = start + torch.arange(table.shape[1] * page, device=table.device).view(-1, page)
    at[table.long().view(-1)] = index.repeat(table.shape[0], 1)
    return at


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,kv,share,dim,page,lengths", [
    (2, 8, 4, 128, 64, [700, 129]), (4, 1, 16, 80, 24, [5, 64, 65, 300]), (1, 1, 40, 128, 7, [1025]),
    (2, 4, 7, 256, 32, [90, 513]), (1, 2, 3, 200, 100, [2111]), (1, 2, 4, 128, 16, [12001]), (3, 2, 5, 64, 16, [1, 33, 4000]),
    (260, 1, 20, 72, 16, [2000] + 259 * [1793])])
def test_every_own_value_is_in_its_place(dev, dtype, rows, kv, share, dim, page, lengths):
    print("own values", dtype, rows, kv, share, dim, page, lengths[:4], flush=True)
    gen = _gen(dev, rows + dim)
    width = -(-max(lengths) // page)
    table = _pages(gen, dev, rows, width)
    k, v = _values(gen, dev, dtype, _positions(table, page, rows * width), rows * width, page, kv, dim)
    cache = A.PagedCache(k, v)
    n = torch.tensor(lengths, dtype=torch.int32, device=dev)
    q = torch.randn((rows, kv * share, dim), generator=gen, device=dev).to(dtype)
    out = A.attend(cache, q, table, n)
    few = range(0, rows, max(1, rows // 12))
    _check(cache, q, out, few, lambda b: _context(cache, b, table, lengths, None, 0, None, 0))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,kv,share,dim,page,shared,own,first", [
    (9, 2, 4, 64, 16, 300, 3, 0), (130, 1, 2, 128, 16, 513, 1, 0), (300, 2, 4, 128, 32, 1290, 2, 5), (70, 4, 3, 256, 5, 140, 2, 33),
    (300, 1, 4, 256, 16, 900, 0, 0), (150, 2, 4, 64, 64, 2000, 3, 100), (70, 1, 8, 80, 24, 700, 0, 9), (67, 1, 32, 64, 128, 1100, 9, 1),
    (40, 2, 4, 64, 16, 130, 19, 3), (1, 2, 8, 128, 16, 333, 70, 100), (2100, 2, 4, 128, 16, 417, 4, 17)])
def test_every_value_that_a_coalition_keeps_is_in_its_place(dev, dtype, rows, kv, share, dim, page, shared, own, first):
    print("kept values", dtype, rows, kv, share, dim, page, shared, own, first, flush=True)
    gen = _gen(dev, rows + dim)
    sw, ow = -(-shared // page), max(1, -(-own // page))
    common, table = _pages(gen, dev, 1, sw), _pages(gen, dev, rows, ow, sw)
    pages = sw + rows * ow
    place = _positions(common, page, pages)
    place[sw:] = _positions(table, page, pages, shared)[sw:]
    k, v = _values(gen, dev, dtype, place, pages, page, kv, dim)
    cache = A.PagedCache(k, v)
    n = torch.randint(0, own + 1, (rows,), generator=gen, device=dev).to(torch.int32)
    keep = torch.rand((rows, shared - first), generator=gen, device=dev) < 0.25 + 0.75 * torch.rand((rows, 1), generator=gen,
                                                                                                 device=dev)
    keep[-1] = True
    q = torch.randn((rows, kv * share, dim), generator=gen, device=dev).to(dtype)
    sl = torch.tensor([shared], dtype=torch.int32, device=dev)
    out = A.attend(cache, q, table, n, shared_table=common, shared_lengths=sl, masks=_pack(keep), num_players=shared - first,
                   first_player=first)
    few = sorted({*range(0, rows, max(1, rows // 12)), rows - 1})
    _check(cache, q, out, few, lambda b: _context(cache, b, table, n, common, shared, keep, first))
