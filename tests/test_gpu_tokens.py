"""The operators of token models (cache append, attention under coalition
masks, log probabilities and their gradient) against plain implementations in
float64.

Tolerances, with u the element type's half unit (2^-24, 2^-11, 2^-8):
  - attention: a score is a sum of head_dim products and a scaling, off by at
    most ds = (head_dim + 8) 2^-24 scale sum |q k|; a weight by 2 ds + 2^-22
    relative, their sum and the output's by n 2^-24 more, and 16-bit weights
    by u relative (f16: n 2^-25 absolute, below its normal numbers), so the
    output is off by at most (4 ds + (n + 32) 2^-24 + 3 u + n 2^-25) max |v|.
  - log probabilities: see the constants beside each check.
"""
import math

import numpy as np
import pytest
import torch

from paper_2401_04829_amd import _lib as L
from paper_2401_04829_amd import answers as A
from tests.gpu_util import require_gpu

pytestmark = pytest.mark.gpu

HALF = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TYPES = [torch.float32, torch.float16, torch.bfloat16]


@pytest.fixture(scope="module")
def dev():
    return require_gpu()


def _gen(dev, seed):
    return torch.Generator(device=dev).manual_seed(seed)


def _cache(gen, dev, dtype, pages, page, kv, dim, layout="slots"):
    shape = (pages, page, kv, dim) if layout == "slots" else (pages, kv, page, dim)
    k, v = (torch.randn(shape, generator=gen, device=dev).to(dtype) for _ in range(2))
    return A.PagedCache(k, v) if layout == "slots" else A.PagedCache(k.transpose(1, 2), v.transpose(1, 2))


def _pack(keep):
    """bool [rows, players] -> the sampler's words, int64 [rows, words]."""
    rows, m = keep.shape
    words = max(1, -(-m // 64))
    bits = torch.zeros((rows, words * 64), dtype=torch.int64, device=keep.device)
    bits[:, :m] = keep
    return (bits.view(rows, words, 64) << torch.arange(64, device=keep.device)).sum(2)


def _attend64(cache, q, scale, table=None, lengths=None, shared_table=None, shared_lengths=None, keep=None, first=0):
    """Row by row in float64; also the bound of a score's rounding and the longest context."""
    rows, heads, dim = q.shape
    share, page = heads // cache.kv_heads, cache.page_size
    out = torch.zeros((rows, heads, dim), dtype=torch.float64)
    lse = torch.full((rows, heads), -math.inf, dtype=torch.float64)
    kk, vv, qq = cache.k.cpu(), cache.v.cpu(), q.cpu().double()
    ds, longest = 0.0, 1
    for b in range(rows):
        slots = []
        if shared_table is not None:
            g = b // (rows // shared_table.shape[0])
            slots += [(int(shared_table[g, i // page]), i % page) for i in range(int(shared_lengths[g]))]
        if table is not None:
            slots += [(int(table[b, i // page]), i % page) for i in range(int(lengths[b]))]
        if keep is not None:
            m = keep.shape[1]
            slots = [s for i, s in enumerate(slots) if not first <= i < first + m or bool(keep[b, i - first])]
        longest = max(longest, len(slots))
        if not slots:
            continue
        p, s = np.array(slots).T
        for h in range(heads):
            k, v = kk[p, s, h // share].double(), vv[p, s, h // share].double()
            x = scale * (k @ qq[b, h])
            ds = max(ds, float((k.abs() @ qq[b, h].abs()).max()) * abs(scale) * (dim + 8) * 2.0 ** -24)
            lse[b, h] = torch.logsumexp(x, 0)
            out[b, h] = torch.softmax(x, 0) @ v
    return out, lse, ds, longest


def _check_attend(cache, q, out, lse, ref, vmax):
    want, want_lse, ds, n = ref
    u = HALF[q.dtype]
    tol = (4 * ds + (n + 32) * 2.0 ** -24 + (3 * u + n * 2.0 ** -25 if q.dtype != torch.float32 else 3 * u)) * vmax
    assert float((out.cpu().double() - want).abs().max()) <= tol
    got = lse.cpu().double()
    dead = want_lse == -math.inf
    assert torch.equal(got == -math.inf, dead)
    assert (out.cpu()[dead] == 0).all()
    d = (got - want_lse)[~dead].abs()
    assert d.numel() == 0 or float((d - 2.0 ** -22 * want_lse[~dead].abs()).max()) <= 2 * ds + (n + 32) * 2.0 ** -24


def _pages(gen, dev, rows, width, start=0):
    return (start + torch.randperm(rows * width, generator=gen, device=dev)).view(rows, width).to(torch.int32)


OWN = [  # rows, kv heads, query heads per kv head, head dim, page, lengths
    (1, 1, 1, 8, 1, [1]), (3, 2, 4, 64, 16, [1, 0, 37]), (2, 8, 4, 128, 64, [700, 129]), (4, 1, 16, 80, 24, [5, 64, 65, 300]),
    (2, 2, 17, 40, 5, [33, 31]), (1, 1, 40, 128, 7, [1025]), (2, 4, 7, 256, 32, [90, 513]), (1, 2, 3, 200, 100, [2111]),
]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,kv,share,dim,page,lengths", OWN)
def test_attention_over_own_tokens(dev, dtype, rows, kv, share, dim, page, lengths):
    print("own", dtype, rows, kv, share, dim, page, lengths, flush=True)
    gen = _gen(dev, rows + dim)
    width = -(-max(lengths) // page) + 1
    cache = _cache(gen, dev, dtype, rows * width, page, kv, dim, "slots" if dim % 3 else "heads")
    table = _pages(gen, dev, rows, width)
    q = torch.randn((rows, kv * share, dim), generator=gen, device=dev).to(dtype)
    n = torch.tensor(lengths, dtype=torch.int32, device=dev)
    out, lse = A.attend(cache, q, table, n, return_lse=True)
    ref = _attend64(cache, q, dim ** -0.5, table, n)
    _check_attend(cache, q, out, lse, ref, float(cache.v.abs().max()))


SHARED = [  # groups, rows of a group, kv heads, share, dim, page, shared lengths, own lengths up to, first player
    (1, 9, 2, 4, 64, 16, [59], 3, 0), (2, 20, 2, 1, 128, 64, [300, 117], 4, 17), (3, 5, 1, 7, 80, 24, [0, 1, 64], 0, 0),
    (1, 130, 1, 2, 128, 16, [513], 1, 0), (1, 70, 4, 3, 256, 5, [40], 2, 33), (2, 300, 2, 4, 128, 32, [129, 257], 2, 5),
    (1, 67, 1, 32, 64, 128, [1100], 9, 1), (1, 1, 2, 8, 128, 16, [333], 70, 100),
]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("groups,per,kv,share,dim,page,lengths,own,first", SHARED)
def test_attention_of_coalitions(dev, dtype, groups, per, kv, share, dim, page, lengths, own, first):
    """Coalitions of every density over a shared prompt, the empty and the
    full one among them, with own tokens (none for some rows); players may
    reach into the rows' own tokens."""
    print("shared", dtype, groups, per, kv, share, dim, page, lengths, own, first, flush=True)
    gen = _gen(dev, per + dim)
    rows, sw, ow = groups * per, max(1, -(-max(lengths) // page)), max(1, -(-own // page))
    cache = _cache(gen, dev, dtype, groups * sw + rows * ow, page, kv, dim)
    shared, table = _pages(gen, dev, groups, sw), _pages(gen, dev, rows, ow, groups * sw)
    sl = torch.tensor(lengths, dtype=torch.int32, device=dev)
    n = torch.randint(0, own + 1, (rows,), generator=gen, device=dev).to(torch.int32)
    m = max(1, max(lengths) - first + (1 if own > 2 else 0))
    keep = torch.rand((rows, m), generator=gen, device=dev) < torch.rand((rows, 1), generator=gen, device=dev)
    keep[0] = False
    keep[-1] = True
    q = torch.randn((rows, kv * share, dim), generator=gen, device=dev).to(dtype)
    out, lse = A.attend(cache, q, table, n, shared_table=shared, shared_lengths=sl, masks=_pack(keep), num_players=m,
                        first_player=first, return_lse=True)
    few = torch.unique(torch.cat([torch.arange(0, rows, max(1, rows // 40)), torch.tensor([rows - 1])]))
    if groups == 1:                                   # the reference of some rows is enough, of every tile
        ref = _attend64(cache, q[few], dim ** -0.5, table[few], n[few], shared, sl, keep[few], first)
        _check_attend(cache, q[few], out[few], lse[few], ref, float(cache.v.abs().max()))
    else:
        ref = _attend64(cache, q, dim ** -0.5, table, n, shared, sl, keep, first)
        _check_attend(cache, q, out, lse, ref, float(cache.v.abs().max()))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("per,share", [(6, 2), (150, 4)])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_what_a_row_does_not_see_does_not_reach_it(dev, dtype, per, share, bad):
    """NaN and infinities in keys and values of absent players and behind the
    lengths: rows that do not see them are as without them, rows that see a
    NaN or infinite value have it."""
    print("unseen", dtype, per, share, bad, flush=True)
    gen = _gen(dev, 5)
    kv, dim, page, length = 2, 128, 16, 100
    cache = _cache(gen, dev, dtype, 7 + per, page, kv, dim)
    shared, table = _pages(gen, dev, 1, 7), _pages(gen, dev, per, 1, 7)
    sl = torch.tensor([length], dtype=torch.int32, device=dev)
    n = torch.randint(0, 3, (per,), generator=gen, device=dev).to(torch.int32)
    keep = torch.rand((per, length), generator=gen, device=dev) < 0.5
    keep[:, 0] = True
    keep[:, 40] = torch.arange(per, device=dev) % 3 == 0
    q = torch.randn((per, kv * share, dim), generator=gen, device=dev).to(dtype)
    clean = _attend64(cache, q, dim ** -0.5, table, n, shared, sl, keep)
    vmax = float(cache.v.abs().max())
    at = (int(shared[0, 40 // page]), 40 % page)
    cache.v[at] = bad                                  # player 40
    cache.v[int(shared[0, 6]), 5:] = bad               # behind the shared part
    cache.k[int(shared[0, 6]), 5:] = bad
    for b in range(per):                               # behind the own parts
        cache.v[int(table[b, 0]), int(n[b]):] = bad
        cache.k[int(table[b, 0]), int(n[b]):] = bad
    out, lse = A.attend(cache, q, table, n, shared_table=shared, shared_lengths=sl, masks=_pack(keep),
                        num_players=length, return_lse=True)
    free = ~keep[:, 40].cpu()
    part = tuple(x[free] for x in clean[:2]) + clean[2:]
    _check_attend(cache, q[free.to(dev)], out[free.to(dev)], lse[free.to(dev)], part, vmax)
    rest = out.cpu()[~free]
    assert (rest.isnan() if math.isnan(bad) else rest == bad).all()
    d = (lse.cpu().double() - clean[1]).abs()
    assert float(d.max()) <= 1e-4                      # the values do not enter it
    cache.k[at] = bad                                  # now its key too
    out, lse = A.attend(cache, q, table, n, shared_table=shared, shared_lengths=sl, masks=_pack(keep),
                        num_players=length, return_lse=True)
    _check_attend(cache, q[free.to(dev)], out[free.to(dev)], lse[free.to(dev)], part, vmax)


@pytest.mark.parametrize("dtype", TYPES)
def test_attention_of_large_scores(dev, dtype):
    """Scores far apart: the visible ones decide, whatever the absent ones would have scored."""
    print("large", dtype, flush=True)
    gen = _gen(dev, 6)
    kv, dim, page, length, per = 1, 64, 32, 200, 40
    cache = _cache(gen, dev, dtype, 7, page, kv, dim)
    shared = _pages(gen, dev, 1, 7)
    q = torch.ones((per, 2, dim), device=dev).to(dtype)
    cache.k[int(shared[0, 1])] = 60.0                  # scores of 30 * dim * scale
    keep = torch.rand((per, length), generator=gen, device=dev) < 0.5
    keep[:, 32:64] = False
    keep[:, 3] = True
    sl = torch.tensor([length], dtype=torch.int32, device=dev)
    out, lse = A.attend(cache, q, shared_table=shared, shared_lengths=sl, masks=_pack(keep),
                        num_players=length, return_lse=True, scale=0.5)
    _check_attend(cache, q, out, lse, _attend64(cache, q, 0.5, None, None, shared, sl, keep), float(cache.v.abs().max()))


def test_attention_of_views_and_streams(dev):
    """Queries and outputs as slices of larger tensors at odd addresses, a
    cache of odd strides, another stream, and nothing written beside out."""
    gen = _gen(dev, 7)
    rows, kv, share, dim, page = 5, 2, 4, 64, 16
    big = torch.randn((2, 40, page, kv, dim + 3), generator=gen, device=dev).bfloat16()
    cache = A.PagedCache(big[0, :, :, :, 1:dim + 1], big[1, :, :, :, 1:dim + 1])
    wide = torch.randn((rows, kv * share + 2, dim + 5), generator=gen, device=dev).bfloat16()
    q = wide[:, 1:-1, 3:3 + dim]
    room = torch.full((rows, kv * share + 1, dim + 1), 7.0, device=dev).bfloat16()
    out = room[:, 1:, 1:]
    table = _pages(gen, dev, rows, 8)
    n = torch.tensor([128, 1, 17, 0, 100], dtype=torch.int32, device=dev)
    s = torch.cuda.Stream(dev)
    s.wait_stream(torch.cuda.current_stream(dev))
    with torch.cuda.stream(s):
        _, lse = A.attend(cache, q, table, n, out=out, return_lse=True)
    s.synchronize()
    _check_attend(cache, q, out, lse, _attend64(cache, q, dim ** -0.5, table, n), float(cache.v.abs().max()))
    assert (room[:, 0] == 7).all() and (room[:, :, 0] == 7).all()
    no = A.attend(cache, q, return_lse=True)           # no context at all
    assert (no[0] == 0).all() and (no[1] == -math.inf).all()
    assert A.attend(cache, q[:0], table[:0], n[:0]).shape == (0, kv * share, dim)


def test_attention_marks_what_is_out_of_range(dev):
    gen = _gen(dev, 8)
    cache = _cache(gen, dev, torch.float16, 4, 16, 1, 64)
    q = torch.randn((2, 1, 64), generator=gen, device=dev).half()
    for table, n, want in [([[0, 1], [2, 3]], [32, 5], 0), ([[0, 4], [2, 3]], [32, 5], 1),
                           ([[0, -1], [2, 3]], [32, 5], 1), ([[0, 1], [2, 3]], [33, 5], 1),
                           ([[0, 1], [2, 3]], [32, -1], 1), ([[0, 9], [2, 3]], [16, 5], 0)]:
        info = torch.zeros(1, dtype=torch.int32, device=dev)
        A.attend(cache, q, torch.tensor(table, dtype=torch.int32, device=dev),
                 torch.tensor(n, dtype=torch.int32, device=dev), info=info)
        assert int(info) == want, (table, n)


# -- append -------------------------------------------------------------------------------------

def _append64(x, pos, cos, sin, rot, interleaved):
    y = x.cpu().double()
    i = torch.arange(rot // 2)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
    for t in range(y.shape[0]):
        if pos[t] < 0 or rot == 0:
            continue
        c, s = cos[pos[t]].cpu().double(), sin[pos[t]].cpu().double()
        y[t, :, a], y[t, :, b] = (x[t].cpu().double()[:, a] * c - x[t].cpu().double()[:, b] * s,
                                  x[t].cpu().double()[:, b] * c + x[t].cpu().double()[:, a] * s)
    return y


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("kv,heads,dim,rot,page", [(1, 1, 8, 2, 1), (2, 6, 64, 64, 16), (8, 32, 128, 128, 64),
                                                   (3, 3, 80, 40, 24), (2, 7, 256, 64, 5), (1, 0, 72, 70, 7),
                                                   (2, 4, 128, 0, 16)])
def test_append(dev, dtype, interleaved, kv, heads, dim, rot, page):
    """Tokens of several sequences in any order, some not stored, with
    positions of their own or their index, against the rotation in float64
    (three roundings of fp32 and one to the element type)."""
    print("append", dtype, interleaved, kv, heads, dim, rot, page, flush=True)
    gen = _gen(dev, dim + rot)
    n, seqs, width = 23, 4, -(-40 // page)
    cache = _cache(gen, dev, dtype, seqs * width, page, kv, dim, "heads" if dim == 64 else "slots")
    before = cache.k.clone(), cache.v.clone()
    table = _pages(gen, dev, seqs, width)
    qkv = torch.randn((n, heads + 2 * kv, dim), generator=gen, device=dev).to(dtype)
    q, k, v = qkv.split([heads, kv, kv], 1)
    place = torch.randperm(seqs * 40, generator=gen, device=dev)[:n]
    rows, index = (place // 40).to(torch.int32), (place % 40).to(torch.int32)
    index[::7] = -1
    positions = None if dim == 256 else torch.randint(0, 50, (n,), generator=gen, device=dev).to(torch.int32)
    if positions is not None:
        positions[5] = -3
    angle = torch.rand((50, rot // 2), generator=gen, device=dev) * 6.28
    cos, sin = (angle.cos(), angle.sin()) if rot else (None, None)
    info = torch.zeros(1, dtype=torch.int32, device=dev)
    got = A.append_tokens(cache, k, v, table, index, rows=rows, positions=positions, q=q if heads else None, cos=cos,
                          sin=sin, interleaved=interleaved, info=info)
    assert int(info) == 0
    pos = (index if positions is None else positions).cpu().tolist()
    wk, wq = (_append64(x, pos, cos, sin, rot, interleaved) for x in (k, q))
    if heads:
        tol = HALF[dtype] * wq.abs() + 2.0 ** -22 * float(q.abs().max())
        assert ((got.cpu().double() - wq).abs() <= tol).all()
    want_k, want_v = (x.cpu().double().clone() for x in before)
    for t in range(n):
        if int(index[t]) >= 0:
            at = int(table[int(rows[t]), int(index[t]) // page]), int(index[t]) % page
            want_k[at], want_v[at] = wk[t], v[t].cpu().double()
    assert torch.equal(cache.v.cpu().double(), want_v)
    assert ((cache.k.cpu().double() - want_k).abs() <= HALF[dtype] * want_k.abs() + 2.0 ** -22 * float(k.abs().max())).all()


def test_append_in_place_and_out_of_range(dev):
    gen = _gen(dev, 9)
    cache = A.PagedCache.empty(4, 8, 2, 64, torch.float32, dev)
    table = torch.tensor([[0, 1], [2, 9]], dtype=torch.int32, device=dev)
    x = torch.randn((3, 2, 64), generator=gen, device=dev)
    angle = torch.rand((16, 32), generator=gen, device=dev)
    a = dict(cos=angle.cos(), sin=angle.sin())
    i32 = dict(dtype=torch.int32, device=dev)

    def call(index, rows, q=None, **kw):
        info = torch.zeros(1, **i32)
        r = A.append_tokens(cache, x, x, table, torch.tensor(index, **i32), rows=torch.tensor(rows, **i32), q=q,
                            info=info, **a, **kw)
        return r, int(info)
    q = torch.randn((3, 5, 64), generator=gen, device=dev)
    want, bad = call([0, 9, 3], [0, 0, 1], q)
    assert bad == 0
    got, _ = call([0, 9, 3], [0, 0, 1], q, q_out=q)
    assert got is q and torch.equal(got, want)
    before = cache.k.clone()
    for index, rows in [([0, 9, 9], [0, 0, 1]), ([16, 0, 0], [0, 0, 1]), ([0, 0, 0], [2, 0, 1]), ([0, 0, 0], [-1, 0, 1])]:
        assert call(index, rows)[1] == 1
    assert torch.equal(cache.k[3], before[3])
    assert call([0, 1, 2], [0, 0, 0], positions=torch.tensor([15, 16, 0], **i32))[1] == 1


# -- log probabilities --------------------------------------------------------------------------

def _logits_of(gen, dev, rows, vocab, dtype, kind):
    x = torch.randn((rows, vocab), generator=gen, device=dev) * (8 if kind == "wide" else 2)
    if kind == "ties":
        x = torch.randint(-2, 3, (rows, vocab), generator=gen, device=dev).float()
    if kind == "banned":
        x[torch.rand((rows, vocab), generator=gen, device=dev) < 0.9] = -math.inf
    if kind == "lowest":
        x[torch.rand((rows, vocab), generator=gen, device=dev) < 0.7] = torch.finfo(dtype).min
        x[0] = torch.finfo(dtype).min
    if kind == "rising":
        x = torch.sort(x, 1).values
    if kind == "far":
        x += 20000.0
    return x.to(dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,vocab,top,kind", [
    (1, 1, 1, "plain"), (5, 2, 2, "plain"), (70, 41, 5, "plain"), (3, 64, 64, "ties"), (9, 1000, 20, "wide"),
    (2, 2049, 64, "ties"), (7, 5001, 1, "rising"), (4, 32768, 5, "plain"), (1, 131072, 20, "plain"),
    (3, 50021, 7, "banned"), (5, 4097, 33, "lowest"), (2, 70001, 20, "far"), (4100, 301, 3, "ties"),
    (5000, 8193, 4, "plain"), (6, 257, 0, "rising"), (130, 16, 9, "banned"), (33, 129, 64, "lowest")])
def test_logprobs(dev, dtype, rows, vocab, top, kind):
    print("logprobs", dtype, rows, vocab, top, kind, flush=True)
    gen = _gen(dev, vocab)
    x = _logits_of(gen, dev, rows, vocab, dtype, kind)
    t = torch.randint(0, vocab, (rows,), generator=gen, device=dev)
    if rows > 2:
        t[2] = -1
    info = torch.zeros(1, dtype=torch.int32, device=dev)
    r = A.token_logprobs(x, t, top, info=info)
    assert int(info) == 0
    y = x.double()
    has = t >= 0
    m = y.amax(1)
    dead = m == -math.inf
    z = y - m.masked_fill(dead, 0.0)[:, None]         # so that rows of the lowest value alone are uniform
    logs = torch.log(z.exp().sum(1))
    lse = torch.where(dead, -math.inf, m + logs)
    logp = torch.where(dead[:, None], -math.inf, z - logs[:, None])
    p = torch.where(dead[:, None], 0.0, logp.exp())
    plogp = torch.where(p == 0, 0.0, p * logp)
    # sums of at most 32 + vocab / 1024 + 16 fp32 additions in a row, exponentials off by 2^-23 |x - m| + 2^-22,
    # whose average is at most log(vocab) + 1 (both relative to the sum)
    lg = math.log(vocab) + 2
    depth = 64 + vocab / 1024
    tol = 2.0 ** -24 * (depth + 4 * lg)

    def near(got, want, tol):
        got = got.double()
        dead = want == -math.inf
        assert torch.equal(got == -math.inf, dead)
        ok = (got - want)[~dead].abs() <= (tol + torch.zeros_like(want))[~dead]
        assert ok.all(), float((got - want)[~dead].abs().max())
    near(r.lse, lse, tol + 2.0 ** -23 * lse.abs().nan_to_num(posinf=0))
    near(r.entropy, -plogp.sum(1), 2.0 ** -23 * ((depth + 8) * lg + lg * lg))
    chosen = logp.gather(1, t.clamp(min=0)[:, None])[:, 0]
    rank = (y > y.gather(1, t.clamp(min=0)[:, None])).sum(1)
    far = 2.0 ** -22 * ((y.gather(1, t.clamp(min=0)[:, None])[:, 0] - m).abs().nan_to_num(nan=0, posinf=0) + lg)
    near(r.logprob, torch.where(has, chosen, 0.0), tol + far)
    assert torch.equal(r.rank.long(), torch.where(has, rank, -1))
    order = torch.sort(y, dim=1, descending=True, stable=True).indices[:, :top]
    assert torch.equal(r.top_id.long(), order)
    best = logp.gather(1, order)
    near(r.top_logprob, best, tol + 2.0 ** -22 * ((y.gather(1, order) - m[:, None]).abs().nan_to_num(nan=0, posinf=0) + lg))


def test_logprobs_of_rows_without_numbers(dev):
    """Rows of -inf alone, with a NaN, with +inf; odd row strides and addresses; optional outputs."""
    gen = _gen(dev, 3)
    for vocab in (41, 3001):
        room = torch.randn((6, vocab + 3), generator=gen, device=dev).bfloat16()
        x = room[:, 1:vocab + 1]
        x[1] = -math.inf
        x[2, 7] = math.nan
        x[3, 5] = math.inf
        x[4] = math.nan
        t = torch.tensor([3, 4, 5, 6, 7, 8], device=dev)
        r = A.token_logprobs(x, t, 3)
        assert r.lse[1] == -math.inf and r.logprob[1] == -math.inf and r.entropy[1] == 0
        assert (r.top_logprob[1] == -math.inf).all() and r.top_id[1].tolist() == [0, 1, 2] and int(r.rank[1]) == 0
        for b in (2, 3, 4):
            assert all(bool(z[b].isnan().all()) for z in (r.lse, r.logprob, r.entropy, r.top_logprob))
            assert (r.top_id[b] >= 0).all() and (r.top_id[b] < vocab).all()
        for b in (0, 5):
            want = torch.log_softmax(x[b].double(), 0)
            assert abs(float(r.logprob[b]) - float(want[t[b]])) < 1e-5
        info = torch.zeros(1, dtype=torch.int32, device=dev)
        r2 = A.token_logprobs(x, torch.tensor([vocab, 4, 5, 6, 7, 8], device=dev), 0, info=info)
        assert int(info) == 1 and float(r2.logprob[0]) == 0 and int(r2.rank[0]) == -1
    assert A.token_logprobs(x[:0], t[:0], 2).top_id.shape == (0, 2)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,vocab,kind", [(1, 1, "plain"), (70, 41, "plain"), (3, 5001, "banned"), (2, 50021, "wide"),
                                             (5, 300, "lowest")])
def test_logprobs_gradient(dev, dtype, rows, vocab, kind):
    """The formula in float64: p is off by 2^-23 (|log p| + 4) relative."""
    print("gradient", dtype, rows, vocab, kind, flush=True)
    gen = _gen(dev, vocab)
    x = _logits_of(gen, dev, rows, vocab, dtype, kind)
    t = torch.randint(0, vocab, (rows,), generator=gen, device=dev)
    if rows > 2:
        t[2] = -1
    gl, ge = (torch.randn(rows, generator=gen, device=dev) for _ in range(2))
    r = A.token_logprobs(x, t)
    for has_l, has_e in ((True, True), (True, False), (False, True)):
        got = A.token_logprobs_backward(x, t, r.lse, r.entropy if has_e else None, gl if has_l else None,
                                        ge if has_e else None).double()
        y, lse, ent = x.double(), r.lse.double()[:, None], r.entropy.double()[:, None]
        logp = y - lse
        p = logp.exp()
        a = (gl.double() if has_l else torch.zeros(rows, device=dev).double()) * (t >= 0)
        b = (ge.double() if has_e else torch.zeros(rows, device=dev).double())[:, None]
        lp = torch.where(p == 0, 0.0, logp)
        want = -p * (a[:, None] + b * (lp + ent))
        hit = torch.arange(vocab, device=dev) == t[:, None]
        want = want + torch.where(hit, a[:, None], 0.0)
        tol = HALF[dtype] * want.abs() + 2.0 ** -22 * (lp.abs() + 4) * p * (a.abs()[:, None] + b.abs() * (lp.abs() + ent + 1)) \
            + 2.0 ** -23 * a.abs()[:, None] * hit + 2.0 ** -25 * (dtype == torch.float16) + 1e-37
        assert ((got - want).abs() <= tol).all(), float(((got - want).abs() - tol).max())
        inplace = x.clone()
        A.token_logprobs_backward(inplace, t, r.lse, r.entropy if has_e else None, gl if has_l else None,
                                  ge if has_e else None, out=inplace)
        assert torch.equal(inplace.double(), got)


def test_logprobs_gradient_against_differences(dev):
    """Central differences of the forward call's own outputs, at a step of
    2^-6: off by the third derivative, at most 2^-12, and the forward's
    rounding, at most 2^-19 / 2^-6."""
    gen = _gen(dev, 4)
    x = torch.randn((1, 37), generator=gen, device=dev)
    t = torch.tensor([11], device=dev)
    r = A.token_logprobs(x, t)
    step = 2.0 ** -6
    up, down = (A.token_logprobs(x + s * torch.eye(37, device=dev) * step, t.expand(37).contiguous()) for s in (1, -1))
    one = torch.ones(1, device=dev)
    for name, args in (("logprob", (r.lse, None, one, None)), ("entropy", (r.lse, r.entropy, None, one))):
        d = (getattr(up, name) - getattr(down, name)) / (2 * step)
        got = A.token_logprobs_backward(x, t, *args)[0]
        assert float((d - got).abs().max()) <= 3 * (2.0 ** -12 + 2.0 ** -13), name


def test_gradient_of_a_row_without_numbers_is_zero(dev):
    x = torch.full((2, 9), -math.inf, device=dev)
    x[1, 3] = 1.0
    t = torch.tensor([2, 3], device=dev)
    r = A.token_logprobs(x, t)
    one = torch.ones(2, device=dev)
    g = A.token_logprobs_backward(x, t, r.lse, r.entropy, one, one)
    assert (g == 0).all()


# sizes on either side of the ways in which the work is laid out: two tiles of
# queries to a wavefront, more parts than the lanes that join them, splits of
# 64 keys, own tokens beside the shared part and apart from it
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,kv,share,dim,page,lengths", [
    (260, 1, 20, 72, 16, [2000] + 259 * [1793]), (1, 2, 4, 128, 16, [12001]), (1, 1, 1, 64, 8, [8193]),
    (5, 2, 3, 128, 16, [64, 65, 128, 0, 1000])])
def test_attention_over_own_tokens_laid_out(dev, dtype, rows, kv, share, dim, page, lengths):
    test_attention_over_own_tokens(dev, dtype, rows, kv, share, dim, page, lengths)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("groups,per,kv,share,dim,page,lengths,own,first", [
    (1, 4100, 2, 4, 72, 16, [300], 2, 0), (1, 2000, 2, 4, 64, 16, [70], 19, 3), (1, 40, 2, 4, 64, 16, [130], 19, 3),
    (1, 31, 1, 1, 128, 16, [200], 2, 0), (1, 33, 1, 1, 128, 16, [200], 33, 0), (1, 35, 1, 2, 256, 16, [97], 5, 9),
    (1, 70, 1, 2, 200, 16, [97], 5, 9), (1, 128, 1, 1, 256, 16, [65], 1, 0)])
def test_attention_of_coalitions_laid_out(dev, dtype, groups, per, kv, share, dim, page, lengths, own, first):
    test_attention_of_coalitions(dev, dtype, groups, per, kv, share, dim, page, lengths, own, first)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,vocab,top,kind", [(3, 256, 6, "plain"), (3, 257, 6, "plain"), (3, 700, 0, "plain"),
                                                 (3, 1024, 3, "plain"), (4100, 1000, 2, "plain")])
def test_logprobs_laid_out(dev, dtype, rows, vocab, top, kind):
    test_logprobs(dev, dtype, rows, vocab, top, kind)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,vocab,kind", [(2, 4096, "plain"), (2, 8191, "plain"), (2, 8193, "plain")])
def test_logprobs_gradient_laid_out(dev, dtype, rows, vocab, kind):
    test_logprobs_gradient(dev, dtype, rows, vocab, kind)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,kv,share,dim,page,longest", [(700, 32, 1, 8, 64, 1500), (2100, 32, 2, 16, 16, 600)])
def test_attention_of_more_keys_than_the_splits_hold(dev, dtype, rows, kv, share, dim, page, longest):
    """So many rows that a wavefront comes back for further keys of its row;
    the rows draw on one pool of pages, as rows with a common beginning do."""
    print("further keys", dtype, rows, kv, share, dim, page, longest, flush=True)
    gen = _gen(dev, rows)
    cache = _cache(gen, dev, dtype, 97, page, kv, dim)
    width = -(-longest // page)
    table = torch.randint(0, 97, (rows, width), generator=gen, device=dev).to(torch.int32)
    n = torch.randint(0, 300, (rows,), generator=gen, device=dev).to(torch.int32)
    n[::50] = longest
    n[1::50] = longest - 243
    q = torch.randn((rows, kv * share, dim), generator=gen, device=dev).to(dtype)
    out, lse = A.attend(cache, q, table, n, max_length=longest, return_lse=True)
    few = torch.unique(torch.cat([torch.arange(0, rows, 50), torch.arange(1, rows, 50), torch.tensor([2, rows - 1])]))
    ref = _attend64(cache, q[few], dim ** -0.5, table[few], n[few])
    _check_attend(cache, q[few], out[few], lse[few], ref, float(cache.v.abs().max()))


@pytest.mark.parametrize("dtype", TYPES)
def test_coalitions_of_more_keys_than_the_splits_hold(dev, dtype):
    test_attention_of_coalitions(dev, dtype, 1, 20000, 32, 1, 8, 16, [600], 1, 0)


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_a_cache_past_32_bits(dev, dim):
    """Pages whose elements lie beyond 2^31 give what the same pages give in a
    small cache, bit for bit: append, own tokens, shared parts of few and of
    many queries."""
    print("large cache", dim, flush=True)
    gen, page, kv, rows = _gen(dev, dim), 16, 2, 64
    per = page * kv * dim
    last = 2 ** 31 // per + 80                    # pages; the last ones are used
    big = A.PagedCache(torch.empty((last, page, kv, dim), dtype=torch.bfloat16, device=dev),
                       torch.empty((last, page, kv, dim), dtype=torch.bfloat16, device=dev))
    small = _cache(gen, dev, torch.bfloat16, 80, page, kv, dim)
    big.k[-80:], big.v[-80:] = small.k, small.v
    table = torch.arange(rows, device=dev).view(rows, 1).to(torch.int32)
    shared = (64 + torch.randperm(16, generator=gen, device=dev)).view(1, 16).to(torch.int32)
    n = torch.randint(1, 16, (rows,), generator=gen, device=dev).to(torch.int32)
    sl = torch.tensor([251], dtype=torch.int32, device=dev)
    masks = torch.randint(-2 ** 62, 2 ** 62, (rows, 4), generator=gen, device=dev)
    q = torch.randn((rows, 2 * kv, dim), generator=gen, device=dev).to(torch.bfloat16)
    new = torch.randn((rows, kv, dim), generator=gen, device=dev).to(torch.bfloat16)
    got = []
    for cache, add in ((small, 0), (big, last - 80)):
        A.append_tokens(cache, new, -new, table + add, n)
        got.append([A.attend(cache, q, table + add, n + 1, return_lse=True),
                    A.attend(cache, q, table + add, n + 1, shared_table=shared + add, shared_lengths=sl, masks=masks,
                             num_players=251, return_lse=True),
                    A.attend(cache, q[:5], table[:5] + add, n[:5] + 1, shared_table=shared + add, shared_lengths=sl,
                             masks=masks[:5], num_players=251, return_lse=True), (cache.k[-80:], cache.v[-80:])])
    for a, b in zip(*got):
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    ref = _attend64(small, q, dim ** -0.5, table, n + 1)
    _check_attend(small, q, *got[1][0], ref, float(small.v.abs().max()))


def test_logits_past_32_bits(dev):
    gen, vocab = _gen(dev, 5), 5001
    flat = torch.empty(2 ** 31 + 4 * vocab, dtype=torch.bfloat16, device=dev)
    x = flat.as_strided((2, vocab), (2 ** 31 + 3, 1))
    x.copy_(torch.randn((2, vocab), generator=gen, device=dev))
    t = torch.tensor([17, 4999], device=dev)
    a, b = A.token_logprobs(x, t, 7), A.token_logprobs(x.contiguous(), t, 7)
    assert all(torch.equal(i, j) for i, j in zip(a, b))
    g = torch.tensor([1.0, -2.0], device=dev)
    want = A.token_logprobs_backward(x.contiguous(), t, b.lse, b.entropy, g, g)
    assert torch.equal(A.token_logprobs_backward(x, t, a.lse, a.entropy, g, g, out=x), want)


def test_calls_replay_from_a_graph(dev):
    """Append, attention (split and joined, with a shared part and masks), log
    probabilities and their gradient, captured once and replayed on new inputs
    with other work between, give what the calls themselves give."""
    gen, kv, dim, rows, page = _gen(dev, 3), 2, 64, 40, 16
    cache = _cache(gen, dev, torch.bfloat16, 200, page, kv, dim)
    table = (100 + torch.arange(rows, device=dev)).view(rows, 1).to(torch.int32)
    shared = torch.randperm(100, generator=gen, device=dev).view(1, 100).to(torch.int32)
    sl = torch.tensor([1511], dtype=torch.int32, device=dev)
    n = torch.zeros(rows, dtype=torch.int32, device=dev)
    ins = [torch.empty((rows, kv, dim), dtype=torch.bfloat16, device=dev) for _ in range(2)]
    q = torch.empty((rows, 2 * kv, dim), dtype=torch.bfloat16, device=dev)
    masks = torch.empty((rows, 24), dtype=torch.int64, device=dev)
    head = torch.randn((2 * kv * dim, 5001), generator=gen, device=dev)
    logits, t = torch.empty((rows, 5001), device=dev), torch.randint(0, 5001, (rows,), generator=gen, device=dev)

    def draw():
        for x in (*ins, q, logits):
            x.copy_(torch.randn(x.shape, generator=gen, device=dev))
        masks.copy_(torch.randint(-2 ** 62, 2 ** 62, masks.shape, generator=gen, device=dev))

    def calls():
        A.append_tokens(cache, *ins, table, n)
        out, lse = A.attend(cache, q, table, n + 1, shared_table=shared, shared_lengths=sl, masks=masks, num_players=1511,
                            return_lse=True)
        r = A.token_logprobs(logits, t, 9)
        return [out, lse, *r, A.token_logprobs_backward(logits, t, r.lse, grad_logprob=r.logprob)]
    draw()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = calls()
    for _ in range(4):
        draw()
        graph.replay()
        torch.cuda.synchronize()
        kept = [x.clone() for x in got]
        assert all(torch.equal(a, b) for a, b in zip(kept, calls()))
        (head @ head.T).sum().item()
