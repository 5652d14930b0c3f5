"""Torch-facing calls that explain a token model's answer.

The players are tokens of a prompt.  Their keys and values are cached once
(`append_tokens` into a `PagedCache`); under a coalition, the new token
attends over the cached prompt, seeing the positions its mask keeps, and over
tokens of its own (`attend`); the answer's log probability is the coalition's
value (`token_logprobs`), from which `AnswerExplainer` takes the Shapley
values with the library's sampler and least squares.  Around these: norms of
heads with the rotation (`norm_rotate`, and on the way into the cache), the
weights that attention gave cached tokens (`attention_weights`) and eviction of
those that got least (`evict_tokens`), log probabilities straight from hidden
states (`linear_logprobs`).

Torch provides device memory and streams; the work runs in libgnnshap.so on
the current stream.  Every tensor must be on the cache's (the logits') device.
Of these calls only those named `differentiable_` have a derivative: the others
refuse tensors that require a gradient (unless under torch.no_grad()) or carry
a tangent.  A backward pass is captured into a graph as any of torch's is: only
while no other graph of the same leaves lives that was built outside of the
capture (torch would wait for its stream, which ends the capture).
"""
import math
from functools import partial
from typing import NamedTuple

import torch
from torch.autograd import forward_ad

from . import _lib as L

_DTYPES = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}


_raw_stream = torch._C._cuda_getCurrentRawStream   # torch.cuda.current_stream(device).cuda_stream without its object
_grad_enabled, _any_requires_grad = torch.is_grad_enabled, torch._C._any_requires_grad


def _need(ok, what):
    if not ok:
        raise ValueError(what)


def _ptr(t):
    return None if t is None else t.data_ptr()


def _no_derivative(call, *tensors):
    """Refuses tensors through which autograd would miss `call`'s derivative."""
    if _grad_enabled() and _any_requires_grad(*tensors):
        raise ValueError(f"{call} has no derivative, and a tensor that it got requires a gradient: call it under "
                         "torch.no_grad() or with that tensor detached")
    if forward_ad._current_level >= 0:
        for t in tensors:
            if t is not None and forward_ad.unpack_dual(t).tangent is not None:
                raise ValueError(f"{call} has no derivative, and a tensor that it got carries a tangent")


def _on(device, call, *args):
    """call(*args, stream) with `device` current and its current stream."""
    index = device.index
    if torch.cuda.current_device() == index:
        return call(*args, _raw_stream(index))
    with torch.cuda.device(device):
        return call(*args, _raw_stream(index))


def _vector(t, name, dtype, size, device):
    """The address of an optional contiguous tensor of `dtype` and `size` (None: any shape)."""
    if t is None:
        return None
    if t.dtype != dtype or t.device != device or not t.is_contiguous() or (size is not None and t.shape != size):
        raise ValueError(f"{name}: a contiguous {dtype} tensor of shape {size} on {device} is needed, got {t.dtype} "
                         f"{tuple(t.shape)} on {t.device}")
    return t.data_ptr()


def _heads(t, name, heads, dim, dtype, device):
    """Checks a [rows, heads, dim] tensor whose last axis is contiguous; its address and two strides."""
    shape, stride = t.shape, t.stride()
    if (len(shape) != 3 or t.dtype != dtype or t.device != device or shape[2] != dim
            or (heads is not None and shape[1] != heads) or (stride[2] != 1 and t.numel() > 0)):
        raise ValueError(f"{name}: a [rows, {heads or 'heads'}, {dim}] {dtype} tensor on {device} with a contiguous "
                         f"last axis is needed, got {t.dtype} {tuple(shape)} with strides {stride} on {t.device}")
    return t.data_ptr(), stride[0], stride[1]


class PagedCache:
    """Keys and values in pages: `k` and `v` are [pages, page size, kv heads,
    head dim] tensors (or views, such as of [pages, kv heads, page size, head
    dim]) of one type and one set of strides, the head dim contiguous.  A page
    table, int32 [rows, pages of a row], names the pages of each sequence."""

    def __init__(self, k, v):
        _need(k.dim() == 4 and k.shape == v.shape and k.stride() == v.stride() and k.dtype == v.dtype
              and k.device == v.device, "keys and values: two [pages, page size, kv heads, head dim] tensors of one "
              "type, device and set of strides are needed")
        _need(k.dtype in _DTYPES, f"cache type {k.dtype} is not one of float32, float16, bfloat16")
        _need(k.is_cuda and k.stride(3) == 1, "the cache must be on a GPU, its head dim contiguous")
        self.k, self.v = k, v
        pages, page, heads, dim = k.shape
        self.kv_heads, self.head_dim, self.page_size = heads, dim, page
        self.dtype, self.device = k.dtype, k.device
        self._c = L.gnnshap_cache(_DTYPES[k.dtype], heads, dim, page, pages, k.stride(0), k.stride(1), k.stride(2),
                                  k.data_ptr(), v.data_ptr())

    @classmethod
    def empty(cls, pages, page_size, kv_heads, head_dim, dtype=torch.bfloat16, device="cuda"):
        kv = torch.zeros((2, pages, page_size, kv_heads, head_dim), dtype=dtype, device=device)
        return cls(kv[0], kv[1])


def append_tokens(cache, k, v, table, index, rows=None, positions=None, q=None, cos=None, sin=None, interleaved=False,
                  q_out=None, info=None, q_norm=None, k_norm=None, eps=1e-6):
    """gnnshap_cache_append: writes keys and values [tokens, kv heads, head
    dim] of new tokens into the cache, token t at place index[t] (int32;
    negative: not stored) of the sequence in row rows[t] (int32; None: t) of
    `table`.  With cos and sin (float32 [positions, rot dim / 2]) keys are
    rotated by positions[t] (int32; None: index), and so are the queries q
    [tokens, heads, head dim] of the same tokens, which are returned (in
    q_out, which may be q).  With q_norm or k_norm ([head dim] weights in the
    cache's type) each head of the queries (the keys) is normed before it is
    rotated: x w / sqrt(mean x^2 + eps).  info: int32 [1], set to 1 on an index
    out of range."""
    _no_derivative("append_tokens", k, v, q, cache.k, cache.v, q_norm, k_norm)
    dtype, dev, dim = cache.dtype, cache.device, cache.head_dim
    n = k.shape[0]
    kp = _heads(k, "k", cache.kv_heads, dim, dtype, dev)
    vp = _heads(v, "v", cache.kv_heads, dim, dtype, dev)
    _need(v.shape[0] == n, "as many values as keys are needed")
    _need(table.dim() == 2, "table: [rows, pages of a row]")
    _need(q is not None or q_norm is None, "q_norm without queries")
    heads, qp, op = 0, (None, 0, 0), (None, 0, 0)
    if q is not None:
        heads = q.shape[1]
        qp = _heads(q, "q", heads, dim, dtype, dev)
        q_out = torch.empty((n, heads, dim), dtype=dtype, device=dev) if q_out is None else q_out
        op = _heads(q_out, "q_out", heads, dim, dtype, dev)
        _need(q.shape[0] == n and q_out.shape[0] == n, "as many queries as keys are needed")
    angles = (0, 0)
    if cos is not None:
        _need(sin is not None and cos.dim() == 2, "cos and sin: two [positions, rot dim / 2] tensors")
        angles = tuple(cos.shape)
    t = L.gnnshap_new_tokens(
        n, *kp, *vp, _vector(rows, "rows", torch.int32, (n,), dev), _vector(index, "index", torch.int32, (n,), dev),
        _vector(positions, "positions", torch.int32, (n,), dev), _vector(table, "table", torch.int32, None, dev),
        table.shape[0], table.shape[1], _vector(cos, "cos", torch.float32, angles, dev),
        _vector(sin, "sin", torch.float32, angles, dev), angles[0], 2 * angles[1], int(interleaved), heads, 0, *qp, *op,
        _vector(q_norm, "q_norm", dtype, (dim,), dev), _vector(k_norm, "k_norm", dtype, (dim,), dev), eps)
    _on(dev, L.gnnshap_cache_append, cache._c, t, _vector(info, "info", torch.int32, (1,), dev))
    return q_out


def _normed(q, k, q_norm, k_norm, cos, sin, positions, interleaved, eps):
    """The library's description of heads to norm and rotate, without outputs."""
    if q.dim() != 3 or not q.is_cuda or q.dtype not in _DTYPES:
        raise ValueError(f"q: a [tokens, heads, head dim] float32, float16 or bfloat16 tensor on a GPU is needed, got "
                         f"{q.dtype} {tuple(q.shape)} on {q.device}")
    n, heads, dim = q.shape
    dtype, dev = q.dtype, q.device
    kinds = [L.gnnshap_heads(heads, 0, *_heads(q, "q", heads, dim, dtype, dev)), L.gnnshap_heads()]
    if k is not None:
        kp = _heads(k, "k", None, dim, dtype, dev)
        _need(k.shape[0] == n, "as many keys as queries are needed")
        kinds[1] = L.gnnshap_heads(k.shape[1], 0, *kp)
    else:
        _need(k_norm is None, "k_norm without keys")
    angles = (0, 0)
    if cos is not None:
        _need(sin is not None and cos.dim() == 2, "cos and sin: two [positions, rot dim / 2] tensors")
        angles = tuple(cos.shape)
    return L.gnnshap_normed(
        _DTYPES[dtype], dim, n, *kinds, _vector(q_norm, "q_norm", dtype, (dim,), dev),
        _vector(k_norm, "k_norm", dtype, (dim,), dev), _vector(positions, "positions", torch.int32, (n,), dev),
        _vector(cos, "cos", torch.float32, angles, dev), _vector(sin, "sin", torch.float32, angles, dev), angles[0],
        2 * angles[1], int(interleaved), eps)


def norm_rotate(q, k=None, q_norm=None, k_norm=None, cos=None, sin=None, positions=None, interleaved=False, eps=1e-6,
                info=None):
    """gnnshap_norm_rotate: each head of the queries q [tokens, heads, head dim]
    and of the keys k (other heads, or None) normed and, with cos and sin
    (float32 [positions, rot dim / 2]), rotated by positions[t] (int32; None: t;
    negative: not rotated), as append_tokens does on the way into a cache.
    q_norm and k_norm: [head dim] weights in the heads' type; None: all 1.
    Returns both, new and contiguous (None for no keys).  info: int32 [1], set
    to 1 on a position out of range."""
    _no_derivative("norm_rotate (but for differentiable_norm_rotate)", q, k, q_norm, k_norm, cos, sin)
    a = _normed(q, k, q_norm, k_norm, cos, sin, positions, interleaved, eps)
    out = [None if x is None else torch.empty(x.shape, dtype=x.dtype, device=x.device) for x in (q, k)]
    for kind, x in zip((a.q, a.k), out):
        if x is not None:
            kind.out, kind.out_token_stride, kind.out_head_stride = x.data_ptr(), x.stride(0), x.stride(1)
    _on(q.device, L.gnnshap_norm_rotate, a, _vector(info, "info", torch.int32, (1,), q.device))
    return tuple(out)


def norm_rotate_backward(grad_q, grad_k, q, k=None, q_norm=None, k_norm=None, cos=None, sin=None, positions=None,
                         interleaved=False, eps=1e-6, weights=True, info=None):
    """gnnshap_norm_rotate_backward: the gradients by q, k, q_norm and k_norm of
    norm_rotate's outputs, whose gradients are grad_q and grad_k.  Returns the
    four, None where the input is None (with weights=False for both weights)."""
    _no_derivative("norm_rotate_backward", grad_q, grad_k, q, k, q_norm, k_norm, cos, sin)
    a = _normed(q, k, q_norm, k_norm, cos, sin, positions, interleaved, eps)
    dev, dtype, dim = q.device, q.dtype, q.shape[2]
    out, kinds = [], []
    for x, g, name in ((q, grad_q, "grad_q"), (k, grad_k, "grad_k")):
        if x is None:
            out.append(None)
            kinds.append(L.gnnshap_heads())
            continue
        gp = _heads(g, name, x.shape[1], dim, dtype, dev)
        _need(g.shape[0] == x.shape[0], f"{name} of as many tokens is needed")
        out.append(torch.empty(x.shape, dtype=dtype, device=dev))
        kinds.append(L.gnnshap_heads(x.shape[1], 0, *gp, out[-1].data_ptr(), out[-1].stride(0), out[-1].stride(1)))
    out += [torch.empty(dim, dtype=dtype, device=dev) if weights and w is not None else None for w in (q_norm, k_norm)]
    nbytes = L.gnnshap_norm_rotate_backward_workspace(a) if out[2] is not None or out[3] is not None else 0
    ws = torch.empty(nbytes, dtype=torch.uint8, device=dev) if nbytes else None
    _on(dev, L.gnnshap_norm_rotate_backward, a, *kinds, _ptr(out[2]), _ptr(out[3]),
        _vector(info, "info", torch.int32, (1,), dev), _ptr(ws), nbytes)
    return tuple(out)


class _NormRotate(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, q_norm, k_norm, cos, sin, positions, interleaved, eps):
        ctx.save_for_backward(q, k, q_norm, k_norm, cos, sin, positions)
        ctx.rest = interleaved, eps
        return norm_rotate(q, k, q_norm, k_norm, cos, sin, positions, interleaved, eps)

    @staticmethod
    def backward(ctx, grad_q, grad_k):
        # a node of its own costs about 30 us on the host: only where a second derivative may follow
        gradient = _NormRotateGradient.apply if _grad_enabled() else partial(_NormRotateGradient.forward, None)
        return (*gradient(grad_q, grad_k, *ctx.saved_tensors, *ctx.rest, any(ctx.needs_input_grad[2:4])),
                None, None, None, None, None)


class _NormRotateGradient(torch.autograd.Function):
    """The gradient as a node of its own, so that differentiating it again raises."""
    @staticmethod
    def forward(ctx, grad_q, grad_k, *rest):
        grads = (g if g is None or g.stride(2) == 1 else g.contiguous() for g in (grad_q, grad_k))
        return norm_rotate_backward(*grads, *rest)

    @staticmethod
    def backward(ctx, *grads):
        raise RuntimeError("differentiable_norm_rotate has a first derivative only")


def differentiable_norm_rotate(q, k=None, q_norm=None, k_norm=None, cos=None, sin=None, positions=None,
                               interleaved=False, eps=1e-6):
    """norm_rotate with its gradient by q, k, q_norm and k_norm (autograd), for
    training.  The gradient is of first order, and the angles have none: cos and
    sin that require a gradient are refused."""
    _no_derivative("differentiable_norm_rotate by cos and sin", cos, sin)
    return _NormRotate.apply(q, k, q_norm, k_norm, cos, sin, positions, interleaved, eps)


def attend(cache, q, table=None, lengths=None, max_length=None, shared_table=None, shared_lengths=None,
           max_shared=None, masks=None, num_players=None, first_player=0, scale=None, out=None, return_lse=False,
           info=None):
    """gnnshap_cache_attend: attention of one new token per row, q [rows,
    heads, head dim].  Row b sees lengths[b] tokens of row b of `table` and,
    before them, the shared part of its group: shared_lengths[g] tokens of row
    g of shared_table, whose rows are the groups of rows / groups consecutive
    rows.  max_length and max_shared bound the lengths (None: what the table's
    pages hold).  masks (int64 [rows, words], the sampler's bits): position
    first_player + j of the context is player j of num_players, seen where bit
    j is set; other positions are always seen.  scale:
    None for 1 / sqrt(head dim).  out must not overlap q.  Returns out, or (out, lse) with the log of
    the sum of exponentials, float32 [rows, heads]; a row that sees nothing
    has out 0 and lse -inf."""
    _no_derivative("attend", q, cache.k, cache.v)
    dtype, dev, dim = cache.dtype, cache.device, cache.head_dim
    qp = _heads(q, "q", None, dim, dtype, dev)
    rows, heads = q.shape[0], q.shape[1]
    out = torch.empty((rows, heads, dim), dtype=dtype, device=dev) if out is None else out
    op = _heads(out, "out", heads, dim, dtype, dev)
    _need(out.shape[0] == rows, "out of as many rows as q is needed")
    lse = torch.empty((rows, heads), dtype=torch.float32, device=dev) if return_lse else None
    width = shared_width = per = 0
    if table is not None:
        _need(table.dim() == 2 and table.shape[0] == rows and lengths is not None, "table: [rows, pages], with lengths")
        width = table.shape[1]
        max_length = width * cache.page_size if max_length is None else max_length
    if shared_table is not None:
        _need(shared_table.dim() == 2 and shared_lengths is not None, "shared_table: [groups, pages], with lengths")
        groups, shared_width = shared_table.shape
        _need(groups > 0 and rows % groups == 0, "rows that the groups divide are needed")
        per = rows // groups
        max_shared = shared_width * cache.page_size if max_shared is None else max_shared
    words = 0
    if masks is not None:
        _need(num_players is not None, "masks without num_players")
        words = masks.shape[-1]
    else:
        _need(not num_players, "players without masks")
        num_players = first_player = 0
    a = L.gnnshap_queries(
        rows, heads, 0, *qp, *op, _ptr(lse), _vector(table, "table", torch.int32, None, dev),
        _vector(lengths, "lengths", torch.int32, (rows,), dev), width, max_length or 0,
        _vector(shared_table, "shared_table", torch.int32, None, dev),
        _vector(shared_lengths, "shared_lengths", torch.int32, None if per == 0 else (rows // per,), dev), shared_width,
        max_shared or 0, max(per, 1) if shared_table is not None else 0,
        _vector(masks, "masks", torch.int64, (rows, words), dev), words, num_players, first_player,
        1.0 / math.sqrt(dim) if scale is None else scale)
    nbytes = L.gnnshap_cache_attend_workspace(cache._c, a)
    ws = torch.empty(nbytes, dtype=torch.uint8, device=dev) if nbytes else None
    _on(dev, L.gnnshap_cache_attend, cache._c, a, _vector(info, "info", torch.int32, (1,), dev), _ptr(ws), nbytes)
    return (out, lse) if return_lse else out


def _weights_of(t, name, rows, columns, device):
    """Checks float32 [rows, columns or more] with a contiguous last axis; its address and stride."""
    if (t.dim() != 2 or t.dtype != torch.float32 or t.device != device or t.shape[0] != rows or t.shape[1] < columns
            or (t.stride(1) != 1 and t.shape[1] > 1)):
        raise ValueError(f"{name}: a float32 [{rows}, {columns} or more] tensor on {device} with a contiguous last axis "
                         f"is needed, got {t.dtype} {tuple(t.shape)} with strides {t.stride()} on {t.device}")
    return t.data_ptr(), t.stride(0)


def attention_weights(cache, q, lse, table, lengths, weights, max_length=None, masks=None, num_players=None,
                      first_player=0, scale=None, info=None):
    """gnnshap_cache_weights: adds to weights [sequences, tokens] (float32) what
    the queries q [rows, heads, head dim], whose attention left lse (float32
    [rows, heads]), gave each token of their sequence, summed over rows and heads.
    The rows of q are, rows / sequences at a time, those of a row of `table`; row
    b sees its first lengths[b] (int32 [rows]) tokens: a new token's row all of
    them, a prompt's rows each those up to its own, coalitions all the prompt's
    through their masks (as for attend, position first_player + j of the sequence
    is player j).  max_length bounds the lengths (None: what the table's pages and
    the weights hold).  Returns weights."""
    _no_derivative("attention_weights", q, lse, cache.k, weights)
    dtype, dev, dim = cache.dtype, cache.device, cache.head_dim
    qp = _heads(q, "q", None, dim, dtype, dev)
    rows, heads = q.shape[0], q.shape[1]
    _need(table.dim() == 2 and (rows % table.shape[0] == 0 if table.shape[0] else rows == 0),
          "table: [sequences, pages], the rows a multiple of the sequences")
    seqs, width = table.shape
    max_length = min(width * cache.page_size, weights.shape[-1]) if max_length is None else max_length
    wp = _weights_of(weights, "weights", seqs, max_length, dev)
    words = 0
    if masks is not None:
        _need(num_players is not None, "masks without num_players")
        words = masks.shape[-1]
    else:
        _need(not num_players, "players without masks")
        num_players = first_player = 0
    a = L.gnnshap_observed(
        rows, heads, 0, *qp, _vector(lse, "lse", torch.float32, (rows, heads), dev),
        _vector(table, "table", torch.int32, None, dev), _vector(lengths, "lengths", torch.int32, (rows,), dev),
        max(rows // max(seqs, 1), 1), width, max_length, _vector(masks, "masks", torch.int64, (rows, words), dev), words,
        num_players, first_player, 1.0 / math.sqrt(dim) if scale is None else scale, *wp)
    nbytes = L.gnnshap_cache_weights_workspace(cache._c, a)
    ws = torch.empty(nbytes, dtype=torch.uint8, device=dev) if nbytes else None
    _on(dev, L.gnnshap_cache_weights, cache._c, a, _vector(info, "info", torch.int32, (1,), dev), _ptr(ws), nbytes)
    return weights


class Evicted(NamedTuple):
    kept: torch.Tensor          # int32 [sequences, keep]: former places of the kept tokens, rising; then -1
    lengths: torch.Tensor       # int32 [sequences]
    weights: torch.Tensor       # float32 [sequences, tokens]: the kept tokens', then 0


def evict_tokens(cache, table, lengths, weights, keep, first=0, recent=0, max_length=None, lengths_out=None,
                 weights_out=None, info=None):
    """gnnshap_cache_evict: cuts each sequence (a row of `table`, whose pages are
    its own, lengths int32 [sequences]) to `keep` tokens: its `first` and `recent`
    last ones and, of the others, those of the largest weights (float32
    [sequences, tokens], as attention_weights adds them up; of equal ones the
    lower place).  The kept tokens' keys and values move up in the cache, in their
    order.  max_length bounds the lengths (None: what the table's pages and the
    weights hold).  Returns an Evicted; lengths_out and weights_out may be given,
    and be lengths and weights themselves.  Columns of weights_out from
    max_length on are left as they are."""
    _no_derivative("evict_tokens", cache.k, cache.v, weights)
    dev = cache.device
    _need(table.dim() == 2, "table: [sequences, pages]")
    seqs, width = table.shape
    max_length = min(width * cache.page_size, weights.shape[-1]) if max_length is None else max_length
    wp = _weights_of(weights, "weights", seqs, max_length, dev)
    lengths_out = torch.empty(seqs, dtype=torch.int32, device=dev) if lengths_out is None else lengths_out
    weights_out = torch.empty((seqs, max_length), dtype=torch.float32, device=dev) if weights_out is None else weights_out
    op = _weights_of(weights_out, "weights_out", seqs, max_length, dev)
    _need(keep >= 1, "at least one token is kept")
    kept = torch.empty((seqs, keep), dtype=torch.int32, device=dev)
    a = L.gnnshap_eviction(seqs, _vector(table, "table", torch.int32, None, dev), width, max_length,
                           _vector(lengths, "lengths", torch.int32, (seqs,), dev), *wp, keep, first, recent,
                           kept.data_ptr(), _vector(lengths_out, "lengths_out", torch.int32, (seqs,), dev), *op)
    nbytes = L.gnnshap_cache_evict_workspace(cache._c, a)
    ws = torch.empty(nbytes, dtype=torch.uint8, device=dev) if nbytes else None
    _on(dev, L.gnnshap_cache_evict, cache._c, a, _vector(info, "info", torch.int32, (1,), dev), _ptr(ws), nbytes)
    return Evicted(kept, lengths_out, weights_out)


class TokenLogprobs(NamedTuple):
    logprob: torch.Tensor       # float32 [rows]: log probability of the given token
    entropy: torch.Tensor       # float32 [rows]
    lse: torch.Tensor           # float32 [rows]: log of the sum of exponentials
    rank: torch.Tensor          # int32 [rows]: logits larger than the given token's
    top_logprob: torch.Tensor   # float32 [rows, top], falling
    top_id: torch.Tensor        # int32 [rows, top]


def _check_logits(x):
    if x.dim() != 2 or not x.is_cuda or x.dtype not in _DTYPES or (x.stride(1) != 1 and x.shape[1] > 1):
        raise ValueError(f"logits: a [rows, vocabulary] float32, float16 or bfloat16 tensor on a GPU with a contiguous "
                         f"last axis is needed, got {x.dtype} {tuple(x.shape)} with strides {x.stride()} on {x.device}")
    return _DTYPES[x.dtype]


def _give_parts(a, maximum, log_sum, size, device):
    """Sets the two parts of lse, where they are given."""
    if maximum is not None:
        a.maximum = _vector(maximum, "maximum", torch.float32, size, device)
    if log_sum is not None:
        a.log_sum = _vector(log_sum, "log_sum", torch.float32, size, device)


def token_logprobs(logits, targets=None, top=0, info=None, maximum=None, log_sum=None):
    """gnnshap_token_logprobs of logits [rows, vocabulary]: log probability and
    rank of the tokens `targets` (int64 [rows]; negative or None: no token, 0
    and -1), entropy, and the `top` most likely tokens (at most 64; of equal
    logits the lowest token first).  Returns a TokenLogprobs.  maximum and
    log_sum (float32 [rows], if given) get the largest logit and the log of the
    sum of exp(x - maximum), for the gradient of logits far from 0."""
    _no_derivative("token_logprobs (but for differentiable_logprobs)", logits)
    dtype = _check_logits(logits)
    (rows, vocab), dev = logits.shape, logits.device
    logprob, entropy, lse = torch.empty((3, rows), dtype=torch.float32, device=dev).unbind(0)
    rank, top_id = torch.empty(rows * (top + 1), dtype=torch.int32, device=dev).split((rows, rows * top))
    r = TokenLogprobs(logprob, entropy, lse, rank, torch.empty((rows, top), dtype=torch.float32, device=dev),
                      top_id.view(rows, top))
    a = L.gnnshap_logits(dtype, top, rows, vocab, logits.data_ptr(), logits.stride(0),
                         _vector(targets, "targets", torch.int64, (rows,), dev), logprob.data_ptr(),
                         entropy.data_ptr(), lse.data_ptr(), rank.data_ptr(), r.top_logprob.data_ptr(),
                         top_id.data_ptr())
    _give_parts(a, maximum, log_sum, (rows,), dev)
    nbytes = L.gnnshap_token_logprobs_workspace(a)
    ws = torch.empty(nbytes, dtype=torch.uint8, device=dev) if nbytes else None
    _on(dev, L.gnnshap_token_logprobs, a, _vector(info, "info", torch.int32, (1,), dev), _ptr(ws), nbytes)
    return r


def token_logprobs_backward(logits, targets, lse, entropy=None, grad_logprob=None, grad_entropy=None, out=None,
                            info=None, maximum=None, log_sum=None):
    """gnnshap_token_logprobs_backward: the gradient by the logits of
    sum(grad_logprob * logprob) + sum(grad_entropy * entropy), in the logits'
    type.  lse and entropy as token_logprobs gave them; out may be the logits
    themselves.  With maximum and log_sum, as token_logprobs gave them, which
    are then read in place of lse, the gradient of logits far from 0 is as exact
    as that of others (by lse, p is off by 2^-24 |lse|)."""
    _no_derivative("token_logprobs_backward", logits, lse, entropy, grad_logprob, grad_entropy, maximum, log_sum)
    dtype = _check_logits(logits)
    (rows, vocab), dev = logits.shape, logits.device
    out = torch.empty((rows, vocab), dtype=logits.dtype, device=dev) if out is None else out
    _need(out.shape == logits.shape and out.dtype == logits.dtype and out.device == dev
          and (out.stride(1) == 1 or vocab == 1), "out: a tensor like the logits is needed")
    a = L.gnnshap_logits(dtype, 0, rows, vocab, logits.data_ptr(), logits.stride(0),
                         _vector(targets, "targets", torch.int64, (rows,), dev), None,
                         _vector(entropy, "entropy", torch.float32, (rows,), dev),
                         _vector(lse, "lse", torch.float32, (rows,), dev))
    _give_parts(a, maximum, log_sum, (rows,), dev)
    _on(dev, L.gnnshap_token_logprobs_backward, a,
        _vector(grad_logprob, "grad_logprob", torch.float32, (rows,), dev),
        _vector(grad_entropy, "grad_entropy", torch.float32, (rows,), dev), out.data_ptr(), out.stride(0),
        _vector(info, "info", torch.int32, (1,), dev))
    return out


class _Logprob(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, targets):
        maximum, log_sum = torch.empty((2, logits.shape[0]), dtype=torch.float32, device=logits.device).unbind(0)
        r = token_logprobs(logits, targets, maximum=maximum, log_sum=log_sum)
        logprob, entropy = r.logprob.data, r.entropy.data   # (autograd refuses to change views in place)
        ctx.save_for_backward(logits, targets, r.lse, entropy, maximum, log_sum)
        return logprob, entropy

    @staticmethod
    def backward(ctx, grad_logprob, grad_entropy):
        return _LogprobGradient.apply(*ctx.saved_tensors, grad_logprob, grad_entropy), None


class _LogprobGradient(torch.autograd.Function):
    """The gradient as a node of its own, so that differentiating it again (by
    the logits or the incoming gradients) raises and is not taken for 0."""
    @staticmethod
    def forward(ctx, logits, targets, lse, entropy, maximum, log_sum, grad_logprob, grad_entropy):
        grads = (None if g is None else g.float().contiguous() for g in (grad_logprob, grad_entropy))
        return token_logprobs_backward(logits, targets, lse, entropy, *grads, maximum=maximum, log_sum=log_sum)

    @staticmethod
    def backward(ctx, grad):
        raise RuntimeError("differentiable_logprobs has a first derivative only")


def differentiable_logprobs(logits, targets):
    """Log probabilities of `targets` (int64 [rows]) and entropies of logits
    [rows, vocabulary] with their gradient by the logits (autograd), for
    gradient attributions and training.  The gradient is of first order:
    differentiating it again raises."""
    return _Logprob.apply(logits, targets)


class LinearLogprobs(NamedTuple):
    logprob: torch.Tensor       # float32 [rows]: log probability of the given token
    entropy: torch.Tensor       # float32 [rows]
    lse: torch.Tensor           # float32 [rows]: log of the sum of exponentials
    maximum: torch.Tensor       # float32 [rows]: the largest logit
    log_sum: torch.Tensor       # float32 [rows]: log of the sum of exp(x - maximum)


def _linear(hidden, weight, targets, **outputs):
    """The library's description of hidden states [rows, width] and weights [vocabulary, width]."""
    if (hidden.dim() != 2 or not hidden.is_cuda or hidden.dtype not in _DTYPES
            or (hidden.stride(1) != 1 and hidden.shape[1] > 1)):
        raise ValueError(f"hidden: a [rows, width] float32, float16 or bfloat16 tensor on a GPU with a contiguous last "
                         f"axis is needed, got {hidden.dtype} {tuple(hidden.shape)} with strides {hidden.stride()} on "
                         f"{hidden.device}")
    (rows, width), dev = hidden.shape, hidden.device
    if (weight.dim() != 2 or weight.dtype != hidden.dtype or weight.device != dev or weight.shape[1] != width
            or (weight.stride(1) != 1 and width > 1)):
        raise ValueError(f"weight: a [vocabulary, {width}] {hidden.dtype} tensor on {dev} with a contiguous last axis "
                         f"is needed, got {weight.dtype} {tuple(weight.shape)} with strides {weight.stride()} on "
                         f"{weight.device}")
    return L.gnnshap_linear(_DTYPES[hidden.dtype], 0, rows, weight.shape[0], width, hidden.data_ptr(), hidden.stride(0),
                            weight.data_ptr(), weight.stride(0), _vector(targets, "targets", torch.int64, (rows,), dev),
                            **outputs)


def linear_logprobs(hidden, weight, targets=None, info=None):
    """gnnshap_linear_logprobs: what token_logprobs gives of the logits hidden
    [rows, width] @ weight [vocabulary, width]^T, without keeping them: log
    probabilities of the tokens `targets` (int64 [rows]; negative or None: no
    token, 0), entropies and lse, and its two parts for the gradient.  The logits
    are in fp32 and not rounded to the weights' type.  Returns a LinearLogprobs."""
    _no_derivative("linear_logprobs (but for differentiable_linear_logprobs)", hidden, weight)
    a = _linear(hidden, weight, targets)
    rows, dev = hidden.shape[0], hidden.device
    r = LinearLogprobs(*torch.empty((5, rows), dtype=torch.float32, device=dev).unbind(0))
    a.logprob, a.entropy, a.lse, a.maximum, a.log_sum = (x.data_ptr() for x in r)
    nbytes = L.gnnshap_linear_logprobs_workspace(a)
    ws = torch.empty(nbytes, dtype=torch.uint8, device=dev) if nbytes else None
    _on(dev, L.gnnshap_linear_logprobs, a, _vector(info, "info", torch.int32, (1,), dev), _ptr(ws), nbytes)
    return r


def linear_logprobs_backward(hidden, weight, targets, maximum, log_sum, entropy=None, grad_logprob=None,
                             grad_entropy=None, of_hidden=True, of_weight=True, info=None):
    """gnnshap_linear_logprobs_backward: the gradients by hidden and by weight
    (None for one that is not wanted) of sum(grad_logprob * logprob) +
    sum(grad_entropy * entropy), in their type; maximum, log_sum and entropy as
    linear_logprobs gave them.  The logits are computed again, a piece of the
    vocabulary at a time."""
    _no_derivative("linear_logprobs_backward", hidden, weight, maximum, log_sum, entropy, grad_logprob, grad_entropy)
    a = _linear(hidden, weight, targets)
    size, dev = (hidden.shape[0],), hidden.device
    _give_parts(a, maximum, log_sum, size, dev)
    a.entropy = _vector(entropy, "entropy", torch.float32, size, dev)
    out = [torch.empty(x.shape, dtype=x.dtype, device=dev) if wanted else None
           for x, wanted in ((hidden, of_hidden), (weight, of_weight))]
    nbytes = L.gnnshap_linear_logprobs_backward_workspace(a)
    ws = torch.empty(nbytes, dtype=torch.uint8, device=dev) if nbytes else None
    _on(dev, L.gnnshap_linear_logprobs_backward, a,
        _vector(grad_logprob, "grad_logprob", torch.float32, size, dev),
        _vector(grad_entropy, "grad_entropy", torch.float32, size, dev), _ptr(out[0]), hidden.shape[1], _ptr(out[1]),
        hidden.shape[1], _vector(info, "info", torch.int32, (1,), dev), _ptr(ws), nbytes)
    return tuple(out)


class _LinearLogprob(torch.autograd.Function):
    @staticmethod
    def forward(ctx, hidden, weight, targets):
        r = linear_logprobs(hidden, weight, targets)
        logprob, entropy = r.logprob.data, r.entropy.data   # (autograd refuses to change views in place)
        ctx.save_for_backward(hidden, weight, targets, r.maximum, r.log_sum, entropy)
        return logprob, entropy

    @staticmethod
    def backward(ctx, grad_logprob, grad_entropy):
        gradient = _LinearLogprobGradient.apply if _grad_enabled() else partial(_LinearLogprobGradient.forward, None)
        return (*gradient(*ctx.saved_tensors, grad_logprob, grad_entropy, *ctx.needs_input_grad[:2]), None)


class _LinearLogprobGradient(torch.autograd.Function):
    """The gradient as a node of its own, so that differentiating it again raises."""
    @staticmethod
    def forward(ctx, hidden, weight, targets, maximum, log_sum, entropy, grad_logprob, grad_entropy, *wanted):
        grads = (None if g is None else g.float().contiguous() for g in (grad_logprob, grad_entropy))
        return linear_logprobs_backward(hidden, weight, targets, maximum, log_sum, entropy, *grads, *wanted)

    @staticmethod
    def backward(ctx, *grads):
        raise RuntimeError("differentiable_linear_logprobs has a first derivative only")


def differentiable_linear_logprobs(hidden, weight, targets):
    """Log probabilities of `targets` (int64 [rows]) and entropies of the logits
    hidden @ weight^T with their gradient by hidden and weight (autograd), for
    training and attributions: neither pass keeps the logits.  The gradient is
    of first order: differentiating it again raises."""
    return _LinearLogprob.apply(hidden, weight, targets)


def _batches(rows, batch):
    """Bounds of batches of at most `batch` rows, of which the last has two at
    least: one row alone would be the full coalition, so the batch before it
    gives it one."""
    ends = list(range(batch, rows, batch)) + [rows]
    if len(ends) > 1 and rows - ends[-2] == 1:
        ends[-2] -= 1
    return list(zip([0] + ends[:-1], ends))


class AnswerExplainer:
    """Shapley values of prompt tokens for a model's answer (Alg. 1 of the
    paper with tokens as players): the sampler's coalitions, their values from
    the caller's model, the constrained least squares.

    `value(masks, num_players)` gives the model's value under each coalition,
    float32 [rows], such as the answer's log probability by `attend` and
    `token_logprobs`; masks are int64 [rows, words] (the sampler's bits).  It is
    called with batches of at most `batch` coalitions, of which the last one
    ends with the empty and the full coalition."""

    def __init__(self, value, device="cuda", batch=16384):
        _need(batch >= 2, "batches of at least two coalitions are needed")
        L.load()
        self.value, self.device, self.batch = value, torch.device(device), int(batch)

    def explain(self, num_players, num_samples, seed, stream_id=0, iterative_threshold=0):
        """Returns an AnswerExplanation, valid once the current stream has run."""
        dev = self.device
        plan, classes = L.gnnshap_plan_samples(int(num_players), int(num_samples), int(seed), int(stream_id),
                                               int(iterative_threshold))
        k, words, m = plan.num_rows, plan.words_per_row, plan.num_players
        masks = torch.zeros((k + 2, words), dtype=torch.int64, device=dev)   # then none and all
        masks[k + 1] = -1
        if m % 64:
            masks[k + 1, -1] = (1 << (m % 64)) - 1
        weights = torch.empty(k, dtype=torch.float32, device=dev)
        nbytes = L.gnnshap_sample_workspace(plan)
        ws = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=dev)
        _on(masks.device, L.gnnshap_sample_coalitions, plan, classes, masks.data_ptr(), weights.data_ptr(),
            ws.data_ptr(), ws.numel())
        y = torch.empty(k + 2, dtype=torch.float32, device=dev)
        for b, end in _batches(k + 2, self.batch):
            part = masks[b:end]
            got = self.value(part, m)
            _need(got.shape == (part.shape[0],) and got.dtype == torch.float32,
                  "value: one float32 number per coalition is needed")
            y[b:end] = got
        phi = torch.empty(m, dtype=torch.float32, device=dev)
        info = torch.empty(1, dtype=torch.int32, device=dev)
        nbytes = L.gnnshap_solve_workspace(plan)
        ws = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=dev)
        _on(masks.device, L.gnnshap_solve_wls, plan, classes, masks.data_ptr(), y.data_ptr(), y[k:].data_ptr(),
            phi.data_ptr(), info.data_ptr(), ws.data_ptr(), ws.numel())
        return AnswerExplanation(phi, y[:k], y[k:], masks[:k], weights, info, plan)


class AnswerExplanation(NamedTuple):
    phi: torch.Tensor           # float32 [players]
    y: torch.Tensor             # float32 [rows]: the coalitions' values
    f_empty_full: torch.Tensor  # float32 [2]
    masks: torch.Tensor         # int64 [rows, words]
    weights: torch.Tensor       # float32 [rows]
    info: torch.Tensor          # int32 [1], as gnnshap_solve_wls sets it
    plan: L.gnnshap_sample_plan
