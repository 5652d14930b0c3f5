"""Torch-facing calls that explain a token model's answer.

The players are tokens of a prompt.  Their keys and values are cached once
(`append_tokens` into a `PagedCache`); under a coalition, the new token
attends over the cached prompt, seeing the positions its mask keeps, and over
tokens of its own (`attend`); the answer's log probability is the coalition's
value (`token_logprobs`), from which `AnswerExplainer` takes the Shapley
values with the library's sampler and least squares.

Torch provides device memory and streams; the work runs in libgnnshap.so on
the current stream.  Every tensor must be on the cache's (the logits') device.
Of these calls only `differentiable_logprobs` has a derivative: the others
refuse tensors that require a gradient (unless under torch.no_grad()) or carry
a tangent.
"""
import math
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
                  q_out=None, info=None):
    """gnnshap_cache_append: writes keys and values [tokens, kv heads, head
    dim] of new tokens into the cache, token t at place index[t] (int32;
    negative: not stored) of the sequence in row rows[t] (int32; None: t) of
    `table`.  With cos and sin (float32 [positions, rot dim / 2]) keys are
    rotated by positions[t] (int32; None: index), and so are the queries q
    [tokens, heads, head dim] of the same tokens, which are returned (in
    q_out, which may be q).  info: int32 [1], set to 1 on an index out of
    range."""
    _no_derivative("append_tokens", k, v, q, cache.k, cache.v)
    dtype, dev, dim = cache.dtype, cache.device, cache.head_dim
    n = k.shape[0]
    kp = _heads(k, "k", cache.kv_heads, dim, dtype, dev)
    vp = _heads(v, "v", cache.kv_heads, dim, dtype, dev)
    _need(v.shape[0] == n, "as many values as keys are needed")
    _need(table.dim() == 2, "table: [rows, pages of a row]")
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
        _vector(sin, "sin", torch.float32, angles, dev), angles[0], 2 * angles[1], int(interleaved), heads, 0, *qp, *op)
    _on(dev, L.gnnshap_cache_append, cache._c, t, _vector(info, "info", torch.int32, (1,), dev))
    return q_out


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
        ctx.save_for_backward(logits, targets, r.lse, r.entropy, maximum, log_sum)
        return r.logprob, r.entropy

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
