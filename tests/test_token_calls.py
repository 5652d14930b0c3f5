"""What the token operators refuse, before any launch (CPU)."""
import ctypes

import pytest
import torch

from paper_2401_04829_amd import _lib as L
from paper_2401_04829_amd import answers as A

P = 4096   # an address that is never read


def _cache(**kw):
    return L.gnnshap_cache(**{**dict(dtype=2, kv_heads=2, head_dim=64, page_size=16, num_pages=4, page_stride=2048,
                                     slot_stride=128, head_stride=64, k=P, v=P), **kw})


def _tokens(**kw):
    return L.gnnshap_new_tokens(**{**dict(num_tokens=3, k=P, k_token_stride=128, k_head_stride=64, v=P,
                                          v_token_stride=128, v_head_stride=64, index=P, table=P, num_rows=1,
                                          table_width=4, cos=P, sin=P, num_positions=64, rot_dim=64), **kw})


def _queries(**kw):
    return L.gnnshap_queries(**{**dict(num_rows=4, heads=4, q=P, q_row_stride=256, q_head_stride=64, out=P,
                                       out_row_stride=256, out_head_stride=64, table=P, lengths=P, table_width=4,
                                       max_length=64, scale=0.125), **kw})


def _logits(**kw):
    return L.gnnshap_logits(**{**dict(dtype=0, top=2, num_rows=3, vocab=10, logits=P, row_stride=10, lse=P, entropy=P),
                               **kw})


BAD_CACHES = [(dict(dtype=3), L.EUNSUPPORTED), (dict(dtype=-1), L.EUNSUPPORTED), (dict(kv_heads=0), L.EINVAL),
              (dict(head_dim=0), L.EINVAL), (dict(head_dim=12), L.EUNSUPPORTED), (dict(head_dim=264), L.EUNSUPPORTED),
              (dict(page_size=0), L.EINVAL), (dict(num_pages=0), L.EINVAL), (dict(num_pages=1 << 31), L.EINVAL),
              (dict(k=None), L.EINVAL), (dict(v=None), L.EINVAL), (dict(slot_stride=-1), L.EINVAL)]


@pytest.mark.parametrize("change,status", BAD_CACHES)
def test_caches_that_are_refused(change, status):
    lib, n = L.load(), ctypes.c_size_t()
    c = _cache(**change)
    assert lib.gnnshap_cache_append(c, _tokens(), None, None) == status
    assert lib.gnnshap_cache_attend_workspace(c, _queries(), n) == status
    assert lib.gnnshap_cache_attend(c, _queries(), None, None, 0, None) == status
    assert lib.gnnshap_last_error()


@pytest.mark.parametrize("change,status", [
    (dict(num_tokens=-1), L.EINVAL), (dict(num_tokens=1 << 31), L.EUNSUPPORTED), (dict(sin=None), L.EINVAL),
    (dict(num_positions=0), L.EINVAL), (dict(rot_dim=63), L.EINVAL), (dict(rot_dim=66), L.EINVAL),
    (dict(rot_dim=-2), L.EINVAL), (dict(q=P, heads=4), L.EINVAL), (dict(q=P, q_out=P), L.EINVAL),
    (dict(num_rows=0), L.EINVAL), (dict(table_width=0), L.EINVAL), (dict(k=None), L.EINVAL), (dict(v=None), L.EINVAL),
    (dict(index=None), L.EINVAL), (dict(table=None), L.EINVAL)])
def test_tokens_that_are_refused(change, status):
    lib = L.load()
    assert lib.gnnshap_cache_append(_cache(), _tokens(**change), None, None) == status
    assert lib.gnnshap_cache_append(_cache(), None, None, None) == L.EINVAL
    assert lib.gnnshap_cache_append(None, _tokens(), None, None) == L.EINVAL
    assert lib.gnnshap_cache_append(_cache(), _tokens(num_tokens=0), None, None) == L.OK


@pytest.mark.parametrize("change,status", [
    (dict(num_rows=-1), L.EINVAL), (dict(num_rows=1 << 31), L.EUNSUPPORTED), (dict(heads=3), L.EINVAL),
    (dict(heads=0), L.EINVAL), (dict(scale=0.0), L.EINVAL), (dict(scale=float("nan")), L.EINVAL),
    (dict(lengths=None), L.EINVAL), (dict(max_length=65), L.EINVAL), (dict(max_length=-1), L.EINVAL),
    (dict(max_length=2 ** 31, table_width=2 ** 31), L.EUNSUPPORTED),
    (dict(shared_table=P, shared_lengths=P, shared_width=2, max_shared=32), L.EINVAL),
    (dict(shared_table=P, shared_lengths=P, shared_width=2, max_shared=32, rows_per_group=3), L.EINVAL),
    (dict(shared_table=P, shared_lengths=P, shared_width=2, max_shared=33, rows_per_group=4), L.EINVAL),
    (dict(shared_table=P, shared_width=2, max_shared=32, rows_per_group=4), L.EINVAL),
    (dict(num_players=5), L.EINVAL), (dict(num_players=65, masks=P, mask_words=1), L.EINVAL),
    (dict(num_players=-1), L.EINVAL), (dict(first_player=-1), L.EINVAL)])
def test_queries_that_are_refused(change, status):
    lib, n = L.load(), ctypes.c_size_t()
    assert lib.gnnshap_cache_attend_workspace(_cache(), _queries(**change), n) == status
    assert lib.gnnshap_cache_attend(_cache(), _queries(**change), None, P, 1 << 40, None) == status


def test_attention_workspace_and_null_arrays():
    lib, n = L.load(), ctypes.c_size_t()
    assert lib.gnnshap_cache_attend_workspace(_cache(), _queries(), None) == L.EINVAL
    for change in (dict(q=None), dict(out=None)):
        assert lib.gnnshap_cache_attend(_cache(), _queries(**change), None, None, 0, None) == L.EINVAL
    assert lib.gnnshap_cache_attend(_cache(), _queries(num_rows=0, q=None, out=None), None, None, 0, None) == L.OK
    big = dict(num_rows=1, table_width=1000, max_length=16000)
    assert lib.gnnshap_cache_attend_workspace(_cache(), _queries(**big), n) == L.OK and n.value > 0
    assert lib.gnnshap_cache_attend(_cache(), _queries(**big), None, P, n.value - 1, None) == L.ECAPACITY
    assert lib.gnnshap_cache_attend(_cache(), _queries(**big), None, None, n.value, None) == L.ECAPACITY


@pytest.mark.parametrize("change,status", [
    (dict(dtype=7), L.EUNSUPPORTED), (dict(num_rows=-1), L.EINVAL), (dict(vocab=0), L.EINVAL),
    (dict(num_rows=1 << 31), L.EUNSUPPORTED), (dict(vocab=(1 << 30) + 1), L.EUNSUPPORTED), (dict(top=-1), L.EINVAL),
    (dict(top=11), L.EINVAL), (dict(top=65, vocab=100), L.EINVAL), (dict(row_stride=-1), L.EINVAL)])
def test_logits_that_are_refused(change, status):
    lib, n = L.load(), ctypes.c_size_t()
    assert lib.gnnshap_token_logprobs_workspace(_logits(**change), n) == status
    assert lib.gnnshap_token_logprobs(_logits(**change), None, None, 0, None) == status
    assert lib.gnnshap_token_logprobs_backward(_logits(**change), P, P, P, 10, None, None) == status


def test_logprobs_workspace_and_null_arrays():
    lib, n = L.load(), ctypes.c_size_t()
    assert lib.gnnshap_token_logprobs_workspace(None, n) == L.EINVAL
    assert lib.gnnshap_token_logprobs_workspace(_logits(), None) == L.EINVAL
    assert lib.gnnshap_token_logprobs(_logits(logits=None), None, None, 0, None) == L.EINVAL
    assert lib.gnnshap_token_logprobs(_logits(logits=None, num_rows=0), None, None, 0, None) == L.OK
    one = dict(num_rows=1, vocab=100000, row_stride=100000)
    assert lib.gnnshap_token_logprobs_workspace(_logits(**one), n) == L.OK and n.value > 0
    assert lib.gnnshap_token_logprobs(_logits(**one), None, P, n.value - 1, None) == L.ECAPACITY
    assert lib.gnnshap_token_logprobs(_logits(**one), None, None, n.value, None) == L.ECAPACITY
    for call in (dict(lse=None), dict(entropy=None), dict(logits=None)):
        assert lib.gnnshap_token_logprobs_backward(_logits(**call), P, P, P, 10, None, None) == L.EINVAL
    assert lib.gnnshap_token_logprobs_backward(_logits(), P, P, None, 10, None, None) == L.EINVAL
    assert lib.gnnshap_token_logprobs_backward(_logits(), P, P, P, -1, None, None) == L.EINVAL


def test_tensors_that_are_refused():
    """The torch-facing calls check types, shapes and devices before they call the library."""
    x = torch.zeros((4, 16, 2, 64))
    with pytest.raises(ValueError):
        A.PagedCache(x, x)                              # not on a GPU
    with pytest.raises(ValueError):
        A.PagedCache(x, x.half())
    with pytest.raises(ValueError):
        A.PagedCache(x[0], x[0])
    with pytest.raises(ValueError):
        A.token_logprobs(torch.zeros((2, 5)), None)     # not on a GPU


@pytest.mark.parametrize("batch", [2, 3, 4, 7, 100])
def test_batches_of_coalitions(batch):
    """All rows once, in order, and the last two, the empty and the full coalition, in one batch."""
    for rows in range(2, 60):
        parts = A._batches(rows, batch)
        assert [b for b, _ in parts] == [0] + [e for _, e in parts[:-1]] and parts[-1][1] == rows
        sizes = [e - b for b, e in parts]
        assert all(1 <= n <= batch for n in sizes) and sizes[-1] >= 2


def test_gradient_needs_both_parts_of_lse():
    lib = L.load()
    for change in (dict(maximum=P), dict(log_sum=P), dict(lse=None, maximum=P), dict(lse=None, log_sum=P)):
        assert lib.gnnshap_token_logprobs_backward(_logits(**change), P, P, P, 10, None, None) == L.EINVAL
    both = dict(lse=None, maximum=P, log_sum=P)
    assert lib.gnnshap_token_logprobs_backward(_logits(**both, entropy=None), P, P, P, 10, None, None) == L.EINVAL
    assert lib.gnnshap_token_logprobs_backward(_logits(**both, num_rows=0), P, P, P, 10, None, None) == L.OK


def test_more_threads_than_a_launch_takes_are_refused():
    """HIP takes fewer than 2^32 threads along an axis of a launch: sizes past
    it are unsupported (and no launch of the call is made), those up to it get
    to the checks behind."""
    lib, n = L.load(), ctypes.c_size_t()
    # rows of a workgroup of 256 threads: 16 where rows are short, 4 to 1 where they are longer
    for vocab, top, rows in ((41, 2, 16), (64, 0, 16), (200, 2, 4), (1000, 0, 4), (1000, 2, 4), (20000, 2, 2), (100000, 2, 1)):
        a = dict(vocab=vocab, top=top, row_stride=vocab)
        over, upto = rows << 24, (rows << 24) - rows
        assert lib.gnnshap_token_logprobs_workspace(_logits(num_rows=over, **a), n) == L.EUNSUPPORTED, vocab
        assert lib.gnnshap_token_logprobs(_logits(num_rows=over, **a), None, P, 1 << 40, None) == L.EUNSUPPORTED
        assert lib.gnnshap_token_logprobs_workspace(_logits(num_rows=upto, **a), n) == L.OK
    # the gradient: x threads side by side, 256 / x rows
    for vocab, x in ((300, 128), (1025, 256), (50000, 256)):
        a = _logits(num_rows=(1 << 32) // x * (256 // x), vocab=vocab, row_stride=vocab)
        assert lib.gnnshap_token_logprobs_backward(a, P, P, P, vocab, None, None) == L.EUNSUPPORTED, vocab
    # a token's heads: 1 to 16 threads side by side in 16 bits
    for dim, x in ((256, 16), (128, 8), (8, 1)):
        c, t = _cache(head_dim=dim), _tokens(num_tokens=min((1 << 32) // x, 1 << 31), rot_dim=0)
        assert lib.gnnshap_cache_append(c, t, None, None) == L.EUNSUPPORTED, dim
    # attention: a wavefront to a row and kv head
    a = dict(num_rows=1 << 25, lengths=P, max_length=16, table_width=1)
    assert lib.gnnshap_cache_attend_workspace(_cache(), _queries(**a), n) == L.EUNSUPPORTED
    assert lib.gnnshap_cache_attend(_cache(), _queries(**a), None, None, 0, None) == L.EUNSUPPORTED
    assert lib.gnnshap_cache_attend_workspace(_cache(), _queries(**dict(a, num_rows=(1 << 25) - 2)), n) == L.OK
    # the join: one to a row and head (here of no context)
    a = dict(table=None, num_rows=1 << 24)
    assert lib.gnnshap_cache_attend_workspace(_cache(), _queries(**a), n) == L.EUNSUPPORTED
    assert lib.gnnshap_cache_attend(_cache(), _queries(**a), None, None, 0, None) == L.EUNSUPPORTED
    assert lib.gnnshap_cache_attend_workspace(_cache(), _queries(**dict(a, num_rows=(1 << 24) - 1)), n) == L.OK


@pytest.mark.parametrize("scale,status", [(1e39, L.EINVAL), (-1e39, L.EINVAL), (float("inf"), L.EINVAL), (3e38, L.EINVAL),
                                          (2e38, L.OK), (-0.125, L.OK), (1e-50, L.OK)])
def test_scales_that_fp32_cannot_hold_are_refused(scale, status):
    lib, n = L.load(), ctypes.c_size_t()
    assert lib.gnnshap_cache_attend_workspace(_cache(), _queries(scale=scale), n) == status
    if status:
        assert lib.gnnshap_cache_attend(_cache(), _queries(scale=scale), None, None, 0, None) == status


def test_queries_as_their_own_output_are_refused():
    """Where a result is not finite a query is read again after outputs have been written."""
    assert L.load().gnnshap_cache_attend(_cache(), _queries(q=P, out=P), None, None, 0, None) == L.EINVAL
    assert b"out is q" in L.load().gnnshap_last_error()
