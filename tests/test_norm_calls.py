"""What the norm of heads refuses, before any launch (CPU)."""
import ctypes

import pytest
import torch

from paper_2401_04829_amd import _lib as L
from paper_2401_04829_amd import answers as A

P = 4096   # an address that is never read


def _heads(**kw):
    return L.gnnshap_heads(**{**dict(heads=4, x=P, token_stride=256, head_stride=64, out=P, out_token_stride=256,
                                     out_head_stride=64), **kw})


def _normed(**kw):
    return L.gnnshap_normed(**{**dict(dtype=2, head_dim=64, num_tokens=3, q=_heads(), k=_heads(heads=2), q_norm=P,
                                      k_norm=P, cos=P, sin=P, num_positions=64, rot_dim=64, eps=1e-6), **kw})


@pytest.mark.parametrize("change,status", [
    (dict(dtype=3), L.EUNSUPPORTED), (dict(dtype=-1), L.EUNSUPPORTED), (dict(head_dim=0), L.EINVAL),
    (dict(head_dim=12), L.EUNSUPPORTED), (dict(head_dim=264), L.EUNSUPPORTED), (dict(num_tokens=-1), L.EINVAL),
    (dict(num_tokens=1 << 31), L.EUNSUPPORTED), (dict(q=_heads(heads=-1)), L.EINVAL),
    (dict(k=_heads(heads=300000)), L.EUNSUPPORTED), (dict(sin=None), L.EINVAL), (dict(num_positions=0), L.EINVAL),
    (dict(rot_dim=63), L.EINVAL), (dict(rot_dim=66), L.EINVAL), (dict(rot_dim=-2), L.EINVAL),
    (dict(eps=-1e-6), L.EINVAL), (dict(eps=float("nan")), L.EINVAL), (dict(eps=1e39), L.EINVAL),
    (dict(q=_heads(x=None)), L.EINVAL)])
def test_heads_that_are_refused(change, status):
    lib, n, g = L.load(), ctypes.c_size_t(), _heads()
    a = _normed(**change)
    assert lib.gnnshap_norm_rotate(a, None, None) == status
    assert lib.gnnshap_norm_rotate_backward(a, g, _heads(heads=2), P, P, None, P, 1 << 40, None) == status
    if "q" not in change or change["q"].heads < 0:
        assert lib.gnnshap_norm_rotate_backward_workspace(a, n) == status


def test_null_arrays_and_workspace():
    lib, n = L.load(), ctypes.c_size_t()
    assert lib.gnnshap_norm_rotate(None, None, None) == L.EINVAL
    assert lib.gnnshap_norm_rotate(_normed(q=_heads(out=None)), None, None) == L.EINVAL
    assert lib.gnnshap_norm_rotate(_normed(num_tokens=0, q=_heads(x=None, out=None)), None, None) == L.OK
    assert lib.gnnshap_norm_rotate(_normed(q=_heads(heads=0), k=_heads(heads=0)), None, None) == L.OK
    assert lib.gnnshap_norm_rotate_backward_workspace(_normed(), None) == L.EINVAL
    assert lib.gnnshap_norm_rotate_backward_workspace(_normed(), n) == L.OK and n.value > 0
    two = _heads(heads=2)
    for g, h in ((None, two), (_heads(), None), (_heads(heads=3), two), (_heads(x=None), two), (_heads(out=None), two)):
        assert lib.gnnshap_norm_rotate_backward(_normed(), g, h, P, P, None, P, n.value, None) == L.EINVAL
    assert lib.gnnshap_norm_rotate_backward(_normed(), _heads(), two, P, P, None, P, n.value - 1, None) == L.ECAPACITY
    assert lib.gnnshap_norm_rotate_backward(_normed(), _heads(), two, P, None, None, None, n.value, None) == L.ECAPACITY
    # more threads than a launch takes: 8 lanes to a head of 64 bf16 elements in packs of 4
    assert lib.gnnshap_norm_rotate(_normed(num_tokens=(1 << 31) - 1, rot_dim=8), None, None) == L.EUNSUPPORTED


@pytest.mark.parametrize("change", [dict(norm_eps=-1.0), dict(norm_eps=float("inf")), dict(norm_eps=float("nan"))])
@pytest.mark.parametrize("which", ["q_norm", "k_norm"])
def test_norms_on_the_way_into_the_cache_that_are_refused(which, change):
    lib = L.load()
    c = L.gnnshap_cache(dtype=2, kv_heads=2, head_dim=64, page_size=16, num_pages=4, page_stride=2048, slot_stride=128,
                        head_stride=64, k=P, v=P)
    t = dict(num_tokens=0, index=P, table=P, num_rows=1, table_width=4)
    assert lib.gnnshap_cache_append(c, L.gnnshap_new_tokens(**t, **change), None, None) == L.OK   # not read
    assert lib.gnnshap_cache_append(c, L.gnnshap_new_tokens(**t, **change, **{which: P}), None, None) == L.EINVAL


def test_tensors_that_are_refused():
    x = torch.zeros((3, 4, 64))
    for call in (A.norm_rotate, A.differentiable_norm_rotate, lambda q: A.norm_rotate_backward(q, None, q)):
        with pytest.raises(ValueError, match="on a GPU"):
            call(x)
    with pytest.raises(ValueError, match="has no derivative"):
        A.norm_rotate(x.requires_grad_())
    with pytest.raises(ValueError, match="has no derivative"):
        A.norm_rotate_backward(x.detach(), None, x)


def test_a_norm_of_queries_needs_queries():
    c = A.PagedCache.__new__(A.PagedCache)
    c.k = c.v = torch.zeros((4, 16, 2, 64))
    c.kv_heads, c.head_dim, c.page_size, c.dtype, c.device, c._c = 2, 64, 16, torch.float32, torch.device("cpu"), None
    x, at = torch.zeros((3, 2, 64)), torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError, match="q_norm without queries"):
        A.append_tokens(c, x, x, at[None], at, q_norm=torch.ones(64))
