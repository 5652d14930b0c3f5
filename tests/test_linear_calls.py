"""What the log probabilities from hidden states refuse, before any launch (CPU)."""
import ctypes

import pytest
import torch

from paper_2401_04829_amd import _lib as L
from paper_2401_04829_amd import answers as A

P = 4096   # an address that is never read


def _linear(**kw):
    return L.gnnshap_linear(**{**dict(dtype=2, num_rows=3, vocab=10, width=64, hidden=P, hidden_stride=64, weight=P,
                                      weight_stride=64, targets=P, entropy=P, maximum=P, log_sum=P), **kw})


@pytest.mark.parametrize("change,status", [
    (dict(dtype=3), L.EUNSUPPORTED), (dict(dtype=-1), L.EUNSUPPORTED), (dict(num_rows=-1), L.EINVAL),
    (dict(vocab=0), L.EINVAL), (dict(width=0), L.EINVAL), (dict(vocab=(1 << 30) + 1), L.EUNSUPPORTED),
    (dict(num_rows=(1 << 30) + 1), L.EUNSUPPORTED), (dict(width=(1 << 24) + 1), L.EUNSUPPORTED),
    (dict(hidden_stride=-1), L.EINVAL), (dict(weight_stride=-1), L.EINVAL)])
def test_calls_that_are_refused(change, status):
    lib, n = L.load(), ctypes.c_size_t()
    a = _linear(**change)
    assert lib.gnnshap_linear_logprobs_workspace(a, n) == status
    assert lib.gnnshap_linear_logprobs(a, None, P, 1 << 40, None) == status
    assert lib.gnnshap_linear_logprobs_backward_workspace(a, n) == status
    assert lib.gnnshap_linear_logprobs_backward(a, P, P, P, 64, P, 64, None, P, 1 << 40, None) == status
    assert lib.gnnshap_last_error()


def test_null_arrays_and_workspace():
    lib, n = L.load(), ctypes.c_size_t()
    for query in (lib.gnnshap_linear_logprobs_workspace, lib.gnnshap_linear_logprobs_backward_workspace):
        assert query(None, n) == L.EINVAL and query(_linear(), None) == L.EINVAL
    assert lib.gnnshap_linear_logprobs(_linear(hidden=None), None, P, 1 << 40, None) == L.EINVAL
    assert lib.gnnshap_linear_logprobs(_linear(weight=None), None, P, 1 << 40, None) == L.EINVAL
    assert lib.gnnshap_linear_logprobs(_linear(num_rows=0, hidden=None), None, None, 0, None) == L.OK
    assert lib.gnnshap_linear_logprobs_workspace(_linear(), n) == L.OK and n.value > 0
    assert lib.gnnshap_linear_logprobs(_linear(), None, P, n.value - 1, None) == L.ECAPACITY
    assert lib.gnnshap_linear_logprobs(_linear(), None, None, n.value, None) == L.ECAPACITY

    def backward(a, *args, out=(P, 64, P, 64), ws=(P, 1 << 40)):
        return lib.gnnshap_linear_logprobs_backward(a, *args, *out, None, *ws, None)
    for change in (dict(hidden=None), dict(weight=None), dict(maximum=None), dict(log_sum=None), dict(entropy=None)):
        assert backward(_linear(**change), P, P) == L.EINVAL
    for out in ((P, -1, P, 64), (P, 64, P, -1)):
        assert backward(_linear(), P, P, out=out) == L.EINVAL
    assert backward(_linear(), P, P, out=(None, 64, None, 64)) == L.OK
    assert lib.gnnshap_linear_logprobs_backward_workspace(_linear(), n) == L.OK and n.value > 0
    assert backward(_linear(), P, P, ws=(P, n.value - 1)) == L.ECAPACITY
    assert backward(_linear(), P, P, ws=(None, n.value)) == L.ECAPACITY


def test_more_threads_than_a_launch_takes_are_refused():
    lib, n = L.load(), ctypes.c_size_t()
    a = _linear(num_rows=1 << 30, vocab=1 << 30)
    assert lib.gnnshap_linear_logprobs_workspace(a, n) == L.EUNSUPPORTED
    assert lib.gnnshap_linear_logprobs(a, None, P, 1 << 60, None) == L.EUNSUPPORTED


def test_tensors_that_are_refused():
    x = torch.zeros((3, 64))
    for call in (lambda: A.linear_logprobs(x, x), lambda: A.differentiable_linear_logprobs(x, x, None),
                 lambda: A.linear_logprobs_backward(x, x, None, x[:, 0], x[:, 0])):
        with pytest.raises(ValueError, match="on a GPU"):
            call()
    with pytest.raises(ValueError, match="has no derivative"):
        A.linear_logprobs(x.requires_grad_(), x)
