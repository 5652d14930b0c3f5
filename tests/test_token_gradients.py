"""What the token operators' calls tell autograd (CPU: torch's own functions
stand in for the library's)."""
import pytest
import torch

from paper_2401_04829_amd import answers as A


@pytest.fixture
def stand_ins(monkeypatch):
    def forward(x, targets=None, top=0, info=None, **_):
        logp = torch.log_softmax(x, 1)
        entropy = -(logp.exp() * logp).sum(1)
        return A.TokenLogprobs(logp.gather(1, targets[:, None])[:, 0], entropy, torch.logsumexp(x, 1), None, None, None)

    def backward(x, targets, lse, entropy=None, grad_logprob=None, grad_entropy=None, out=None, info=None, **_):
        x, lse = x.detach(), lse.detach()             # the library gets addresses: its result has no graph
        logp = x - lse[:, None]
        d = torch.nn.functional.one_hot(targets, x.shape[1]) - logp.exp()
        return (grad_logprob[:, None] * d - grad_entropy[:, None] * logp.exp() * (logp + entropy[:, None])).detach()
    monkeypatch.setattr(A, "token_logprobs", forward)
    monkeypatch.setattr(A, "token_logprobs_backward", backward)


def test_a_second_derivative_raises(stand_ins):
    """A gradient penalty through differentiable_logprobs would lack the
    second derivative's terms, so it is refused."""
    gen = torch.Generator().manual_seed(1)
    x, t = torch.randn((3, 5), generator=gen), torch.tensor([0, 4, 2])
    u = torch.ones(3, requires_grad=True)             # weighs the rows
    for of_logits in (True, False):                   # the first gradient depends on w (and u): its logits (their weights)
        w = torch.ones(5, requires_grad=True)
        logp, entropy = A.differentiable_logprobs(x * w, t)
        first, = torch.autograd.grad((u * (logp + entropy)).sum(), w, create_graph=True)
        y = (x * w.detach()).requires_grad_()
        logp = torch.log_softmax(y, 1)
        (logp.gather(1, t[:, None]).sum() - (logp.exp() * logp).sum()).backward()
        assert torch.allclose(first, (y.grad * x).sum(0), atol=1e-6)
        with pytest.raises(RuntimeError, match="first derivative only"):
            torch.autograd.grad(first.pow(2).sum(), w if of_logits else u)


def test_a_second_derivative_raises_where_another_path_has_one(stand_ins):
    """Where torch differentiates a part of the path twice, no error of its own
    would tell that the rest is missing."""
    gen = torch.Generator().manual_seed(2)
    x, t = torch.randn((3, 5), generator=gen, requires_grad=True), torch.tensor([0, 4, 2])
    logp, _ = A.differentiable_logprobs(x * x, t)
    first, = torch.autograd.grad(logp.sum() + x.pow(3).sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="first derivative only"):
        first.sum().backward()


def test_a_first_derivative_with_a_graph_and_without(stand_ins):
    x, t = torch.randn((3, 5), generator=torch.Generator().manual_seed(3), requires_grad=True), torch.tensor([0, 4, 2])
    a, = torch.autograd.grad(A.differentiable_logprobs(x, t)[0].sum(), x)
    b, = torch.autograd.grad(A.differentiable_logprobs(x, t)[0].sum(), x, create_graph=True)
    assert not a.requires_grad and torch.equal(a, b)
    A.differentiable_logprobs(x, t)[0].sum().backward()
    assert torch.equal(x.grad, a)


class _Reached(Exception):
    pass


@pytest.fixture
def calls(monkeypatch):
    """Each call without a derivative, given its floating tensors by name, up
    to where the library would be called."""
    def reached(*_):
        raise _Reached
    for name in ("gnnshap_cache_append", "gnnshap_cache_attend_workspace", "gnnshap_token_logprobs_workspace",
                 "gnnshap_token_logprobs_backward"):
        monkeypatch.setattr(A.L, name, reached)
    monkeypatch.setattr(A, "_on", reached)
    monkeypatch.setattr(A, "_check_logits", lambda x: 0)
    i32 = dict(dtype=torch.int32)
    t, table = torch.zeros(3, dtype=torch.int64), torch.zeros((3, 1), **i32)

    def cache(x):
        c = A.PagedCache.__new__(A.PagedCache)
        c.k, c.v, c.kv_heads, c.head_dim, c.page_size = x["ck"], x["cv"], 2, 8, 4
        c.dtype, c.device, c._c = torch.float32, torch.device("cpu"), None
        return c
    return {
        "append": (dict(k=(3, 2, 8), v=(3, 2, 8), q=(3, 4, 8), ck=(1, 4, 2, 8), cv=(1, 4, 2, 8)),
                   lambda x: A.append_tokens(cache(x), x["k"], x["v"], table, torch.zeros(3, **i32), q=x["q"])),
        "attend": (dict(q=(3, 4, 8), ck=(1, 4, 2, 8), cv=(1, 4, 2, 8)),
                   lambda x: A.attend(cache(x), x["q"], table, torch.zeros(3, **i32))),
        "logprobs": (dict(x=(3, 5)), lambda x: A.token_logprobs(x["x"], t)),
        "backward": (dict(x=(3, 5), lse=(3,), entropy=(3,), gl=(3,), ge=(3,)),
                     lambda x: A.token_logprobs_backward(x["x"], t, x["lse"], x["entropy"], x["gl"], x["ge"]))}


@pytest.mark.parametrize("name", ["append", "attend", "logprobs", "backward"])
def test_calls_without_a_derivative_refuse_what_needs_one(calls, name):
    shapes, call = calls[name]
    x = {k: torch.zeros(s) for k, s in shapes.items()}
    with pytest.raises(_Reached):
        call(x)
    for one in shapes:
        y = dict(x, **{one: torch.zeros(shapes[one], requires_grad=True)})
        with pytest.raises(ValueError, match="has no derivative"):
            call(y)
        with torch.no_grad(), pytest.raises(_Reached):
            call(y)
        with pytest.raises(_Reached):
            call({k: v.detach() for k, v in y.items()})
        with torch.autograd.forward_ad.dual_level():
            with pytest.raises(_Reached):
                call(x)
            with pytest.raises(ValueError, match="carries a tangent"):
                call(dict(x, **{one: torch.autograd.forward_ad.make_dual(x[one], torch.ones(shapes[one]))}))
