"""token_logprobs under autograd: the gradients that a training program gets, against the same computed by autograd in 64 bits, and what
is refused.  Tolerances as derived in test_gpu_outputs.py."""
import math

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from paper_2311_04996_amd import token_logprobs, token_logprobs_backward  # noqa: E402
from test_gpu_outputs import DT, backward64, close, gen, loss64, randn, round_off, some_tokens  # noqa: E402


def weights(g, x, tokens, top):
    lead = x.shape[:-1]
    return dict(gl=randn(g, *tokens.shape) if tokens is not None else None, gs=randn(g, *lead), gh=randn(g, *lead), gt=randn(g, *lead, top) if top else None)


def loss_of(r, w):
    pairs = ((r.logprobs, w["gl"]), (r.lse, w["gs"]), (r.entropy, w["gh"]), (r.top_logprobs, w["gt"]))
    return sum((a * c).sum() for a, c in pairs if a is not None and c is not None)


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("v", [2, 29, 129, 1000, 2048, 2049, 30000])
def test_a_loss_of_token_logprobs_has_its_gradient(v, dt):
    g = gen(v, 200)
    for rows, given, top in ((1, 1, 0), (7, 3, 2), (5, 0, 1)):
        x = (randn(g, rows, v) * 3).to(DT[dt]).requires_grad_()
        tokens = some_tokens(g, rows, v, given) if given else None
        w = weights(g, x, tokens, top)
        r = token_logprobs(x, tokens, top=top)
        plain = token_logprobs(x.detach(), tokens, top=top)
        for name, a, c in zip(r._fields, r, plain):                                # the same results, and no more constants than said
            assert (a is None) == (c is None) and (a is None or torch.equal(a, c))
            assert a is None or a.requires_grad == (name in ("logprobs", "lse", "entropy", "top_logprobs"))
            assert c is None or not c.requires_grad
        loss_of(r, w).backward()
        want, tol = backward64(x.detach(), tokens, r.top_ids, w["gl"], w["gs"], w["gh"], w["gt"])
        close(x.grad, want, tol + round_off(want, x.dtype))
        assert torch.equal(x.grad, token_logprobs_backward(x.detach(), plain, tokens, grad_logprobs=w["gl"], grad_lse=w["gs"], grad_entropy=w["gh"], grad_top=w["gt"]))
        x64 = x.detach().double().cpu().requires_grad_()                           # the formula against autograd's own
        loss64(x64, tokens, r.top_ids, w["gl"], w["gs"], w["gh"], w["gt"]).backward()
        close(x.grad, x64.grad.cuda(), tol + round_off(want, x.dtype))


@pytest.mark.parametrize("name", ["logprobs", "lse", "entropy", "top_logprobs"])
def test_one_result_alone_with_an_expanded_gradient(name):
    """... of scores that are no leaf but a view.  (The gradient of a sum is one number, expanded.)"""
    g = gen(201)
    x = randn(g, 6, 129).requires_grad_()
    tokens = some_tokens(g, 6, 129, 3)
    r = token_logprobs((x * 2.0).view(2, 3, 129), tokens.view(2, 3, 3), top=2)
    (got,) = torch.autograd.grad(getattr(r, name).sum(), x)
    one = {n: torch.ones(s, device="cuda") if n == name else None for n, s in (("logprobs", (6, 3)), ("lse", 6), ("entropy", 6), ("top_logprobs", (6, 2)))}
    want, tol = backward64((x * 2.0).detach(), tokens, r.top_ids.view(6, 2), one["logprobs"], one["lse"], one["entropy"], one["top_logprobs"])
    close(got, 2 * want, 2 * tol + round_off(2 * want, torch.float32))


def test_one_token_per_row():
    x = randn(gen(208), 6, 129).requires_grad_()
    t = torch.arange(6, dtype=torch.int32, device="cuda")
    r = token_logprobs(x, t)
    assert r.logprobs.shape == (6,)
    (got,) = torch.autograd.grad(r.logprobs.sum(), x)
    want, tol = backward64(x.detach(), t[:, None], None, torch.ones(6, 1), None, None, None)
    close(got, want, tol)


def test_padded_batches_have_no_gradient_behind_a_length():
    g = gen(202)
    lengths = torch.tensor([5, 0, 3], dtype=torch.int32, device="cuda")
    valid = torch.arange(5, device="cuda")[None] < lengths[:, None]
    x = randn(g, 3, 5, 300)
    x[~valid] = math.nan
    x.requires_grad_()
    tokens = some_tokens(g, 15, 300, 2).view(3, 5, 2)
    r = token_logprobs(x, tokens, top=2, lengths=lengths)
    w = weights(g, x, tokens, 2)
    loss_of(r, w).backward()
    assert bool((x.grad[~valid] == 0).all())
    want, tol = backward64(x.detach(), tokens, r.top_ids, w["gl"], w["gs"], w["gh"], w["gt"])
    close(x.grad[valid], want[valid], tol[valid])


def test_nothing_is_recorded_where_nothing_is_asked_for():
    x = randn(gen(203), 4, 50).requires_grad_()
    with torch.no_grad():
        assert not any(t is not None and t.requires_grad for t in token_logprobs(x, top=2))
    assert not any(t is not None and t.requires_grad for t in token_logprobs(x.detach(), top=2))
    # the function for the gradient takes what the recorded call returned, too
    r = token_logprobs(x)
    a = token_logprobs_backward(x, r, grad_lse=torch.ones(4, device="cuda"))
    assert not a.requires_grad and torch.equal(a, torch.autograd.grad(r.lse.sum(), x)[0])


def test_what_autograd_cannot_do_is_told():
    g = gen(204)
    x = randn(g, 4, 50).requires_grad_()
    r = token_logprobs(x)
    first = torch.autograd.grad(r.lse.sum(), x, create_graph=True)[0]
    with pytest.raises(RuntimeError):                                              # no second derivative
        first.sum().backward()
    y = x * 1.0
    r = token_logprobs(y)
    y.mul_(2.0)                                                                    # the scores are no longer what they were
    with pytest.raises(RuntimeError, match="modified by an inplace"):
        r.lse.sum().backward()


def test_on_another_stream():
    """The forward call on a stream of its own; the loss, and the rest of the backward pass, on the current one."""
    g = gen(205)
    x = randn(g, 40, 40000).requires_grad_()
    tokens = some_tokens(g, 40, 40000, 1)
    (want,) = torch.autograd.grad(token_logprobs(x, tokens).logprobs.mean(), x)
    stream = torch.cuda.Stream()
    for _ in range(3):
        stream.wait_stream(torch.cuda.current_stream())
        r = token_logprobs(x, tokens, stream=stream)
        torch.cuda.current_stream().wait_stream(stream)
        (got,) = torch.autograd.grad(r.logprobs.mean(), x)
        assert torch.equal(got, want)


def test_what_autograd_keeps_is_known_to_the_stream_that_reads_it(monkeypatch):
    """The backward pass reads scores, tokens and lengths on the given stream after the program may have let go of them: their memory is
    not another's before that stream is done."""
    told = []
    real = torch.Tensor.record_stream
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: (told.append((t.data_ptr(), s)), real(t, s))[1])
    x = randn(gen(209), 2, 3, 50).requires_grad_()
    tokens, lengths = torch.zeros((2, 3, 1), dtype=torch.int32, device="cuda"), torch.tensor([3, 1], dtype=torch.int32, device="cuda")
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    token_logprobs(x, tokens, lengths=lengths, stream=stream)
    assert [(t.data_ptr(), stream) for t in (x, tokens, lengths)] == told
    torch.cuda.synchronize()


def test_in_a_graph_the_gradient_is_called_itself():
    g = gen(206)
    x = randn(g, 6, 3000).requires_grad_()
    tokens, ones = some_tokens(g, 6, 3000, 1), torch.ones(6, 1, device="cuda")
    (want,) = torch.autograd.grad(token_logprobs(x, tokens).logprobs.sum(), x)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph), torch.no_grad():
        r = token_logprobs(x, tokens)
        d = token_logprobs_backward(x, r, tokens, grad_logprobs=ones)
    for _ in range(3):
        d.zero_()
        graph.replay()
        again = torch.autograd.grad(token_logprobs(x, tokens).logprobs.sum(), x)[0]
        torch.cuda.synchronize()
        assert torch.equal(d, want) and torch.equal(again, want)


def test_a_captured_backward_pass_is_refused():
    """The function that autograd calls says so before it does anything; the stream's state is the caller's to say here."""
    from unittest import mock
    x = randn(gen(207), 4, 50).requires_grad_()
    r = token_logprobs(x)
    with mock.patch("torch.cuda.is_current_stream_capturing", lambda: True), pytest.raises(RuntimeError, match="token_logprobs_backward"):
        r.lse.sum().backward()
    assert x.grad is None
    r.entropy.sum().backward()
    assert bool(torch.isfinite(x.grad).all())
