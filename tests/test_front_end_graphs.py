"""The autograd front end around the library's calls, on CPU tensors with the calls themselves left out: what it remembers of living losses,
and what that costs."""
import gc
import sys

import pytest
import torch

from paper_2511_17599_amd import binding as B
from paper_2511_17599_amd import torch_api as A


@pytest.fixture
def capturing(monkeypatch):
    """The front end on CPU tensors; the returned list says whether a capture is to be seen."""
    state = [False]
    monkeypatch.setattr(A, "_capturing", lambda tensor: state[0])
    monkeypatch.setattr(A, "_stream", lambda device: 0)
    monkeypatch.setattr(A, "_prepare", lambda H, W, y: (H.reshape(-1, H.shape[-1]), W, y.reshape(-1)))
    monkeypatch.setattr(A, "_operands", lambda H, W: (H.reshape(-1, H.shape[-1]), W))
    monkeypatch.setattr(A, "_launch", lambda *args: None)
    for name in ("flce_forward", "flce_backward_device_grad", "flce_forward_rows", "flce_backward_rows"):
        monkeypatch.setattr(B, name, lambda *args: B.FLCE_OK)
    return state


def case():
    H, W = torch.randn(4, 8, requires_grad=True), torch.randn(30, 8, requires_grad=True)
    return H, W, torch.zeros(4, dtype=torch.int64), (torch.zeros(4, 2, dtype=torch.int64), torch.zeros(4, 2))


def test_losses_are_remembered_as_long_as_their_graphs_live(capturing):
    H, W, y, lists = case()
    before = len(A._eager_nodes)
    losses = [A.linear_cross_entropy(H, W, y), 2 * A.linear_cross_entropy(H, W, y, reduction="none").sum(), A.linear_distillation(H, W, *lists)]
    assert len(A._eager_nodes) == before + 3
    losses[1].backward()
    assert len(A._eager_nodes) == before + 3                      # its accumulators live as long as the graph's nodes do
    losses.clear()
    with torch.no_grad():
        A.linear_cross_entropy(H, W, y), A.linear_distillation(H, W, *lists)
    A.linear_cross_entropy(H.detach(), W.detach(), y)
    assert len(A._eager_nodes) == before
    capturing[0] = True
    loss = A.linear_cross_entropy(H, W, y)
    assert loss.requires_grad and len(A._eager_nodes) == before


@pytest.mark.parametrize("front", ["cross_entropy", "distillation"])
def test_compiled_callers_end_silently(capturing, monkeypatch, front):
    """Whatever the tracer makes of a call's objects, none of them fails where it is dropped."""
    H, W, y, lists = case()
    call = (lambda h, w: A.linear_cross_entropy(h, w, y)) if front == "cross_entropy" else (lambda h, w: A.linear_distillation(h, w, *lists))
    seen = []
    monkeypatch.setattr(sys, "unraisablehook", lambda u: seen.append(u.exc_value))
    loss = torch.compile(call, backend="eager")(H, W)
    loss.backward()
    assert H.grad is not None and W.grad is not None
    del loss
    torch._dynamo.reset()
    gc.collect()
    assert not seen


def test_a_loss_costs_little_to_remember(capturing, monkeypatch):
    """In calls, of Python and of C functions, that an eager loss makes from its forward to its end: the function itself, the capture's query,
    a weak reference, its way into the set and out of it.  (A call without gradients makes some forty.)"""
    H, W, y, _ = case()

    def calls():
        count = [0]

        def seen(frame, event, arg):
            count[0] += event in ("call", "c_call")
        A.linear_cross_entropy(H, W, y)
        gc.disable()
        sys.setprofile(seen)
        A.linear_cross_entropy(H, W, y)
        sys.setprofile(None)
        gc.enable()
        return count[0]

    here = calls()
    monkeypatch.setattr(A, "_remember", lambda *args: None)
    without = calls()
    print(here, without)
    assert here - without <= 5


def test_accumulators_behind_the_states(capturing):
    """In a model the leaves are the parameters that the states were computed from."""
    H, W, y, _ = case()
    P, x = torch.randn(8, 8, requires_grad=True), torch.randn(4, 8)
    loss = A.linear_cross_entropy(torch.tanh(x @ P), W, y)
    node = [r() for r in A._eager_nodes if r() is loss.grad_fn]
    at = [torch.autograd.graph.get_gradient_edge(t).node for t in (P, W)]
    assert len(node) == 1 and A._accumulators(node) == set(at)
    other = torch.relu(x @ P)
    assert A._accumulators([torch.autograd.graph.get_gradient_edge(other).node]) == {at[0]}
    assert A._accumulators([torch.autograd.graph.get_gradient_edge(H).node]).isdisjoint(at)


@pytest.mark.parametrize("reduction", ["mean", "none"])
@pytest.mark.parametrize("eager", ["cross_entropy", "distillation"])
def test_captured_cross_entropy_beside_a_living_eager_loss(capturing, reduction, eager):
    H, W, y, lists = case()
    x = torch.randn(8, 8, requires_grad=True)
    call = (lambda: A.linear_cross_entropy(H @ x, W, y)) if eager == "cross_entropy" else (lambda: A.linear_distillation(H @ x, W, *lists))
    living = 2 * call()
    capturing[0] = True
    for h, w in ((H, W), (H.detach(), W), (H, W.detach()), (torch.relu(torch.ones(4, 8) @ x), W.detach())):
        loss = A.linear_cross_entropy(h, w, y, reduction=reduction).sum()          # the forward alone is none of it
        with pytest.raises(RuntimeError, match="alive"):
            loss.backward()
    A.linear_cross_entropy(torch.randn(4, 8, requires_grad=True), W.detach(), y, reduction=reduction).sum().backward()
    del living, loss
    A.linear_cross_entropy(H, W, y, reduction=reduction).sum().backward()
    assert H.grad is not None and W.grad is not None


def test_captures_beside_losses_of_a_side_stream(capturing, monkeypatch):
    """A stream that a capture can take in: the usual warm-up on one, whose last loss may still be alive."""
    H, W, y, _ = case()
    monkeypatch.setattr(A, "_stream", lambda device: 4096)
    living = A.linear_cross_entropy(H, W, y)
    living.backward()
    capturing[0] = True
    A.linear_cross_entropy(H, W, y).backward()
    assert living.requires_grad


@pytest.mark.parametrize("lead", [(4,), (2, 2)])
@pytest.mark.parametrize("strided", [False, True])
def test_distillation_is_differentiated_once(capturing, monkeypatch, lead, strided):
    """The library's gradients have no graph of their own: a penalty on what follows from them raises where it would lose the loss's part,
    however it is differentiated."""
    _, W, _, lists = case()
    lists = tuple(t.reshape(*lead, 2) for t in lists)
    W.requires_grad_(False)
    monkeypatch.setattr(A, "_launch", lambda call, device, *args: [t.fill_(1) for t in args if torch.is_tensor(t) and t.shape == W.shape])
    P, x = torch.randn(8, 8, requires_grad=True), torch.randn(*lead, 8)

    def states():
        h = torch.tanh(x @ P)
        return torch.stack([h, h], -1)[..., 0] if strided else h

    for take in (lambda g: torch.autograd.grad((g * g).sum(), P), lambda g: (g * g).sum().backward()):
        loss = A.linear_distillation(states(), W, *lists)
        g, = torch.autograd.grad(loss, P, create_graph=True)
        assert g.requires_grad
        with pytest.raises(RuntimeError, match="cannot be differentiated"):
            take(g)
    A.linear_distillation(states(), W, *lists).backward()
    assert P.grad is not None and not P.grad.requires_grad
