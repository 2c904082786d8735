"""The autograd front end around the library's calls, on CPU tensors with the calls themselves left out: what it remembers of living losses,
and what that costs."""
import gc
import sys
import time

import pytest
import torch

from paper_2511_17599_amd import binding as B
from paper_2511_17599_amd import torch_api as A


@pytest.fixture
def capturing(monkeypatch):
    """The front end on CPU tensors; the returned list says whether a capture is to be seen."""
    state = [False]
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: state[0])
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
    """Forward calls with and without it in turn; 3 us are several times what it takes here."""
    H, W, y, _ = case()
    kept = A._remember

    def best(n=300):
        t = time.perf_counter()
        for _ in range(n):
            A.linear_cross_entropy(H, W, y)
        return (time.perf_counter() - t) / n

    best()
    times = {False: [], True: []}
    for rep in range(30):
        for left_out in (False, True):
            monkeypatch.setattr(A, "_remember", (lambda ctx: None) if left_out else kept)
            times[left_out].append(best())
    cost = min(times[False]) - min(times[True])
    print(f"{cost * 1e6:.2f} us of {min(times[False]) * 1e6:.1f}")
    assert cost < 3e-6


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
