"""GPU: which captures the front end refuses (the checks alone, nothing is captured there), and that others go through."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2511_17599_amd.torch_api import linear_cross_entropy, linear_distillation     # noqa: E402


def case():
    x, P, W = torch.randn(8, 16, device="cuda"), *(torch.randn(n, 16, device="cuda", requires_grad=True) for n in (16, 30))
    lists = torch.zeros(8, 2, dtype=torch.int64, device="cuda"), torch.zeros(8, 2, device="cuda")
    return x, P, W, lists, torch.zeros(8, dtype=torch.int64, device="cuda")


@pytest.mark.parametrize("eager", ["distillation", "cross_entropy"])
def test_distillation_beside_a_living_loss_of_the_same_parameters(monkeypatch, eager):
    x, P, W, lists, y = case()
    H = torch.tanh(x @ P)
    loss = linear_distillation(H, W.detach(), *lists) if eager == "distillation" else linear_cross_entropy(H, W.detach(), y)
    del H
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
    with pytest.raises(RuntimeError, match="alive"):
        linear_distillation(torch.relu(x @ P), W, *lists)
    linear_distillation(x, W, *lists)                              # (no leaf in common)
    with torch.no_grad():
        linear_distillation(x @ P, W, *lists)
    del loss
    linear_distillation(torch.relu(x @ P), W, *lists).backward()
    assert P.grad is not None and W.grad is not None


@pytest.mark.parametrize("reduction", ["mean", "none"])
@pytest.mark.parametrize("eager", ["distillation", "cross_entropy"])
def test_cross_entropy_beside_a_living_loss_of_the_same_parameters(monkeypatch, eager, reduction):
    x, P, W, lists, y = case()
    H = torch.tanh(x @ P)
    loss = linear_distillation(H, W, *lists) if eager == "distillation" else linear_cross_entropy(H, W, y, reduction=reduction)
    del H
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
    again = linear_cross_entropy(x @ P, W, y, reduction=reduction).sum()
    with pytest.raises(RuntimeError, match="alive"):
        again.backward()
    del loss, again
    linear_cross_entropy(x @ P, W, y, reduction=reduction).sum().backward()
    assert P.grad is not None and W.grad is not None


@pytest.mark.parametrize("reduction", ["mean", "none"])
def test_a_captured_cross_entropy_step(reduction):
    _, P, W, _, y = case()
    up = None if reduction == "mean" else torch.linspace(0.5, 1, 8, device="cuda")
    H = torch.randn(8, 16, device="cuda", requires_grad=True)

    def step():
        loss = linear_cross_entropy(H, W, y, reduction=reduction)
        return (loss.detach(), *torch.autograd.grad(loss, (H, W), up))

    want = [t.clone() for t in step()]                             # (no eager graph lives behind it)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = step()
    for rep in range(3):
        for t in got:
            t.fill_(7)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), rep
