"""GPU: which captures the front end refuses.  (The checks alone: nothing is captured here.)"""
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
