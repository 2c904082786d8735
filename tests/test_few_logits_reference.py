"""The plain forms that the GPU tests compare with, held to closed forms, to torch in 64 bits and to differences (CPU)."""
import numpy as np
import pytest
import torch

import few_logits as F


def case(seed, N=7, d=8, V=23, K=5):
    rng = np.random.default_rng(seed)
    H, W = rng.standard_normal((N, d)), rng.standard_normal((V, d))
    ids = np.stack([rng.permutation(V)[:K] for _ in range(N)])
    return H, W, ids, 3 * rng.standard_normal((N, K))


def test_topk_orders_ties_and_nan():
    z = np.array([[1.0, 3.0, 3.0, -0.0, 0.0, np.nan, -np.inf, np.inf]])
    v, ids, lse = F.topk(z, 8)
    assert ids.tolist() == [[5, 7, 1, 2, 0, 3, 4, 6]]
    z = np.random.default_rng(1).standard_normal((5, 40))
    v, ids, lse = F.topk(z, 7)
    t = torch.topk(torch.from_numpy(z), 7)
    assert np.array_equal(v, t.values.numpy()) and np.array_equal(ids, t.indices.numpy())
    assert np.allclose(lse, torch.logsumexp(torch.from_numpy(z), 1).numpy(), rtol=1e-14)
    assert F.logsumexp(np.full((1, 3), -np.inf))[0] == -np.inf and F.logsumexp(np.array([[np.inf, 0.0]]))[0] == np.inf


@pytest.mark.parametrize("T", [1.0, 2.5])
def test_distillation_is_torch_kl(T):
    H, W, ids, t = case(2)
    r = F.distill(H, W, ids, t, T, np.ones(7))
    Ht, Wt = (torch.from_numpy(x).requires_grad_() for x in (H, W))
    logq = torch.log_softmax(Ht @ Wt.t() / T, 1).gather(1, torch.from_numpy(ids))
    p = torch.softmax(torch.from_numpy(t) / T, 1)
    rows = T * T * torch.nn.functional.kl_div(logq, p, reduction="none").sum(1)
    assert np.allclose(r["rows"], rows.detach().numpy(), rtol=1e-12)
    rows.sum().backward()
    assert np.allclose(r["dH"], Ht.grad.numpy(), atol=1e-13) and np.allclose(r["dW"], Wt.grad.numpy(), atol=1e-13)


def test_distillation_gradient_by_differences():
    H, W, ids, t = case(3)
    ids[2, 1:] = -1
    ids[4] = -1
    ids[5, 3] = ids[5, 0]                      # the same id twice
    t[6, 2] = -np.inf
    gamma = np.linspace(0.5, 2.0, 7)
    r = F.distill(H, W, ids, t, 1.7, gamma)
    assert not r["counts"][4] and r["rows"][4] == 0 and not r["dH"][4].any()
    f = lambda: (F.distill(H, W, ids, t, 1.7, gamma)["rows"] * gamma).sum()
    for A, g in ((H, r["dH"]), (W, r["dW"])):
        for at in ((0, 1), (2, 3), (5, 7), (6, 0)):
            keep, e = A[at], 1e-5
            A[at] = keep + e
            up = f()
            A[at] = keep - e
            down = f()
            A[at] = keep
            assert abs((up - down) / (2 * e) - g[at]) < 1e-8


def test_distillation_of_a_teacher_that_is_the_student_is_zero():
    H, W, _, _ = case(4)
    z = H @ W.T
    r = F.distill(H, W, np.tile(np.arange(23), (7, 1)), z, 2.0, np.ones(7))
    assert np.abs(r["rows"]).max() < 1e-13 and np.abs(r["dH"]).max() < 1e-13


def test_beam_is_a_search_over_all_continuations():
    rng = np.random.default_rng(5)
    H, W = rng.standard_normal((2, 3, 8)), rng.standard_normal((11, 8))
    s = rng.standard_normal((2, 3))
    got = F.beam(H, W, s, None, 5, -1, 0)
    total = torch.log_softmax(torch.from_numpy(H @ W.T), -1) + torch.from_numpy(s)[..., None]
    want = torch.topk(total.flatten(1), 5)
    assert np.allclose(got[0], want.values.numpy()) and np.array_equal(got[2] * 11 + got[1], want.indices.numpy())
    done = np.array([[True, True, True], [False, True, False]])
    got = F.beam(H, W, s, done, 5, 4, 9)
    assert np.array_equal(got[0][0, :3], -np.sort(-s[0])) and (got[1][0] == 9).all() and (got[0][0, 3:] == -np.inf).all()
