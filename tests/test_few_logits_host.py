"""Host-only: what the calls on a few logits per row refuse, before any device is touched, and what their workspaces hold."""
import pytest
import torch

from paper_2511_17599_amd import binding as B
from paper_2511_17599_amd import torch_api as A

P = 4096            # a fake, aligned, never dereferenced device address
BF16, F32 = B.FLCE_DTYPE_BF16, B.FLCE_DTYPE_F32
ARG, SHAPE, WS = B.FLCE_ERR_BAD_ARG, B.FLCE_ERR_BAD_SHAPE, B.FLCE_ERR_WORKSPACE


def topk(H=P, W=P, N=8, d=64, V=512, K=4, dt=F32, z=P, ids=P, lse=P, ws=P, nb=1 << 40):
    return B.flce_topk(H, W, N, d, V, K, dt, z, ids, lse, ws, nb)


@pytest.mark.parametrize("kw,want", [
    (dict(H=None), ARG), (dict(W=None), ARG), (dict(z=None), ARG), (dict(ids=None), ARG), (dict(lse=None), ARG), (dict(dt=2), ARG),
    (dict(H=P + 8), ARG), (dict(W=P + 4), ARG), (dict(N=0), SHAPE), (dict(N=-3), SHAPE), (dict(d=60), SHAPE), (dict(d=0), SHAPE),
    (dict(V=0), SHAPE), (dict(K=0), SHAPE), (dict(K=257), SHAPE), (dict(K=5, V=4), SHAPE), (dict(V=(1 << 22) + 1), SHAPE),
    (dict(ws=None), WS), (dict(ws=P + 16), WS), (dict(nb=16), WS), (dict(N=1 << 40), SHAPE)])
def test_topk_refuses(kw, want):
    assert topk(**kw) == want


def test_topk_workspace():
    need = B.flce_topk_workspace_bytes(8, 64, 512, 4, F32)
    assert need > 0 and topk(nb=need - 1) == WS
    for bad in ((0, 64, 512, 4), (8, 63, 512, 4), (8, 64, 512, 0), (8, 64, 512, 513), (8, 64, 3, 4)):
        assert B.flce_topk_workspace_bytes(*bad, BF16) == 0
    assert B.flce_topk_workspace_bytes(8, 64, 512, 4, 5) == 0
    # a few rows: their logits; more: whole tiles of 256 rows, a chunk of them however many
    assert B.flce_topk_workspace_bytes(32, 4096, 128256, 64, BF16) < 32 * 128256 * 4 * 1.1
    assert B.flce_topk_workspace_bytes(64, 4096, 128256, 64, BF16) < 256 * 128256 * 4 * 1.1
    for N in (8192, 131072):
        assert B.flce_topk_workspace_bytes(N, 4096, 128256, 64, BF16) < (1 << 30) * 1.05 + N * 4096 * 2 * 1.01 + (1 << 20)


def fwd(H=P, W=P, ids=P, t=P, N=8, d=64, V=512, K=4, T=1.0, red=0, dt=F32, loss=P, rows=None, lse=P, saved=P, ws=P, nb=1 << 40):
    return B.flce_distill_forward(H, W, ids, t, N, d, V, K, T, red, dt, loss, rows, lse, saved, ws, nb)


def bwd(H=P, W=P, ids=P, lse=P, saved=P, N=8, d=64, V=512, K=4, T=1.0, red=0, dt=F32, g=P, gr=None, dH=P, dW=P, ws=P, nb=1 << 40):
    return B.flce_distill_backward(H, W, ids, lse, saved, N, d, V, K, T, red, dt, g, gr, dH, dW, ws, nb)


COMMON = [(dict(H=None), ARG), (dict(W=None), ARG), (dict(ids=None), ARG), (dict(lse=None), ARG), (dict(saved=None), ARG), (dict(saved=P + 8), ARG),
          (dict(red=2), ARG), (dict(dt=-1), ARG), (dict(H=P + 8), ARG), (dict(T=0.0), ARG), (dict(T=-1.0), ARG),
          (dict(T=float("nan")), ARG), (dict(T=float("inf")), ARG), (dict(T=1e-40), ARG), (dict(T=1e30), ARG), (dict(K=0), SHAPE),
          (dict(K=257), SHAPE), (dict(N=0), SHAPE), (dict(d=4), SHAPE), (dict(V=-1), SHAPE), (dict(ws=None), WS), (dict(ws=P + 128), WS),
          (dict(nb=300), WS)]


@pytest.mark.parametrize("kw,want", COMMON + [(dict(loss=None), ARG), (dict(t=None), ARG)])
def test_distill_forward_refuses(kw, want):
    assert fwd(**kw) == want


@pytest.mark.parametrize("kw,want", COMMON + [(dict(g=None), ARG), (dict(gr=P), ARG), (dict(dH=None), ARG), (dict(dW=None), ARG),
                                              (dict(dW=P + 4), ARG)])
def test_distill_backward_refuses(kw, want):
    assert bwd(**kw) == want


def test_distill_workspaces():
    for back, call in ((0, fwd), (1, bwd)):
        need = B.flce_distill_workspace_bytes(8, 64, 512, 4, F32, back)
        assert need > 0 and call(nb=need - 1) == WS
        for bad in ((0, 64, 512, 4), (8, 63, 512, 4), (8, 64, 0, 4), (8, 64, 512, 257)):
            assert B.flce_distill_workspace_bytes(*bad, BF16, back) == 0
    # the copy of H, the lists, a few words per row
    N, d, V, K = 131072, 4096, 128256, 32
    assert B.flce_distill_workspace_bytes(N, d, V, K, BF16, 0) < N * d * 2 * 1.01 + N * K * 4 + (64 << 20)
    assert B.flce_distill_workspace_bytes(N, d, V, K, BF16, 1) == B.flce_workspace_bytes(N, d, V, BF16, 1)
    assert 8 * N * (K + 1) <= B.flce_distill_saved_bytes(N, K) < 8 * N * (K + 1) + 256
    assert B.flce_distill_saved_bytes(0, 4) == B.flce_distill_saved_bytes(4, 0) == B.flce_distill_saved_bytes(4, 257) == 0


def step(H=P, W=P, s=P, f=None, batch=2, beams=4, d=64, V=512, n_out=4, dt=F32, so=1 << 20, to=P, po=P, fo=1 << 21, ws=P, nb=1 << 40):
    return B.flce_beam_step(H, W, s, f, batch, beams, d, V, n_out, 2, 0, dt, so, to, po, fo, ws, nb)


@pytest.mark.parametrize("kw,want", [
    (dict(H=None), ARG), (dict(W=None), ARG), (dict(s=None), ARG), (dict(so=None), ARG), (dict(to=None), ARG), (dict(po=None), ARG),
    (dict(fo=None), ARG), (dict(dt=9), ARG), (dict(H=P + 2), ARG), (dict(so=P), ARG), (dict(s=P, so=P + 4), ARG), (dict(f=1 << 21), ARG),
    (dict(batch=0), SHAPE), (dict(beams=0), SHAPE), (dict(beams=65), SHAPE), (dict(n_out=0), SHAPE), (dict(n_out=65), SHAPE),
    (dict(d=12), SHAPE), (dict(V=0), SHAPE), (dict(batch=1 << 40), SHAPE), (dict(ws=None), WS), (dict(nb=100), WS)])
def test_beam_step_refuses(kw, want):
    assert step(**kw) == want


def test_beam_workspace():
    need = B.flce_beam_workspace_bytes(2, 4, 64, 512, 4, F32)
    assert need > B.flce_topk_workspace_bytes(8, 64, 512, 4, F32) and step(nb=need - 1) == WS
    assert B.flce_beam_workspace_bytes(2, 4, 64, 3, 8, F32) > 0            # fewer tokens than results: all of them are candidates
    assert B.flce_beam_workspace_bytes(2, 65, 64, 512, 4, F32) == 0


def reorder(src=P, dst=1 << 30, par=P, outer=2, batch=3, bi=4, bo=4, row=64, sr=64, so=768, dr=64, do=768):
    return B.flce_beam_reorder(src, dst, par, outer, batch, bi, bo, row, sr, so, dr, do)


@pytest.mark.parametrize("kw,want", [
    (dict(src=None), ARG), (dict(dst=None), ARG), (dict(par=None), ARG), (dict(outer=0), SHAPE), (dict(batch=0), SHAPE),
    (dict(bi=0), SHAPE), (dict(bo=0), SHAPE), (dict(bi=65), SHAPE), (dict(bo=65), SHAPE), (dict(row=0), SHAPE), (dict(row=65), SHAPE),
    (dict(sr=63), SHAPE), (dict(dr=-64), SHAPE), (dict(so=767), SHAPE), (dict(do=0), SHAPE), (dict(sr=1 << 60), SHAPE),
    (dict(dst=P + 64), ARG), (dict(dst=P + 1535), ARG), (dict(dst=P, sr=128, so=1536), ARG), (dict(dst=P, bo=2, dr=64, do=384), ARG),
    (dict(dst=P, bi=17, bo=17, so=17 * 192, do=17 * 192), SHAPE)])
def test_reorder_refuses(kw, want):
    assert reorder(**kw) == want


def test_front_end_refuses():
    H, W = torch.zeros(4, 3, 16), torch.zeros(50, 16)
    with pytest.raises(ValueError):
        A.linear_topk(H, W, 4)                                             # not on a GPU
    with pytest.raises(TypeError):
        A.linear_topk(H.double(), W.double(), 4)
    with pytest.raises(TypeError):
        A.linear_topk(H, W.bfloat16(), 4)
    ids, t = torch.zeros(4, 3, 5, dtype=torch.int64), torch.zeros(4, 3, 5)
    with pytest.raises(ValueError):
        A.linear_distillation(H, W, ids, t, reduction="max")
    with pytest.raises(TypeError):
        A.linear_distillation(H, W, t, t)
    with pytest.raises(TypeError):
        A.linear_distillation(H, W, ids, ids)
    with pytest.raises(ValueError):
        A.linear_distillation(H, W, ids[:, :2], t[:, :2])
    with pytest.raises(ValueError):
        A.linear_distillation(H, W, ids, t[..., :4])
    with pytest.raises(ValueError):
        A.beam_step(H[0], W, torch.zeros(4, 3))
    with pytest.raises(ValueError):
        A.beam_step(H, W, torch.zeros(4, 2))
    with pytest.raises(ValueError):
        A.beam_step(H, W, torch.zeros(4, 3), finished=torch.zeros(4, 2, dtype=torch.bool))
    with pytest.raises(ValueError):
        A.reorder_states(torch.zeros(4, 3, dtype=torch.int64), torch.zeros(1, 4, 3, 8))
