"""GPU: distillation from a teacher's largest logits, loss and gradients, against the definition in 64 bits."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import few_logits as F                                    # noqa: E402
from conftest import set_plan, tile_edges                 # noqa: E402
from paper_2511_17599_amd import binding as B             # noqa: E402
from paper_2511_17599_amd.torch_api import linear_cross_entropy, linear_distillation, linear_topk   # noqa: E402

CODE = {"bf16": B.FLCE_DTYPE_BF16, "f32": B.FLCE_DTYPE_F32}


def operands(rng, N, d, V, dtype):
    """numpy values that dtype holds."""
    def stored(x):
        return F.f64(torch.from_numpy(x).to(F.DT[dtype]))
    return stored(rng.standard_normal((N, d))), stored(0.08 * rng.standard_normal((V, d)))


def lists(rng, N, V, K, kind="full"):
    ids = np.stack([rng.permutation(V)[:K] for _ in range(N)]) if V >= K else rng.integers(0, V, (N, K))
    t = np.float32(6 - 2 * np.log1p(np.arange(K)) + rng.standard_normal((N, K)))
    if kind != "full":
        ids = np.where(np.arange(K) < rng.integers(1, K + 1, (N, 1)), ids, -1)
        ids[rng.permutation(N)[:max(1, N // 6)]] = -1     # rows without an entry
        t[ids < 0] = np.nan                               # what is absent is not looked at
    if kind == "wild":
        ids[N // 2] = rng.permutation(np.where(np.arange(K) % 2 == 0, ids[N // 2].max(), ids[N // 2]))
        t[N // 2] = 1.0
        ids[N // 3] = rng.integers(0, V, K)
        t[N // 3] = -np.inf                               # entries, but no share
        ids[N // 4], t[N // 4] = rng.integers(0, V, K), 0.0
        t[N // 4, ::2] = -np.inf
        t[N // 4, 1:2] = np.finfo(np.float32).min         # the lowest value is a logit like another
        ids[1], t[1] = rng.integers(0, V, K), np.finfo(np.float32).min
    return ids, t


def call(H, W, ids, t, T, reduction="mean", grad=1.0, grad_rows=None, stream=None):
    """Forward and backward on poisoned workspaces; loss, losses per row, lse, dH, dW, number of rows that count, status."""
    (N, d), V, K = H.shape, W.shape[0], ids.shape[1]
    dt = CODE["bf16" if H.dtype is torch.bfloat16 else "f32"]
    red = {"mean": B.FLCE_REDUCE_MEAN, "sum": B.FLCE_REDUCE_SUM}[reduction]
    f = lambda *s: torch.full(s, 7.0, device="cuda")
    loss, rows, lse = f(1), f(N + 16), f(N + 16)
    nf, nb = (B.flce_distill_workspace_bytes(N, d, V, K, dt, b) for b in (0, 1))
    ns = B.flce_distill_saved_bytes(N, K)
    wf, wb, saved = (torch.full((n + 64,), 0xFF, dtype=torch.uint8, device="cuda") for n in (nf, nb, ns))
    dH, dW = torch.full((N * d + 64,), 7.0, dtype=H.dtype, device="cuda"), torch.full((V * d + 64,), 7.0, dtype=H.dtype, device="cuda")
    assert B.flce_distill_forward(H, W, ids, t, N, d, V, K, T, red, dt, loss, rows, lse, saved, wf, nf, stream) == B.FLCE_OK
    status = B.flce_last_device_status(wf, stream)
    up = None if grad_rows is not None else torch.full((1,), grad, device="cuda")
    torch.cuda.synchronize()
    kept = saved.clone()
    assert B.flce_distill_backward(H, W, ids, lse, saved, N, d, V, K, T, red, dt, up, grad_rows, dH, dW, wb, nb, stream) == B.FLCE_OK
    assert B.flce_last_device_status(wb, stream) == status
    torch.cuda.synchronize()
    for x in (rows[N:], lse[N:], dH[N * d:], dW[V * d:]):
        assert (x == 7).all()
    assert (wf[nf:] == 0xFF).all() and (wb[nb:] == 0xFF).all() and (saved[ns:] == 0xFF).all() and torch.equal(saved, kept)
    pairs = saved[ns - 8 * N * K:ns].view(torch.float32).reshape(N, K, 2)     # (share, logit) of each entry
    return dict(loss=loss, rows=rows[:N], lse=lse[:N], zt=pairs[..., 1], share=pairs[..., 0], dH=dH[:N * d].reshape(N, d),
                dW=dW[:V * d].reshape(V, d), status=status)


def check(rng, N, d, V, K, dtype, T, reduction="mean", kind="full", per_row=False):
    print(f"[case] distill {dtype} N={N} d={d} V={V} K={K} T={T} {reduction} {kind} per_row={per_row}", flush=True)
    H, W = operands(rng, N, d, V, dtype)
    ids, t = lists(rng, N, V, K, kind)
    counts = F.shares(ids, t, T, V)[2]
    wr = rng.uniform(-1, 2, N).astype(np.float32)
    gamma = wr.astype(np.float64) if per_row else np.full(N, 1.25 / max(1, counts.sum()) if reduction == "mean" else 1.25)
    r = F.distill(H, W, ids, t.astype(np.float64), T, gamma)
    got = call(F.on_gpu(H, dtype), F.on_gpu(W, dtype), torch.from_numpy(ids).cuda(), torch.from_numpy(t).cuda(), T, reduction, 1.25,
               torch.from_numpy(wr).cuda() if per_row else None)
    dz = F.logit_bound(H, W)
    assert (np.abs(F.f64(got["lse"]) - r["lse"]) <= dz.max(1) / T + F.lse_bound(r["lse"], V)).all()
    assert (np.abs(F.f64(got["zt"]) - r["zt"]) <= dz.max()).all()
    bound = F.loss_bound(r, H, W, T)
    assert (np.abs(F.f64(got["rows"]) - r["rows"]) <= bound).all()
    n = r["counts"].sum()
    total, tb = r["rows"].sum(), bound.sum() + (N + 10) * F.U32 * np.abs(r["rows"]).sum()
    scale = 1 / max(1, n) if reduction == "mean" else 1.0
    assert abs(got["loss"].item() - total * scale) <= tb * scale
    assert got["status"] == (B.FLCE_ERR_TARGET_RANGE if r["bad"].any() else B.FLCE_OK, n)
    bH, bW = F.grad_bounds(r, H, W, T, dtype, per_row)
    for k, b in (("dH", bH), ("dW", bW)):
        x = F.f64(got[k])
        assert (np.abs(x - r[k]) <= b).all(), (k, np.max(np.abs(x - r[k]) / b))
        norm = np.linalg.norm(r[k])
        if norm > 0:
            err = np.linalg.norm(x - r[k]) / norm
            print(f"       {k} {err:.2e} of its norm", flush=True)
            # two roundings to the type, each at most u, where the terms of a sum do not cancel
            assert err <= (2 * F.U["bf16"] if dtype == "bf16" else 2e-5)
    assert not got["dH"][torch.from_numpy(~r["counts"]).cuda()].any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,d,V,K,T,reduction,kind,per_row", [
    (1, 8, 2, 1, 1.0, "mean", "full", False), (1, 64, 300, 256, 2.0, "sum", "full", False), (5, 40, 17, 16, 1.0, "mean", "full", True),
    (64, 32, 1000, 7, 0.5, "mean", "ragged", False), (130, 104, 3001, 33, 3.0, "sum", "wild", False),
    (300, 200, 2000, 64, 1.0, "mean", "wild", True), (257, 264, 5003, 20, 2.0, "mean", "ragged", True),
    (600, 128, 4099, 100, 1.0, "mean", "wild", False), (40, 72, 9000, 256, 4.0, "mean", "ragged", False),
    (1100, 72, 700, 3, 1.0, "sum", "ragged", True)])
def test_sizes(dtype, N, d, V, K, T, reduction, kind, per_row):
    check(np.random.default_rng(N + V), N, d, V, K, dtype, T, reduction, kind, per_row)


@pytest.mark.parametrize("knobs", [dict(FLCE_GENERIC=1), dict(FLCE_TILE=128), dict(FLCE_TILE=256), dict(FLCE_VC_TILES=3, FLCE_NC_TILES=1),
                                   dict(FLCE_TILE=128, FLCE_VC_TILES=2, FLCE_NC_TILES=2), dict(FLCE_GENERIC=1, FLCE_VC_TILES=3, FLCE_NC_TILES=1)])
@pytest.mark.parametrize("d,per_row", [(96, False), (104, True)])
def test_every_loop_and_chunks(monkeypatch, knobs, d, per_row):
    set_plan(monkeypatch, **knobs)
    check(np.random.default_rng(7), 700, d, 3333, 40, "bf16", 1.5, "mean", "wild", per_row)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [0.05, 40.0])
def test_far_temperatures(dtype, T):
    check(np.random.default_rng(13), 210, 72, 1500, 30, dtype, T, "mean", "wild", False)


@pytest.mark.parametrize("edges,N,d,V", [((64, 64), 300, 96, 3000), ((128, 128), 1300, 96, 4100)])
def test_f32_edges_in_chunks(monkeypatch, edges, N, d, V):
    set_plan(monkeypatch, FLCE_VC_TILES=5, FLCE_NC_TILES=2)
    assert tile_edges(N, d, V, "f32") == edges
    check(np.random.default_rng(8), N, d, V, 25, "f32", 2.0, "mean", "wild", True)


def test_all_entries_in_one_tile():
    """Lists that crowd a few positions: thousands of entries of one tile, 64 and 65 of one block among them."""
    rng = np.random.default_rng(12)
    N, d, V, K = 300, 64, 2000, 200
    H, W = operands(rng, N, d, V, "bf16")
    ids = np.tile(700 + np.arange(K), (N, 1))
    ids[:8] = 700 + np.arange(K)[::-1]
    t = rng.standard_normal((N, K)).astype(np.float32)
    r = F.distill(H, W, ids, t.astype(np.float64), 1.0, np.ones(N))
    got = call(F.on_gpu(H, "bf16"), F.on_gpu(W, "bf16"), torch.from_numpy(ids).cuda(), torch.from_numpy(t).cuda(), 1.0, "sum")
    assert (np.abs(F.f64(got["zt"]) - r["zt"]) <= F.logit_bound(H, W).max()).all()
    assert (np.abs(F.f64(got["rows"]) - r["rows"]) <= F.loss_bound(r, H, W, 1.0)).all()
    bH, bW = F.grad_bounds(r, H, W, 1.0, "bf16", False)
    assert (np.abs(F.f64(got["dH"]) - r["dH"]) <= bH).all() and (np.abs(F.f64(got["dW"]) - r["dW"]) <= bW).all()


def test_more_tiles_than_buckets():
    """A vocabulary of more tiles than the sort of the lists takes at a time (64-row tiles: 8192 x 64)."""
    N, d, V, K = 20, 8, 540_000, 50
    assert tile_edges(N, d, V, "f32")[0] in (64, 128)
    rng = np.random.default_rng(13)
    for dtype in ("f32", "bf16"):
        H, W = operands(rng, N, d, V, dtype)
        ids, t = lists(rng, N, V, K)
        ids[:, 0], ids[:, 1], ids[:, 2] = V - 1, 0, 8192 * 64
        got = call(F.on_gpu(H, dtype), F.on_gpu(W, dtype), torch.from_numpy(ids).cuda(), torch.from_numpy(t).cuda(), 1.0, "sum")
        z = np.einsum("nd,nkd->nk", H, W[ids])
        assert (np.abs(F.f64(got["zt"]) - z) <= 4 * (d + 2) * F.U32 * np.einsum("nd,nkd->nk", np.abs(H), np.abs(W[ids]))).all()


def test_ids_beyond_the_vocabulary():
    rng = np.random.default_rng(14)
    N, d, V, K = 90, 64, 500, 6
    H, W = operands(rng, N, d, V, "f32")
    ids, t = lists(rng, N, V, K)
    ids[3, 2], ids[50, 5], ids[60, 0] = V, 1 << 40, (1 << 32) + 5
    r = F.distill(H, W, np.where(ids >= V, V, ids), t.astype(np.float64), 1.0, np.ones(N))
    got = call(F.on_gpu(H, "f32"), F.on_gpu(W, "f32"), torch.from_numpy(ids).cuda(), torch.from_numpy(t).cuda(), 1.0, "sum")
    assert got["status"] == (B.FLCE_ERR_TARGET_RANGE, N - 3)
    assert (np.abs(F.f64(got["rows"]) - r["rows"]) <= F.loss_bound(r, H, W, 1.0)).all() and got["rows"][3] == 0
    assert not got["dH"][[3, 50, 60]].any()
    assert (np.abs(F.f64(got["dW"]) - r["dW"]) <= F.grad_bounds(r, H, W, 1.0, "f32", False)[1]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_no_row_counts(dtype):
    rng = np.random.default_rng(15)
    H, W = operands(rng, 70, 64, 300, dtype)
    ids = torch.full((70, 4), -1, dtype=torch.int64, device="cuda")
    got = call(F.on_gpu(H, dtype), F.on_gpu(W, dtype), ids, torch.zeros(70, 4, device="cuda"), 1.0)
    assert got["loss"].item() == 0 and not got["rows"].any() and not got["dH"].any() and not got["dW"].any()
    assert not got["zt"].any() and (got["share"] == -1).all()
    assert got["status"] == (B.FLCE_OK, 0)


def test_one_entry_is_cross_entropy():
    """A list of one id is a target: losses agree to the bounds of both, gradients too (bf16: bit for bit, one G)."""
    rng = np.random.default_rng(16)
    for dtype, N, d, V in (("bf16", 600, 128, 3000), ("f32", 200, 64, 1000)):
        H, W = operands(rng, N, d, V, dtype)
        y = torch.from_numpy(rng.integers(0, V, N)).cuda()
        a, b = ((F.on_gpu(H, dtype).requires_grad_(), F.on_gpu(W, dtype).requires_grad_()) for _ in range(2))
        ce = linear_cross_entropy(*a, y, reduction="none")
        kd = linear_distillation(*b, y[:, None], torch.zeros(N, 1, device="cuda"), reduction="none")
        assert np.abs(F.f64(ce) - F.f64(kd)).max() <= 4 * F.lse_bound(np.abs(F.f64(ce)).max() + 20, V)
        w = torch.linspace(0.5, 1, N, device="cuda")
        g1, g2 = torch.autograd.grad(ce, a, w), torch.autograd.grad(kd, b, w)
        for x, z in zip(g1, g2):
            assert (x.float() - z.float()).norm() <= (2 * F.U["bf16"] if dtype == "bf16" else 2e-5) * x.float().norm()


@pytest.mark.parametrize("logit", [40.0, 165.0])
@pytest.mark.parametrize("dtype,N,d,V", [("f32", 250, 520, 4100), ("f32", 1300, 512, 4000), ("bf16", 268, 512, 1029), ("bf16", 2060, 1032, 20011)])
def test_confident_rows_of_a_confident_teacher(dtype, N, d, V, logit):
    """exp(z - lse) - 1 is zero but for the exponent's rounding where list and softmax hold the same logit (half a unit in the last place
    of the larger of z log2(e), lse log2(e))."""
    g = torch.Generator(device="cuda").manual_seed(60 + d)
    W = torch.randn(V, d, device="cuda", generator=g)
    y = torch.randint(0, V, (N,), device="cuda", generator=g)
    H = W[y] * (logit / (W[y] ** 2).sum(1, keepdim=True))
    H, W = H.to(F.DT[dtype]), W.to(F.DT[dtype])
    ids = torch.stack([y, (y + 1) % V], 1)
    t = torch.tensor([0.0, -float("inf")], device="cuda").expand(N, 2).contiguous()
    print(f"[case] confident distill {dtype} N={N} d={d} V={V} logit={logit}", flush=True)
    got = call(H, W, ids, t, 1.0, "sum")
    Wy = W[y].double()
    gy = (got["dH"].double() * Wy).sum(1) / (Wy ** 2).sum(1)
    bound = np.log(2) * 2.0 ** (np.floor(np.log2(1.02 * logit * np.log2(np.e))) - 24) + 3e-7
    assert gy.abs().max().item() <= 1.02 * bound


def test_nan_and_infinity_stay_in_their_rows():
    rng = np.random.default_rng(17)
    N, d, V, K = 100, 64, 400, 5
    H, W = operands(rng, N, d, V, "f32")
    ids, t = lists(rng, N, V, K)
    t[7, 1], t[8, 0] = np.nan, np.inf
    H[20, 3] = np.nan
    ids[30] = -1
    H[30] = np.inf                                        # a row that does not count
    Hg, Wg = F.on_gpu(H, "f32"), F.on_gpu(W, "f32")
    got = call(Hg, Wg, torch.from_numpy(ids).cuda(), torch.from_numpy(t).cuda(), 1.0, "sum")
    odd = np.isin(np.arange(N), (7, 8, 20))
    assert torch.isnan(got["rows"]).cpu().numpy().tolist() == odd.tolist() and got["rows"][30] == 0
    assert not got["dH"][30].any() and torch.isnan(got["dH"][7]).any() and torch.isnan(got["dH"][20]).all()
    keep = np.flatnonzero(~odd & (np.arange(N) != 30))
    r = F.distill(H[keep], W, ids[keep], t[keep].astype(np.float64), 1.0, np.ones(len(keep)))
    assert (np.abs(F.f64(got["rows"])[keep] - r["rows"]) <= F.loss_bound(r, H[keep], W, 1.0)).all()
    assert (np.abs(F.f64(got["dH"])[keep] - r["dH"]) <= F.grad_bounds(r, H[keep], W, 1.0, "f32", False)[0]).all()


def test_gradients_by_differences():
    """fp32, in the direction of random vectors: the loss of both sides in 64 bits would be the definition's; the kernels' own differences
    see what forward and backward disagree on.  Step 2^-6: truncation below 1e-4 of the derivative, rounding of two losses (1e-6) / 2^-5."""
    rng = np.random.default_rng(18)
    N, d, V, K, T = 64, 64, 500, 12, 2.0
    H, W = operands(rng, N, d, V, "f32")
    ids, t = lists(rng, N, V, K, "ragged")
    idg, tg = torch.from_numpy(ids).cuda(), torch.from_numpy(t).cuda()
    Hg, Wg = (F.on_gpu(x, "f32").requires_grad_() for x in (H, W))
    loss = linear_distillation(Hg, Wg, idg, tg, T, "mean")
    dH, dW = torch.autograd.grad(loss, (Hg, Wg))
    for X, dX, k in ((H, dH, 0), (W, dW, 1)):
        u = rng.standard_normal(X.shape)
        u *= (1.0 if k == 0 else 0.1)
        e = 2.0 ** -6
        ls = []
        for s in (e, -e):
            a = [H, W]
            a[k] = X + s * u
            ls.append(linear_distillation(F.on_gpu(a[0], "f32"), F.on_gpu(a[1], "f32"), idg, tg, T, "mean").item())
        want = (F.f64(dX) * u).sum()
        assert abs((ls[0] - ls[1]) / (2 * e) - want) <= 1e-3 * np.abs(F.f64(dX) * u).sum() + 1e-4


def test_front_end():
    rng = np.random.default_rng(19)
    N, d, V, K = 96, 64, 700, 9
    H, W = operands(rng, N, d, V, "bf16")
    ids, t = lists(rng, N, V, K, "ragged")
    idg, tg = torch.from_numpy(ids).cuda(), torch.from_numpy(t).cuda()
    want = call(F.on_gpu(H, "bf16"), F.on_gpu(W, "bf16"), idg, tg, 2.0, "mean", 1.0)
    for red in ("mean", "sum", "none"):
        Hg, Wg = F.on_gpu(H, "bf16").reshape(4, 24, d).requires_grad_(), F.on_gpu(W, "bf16").requires_grad_()
        loss = linear_distillation(Hg, Wg, idg.reshape(4, 24, K), tg.reshape(4, 24, K).double(), 2.0, red)
        n = want["status"][1]
        if red == "none":
            assert loss.shape == (4, 24) and torch.equal(loss.reshape(-1), want["rows"])
            loss = loss.sum() / n                         # (its gradient is an expanded scalar)
        elif red == "sum":
            loss = loss / n
        loss.backward()
        assert Hg.grad.shape == Hg.shape and Wg.grad.shape == Wg.shape
        err = (Hg.grad.reshape(N, d).float() - want["dH"].float()).norm() / want["dH"].float().norm()
        assert err <= 2 * F.U["bf16"]
    # a gradient that torch marks as negated, int32 ids, lists that are views
    Hg, Wg = F.on_gpu(H, "bf16").requires_grad_(), F.on_gpu(W, "bf16").requires_grad_()
    loss = linear_distillation(Hg, Wg, idg.int().t().contiguous().t(), tg.t().contiguous().t(), 2.0)
    g = torch.autograd.grad(loss, (Hg, Wg), torch.tensor(1.0j, device="cuda").conj().imag)
    assert torch.equal(g[0], -want["dH"]) and torch.equal(g[1], -want["dW"])


@pytest.mark.parametrize("dtype,N,d,V,K", [("bf16", 1030, 256, 5000, 30), ("f32", 300, 64, 700, 10)])
def test_repeats_streams_and_a_graph(dtype, N, d, V, K):
    rng = np.random.default_rng(20)
    H, W = operands(rng, N, d, V, dtype)
    ids, t = lists(rng, N, V, K, "ragged")
    a = F.on_gpu(H, dtype), F.on_gpu(W, dtype), torch.from_numpy(ids).cuda(), torch.from_numpy(t).cuda()
    want = call(*a, 1.5)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for got in (call(*a, 1.5), call(*a, 1.5, stream=side)):
        assert all(torch.equal(want[k], got[k]) for k in ("loss", "rows", "lse", "zt", "dH", "dW"))
    Hg, Wg = a[0].clone().requires_grad_(), a[1].clone().requires_grad_()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        loss = linear_distillation(Hg, Wg, *a[2:], 1.5)
        dH, dW = torch.autograd.grad(loss, (Hg, Wg))
    eager = linear_distillation(Hg, Wg, *a[2:], 1.5)      # afterwards, with the graph's own autograd graph alive
    up = torch.autograd.grad(eager, (Hg, Wg))
    assert torch.equal(up[0], want["dH"]) and torch.equal(up[1], want["dW"])
    for rep in range(3):
        for x in (loss, dH, dW):
            x.detach().fill_(7)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(loss, want["loss"][0]) and torch.equal(dH, want["dH"]) and torch.equal(dW, want["dW"]), rep


def test_capture_beside_a_living_eager_graph_is_refused(monkeypatch):
    """(The check alone: nothing is captured here.)"""
    H, W = torch.randn(8, 16, device="cuda", requires_grad=True), torch.randn(30, 16, device="cuda", requires_grad=True)
    ids, t = torch.zeros(8, 2, dtype=torch.int64, device="cuda"), torch.zeros(8, 2, device="cuda")
    loss = linear_distillation(H, W, ids, t)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
    with pytest.raises(RuntimeError, match="alive"):
        linear_distillation(H, W, ids, t)
    with pytest.raises(RuntimeError, match="alive"):
        linear_distillation(H.detach(), W, ids, t)
    with torch.no_grad():
        assert linear_distillation(H, W, ids, t) == loss
    assert linear_distillation(H.detach(), W.detach(), ids, t) == loss
    value = loss.item()
    del loss
    assert linear_distillation(H, W, ids, t).item() == value


@pytest.mark.parametrize("reduction", ["mean", "none"])
def test_capture_beside_a_living_eager_cross_entropy_is_refused(monkeypatch, reduction):
    """(The check alone, as above.)  The refusal ends with the graph of the loss, not with the loss's own name."""
    H, W = torch.randn(8, 16, device="cuda", requires_grad=True), torch.randn(30, 16, device="cuda", requires_grad=True)
    ids, t = torch.zeros(8, 2, dtype=torch.int64, device="cuda"), torch.zeros(8, 2, device="cuda")
    y = torch.zeros(8, dtype=torch.int64, device="cuda")
    loss = 2 * linear_cross_entropy(H, W, y, reduction=reduction)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
    with pytest.raises(RuntimeError, match="alive"):
        linear_distillation(H, W, ids, t)
    del loss
    linear_distillation(H, W, ids, t)


def test_teacher_to_student():
    """A teacher's lists as linear_topk writes them, and a student trained on them: the losses are the definition's on those lists."""
    rng = np.random.default_rng(23)
    N, V, K, T = 400, 3001, 32, 2.0
    Ht, Wt = operands(rng, N, 128, V, "bf16")
    H, W = operands(rng, N, 72, V, "bf16")
    z, ids, _ = linear_topk(F.on_gpu(Ht, "bf16"), F.on_gpu(Wt, "bf16"), K)
    Hg, Wg = F.on_gpu(H, "bf16").requires_grad_(), F.on_gpu(W, "bf16").requires_grad_()
    loss = linear_distillation(Hg, Wg, ids, z, T)
    loss.backward()
    r = F.distill(H, W, ids.cpu().numpy(), F.f64(z), T, np.full(N, 1 / N))
    assert abs(loss.item() - r["rows"].mean()) <= F.loss_bound(r, H, W, T).mean() + (N + 10) * F.U32 * r["rows"].mean()
    bH, bW = F.grad_bounds(r, H, W, T, "bf16", False)
    assert (np.abs(F.f64(Hg.grad) - r["dH"]) <= bH).all() and (np.abs(F.f64(Wg.grad) - r["dW"]) <= bW).all()
