"""GPU: logits near the largest number of 32 bits (vocabularies masked with the type's lowest value, whole groups of them, whole rows,
the end of the vocabulary) through every call that keeps a few logits per row.  The masks come in as a column of W that some rows of H
multiply by one: such a logit is the mask's value exactly, whatever the other columns add to it."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import few_logits as F                                    # noqa: E402
import test_gpu_beam as TB                                # noqa: E402
import test_gpu_distill as TD                             # noqa: E402
import test_gpu_topk as TK                                # noqa: E402
from conftest import set_plan                             # noqa: E402

LOW = float(torch.finfo(torch.bfloat16).min)              # -3.39e38, held by both types
HIGH = -LOW


def masked_operands(rng, N, d, V):
    """Column 0: groups are masked (in all rows but 1, 3 and the last of five or more); row 1: every logit is; row 2: one large logit; row 3:
    all but three are masked."""
    H, W = F.grid_operands(rng, N, d, V)
    H[:, :4], W[:, :4] = 0, 0
    H[:, 0] = 1
    W[:min(64, V // 2), 0] = LOW
    W[V // 2:V // 2 + V // 4, 0] = LOW                    # groups in the middle, each whole
    W[V - V // 16 - 1:, 0] = LOW                          # and the last ones, whatever the last one holds
    if N > 3:
        H[1, :2] = 0, 1
        W[:, 1] = LOW
        H[2, 2] = 1
        W[V // 2 - 1, 2] = HIGH
        H[3, 0], H[3, 3] = 0, 1
        W[:, 3] = LOW
        W[V // 2 - 3:V // 2, 3] = 0
    if N > 4:
        H[N - 1, 0] = 0
    return H, W


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("K", [1, 20, 200])
@pytest.mark.parametrize("N,d,V", [(1, 8, 300), (4, 64, 301), (5, 72, 20011), (4, 64, 40007), (20, 64, 66003), (64, 64, 333), (70, 96, 333), (300, 104, 5003)])
def test_masks_in_topk(dtype, K, N, d, V):
    H, W = masked_operands(np.random.default_rng(V + N), N, d, V)
    TK.check(H, W, K, dtype)


@pytest.mark.parametrize("knobs", [dict(FLCE_GENERIC=1), dict(FLCE_TILE=128), dict(FLCE_TILE=256)])
def test_masks_in_every_loop(monkeypatch, knobs):
    set_plan(monkeypatch, **knobs)
    H, W = masked_operands(np.random.default_rng(4), 300, 96, 3333)
    TK.check(H, W, 20, "bf16")


@pytest.mark.parametrize("K", [1, 60])
def test_masks_beside_a_floor(K):
    """Many rounds of tiles: what the vocabulary's first part gives as a floor for the rest."""
    N, d, V = 2100, 1024, 50000
    rng = np.random.default_rng(K)
    H, W = masked_operands(rng, N, d, V)
    Hg, Wg = F.on_gpu(H, "bf16"), F.on_gpu(W, "bf16")
    z, ids, lse = TK.call(Hg, Wg, K)
    for rows in (slice(0, 40), slice(N - 40, N)):
        full = Hg[rows].float() @ Wg.float().t()
        wz, wids, wlse = F.topk(F.f64(full), K)
        assert np.array_equal(ids[rows].cpu().numpy(), wids) and np.array_equal(F.f64(z[rows]), wz)
        assert (np.abs(F.f64(lse[rows]) - wlse) <= F.lse_bound(wlse, V)).all()


@pytest.mark.parametrize("K", [5, 60])
def test_infinities_and_nan_beside_a_floor(K):
    """Every place of the lists of rows with infinities in the first part, with and without NaN behind it, and of rows of nothing but NaN."""
    N, d, V = 2100, 1024, 50000
    H, W = F.grid_operands(np.random.default_rng(V + K), N, d, V)
    H[:, 1:4], W[:, 1:4] = 0, 0
    Hg, Wg = F.on_gpu(H, "bf16"), F.on_gpu(W, "bf16")
    Wg[100:100 + 64 * (K + 3):64, 2] = HIGH               # rows 2 .. 5: more infinities than places (a product past 32 bits)
    Wg[V - 9, 2] = LOW
    Hg[2:6, 2] = 4
    Hg[10:12, 2] = -4                                     # rows 10, 11: -inf there, one infinity at the end
    Wg[:, 3] = 1
    Wg[V - 9, 3] = 0
    Hg[6:10, 3] = float("inf")                            # rows 6 .. 9: infinities everywhere, NaN at one place of the end
    Hg[12] = float("nan")
    Hg[13, 5] = float("inf")                              # both infinities, and NaN where W is 0
    z, ids, lse = TK.call(Hg, Wg, K)
    full = Hg[:16].float() @ Wg.float().t()
    wz, wids, wlse = F.topk(F.f64(full), K)
    assert np.isinf(wz[2:6]).all() and np.isnan(wz[6:10, 0]).all() and np.isnan(wz[12]).all()
    assert np.array_equal(ids[:16].cpu().numpy(), wids) and np.array_equal(F.f64(z[:16]), wz, equal_nan=True)
    got, fin = F.f64(lse[:16]), np.isfinite(wlse)
    assert np.array_equal(got[~fin], wlse[~fin], equal_nan=True)
    assert (np.abs(got[fin] - wlse[fin]) <= F.lse_bound(wlse[fin], V)).all()


def log_softmax(z):
    m = z.max(-1, keepdims=True)
    return (z - m) - np.log(np.exp(z - m).sum(-1, keepdims=True))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("batch,beams,d,V,n_out", [(1, 4, 64, 301, 4), (3, 5, 72, 20011, 10), (30, 4, 64, 1501, 8)])
def test_masks_in_a_beam_step(dtype, batch, beams, d, V, n_out):
    """A beam whose logits are all the mask is uniform: its candidates are behind by log V, not level with its score."""
    rng = np.random.default_rng(batch)
    H, W = masked_operands(rng, batch * beams, d, V)
    scores = np.float32(np.tile(-4 - 0.25 * np.arange(beams), (batch, 1)))
    got = TB.step(H.reshape(batch, beams, d), W, scores, None, n_out, 2, 0, dtype)
    logp = log_softmax(H @ W.T).reshape(batch, beams, V)
    total = (scores.astype(np.float64)[..., None] + logp).reshape(batch, -1)
    # equal logits of a beam are equal scores: by beam, then by token; scores of different logits are no nearer than a grid's step
    order = np.argsort(-total, axis=1, kind="stable")[:, :n_out]
    want = np.take_along_axis(total, order, 1)
    assert np.array_equal(got[2], order // V) and np.array_equal(got[1], order % V)
    assert (np.abs(got[0] - want) <= F.lse_bound(0.0, V) + 4 * F.U32 * (np.abs(want) + 40)).all()


def masked_student(rng, N, d, V, dtype):
    """Operands, and the same without the mask's column: groups at the vocabulary's start, in its middle and at its end are masked in all
    rows but row 0."""
    H, W = TD.operands(rng, N, d, V, dtype)
    H[:, 0], W[:, 0] = 0, 0
    plain = H.copy(), W.copy()
    H[1:, 0] = 1
    free = np.arange(V // 3, V // 2)
    W[:, 0] = LOW
    W[free, 0] = 0
    return H, W, free, plain


@pytest.mark.parametrize("dtype,knobs", [("bf16", {}), ("f32", {}), ("bf16", dict(FLCE_GENERIC=1)), ("bf16", dict(FLCE_TILE=128)),
                                         ("bf16", dict(FLCE_TILE=256))])
@pytest.mark.parametrize("T", [1.0, 0.5, 3.0])
@pytest.mark.parametrize("N,d,V", [(130, 72, 1601), (600, 96, 5003)])
def test_masks_in_distillation(monkeypatch, dtype, knobs, T, N, d, V):
    set_plan(monkeypatch, **knobs)
    K = 20
    rng = np.random.default_rng(N)
    H, W, free, (H0, W0) = masked_student(rng, N, d, V, dtype)
    ids = np.stack([rng.permutation(free)[:K] for _ in range(N)])
    t = np.float32(rng.standard_normal((N, K)))
    ids[::7, 3:] = -1
    print(f"[case] masked distill {dtype} N={N} V={V} T={T} {knobs}", flush=True)
    r = F.distill(H, W, ids, t.astype(np.float64), T, np.ones(N))
    got = TD.call(F.on_gpu(H, dtype), F.on_gpu(W, dtype), torch.from_numpy(ids).cuda(), torch.from_numpy(t).cuda(), T, "sum")
    # bounds: those of the same operands without the mask's column, whose products are exact (a probability of 0 where it masks)
    assert (np.abs(F.f64(got["lse"]) - r["lse"]) <= F.logit_bound(H0, W0).max(1) / T + F.lse_bound(r["lse"], V)).all()
    assert (np.abs(F.f64(got["rows"]) - r["rows"]) <= F.loss_bound(r, H0, W0, T)).all()
    bH, bW = F.grad_bounds(r, H0, W0, T, dtype, False)    # (all columns but the mask's)
    assert (np.abs(F.f64(got["dH"]) - r["dH"])[:, 1:] <= bH[:, 1:]).all()
    assert (np.abs(F.f64(got["dW"]) - r["dW"])[:, 1:] <= bW[:, 1:]).all()


def test_temperatures_that_take_logits_past_32_bits():
    """Logits of 1e30 at a temperature of 1e-10: z / T is no number of 32 bits, the losses of rows with them are."""
    N, d, V, K, T = 40, 64, 700, 5, 1e-10
    H, W = np.zeros((N, d)), np.zeros((V, d))
    H[:, 0], W[:, 0] = 1, -np.ldexp(1.0, 100)
    W[100:110, 0] = 0
    ids = np.tile(100 + np.arange(K), (N, 1))
    t = np.zeros((N, K), np.float32)
    got = TD.call(F.on_gpu(H, "f32"), F.on_gpu(W, "f32"), torch.from_numpy(ids).cuda(), torch.from_numpy(t).cuda(), T, "sum")
    bound = F.lse_bound(np.log(10), V)
    assert (np.abs(F.f64(got["lse"]) - np.log(10)) <= bound).all()
    assert (np.abs(F.f64(got["rows"]) / T ** 2 - np.log(10 / K)) <= bound + (256 + 100) * F.U32 * (1 + np.log(K) + np.log(10))).all()
    q = np.where(np.arange(V) < 100, 0, np.where(np.arange(V) < 100 + K, 0.1 - 1 / K, np.where(np.arange(V) < 110, 0.1, 0.0)))
    assert (np.abs(F.f64(got["dW"])[:, 0] - T * N * q) <= T * N * (bound + 400 * F.U32)).all() and not got["dW"][:, 1:].any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_losses_of_rows_that_are_all_mask(dtype):
    """Such a row is uniform: its loss is log V minus the entropy of its list."""
    N, d, V, K = 90, 64, 1501, 9
    rng = np.random.default_rng(8)
    H, W = TD.operands(rng, N, d, V, dtype)
    H[:, 0], W[:, 0] = 0, LOW
    H[5:9, 0] = 1
    ids = np.stack([rng.permutation(V)[:K] for _ in range(N)])
    t = np.float32(rng.standard_normal((N, K)))
    got = TD.call(F.on_gpu(H, dtype), F.on_gpu(W, dtype), torch.from_numpy(ids).cuda(), torch.from_numpy(t).cuda(), 1.0, "sum")
    p = F.shares(ids, t.astype(np.float64), 1.0, V)[0]
    want = (p * (np.log(p) + np.log(V))).sum(1)
    assert (np.abs(F.f64(got["rows"]) - want)[5:9] <= F.lse_bound(0.0, V) + (256 + 100) * F.U32 * (1 + np.log(V) + 8)).all()
