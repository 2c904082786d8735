"""GPU: a row's largest logits.  On operands whose products are exact in 32 bits the logits are the plain form's bit for bit and the ids
are compared one by one, equal logits among them."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import few_logits as F                                    # noqa: E402
from conftest import set_plan                             # noqa: E402
from paper_2511_17599_amd import binding as B             # noqa: E402
from paper_2511_17599_amd.torch_api import linear_topk    # noqa: E402

CODE = {"bf16": B.FLCE_DTYPE_BF16, "f32": B.FLCE_DTYPE_F32}


def call(H, W, K, stream=None):
    """The call on a poisoned workspace, with words behind every output that have to stay."""
    (N, d), V, dt = H.shape, W.shape[0], CODE["bf16" if H.dtype is torch.bfloat16 else "f32"]
    nb = B.flce_topk_workspace_bytes(N, d, V, K, dt)
    ws = torch.full((nb + 256,), 0xFF, dtype=torch.uint8, device="cuda")
    z = torch.full((N * K + 64,), 7.0, device="cuda")
    ids = torch.full((N * K + 64,), -9, dtype=torch.int64, device="cuda")
    lse = torch.full((N + 64,), 7.0, device="cuda")
    assert B.flce_topk(H, W, N, d, V, K, dt, z, ids, lse, ws, nb, stream) == B.FLCE_OK
    torch.cuda.synchronize()
    assert (z[N * K:] == 7).all() and (ids[N * K:] == -9).all() and (lse[N:] == 7).all() and (ws[nb:] == 0xFF).all()
    return z[:N * K].reshape(N, K), ids[:N * K].reshape(N, K), lse[:N]


def check(H, W, K, dtype):
    """numpy operands, exact in dtype."""
    print(f"[case] topk {dtype} N={H.shape[0]} d={H.shape[1]} V={W.shape[0]} K={K}", flush=True)
    z, ids, lse = call(F.on_gpu(H, dtype), F.on_gpu(W, dtype), K)
    with np.errstate(invalid="ignore"):
        full = H @ W.T
    wz, wids, wlse = F.topk(full, K)
    assert np.array_equal(ids.cpu().numpy(), wids)
    assert np.array_equal(F.f64(z), wz, equal_nan=True)
    got, fin = F.f64(lse), np.isfinite(wlse)
    assert np.array_equal(got[~fin], wlse[~fin], equal_nan=True)
    assert (np.abs(got[fin] - wlse[fin]) <= F.lse_bound(wlse[fin], W.shape[0])).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,d,V,K", [
    (1, 8, 1, 1), (1, 64, 15, 15), (2, 40, 16, 3), (3, 104, 17, 17), (16, 32, 257, 256), (17, 72, 1000, 20), (32, 128, 20011, 5),
    (33, 256, 4099, 64), (64, 520, 33000, 10), (64, 64, 300, 200), (5, 1032, 16385, 1), (65, 8, 5, 5), (65, 64, 40, 33), (100, 96, 1, 1),
    (300, 200, 3001, 50), (257, 128, 20011, 256), (1030, 264, 2049, 17)])
def test_sizes(dtype, N, d, V, K):
    rng = np.random.default_rng(N * 1000003 + V)
    H, W = F.grid_operands(rng, N, d, V)
    check(H, W, K, dtype)


@pytest.mark.parametrize("knobs", [dict(FLCE_GENERIC=1), dict(FLCE_TILE=128), dict(FLCE_TILE=256)])
@pytest.mark.parametrize("d", [96, 104])
def test_every_loop(monkeypatch, knobs, d):
    set_plan(monkeypatch, **knobs)
    H, W = F.grid_operands(np.random.default_rng(3), 600, d, 3333)
    check(H, W, 40, "bf16")


def test_the_copy_of_h():
    """Large enough that the forward makes its pre-tiled copy of H, with both edges of the tuned loop's hidden-size forms."""
    for N, d, V in ((2100, 1024, 33000), (2100, 1032, 33000)):
        assert " h_copy=1/" in B.flce_plan_describe(N, d, V, B.FLCE_DTYPE_BF16)
        H, W = F.grid_operands(np.random.default_rng(d), N, d, V)
        Hg, Wg = F.on_gpu(H, "bf16"), F.on_gpu(W, "bf16")
        z, ids, lse = call(Hg, Wg, 30)
        full = Hg.float() @ Wg.float().t()                # exact, in any order
        for rows in (slice(0, 64), slice(1000, 1064), slice(N - 64, N)):
            wz, wids, wlse = F.topk(F.f64(full[rows]), 30)
            assert np.array_equal(ids[rows].cpu().numpy(), wids) and np.array_equal(F.f64(z[rows]), wz)
            assert (np.abs(F.f64(lse[rows]) - wlse) <= F.lse_bound(wlse, V)).all()
        assert torch.equal(z[:, 0], full.max(1).values)


@pytest.mark.parametrize("knobs,N,d,V,K", [(dict(), 2100, 1024, 50000, 5), (dict(), 2100, 1024, 50000, 60), (dict(FLCE_TILE=128), 1100, 1024, 60000, 20)])
def test_floors(monkeypatch, knobs, N, d, V, K):
    """Calls of many rounds keep only the groups that reach a floor from the vocabulary's first part: rows whose largest logits all lie
    in that part, all behind it, are all equal, NaN, infinite or -inf."""
    set_plan(monkeypatch, **knobs)
    rng = np.random.default_rng(V + K)
    H, W = F.grid_operands(rng, N, d, V)
    H[0] = 0
    W[:, :4] = 0
    H[:, :4] = 0
    H[1:40, 0], W[:200, 0] = 7, 0.12                      # large at the start
    H[1:20, 1], W[V - 300:, 1] = 7, 0.12                  # and at the end
    H[40:60, 2], W[V // 2:, 2] = -7.9375, 0.12            # low behind the middle
    Hg, Wg = F.on_gpu(H, "bf16"), F.on_gpu(W, "bf16")

    def compare(rows):
        z, ids, lse = call(Hg, Wg, K)
        full = Hg[rows].float() @ Wg.float().t()
        wz, wids, wlse = F.topk(F.f64(full), K)
        assert np.array_equal(ids[rows].cpu().numpy(), wids) and np.array_equal(F.f64(z[rows]), wz, equal_nan=True)
        fin = np.isfinite(wlse)
        got = F.f64(lse[rows])
        assert (np.abs(got[fin] - wlse[fin]) <= F.lse_bound(wlse[fin], V)).all() and np.array_equal(got[~fin], wlse[~fin], equal_nan=True)

    compare(slice(0, 64))
    compare(slice(N - 64, N))
    Wg[7, 3] = float("inf")                               # K and more infinities in the first part for rows 2 .. 9, NaN behind it
    Wg[100:100 + 64 * K:64, 3] = float("inf")
    Wg[V - 9, 3] = float("nan")
    Hg[2:10, 3] = 1
    Hg[10:12, 3] = -1
    torch.cuda.synchronize()
    z, ids, lse = call(Hg[:N].contiguous(), Wg, K)
    assert (ids[2:12, 0] == V - 9).all() and torch.isnan(z[:, 0]).all()      # (0 times an infinity: every row)


@pytest.mark.parametrize("N", [3, 70])
def test_more_groups_than_lds_holds_and_chunks_of_rows(N):
    V, d = 600_001, 8
    rng = np.random.default_rng(N)
    H, W = F.grid_operands(rng, N, d, V)
    check(H, W, 100, "bf16")
    check(H, W, 100, "f32")


def test_rows_in_several_chunks():
    N, d, V = 700, 8, 600_001                             # 256 rows of fp32 logits at a time
    assert B.flce_topk_workspace_bytes(N, d, V, 4, B.FLCE_DTYPE_BF16) < 2 * 256 * V * 4
    rng = np.random.default_rng(9)
    H, W = F.grid_operands(rng, N, d, V)
    z, ids, lse = call(F.on_gpu(H, "bf16"), F.on_gpu(W, "bf16"), 4)
    for i in (0, 255, 256, 511, 512, 699):
        wz, wids, wlse = F.topk(H[i:i + 1] @ W.T, 4)
        assert np.array_equal(ids[i:i + 1].cpu().numpy(), wids) and np.array_equal(F.f64(z[i:i + 1]), wz)
        assert (np.abs(F.f64(lse[i:i + 1]) - wlse) <= F.lse_bound(wlse, V)).all()


@pytest.mark.parametrize("N", [2, 40, 300])
def test_w_beyond_32_bits_of_bytes(N):
    """Largest logits whose rows of W lie on both sides of 2^31 and 2^32 bytes."""
    V, d = 600_007, 4096                                  # 4.9 GB
    W = torch.zeros(V, d, dtype=torch.bfloat16, device="cuda")
    at = [V - 1, (1 << 32) // (2 * d), (1 << 32) // (2 * d) - 1, (1 << 31) // (2 * d), 0, V - 300]
    for i, v in enumerate(at):
        W[v, d - 1 - i] = 6 - i
    H = torch.ones(N, d, dtype=torch.bfloat16, device="cuda")
    z, ids, lse = call(H, W, 8)
    assert ids.tolist() == [at + [1, 2]] * N and z.tolist() == [[6., 5., 4., 3., 2., 1., 0., 0.]] * N
    want = np.log(V - 6 + np.exp(np.arange(1.0, 7.0)).sum())
    assert (np.abs(F.f64(lse) - want) <= F.lse_bound(want, V)).all()


@pytest.mark.parametrize("N", [4, 130])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("K", [1, 60, 256])
def test_equal_logits_go_to_the_lowest_id(N, dtype, K):
    rng = np.random.default_rng(11)
    H, W = F.grid_operands(rng, N, 64, 9001)
    H[0] = 0                                              # every logit equal
    W[5000:8000] = W[5000]                                # a run of equal ones
    W[100:9000:97] = W[42]                                # and some far apart
    H[1] = W[5000] * 16                                   # the run is the largest
    H[2] = W[42] * 16
    H[3] = -np.abs(H[3])
    W[7000] = 0
    check(H, W, K, dtype)


@pytest.mark.parametrize("N", [2, 90])
@pytest.mark.parametrize("K", [7, 256])
def test_a_band_of_large_logits(N, K):
    """Thousands of candidates above the bound that the groups' maxima give: in consecutive positions, every one different."""
    V = 20000
    H, W = np.zeros((N, 16)), np.zeros((V, 16))
    H[:, 0], H[:, 1] = 1, 2.0 ** -7
    band = np.arange(3000, 3000 + 12000)
    x = np.random.default_rng(5).permutation(12000)
    W[band, 0] = 1 + x // 128 / 128.0
    W[band, 1] = x % 128 / 128.0
    check(H, W, K, "bf16")
    check(H, W, K, "f32")


@pytest.mark.parametrize("N", [6, 80])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_infinities_and_nan(N, dtype):
    V, d, K = 3000, 32, 20
    H, W = F.grid_operands(np.random.default_rng(21), N, d, V)
    H[:, 0] = np.abs(H[:, 0]) + 0.5
    W[17, 0] = np.inf                                     # +inf in every row's logit 17
    W[1900, 0] = -np.inf
    check(H, W, K, dtype)
    W[2500, 3] = np.nan                                   # NaN in every row: above +inf, and the log-sum-exp's value
    W[40, 3] = np.nan
    check(H, W, K, dtype)
    H2, W2 = F.grid_operands(np.random.default_rng(22), N, d, 40)
    H2[1] = 0
    H2[1, 0] = 1
    W2[:, 0] = -np.inf
    H2[:, 0] = np.where(np.arange(N) == 1, 1.0, 0.5)
    check(H2, W2, 40, dtype)                              # nothing but -inf


@pytest.mark.parametrize("dtype,N,d,V,K", [("bf16", 4, 768, 50257, 20), ("bf16", 500, 256, 8000, 64), ("f32", 200, 128, 3000, 9)])
def test_repeats_streams_and_a_graph(dtype, N, d, V, K):
    rng = np.random.default_rng(31)
    H, W = (F.on_gpu(x, dtype) for x in (rng.standard_normal((N, d)), 0.05 * rng.standard_normal((V, d))))
    want = call(H, W, K)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for got in (call(H, W, K), call(H, W, K, side)):
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    with torch.cuda.stream(side):
        got = linear_topk(H, W, K)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    nb = B.flce_topk_workspace_bytes(N, d, V, K, CODE[dtype])
    ws = torch.empty(nb, dtype=torch.uint8, device="cuda")
    out = [torch.empty_like(t.contiguous()) for t in want]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        assert B.flce_topk(H, W, N, d, V, K, CODE[dtype], *out, ws, nb, torch.cuda.current_stream()) == B.FLCE_OK
    for rep in range(3):
        ws.fill_(rep * 77)
        for t in out:
            t.fill_(3)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)), rep


def test_front_end_shapes_and_strides():
    rng = np.random.default_rng(41)
    H, W = F.grid_operands(rng, 24, 64, 500)
    Hg, Wg = F.on_gpu(H, "f32"), F.on_gpu(W, "f32")
    z, ids, lse = linear_topk(Hg.reshape(2, 3, 4, 64), Wg, 6)
    assert z.shape == ids.shape == (2, 3, 4, 6) and lse.shape == (2, 3, 4) and not z.requires_grad
    wz, wids, _ = F.topk(H @ W.T, 6)
    assert np.array_equal(ids.reshape(24, 6).cpu().numpy(), wids)
    one = linear_topk(Hg[5], Wg, 6)                       # a single token's vector
    assert one[1].shape == (6,) and np.array_equal(one[1].cpu().numpy(), wids[5]) and one[2].shape == ()
    wide = torch.zeros(24, 128, device="cuda")
    wide[:, 1::2] = Hg
    got = linear_topk(wide[:, 1::2], Wg.t().contiguous().t(), 6)
    assert torch.equal(got[1].reshape(-1), ids.reshape(-1))
    off = torch.zeros(24 * 64 + 1, device="cuda")         # contiguous, but not 16-byte aligned: the library refuses it
    off[1:] = Hg.reshape(-1)
    with pytest.raises(RuntimeError):
        linear_topk(off[1:].reshape(24, 64), Wg, 6)
    for k in (0, 257, 501):
        with pytest.raises(ValueError):
            linear_topk(Hg, Wg, k)
    with pytest.raises(ValueError):
        linear_topk(Hg[:0], Wg, 3)
