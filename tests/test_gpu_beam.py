"""GPU: a beam search's step and the reordering of its states, against brute force over every candidate."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import few_logits as F                                    # noqa: E402
from paper_2511_17599_amd import binding as B             # noqa: E402
from paper_2511_17599_amd.torch_api import beam_step, linear_topk, reorder_states   # noqa: E402


def step(H, W, s, fin, n_out, eos, pad, dtype):
    """beam_step on numpy operands."""
    out = beam_step(F.on_gpu(H, dtype), F.on_gpu(W, dtype), torch.from_numpy(s).cuda().float(),
                    None if fin is None else torch.from_numpy(fin).cuda(), n_out, eos, pad)
    return [x.cpu().numpy() for x in out]


def score_bound(s, V):
    """z - lse and the sum with the score, one rounding each; the log-sum-exp's own."""
    s = np.where(np.isfinite(s), s, 0)
    return 4 * F.U32 * (np.abs(s) + 64) + F.lse_bound(32.0, V)


def check(rng, batch, beams, d, V, n_out, dtype, share=0.2, eos=3, pad=1):
    print(f"[case] beam {dtype} batch={batch} beams={beams} d={d} V={V} n_out={n_out}", flush=True)
    H, W = F.grid_operands(rng, batch * beams, d, V)
    H = H.reshape(batch, beams, d)
    s = np.sort(-20 + 4 * rng.standard_normal((batch, beams)).astype(np.float32), 1)[:, ::-1].copy()
    fin = rng.random((batch, beams)) < share if share is not None else None
    want = F.beam(H, W, s.astype(np.float64), fin, n_out, eos, pad)
    got = step(H, W, s, fin, n_out, eos, pad, dtype)
    # (no two candidates of different beams lie closer than the kernel's scores are exact: the seeds were not chosen, the gaps are)
    same = np.isclose(got[0], want[0], rtol=0, atol=score_bound(want[0], V)) | (got[0] == want[0])
    assert same.all()
    assert np.array_equal(got[1], want[1]) and np.array_equal(got[2], want[2]) and np.array_equal(got[3], want[3])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("batch,beams,d,V,n_out", [(1, 1, 8, 5, 5), (1, 1, 64, 1000, 4), (1, 4, 64, 5003, 4), (3, 2, 104, 300, 4),
                                                   (2, 64, 32, 700, 64), (16, 5, 72, 2049, 10), (30, 12, 40, 999, 12), (70, 3, 200, 1500, 3),
                                                   (5, 1, 16, 40, 8)])
def test_sizes(dtype, batch, beams, d, V, n_out):
    check(np.random.default_rng(batch * 100 + beams), batch, beams, d, V, n_out, dtype)


def test_without_flags_and_eos():
    check(np.random.default_rng(2), 4, 4, 64, 300, 4, "bf16", share=None, eos=-1)
    check(np.random.default_rng(3), 6, 3, 64, 12, 6, "f32", share=0.0, eos=5)          # the token is among the best now and then


def test_all_finished_and_fewer_candidates_than_results():
    rng = np.random.default_rng(4)
    check(rng, 3, 4, 64, 300, 10, "bf16", share=1.0)                                    # four candidates for ten results
    H, W = F.grid_operands(rng, 2, 16, 3)
    got = step(H.reshape(2, 1, 16), W, np.zeros((2, 1), np.float32), None, 8, -1, 7, "f32")      # three tokens for eight results
    assert (got[0][:, 3:] == -np.inf).all() and (got[1][:, 3:] == 7).all() and (got[2] == 0).all() and got[3][:, 3:].all()
    assert not got[3][:, :3].any() and sorted(got[1][0, :3]) == [0, 1, 2]


@pytest.mark.parametrize("rows", [(1, 4), (30, 4)])
def test_equal_scores_go_to_the_lower_beam(rows):
    batch, beams = rows
    rng = np.random.default_rng(5)
    H, W = F.grid_operands(rng, batch, 64, 800)
    H = np.repeat(H[:, None], beams, 1)                   # the same state in every beam
    W[500:520] = W[500]
    got = step(H, W, np.full((batch, beams), -3, np.float32), None, 6, -1, 0, "bf16")
    want = F.beam(H, W, np.full((batch, beams), -3.0), None, 6, -1, 0)
    assert np.array_equal(got[1], want[1]) and np.array_equal(got[2], want[2])
    assert (got[2][:, 0] == 0).all() and (got[2][:, 1] == 1).all()                      # one token, beam after beam


def test_dead_and_odd_scores():
    rng = np.random.default_rng(6)
    H, W = F.grid_operands(rng, 12, 32, 200)
    H = H.reshape(3, 4, 32)
    s = np.full((3, 4), -np.inf, np.float32)              # a first step: one live beam of four
    s[:, 0] = 0
    got, want = step(H, W, s, None, 4, -1, 0, "bf16"), F.beam(H, W, s.astype(np.float64), None, 4, -1, 0)
    assert (got[2] == 0).all() and np.array_equal(got[1], want[1])
    s[1] = -np.inf                                        # nothing live: every place is taken, in order of beams
    got = step(H, W, s, None, 4, -1, 0, "bf16")
    assert (got[0][1] == -np.inf).all() and (got[2][1] == 0).all() and len(set(got[1][1])) == 4
    s[2] = [0, np.nan, np.inf, 0]
    W[9, 0] = np.inf                                      # beams whose log-sum-exp is +inf, NaN where the state is 0 there
    got = step(H, W, s, None, 64, -1, 0, "f32")
    assert np.isnan(got[0][2, 0]) and got[0].shape == (3, 64)
    for b in range(3):                                    # every place written, with a candidate of its own
        assert len({(p, t) for p, t in zip(got[2][b], got[1][b])}) == 64 and (got[2][b] < 4).all() and (got[1][b] < 200).all()


@pytest.mark.parametrize("dtype,batch,beams,d,V,n_out", [("bf16", 2, 3, 64, 900, 5), ("f32", 30, 4, 40, 700, 4), ("bf16", 60, 5, 8, 600_001, 3)])
def test_outputs_and_workspace_end_where_they_say(dtype, batch, beams, d, V, n_out):
    """Poisoned workspace, words behind every output; the last shape's rows go through in chunks that cut a search."""
    rng = np.random.default_rng(8)
    H, W = F.grid_operands(rng, batch * beams, d, V)
    s = rng.standard_normal((batch, beams)).astype(np.float32)
    code = {"bf16": B.FLCE_DTYPE_BF16, "f32": B.FLCE_DTYPE_F32}[dtype]
    nb = B.flce_beam_workspace_bytes(batch, beams, d, V, n_out, code)
    ws = torch.full((nb + 256,), 0xFF, dtype=torch.uint8, device="cuda")
    n = batch * n_out
    out = [torch.full((n + 32,), 9, dtype=t, device="cuda") for t in (torch.float32, torch.int64, torch.int64, torch.uint8)]
    want = step(H.reshape(batch, beams, d), W, s, None, n_out, 3, 1, dtype)
    for rep in range(2):                                  # the second time on what the first left in the workspace
        assert B.flce_beam_step(F.on_gpu(H, dtype), F.on_gpu(W, dtype), torch.from_numpy(s).cuda(), None, batch, beams, d, V, n_out, 3, 1,
                                code, *out, ws, nb) == B.FLCE_OK
        torch.cuda.synchronize()
        assert (ws[nb:] == 0xFF).all()
        for x, w in zip(out, want):
            assert (x[n:] == 9).all() and np.array_equal(x[:n].cpu().numpy().reshape(batch, n_out), w)
    for b in (0, batch // 2, batch - 1):
        one = F.beam(H.reshape(batch, beams, d)[b:b + 1], W, s[b:b + 1].astype(np.float64), None, n_out, 3, 1)
        assert np.array_equal(want[1][b:b + 1], one[1]) and np.array_equal(want[2][b:b + 1], one[2])


def test_a_graph_and_other_streams():
    rng = np.random.default_rng(7)
    batch, beams, d, V = 4, 4, 256, 8000
    H, W = (F.on_gpu(x, "bf16") for x in (rng.standard_normal((batch, beams, d)), 0.05 * rng.standard_normal((V, d))))
    s = torch.from_numpy(rng.standard_normal((batch, beams)).astype(np.float32)).cuda()
    fin = torch.zeros(batch, beams, dtype=torch.bool, device="cuda")
    fin[1, 2] = True
    src = torch.randn(6, batch, beams, 50, device="cuda")
    want = beam_step(H, W, s, fin, eos_id=2)
    moved = reorder_states(want[2], src)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = beam_step(H, W, s, fin, eos_id=2)
        m2 = reorder_states(got[2], src)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and torch.equal(moved, m2)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = beam_step(H, W, s, fin, eos_id=2)
        m3 = reorder_states(out[2], src)
    for rep in range(3):
        out[0].fill_(0), out[1].fill_(-1), out[2].fill_(0), m3.fill_(0)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)) and torch.equal(m3, moved), rep


def plain_reorder(src, parents):
    return torch.stack([src[:, b][:, parents[b]] for b in range(parents.shape[0])], 1)


@pytest.mark.parametrize("dtype", [torch.uint8, torch.bfloat16, torch.float32, torch.int64])
@pytest.mark.parametrize("outer,batch,bi,bo,n", [(1, 1, 1, 1, 1), (3, 2, 1, 4, 33), (2, 5, 4, 4, 128), (1, 3, 8, 6, 1000), (4, 2, 16, 16, 77),
                                                 (2, 3, 64, 64, 40), (1, 2, 20, 33, 515), (7, 1, 3, 2, 100_003)])
def test_reorder(dtype, outer, batch, bi, bo, n):
    g = torch.Generator(device="cuda").manual_seed(n)
    src = torch.randint(0, 200, (outer, batch, bi, n), device="cuda", generator=g).to(dtype)
    par = torch.randint(0, bi, (batch, bo), device="cuda", generator=g)
    print(f"[case] reorder {dtype} {outer} {batch} {bi}->{bo} n={n}", flush=True)
    assert torch.equal(reorder_states(par, src), plain_reorder(src, par))
    wide = torch.full((outer, batch, bo, n + 13), 3, device="cuda").to(dtype)        # a part of longer rows: the rest stays
    reorder_states(par, src, out=wide[..., :n])
    assert torch.equal(wide[..., :n], plain_reorder(src, par)) and (wide[..., n:] == 3).all()
    if bi == bo and bo <= 16:
        same = src.clone()
        assert reorder_states(par, same, out=same) is same and torch.equal(same, plain_reorder(src, par))


@pytest.mark.parametrize("pad", [0, 12])
def test_reorder_states_beyond_32_bits(pad):
    """Rows of more than 2^31 bytes, slabs of more than 2^32, as wide vectors and (pad: rows 4 bytes off) as narrow ones; in place too."""
    n = (1 << 31) + 64
    src = torch.empty(2, 1, 2, n + pad, dtype=torch.uint8, device="cuda")
    for o in range(2):
        for j in range(2):
            src[o, 0, j] = (torch.arange(n + pad, device="cuda") % 251 + 2 * o + j).to(torch.uint8)
    par = torch.tensor([[1, 0]], device="cuda")
    part = src[..., :n]
    moved = reorder_states(par, part)
    for o in range(2):
        for j in range(2):
            assert torch.equal(moved[o, 0, j], part[o, 0, 1 - j])
    reorder_states(par, part, out=part)
    for o in range(2):
        for j in range(2):
            assert torch.equal(moved[o, 0, j], part[o, 0, j])


def test_reorder_rows_of_odd_addresses_and_in_place_parts():
    par = torch.tensor([[1, 1, 0], [2, 0, 1]], device="cuda")
    base = torch.arange(4 * 6 * 37 + 5, device="cuda").to(torch.uint8)
    src = base[5:].reshape(4, 2, 3, 37)
    assert torch.equal(reorder_states(par, src), plain_reorder(src, par))
    room = torch.randn(4, 2, 3, 64, device="cuda")
    want = room.clone()
    want[..., :40] = plain_reorder(room[..., :40], par)
    reorder_states(par, room[..., :40], out=room[..., :40])
    assert torch.equal(room, want)
    first = torch.randn(2, 3, 9, 4, device="cuda")        # the batch is the first dimension
    assert torch.equal(reorder_states(par, first, dim=0), plain_reorder(first[None], par)[0])


def test_reorder_refuses_and_reports():
    par = torch.tensor([[0, 3], [-1, 1]], device="cuda")
    src = torch.randn(3, 2, 2, 20, device="cuda")
    dst = torch.full_like(src, 5.0)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    reorder_states(torch.zeros_like(par), src, status=status)
    assert status.item() == 0
    reorder_states(par, src, out=dst, status=status)
    assert status.item() == B.FLCE_ERR_TARGET_RANGE
    assert torch.equal(dst[:, 0, 0], src[:, 0, 0]) and (dst[:, 0, 1] == 5).all() and (dst[:, 1, 0] == 5).all() and torch.equal(dst[:, 1, 1], src[:, 1, 1])
    with pytest.raises(ValueError):
        reorder_states(par, src.transpose(2, 3))
    with pytest.raises(ValueError):
        reorder_states(par, src[..., ::2])
    with pytest.raises(ValueError):
        reorder_states(par, src, out=torch.empty(3, 2, 3, 20, device="cuda"))
    with pytest.raises(ValueError):
        reorder_states(par, src.transpose(0, 1))
    with pytest.raises(TypeError):
        reorder_states(par, src, status=torch.zeros(1, device="cuda"))
    with pytest.raises(RuntimeError):                     # part of itself
        room = torch.randn(1, 2, 2, 30, device="cuda")
        reorder_states(par, room[..., :20], out=room[..., 5:25])
    empty = reorder_states(par, src[..., :0])
    assert empty.shape == (3, 2, 2, 0)


def test_a_whole_search():
    """A search as a program runs it: one beam widened to four, a step, the states reordered in place, until all have ended.  The
    model's state is a vector that takes up the token; every step is compared with brute force on the same states."""
    rng = np.random.default_rng(11)
    batch, beams, d, V, eos, pad = 3, 4, 32, 300, 5, 0
    E = F.grid(rng.standard_normal((V, d)), 2.0 ** -4, 1.0)
    W = F.grid(rng.standard_normal((V, d)), 2.0 ** -10, 0.1)
    W[eos] += 2.0 ** -6
    W = np.clip(W, -127 * 2.0 ** -10, 127 * 2.0 ** -10)
    h = F.grid(rng.standard_normal((batch, 1, d)), 2.0 ** -4, 1.0)
    Wg, Eg = F.on_gpu(W, "bf16"), F.on_gpu(E, "bf16")
    state = F.on_gpu(h, "bf16")
    scores = torch.zeros(batch, 1, device="cuda")
    fin = torch.zeros(batch, 1, dtype=torch.bool, device="cuda")
    history = torch.zeros(batch, 1, 0, dtype=torch.int64, device="cuda")
    for n in range(6):
        want = F.beam(F.f64(state), W, F.f64(scores), fin.cpu().numpy(), beams, eos, pad)
        scores, tokens, parents, fin = beam_step(state, Wg, scores, fin, beams, eos, pad)
        assert np.allclose(F.f64(scores), want[0], rtol=0, atol=score_bound(want[0], V).max())
        assert np.array_equal(tokens.cpu().numpy(), want[1]) and np.array_equal(parents.cpu().numpy(), want[2])
        state = reorder_states(parents, state, dim=0) if n == 0 else reorder_states(parents, state, out=state, dim=0)
        history = torch.cat([reorder_states(parents, history, dim=0), tokens[..., None]], 2)
        state.copy_((torch.round((state.float() * 0.5 + Eg[tokens].float()) * 16).clamp(-127, 127) / 16))
    assert history.shape == (batch, beams, 6)
    total = torch.zeros(batch, beams, dtype=torch.float64)    # the scores are the sums of their tokens' log-probabilities
    for b in range(batch):
        for j in range(beams):
            x, done = h[b, 0], False
            for v in history[b, j].tolist():
                if not done:
                    z = W @ x
                    total[b, j] += z[v] - F.logsumexp(z[None])[0]
                done = done or v == eos
                x = np.clip(np.round((x * 0.5 + E[v]) * 16), -127, 127) / 16
    assert np.allclose(total.numpy(), F.f64(scores), rtol=0, atol=6 * score_bound(np.array(60.0), V))
    assert linear_topk(state, Wg, 3)[1].shape == (batch, beams, 3)
