"""Plain 64-bit forms of the operators that keep a few logits per row, and the bounds that their results are held to.

Written from the definitions, without the library.  Bounds count roundings: u(t) = finfo(t).eps / 2 relative to each value that
is rounded to t, a sum of n terms in 32 bits is off by at most n 2^-24 of the sum of their magnitudes, in any order."""
import numpy as np
import torch

U32 = 2.0 ** -24
U = {"bf16": 2.0 ** -8, "f32": U32}
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def grid(x, step, scale):
    """Multiples of a step, at most 127: products and sums of such values are exact in 32 bits."""
    return np.clip(np.round(x * (scale / step)), -127, 127) * step


def grid_operands(rng, N, d, V):
    return grid(rng.standard_normal((N, d)), 2.0 ** -4, 1.0), grid(rng.standard_normal((V, d)), 2.0 ** -10, 0.05)


def on_gpu(x, dtype):
    return torch.from_numpy(np.asarray(x)).to("cuda", torch.float32).to(DT[dtype])


def f64(t):
    return t.detach().double().cpu().numpy()


def logsumexp(z):
    m = z.max(-1, keepdims=True)
    m0 = np.where(np.isfinite(m), m, 0.0)
    with np.errstate(divide="ignore", over="ignore"):
        return (m0 + np.log(np.exp(z - m0).sum(-1, keepdims=True)))[..., 0]


def topk(z, K):
    """NaN above all, then by value, equal ones by position."""
    v = np.where(np.isnan(z), np.inf, z) + 0.0
    ids = np.lexsort((np.broadcast_to(np.arange(z.shape[1]), z.shape), -v, ~np.isnan(z)), axis=-1)[:, :K]
    return np.take_along_axis(z, ids, 1), ids, logsumexp(z)


def lse_bound(lse, V):
    """The sum of V exponentials: 18 additions inside a group of 16 per lane, at most V / 4096 + 20 from group to group and lane to
    lane; an exponent is rounded twice (at most 64 of it counts: 2^-64 adds nothing); logarithm and the last sum."""
    return (18 + V / 4096 + 20 + 2 * 64 * 0.7 + 4) * U32 + 2 * U32 * np.abs(lse)


def shares(ids, t, T, V):
    """(share of each entry, 0 where there is none; whether the row counts; whether it is out of range)"""
    bad = (ids >= V).any(1)
    here = (ids >= 0) & (ids < V) & ~(t == -np.inf)
    counts = here.any(1) & ~bad
    x = np.where(here, t / T, -np.inf)
    m = np.where(here.any(1), x.max(1), 0.0)[:, None]
    e = np.where(here, np.exp(x - m), 0.0)
    s = e.sum(1, keepdims=True)
    return e / np.where(s > 0, s, 1.0), here, counts, bad


def distill(H, W, ids, t, T, gamma):
    """Losses per row, lse, and the gradients for upstream gradients gamma per row (those of rows that do not count are not used);
    with what the bounds need."""
    V = W.shape[0]
    z = H @ W.T
    p, here, counts, bad = shares(ids, t, T, V)
    at = np.where(here, ids, 0)
    lse = logsumexp(z / T)
    zt = np.where(here, np.take_along_axis(z, at, 1), 0.0)
    logp = np.log(np.where(p > 0, p, 1.0))
    rows = T * T * (p * (logp - zt / T + lse[:, None])).sum(1) * counts
    q = np.exp(z / T - lse[:, None])
    g = q.copy()
    np.add.at(g, (np.arange(len(g))[:, None], at), -p)
    gam = np.where(counts, gamma, 0.0)
    G = T * gam[:, None] * g
    return dict(z=z, p=p, here=here, counts=counts, bad=bad, zt=zt, lse=lse, rows=rows, q=q, g=g, G=G, gam=gam, dH=G @ W, dW=G.T @ H)


def logit_bound(H, W):
    """A logit's sum over d, and as much again for the fp32 loop's parts."""
    return 2 * (H.shape[1] + 2) * U32 * (np.abs(H) @ np.abs(W).T)


def loss_bound(r, H, W, T):
    """Per row: logits and lse as they are bounded, the list's own softmax (256 terms at most, exponents as in lse_bound)."""
    dz = logit_bound(H, W).max(1) / T
    dl = dz + lse_bound(r["lse"], W.shape[0])
    size = (r["p"] * (np.abs(np.log(np.where(r["p"] > 0, r["p"], 1.0))) + np.abs(r["zt"]) / T + np.abs(r["lse"])[:, None])).sum(1)
    return T * T * (dz + dl + (256 + 100) * U32 * (1 + size)) * r["counts"]


def grad_bounds(r, H, W, T, dtype, per_row):
    """G rounded to dtype (its probability off by the logit's and lse's error first), products and sums in 32 bits, the result rounded."""
    V, N = W.shape[0], H.shape[0]
    dq = (2 * logit_bound(H, W) / T + lse_bound(r["lse"], V)[:, None] + 8 * U32 + 2 * U32 * np.abs(r["z"] / T - r["lse"][:, None])) * r["q"]
    listed = np.abs(r["g"] - r["q"])                       # the shares, at their places
    dg = dq + (256 + 100) * U32 * listed
    scale = T * np.abs(r["gam"])[:, None]
    eG = scale * (dg + U[dtype] * (np.abs(r["g"]) + dg) + 4 * U32 * np.abs(r["g"]))
    aG = np.abs(r["G"])
    dH = eG @ np.abs(W) + (V + 4) * U32 * (aG @ np.abs(W))
    dW = eG.T @ np.abs(H) + (N + 4) * U32 * (aG.T @ np.abs(H))
    return dH + U[dtype] * (np.abs(r["dH"]) + dH) + 1e-38, dW + U[dtype] * (np.abs(r["dW"]) + dW) + 1e-38


def beam(H, W, scores, finished, n_out, eos, pad):
    """[batch, beams, d] -> (scores, tokens, parents, finished), brute force over every candidate."""
    batch, beams, _ = H.shape
    V = W.shape[0]
    out = np.full((batch, n_out), -np.inf), np.full((batch, n_out), pad), np.zeros((batch, n_out), int), np.ones((batch, n_out), bool)
    for b in range(batch):
        cand = []
        for j in range(beams):
            if finished is not None and finished[b, j]:
                cand.append((-scores[b, j], j, 0, pad, True))
                continue
            z = W @ H[b, j]
            s = scores[b, j] + (z - logsumexp(z[None])[0])
            cand += [(-s[v], j, k, v, v == eos) for k, v in enumerate(np.lexsort((np.arange(V), -z))[:n_out])]
        for r, (s, j, _, v, f) in enumerate(sorted(cand)[:n_out]):
            out[0][b, r], out[1][b, r], out[2][b, r], out[3][b, r] = -s, v, j, f
    return out
