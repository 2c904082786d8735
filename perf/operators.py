"""Performance cases of the operators around the projection that keep a few logits per row: the largest logits of each row,
distillation from a teacher's largest logits, the step of a beam search and the reordering of its states.

Hidden states ~ N(0, 1), vocabulary weights ~ N(0, 0.02^2), as the repository's recipe has them.  The selections take both
on the grids of an 8-bit quantised model (multiples of 2^-4 and of 2^-10, at most 127 steps): every product and every sum of
them is exact in 32 bits, so that two computations of a row have the same logits, equal logits among them, and the selected
ids can be compared one by one.

A case: "op" and the sizes it takes.
  topk    : N rows, d, V, K largest logits, dtype
  distill : N, d, V, K entries a list, dtype, T (temperature), reduction, "empty" (share of rows without entries), "ragged"
            (lists end early, as lists cut by probability do)
  beam    : batch x beams rows, d, V, n_out results per batch element, dtype, "done" (share of finished beams)
  reorder : outer (tensors of a state: layers x keys and values), batch, beams, `used` of `room` bf16 values per row
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _topk(name, N, d, V, K, dtype="bf16"):
    return dict(name=name, op="topk", N=N, d=d, V=V, K=K, dtype=dtype)


def _distill(name, N, d, V, K, dtype="bf16", T=1.0, reduction="mean", empty=0.0, ragged=False):
    return dict(name=name, op="distill", N=N, d=d, V=V, K=K, dtype=dtype, T=T, reduction=reduction, empty=empty, ragged=ragged)


def _beam(name, batch, beams, d, V, n_out, dtype="bf16", done=0.0):
    return dict(name=name, op="beam", batch=batch, beams=beams, d=d, V=V, n_out=n_out, dtype=dtype, done=done)


def _reorder(name, outer, batch, beams, used, room):
    return dict(name=name, op="reorder", outer=outer, batch=batch, beams=beams, used=used, room=room)


def listed():
    return [
        # the largest log-probabilities of one new token with a GPT-2-sized head: latency counts
        _topk("one_token_topk", 1, 768, 50257, 20),
        # a small fp32 model that writes its lists for a batch, ragged sizes
        _topk("small_f32_topk", 1000, 512, 10007, 50, "f32"),
        # a Llama-3-8B-sized teacher that writes its lists for half a batch
        _topk("teacher_topk", 4096, 4096, 128256, 64),
        # the repository's fp32 workload's sizes: a unit-test sized student, every launch counts
        _distill("tiny_f32_distill", 256, 256, 4096, 16, "f32", T=2.0, empty=0.05),
        # bf16 with a hidden size that is no multiple of 32, lists cut by probability, summed loss
        _distill("odd_width_distill", 1030, 200, 20011, 50, reduction="sum", ragged=True, empty=0.1),
        # one loss per row, weighted by the caller: a translation-sized head
        _distill("weighted_rows_distill", 2048, 1024, 32000, 32, T=2.0, reduction="none", empty=0.1),
        # a Llama-3-8B-sized student on the lists of a teacher of the same vocabulary
        _distill("llama3_8b_distill", 8192, 4096, 128256, 32, T=1.5, empty=0.1),
        # one sentence translated or summarised with a GPT-2-sized head: latency counts
        _beam("one_sentence_beams", 1, 4, 768, 50257, 4),
        # a batch of sentences with a Llama-3-8B-sized head, one new token each: the weights are what is read
        _beam("batch_of_beams", 8, 4, 4096, 128256, 4, done=0.1),
        # a large batch, candidates for twice the beams, ragged sizes
        _beam("large_batch_of_beams", 60, 5, 1024, 32003, 10, done=0.2),
        # the states of the one sentence: keys and values of 12 layers, 100 of 1024 positions of 768 values
        _reorder("one_sentence_states", 24, 1, 4, 100 * 768, 1024 * 768),
        # the states of the batch of sentences: keys and values of 32 layers, 600 of 1024 positions of 8 heads of 128
        _reorder("batch_of_states", 64, 8, 4, 600 * 1024, 1024 * 1024),
    ]


def _cost(c):
    if c["op"] == "reorder":
        return 4.0 * c["outer"] * c["batch"] * c["beams"] * c["used"]
    rows = c["batch"] * c["beams"] if c["op"] == "beam" else c["N"]
    return (8.0 if c["op"] == "distill" else 2.0) * rows * c["d"] * c["V"] * (16 if c["dtype"] == "f32" else 1)


def draw(rng):
    """A case of the same ranges: sizes spread over their logarithm, odd ones among them."""
    def size(lo, hi, step=1):
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / step)) * step))

    while True:
        op = rng.choice(("topk", "topk", "distill", "distill", "beam", "beam", "reorder"))
        top = max(_cost(c) for c in listed() if c["op"] == op)
        dtype = "f32" if rng.random() < 0.25 else "bf16"
        if dtype == "f32":
            d, V, rows = size(64, 1024, 8), size(512, 32768), 2048
        else:
            d = size(128, 4096, 64) if rng.random() < 5 / 6 else size(40, 1024, 32) + 8
            V, rows = size(2048, 131072), 8192
        if op == "topk":
            c = _topk("", size(1, rows), d, V, size(1, 200), dtype)
        elif op == "distill":
            c = _distill("", size(64, rows), d, V, size(1, 128), dtype, rng.choice((1.0, 1.0, 2.0, 3.5)),
                         rng.choice(("mean", "sum", "none")), rng.choice((0.0, 0.05, 0.3)), rng.random() < 0.5)
        elif op == "beam":
            beams = rng.choice((1, 2, 3, 4, 5, 8, 12))
            c = _beam("", size(1, 64), beams, d, V, rng.choice((beams, 2 * beams, size(1, 16))), dtype, rng.choice((0.0, 0.1, 0.4)))
        else:
            width = size(128, 2048, 8)
            c = _reorder("", size(1, 96), size(1, 32), rng.choice((1, 2, 3, 4, 5, 8, 12)), width * size(1, 900), width * 1024)
        del c["name"]
        if op == "reorder" and c["outer"] * c["batch"] * c["beams"] * c["room"] > 2.5e9:
            continue                     # what the card holds several times over
        if _cost(c) <= top:
            return c


def _grid(t, step, scale):
    """Values of an 8-bit quantised tensor: at most 127 steps to either side."""
    return (t * (scale / step)).round_().clamp_(-127, 127).mul_(step)


def _operands(case, rows, g, exact_products):
    d, V, dt = case["d"], case["V"], DTYPES[case["dtype"]]
    H = torch.randn(rows, d, device="cuda", generator=g)
    H = (_grid(H, 2.0 ** -4, 1.0) if exact_products else H).to(dt)
    W = torch.empty(V, d, dtype=dt, device="cuda")
    for v in range(0, V, 32768):
        n = min(32768, V - v)
        w = torch.randn(n, d, device="cuda", generator=g)
        W[v:v + n] = _grid(w, 2.0 ** -10, 0.02) if exact_products else w * 0.02
    return H, W


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    st = dict(case=case)
    dev = dict(device="cuda")
    if case["op"] == "topk":
        st["H"], st["W"] = _operands(case, case["N"], g, True)
    elif case["op"] == "distill":
        N, V, K = case["N"], case["V"], case["K"]
        H, W = _operands(case, N, g, False)
        # distinct ids in no order, logits that fall off from the first to the last as a teacher's do
        first = torch.randint(0, V, (N, 1), generator=g, **dev)
        step = torch.randint(1, max(2, V // K), (N, 1), generator=g, **dev)
        k = torch.arange(K, **dev)
        ids = (first + k * step) % V
        t = 14.0 - 2.2 * torch.log1p(k.float()) + 0.7 * torch.randn(N, K, generator=g, **dev)
        if case["ragged"]:
            n = torch.randint(1, K + 1, (N, 1), generator=g, **dev)
            ids = torch.where(k < n, ids, torch.full_like(ids, -1))
        ids[torch.randperm(N, generator=g, **dev)[:min(N - 1, round(case["empty"] * N))]] = -1
        st.update(H=H, W=W, ids=ids, t=t, wr=torch.rand(N, generator=g, **dev) * (2.0 / N))
        if own:
            H.requires_grad_()
            W.requires_grad_()
    elif case["op"] == "beam":
        rows = case["batch"] * case["beams"]
        st["H"], st["W"] = _operands(case, rows, g, True)
        s = -20.0 + 3.0 * torch.randn(case["batch"], case["beams"], generator=g, **dev)
        st["scores"] = s.sort(1, descending=True).values
        st["finished"] = torch.rand(case["batch"], case["beams"], generator=g, **dev) < case["done"]
        st["eos"], st["pad"] = 2, 0
        if own:
            from paper_2511_17599_amd import binding as B
            n = (case["batch"], case["n_out"])
            st["out"] = (torch.empty(n, dtype=torch.float32, **dev), torch.empty(n, dtype=torch.int64, **dev),
                         torch.empty(n, dtype=torch.int64, **dev), torch.empty(n, dtype=torch.bool, **dev))
            st["dt"] = {"bf16": B.FLCE_DTYPE_BF16, "f32": B.FLCE_DTYPE_F32}[case["dtype"]]
            nb = B.flce_beam_workspace_bytes(case["batch"], case["beams"], case["d"], case["V"], case["n_out"], st["dt"])
            st["ws"] = torch.empty(nb, dtype=torch.uint8, **dev)
    else:
        shape = (case["outer"], case["batch"], case["beams"])
        st["src"] = torch.zeros(shape + (case["room"],), dtype=torch.bfloat16, **dev)
        for o in range(case["outer"]):
            st["src"][o, ..., :case["used"]] = torch.randn(shape[1:] + (case["used"],), generator=g, **dev)
        st["dst"] = torch.zeros_like(st["src"])
        st["parents"] = torch.randint(0, case["beams"], shape[1:], generator=g, **dev)
    return st


def _largest(z, K):
    """The K largest of each row, ties to the lowest index: 64-bit keys of the value's order and the index."""
    bits = z.contiguous().view(torch.int32).long()
    order = torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits)          # -0 and +0 are equal
    V = z.shape[1]
    keys = torch.topk((order << 32) + (V - 1 - torch.arange(V, device=z.device)), K, dim=1).values
    ids = V - 1 - (keys & 0xFFFFFFFF)
    return z.gather(1, ids), ids


def _plain_topk(st):
    H, W, K = st["H"], st["W"].float().t(), st["case"]["K"]
    step = max(1, (1 << 27) // W.shape[1])
    parts = []
    for i in range(0, H.shape[0], step):
        z = H[i:i + step].float() @ W
        m = z.max(1, keepdim=True).values
        lse = (m[:, 0].double() + (z - m).double().exp().sum(1).log()).float()
        parts.append(_largest(z, K) + (lse,))
    return tuple(torch.cat(p) for p in zip(*parts))


def _plain_distill(st):
    case = st["case"]
    H, W, ids, t, T = st["H"], st["W"], st["ids"], st["t"], case["T"]
    here = ids >= 0
    counts = here.any(1)
    n = counts.sum()
    p = torch.where(here, t / T, torch.full_like(t, -math.inf))
    p = torch.exp(p - torch.where(counts, p.max(1).values, torch.zeros_like(t[:, 0]))[:, None])
    p = p / p.sum(1, keepdim=True).clamp_min(1e-30)
    gam = torch.where(counts, st["wr"] if case["reduction"] == "none" else
                      (1.0 / n if case["reduction"] == "mean" else torch.ones_like(n)).float(), torch.zeros_like(st["wr"]))
    Wf = W.float()
    dH, dW = torch.empty(H.shape, device=H.device), torch.zeros(W.shape, device=H.device)
    rows = torch.empty(H.shape[0], device=H.device)
    at = ids.clamp_min(0)
    step = max(1, (1 << 28) // W.shape[0])
    for i in range(0, H.shape[0], step):
        s = slice(i, i + step)
        h = H[s].float()
        z = (h @ Wf.t()).div_(T)
        m = z.max(1, keepdim=True).values
        lse = m[:, 0] + (z - m).exp_().sum(1, dtype=torch.float64).log().float()
        term = p[s] * (torch.log(p[s].clamp_min(1e-38)) - z.gather(1, at[s]) + lse[:, None])
        rows[s] = T * T * term.sum(1)
        q = z.sub_(lse[:, None]).exp_()
        q.scatter_add_(1, at[s], -p[s])
        q *= (T * gam[s])[:, None]
        dH[s] = q @ Wf
        dW += q.t() @ h
    rows = torch.where(counts, rows, torch.zeros_like(rows))
    out = rows if case["reduction"] == "none" else rows.sum() / n if case["reduction"] == "mean" else rows.sum()
    return out, dH.to(H.dtype), dW.to(W.dtype)


def _plain_beam(st):
    case = st["case"]
    batch, beams, V, n_out = case["batch"], case["beams"], case["V"], case["n_out"]
    z = (st["H"].float() @ st["W"].float().t()).double()
    k = min(n_out, V)
    zk, tok = _largest(z.float(), k)
    # sums of log-probabilities decide between beams: 64 bits, rounded at the end
    m = z.max(1, keepdim=True).values
    lse = m[:, 0] + (z - m).exp().sum(1).log()
    s = (st["scores"].double().reshape(-1, 1) + zk.double() - lse[:, None]).reshape(batch, beams, k)
    done = st["finished"]
    once = torch.full((batch, beams, k), -math.inf, dtype=torch.float64, device=s.device)
    once[..., 0] = st["scores"].double()
    s = torch.where(done[..., None], once, s).reshape(batch, -1)
    tok = torch.where(done[..., None], torch.full_like(tok.reshape(batch, beams, k), st["pad"]),
                      tok.reshape(batch, beams, k)).reshape(batch, -1)
    best = torch.sort(s, dim=1, descending=True, stable=True)
    at = best.indices[:, :n_out]
    token, parent = tok.gather(1, at), at // k
    return best.values[:, :n_out].float(), token, parent, done.gather(1, parent) | (token == st["eos"])


def _plain_reorder(st):
    n, rows = st["case"]["used"], torch.arange(st["case"]["batch"], device="cuda")[:, None]
    st["dst"][..., :n] = st["src"][:, rows, st["parents"], :n]
    return st["dst"]


def run(st):
    case = st["case"]
    if not own:
        with torch.no_grad():
            return {"topk": _plain_topk, "distill": _plain_distill, "beam": _plain_beam, "reorder": _plain_reorder}[case["op"]](st)
    from paper_2511_17599_amd import binding as B
    from paper_2511_17599_amd import torch_api as A
    if case["op"] == "topk":
        return A.linear_topk(st["H"], st["W"], case["K"])
    if case["op"] == "distill":
        loss = A.linear_distillation(st["H"], st["W"], st["ids"], st["t"], temperature=case["T"], reduction=case["reduction"])
        up = st["wr"] if case["reduction"] == "none" else None
        return (loss.detach(),) + torch.autograd.grad(loss, (st["H"], st["W"]), up)
    if case["op"] == "beam":
        rc = B.flce_beam_step(st["H"], st["W"], st["scores"], st["finished"], case["batch"], case["beams"], case["d"], case["V"],
                              case["n_out"], st["eos"], st["pad"], st["dt"], *st["out"], st["ws"], st["ws"].numel(),
                              torch.cuda.current_stream())
        if rc != B.FLCE_OK:
            raise RuntimeError(B.flce_status_string(rc))
        return st["out"]
    n = case["used"]
    A.reorder_states(st["parents"], st["src"][..., :n], out=st["dst"][..., :n])
    return st["dst"]


def work(case):
    """Inputs read once, outputs written once; logits once, and once more for the gradients with their two products."""
    if case["op"] == "reorder":
        return {"bytes": _cost(case), "flops": 0.0}
    d, V, e = case["d"], case["V"], 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "beam":
        N, few = case["batch"] * case["beams"], case["batch"] * case["n_out"] * 21
    else:
        N, few = case["N"], case["N"] * (12 * case["K"] + 4)
    if case["op"] == "distill":
        counted = N - min(N - 1, round(case["empty"] * N))
        return {"bytes": 3.0 * (N + V) * d * e + 2.0 * few, "flops": (2.0 * N + 6.0 * counted) * d * V}
    return {"bytes": (N + V) * d * e + few, "flops": 2.0 * N * d * V}


def exact(case, seed):
    """The definitions in 64 bits on the same inputs."""
    st = prepare(case, seed)
    if case["op"] == "reorder":
        at = (st["parents"] + case["beams"] * torch.arange(case["batch"], device="cuda")[:, None]).flatten()
        return torch.index_select(st["src"].flatten(1, 2), 1, at).view_as(st["src"])
    H, W = st["H"].detach(), st["W"].detach().double()
    N, V = H.shape[0], W.shape[0]
    step = max(1, (1 << 27) // V)
    f64 = dict(dtype=torch.float64, device="cuda")
    if case["op"] == "topk":
        vals, lse = torch.empty(N, case["K"], **f64), torch.empty(N, **f64)
        for i in range(0, N, step):
            z = H[i:i + step].double() @ W.t()
            vals[i:i + step] = torch.topk(z, case["K"], dim=1).values
            lse[i:i + step] = torch.logsumexp(z, 1)
        return vals, None, lse
    if case["op"] == "beam":
        b, nb, n_out = case["batch"], case["beams"], case["n_out"]
        logp = torch.log_softmax(H.double() @ W.t(), 1).reshape(b, nb, V)
        total = (st["scores"].double()[..., None] + torch.topk(logp, min(n_out, V), dim=2).values)
        rest = torch.full_like(total, -math.inf)
        rest[..., 0] = st["scores"].double()
        total = torch.where(st["finished"][..., None], rest, total).flatten(1)
        return torch.topk(total, n_out, dim=1).values, None, None, None
    T, ids = case["T"], st["ids"]
    logp = torch.where(ids >= 0, st["t"].double() / T, torch.tensor(-math.inf, **f64))
    counts = (ids >= 0).any(1)
    logp = torch.where(counts[:, None], torch.log_softmax(logp, 1), torch.tensor(-math.inf, **f64))
    p = logp.exp()
    weight = counts.double()
    if case["reduction"] == "mean":
        weight = weight / counts.sum()
    elif case["reduction"] == "none":
        weight = weight * st["wr"].double()
    rows = torch.zeros(N, **f64)
    dH, dW = torch.zeros(N, case["d"], **f64), torch.zeros(V, case["d"], **f64)
    for i in range(0, N, step):
        s = slice(i, i + step)
        h = H[s].double()
        logq = torch.log_softmax(h @ W.t() / T, 1)
        at = ids[s].clamp_min(0)
        kl = p[s] * (torch.where(p[s] > 0, logp[s], torch.zeros_like(p[s])) - logq.gather(1, at))
        rows[s] = T * T * kl.sum(1)
        G = logq.exp_()
        G.scatter_add_(1, at, -p[s])
        G.mul_(T * weight[s][:, None])
        dH[s] = G @ W
        dW += G.t() @ h
    loss = rows if case["reduction"] == "none" else rows.sum() / (counts.sum() if case["reduction"] == "mean" else 1)
    return loss, dH, dW
