"""torch.autograd front end of libflce: hidden states and vocabulary weights in, loss out, gradients through
``backward()``.  Plumbing only: every step of the computation runs inside the library's kernels; torch holds the
tensors, names the stream and chains the autograd graph.

    loss = linear_cross_entropy(H, W, targets)                       # mean over counted rows
    rows = linear_cross_entropy(H, W, targets, reduction="none")     # one loss per row
    loss.backward()                                                   # H.grad, W.grad

H is [..., d] (leading dimensions are flattened to N rows), W is [V, d], both bf16 or both fp32, contiguous, on the
same GPU; targets are int64 with the leading shape of H.  The N x V logits are never formed.

On a few logits per row:

    logits, ids, lse = linear_topk(H, W, k)                           # the k largest of each row
    loss = linear_distillation(H, W, ids, logits, temperature=2.0)    # a student on a teacher's lists
    scores, tokens, parents, finished = beam_step(H, W, scores, finished, eos_id=2)
    reorder_states(parents, cache, out=cache)                         # the beams' states follow
"""
from __future__ import annotations

import functools
import weakref

import torch

from . import binding as B

_DT = {torch.bfloat16: B.FLCE_DTYPE_BF16, torch.float32: B.FLCE_DTYPE_F32}
_RED = {"mean": B.FLCE_REDUCE_MEAN, "sum": B.FLCE_REDUCE_SUM}


# the current stream's handle, without a Stream object around it where torch offers that
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(device):
    return _raw_stream(device.index) if _raw_stream else torch.cuda.current_stream(device).cuda_stream


def _check(rc):
    if rc != B.FLCE_OK:
        raise RuntimeError(f"libflce: {B.flce_status_string(rc)}")


def _prepare(H, W, targets):
    if H.dtype not in _DT or W.dtype != H.dtype:
        raise TypeError("H and W must both be bfloat16 or both float32")
    if not (H.is_cuda and W.is_cuda and targets.is_cuda):
        raise ValueError("libflce works on GPU tensors only")
    # A small call is bound by this host work: what is as the library wants it goes through untouched (64 x 64 x 600, forward
    # and backward 131 -> 121 us with the same elsewhere in this file).
    H2 = H if H.dim() == 2 and H.is_contiguous() else H.reshape(-1, H.shape[-1]).contiguous()
    W2 = W.contiguous()
    if targets.dim() == 1 and targets.dtype is torch.int64 and targets.is_contiguous():
        y = targets
    else:
        y = targets.reshape(-1).to(torch.int64).contiguous()
    if y.numel() != H2.shape[0] or W2.shape[1] != H2.shape[1]:
        raise ValueError("shapes: H [..., d], W [V, d], targets [...]")
    return H2, W2, y


def _workspace(N, d, V, dt, backward, device):
    nb = B.flce_workspace_bytes(N, d, V, dt, backward)
    if nb == 0:
        raise ValueError("unsupported shape (d must be a multiple of 8)")
    return torch.empty(nb, dtype=torch.uint8, device=device), nb


# The autograd nodes of the living losses that were made outside of a HIP graph's capture.  While such a graph lives, torch's gradient
# accumulators of its leaves belong to the stream it was made on, and a backward captured for the same leaves waits for that stream; where
# that is the default stream, which no capture can take in, it ends the process.  One weak reference per loss: 0.7 us of a call's 20.
_eager_nodes = set()


def _capturing(t):
    return t.is_cuda and torch.cuda.is_current_stream_capturing()


def _remember(ctx, loss, stream):
    if _capturing(loss):
        ctx.stream = None
    else:
        ctx.stream = stream
        _eager_nodes.add(weakref.ref(ctx, _eager_nodes.discard))


def _accumulators(nodes):
    """The gradient accumulators that the autograd graphs behind `nodes` end in."""
    seen, todo = set(), list(nodes)
    while todo:
        node = todo.pop()
        if node not in seen:
            seen.add(node)
            todo += [n for n, _ in node.next_functions if n is not None]
    return {node for node in seen if not node.next_functions}


def _living(nodes):
    """Eager losses that have a gradient accumulator in common with the graphs behind `nodes`."""
    mine = _accumulators(nodes)
    return [node for node in (ref() for ref in _eager_nodes.copy()) if node is not None and not mine.isdisjoint(_accumulators([node]))]


def _refuse_captured_backward(ctx, grad):
    """The captured backward of a captured forward is refused beside an eager loss of the same leaves from the default stream."""
    if _capturing(grad) and any(node.stream == 0 for node in _living([ctx])):
        raise RuntimeError("an eager loss of the same leaves, made on the default stream, is alive: drop it before capturing a backward")


class _ScalarLoss(torch.autograd.Function):
    """Alg. 1 forward, Alg. 2 backward; mean or sum over the counted rows."""

    @staticmethod
    def forward(ctx, H, W, targets, ignore_index, reduction):
        H2, W2, y = _prepare(H, W, targets)
        N, d = H2.shape
        V = W2.shape[0]
        dt = _DT[H2.dtype]
        st = _stream(H2.device)
        loss = torch.empty((), dtype=torch.float32, device=H2.device)
        lse = torch.empty(N, dtype=torch.float32, device=H2.device)
        ws, nb = _workspace(N, d, V, dt, 0, H2.device)
        _check(B.flce_forward(H2, W2, y, N, d, V, ignore_index, _RED[reduction], dt, loss, lse, ws, nb, st))
        ctx.save_for_backward(H2, W2, y, lse)
        ctx.meta = (H.shape, ignore_index, reduction)
        _remember(ctx, loss, st)
        return loss

    @staticmethod
    def backward(ctx, grad_out):
        if ctx.stream is None:
            _refuse_captured_backward(ctx, grad_out)
        H2, W2, y, lse = ctx.saved_tensors
        shape, ignore_index, reduction = ctx.meta
        N, d = H2.shape
        V = W2.shape[0]
        dt = _DT[H2.dtype]
        st = _stream(H2.device)
        dH = torch.empty_like(H2)
        dW = torch.empty_like(W2)
        ws, nb = _workspace(N, d, V, dt, 1, H2.device)
        # The kernels read the upstream gradient where it is: no wait for the stream between forward and backward.  (The
        # autograd engine runs this on the forward's stream and keeps gradients made on another one alive for it.)
        g = grad_out
        if g.dtype is not torch.float32 or g.device != H2.device:
            g = g.to(device=H2.device, dtype=torch.float32)
        if g.is_neg() or g._is_zerotensor():     # marked, not stored: the word in memory is not the value, or there is none
            g = g.clone().resolve_neg()
        _check(B.flce_backward_device_grad(H2, W2, y, lse, N, d, V, ignore_index, _RED[reduction], dt, g, dH, dW, ws, nb,
                                           st))
        return dH if dH.shape == shape else dH.reshape(shape), dW, None, None, None


class _RowLosses(torch.autograd.Function):
    """One loss per row (optionally label-smoothed); the backward takes one upstream gradient per row."""

    @staticmethod
    def forward(ctx, H, W, targets, ignore_index, label_smoothing):
        H2, W2, y = _prepare(H, W, targets)
        N, d = H2.shape
        V = W2.shape[0]
        dt = _DT[H2.dtype]
        st = _stream(H2.device)
        rows = torch.empty(N, dtype=torch.float32, device=H2.device)
        lse = torch.empty(N, dtype=torch.float32, device=H2.device)
        ws, nb = _workspace(N, d, V, dt, 0, H2.device)
        _check(B.flce_forward_rows(H2, W2, y, N, d, V, ignore_index, label_smoothing, dt, rows, lse, ws, nb, st))
        ctx.save_for_backward(H2, W2, y, lse)
        ctx.meta = (H.shape, ignore_index, label_smoothing)
        _remember(ctx, rows, st)
        return rows if targets.dim() == 1 else rows.reshape(targets.shape)

    @staticmethod
    def backward(ctx, grad_rows):
        if ctx.stream is None:
            _refuse_captured_backward(ctx, grad_rows)
        H2, W2, y, lse = ctx.saved_tensors
        shape, ignore_index, label_smoothing = ctx.meta
        N, d = H2.shape
        V = W2.shape[0]
        dt = _DT[H2.dtype]
        st = _stream(H2.device)
        dH = torch.empty_like(H2)
        dW = torch.empty_like(W2)
        gr = grad_rows.reshape(-1).to(torch.float32).contiguous()
        ws, nb = _workspace(N, d, V, dt, 1, H2.device)
        _check(B.flce_backward_rows(H2, W2, y, lse, gr, N, d, V, ignore_index, label_smoothing, dt, dH, dW, ws, nb,
                                    st))
        return dH if dH.shape == shape else dH.reshape(shape), dW, None, None, None


def linear_cross_entropy(H, W, targets, ignore_index=-100, reduction="mean", label_smoothing=0.0):
    """Cross-entropy of softmax(H . W^T) against `targets` without the logits tensor.

    reduction: "mean" (over rows whose target is not `ignore_index`), "sum" or "none".  Label smoothing comes
    with one loss per row only (reduction="none", the library's per-row call): reduce the rows with torch as
    needed, autograd hands the per-row upstream gradients back to the library.

    Forward and backward can be captured into a HIP graph.  The backward is refused there while an eager loss of this module that was
    made on the default stream and has a leaf in common (H, W or the parameters they come from) is alive.
    """
    if reduction not in ("mean", "sum", "none"):
        raise ValueError("reduction must be 'mean', 'sum' or 'none'")
    if reduction != "none":
        if label_smoothing != 0.0:
            raise ValueError("label smoothing is available with reduction='none' only")
        return _ScalarLoss.apply(H, W, targets, int(ignore_index), reduction)
    return _RowLosses.apply(H, W, targets, int(ignore_index), float(label_smoothing))


def _launch(call, device, *args):
    """The library launches on the current device: the tensors' own, whichever is current for the caller."""
    if torch.cuda.current_device() == device.index:
        rc = call(*args, _stream(device))
    else:
        with torch.cuda.device(device):
            rc = call(*args, _stream(device))
    _check(rc)


def _operands(H, W):
    if H.dtype not in _DT or W.dtype != H.dtype:
        raise TypeError("H and W must both be bfloat16 or both float32")
    if not (H.is_cuda and W.is_cuda):
        raise ValueError("libflce works on GPU tensors only")
    if H.device != W.device:
        raise ValueError("H and W are on different devices")
    if H.dim() < 1 or W.dim() != 2 or W.shape[1] != H.shape[-1]:
        raise ValueError("shapes: H [..., d], W [V, d]")
    return H if H.dim() == 2 and H.is_contiguous() else H.reshape(-1, H.shape[-1]).contiguous(), W.contiguous()


def _beside(device, t, dtype, name):
    """A further argument as the library wants it: on H's device, contiguous, of one type."""
    if t.device != device:
        raise ValueError(f"{name} is on another device than H")
    return t if t.dtype is dtype and t.is_contiguous() else t.to(dtype).contiguous()


def _scratch(nbytes, device, what):
    if nbytes == 0:
        raise ValueError(f"unsupported shape ({what})")
    return torch.empty(nbytes, dtype=torch.uint8, device=device), nbytes


def linear_topk(H, W, k):
    """The k largest logits of each row of H . W^T, in descending order (equal ones by id), without the logits tensor.

    Returns (logits [..., k] float32, ids [..., k] int64, lse [...] float32); lse is the log-sum-exp over the whole
    vocabulary, so logits - lse[..., None] are log-probabilities.  1 <= k <= 256.  Not differentiable.
    """
    with torch.no_grad():
        H2, W2 = _operands(H.detach(), W.detach())
        (N, d), V, dt, dev = H2.shape, W2.shape[0], _DT[H2.dtype], H2.device
        k = int(k)
        ws, nb = _scratch(B.flce_topk_workspace_bytes(N, d, V, k, dt), dev,
                          "d must be a multiple of 8, 1 <= k <= min(256, V), V <= 2^22, at least one row")
        logits = torch.empty(N, k, dtype=torch.float32, device=dev)
        ids = torch.empty(N, k, dtype=torch.int64, device=dev)
        lse = torch.empty(N, dtype=torch.float32, device=dev)
        _launch(B.flce_topk, dev, H2, W2, N, d, V, k, dt, logits, ids, lse, ws, nb)
    if H.dim() == 2:
        return logits, ids, lse
    lead = H.shape[:-1]
    return logits.reshape(*lead, k), ids.reshape(*lead, k), lse.reshape(lead)


def _refuse_capture(H, W):
    """A distillation is refused under capture beside any living eager loss of the same leaves (H, W or what they were computed from)."""
    if torch.is_grad_enabled() and _capturing(H):
        if _living([torch.autograd.graph.get_gradient_edge(t).node for t in (H, W) if t.requires_grad]):
            raise RuntimeError("an eager loss of the same leaves is alive: drop it before capturing a distillation")


class _Once(torch.autograd.Function):
    """Gradients that the library has filled have no graph of their own: where torch is to keep one (create_graph), it ends here."""

    @staticmethod
    def forward(ctx, dH, dW, H, W, grad):
        return dH, dW

    @staticmethod
    def backward(ctx, *grads):
        raise RuntimeError("the gradients of linear_distillation cannot be differentiated")


class _Distillation(torch.autograd.Function):
    """Loss over a teacher's lists; mean or sum over the rows that count, or one loss per row."""

    @staticmethod
    def forward(ctx, H, W, ids, logits, temperature, reduction):
        H2, W2 = _operands(H, W)
        (N, d), V, dt, dev = H2.shape, W2.shape[0], _DT[H2.dtype], H2.device
        K = ids.shape[-1]
        ids2 = _beside(dev, ids, torch.int64, "teacher_ids")
        t2 = _beside(dev, logits, torch.float32, "teacher_logits")
        ws, nb = _scratch(B.flce_distill_workspace_bytes(N, d, V, K, dt, 0), dev,
                          "d must be a multiple of 8, 1 <= K <= 256, at least one row")
        rows = reduction == "none"
        out = torch.empty(H.shape[:-1] if rows else (), dtype=torch.float32, device=dev)
        ns = B.flce_distill_saved_bytes(N, K)
        keep = torch.empty(ns + 4 * N, dtype=torch.uint8, device=dev)        # what the backward takes, lse behind it
        saved = keep.data_ptr()
        _launch(B.flce_distill_forward, dev, H2, W2, ids2, t2, N, d, V, K, temperature, _RED.get(reduction, B.FLCE_REDUCE_SUM), dt,
                None if rows else out, out if rows else None, saved + ns, saved, ws, nb)
        ctx.save_for_backward(H, W, ids2, keep)
        ctx.meta = (temperature, reduction, K, ns)
        _remember(ctx, out, _stream(dev))
        return out

    @staticmethod
    def backward(ctx, grad):
        if ctx.stream is None:
            _refuse_captured_backward(ctx, grad)
        H, W, ids2, keep = ctx.saved_tensors
        temperature, reduction, K, ns = ctx.meta
        N, (V, d), dt, dev = ids2.numel() // K, W.shape, _DT[H.dtype], H.device
        # The kernels read the gradient where it is; one that is only marked as negated or zero is made first.
        g = grad
        if g.dtype is not torch.float32 or g.device != dev:
            g = g.to(device=dev, dtype=torch.float32)
        if g.is_neg() or g._is_zerotensor():
            g = g.clone().resolve_neg()
        rows = reduction == "none"
        if rows:
            g = g.contiguous()
        dH = torch.empty_like(H)
        dW = torch.empty_like(W)
        ws, nb = _scratch(B.flce_distill_workspace_bytes(N, d, V, K, dt, 1), dev, "as in the forward")
        saved = keep.data_ptr()
        _launch(B.flce_distill_backward, dev, H, W, ids2, saved + ns, saved, N, d, V, K, temperature,
                _RED.get(reduction, B.FLCE_REDUCE_SUM), dt, None if rows else g, g if rows else None, dH, dW, ws, nb)
        if torch.is_grad_enabled():
            dH, dW = _Once.apply(dH, dW, H, W, grad)
        return dH, dW, None, None, None, None


def linear_distillation(H, W, teacher_ids, teacher_logits, temperature=1.0, reduction="mean"):
    """Distillation of softmax(H . W^T) from a teacher's largest logits, without the logits tensor.

    teacher_ids [..., K] (int64, negative: no entry) and teacher_logits [..., K] (float, no gradient) with the leading shape
    of H, K <= 256, as linear_topk gives them.  Per row T^2 KL(p || q) with p = softmax over the list's logits / T and q = softmax over
    the vocabulary's logits / T, T = temperature.  reduction: "mean" (over the rows that have an entry), "sum" or "none".
    Rows without an entry, and rows with an id beyond the vocabulary, have loss and gradient 0.  The gradients cannot be differentiated
    again: that raises.

    Forward and backward can be captured into a HIP graph while no autograd graph made outside of it has a leaf in common with them (H, W or
    the parameters they come from).  Beside a living eager loss of this module the call is refused, under torch.no_grad() it is not.
    """
    if reduction not in ("mean", "sum", "none"):
        raise ValueError("reduction must be 'mean', 'sum' or 'none'")
    if teacher_ids.dtype.is_floating_point or not teacher_logits.dtype.is_floating_point:
        raise TypeError("teacher_ids are integers, teacher_logits are floating point")
    if teacher_ids.shape != teacher_logits.shape or teacher_ids.dim() != H.dim() or teacher_ids.shape[:-1] != H.shape[:-1]:
        raise ValueError("shapes: H [..., d], teacher_ids and teacher_logits [..., K]")
    _refuse_capture(H, W)
    # (copies are made here, in the autograd graph, so that H and W are what the backward keeps)
    return _Distillation.apply(H.contiguous(), W.contiguous(), teacher_ids, teacher_logits, float(temperature), reduction)


def beam_step(H, W, scores, finished=None, n_out=None, eos_id=-1, pad_id=0):
    """One step of a beam search on softmax(H . W^T), without the logits tensor.

    H [batch, beams, d], scores [batch, beams] (sums of log-probabilities), finished [batch, beams] (bool) or None.  Returns the
    n_out (default: beams) best continuations of each search in order: scores [batch, n_out] float32, tokens and parents
    (the beam each comes from) int64, finished bool.  A finished beam stays a candidate with its score and `pad_id`.
    """
    if H.dim() != 3 or scores.shape != H.shape[:2] or (finished is not None and finished.shape != H.shape[:2]):
        raise ValueError("shapes: H [batch, beams, d], scores and finished [batch, beams]")
    with torch.no_grad():
        H2, W2 = _operands(H.detach(), W.detach())
        (batch, beams, d), V, dt, dev = H.shape, W2.shape[0], _DT[H2.dtype], H2.device
        n_out = beams if n_out is None else int(n_out)
        s = _beside(dev, scores, torch.float32, "scores")
        f = None if finished is None else _beside(dev, finished, torch.bool, "finished")
        ws, nb = _scratch(B.flce_beam_workspace_bytes(batch, beams, d, V, n_out, dt), dev,
                          "d must be a multiple of 8, beams and n_out 1 .. 64, V <= 2^22, at least one search")
        out = (torch.empty(batch, n_out, dtype=torch.float32, device=dev), torch.empty(batch, n_out, dtype=torch.int64, device=dev),
               torch.empty(batch, n_out, dtype=torch.int64, device=dev), torch.empty(batch, n_out, dtype=torch.bool, device=dev))
        _launch(B.flce_beam_step, dev, H2, W2, s, f, batch, beams, d, V, n_out, int(eos_id), int(pad_id), dt, *out, ws, nb)
    return out


@functools.lru_cache(1024)
def _rows_of(shape, stride, dim, size):
    """(bytes of a beam's row, number of outer slabs, bytes from row to row, bytes from slab to slab) of a states tensor."""
    run = 1
    for n, s in zip(shape[:dim + 1:-1], stride[:dim + 1:-1]):
        if n > 1 and s != run:
            raise ValueError("a beam's state must be contiguous")
        run *= n
    batch, beams = shape[dim], shape[dim + 1]
    row = stride[dim + 1] if beams > 1 else stride[dim] if batch > 1 else run
    if batch > 1 and stride[dim] != beams * row:
        raise ValueError("batch and beams must be one run of rows")
    outer, step = 1, None
    for n, s in zip(shape[:dim][::-1], stride[:dim][::-1]):
        if n > 1:
            if step is not None and s != step * outer:
                raise ValueError("the dimensions ahead of the batch must be strided once")
            step = s if step is None else step
            outer *= n
    return run * size, outer, row * size, (step or 0) * size


def reorder_states(parents, states, out=None, dim=1, status=None):
    """The beams' states after a step: out[..., b, j, ...] = states[..., b, parents[b, j], ...].

    parents [batch, beams_out] (int64); dimension `dim` of `states` is the batch, the next one the beams; what lies ahead of it
    (layers, keys and values) may be strided once, a beam's row is contiguous.  out: a tensor of states' shape with beams_out
    beams (a new one by default); out=states reorders in place (up to 16 beams).  status: an int32 tensor that becomes
    FLCE_ERR_TARGET_RANGE where a parent is no beam (whose row is left as it was).  Returns out.  Not differentiable.
    """
    if not states.is_cuda or parents.device != states.device or (out is not None and out.device != states.device):
        raise ValueError("parents, states and out must be on one GPU")
    if parents.dim() != 2 or states.dim() < dim + 2 or dim < 0 or states.shape[dim] != parents.shape[0]:
        raise ValueError("shapes: parents [batch, beams_out], states [..., batch, beams, ...] with the batch at `dim`")
    if status is not None and (status.dtype is not torch.int32 or status.device != states.device or status.numel() != 1):
        raise TypeError("status is one int32 on the states' GPU")
    batch, beams_out = parents.shape
    beams_in = states.shape[dim + 1]
    want = states.shape[:dim + 1] + (beams_out,) + states.shape[dim + 2:]
    if out is None:
        out = torch.empty(want, dtype=states.dtype, device=states.device)
    if out.shape != want or out.dtype != states.dtype:
        raise ValueError("out does not have the shape and type of the reordered states")
    if out.numel() == 0:
        return out

    row_bytes, outer, src_row, src_outer = _rows_of(states.shape, states.stride(), dim, states.element_size())
    _, _, dst_row, dst_outer = _rows_of(want, out.stride(), dim, out.element_size())
    _launch(B.flce_beam_reorder, states.device, states, out, _beside(states.device, parents, torch.int64, "parents"), outer, batch, beams_in,
            beams_out, row_bytes, src_row, src_outer, dst_row, dst_outer, status)
    return out
