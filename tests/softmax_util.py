"""Inputs, 64-bit references and error bounds of the operators on whole tables, shared by their GPU tests."""
import math

import torch

import paper_2101_08358_amd as mar

DEV = "cuda:0"
TYPES = {"fp32": (torch.float32, mar.DTYPE_FP32), "bf16": (torch.bfloat16, mar.DTYPE_BF16), "fp16": (torch.float16, mar.DTYPE_FP16)}
# relative error of a softmax weight when it enters a product: half a step of the 16-bit types, 2^-22 as a pair of f16
WEIGHT_EPS = {"fp32": 2.0 ** -22, "bf16": 2.0 ** -8, "fp16": 2.0 ** -11}


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def rows(g, n, dim, dtype, std=0.3, stride=None, offset=0):
    """n rows of dim values whose stride and start are as asked for; what lies between the rows is NaN."""
    stride = stride or dim
    buf = torch.full((offset + max(n, 1) * stride,), float("nan"), dtype=dtype, device=DEV)
    view = buf[offset:].view(max(n, 1), stride)[:n, :dim]
    view.copy_((torch.randn((n, dim), generator=g, device=DEV) * std).to(dtype))
    return view


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def problem(q, w, tname, scale=1.0):
    return mar.MarSoftmax(w.shape[0], w.stride(0) if w.shape[0] > 1 else max(w.stride(0), w.shape[1]),
                          q.stride(0) if q.shape[0] > 1 else max(q.stride(0), q.shape[1]), q.shape[0], w.shape[1], TYPES[tname][1], scale)


def workspace(nbytes):
    return torch.full((nbytes,), 0xA5, dtype=torch.uint8, device=DEV)


def score_error(q, w, scale):
    """Bound of a score's error: d sums in fp32 of exact products (or of pairs whose product is good to 2^-22), the factor
    to log2 units and back."""
    d = w.shape[1]
    size = scale * float(q.double().norm(dim=1).max() if q.shape[0] else 0.0) * float(w.double().norm(dim=1).max())
    return size * (d + 16) * 2.0 ** -24


def sum_error(V):
    """Relative error of a sum of V weights: a lane's chain of V / 32 sums of four, the weights' own exponentials."""
    return (V / 32 + 256) * 2.0 ** -24


def scores(q, w, scale, allowed=None):
    s = torch.matmul(q.double(), w.double().t().contiguous()) * scale
    return s if allowed is None else s.masked_fill(~allowed, -math.inf)


def pack(allowed):
    """[T, V] truth values -> [T, words] int32."""
    T, V = allowed.shape
    words = (V + 31) // 32
    bits = torch.zeros((T, words * 32), dtype=torch.int64, device=DEV)
    bits[:, :V] = allowed.long()
    v = (bits.view(T, words, 32) << torch.arange(32, device=DEV)).sum(2)
    return torch.where(v >= 1 << 31, v - (1 << 32), v).to(torch.int32).contiguous()


def run_log_probs(q, w, tname, targets=None, words=None, words_stride=0, top=0, scale=1.0, stream=None, ws=None):
    T = q.shape[0]
    p = problem(q, w, tname, scale)
    ws = workspace(mar.mar_log_probs_workspace_bytes(p, top)) if ws is None else ws
    lp = torch.full((T,), 7.0, device=DEV) if targets is not None else None
    en = torch.full((T,), 7.0, device=DEV)
    ids = torch.full((T, top), -7, dtype=torch.int32, device=DEV)
    tp = torch.full((T, top), 7.0, device=DEV)
    mar.mar_log_probs(p, q, w, targets, words, words_stride, top, lp, en, ids, tp, ws, ws.numel(), stream)
    return lp, en, ids, tp


def run_loss(q, w, tname, targets, weights=None, scale=1.0, want=("loss", "lse", "gq", "gw"), gq=None, gw=None, ws=None, stream=None):
    T, V = q.shape[0], w.shape[0]
    p = problem(q, w, tname, scale)
    ws = workspace(mar.mar_softmax_loss_workspace_bytes(p)) if ws is None else ws
    loss = torch.full((T,), 7.0, device=DEV) if "loss" in want else None
    lse = torch.full((T,), 7.0, device=DEV) if "lse" in want else None
    if gq is None and "gq" in want:
        gq = torch.full(tuple(q.shape), 7.0, dtype=q.dtype, device=DEV)
    if gw is None and "gw" in want:
        gw = torch.full(tuple(w.shape), 7.0, dtype=w.dtype, device=DEV)
    d = w.shape[1]
    mar.mar_softmax_loss(p, q, w, targets, weights, loss, lse, gq, gq.stride(0) if gq is not None and T > 1 else d, gw,
                         gw.stride(0) if gw is not None and V > 1 else d, ws, ws.numel(), stream)
    return loss, lse, gq, gw


def loss_reference(q, w, targets, weights, scale):
    """loss, lse, the weights' matrix u (p - [target]), and |u| (p + [target]) for the bounds, in 64 bits."""
    T, V = q.shape[0], w.shape[0]
    s = scores(q, w, scale)
    lse = torch.logsumexp(s, 1)
    has = (targets >= 0) & (targets < V)
    u = torch.ones(T, dtype=torch.float64, device=DEV) if weights is None else weights.double()
    u = torch.where(has, u, torch.zeros_like(u))
    t = targets.long().clamp(0, V - 1)
    at = torch.arange(T, device=DEV)
    loss = torch.where(has, u * (lse - s[at, t]), torch.zeros_like(lse))
    p = torch.exp(s - lse[:, None])
    one = torch.zeros_like(p)
    one[at, t] = 1.0
    D = torch.where(has[:, None], (p - one) * u[:, None], torch.zeros_like(p))
    A = torch.where(has[:, None], (p + one) * u.abs()[:, None], torch.zeros_like(p))
    return loss, lse, D, A


def check_loss(out, q, w, tname, targets, weights, scale):
    loss, lse, gq, gw = out
    T, V = q.shape[0], w.shape[0]
    q = torch.nan_to_num(q) if T else q
    rl, rlse, D, A = loss_reference(q, w, targets, weights, scale)
    delta, total = score_error(q, w, scale), sum_error(V)
    u = (torch.ones(T, device=DEV) if weights is None else weights).double().abs()
    if lse is not None:
        err = (lse.double() - rlse).abs()
        assert (err <= delta + total + rlse.abs() * 2.0 ** -23).all(), float(err.max())
    if loss is not None:
        err = (loss.double() - rl).abs()
        assert (err <= u * (2 * delta + total) + rl.abs() * 2.0 ** -23).all(), float(err.max())
    dtype = TYPES[tname][0]
    per = 2 * (delta + total) + WEIGHT_EPS[tname]
    smallest = torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps     # a subnormal result's half step and more
    if gq is not None:
        ref, size = scale * D @ w.double(), scale * A @ w.double().abs()
        floor = scale * V * 2.0 ** -36 * u[:, None] * float(w.double().abs().max())
        err = (gq.double() - ref).abs()
        bound = size * (per + (V / 8 + 64) * 2.0 ** -24) + floor + ref.abs() * half_step(dtype) + smallest
        assert (err <= bound).all(), (float((err / bound).max()), float(err.max()))
    if gw is not None:
        Dt, At = D.t().contiguous(), A.t().contiguous()
        ref, size = scale * Dt @ q.double(), scale * At @ q.double().abs()
        floor = scale * max(T, 1) * 2.0 ** -36 * (At.amax(1, keepdim=True) if T else 0.0) * (float(q.double().abs().max()) if T else 0.0)
        # a weight below the smallest normal float, 2^-126, may count as zero: T of them times |u| and the largest value (bf16 results
        # go down to 2^-133, so that this shows beside a row all of whose probabilities are below 2^-126)
        floor = floor + (scale * T * 2.0 ** -126 * float(u.max()) * float(q.double().abs().max()) if T else 0.0)
        err = (gw.double() - ref).abs()
        bound = size * (per + (T / 8 + 64) * 2.0 ** -24) + floor + ref.abs() * half_step(dtype) + smallest
        assert (err <= bound).all(), (float((err / bound).max()), float(err.max()))
