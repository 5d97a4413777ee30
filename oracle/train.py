"""Attention with its gradients and the residual step between blocks with its gradients,
from their formulas in 64 bits, with bounds on what the library's roundings may add."""
import math

import torch

# half a step of each type, relative to the value
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}

# The 2-norm of what attention's results are off by, relative to them, for scores of a few
# units: up to three roundings to bf16 that do not know of each other (of p or e, of the
# output in delta, of the result), each uniform within 2^-8 of the value and so 2^-8 / sqrt(3)
# in the mean, 2^-8 together; twice that.
NORM = 2.0 ** -7


def attention(q, k, v, grad, kept):
    """q, k, v, grad [H, N, d] in float64, kept [N, N] boolean.  A dict of out, lse, dq, dk,
    dv and, under "bound", the most that each may be off by when probabilities (p) and
    their gradients (e) are rounded to bf16 before products, the output before
    delta = rowsum(grad out), results once at the end, and sums are in fp32."""
    d = q.shape[-1]
    half, f32 = 2.0 ** -8, 2.0 ** -24
    terms = (k.shape[1] + d) * f32
    s = q @ k.transpose(1, 2) / math.sqrt(d)
    size = q.abs() @ k.abs().transpose(1, 2) / math.sqrt(d)
    s = s.masked_fill(~kept, -math.inf)
    lse = torch.logsumexp(s, -1)
    p = torch.where(kept, torch.exp(s - torch.where(lse > -math.inf, lse, 0.0)[..., None]), 0.0)
    # exp of a score and a log-sum-exp that are off by fp32 roundings: of the 128 products'
    # sum, of the scale, and of the result's place (log2)
    off_s = size * (d + 4) * f32 + (s.abs().masked_fill(~kept, 0.0) + lse.abs().nan_to_num(
        posinf=0.0)[..., None]) * 8 * f32 + 16 * f32
    out = p @ v
    dp = grad @ v.transpose(1, 2)
    delta = (grad * out).sum(-1, keepdim=True)
    e = p * (dp - delta)
    off_delta = (half + terms + 2 * f32) * (grad.abs() * (p @ v.abs())).sum(-1, keepdim=True)
    off_dp = d * f32 * (grad.abs() @ v.abs().transpose(1, 2))
    off_e = e.abs() * (half + off_s) + p * (off_delta + off_dp) * (1 + half)
    off_p = p * (half + off_s)
    c = 1 / math.sqrt(d)
    r = {"out": out, "lse": lse, "dq": c * e @ k, "dk": c * e.transpose(1, 2) @ q,
         "dv": p.transpose(1, 2) @ grad}
    r["bound"] = {
        "lse": off_s.masked_fill(~kept, 0.0).amax(-1) + terms,
        "out": (2 * half + terms) * (p @ v.abs()) + (off_p @ v.abs()),
        "dq": c * (off_e @ k.abs()) + (half + terms) * c * (e.abs() @ k.abs()),
        "dk": c * (off_e.transpose(1, 2) @ q.abs())
        + (half + terms) * c * (e.abs().transpose(1, 2) @ q.abs()),
        "dv": off_p.transpose(1, 2) @ grad.abs()
        + (half + terms) * (p.transpose(1, 2) @ grad.abs()),
    }
    return r


def kept_tokens(kept, block, n):
    """Boolean [n, n] of a block mask [nb, nb]."""
    kept = torch.as_tensor(kept)
    return kept.repeat_interleave(block, 0).repeat_interleave(block, 1)[:n, :n]


def unit(x, kind, eps):
    """Rows normalised; kind "none", "layer" or "rms"."""
    if kind == "none":
        return x
    if kind == "layer":
        x = x - x.mean(-1, keepdim=True)
    return x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)


def residual_norm(x, y, kind, post, eps, a, frame, gate=None, scale=None, shift=None, weight=None,
                  bias=None, post_weight=None):
    """(r, h) in the inputs' precision; h None for kind "none"."""
    of = torch.arange(x.shape[0], device=x.device) // (frame or x.shape[0])
    r = x
    if y is not None:
        u = unit(y, post, eps)
        u = u if post_weight is None else u * post_weight
        r = a * x + (u if gate is None else gate[of] * u)
    if kind == "none":
        return r, None
    return r, after(r, kind, eps, of, scale, shift, weight, bias)


def after(r, kind, eps, of, scale=None, shift=None, weight=None, bias=None):
    """h of r."""
    h = unit(r, kind, eps)
    h = h if weight is None else h * weight
    h = h if bias is None else h + bias
    return h if scale is None else h * (1 + scale[of]) + shift[of]
