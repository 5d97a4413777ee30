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


# -------------------------------------- the residual step's gradients in whole numbers
#
# Rows of eight-column groups, each a whole number times one of the rows h_i of an 8 x 8
# Hadamard matrix (h_i h_j = h_(i xor j), of sum 0 for i != j), so that with eps 0 every
# quantity on the way is a whole number and fp32 holds it and every sum exactly:
#   r = +-h_1 and, under a norm, y = +-h_2 are their own normalised rows;
#   grad_h = t h_3, grad_r = u h_4, parameters constant over a group: the means over a row of
#   grad_h M, of its product with r, of e G and of its product with y are 0.
# t and u have no zeros: every row counts in every sum.

def _hadamard(i):
    return torch.tensor([(-1.0) ** bin(i & j).count("1") for j in range(8)], dtype=torch.double)


def whole_step(n, dim, frame, post, names, with_y=True, seed=0):
    """(tensors by name, grad_r, grad_h) in float64."""
    g = torch.Generator().manual_seed(seed)

    def rows(count, *values):
        at = torch.randint(len(values), (count, dim // 8, 1), generator=g)
        return torch.tensor(values, dtype=torch.double)[at]

    def along(x, i=0):
        return (x * _hadamard(i)).reshape(x.shape[0], dim)

    t = {"x": along(rows(n, -1, 1), 1)}
    if with_y:
        t["y"] = along(rows(n, -1, 1) if post != "none" else rows(n, -2, -1, 1, 2), 2)
    frames = -(-n // (frame or n))
    for name in names:
        if name in ("gate", "scale", "shift"):
            t[name] = along(rows(frames, -1, 1, 2) - float(name == "scale"))
        else:
            t[name] = along(rows(1, -1, 1, 2))[0]
    return t, along(rows(n, -2, -1, 1, 2), 4), along(rows(n, -2, -1, 1, 2), 3)


def whole_gradients(t, gr, gh, kind, a, frame):
    """Every gradient of that step by name, in float64, at r = t["x"]."""
    n, dim = t["x"].shape
    of = torch.arange(n, device=gr.device) // (frame or n)
    frames = int(of[-1]) + 1

    def param(name, none):
        p = t.get(name)
        return none if p is None else p[of] if name in ("gate", "scale", "shift") else p

    def add(x):       # a frame's rows
        return torch.zeros(frames, dim, dtype=torch.double, device=x.device).index_add_(0, of, x)

    e, found = gr, {}
    if kind != "none":
        wide = 1 + param("scale", 0.0)
        e = gr + gh * param("weight", 1.0) * wide
        found["shift"] = add(gh)
        found["scale"] = add(gh * (t["x"] * param("weight", 1.0) + param("bias", 0.0)))
        found["weight"] = (gh * t["x"] * wide).sum(0)
        found["bias"] = (gh * wide).sum(0)
    found["x"] = a * e
    if "y" in t:
        found["gate"] = add(e * t["y"] * param("post_weight", 1.0))
        found["post_weight"] = (e * t["y"] * param("gate", 1.0)).sum(0)
        found["y"] = e * param("gate", 1.0) * param("post_weight", 1.0)
    return {k: x for k, x in found.items() if k in t}


# The 2-norm of what a row of r, h, dx or dy is off by in fp32, relative to its own, for rows
# whose mean is below their deviations and terms that do not cancel, u = 2^-24.  A sum over a
# row has at most 16 additions in a thread, 6 over a wave, 4 over waves: 26 u of the sizes added.
# A mean is then off by 28 u of them, a factor by half of (26 + 3) u + 2 (28 + 1) u and 3 u,
# 47 u, a normalised element by 28 u + 1 u and 47 u of itself: 76 u, with the parameters 80 u, of
# sizes that together are no larger than twice the result; h behind a norm of y has both norms',
# a gradient through a norm two more such means beside it, of terms that are off by those 80 u,
# and dy twice that.
ROW_NORM = {"r": 160 * 2.0 ** -24, "h": 240 * 2.0 ** -24, "x": 480 * 2.0 ** -24, "y": 960 * 2.0 ** -24}


def row_case(dim, post, n=60, seed=0):
    """Tensors by name, grad_r and grad_h, in float32, frames of 25 rows."""
    g = torch.Generator().manual_seed(seed + dim)

    def normal(rows, size, mean=0.0):
        return torch.randn(rows, dim, generator=g) * size + mean

    t = {"x": normal(n, 1.5, 0.3), "y": normal(n, 0.7, 0.2), "gate": normal(3, 0.1, 0.5),
         "scale": normal(3, 0.1), "shift": normal(3, 0.4), "weight": normal(1, 0.1, 1.0)[0]}
    if post != "none":
        t["post_weight"] = normal(1, 0.1, 1.0)[0]
    return t, normal(n, 0.5, 0.2), normal(n, 0.5, 0.2)


def row_results(t, gr, gh, kind, post, eps, frame, left=None):
    """r and h of the step, dx and dy at t["x"] in r's place, in float64; `left`: a column that
    the rows' means leave out."""
    dim = t["x"].shape[-1]
    of = torch.arange(t["x"].shape[0], device=gr.device) // frame
    keep = torch.ones(dim, dtype=torch.double, device=gr.device)
    if left is not None:
        keep[left] = 0.0

    def mean(x):
        return (x * keep).sum(-1, keepdim=True) / dim

    def norm(x, kind):
        if kind == "none":
            return x, 1.0
        x = x - mean(x) if kind == "layer" else x
        f = 1 / torch.sqrt(mean(x * x) + eps)
        return x * f, f

    def back(g, u, f, kind):
        if kind == "none":
            return g
        return f * (g - (mean(g) if kind == "layer" else 0.0) - u * mean(g * u))

    v, fv = norm(t["y"], post)
    scale = t["gate"][of] * t.get("post_weight", 1.0)
    r = t["x"] + scale * v
    m = t["weight"] * (1 + t["scale"][of])
    u, f = norm(t["x"], kind)
    e = gr + back(gh * m, u, f, kind)
    return {"r": r, "h": norm(r, kind)[0] * m + t["shift"][of], "x": e,
            "y": back(e * scale, v, fv, post)}
