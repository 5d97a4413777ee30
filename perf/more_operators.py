"""Timed cases of the training operators of a video transformer's block.

What a program that fine-tunes a model under a block mask runs around its matrix
products:

    attention   softmax attention over every key or over the kept blocks of a
                block CSR, with each row's log-sum-exp, and the gradients of q, k
                and v from that of its output (one training pass: both)
    norm        the step from one block of a layer to the next on the residual
                stream:   r = a x + gate * P(y),   h = N(r) * (1 + scale) + shift
                (y the block's output, P a norm of it or nothing, N the next
                block's norm; gate, scale and shift one row for each frame)
    back        its gradients from those of r and h: of x, of y, of each frame's
                gate, scale and shift, of the norms' weights

Attention is of heads of 128 in bf16, scores divided by sqrt(128):
    p = exp(s - lse),  o = p v,  dv = p' do,  ds = p * (do v' - rowsum(do * o)),
    dq = ds k / sqrt(128),  dk = ds' q / sqrt(128).
A row without keys has o = 0, lse = -inf and no gradient.

The shapes are those of the repository's workloads (Wan 2.1 1.3B and 14B, 30x52
latents, 12 and 40 heads; HunyuanVideo 1.5, 30x53 latents, 16 heads, 512 text
tokens) and generic ones.
"""
import math

import numpy as np
import torch

own = False

D = 128
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
BYTES = {"bf16": 2, "f16": 2, "f32": 4}
KINDS = ("none", "layer", "rms")
EPS = 1e-6
PARAMS = ("gate", "scale", "shift", "weight", "bias", "post_weight")


def _attention(name, H, N, B=128, layout="hnd", mask="", P=0, W=0, tper=0, share=0.0, rows=0):
    """H heads of N tokens; mask "": every key, "frames": frames of P tokens within
    W frames and every tper-th frame, "random": each block of B with probability
    `share`, the fourth query block of each five empty (`rows` seeds them)."""
    return _named(name, dict(op="attention", H=H, N=N, B=B, layout=layout, mask=mask, P=P, W=W,
                             tper=tper, share=share, rows=rows))


def _norm(name, op, n, dim, frame, stream="bf16", block="bf16", params="f32", kind="layer",
          post="none", y=True, gate=True, scale=True, weight=False, bias=False, a=1.0):
    """n tokens of `dim` channels, a row of gate, scale and shift for each `frame`
    tokens; `stream`: the type of x and r, `block`: of y and h, `params`: of the rest;
    `weight`: N and P have weights, `bias`: N has a bias."""
    return _named(name, dict(op=op, n=n, dim=dim, frame=frame, stream=stream, block=block,
                             params=params, kind=kind, post=post, y=y, gate=gate, scale=scale,
                             weight=weight, bias=bias, a=a))


def _named(name, c):
    return dict(c, name=name) if name else c


def listed():
    return [
        # One head over the tiny workload's 4 frames of 16x16, own frame and one
        # global: the smallest training pass, latency.
        _attention("attention_tiny", 1, 1024, B=64, mask="frames", P=256, W=0, tper=4),
        # A layer over 8 frames, heads as views of a fused projection.
        _attention("attention_frames_nhd", 12, 8 * 1560, layout="nhd", mask="frames", P=1560,
                   W=2, tper=4),
        # A caller's own mask: an odd length, small blocks, empty rows.
        _attention("attention_random_odd", 5, 4999, B=64, mask="random", share=0.3, rows=16),
        # A whole clip at the training horizon, every key.
        _attention("attention_clip", 12, 21 * 1560),
        # Two heads (a head-parallel share) of a 121-frame video under its mask: the
        # longest axis, and key blocks that every query keeps beside ones that few do.
        _attention("attention_long", 2, 121 * 1560, mask="frames", P=1560, W=6, tper=16),
        # One token of text into a layer: the smallest call, latency.
        _norm("norm_token", "norm", 1, 1536, 1),
        # The newest frame of the 14B model, its residual stream in 32 bits.
        _norm("norm_frame", "norm", 1560, 5120, 1560, stream="f32"),
        # Queries or keys of a chunk, each head's 128 normalised, no residual.
        _norm("norm_heads", "norm", 16 * 8 * 1590, 128, 1590, params="bf16", kind="rms", y=False,
              gate=False, scale=False, weight=True),
        # A whole clip of the 1.3B model.
        _norm("norm_clip", "norm", 21 * 1560, 1536, 1560),
        # Its gradients, the way back.
        _norm("back_clip", "back", 21 * 1560, 1536, 1560),
        # Frames and text of odd sizes, a norm before and behind the block, weights
        # with gradients, half precision.
        _norm("back_sandwich", "back", 4 * 1590 + 509, 2048, 1590, stream="f16", block="f16",
              kind="rms", post="rms", scale=False, weight=True, a=0.5),
        # A whole clip of the 14B model, its residual stream in 32 bits: the largest.
        _norm("back_clip_wide", "back", 21 * 1560, 5120, 1560, stream="f32", kind="layer",
              weight=True, bias=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    caps = {c["op"]: work(c) for c in listed()}
    caps["attention"] = work(next(c for c in listed() if c["name"] == "attention_clip"))
    while True:
        op = rng.choice(["attention", "attention", "norm", "back"])
        if op == "attention":
            mask = rng.choice(["", "frames", "frames", "random"])
            P = _log_int(rng, 4, 34) * _log_int(rng, 4, 60)
            N = (_log_int(rng, 1, 121) * P + (_log_int(rng, 1, 512) if rng.random() < 0.3 else 0)
                 if mask == "frames" else _log_int(rng, 2, 60000))
            c = _attention(None, _log_int(rng, 1, 40), N, B=rng.choice([64, 128]),
                           layout=rng.choice(["hnd", "nhd"]), mask=mask,
                           P=P if mask == "frames" else 0,
                           W=rng.randint(0, 6) if mask == "frames" else 0,
                           tper=rng.randint(2, 18) if mask == "frames" else 0,
                           share=rng.uniform(0.05, 0.7) if mask == "random" else 0.0,
                           rows=rng.randint(0, 1 << 30) if mask == "random" else 0)
            fits = (N <= 190000 and c["H"] * N <= 2e6
                    and 0 < work(c)["flops"] <= caps["attention"]["flops"])
        else:
            stream, block = rng.choice([("bf16", "bf16"), ("f16", "f16"), ("f32", "f32"),
                                        ("f32", "bf16"), ("f32", "f16")])
            n, y = _log_int(rng, 1, 400000), rng.random() < 0.8
            c = _norm(None, op, n, 8 * _log_int(rng, 8, 1024), _log_int(rng, 1, 4000),
                      stream=stream, block=block, params=rng.choice(["f32", block]),
                      kind=rng.choice(["layer", "rms"]),
                      post=rng.choice(KINDS) if y else "none", y=y,
                      gate=y and rng.random() < 0.8, scale=rng.random() < 0.7,
                      weight=rng.random() < 0.5, bias=rng.random() < 0.3,
                      a=rng.choice([1.0, 1.0, 0.5]) if y else 1.0)
            fits = (n // c["frame"] <= 4000 and work(c)["bytes"] <= caps["back"]["bytes"]
                    and c["n"] * c["dim"] <= 1.7e8)
        if fits:
            return c


# ------------------------------------------------------------------ masks

def _kept_blocks(c):
    """The kept blocks [nb][nb] of a mask as a boolean array."""
    N, B = c["N"], c["B"]
    nb = -(-N // B)
    if c["mask"] == "random":
        kept = np.random.default_rng(c["rows"]).random((nb, nb)) < c["share"]
        kept[3::5] = False
        return kept
    # Blocks that touch a kept pair of frames; tokens behind the last whole frame are
    # text: they see, and are seen by, every token.
    T, W = N // c["P"], c["W"]
    t = np.arange(T + 1)
    frames = ((np.abs(t[:, None] - t[None, :]) <= W) | (t[None, :] % c["tper"] == 0)
              | (t[:, None] == T) | (t[None, :] == T))
    first = np.minimum(np.arange(nb) * B // c["P"], T)
    last = np.minimum((np.minimum((np.arange(nb) + 1) * B, N) - 1) // c["P"], T)
    touch = ((t[None, :] >= first[:, None]) & (t[None, :] <= last[:, None])).astype(np.float32)
    return (touch @ frames.astype(np.float32) @ touch.T) > 0


def _pairs(c):
    """Query and key token pairs that one head attends."""
    N, B = c["N"], c["B"]
    if not c["mask"]:
        return N * N
    kept = _kept_blocks(c)
    size = np.minimum(np.arange(1, len(kept) + 1) * B, N) - np.arange(len(kept)) * B
    return int(size @ (kept @ size))


def work(c):
    """Attention: the two products forward and the five back (scores once more);
    q, k, v and the gradient of the output in, the output, the log-sum-exp and three
    gradients out.  Norms: each input once, each output once, and what an element
    takes (a norm 8 operations forward and 12 back, a gate or a scale 2 and 4)."""
    if c["op"] == "attention":
        H, N = c["H"], c["N"]
        return {"bytes": H * N * (8 * 2 * D + 4), "flops": 7 * 2 * H * D * _pairs(c)}
    n, dim, s, b, p = c["n"], c["dim"], BYTES[c["stream"]], BYTES[c["block"]], BYTES[c["params"]]
    rows = -(-n // c["frame"])
    params = dim * p * ((rows if c["gate"] else 0) + (2 * rows if c["scale"] else 0)
                        + (1 if c["weight"] else 0) + (1 if c["bias"] else 0)
                        + (1 if c["weight"] and c["post"] != "none" else 0))
    norms = 1 + (c["post"] != "none")
    ops = 2 if c["op"] == "norm" else 4
    flops = n * dim * ((8 if c["op"] == "norm" else 12) * norms
                       + ops * (c["y"] + c["gate"] + c["scale"] + c["weight"]))
    if c["op"] == "norm":
        elements = (2 * s + 2 * b) if c["y"] else s + b
        return {"bytes": n * dim * elements + params, "flops": flops}
    # r, the gradients of r and h, y; gradients of x and y; parameters in and out
    elements = 3 * s + b + (2 * b if c["y"] else 0)
    return {"bytes": n * dim * elements + 2 * params, "flops": flops}


# ----------------------------------------------------------------- inputs

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed) % (1 << 62))


def _rows(g, H, n, layout, spread):
    """Values [H, n, 128] in bf16, each head with a spread of its own as a model's
    layers have them; "nhd": a view of one [n, H, 128] buffer."""
    wide = torch.exp(spread * torch.randn(H, 1, 1, generator=g, device="cuda"))
    if layout == "nhd":
        x = torch.randn(n, H, D, generator=g, device="cuda") * wide.transpose(0, 1)
        return x.bfloat16().transpose(0, 1)
    return (torch.randn(H, n, D, generator=g, device="cuda") * wide).bfloat16()


def prepare(c, seed):
    g = _gen(seed)
    s = {"c": c}
    if c["op"] == "attention":
        for name, spread in (("q", 0.3), ("k", 0.3), ("v", 0.5), ("grad", 0.5)):
            s[name] = _rows(g, c["H"], c["N"], c["layout"], spread)
        if c["mask"]:
            kept = _kept_blocks(c)
            s["row_ptr"] = torch.from_numpy(np.concatenate(
                [[0], kept.sum(1).cumsum()]).astype(np.int32)).cuda()
            s["col_idx"] = torch.from_numpy(np.nonzero(kept)[1].astype(np.int32)).cuda()
            s["widest"] = int(kept.sum(1).max())
    else:
        n, dim, frames = c["n"], c["dim"], -(-c["n"] // c["frame"])

        def normal(rows, kind, size=1.0, mean=0.0):
            x = torch.randn(rows, dim, generator=g, device="cuda")
            return (x * size + mean).to(TYPES[c[kind]])

        # A stream whose tokens and channels differ in size, as it is deep in a model.
        size = torch.exp(0.5 * torch.randn(1, dim, generator=g, device="cuda"))
        s["r" if c["op"] == "back" else "x"] = normal(n, "stream", size, 0.1)
        if c["y"]:
            s["y"] = normal(n, "block", 0.7)
        if c["op"] == "back":
            s["grad_r"], s["grad_h"] = normal(n, "stream", 0.1), normal(n, "block", 0.1)
        if c["gate"]:
            s["gate"] = normal(frames, "params", 0.3, 0.2)
        if c["scale"]:
            # neighbouring rows of one modulation tensor, as a model computes them
            both = torch.randn(frames, 2, dim, generator=g, device="cuda") * 0.3
            s["scale"], s["shift"] = both.to(TYPES[c["params"]]).unbind(1)
        if c["weight"]:
            s["weight"] = normal(1, "params", 0.2, 1.0)[0]
            if c["post"] != "none":
                s["post_weight"] = normal(1, "params", 0.2, 1.0)[0]
        if c["bias"]:
            s["bias"] = normal(1, "params", 0.2)[0]
    if own:
        _handles(s)
    return s


def _handles(s):
    """The objects that a program keeps beside its buffers."""
    import paper_2605_31057_amd as lvsa
    c = s["c"]
    s["lvsa"] = lvsa
    if c["op"] == "attention":
        s["mask"] = (lvsa.csr_mask(s["row_ptr"], s["col_idx"], c["N"], c["B"]) if c["mask"]
                     else None)
    else:
        kinds = {"none": lvsa.NORM_NONE, "layer": lvsa.NORM_LAYER, "rms": lvsa.NORM_RMS}
        s["plan"] = lvsa.ResidualNorm(c["dim"], norm=kinds[c["kind"]], post=kinds[c["post"]],
                                      eps=EPS, residual=c["a"], frame_tokens=c["frame"])
        s["params"] = {k: s[k] for k in PARAMS if k in s}


# -------------------------------------------------------------------- run

def run(s):
    if own:
        return _run_own(s)
    if s["c"]["op"] == "attention":
        return _plain_attention(s, s["c"])
    return _plain_norm(s, s["c"]) if s["c"]["op"] == "norm" else _plain_back(s, s["c"])


def _run_own(s):
    c, lvsa = s["c"], s["lvsa"]
    if c["op"] == "attention":
        out, lse = lvsa.attention_lse(s["q"], s["k"], s["v"], s["mask"])
        dq, dk, dv = lvsa.attention_backward(s["grad"], s["q"], s["k"], s["v"], out, lse, s["mask"])
        return {"out": out, "lse": lse, "dq": dq, "dk": dk, "dv": dv}
    if c["op"] == "norm":
        if not c["y"]:
            return {"h": lvsa.residual_norm(s["plan"], s["x"], dtype=TYPES[c["block"]],
                                            **s["params"])}
        r, h = lvsa.residual_norm(s["plan"], s["x"], s["y"], **s["params"])
        return {"r": r, "h": h}
    return lvsa.residual_norm_backward(s["plan"], s["grad_h"], s["grad_r"], s["r"], s.get("y"),
                                       **s["params"])


# ------------------------------------------------------------ plain forms

def _plain_attention(s, c):
    """Some query blocks at a time (all scores of a long video do not fit the card),
    each with its kept key blocks gathered, short rows filled up and masked."""
    H, N, B = c["H"], c["N"], c["B"]
    nb = -(-N // B)

    def blocks(x):
        x = torch.nn.functional.pad(x.float(), (0, 0, 0, nb * B - N))
        return x.reshape(H, nb, B, D)

    q, k, v, grad = (blocks(s[x]) for x in ("q", "k", "v", "grad"))
    widest = s["widest"] if c["mask"] else nb
    at = torch.arange(widest, device="cuda").expand(nb, widest)
    there = torch.ones(nb, widest, dtype=torch.bool, device="cuda")
    if c["mask"]:
        rows = s["row_ptr"].long()
        there = at < rows.diff()[:, None]
        at = s["col_idx"][torch.where(there, rows[:-1, None] + at, 0)].long()
    keys = at[..., None] * B + torch.arange(B, device="cuda")
    there = (there[..., None] & (keys < N)).reshape(nb, 1, widest * B)
    out, dq, dk, dv = (torch.zeros_like(q) for _ in range(4))
    lse = torch.empty(H, nb, B, device="cuda")
    group = max(1, int(3e9) // max(1, H * widest * B * 16 * (D + B)))
    for i in range(0, nb, group):
        e = min(nb, i + group)
        kk, vv = (x[:, at[i:e]].reshape(H, e - i, widest * B, D) for x in (k, v))
        p = torch.matmul(q[:, i:e] / math.sqrt(D), kk.transpose(2, 3))
        p.masked_fill_(~there[i:e], -math.inf)
        most = p.amax(-1, keepdim=True) if widest else torch.full_like(p[..., :1], -math.inf)
        p.sub_(torch.where(most > -math.inf, most, 0.0)).exp_()
        total = p.sum(-1, keepdim=True)
        lse[:, i:e] = torch.where(total > 0, most + total.log(), -math.inf)[..., 0]
        p.div_(torch.where(total > 0, total, 1.0))
        out[:, i:e] = torch.matmul(p, vv)
        ds = torch.matmul(grad[:, i:e], vv.transpose(2, 3))
        ds.sub_((grad[:, i:e] * out[:, i:e]).sum(-1, keepdim=True)).mul_(p)
        dq[:, i:e] = torch.matmul(ds, kk) / math.sqrt(D)
        where = at[i:e].reshape(-1)
        dv.index_add_(1, where, torch.matmul(p.transpose(2, 3), grad[:, i:e]).view(H, -1, B, D))
        dk.index_add_(1, where, torch.matmul(ds.transpose(2, 3), q[:, i:e]).view(H, -1, B, D),
                      alpha=1 / math.sqrt(D))
    found = {"out": out, "lse": lse, "dq": dq, "dk": dk, "dv": dv}
    return {name: x.reshape(H, nb * B)[:, :N].contiguous() if name == "lse"
            else x.reshape(H, nb * B, D)[:, :N].bfloat16() for name, x in found.items()}


def _plain_unit(x, kind):
    """x normalised over its channels, and the factor that did it."""
    if kind == "layer":
        x = x - x.mean(-1, keepdim=True)
    factor = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    return x * factor, factor


def _plain_unit_back(grad, unit, factor, kind):
    """Gradient of x from that of its normalised form."""
    less = unit * (grad * unit).mean(-1, keepdim=True)
    if kind == "layer":
        less = less + grad.mean(-1, keepdim=True)
    return factor * (grad - less)


def _plain_norm(s, c):
    frame = torch.arange(c["n"], device="cuda") // c["frame"]
    x = s["x"].float()
    if c["y"]:
        y = s["y"].float()
        if c["post"] != "none":
            y = _plain_unit(y, c["post"])[0]
            if c["weight"]:
                y = y * s["post_weight"].float()
        if c["gate"]:
            y = y * s["gate"].float()[frame]
        x = c["a"] * x + y
    h = _plain_unit(x, c["kind"])[0]
    if c["weight"]:
        h = h * s["weight"].float()
    if c["bias"]:
        h = h + s["bias"].float()
    if c["scale"]:
        h = h * (1 + s["scale"].float()[frame]) + s["shift"].float()[frame]
    h = h.to(TYPES[c["block"]])
    return {"r": x.to(TYPES[c["stream"]]), "h": h} if c["y"] else {"h": h}


def _frame_sums(x, c):
    """Sums of x [n, dim] over each frame's tokens, in 64 bits: they may be many."""
    frames = -(-c["n"] // c["frame"])
    x = torch.nn.functional.pad(x.double(), (0, 0, 0, frames * c["frame"] - c["n"]))
    return x.view(frames, c["frame"], -1).sum(1)


def _plain_back(s, c):
    frame = torch.arange(c["n"], device="cuda") // c["frame"]
    params = TYPES[c["params"]]
    found = {}
    dh = s["grad_h"].float()
    unit, factor = _plain_unit(s["r"].float(), c["kind"])
    a = unit
    if c["weight"]:
        a = a * s["weight"].float()
    if c["bias"]:
        a = a + s["bias"].float()
    if c["scale"]:
        found["scale"] = _frame_sums(dh * a, c).to(params)
        found["shift"] = _frame_sums(dh, c).to(params)
        dh = dh * (1 + s["scale"].float()[frame])
    if c["bias"]:
        found["bias"] = dh.double().sum(0).to(params)
    if c["weight"]:
        found["weight"] = (dh * unit).double().sum(0).to(params)
        dh = dh * s["weight"].float()
    dr = s["grad_r"].float() + _plain_unit_back(dh, unit, factor, c["kind"])
    found["x"] = (c["a"] * dr).to(TYPES[c["stream"]])
    if c["y"]:
        y, dy = s["y"].float(), dr
        if c["post"] != "none":
            unit, factor = _plain_unit(y, c["post"])
            y = unit * s["post_weight"].float() if c["weight"] else unit
        if c["gate"]:
            found["gate"] = _frame_sums(dr * y, c).to(params)
            dy = dr * s["gate"].float()[frame]
        if c["post"] != "none":
            if c["weight"]:
                found["post_weight"] = (dy * unit).double().sum(0).to(params)
                dy = dy * s["post_weight"].float()
            dy = _plain_unit_back(dy, unit, factor, c["post"])
        found["y"] = dy.to(TYPES[c["block"]])
    return {k: found[k] for k in ("x", "y", *PARAMS) if k in found}


# ------------------------------------------------------------------ exact

def exact(c, seed):
    global own
    was, own = own, False
    s = prepare(c, seed)
    own = was
    if c["op"] == "attention":
        return _exact_attention(s, c)
    return _exact_norm(s, c)


def _exact_attention(s, c):
    """One head and some queries of one row at a time: softmax over the kept keys
    alone, and its Jacobian (diag(p) - p p') times the gradient."""
    N, B = c["N"], c["B"]
    found = {x: torch.zeros(c["H"], N, D, dtype=torch.float64, device="cuda")
             for x in ("out", "dq", "dk", "dv")}
    found["lse"] = torch.full((c["H"], N), -math.inf, dtype=torch.float64, device="cuda")
    pieces = []
    if c["mask"]:
        kept = _kept_blocks(c)
        for row, keep in enumerate(kept):
            keys = np.nonzero(np.repeat(keep, B)[:N])[0]
            if len(keys):
                pieces.append((slice(row * B, min(N, row * B + B)), torch.from_numpy(keys).cuda()))
    else:
        step = max(1, int(2.5e8) // N)
        pieces = [(slice(i, min(N, i + step)), slice(None)) for i in range(0, N, step)]
    for head in range(c["H"]):
        q, k, v, grad = (s[x][head].double() for x in ("q", "k", "v", "grad"))
        for rows, keys in pieces:
            kk, vv, qq, gg = k[keys], v[keys], q[rows], grad[rows]
            logits = qq @ kk.T * D ** -0.5
            found["lse"][head, rows] = torch.logsumexp(logits, -1)
            p = torch.softmax(logits, -1)
            found["out"][head, rows] = p @ vv
            found["dv"][head, keys] += p.T @ gg
            dp = gg @ vv.T
            ds = (dp - (p * dp).sum(-1, keepdim=True)) * p * D ** -0.5
            found["dq"][head, rows] = ds @ kk
            found["dk"][head, keys] += ds.T @ qq
    return {x: found[x] for x in ("out", "lse", "dq", "dk", "dv")}


def _exact_norm(s, c):
    """Forward from the definition; backward by automatic differentiation of it
    around the given r."""
    wide = {k: x.double().requires_grad_() for k, x in s.items() if torch.is_tensor(x)}
    of = torch.div(torch.arange(c["n"], device="cuda"), c["frame"], rounding_mode="floor")

    def normed(x, kind):
        if kind == "layer":
            return (x - x.mean(1, keepdim=True)) / torch.sqrt(
                x.var(1, unbiased=False, keepdim=True) + EPS)
        return x / torch.sqrt(x.pow(2).mean(1, keepdim=True) + EPS)

    def added():
        y = wide["y"] if c["post"] == "none" else normed(wide["y"], c["post"])
        if "post_weight" in wide:
            y = y * wide["post_weight"]
        return y * wide["gate"][of] if c["gate"] else y

    def following(r):
        h = normed(r, c["kind"])
        h = h * wide["weight"] if c["weight"] else h
        h = h + wide["bias"] if c["bias"] else h
        return h * (wide["scale"][of] + 1) + wide["shift"][of] if c["scale"] else h

    if c["op"] == "norm":
        with torch.no_grad():
            if not c["y"]:
                return {"h": following(wide["x"])}
            r = c["a"] * wide["x"] + added()
            return {"r": r, "h": following(r)}
    names = [k for k in PARAMS if k in wide]
    after = [k for k in names if k not in ("gate", "post_weight")]
    into = torch.autograd.grad(following(wide["r"]), [wide["r"]] + [wide[k] for k in after],
                               wide["grad_h"].detach())
    found = dict(zip(after, into[1:]))
    dr = into[0] + wide["grad_r"].detach()
    found["x"] = c["a"] * dr
    if c["y"]:
        before = [k for k in names if k not in after]
        back = torch.autograd.grad(added(), [wide["y"]] + [wide[k] for k in before], dr)
        found["y"] = back[0]
        found.update(zip(before, back[1:]))
    return {k: found[k] for k in ("x", "y", *PARAMS) if k in found}
