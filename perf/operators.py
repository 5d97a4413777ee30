"""Timed cases of the chunk-by-chunk generation operators.

A long video can be generated some latent frames at a time: the new frames'
queries attend to the keys and values of every frame so far, which stay in a
cache held in 8 bits.  The operators of that path:

    rope      rotary positions over (frame, row, column) of the latent grid
    back      its gradient
    write     new keys (rotated on the way) and values quantised into the cache
    read      cached tokens back as floating-point values
    attend    attention of a few tokens or whole frames over the cache, over
              every token or over the kept blocks of a block CSR

The cache: e4m3 values with one power-of-two scale per head and block of 64 or
128 tokens, the least 2^k (k >= -117) that keeps the block's largest finite
magnitude within 448.  Keys are [heads, capacity, 128].  Values are tiles
[heads, capacity / 64, 128, 64], one column of a tile after the other: token
16 a + 4 b + r of a tile (a, b, r < 4) is at place 16 b + 4 a + r.  Tokens that
a written block held before keep their values, rounded again to the new scale.

The shapes are those of the repository's workloads (Wan 2.1 1.3B and 14B, 30x52
latents, 12 and 40 heads; HunyuanVideo 1.5, 30x53 latents, 16 heads, 512 text
tokens) with frames arriving one to three at a time, and generic ones with
shared key heads.
"""
import math

import numpy as np
import torch

own = False

D = 128
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
BYTES = {"bf16": 2, "f16": 2, "f32": 4}
PAIRS = (22, 21, 21)     # of the 64 pairs of a head: frame, row, column
THETA = 10000.0


def _rope(name, op, H, n, T, h, w, start=0, halves=False, dtype="bf16", layout="hnd"):
    return _named(name, dict(op=op, H=H, n=n, T=T, h=h, w=w, start=start, halves=halves,
                             dtype=dtype, layout=layout))


def _write(name, H, n, held, T, h, w, B=128, rope=True, dtype="bf16", layout="hnd"):
    return _named(name, dict(op="write", H=H, n=n, held=held, T=T, h=h, w=w, B=B, rope=rope,
                             dtype=dtype, layout=layout))


def _read(name, H, n, start, held, B=128, dtype="bf16"):
    return _named(name, dict(op="read", H=H, n=n, start=start, held=held, B=B, dtype=dtype))


def _attend(name, H, G, n, held, B=128, layout="hnd", mask="", T=0, P=0, W=0, tper=0, hole=False):
    """H key heads, each read by G query heads; `held` cached tokens, the last
    n of which are the queries' own; mask "": every token, "frames": frames
    within W and every tper-th frame, over T frames of P tokens, in blocks of
    B tokens; `hole`: the first query block's row is empty."""
    return _named(name, dict(op="attend", H=H, G=G, n=n, held=held, B=B, layout=layout, mask=mask,
                             T=T, P=P, W=W, tper=tper, hole=hole))


def _named(name, c):
    return dict(c, name=name) if name else c


def listed():
    return [
        # One token's queries (a text token, or a probe of a cached video): latency.
        _rope("rope_token", "rope", 12, 1, 21, 30, 52, start=20 * 1560 + 777),
        # The queries of the newest frame, a view of the fused projection.
        _rope("rope_frame_nhd", "rope", 12, 1560, 21, 30, 52, start=20 * 1560, layout="nhd"),
        # A training step's gradient through the positions of a whole clip, in
        # the other pair order and the gradients' own 32 bits.
        _rope("rope_grad_clip", "back", 12, 21 * 1560, 21, 30, 52, halves=True, dtype="f32"),
        # One more token into a block that is partly filled: latency.
        _write("write_token", 12, 1, 21 * 1560, 22, 30, 52),
        # One denoising step's keys and values of the newest frame; its first
        # and last blocks hold other tokens too.
        _write("write_frame", 12, 1560, 20 * 1560, 21, 30, 52, layout="nhd"),
        # The cache of a whole conditioning clip of the 14B model, small blocks.
        _write("write_clip", 40, 21 * 1560, 0, 21, 30, 52, B=64),
        # A frame of the cache back, from an odd place, for a program's own use.
        _read("read_frame", 12, 1560, 7 * 1560 + 13, 21 * 1560, dtype="f32"),
        # A whole layer's cache back in bf16, text tokens included.
        _read("read_layer", 16, 65 * 1590 + 512, 0, 65 * 1590 + 512),
        # One query token over a clip: the smallest attention call.
        _attend("attend_token", 12, 1, 1, 21 * 1560),
        # Eight query tokens, 40 query heads that share 8 key heads, long cache
        # of an odd length: the cache's bytes count.
        _attend("attend_shared_long", 8, 5, 8, 131071),
        # The newest frame of a 121-frame video over the frames its mask keeps.
        _attend("attend_frame_mask", 12, 1, 1560, 121 * 1560, mask="frames", T=121, P=1560, W=6,
                tper=16),
        # Three new frames of the 14B model over every frame so far (twice the
        # training horizon): the largest.
        _attend("attend_chunk", 40, 1, 3 * 1560, 41 * 1560, layout="nhd"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    cap = listed()[-1]
    most = work(cap)["flops"]
    while True:
        op = rng.choice(["rope", "back", "write", "write", "read", "attend", "attend", "attend"])
        h, w, T = _log_int(rng, 4, 34), _log_int(rng, 4, 60), _log_int(rng, 1, 121)
        P, H = h * w, _log_int(rng, 1, 40)
        B = rng.choice([64, 128])
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        layout = rng.choice(["hnd", "nhd"])
        grid = T * P
        text = _log_int(rng, 1, 512) if rng.random() < 0.25 else 0
        if op in ("rope", "back"):
            n = _log_int(rng, 1, grid + text)
            c = _rope(None, op, H, n, T, h, w, start=rng.randint(0, grid + text - n),
                      halves=rng.random() < 0.5, dtype=dtype, layout=layout)
            fits = H * n <= 2.5e6
        elif op == "write":
            n = _log_int(rng, 1, grid + text)
            c = _write(None, H, n, rng.randint(0, grid + text - n), T, h, w, B=B,
                       rope=rng.random() < 0.7, dtype=dtype, layout=layout)
            fits = H * (n + c["held"]) <= 1.6e6
        elif op == "read":
            held = grid + text
            n = _log_int(rng, 1, held)
            c = _read(None, H, n, rng.randint(0, held - n), held, B=B, dtype=dtype)
            fits = H * held <= 2.5e6
        else:
            G = rng.choice([1, 1, 2, 4, 5, 8])
            H = _log_int(rng, 1, 16 if G > 1 else 40)
            mask = rng.choice(["", "frames"])
            held = grid if mask else _log_int(rng, 1, 150000)
            n = _log_int(rng, 1, min(held, 5000))
            c = _attend(None, H, G, n, held, B=B, layout=layout, mask=mask,
                        T=T if mask else 0, P=P if mask else 0, W=rng.randint(0, 6) if mask else 0,
                        tper=rng.randint(2, 18) if mask else 0,
                        hole=bool(mask) and n > 2 * B and rng.random() < 0.3)
            fits = (held <= 190000 and H * held <= 2.6e6 and H * G * n * held <= 1.2e10
                    and work(c)["flops"] <= most)
        if fits:
            return c


# ------------------------------------------------------------------ masks

def _block_rows(c):
    """The block CSR rows [nb][nb] of a "frames" mask as a boolean array: blocks
    that touch a kept pair of frames."""
    T, P, B, W, tper = c["T"], c["P"], c["B"], c["W"], c["tper"]
    nb = -(-c["held"] // B)
    t = np.arange(T)
    frames = (np.abs(t[:, None] - t[None, :]) <= W) | (t[None, :] % tper == 0)
    first = np.arange(nb) * B // P
    last = np.minimum((np.arange(nb) + 1) * B, c["held"]) - 1
    touch = (t[None, :] >= first[:, None]) & (t[None, :] <= (last // P)[:, None])
    kept = (touch.astype(np.float32) @ frames.astype(np.float32) @ touch.T.astype(np.float32)) > 0
    if c["hole"]:
        kept[(c["held"] - c["n"]) // B] = False
    return kept


def _pairs(c):
    """Query and key token pairs that a call attends, and the key tokens any does."""
    n, held = c["n"], c["held"]
    if not c["mask"]:
        return n * held, held
    B, kept = c["B"], _block_rows(c)
    size = np.minimum(np.arange(1, len(kept) + 1) * B, held) - np.arange(len(kept)) * B
    q = np.bincount((held - n + np.arange(n)) // B, minlength=len(kept))
    return int((q * (kept @ size)).sum()), int(size[kept[q > 0].any(0)].sum())


def work(c):
    """Each input once, each output once; the products of attention, three
    operations an element for a rotation, one multiplication and one comparison
    an element for the cache's scales."""
    H, n = c["H"], c["n"]
    if c["op"] in ("rope", "back"):
        return {"bytes": 2 * H * n * D * BYTES[c["dtype"]], "flops": 3 * H * n * D}
    if c["op"] == "write":
        old = c["held"] % c["B"]     # held tokens of the first block: read, and rounded again
        return {"bytes": 2 * H * D * (n * (BYTES[c["dtype"]] + 1) + old),
                "flops": H * n * D * (7 if c["rope"] else 4)}
    if c["op"] == "read":
        return {"bytes": 2 * H * n * D * (1 + BYTES[c["dtype"]]), "flops": 2 * H * n * D}
    pairs, keys = _pairs(c)
    return {"bytes": 2 * 2 * H * c["G"] * n * D + 2 * H * keys * D,
            "flops": 4 * H * c["G"] * pairs * D}


# ----------------------------------------------------------------- inputs

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed) % (1 << 62))


def _normal(g, H, n, dtype, layout="hnd"):
    """N(0, 1) values [H, n, 128]; "nhd": a view of one [n, H, 128] buffer."""
    if layout == "nhd":
        return torch.randn(n, H, D, generator=g, device="cuda").to(dtype).transpose(0, 1)
    return torch.randn(H, n, D, generator=g, device="cuda").to(dtype)


def _table(c):
    """(cos, sin) of every position of each axis and each of its pairs, [.., 2]
    in 32 bits from angles in 64: frames, then rows, then columns."""
    parts = []
    for size, pairs in zip((c["T"], c["h"], c["w"]), PAIRS):
        at = torch.arange(size, dtype=torch.float64, device="cuda")[:, None]
        angle = at * THETA ** (-torch.arange(pairs, dtype=torch.float64, device="cuda") / pairs)
        parts.append(torch.stack([angle.cos(), angle.sin()], -1).reshape(-1, 2))
    return torch.cat(parts).float()


def _empty_cache(H, tokens, B):
    cap = -(-tokens // 128) * 128
    f8 = torch.float8_e4m3fn
    return {"k": torch.zeros(H, cap, D, dtype=f8, device="cuda"),
            "v": torch.zeros(H, cap // 64, D, 64, dtype=f8, device="cuda"),
            "k_scale": torch.full((H, cap // B), 2.0 ** -117, device="cuda"),
            "v_scale": torch.full((H, cap // B), 2.0 ** -117, device="cuda")}


def _fill(g, cache, held, B):
    """`held` tokens of keys and values with a spread of their own for each
    head, as a model's layers have them."""
    H = cache["k"].shape[0]
    spread = torch.exp(0.5 * torch.randn(2, H, 1, 1, generator=g, device="cuda"))
    k = _normal(g, H, held, torch.float32) * spread[0]
    v = _normal(g, H, held, torch.float32) * spread[1]
    _plain_write(cache, k.bfloat16(), v.bfloat16(), 0, B, None)


def prepare(c, seed):
    g = _gen(seed)
    op, H, n = c["op"], c["H"], c["n"]
    s = {"c": c}
    if op in ("rope", "back"):
        s["x"] = _normal(g, H, n, TYPES[c["dtype"]], c["layout"])
        s["table"] = _table(c)
    elif op == "write":
        s["cache"] = _empty_cache(H, c["held"] + n, c["B"])
        if c["held"]:
            _fill(g, s["cache"], c["held"], c["B"])
        s["k"] = _normal(g, H, n, TYPES[c["dtype"]], c["layout"])
        s["v"] = _normal(g, H, n, TYPES[c["dtype"]], c["layout"])
        s["table"] = _table(c)
    else:
        s["cache"] = _empty_cache(H, c["held"], c["B"])
        _fill(g, s["cache"], c["held"], c["B"])
        if op == "attend":
            s["q"] = _normal(g, H * c["G"], n, torch.bfloat16, c["layout"])
            if c["mask"]:
                kept = _block_rows(c)
                s["row_ptr"] = torch.from_numpy(np.concatenate(
                    [[0], kept.sum(1).cumsum()]).astype(np.int32)).cuda()
                s["col_idx"] = torch.from_numpy(np.nonzero(kept)[1].astype(np.int32)).cuda()
    if own:
        _handles(s)
    return s


def _handles(s):
    """The objects that a program keeps beside its buffers."""
    import paper_2605_31057_amd as lvsa
    c = s["c"]
    s["lvsa"] = lvsa
    if "table" in s:
        s["rope"] = lvsa.Rope(c["T"], c["h"], c["w"], pairs=PAIRS, table=s["table"],
                              layout=lvsa.ROPE_HALVES if c.get("halves") else lvsa.ROPE_PAIRS)
    if "cache" in s:
        b = s["cache"]
        s["kv"] = lvsa.KvCache(c["H"], b["k"].shape[1], c["B"], n_tokens=c["held"],
                               buffers=(b["k"], b["v"], b["k_scale"], b["v_scale"]))
    if "row_ptr" in s:
        s["mask"] = lvsa.csr_mask(s["row_ptr"], s["col_idx"], c["held"], c["B"])


# -------------------------------------------------------------------- run

def run(s):
    c = s["c"]
    if own:
        return _run_own(s)
    if c["op"] in ("rope", "back"):
        y = _plain_rotate(s["x"].float(), s["table"], c, c["start"], c["halves"], c["op"] == "back")
        return y.to(s["x"].dtype)
    if c["op"] == "write":
        rotate = (s["table"], c) if c["rope"] else None
        _plain_write(s["cache"], s["k"], s["v"], c["held"], c["B"], rotate)
        return s["cache"]
    if c["op"] == "read":
        k, v = _plain_values(s["cache"], c["B"], c["start"], c["start"] + c["n"])
        return k.to(TYPES[c["dtype"]]), v.to(TYPES[c["dtype"]])
    return _plain_attend(s, c)


def _run_own(s):
    c, lvsa = s["c"], s["lvsa"]
    if c["op"] == "rope":
        return lvsa.rope(s["x"], s["rope"], start=c["start"])
    if c["op"] == "back":
        return lvsa.rope_backward(s["x"], s["rope"], start=c["start"])
    if c["op"] == "write":
        lvsa.kv_write(s["kv"], s["k"], s["v"], start=c["held"],
                      rope=s["rope"] if c["rope"] else None)
        return s["cache"]
    if c["op"] == "read":
        return lvsa.kv_read(s["kv"], c["start"], c["n"], dtype=TYPES[c["dtype"]])
    return lvsa.attention_cache(s["q"], s["kv"], mask=s.get("mask"), q_start=c["held"] - c["n"])


# ------------------------------------------------------------ plain forms

def _plain_rotate(x, table, c, start, halves=False, back=False):
    """Rotates x [H, n, 128]; the tokens past the grid stay as they are."""
    T, h, w = c["T"], c["h"], c["w"]
    i = start + torch.arange(x.shape[1], device=x.device)
    inside = i < T * h * w
    i = torch.where(inside, i, 0)
    t, y, z = table.to(x.dtype).split([T * PAIRS[0], h * PAIRS[1], w * PAIRS[2]])
    cs = torch.cat([t.view(T, PAIRS[0], 2)[i // (h * w)], y.view(h, PAIRS[1], 2)[i // w % h],
                    z.view(w, PAIRS[2], 2)[i % w]], 1)
    cos = torch.where(inside[:, None], cs[..., 0], 1.0)
    sin = torch.where(inside[:, None], cs[..., 1], 0.0)
    sin = -sin if back else sin
    a, b = (x[..., :64], x[..., 64:]) if halves else (x[..., 0::2], x[..., 1::2])
    p, q = a * cos - b * sin, a * sin + b * cos
    return torch.cat([p, q], -1) if halves else torch.stack([p, q], -1).flatten(-2)


def _order():
    """Token of a 64-token tile at each of its places."""
    at = torch.arange(64, device="cuda")
    return 16 * (at // 4 % 4) + 4 * (at // 16) + at % 4


def _plain_values(cache, B, first, end):
    """The float32 keys and values [H, end - first, 128] of tokens first .. end - 1."""
    lo, hi = first // 128 * 128, -(-end // 128) * 128
    H = cache["k"].shape[0]
    k = cache["k"][:, lo:hi].float()
    tiles = cache["v"][:, lo // 64: hi // 64].float()
    v = torch.empty_like(tiles)
    v[..., _order()] = tiles
    v = v.transpose(2, 3).reshape(H, hi - lo, D)
    ks = cache["k_scale"][:, lo // B: hi // B].repeat_interleave(B, 1)[..., None]
    vs = cache["v_scale"][:, lo // B: hi // B].repeat_interleave(B, 1)[..., None]
    return (k * ks)[:, first - lo: end - lo], (v * vs)[:, first - lo: end - lo]


def _plain_quantise(x, B):
    """x [H, n, 128], n a multiple of B, to e4m3 and scales [H, n / B]."""
    H, n, _ = x.shape
    x = x.reshape(H, n // B, B * D)
    most = torch.where(x.isfinite(), x.abs(), 0.0).amax(-1)
    m, e = torch.frexp(most)                                # most = m 2^e, 0.5 <= m < 1
    e = torch.where(m > 0.875, e - 8, e - 9).clamp(min=-117)   # 448 = 0.875 2^9
    e = torch.where(most > 0, e, -117)
    q = torch.ldexp(x, -e[..., None])
    q = torch.where(x.isfinite(), q, math.nan).to(torch.float8_e4m3fn)
    return q.reshape(H, n, D), torch.ldexp(torch.ones_like(most), e)


def _plain_write(cache, k, v, start, B, rotate):
    """Tokens start .. start + n - 1; the blocks that they touch hold the earlier
    tokens they had and zeros behind the new ones."""
    H, n, _ = k.shape
    end = start + n
    lo, hi = start // 128 * 128, -(-end // 128) * 128
    new_k, new_v = k.float(), v.float()
    if rotate:
        # 64 bits: a rotated value next to a rounding border goes to the right side
        new_k = _plain_rotate(k.double(), rotate[0], rotate[1], start).float()
    whole_k = torch.zeros(H, hi - lo, D, device=k.device)
    whole_v = torch.zeros(H, hi - lo, D, device=k.device)
    if start > lo:
        whole_k[:, : start - lo], whole_v[:, : start - lo] = _plain_values(cache, B, lo, start)
    whole_k[:, start - lo: end - lo] = new_k
    whole_v[:, start - lo: end - lo] = new_v
    # blocks of 64 tokens: the first or last of the 128-token range may stay untouched
    a, z = start // B * B - lo, -(-end // B) * B - lo
    q, ks = _plain_quantise(whole_k[:, a:z], B)
    cache["k"][:, lo + a: lo + z] = q
    cache["k_scale"][:, (lo + a) // B: (lo + z) // B] = ks
    q, vs = _plain_quantise(whole_v[:, a:z], B)
    q = q.view(torch.uint8).reshape(H, (z - a) // 64, 64, D).transpose(2, 3)[..., _order()]
    cache["v"][:, (lo + a) // 64: (lo + z) // 64] = q.view(torch.float8_e4m3fn)
    cache["v_scale"][:, (lo + a) // B: (lo + z) // B] = vs


def _plain_attend(s, c):
    H, G, n, N, B = c["H"], c["G"], c["n"], c["held"], c["B"]
    k, v = _plain_values(s["cache"], B, 0, N)
    q = s["q"].float().reshape(H, G * n, D) / math.sqrt(D)
    p = torch.matmul(q, k.transpose(1, 2))
    if c["mask"]:
        nb = -(-N // B)
        at = torch.repeat_interleave(torch.arange(nb, device="cuda"), s["row_ptr"].diff(),
                                     output_size=s["col_idx"].numel())
        kept = torch.zeros(nb, nb, dtype=torch.bool, device="cuda")
        kept[at, s["col_idx"].long()] = True
        kept = kept[torch.arange(N - n, N, device="cuda") // B]
        kept = kept[:, torch.arange(N, device="cuda") // B]
        p.view(H, G, n, N).masked_fill_(~kept, -math.inf)
    most = p.amax(-1, keepdim=True)
    p.sub_(torch.where(most > -math.inf, most, 0.0)).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, v) / torch.where(total > 0, total, 1.0)
    return o.reshape(H * G, n, D).bfloat16()


# ------------------------------------------------------------------ exact

def _wide_values(cache, B, tokens):
    """Keys and values of the given tokens in 64 bits, by index."""
    held = [cache[x].double() for x in ("k", "v", "k_scale", "v_scale")]
    place = tokens % 64
    place = place // 4 % 4 * 16 + place // 16 * 4 + place % 4
    k = held[0][:, tokens] * held[2][:, tokens // B, None]
    v = held[1][:, tokens // 64, :, place].transpose(0, 1) * held[3][:, tokens // B, None]
    return k, v


def _wide_rotate(x, c, start, halves, sign):
    """x [H, n, 128] times e^(i angle), pairs as complex numbers, the angles'
    cosines and sines as the 32-bit table holds them."""
    table = _table(c).double()
    H, n, _ = x.shape
    turn = torch.ones(n, 64, dtype=torch.complex128, device="cuda")
    tok = start + torch.arange(n, device="cuda")
    video = tok < c["T"] * c["h"] * c["w"]
    tok = tok[video]
    at = (tok // (c["h"] * c["w"]), tok % (c["h"] * c["w"]) // c["w"], tok % c["w"])
    row, pair = 0, 0
    for where, size, pairs in zip(at, (c["T"], c["h"], c["w"]), PAIRS):
        e = table[row + where[:, None] * pairs + torch.arange(pairs, device="cuda")]
        turn[video, pair: pair + pairs] = torch.complex(e[..., 0], sign * e[..., 1])
        row, pair = row + size * pairs, pair + pairs
    z = x.reshape(H, n, 2, 64).transpose(2, 3) if halves else x.reshape(H, n, 64, 2)
    z = torch.view_as_real(torch.complex(z[..., 0], z[..., 1]) * turn)
    return (z.transpose(2, 3) if halves else z).reshape(H, n, D)


def _wide_blocks(x, B):
    """Values [H, n, 128] in 64 bits, n a multiple of B, as the cache holds them
    by the definition: (e4m3 values, scales [H, n / B])."""
    most = x.reshape(x.shape[0], -1, B * D).abs().amax(-1)
    k = torch.ceil(torch.log2(most.clamp(min=2.0 ** -130) / 448)) - 1
    for _ in range(2):
        k = torch.where(most > 448 * torch.exp2(k), k + 1, k)
    scale = torch.exp2(k.clamp(min=-117))
    y = x / scale.repeat_interleave(B, 1)[..., None]
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(y / step) * step, scale


def exact(c, seed):
    global own
    was, own = own, False
    s = prepare(c, seed)
    own = was
    if c["op"] in ("rope", "back"):
        return _wide_rotate(s["x"].double(), c, c["start"], c["halves"],
                            -1 if c["op"] == "back" else 1)
    cache, B = s["cache"], c["B"]
    if c["op"] == "read":
        return _wide_values(cache, B, c["start"] + torch.arange(c["n"], device="cuda"))
    if c["op"] == "write":
        return _exact_write(s, c, cache, B)
    k, v = _wide_values(cache, B, torch.arange(c["held"], device="cuda"))
    q = s["q"].double()
    out = torch.zeros_like(q)
    blocks = _block_rows(c) if c["mask"] else None
    first = c["held"] - c["n"]
    per = max(1, int(2e9 // c["held"]) // B * B)      # queries at a time: scores of 16 GB
    for head in range(q.shape[0]):
        kh, vh = k[head // c["G"]], v[head // c["G"]]
        i = 0
        while i < c["n"]:
            j = min(c["n"], i + per)
            keys = slice(None)
            if blocks is not None:       # one query block, its kept keys alone
                j = min(c["n"], ((first + i) // B + 1) * B - first)
                keep = np.repeat(blocks[(first + i) // B], B)[: c["held"]]
                keys = torch.from_numpy(np.nonzero(keep)[0]).cuda()
            if blocks is None or len(keys):
                p = torch.softmax(q[head, i:j] @ kh[keys].T / math.sqrt(D), -1)
                out[head, i:j] = p @ vh[keys]
            i = j
    return out


def _exact_write(s, c, cache, B):
    n, start = c["n"], c["held"]
    k, v = s["k"].double(), s["v"].double()
    if c["rope"]:
        k = _wide_rotate(k, c, start, False, 1)
    first, end = start // B * B, -(-(start + n) // B) * B
    if start > first:
        old_k, old_v = _wide_values(cache, B, torch.arange(first, start, device="cuda"))
        k, v = torch.cat([old_k, k], 1), torch.cat([old_v, v], 1)
    none = torch.zeros(c["H"], end - start - n, D, dtype=k.dtype, device="cuda")
    tile = torch.arange(64, device="cuda")
    place = tile // 4 % 4 * 16 + tile // 16 * 4 + tile % 4
    out = {}
    for name, x in (("k", k), ("v", v)):
        y, scale = _wide_blocks(torch.cat([x, none], 1), B)
        out[name] = cache[name].double()
        if name == "k":
            out[name][:, first: end] = y
        else:
            y = y.reshape(c["H"], -1, 64, D).transpose(2, 3)
            out[name][:, first // 64: end // 64, :, place] = y
        out[name + "_scale"] = cache[name + "_scale"].double()
        out[name + "_scale"][:, first // B: end // B] = scale
    return out
