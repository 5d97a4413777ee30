"""Plain 64-bit forms of the rotary positions, the 8-bit K/V cache and the
attention over it (test infrastructure; shares no code with the library).

Arrays are [heads, tokens, 128] float64.  The cache is modelled by the values
that it holds: a token's value is an e4m3 number times its block's power of two.
"""
import numpy as np

D = 128


# ------------------------------------------------------------- rotary

def rope_table(grid, pairs, theta=10000.0):
    """Per axis the angles [size, pairs of the axis]."""
    return [np.arange(size)[:, None] * theta ** (-np.arange(n) / max(n, 1))
            for size, n in zip(grid, pairs)]


def token_turns(grid, pairs, cos_sin, tokens):
    """(cos, sin) [tokens, 64] of every pair; cos_sin: [entries, 2], the axes one
    after the other."""
    T, h, w = grid
    cos, sin = np.ones((len(tokens), D // 2)), np.zeros((len(tokens), D // 2))
    for i, tok in enumerate(tokens):
        if tok >= T * h * w:
            continue
        at = (tok // (h * w), tok // w % h, tok % w)
        entry = 0
        pair = 0
        for size, n, pos in zip(grid, pairs, at):
            rows = cos_sin[entry + pos * n: entry + (pos + 1) * n]
            cos[i, pair: pair + n], sin[i, pair: pair + n] = rows[:, 0], rows[:, 1]
            entry += size * n
            pair += n
    return cos, sin


def rotate(x, cos, sin, halves):
    a, b = (x[..., :64], x[..., 64:]) if halves else (x[..., 0::2], x[..., 1::2])
    y = np.empty_like(x)
    p, q = a * cos - b * sin, a * sin + b * cos
    if halves:
        y[..., :64], y[..., 64:] = p, q
    else:
        y[..., 0::2], y[..., 1::2] = p, q
    return y


# -------------------------------------------------------------- cache

def e4m3(x):
    """x rounded to the nearest e4m3 number (ties to even), |x| <= 448."""
    mag = np.maximum(np.abs(x), 2.0 ** -6)
    step = 2.0 ** (np.floor(np.log2(mag)) - 3)
    return np.round(x / step) * step


def block_scale(x):
    """The scale of one block's values."""
    fin = np.abs(x[np.isfinite(x)])
    most = fin.max() if fin.size else 0.0
    e = -117
    while most > 448 * 2.0 ** e and e < 119:
        e += 1
    return 2.0 ** e


class Cache:
    """The values held by a cache of [heads, capacity] tokens."""

    def __init__(self, heads, capacity, block):
        self.block = block
        self.n = 0
        self.k = np.zeros((heads, capacity, D))
        self.v = np.zeros((heads, capacity, D))
        self.k_scale = np.full((heads, capacity // block), np.nan)   # nan: not written
        self.v_scale = np.full((heads, capacity // block), np.nan)

    def write(self, k, v, start):
        end = start + k.shape[1]
        n = max(self.n, end)
        B = self.block
        for held, scale, x in ((self.k, self.k_scale, k), (self.v, self.v_scale, v)):
            held[:, self.n:] = 0.0
            held[:, start:end] = x
            for b in range(start // B, (end - 1) // B + 1):
                for h in range(held.shape[0]):
                    y = held[h, b * B: (b + 1) * B]
                    s = block_scale(y)
                    with np.errstate(invalid="ignore"):
                        q = e4m3(np.clip(y / s, -448, 448)) * s
                    held[h, b * B: (b + 1) * B] = np.where(np.isfinite(y), q, np.nan)
                    scale[h, b] = s
        self.n = n


# ---------------------------------------------------------- attention

def attend(q, k, v, keep=None):
    """softmax(q k^T / sqrt(128)) v for [Hq, n, 128] queries over [H, N, 128] keys
    (Hq a multiple of H), `keep` a boolean [n, N].  Returns (out, spread, size,
    reach): out, and per element of it sum p |v - out|, sum p |v|, and per query the
    largest possible |q| |k| a product of one rounding can be off by, over sqrt(128)."""
    Hq, n, _ = q.shape
    H, N, _ = k.shape
    G = Hq // H
    out, spread, size = (np.zeros((Hq, n, D)) for _ in range(3))
    reach = np.zeros((Hq, n))
    for h in range(Hq):
        kh, vh = k[h // G], v[h // G]
        for i in range(n):
            idx = np.arange(N) if keep is None else np.nonzero(keep[i])[0]
            if not len(idx):
                continue
            s = kh[idx] @ q[h, i] / np.sqrt(D)
            p = np.exp(s - s.max())
            p /= p.sum()
            out[h, i] = p @ vh[idx]
            spread[h, i] = p @ np.abs(vh[idx] - out[h, i])
            size[h, i] = p @ np.abs(vh[idx])
            reach[h, i] = np.abs(q[h, i]).max() * np.abs(kh[idx]).sum(1).max() / np.sqrt(D)
    return out, spread, size, reach


def block_keep(row_ptr, col_idx, block, n_tokens, q_start, n):
    """The boolean [n, n_tokens] of a block CSR's queries q_start, q_start + 1, .."""
    keep = np.zeros((n, n_tokens), dtype=bool)
    for i in range(n):
        b = (q_start + i) // block
        for c in col_idx[row_ptr[b]: row_ptr[b + 1]]:
            if 0 <= c < len(row_ptr) - 1:
                keep[i, c * block: (c + 1) * block] = True
    return keep
