"""Attention's log-sum-exps and gradients against the formulas in 64 bits, element by
element within the bounds that the kernels' roundings give (oracle/train.py)."""
import ctypes
import math

import numpy as np
import pytest
import torch

import paper_2605_31057_amd as L
from oracle import train as OT

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    L.lib()


def _inputs(H, n, seed=0, nhd=False, size=1.0):
    g = torch.Generator().manual_seed(seed)
    made = []
    for wide in (size, 1.0, 1.0, 0.5):
        x = (torch.randn((n, H, 128) if nhd else (H, n, 128), generator=g) * wide).to(BF).cuda()
        made.append(x.transpose(0, 1) if nhd else x)
    return made


def _mask(kept, n, block):
    kept = np.asarray(kept)
    rows = torch.from_numpy(np.concatenate([[0], kept.sum(1).cumsum()]).astype(np.int32)).cuda()
    cols = torch.from_numpy(np.nonzero(kept)[1].astype(np.int32)).cuda()
    if not cols.numel():
        cols = torch.zeros(1, dtype=torch.int32, device="cuda")
    return L.csr_mask(rows, cols, n, block)


def _kept(n, block, share=0.5, seed=1, empty=()):
    nb = -(-n // block)
    kept = np.random.default_rng(seed).random((nb, nb)) < share
    for r in empty:
        kept[r % nb] = False
    return kept


def _pass(q, k, v, grad, mask):
    out, lse = L.attention_lse(q, k, v, mask)
    dq, dk, dv = L.attention_backward(grad, q, k, v, out, lse, mask)
    return {"out": out, "lse": lse, "dq": dq, "dk": dk, "dv": dv}


def _check(got, q, k, v, grad, kept=None, wide=False):
    """`wide`: scores of many units, where a row's few terms cancel; element bounds alone.
    So too where a row has fewer than 8 keys: with a single one e = p (do v' - delta) is 0 and
    what is left of it is rounding, of any size relative to it."""
    n = q.shape[1]
    kept = torch.ones(n, n, dtype=torch.bool) if kept is None else kept
    want = OT.attention(*(x.double().contiguous() for x in (q, k, v, grad)), kept.cuda())
    for name, x in got.items():
        w, bound = want[name], want["bound"][name]
        fine = torch.isfinite(w)
        assert torch.equal(torch.isfinite(x), fine) and torch.equal(x[~fine].double(), w[~fine])
        over = (x.double() - w).abs()[fine] - bound[fine]
        assert (over <= 1e-30).all(), (name, float(over.max()), float(bound.max()))
        if name != "lse" and not wide and kept.sum(1)[kept.any(1)].min() >= 8:
            off = (x.double() - w)[fine].norm()
            assert off <= OT.NORM * w[fine].norm(), (name, float(off / w[fine].norm()))


SIZES = [(1, 1), (2, 2), (1, 63), (2, 64), (1, 65), (3, 127), (1, 128), (2, 129), (1, 191),
         (2, 257), (5, 500), (1, 1000)]


@pytest.mark.parametrize("H,n", SIZES)
def test_dense(H, n):
    x = _inputs(H, n, seed=n)
    _check(_pass(*x, None), *x)


@pytest.mark.parametrize("block", [64, 128])
@pytest.mark.parametrize("H,n", SIZES)
def test_masked(block, H, n):
    kept = _kept(n, block, seed=n, empty=(2,) if n > 3 * block else ())
    kept[:, -1] |= kept.sum(1) == 0 if n <= 3 * block else False
    x = _inputs(H, n, seed=n, nhd=n % 2 == 1)
    _check(_pass(*x, _mask(kept, n, block)), *x, OT.kept_tokens(kept, block, n))


@pytest.mark.parametrize("block", [64, 128])
def test_rows_and_columns_without_blocks(block):
    n = 7 * block + 5
    kept = _kept(n, block, 0.4, seed=3, empty=(0, 3, 7))
    kept[:, 2] = False
    kept[:, 7] = False
    x = _inputs(2, n)
    got = _pass(*x, _mask(kept, n, block))
    _check(got, *x, OT.kept_tokens(kept, block, n))
    assert (got["dk"][:, 2 * block: 3 * block] == 0).all()
    assert (got["dv"][:, 7 * block:] == 0).all()
    assert (got["dq"][:, 3 * block: 4 * block] == 0).all()
    assert (got["lse"][:, 3 * block: 4 * block] == -math.inf).all()


@pytest.mark.parametrize("block", [64, 128])
@pytest.mark.parametrize("blocks", [31, 32, 33, 63, 64, 65, 97])
def test_bitmaps_of_whole_words_and_a_block_more(blocks, block):
    n = blocks * block - 3
    kept = _kept(n, block, 0.3, seed=blocks, empty=(4,)) & ~(np.arange(blocks) == 31)[None]
    kept[:, -1] = True
    x = _inputs(1, n, seed=blocks)
    _check(_pass(*x, _mask(kept, n, block)), *x, OT.kept_tokens(kept, block, n))


@pytest.mark.parametrize("block", [64, 128])
def test_an_empty_mask(block):
    n = 3 * block - 1
    x = _inputs(2, n)
    got = _pass(*x, _mask(np.zeros((3, 3), bool), n, block))
    assert all((got[name] == 0).all() for name in ("out", "dq", "dk", "dv"))


@pytest.mark.parametrize("block", [64, 128])
def test_blocks_that_are_not_kept_never_reach(block):
    """NaN and infinities in a key block (a query block) stay out of the gradients of those
    that it has no pair with."""
    n = 6 * block
    kept = _kept(n, block, 0.5, seed=8)
    kept[:, 0] = True
    kept[1, 3], kept[4, 3] = False, False
    x = _inputs(2, n)
    clean = _pass(*x, _mask(kept, n, block))
    bad = [t.clone() for t in x]
    bad[1][:, 3 * block: 4 * block] = math.nan
    bad[2][:, 3 * block: 4 * block] = math.inf
    got = _pass(*bad, _mask(kept, n, block))
    for row in np.nonzero(~kept[:, 3])[0]:
        at = slice(row * block, (row + 1) * block)
        for name in ("out", "lse", "dq"):
            assert torch.equal(got[name][:, at], clean[name][:, at])
    # key blocks see it through the queries of rows that keep block 3 alone
    for col in range(6):
        if not (kept[:, 3] & kept[:, col]).any():
            at = slice(col * block, (col + 1) * block)
            assert torch.equal(got["dk"][:, at], clean["dk"][:, at])
            assert torch.equal(got["dv"][:, at], clean["dv"][:, at])
    bad = [t.clone() for t in x]
    bad[0][:, 4 * block: 5 * block] = math.nan
    bad[3][:, 4 * block: 5 * block] = -math.inf
    got = _pass(*bad, _mask(kept, n, block))
    for col in np.nonzero(~kept[4])[0]:
        at = slice(col * block, (col + 1) * block)
        assert torch.equal(got["dk"][:, at], clean["dk"][:, at])
        assert torch.equal(got["dv"][:, at], clean["dv"][:, at])


@pytest.mark.parametrize("size", [4.0, 30.0, 300.0])
def test_wide_scores(size):
    n = 300
    x = _inputs(2, n, seed=5, size=size)
    _check(_pass(*x, None), *x, wide=True)


def test_scores_far_from_zero():
    """Every score near -700 or +700 in the natural logarithm: exponentials of the scores
    alone would not be finite, nor those of keys past the last one."""
    for sign in (-1.0, 1.0):
        x = _inputs(1, 70, seed=6)
        x[0][:] = sign * 8.0
        x[1][:] = (8.0 + 0.25 * torch.randn(1, 70, 128, generator=torch.Generator().manual_seed(1))
                   ).to(BF).cuda()
        _check(_pass(*x, None), *x, wide=True)


def test_out_is_attentions():
    """out is bit for bit that of the call without lse; whole and split tiles."""
    for H, n, block in ((1, 1000, 128), (12, 5460, 128), (12, 5460, 64), (40, 4680, 128)):
        q, k, v, _ = _inputs(H, n, seed=H)
        kept = _kept(n, block, 0.6, seed=n)
        m = _mask(kept, n, block)
        assert torch.equal(L.attention_lse(q, k, v, m)[0], L.attention(q, k, v, m))
        every = L.BlockMask(n, block, -(-n // block), -(-n // block), None, None)
        assert torch.equal(L.attention_lse(q, k, v, every)[0],
                           L.dense_attention(q, k, v, block=block))


def test_long_rows_against_blocks_of_the_formula():
    """12 heads of 4,000 tokens under a mask, whole tiles of every kernel: sampled rows and
    keys."""
    H, n, block = 12, 4000, 128
    kept = _kept(n, block, 0.4, seed=2, empty=(5,))
    x = _inputs(H, n, seed=9)
    got = _pass(*x, _mask(kept, n, block))
    for h in (0, 11):
        _check({k: t[h: h + 1] for k, t in got.items()}, *(t[h: h + 1] for t in x),
               OT.kept_tokens(kept, block, n))


@pytest.mark.parametrize("block", [64, 128])
def test_key_blocks_that_every_query_keeps_beside_ones_that_few_do(block):
    """Two key blocks kept by every query block, the others by their own and the next: a
    tile's walk is several times another's, split and whole items in one call; and one head
    beside many."""
    n = 40 * block - 7
    kept = np.eye(40, dtype=bool) | np.eye(40, k=1, dtype=bool)
    kept[:, [3, 30]] = True
    kept[17] = True
    for H in (1, 24):
        x = _inputs(H, n, seed=H)
        got = _pass(*x, _mask(kept, n, block))
        for h in (0, H - 1):
            _check({k: t[h: h + 1] for k, t in got.items()}, *(t[h: h + 1] for t in x),
                   OT.kept_tokens(kept, block, n))


@pytest.mark.parametrize("block", [0, 64, 128])
@pytest.mark.parametrize("more", [0, 1])
@pytest.mark.parametrize("tiles", [4, 16, 32])
def test_as_many_items_as_fit_at_once(tiles, more, block):
    """Tiles of queries and of keys as many as the device takes at once (two workgroups a
    compute unit), whole or with room for parts, and of a token more."""
    slots = 2 * torch.cuda.get_device_properties(0).multi_processor_count
    for H in {max(1, slots // (2 * tiles)), max(1, slots // (5 * tiles))}:
        n = 128 * tiles + more
        kept = _kept(n, block, 0.3, seed=tiles) | np.eye(-(-n // block), dtype=bool) if block else None
        x = _inputs(H, n, seed=tiles + more)
        got = _pass(*x, _mask(kept, n, block) if block else None)
        for h in {0, H - 1}:
            _check({k: t[h: h + 1] for k, t in got.items()}, *(t[h: h + 1] for t in x),
                   OT.kept_tokens(kept, block, n) if block else None)


@pytest.mark.parametrize("tiles", [23, 24, 25])
def test_a_few_items_more_than_fit_at_once(tiles):
    """Every key, as many heads as make a few tiles more than the device takes at once."""
    H = torch.cuda.get_device_properties(0).multi_processor_count // tiles + 1
    n = 128 * tiles - 5
    x = _inputs(H, n, seed=tiles)
    got = _pass(*x, None)
    for h in (0, H - 1):
        _check({k: t[h: h + 1] for k, t in got.items()}, *(t[h: h + 1] for t in x))


def test_masks_of_thousands_of_blocks():
    """8,000 blocks of 64 (the most), each row with a few: queries and keys at both ends and
    between against the formula over the blocks that they meet."""
    block, nb = 64, 8000
    n = nb * block - 5
    kept = np.zeros((nb, nb), bool)
    at = np.arange(nb)
    kept[at, at] = True
    kept[at, (at * 7 + 3) % nb] = True
    kept[::500, 4321] = True
    x = _inputs(1, n, seed=3)
    got = _pass(*x, _mask(kept, n, block))
    for b in (0, 1, 4321, 4500, nb - 1):
        # the tokens that meet block b's queries or keys, or theirs
        rows = np.nonzero(kept[:, b])[0]
        blocks = np.unique(np.concatenate([[b], rows, np.nonzero(kept[rows].any(0))[0],
                                           np.nonzero(kept[b])[0]]))
        tok = np.concatenate([np.arange(c * block, min(n, (c + 1) * block)) for c in blocks])
        sub = [t[:, tok].contiguous() for t in x]
        pairs = torch.from_numpy(kept[np.ix_(tok // block, tok // block)])
        want = OT.attention(*(t.double() for t in sub), pairs.cuda())
        mine = torch.from_numpy(np.nonzero(tok // block == b)[0]).cuda()
        for name in ("out", "lse", "dq", "dk", "dv"):
            # queries of b see all their keys here, and keys of b all their queries
            g = got[name][:, torch.from_numpy(tok).cuda()][:, mine]
            assert ((g.double() - want[name][:, mine]).abs() <= want["bound"][name][:, mine] + 1e-30
                    ).all(), (b, name)


def test_every_key_past_8000_blocks():
    """One head of 8,001 blocks of 64 and some, every key: log-sum-exps and dq of sampled
    queries, dk and dv of sampled keys (with the call's own log-sum-exps and output, which the
    first part checks)."""
    n = 8001 * 64 + 21
    q, k, v, grad = _inputs(1, n, seed=4)
    every = L.BlockMask(n, 64, -(-n // 64), -(-n // 64), None, None)
    out, lse = L.attention_lse(q, k, v, every)
    dq, dk, dv = L.attention_backward(grad, q, k, v, out, lse, every)
    at = torch.tensor([0, 1, 63, 64, 300000, n - 22, n - 21, n - 1], device="cuda")
    wide = [t[0].double() for t in (q, k, v, grad)]
    s = wide[0][at] @ wide[1].T / math.sqrt(128)
    want = torch.logsumexp(s, -1)
    assert ((lse[0, at].double() - want).abs() <= 1e-5 * (1 + want.abs())).all()
    p = torch.exp(s - want[:, None])
    o = p @ wide[2]
    # out and gradients: roundings that do not know of each other, in the 2-norm
    assert (out[0, at].double() - o).norm() <= OT.NORM * o.norm()
    e = p * (wide[3][at] @ wide[2].T - (wide[3][at] * o).sum(-1, keepdim=True))
    w = e @ wide[1] / math.sqrt(128)
    assert (dq[0, at].double() - w).norm() <= OT.NORM * w.norm()
    p = torch.exp(wide[0] @ wide[1][at].T / math.sqrt(128) - lse[0].double()[:, None])
    e = p * (wide[3] @ wide[2][at].T - (wide[3] * out[0].double()).sum(-1, keepdim=True))
    for got, w in ((dv, p.T @ wide[3]), (dk, e.T @ wide[0] / math.sqrt(128))):
        assert (got[0, at].double() - w).norm() <= OT.NORM * w.norm()


def test_the_same_every_time():
    x = _inputs(3, 900, seed=4)
    m = _mask(_kept(900, 64, 0.5), 900, 64)
    first = _pass(*x, m)
    for _ in range(3):
        again = _pass(*x, m)
        assert all(torch.equal(first[k], again[k]) for k in first)


def test_gradients_into_given_tensors_leave_the_rest():
    H, n = 2, 150
    x = _inputs(H, n)
    want = _pass(*x, None)
    out, lse = L.attention_lse(*x[:3])
    room = [torch.full((n + 3, H, 128), 7.0, dtype=BF, device="cuda") for _ in range(3)]
    grads = [r[1: n + 1].transpose(0, 1) for r in room]
    got = L.attention_backward(x[3], *x[:3], out, lse, grads=grads)
    for name, g, r in zip(("dq", "dk", "dv"), got, room):
        assert torch.equal(g, want[name])
        assert (r[0] == 7).all() and (r[n + 1:] == 7).all()


def test_against_differences():
    """The gradients of sum(out * grad) against central differences of the library's own
    output, in a random direction, q, k and v together."""
    x = _inputs(1, 200, seed=12)
    got = _pass(*x, None)
    g = torch.Generator().manual_seed(3)
    step = [torch.randn(1, 200, 128, generator=g).cuda() for _ in range(3)]

    def loss(t):
        q, k, v = (a.double() + t * b.double() for a, b in zip(x, step))
        p = torch.softmax(q @ k.transpose(1, 2) / math.sqrt(128), -1)
        return float(((p @ v) * x[3].double()).sum())

    slope = (loss(1e-4) - loss(-1e-4)) / 2e-4
    mine = sum(float((got[n].double() * s.double()).sum()) for n, s in zip(("dq", "dk", "dv"), step))
    want = OT.attention(*(t.double() for t in x), torch.ones(200, 200, dtype=torch.bool).cuda())
    room = sum(float((want["bound"][n] * s.abs().double()).sum())
               for n, s in zip(("dq", "dk", "dv"), step))
    assert abs(mine - slope) <= room


# ------------------------------------------------------------------ autograd

def _leaves(x):
    return [t.detach().clone().requires_grad_() for t in x[:3]]


@pytest.mark.parametrize("block", [64, 128])
def test_autograd(block):
    n = 500
    x = _inputs(3, n, seed=2)
    m = _mask(_kept(n, block, 0.5), n, block)
    want = _pass(*x, m)
    q, k, v = _leaves(x)
    out = L.attention(q, k, v, m)
    assert torch.equal(out, want["out"])
    out.backward(x[3])
    for t, name in ((q, "dq"), (k, "dk"), (v, "dv")):
        assert torch.equal(t.grad, want[name])
    q, k, v = _leaves(x)
    out = L.dense_attention(q, k, v, block=block)
    assert torch.equal(out, L.dense_attention(*x[:3], block=block))
    out.backward(x[3])
    # the walk of keys does not depend on the forward pass's block
    o, lse = L.attention_lse(*x[:3], L.BlockMask(n, block, -(-n // block), -(-n // block), None, None))
    for t, w in zip((q, k, v), L.attention_backward(x[3], *x[:3], o, lse)):
        assert torch.equal(t.grad, w)


def test_autograd_of_some_and_of_expanded_gradients():
    x = _inputs(2, 100)
    ones = torch.ones(2, 100, 128, dtype=BF, device="cuda")
    want = _pass(*x[:3], ones, None)
    q, k, v = (t.clone() for t in x[:3])
    v.requires_grad_()
    L.dense_attention(q, k, v).backward(ones[:1, :1].expand(2, 100, 128))
    assert torch.equal(v.grad, want["dv"]) and q.grad is None
    with torch.no_grad():
        assert not L.dense_attention(q, k, v).requires_grad
    # one tensor three times: its gradient is the sum
    t = x[0].clone().requires_grad_()
    L.dense_attention(t, t, t).backward(ones)
    want = _pass(x[0], x[0], x[0], ones, None)
    total = sum(want[n].double() for n in ("dq", "dk", "dv"))
    size = sum(want[n].double().abs() for n in ("dq", "dk", "dv"))
    assert ((t.grad.double() - total).abs() <= 2 * 2.0 ** -8 * size).all()


def test_autograd_into_a_given_output():
    x = _inputs(2, 100)
    q, k, v = _leaves(x)
    out = torch.empty_like(x[0])
    got = L.dense_attention(q, k, v, out=out)
    assert got.data_ptr() == out.data_ptr()
    got.backward(x[3])
    assert torch.equal(q.grad, _pass(*x, None)["dq"])


def test_a_mask_that_changes_before_the_backward_pass_is_noticed():
    T, P, B = 8, 40, 64
    nb = -(-T * P // B)
    row_ptr = torch.empty(nb + 1, dtype=torch.int32, device="cuda")
    col_idx = torch.empty(nb * nb, dtype=torch.int32, device="cuda")
    p = L.Params(window=1, tper=3)
    x = _inputs(1, T * P)
    m = L.build_mask_device(T, P, B, 0, row_ptr, col_idx, p)
    q, k, v = _leaves(x)
    out = L.attention(q, k, v, m)
    L.build_mask_device(T, P, B, 1, row_ptr, col_idx, p)
    with pytest.raises(RuntimeError):
        out.backward(x[3])


def test_a_mask_of_a_handle_lives_as_long_as_its_view():
    T, P, B = 8, 40, 64
    x = _inputs(1, T * P)

    def mask():
        return L.build_mask(T, P, B, 0, L.Params(window=1, tper=3)).upload().device_mask()

    q, k, v = _leaves(x)
    out = L.attention(q, k, v, mask())
    junk = [torch.full((64,), -1, dtype=torch.int32, device="cuda") for _ in range(50)]
    out.backward(x[3])
    want = _pass(*x, mask())
    assert torch.equal(out, want["out"]) and torch.equal(k.grad, want["dk"])
    del junk


def test_second_derivatives_are_refused():
    q, k, v = _leaves(_inputs(1, 64))
    out = L.dense_attention(q, k, v)
    grad, = torch.autograd.grad(out.float().pow(2).sum(), q, create_graph=True)
    with pytest.raises(RuntimeError):
        grad.float().sum().backward()


# ------------------------------------------------------------------ streams, graphs

def test_on_another_stream():
    x = _inputs(2, 700)
    m = _mask(_kept(700, 128, 0.6), 700, 128)
    want = _pass(*x, m)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    out, lse = L.attention_lse(*x[:3], m, stream=s)
    grads = L.attention_backward(x[3], *x[:3], out, lse, m, stream=s)
    q, k, v = _leaves(x)
    torch.cuda.synchronize()
    y = L.attention(q, k, v, m, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    y.backward(x[3])
    torch.cuda.synchronize()
    for g, t, name in zip(grads, (q, k, v), ("dq", "dk", "dv")):
        assert torch.equal(g, want[name]) and torch.equal(t.grad, want[name])


def test_two_at_once():
    a, b = _inputs(2, 900, seed=1), _inputs(2, 900, seed=2)
    m = _mask(_kept(900, 64, 0.6), 900, 64)
    want = _pass(*a, m), _pass(*b, m)
    torch.cuda.synchronize()
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    got = []
    for s, x in zip(streams, (a, b)):
        with torch.cuda.stream(s):
            got.append(_pass(*x, m))
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        assert all(torch.equal(g[k], w[k]) for k in w)


def test_captured():
    """A training pass captured into a graph, replayed with new inputs among eager ones."""
    n = 600
    m = _mask(_kept(n, 128, 0.6), n, 128)
    x = _inputs(2, n)

    def step():
        q, k, v = (t.detach().requires_grad_() for t in x[:3])
        out = L.attention(q, k, v, m)
        return out.detach(), *torch.autograd.grad(out, (q, k, v), x[3])

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(3):
            step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for s in range(4):
        fresh = _inputs(2, n, seed=30 + s)
        for t, f in zip(x, fresh):
            t.copy_(f)
        for t in got:
            t.fill_(0.0)
        graph.replay()
        torch.cuda.synchronize()
        want = _pass(*fresh, m)
        for t, name in zip(got, ("out", "dq", "dk", "dv")):
            assert torch.equal(t, want[name])


def test_shared_heads_and_slices_of_a_projection():
    """Keys and values that all heads share (expanded), queries as a slice of a fused
    projection: the shared tensors' gradients are the sums over the heads."""
    H, n = 4, 300
    g = torch.Generator().manual_seed(5)
    qkv = torch.randn(n, H + 2, 128, generator=g).to(BF).cuda()
    grad = torch.randn(H, n, 128, generator=g).to(BF).cuda()
    leaf = qkv.clone().requires_grad_()
    q = leaf[:, :H].transpose(0, 1)
    k, v = (leaf[:, H + i: H + i + 1].transpose(0, 1).expand(H, n, 128) for i in range(2))
    L.dense_attention(q, k, v).backward(grad)
    full = [qkv[:, :H].transpose(0, 1).contiguous(),
            *(qkv[:, H + i].expand(H, n, 128).contiguous() for i in range(2))]
    want = _pass(*full, grad, None)
    assert torch.equal(leaf.grad[:, :H].transpose(0, 1), want["dq"])
    for i, name in ((0, "dk"), (1, "dv")):
        total = want[name].double().sum(0)
        # autograd adds four bf16 gradients, a rounding each time
        room = 4 * 2.0 ** -8 * want[name].double().abs().sum(0)
        assert ((leaf.grad[:, H + i].double() - total).abs() <= room).all()


def test_heads_past_32_bits():
    """90 heads of 190,000 tokens, 2.19e9 elements a tensor, each block of keys kept by its own
    queries: heads at both ends and between as in calls of their own."""
    H, n, block = 90, 190000, 128
    m = _mask(np.eye(-(-n // block), dtype=bool), n, block)
    g = torch.Generator(device="cuda").manual_seed(5)
    x = [torch.randn(H, n, 128, dtype=BF, device="cuda", generator=g) for _ in range(4)]
    got = _pass(*x, m)
    for h in (0, 45, H - 1):
        q, k, v, grad = (t[h: h + 1] for t in x)
        out, lse = L.attention_lse(q, k, v, m)
        # rows' sums may be in other parts: a rounding of out, and fp32 ones
        assert ((got["out"][h].double() - out[0].double()).abs()
                <= 2.0 ** -8 * out[0].double().abs() + 1e-5).all()
        assert ((got["lse"][h] - lse[0]).abs() <= 1e-5 * (1 + lse[0].abs())).all()
        own = L.attention_backward(grad, q, k, v, got["out"][h: h + 1],
                                   got["lse"][h: h + 1].contiguous(), m)
        for name, t in zip(("dq", "dk", "dv"), own):
            assert torch.equal(got[name][h], t[0]), (h, name)


def test_from_two_threads():
    import threading
    m = _mask(_kept(700, 64, 0.6), 700, 64)
    x = [_inputs(2, 700, seed=s) for s in range(2)]
    want = [_pass(*t, m) for t in x]
    torch.cuda.synchronize()
    got = [None, None]

    def work(i):
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(5):
                got[i] = _pass(*x[i], m)
            torch.cuda.current_stream().synchronize()

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    for g, w in zip(got, want):
        assert all(torch.equal(g[k], w[k]) for k in w)


def test_a_training_step_of_a_block():
    """Norm and modulation, rotary positions, attention under an LVSA mask, gate and
    residual, the next norm, as a block of a video transformer has them: gradients of the
    input and of every parameter against the same step in 64 bits."""
    T, h, w, H = 6, 8, 10, 3
    P, n, dim = h * w, T * h * w, H * 128
    g = torch.Generator().manual_seed(11)

    def normal(*shape, size=1.0):
        return torch.randn(*shape, generator=g) * size

    params = {"x": normal(n, dim), "mod": normal(T, 5, dim, size=0.3),
              "wqkv": normal(dim, 3 * dim, size=dim ** -0.5), "wo": normal(dim, dim, size=dim ** -0.5),
              "qk": 1 + normal(2, 128, size=0.1)}
    grad = normal(n, dim), normal(n, dim)
    csr = L.build_mask(T, P, 64, 3, L.Params(window=1, tper=3))
    row_ptr, col_idx = csr.arrays()
    nb = len(row_ptr) - 1
    kept = np.zeros((nb, nb), bool)
    for r in range(nb):
        kept[r, col_idx[row_ptr[r]: row_ptr[r + 1]]] = True
    csr.upload()

    # the library's step: products in bf16, the stream in 32 bits
    leaf = {k: v.cuda().requires_grad_() for k, v in params.items()}
    shift, scale, gate, scale2, shift2 = leaf["mod"].unbind(1)
    first = L.ResidualNorm(dim, frame_tokens=P)
    heads = L.ResidualNorm(128, norm=L.NORM_RMS)
    rope = L.Rope(T, h, w)
    a = L.residual_norm(first, leaf["x"], scale=scale, shift=shift, dtype=BF)
    q, k, v = (a @ leaf["wqkv"].to(BF)).view(n, 3, H, 128).unbind(1)
    q, k = (L.residual_norm(heads, t.contiguous(), weight=leaf["qk"][i]) for i, t in ((0, q), (1, k)))
    q, k = (L.rope(t.transpose(0, 1), rope) for t in (q, k))
    o = L.attention(q, k, v.transpose(0, 1), csr.device_mask())
    y = o.transpose(0, 1).reshape(n, dim) @ leaf["wo"].to(BF)
    r, out = L.residual_norm(first, leaf["x"], y.float(), gate=gate, scale=scale2, shift=shift2)
    torch.autograd.backward((r, out), [t.cuda() for t in grad])

    # in 64 bits
    wide = {k: v.double().cuda().requires_grad_() for k, v in params.items()}
    wide["wqkv"].data.copy_(params["wqkv"].to(BF).double())
    wide["wo"].data.copy_(params["wo"].to(BF).double())
    shift, scale, gate, scale2, shift2 = wide["mod"].unbind(1)
    of = torch.arange(n, device="cuda") // P
    a = OT.after(wide["x"], "layer", 1e-6, of, scale=scale, shift=shift)
    q, k, v = (a @ wide["wqkv"]).view(n, 3, H, 128).unbind(1)
    eye = torch.eye(128, device="cuda")[:, None].expand(128, n, 128).contiguous()
    turn = L.rope(eye, rope).double().permute(1, 0, 2)          # [token, element, rotated]
    q, k = (OT.unit(t, "rms", 1e-6) * wide["qk"][i] for i, t in ((0, q), (1, k)))
    q, k = (torch.bmm(t, turn).transpose(0, 1) for t in (q, k))
    s = q @ k.transpose(1, 2) / math.sqrt(128)
    s = s.masked_fill(~OT.kept_tokens(kept, 64, n).cuda(), -math.inf)
    y = (torch.softmax(s, -1) @ v.transpose(0, 1)).transpose(0, 1).reshape(n, dim) @ wide["wo"]
    r2, out2 = OT.residual_norm(wide["x"], y, "layer", "none", 1e-6, 1.0, P, gate=gate, scale=scale2,
                                shift=shift2)
    torch.autograd.backward((r2, out2), [t.double().cuda() for t in grad])
    # a dozen tensors on the way are rounded to bf16, 2^-8 / sqrt(3) of their values in the
    # mean each, independently: below 12 ** 0.5 * 2^-8 / 3 ** 0.5 = 2^-7 together; twice that
    for got, want in ((r, r2), (out, out2), *((leaf[k].grad, wide[k].grad) for k in leaf)):
        off = (got.detach().double() - want.detach()).norm() / want.detach().norm()
        assert off <= 2.0 ** -6, float(off)


@pytest.mark.parametrize("block", [0, 64, 128])
@pytest.mark.parametrize("H,n", [(1, 1), (2, 5), (2, 70), (1, 127), (3, 150), (1, 321)])
@pytest.mark.parametrize("stride", [8, 64, 120])
def test_inputs_whose_rows_share_elements(stride, H, n, block):
    """Rows a stride of less than 128 apart, each input in turn and all together: the same
    as their contiguous copies, where rows past the last are not a tail of the last."""
    kept = _kept(n, block, 0.6, seed=n) | np.eye(-(-n // block), dtype=bool) if block else None
    m = _mask(kept, n, block) if block else None
    g = torch.Generator().manual_seed(n)

    def shared(size=1.0):
        flat = (torch.randn(H, (n - 1) * stride + 128, generator=g) * size).to(BF).cuda()
        return flat.as_strided((H, n, 128), (flat.stride(0), stride, 1))

    apart = _inputs(H, n, seed=n)
    # queries whose scores, without a log-sum-exp, would have no finite exponential
    whole = [shared(30.0), *(shared() for _ in range(3))]
    out, lse = L.attention_lse(*apart[:3], m)
    for which in ((0,), (1,), (2,), (3,), (0, 1, 2, 3)):
        x = [whole[i] if i in which else apart[i] for i in range(4)]
        alone = [t.contiguous() for t in x]
        want = _pass(*alone, m)
        got = {k: torch.empty_like(alone[0]) for k in ("out", "dq", "dk", "dv")}
        _, got["lse"] = L.attention_lse(*x[:3], m, out=got["out"])
        L.attention_backward(x[3], *x[:3], got["out"], got["lse"], m,
                             grads=[got[k] for k in ("dq", "dk", "dv")])
        assert all(torch.equal(got[k], want[k]) for k in want), which
    # an output read back through such rows, and gradients as autograd hands them on
    want = L.attention_backward(apart[3], *apart[:3], whole[0].contiguous(), lse, m)
    got = L.attention_backward(apart[3], *apart[:3], whole[0], lse, m)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    q, k, v = _leaves(apart)
    y = L.attention(q, k, v, m) if block else L.dense_attention(q, k, v)
    y.backward(whole[3])
    want = L.attention_backward(whole[3].contiguous(), *apart[:3], out, lse, m)
    assert all(torch.equal(t.grad, w) for t, w in zip((q, k, v), want))


def test_a_single_token_of_any_stride():
    """Through the library itself, as the binding gives a single token the stride of a
    contiguous one."""
    ref, f = ctypes.byref, L._fast()
    x = _inputs(1, 1, seed=3)
    want = _pass(*x, None)
    grads = [torch.empty_like(x[0]) for _ in range(3)]
    need = ctypes.c_int64()
    for st in (8, 64, 128, 4096):
        t = [L._Tensor(i.data_ptr(), 1, 1, 128, 128, st) for i in (x[3], *x[:3], want["out"], *grads)]
        assert f.back_workspace(ref(t[1]), None, ref(need)) == L.OK
        work = torch.empty(need.value, dtype=torch.uint8, device="cuda")
        assert f.back(*(ref(i) for i in t[:5]), want["lse"].data_ptr(), None, *(ref(i) for i in t[5:]),
                      work.data_ptr(), need.value, f.stream(f.device())) == L.OK
        for g, name in zip(grads, ("dq", "dk", "dv")):
            assert torch.equal(g, want[name]), (st, name)


@pytest.mark.parametrize("block", [64, 128])
@pytest.mark.parametrize("H,n", [(640, 64), (1, 100), (500, 128), (4096, 17), (256, 256), (512, 250),
                                 (520, 256), (530, 256), (120, 385), (700, 640)])
def test_heads_of_few_tokens_under_a_mask(H, n, block):
    """Calls of so many heads or so few tokens that no item is in parts, and ones on both
    sides of that; every head kept blocks of all sorts, a column that all rows keep."""
    kept = _kept(n, block, 0.4, seed=n + H)
    kept[:, -1] = True
    x = _inputs(H, n, seed=H)
    got = _pass(*x, _mask(kept, n, block))
    for h in {0, H // 2, H - 1}:
        _check({k: t[h: h + 1] for k, t in got.items()}, *(t[h: h + 1] for t in x),
               OT.kept_tokens(kept, block, n))


@pytest.mark.parametrize("block", [0, 64, 128])
def test_against_differences_of_the_librarys_output(block):
    """sum(out * grad) of the library's own forward pass, half a step of h to both sides of the
    inputs along the signs of the gradients, against the gradients: inputs are multiples of h
    below 4, so bf16 holds both ends.  What the difference has beyond the slope, h not being
    small, is the formula's in 64 bits at the same ends."""
    H, n, h = 2, 200, 2.0 ** -3
    kept = _kept(n, block, 0.6, seed=4) | np.eye(-(-n // block), dtype=bool) if block else None
    mask = _mask(kept, n, block) if block else None
    pairs = (OT.kept_tokens(kept, block, n) if block else torch.ones(n, n, dtype=torch.bool)).cuda()
    x = _inputs(H, n, seed=21)
    x[:3] = [((t.float() / h).round() * h).clamp(-3.5, 3.5).to(BF) for t in x[:3]]
    got = _pass(*x, mask)
    names = ("dq", "dk", "dv")
    step = [torch.where(got[k] > 0, 0.5, -0.5).float() * h for k in names]
    ends = [[(t.float() + way * s) for t, s in zip(x, step)] for way in (1, -1)]
    held = [[t.to(BF) for t in end] for end in ends]
    assert all(torch.equal(a.float(), b) for e, f in zip(held, ends) for a, b in zip(e, f))
    grad = x[3].double()
    values, plain, room = [], [], 0.0
    for end in held:
        out = L.attention(*end, mask) if block else L.dense_attention(*end)
        want = OT.attention(*(t.double() for t in end), grad, pairs)["out"]
        values.append(float((out.double() * grad).sum()))
        plain.append(float((want * grad).sum()))
        room += OT.NORM * float(want.norm() * grad.norm())
    want = OT.attention(*(t.double() for t in x), pairs)
    along = sum(float((want[k] * s.double()).sum()) for k, s in zip(names, step)) * 2
    mine = sum(float((got[k].double() * s.double()).sum()) for k, s in zip(names, step)) * 2
    room += sum(OT.NORM * float(want[k].norm() * s.double().norm()) for k, s in zip(names, step)) * 2
    off = values[0] - values[1] - (plain[0] - plain[1] - along) - mine
    assert abs(off) <= room and room <= 0.2 * mine, (off, room, mine)
