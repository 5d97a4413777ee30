"""The C ABI of attention's gradients and of the residual step, as far as it needs no GPU:
refusals before any launch with the documented status, sizes of workspaces, and the plain
64-bit forms themselves against automatic differentiation."""
import ctypes

import pytest
import torch

import paper_2605_31057_amd as L
from oracle import train as OT
from tests import whole_cases as WHOLE

ref = ctypes.byref
PTR = 0x100000


def _tensor(heads=2, n=300, d=128, data=PTR, sh=None, st=None):
    return L._Tensor(data, heads, n, d, n * d if sh is None else sh, d if st is None else st)


def _mask(n=300, block=128, nq=None, nk=None, rows=8 * PTR, cols=9 * PTR):
    nb = -(-n // block) if block > 0 else 0
    return L.BlockMask(n, block, nb if nq is None else nq, nb if nk is None else nk, rows, cols)


BAD_MASKS = [
    (dict(rows=None), L.EINVAL), (dict(cols=None), L.EINVAL), (dict(n=301), L.EINVAL),
    (dict(nq=4), L.EINVAL), (dict(nk=2), L.EINVAL), (dict(block=32), L.EUNSUPPORTED),
    (dict(block=256), L.EUNSUPPORTED),
]
BAD_TENSORS = [
    (dict(n=299), L.EINVAL), (dict(heads=1), L.EINVAL), (dict(data=None), L.EINVAL),
    (dict(d=64), L.EUNSUPPORTED), (dict(data=PTR + 8), L.EUNSUPPORTED), (dict(st=132), L.EUNSUPPORTED),
    (dict(sh=-128), L.EUNSUPPORTED), (dict(st=2 ** 26), L.EUNSUPPORTED),
]


def test_attention_lse_refusals():
    f = L.lib().lvsa_attention_lse
    q, k, v, o = (_tensor(data=i * PTR) for i in range(1, 5))
    lse = 6 * PTR

    def call(q=q, k=k, v=v, mask=None, o=o, lse=lse):
        return f(*(t and ref(t) for t in (q, k, v, mask, o)), lse, None)

    for kw in (dict(q=None), dict(k=None), dict(v=None), dict(o=None), dict(lse=None),
               dict(q=_tensor(n=0)), dict(o=_tensor(data=2 * PTR))):
        assert call(**kw) == L.EINVAL, kw
    assert call(lse=lse + 2) == L.EUNSUPPORTED
    for kw, st in BAD_MASKS:
        assert call(mask=_mask(**kw)) == st, kw
    assert call(mask=_mask(n=8001 * 64, block=64)) == L.EUNSUPPORTED
    for kw, st in BAD_TENSORS:
        if kw.get("data", 0) is not None and "data" not in kw:
            kw = dict(kw, data=2 * PTR)
        assert call(k=_tensor(**kw)) == st, kw


def test_attention_backward_refusals():
    lib = L.lib()
    names = ("go", "q", "k", "v", "out", "gq", "gk", "gv")
    good = {x: _tensor(data=(i + 1) * PTR) for i, x in enumerate(names)}
    lse, work = 20 * PTR, 30 * PTR
    need = ctypes.c_int64()
    assert lib.lvsa_attention_backward_workspace(ref(good["q"]), None, ref(need)) == L.OK
    assert need.value >= 2 * 2 * 300 * 4

    def call(mask=None, lse=lse, work=work, size=1 << 40, **kw):
        t = dict(good, **kw)
        go, q, k, v, out, gq, gk, gv = (t[x] and ref(t[x]) for x in names)
        return lib.lvsa_attention_backward(go, q, k, v, out, lse, mask and ref(mask), gq, gk, gv,
                                           work, size, None)

    for x in names:
        assert call(**{x: None}) == L.EINVAL, x
    assert call(lse=None) == L.EINVAL
    assert call(lse=lse + 1) == L.EUNSUPPORTED
    assert call(work=None) == L.EINVAL
    assert call(size=need.value - 1) == L.EINVAL
    assert call(work=work + 8) == L.EUNSUPPORTED
    for kw, st in BAD_MASKS:
        assert call(mask=_mask(**kw)) == st, kw
        if "n" not in kw:
            assert lib.lvsa_attention_backward_workspace(ref(good["q"]), ref(_mask(**kw)),
                                                         ref(need)) == st, kw
    for kw, st in BAD_TENSORS:
        for x in ("go", "k", "v", "out"):
            t = _tensor(**dict(dict(data=(names.index(x) + 1) * PTR), **kw))
            if "st" in kw and kw["st"] > 1000 and x == "out":
                continue        # out is read with 64-bit offsets
            assert call(**{x: t}) == st, (kw, x)
    # rows of a gradient that share elements, gradients in an input's or in each other's place
    for x in ("gq", "gk", "gv"):
        at = (names.index(x) + 1) * PTR
        assert call(**{x: _tensor(data=at, st=64)}) == L.EINVAL
        assert call(**{x: _tensor(data=at, sh=0)}) == L.EINVAL
        for y in ("go", "q", "k", "v", "out"):
            assert call(**{x: good[y]}) == L.EINVAL
        assert call(**{x: _tensor(data=lse)}) == L.EINVAL
    assert call(gq=good["gk"]) == L.EINVAL
    assert call(gk=good["gv"]) == L.EINVAL
    assert call(gv=good["gq"]) == L.EINVAL


def test_attention_backward_sizes():
    f = L.lib().lvsa_attention_backward_workspace
    need = ctypes.c_int64()
    assert f(None, None, ref(need)) == L.EINVAL
    assert f(ref(_tensor()), None, None) == L.EINVAL
    assert f(ref(_tensor(n=0)), None, ref(need)) == L.EINVAL
    assert f(ref(_tensor(heads=0)), None, ref(need)) == L.EINVAL
    assert f(ref(_tensor(heads=1 << 14, n=1 << 15)), None, ref(need)) == L.EUNSUPPORTED
    assert f(ref(_tensor(n=8001 * 64)), ref(_mask(n=8001 * 64, block=64)), ref(need)) == L.EUNSUPPORTED
    # a mask without rows is every block, in blocks of any size
    sizes = []
    for mask in (None, _mask(block=64, rows=None, cols=None), _mask(block=128, rows=None, cols=None)):
        assert f(ref(_tensor()), mask and ref(mask), ref(need)) == L.OK
        sizes.append(need.value)
    assert len(set(sizes)) == 1
    # parts of items stay within a few hundred megabytes however long the call is
    for H, n in ((1, 128), (1, 188760), (40, 188760), (12, 32760), (500, 1000), (1, 2 ** 28)):
        for mask in (None, _mask(n=n) if n < 8000 * 128 else None):
            assert f(ref(_tensor(heads=H, n=n)), mask and ref(mask), ref(need)) == L.OK
            assert need.value <= 8 * H * n + (600 << 20), (H, n, need.value)


# ------------------------------------------------------------- residual step

def _rows(data=PTR, n=10, stride=256):
    return L._Rows(data, n, stride)


def _plan(dim=256, frame=4, norm=1, post=0, eps=1e-6, a=1.0, st=2, bt=2, pt=2, gate=50 * PTR,
          scale=51 * PTR, shift=52 * PTR, strides=(256, 256, 256), weight=None, bias=None,
          post_weight=None):
    return L._ResidualNorm(dim, frame, norm, post, eps, a, st, bt, pt, gate, scale, shift, *strides,
                           weight, bias, post_weight)


BAD_PLANS = [
    (dict(dim=0), L.EINVAL), (dict(frame=-1), L.EINVAL), (dict(norm=3), L.EINVAL),
    (dict(norm=-1), L.EINVAL), (dict(post=3), L.EINVAL), (dict(st=3), L.EINVAL),
    (dict(bt=-1), L.EINVAL), (dict(pt=7), L.EINVAL), (dict(eps=-1.0), L.EINVAL),
    (dict(eps=float("nan")), L.EINVAL), (dict(eps=float("inf")), L.EINVAL),
    (dict(scale=None), L.EINVAL), (dict(shift=None), L.EINVAL),
    (dict(norm=0), L.EINVAL),                       # a scale without a norm
    (dict(post_weight=53 * PTR), L.EINVAL),         # of no norm
    (dict(strides=(-8, 256, 256)), L.EINVAL),
    (dict(dim=252), L.EUNSUPPORTED), (dict(dim=16392), L.EUNSUPPORTED),
    (dict(st=0, bt=1), L.EUNSUPPORTED), (dict(st=0, bt=2), L.EUNSUPPORTED),
    (dict(st=1, bt=0), L.EUNSUPPORTED), (dict(gate=PTR + 8), L.EUNSUPPORTED),
    (dict(weight=PTR + 4), L.EUNSUPPORTED), (dict(strides=(256, 252, 256)), L.EUNSUPPORTED),
]
X, Y, R, H, GR, GH, GX, GY = (i * PTR for i in range(1, 9))


def test_residual_norm_refusals():
    f = L.lib().lvsa_residual_norm_forward

    def call(p=_plan(), x=_rows(X), y=_rows(Y), r=_rows(R), h=_rows(H)):
        return f(*(t and ref(t) for t in (p, x, y, r, h)), None)

    for kw, st in BAD_PLANS:
        assert call(p=_plan(**kw)) == st, kw
    for x in ("p", "x", "r", "h"):
        assert call(**{x: None}) == L.EINVAL, x
    for x, at in (("x", X), ("y", Y), ("r", R), ("h", H)):
        for t, st in ((_rows(None), L.EINVAL), (_rows(at, n=0 if x == "x" else 9), L.EINVAL),
                      (_rows(at, stride=-256), L.EINVAL), (_rows(at + 8), L.EUNSUPPORTED),
                      (_rows(at, stride=260), L.EUNSUPPORTED)):
            assert call(**{x: t}) == st, (x, st)
    for x, at in (("r", R), ("h", H)):
        assert call(**{x: _rows(at, stride=128)}) == L.EINVAL      # rows that share elements
    # in place: r in x's, h in y's rows, the same strides; nothing else
    assert call(r=_rows(X, stride=512)) == L.EINVAL
    assert call(h=_rows(Y, stride=512)) == L.EINVAL
    assert call(r=_rows(Y)) == L.EINVAL
    assert call(h=_rows(X)) == L.EINVAL
    assert call(h=_rows(R)) == L.EINVAL
    # without y: no r, gate, norm of y, factor
    plain = dict(gate=None)
    assert call(p=_plan(**plain), y=None) == L.EINVAL
    assert call(y=None, r=None) == L.EINVAL
    assert call(p=_plan(post=1, **plain), y=None, r=None) == L.EINVAL
    assert call(p=_plan(a=0.5, **plain), y=None, r=None) == L.EINVAL
    assert call(p=_plan(norm=0, scale=None, shift=None, **plain), y=None, r=None, h=None) == L.EINVAL
    # no norm, no h
    assert call(p=_plan(norm=0, scale=None, shift=None)) == L.EINVAL
    # work-items past a launch
    assert call(p=_plan(frame=1), x=_rows(X, n=2 ** 30), y=_rows(Y, n=2 ** 30), r=_rows(R, n=2 ** 30),
                h=_rows(H, n=2 ** 30)) == L.EUNSUPPORTED


def _grads(x=GX, y=GY, n=10, stride=256, **kw):
    g = L._NormGrads()
    g.x, g.y = L._Rows(x, n, stride), L._Rows(y, n, stride)
    for k, v in kw.items():
        setattr(g, k, v)
    return g


def test_residual_norm_backward_refusals():
    lib = L.lib()
    work = 40 * PTR

    def call(p=_plan(), gh=_rows(GH), gr=_rows(GR), r=_rows(R), y=_rows(Y), g=_grads(), work=work,
             size=1 << 40):
        return lib.lvsa_residual_norm_backward(*(t and ref(t) for t in (p, gh, gr, r, y, g)), work,
                                               size, None)

    for kw, st in BAD_PLANS:
        assert call(p=_plan(**kw)) == st, kw
    for x in ("p", "gh", "r", "y", "g"):
        assert call(**{x: None}) == L.EINVAL, x
    for x, at in (("gh", GH), ("gr", GR), ("r", R), ("y", Y)):
        for t, st in ((_rows(None), L.EINVAL), (_rows(at, n=0 if x == "r" else 9), L.EINVAL),
                      (_rows(at, stride=-256), L.EINVAL), (_rows(at + 8), L.EUNSUPPORTED),
                      (_rows(at, stride=260), L.EUNSUPPORTED)):
            assert call(**{x: t}) == st, (x, st)
    for g in (_grads(stride=128), _grads(n=9), _grads(x=R), _grads(x=Y), _grads(x=GH), _grads(y=GR),
              _grads(y=R), _grads(y=Y), _grads(y=GX)):
        assert call(g=g) == L.EINVAL
    assert call(g=_grads(x=GX + 8)) == L.EUNSUPPORTED
    # gradients of what the step does not have, or in a parameter's place
    for name in ("weight", "bias", "post_weight"):
        assert call(g=_grads(**{name: 60 * PTR})) == L.EINVAL
    assert call(g=_grads(gate=50 * PTR)) == L.EINVAL
    assert call(g=_grads(gate=60 * PTR + 8)) == L.EUNSUPPORTED
    # a workspace where there are sums
    need = ctypes.c_int64()
    g = _grads(gate=60 * PTR, scale=61 * PTR)
    assert lib.lvsa_residual_norm_workspace(ref(_plan()), 10, ref(g), ref(need)) == L.OK
    assert need.value > 0
    assert call(g=g, size=need.value - 1) == L.EINVAL
    assert call(g=g, work=None) == L.EINVAL
    assert call(g=g, work=work + 8) == L.EUNSUPPORTED
    assert lib.lvsa_residual_norm_workspace(ref(_plan()), 10, ref(_grads()), ref(need)) == L.OK
    assert need.value == 0
    assert lib.lvsa_residual_norm_workspace(ref(_plan()), 0, ref(g), ref(need)) == L.EINVAL
    assert lib.lvsa_residual_norm_workspace(ref(_plan()), 10, None, ref(need)) == L.EINVAL
    assert lib.lvsa_residual_norm_workspace(ref(_plan()), 10, ref(g), None) == L.EINVAL
    assert call(p=_plan(frame=1, dim=64), gh=_rows(GH, n=2 ** 23), gr=_rows(GR, n=2 ** 23),
                r=_rows(R, n=2 ** 23), y=_rows(Y, n=2 ** 23), g=_grads(n=2 ** 23)) == L.EUNSUPPORTED
    # no gradient of y without y
    assert call(p=_plan(gate=None), y=None) == L.EINVAL


# ------------------------------------------------------------------- binding

def test_binding_refusals():
    for kw in (dict(dim=2 ** 32 + 8), dict(dim=-8), dict(dim=256, frame_tokens=2 ** 31),
               dict(dim=256, norm=2 ** 32)):
        with pytest.raises(L.LvsaError):
            L.ResidualNorm(**kw)
    x = torch.zeros(256).as_strided((2 ** 31, 256), (0, 1))
    with pytest.raises(L.LvsaError):
        L._channels(x, 256, -1)
    for t in (torch.zeros(4, 128), torch.zeros(256, 4).t(), torch.zeros(4, 3, 512)[:, ::2, :256],
              torch.zeros(4, 3, 512), torch.zeros(512), torch.zeros(())):
        with pytest.raises(ValueError):
            L._channels(t, 256, -1)
    with pytest.raises(ValueError):
        L._channels(torch.zeros(4, 256), 256, 0)


def test_no_rows_are_refused_as_by_the_library():
    L._fast()
    empty = torch.zeros(0, 256)
    for frame in (0, 10):
        plan = L.ResidualNorm(256, frame_tokens=frame)
        with pytest.raises(L.LvsaError) as e:
            L._norm_plan(plan, 0, torch.float32, torch.float32, (None, empty, empty) + (None,) * 3, -1)
        assert e.value.status == L.EINVAL


# ----------------------------------------------------------------- the oracle

@pytest.mark.parametrize("masked", [False, True])
def test_attention_of_the_oracle(masked):
    g = torch.Generator().manual_seed(1)
    q, k, v, grad = (torch.randn(2, 40, 16, generator=g, dtype=torch.double) for _ in range(4))
    kept = OT.kept_tokens([[1, 0, 1], [1, 1, 0], [0, 1, 1]], 16, 40).bool() if masked else \
        torch.ones(40, 40, dtype=torch.bool)
    want = OT.attention(q, k, v, grad, kept)
    leaves = [t.requires_grad_() for t in (q, k, v)]
    out = torch.nn.functional.scaled_dot_product_attention(*leaves, attn_mask=kept)
    assert torch.allclose(out, want["out"], rtol=0, atol=1e-12)
    for name, x in zip(("dq", "dk", "dv"), torch.autograd.grad(out, leaves, grad)):
        assert torch.allclose(x, want[name], rtol=0, atol=1e-11)


@pytest.mark.parametrize("n", [64, 1000])
def test_bounds_see_a_missing_key(n):
    """One key too few passes the bound of a few elements at least, and the bound in the
    2-norm by far."""
    g = torch.Generator().manual_seed(2)
    q, k, v, grad = (torch.randn(1, n, 128, generator=g, dtype=torch.double) for _ in range(4))
    kept = torch.ones(n, n, dtype=torch.bool)
    want = OT.attention(q, k, v, grad, kept)
    kept[:, n - 1] = False
    other = OT.attention(q, k, v, grad, kept)
    for name in ("out", "lse", "dq", "dk", "dv"):
        off = (other[name] - want[name]).abs()
        assert (off > want["bound"][name]).any(), name
        if name != "lse":
            assert off.norm() > 2 * OT.NORM * want[name].norm(), name


@pytest.mark.parametrize("n", [1, 64, 100, 128, 200, 256, 400, 1000])
@pytest.mark.parametrize("block", [0, 64, 128])
def test_workspaces_of_many_short_heads(block, n):
    """Parts are reserved only where an item can be split, and then for as many as the launch's
    workgroup slots call for: beyond the rows' statistics, bitmaps and lists a few hundred
    megabytes at any number of heads, and next to nothing for heads of one tile."""
    need = ctypes.c_int64()
    for heads in (1, 64, 200, 256, 300, 512, 513, 640, 1000, 4096, 65536, 2 ** 20):
        if heads * n >= 2 ** 29:
            continue
        mask = ref(_mask(n=n, block=block)) if block else None
        assert L.lib().lvsa_attention_backward_workspace(ref(_tensor(heads=heads, n=n)), mask,
                                                         ref(need)) == L.OK
        parts = need.value - 8 * heads * n
        assert parts <= (256 << 20), (heads, parts)
        if n <= 128:
            assert parts <= 64 * 1024, (heads, parts)


@pytest.mark.parametrize("mask", [None, _mask(n=1, block=64), _mask(n=1, block=128),
                                  _mask(n=1, block=64, rows=None, cols=None)])
def test_more_heads_than_a_launch_holds(mask):
    """Two items a head of few tokens, a workgroup of 256 each: 2^23 heads would pass 2^32
    work-items, which both entry points refuse before any launch."""
    lib, need = L.lib(), ctypes.c_int64()
    m = mask and ref(mask)
    size = lib.lvsa_attention_backward_workspace
    assert size(ref(_tensor(heads=2 ** 23 - 1, n=1)), m, ref(need)) == L.OK
    for heads in (2 ** 23, 2 ** 24 - 1, 2 ** 29 - 1):
        assert size(ref(_tensor(heads=heads, n=1)), m, ref(need)) == L.EUNSUPPORTED, heads
    t = [_tensor(heads=2 ** 23, n=1, data=(i + 1) * PTR) for i in range(8)]
    assert lib.lvsa_attention_backward(*map(ref, t[:5]), 20 * PTR, m, *map(ref, t[5:]), 30 * PTR,
                                       1 << 60, None) == L.EUNSUPPORTED


# --------------------------------------- the residual step in whole numbers

@pytest.mark.parametrize("kind", ["none", "layer", "rms"])
@pytest.mark.parametrize("post", ["none", "layer", "rms"])
@pytest.mark.parametrize("n,dim,frame", [(1, 8, 0), (7, 24, 3), (12, 16, 1), (9, 40, 0)])
def test_whole_numbers_are_the_formulas(n, dim, frame, kind, post):
    """whole_gradients against automatic differentiation of the step, eps 0."""
    names = [k for k in WHOLE.ALL if (kind != "none" or k in ("gate", "post_weight")) and
             (post != "none" or k != "post_weight")]
    for with_y in (True, False) if kind != "none" and post == "none" else (True,):
        use = [k for k in names if with_y or k not in ("gate", "post_weight")]
        t, gr, gh = OT.whole_step(n, dim, frame, post, use, with_y, seed=n)
        got = OT.whole_gradients(t, gr, gh, kind, 0.5, frame)
        w = {k: x.clone().requires_grad_() for k, x in t.items()}
        of = torch.arange(n) // (frame or n)
        e = gr
        if kind != "none":
            h = OT.after(w["x"], kind, 0.0, of, *(w.get(k) for k in ("scale", "shift", "weight", "bias")))
            later = [k for k in ("x", "scale", "shift", "weight", "bias") if k in w]
            want = dict(zip(later, torch.autograd.grad(h, [w[k] for k in later], gh)))
            e = gr + want["x"]
        else:
            want = {}
        want["x"] = 0.5 * e
        if with_y:
            u = OT.unit(w["y"], post, 0.0) * w.get("post_weight", 1.0)
            u = u * w["gate"][of] if "gate" in w else u
            before = [k for k in ("y", "gate", "post_weight") if k in w]
            want.update(zip(before, torch.autograd.grad(u, [w[k] for k in before], e)))
        assert set(got) == set(want) == set(t)
        for k in got:
            assert (got[k] - want[k]).abs().max() <= 1e-9, k
            assert (got[k] * 2 == (got[k] * 2).round()).all() and got[k].abs().max() < 2 ** 20, k


@pytest.mark.parametrize("n,dim,frame", [s for s in WHOLE.SHAPES if s[0] * s[1] <= 2 ** 21])
@pytest.mark.parametrize("names", WHOLE.NAMES)
def test_whole_numbers_see_a_missing_row(n, dim, frame, names):
    """A row left out, or a stretch of them, changes every gradient, whole numbers that fp32
    holds: no bound hides it."""
    post = "rms" if "post_weight" in names else "none"
    t, gr, gh = OT.whole_step(n, dim, frame, post, names, seed=n)
    want = OT.whole_gradients(t, gr, gh, "layer", 1.0, frame)
    for first, more in ((0, 0), (n // 2, 0), (n - 1, 0), (n // 3, n // 32)):
        left = slice(first, first + more + 1)
        less = [x.clone() for x in (gr, gh)]
        for x in less:
            x[left] = 0.0
        other = OT.whole_gradients(t, *less, "layer", 1.0, frame)
        for k in want:
            assert (other[k] - want[k]).abs().max() >= 1, (k, left)


@pytest.mark.parametrize("dim", WHOLE.WIDTHS)
@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("post", ["none", "layer", "rms"])
def test_the_bound_of_a_row_sees_a_missing_column(dim, kind, post):
    """A column that is left out of a row's means, of any row where its values are not near
    zero, passes the bound on the row; and the plain results are the formula's."""
    t, gr, gh = OT.row_case(dim, post)
    t, gr, gh = {k: x.double() for k, x in t.items()}, gr.double(), gh.double()
    want = OT.row_results(t, gr, gh, kind, post, 1e-5, 25)
    plain = OT.residual_norm(t["x"], t["y"], kind, post, 1e-5, 1.0, 25,
                             **{k: x for k, x in t.items() if k not in ("x", "y")})
    w = {k: t[k].clone().requires_grad_() for k in ("x", "y")}
    of = torch.arange(60) // 25
    h = OT.after(w["x"], kind, 1e-5, of, t["scale"], t["shift"], t["weight"])
    e = gr + torch.autograd.grad(h, w["x"], gh)[0]
    u = OT.unit(w["y"], post, 1e-5) * t.get("post_weight", 1.0) * t["gate"][of]
    for k, x in zip(("r", "h", "x", "y"), (*plain, e, torch.autograd.grad(u, w["y"], e)[0])):
        assert (want[k] - x).abs().max() <= 1e-10, k
    for left in (0, dim // 2 + 1, dim - 1):
        other = OT.row_results(t, gr, gh, kind, post, 1e-5, 25, left)
        for k in want:
            if k == "r" and post == "none":
                continue
            off = (other[k] - want[k]).norm(dim=-1) / want[k].norm(dim=-1)
            assert off.max() > OT.ROW_NORM[k], (k, left, float(off.max()))
