"""The residual step between blocks and its gradients against the formulas in 64 bits."""
import itertools
import math

import pytest
import torch

import paper_2605_31057_amd as L
from oracle import train as OT

pytestmark = pytest.mark.gpu
BF, HF, SF = torch.bfloat16, torch.float16, torch.float32
KIND = {"none": L.NORM_NONE, "layer": L.NORM_LAYER, "rms": L.NORM_RMS}
EPS = 1e-5


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    L.lib()


def _case(n, dim, frame, stream=SF, block=SF, params=SF, kind="layer", post="none", a=1.0,
          with_y=True, names=("gate", "scale", "shift"), seed=0):
    """(plan, inputs as a dict, gradients of r and h)."""
    g = torch.Generator().manual_seed(seed)

    def normal(rows, dtype, size=1.0, mean=0.0):
        return (torch.randn(rows, dim, generator=g) * size + mean).to(dtype).cuda()

    plan = L.ResidualNorm(dim, norm=KIND[kind], post=KIND[post], eps=EPS, residual=a,
                          frame_tokens=frame)
    t = {"x": normal(n, stream, 1.5, 0.3)}
    if with_y:
        t["y"] = normal(n, block, 0.7)
    frames = -(-n // (frame or n))
    for name in names:
        if name in ("gate", "scale", "shift"):
            t[name] = normal(frames, params, 0.4, 0.1)
        else:
            t[name] = normal(1, params, 0.3, 1.0)[0]
    return plan, t, normal(n, stream, 0.5), normal(n, block, 0.5)


def _wide(t):
    return {k: v.double().requires_grad_() for k, v in t.items()}


def _formula(w, kind, post, a, frame):
    w = dict(w)
    x, y = w.pop("x"), w.pop("y", None)
    return OT.residual_norm(x, y, kind, post, EPS, a, frame, **w)


def _near(got, want, dtype, steps, scale):
    """Within `steps` roundings of fp32 at `scale` (the size of what is added up) and one of
    the result's type."""
    room = steps * 2.0 ** -24 * scale + OT.HALF_STEP[dtype] * want.abs() + 1e-30
    over = (got.double() - want).abs() - room
    assert (over <= 0).all(), float((over / room).max())


def _sizes(t, n):
    """How large the terms of a row's results get: inputs here are a few units at most, and
    the rows' deviations are about one."""
    return 40.0


def _forward(plan, t, kind, post, a, frame, **kw):
    got = L.residual_norm(plan, **t, **kw)
    with torch.no_grad():
        r, h = _formula(_wide(t), kind, post, a, frame)
    dim = t["x"].shape[-1]
    # a sum over dim columns of fp32 numbers, by halves: at most dim roundings, and some 16
    steps = dim + 16
    if "y" not in t:
        _near(got, h, got.dtype, steps, _sizes(t, dim))
        return
    got_r, got_h = (got, None) if kind == "none" else got
    assert got_r.dtype == t["x"].dtype
    _near(got_r, r, got_r.dtype, 4 if post == "none" else steps, _sizes(t, dim))
    if got_h is not None:
        assert got_h.dtype == t["y"].dtype
        _near(got_h, h, got_h.dtype, steps, _sizes(t, dim))


def _backward(plan, t, gr, gh, kind, post, a, frame):
    """Gradients at the r that is given as x's place."""
    r = t["x"]
    params = {k: v for k, v in t.items() if k not in ("x", "y")}
    got = L.residual_norm_backward(plan, None if kind == "none" else gh, gr, r, t.get("y"), **params)
    w = _wide(t)
    n, dim = r.shape
    of = torch.arange(n, device="cuda") // (frame or n)
    dr = gr.double()
    want = {}
    if kind != "none":
        later = [k for k in ("scale", "shift", "weight", "bias") if k in w]
        h = OT.after(w["x"], kind, EPS, of, **{k: w[k] for k in later})
        into = torch.autograd.grad(h, [w["x"]] + [w[k] for k in later], gh.double())
        dr = dr + into[0]
        want.update(zip(later, into[1:]))
    want["x"] = a * dr
    if "y" in t:
        u = OT.unit(w["y"], post, EPS)
        u = u * w["post_weight"] if "post_weight" in w else u
        u = w["gate"][of] * u if "gate" in w else u
        before = ["y"] + [k for k in ("gate", "post_weight") if k in w]
        want.update(zip(before, torch.autograd.grad(u, [w[k] for k in before], dr)))
    assert set(got) == set(want)
    for name, x in got.items():
        ref = t[name]
        assert x.dtype == ref.dtype and x.shape == ref.shape
        rows = 1 if name in ("x", "y") else n if name in ("weight", "bias", "post_weight") else frame or n
        # a term of a row is off by its own sums over dim columns; terms of `rows` rows are
        # added: rows roundings of the sum of their sizes
        _near(x, want[name], x.dtype, (dim + 32) * (1 if rows == 1 else 1) + rows,
              _sizes(t, dim) * rows ** (0 if rows == 1 else 1))


SHAPES = [(1, 8, 1), (1, 1536, 1), (3, 128, 2), (17, 136, 4), (50, 512, 7), (33, 520, 0), (9, 1024, 3),
          (70, 1536, 32), (5, 2048, 5), (6, 2056, 4), (7, 5120, 3), (4, 8192, 2), (3, 8200, 2),
          (2, 16384, 1), (40, 16000, 15), (11, 72, 3), (300, 64, 100), (1000, 256, 130)]


FEW = [(1, 1536, 0), (191, 1536, 0), (192, 1536, 0), (400, 1536, 300), (1000, 520, 0), (900, 2056, 400),
       (5000, 128, 0), (9000, 64, 4100), (300, 5120, 0), (420, 9000, 0), (2000, 520, 450)]


@pytest.mark.parametrize("n,dim,frame", FEW)
@pytest.mark.parametrize("names", [("gate", "scale", "shift", "weight", "bias", "post_weight"),
                                   ("gate", "scale", "shift"), ("weight", "bias"), ("post_weight",)])
def test_few_frames(n, dim, frame, names):
    """One frame or a few of many rows, whose sums are added in two steps from some number on."""
    post = "rms" if "post_weight" in names else "none"
    plan, t, gr, gh = _case(n, dim, frame, BF, BF, post=post, names=names, seed=n)
    _backward(plan, t, gr, gh, "layer", post, 1.0, frame)


@pytest.mark.parametrize("n,dim,frame", SHAPES)
@pytest.mark.parametrize("kind", ["layer", "rms"])
def test_shapes(n, dim, frame, kind):
    if dim == 8 and kind == "layer":
        kind = "rms"
    plan, t, gr, gh = _case(n, dim, frame, kind=kind, seed=dim)
    _forward(plan, t, kind, "none", 1.0, frame)
    _backward(plan, t, gr, gh, kind, "none", 1.0, frame)


@pytest.mark.parametrize("n,dim,frame", [(200, 128, 1), (90, 512, 3), (77, 1536, 1), (2100, 640, 2),
                                         (33, 16000, 1)])
@pytest.mark.parametrize("names", [("gate", "scale", "shift"), ("gate",),
                                   ("gate", "scale", "shift", "weight", "bias", "post_weight")])
def test_frames_of_few_tokens(n, dim, frame, names):
    """A row of gate, scale and shift for each token or two: a frame is one team's, its
    gradients written without partial sums (with the weights' too, without)."""
    plan, t, gr, gh = _case(n, dim, frame, params=BF, post="rms", names=names)
    _forward(plan, t, "layer", "rms", 1.0, frame)
    _backward(plan, t, gr, gh, "layer", "rms", 1.0, frame)
    params = {k: v for k, v in t.items() if k not in ("x", "y")}
    every = L.residual_norm_backward(plan, gh, gr, t["x"], t["y"], **params)
    few = [k for k in ("x", "y", "gate", "scale", "shift") if k in t]
    got = L.residual_norm_backward(plan, gh, gr, t["x"], t["y"], wanted=few, **params)
    for k in few:      # the same sums either way, but for fused roundings
        a, b = got[k].double(), every[k].double()
        assert ((a - b).abs() <= 2.0 ** -7 * b.abs() + 2.0 ** -20).all(), k


@pytest.mark.parametrize("n,dim,frame", [(3200, 128, 16), (4001, 136, 21), (800, 1536, 4), (191, 520, 1),
                                         (192, 520, 1), (200, 9000, 1), (7000, 64, 7), (1, 1536, 0)])
@pytest.mark.parametrize("names", [("gate", "scale", "shift", "weight", "bias", "post_weight"),
                                   ("scale", "shift", "weight"), ("gate", "bias")])
def test_weights_over_many_frames(n, dim, frame, names):
    """Weights beside a row of gate, scale and shift for every few tokens: their sums over
    the frames in one step and in two, of frames that are one team's and of longer ones."""
    post = "rms" if "post_weight" in names else "none"
    plan, t, gr, gh = _case(n, dim, frame, post=post, names=names, seed=n)
    _backward(plan, t, gr, gh, "layer", post, 1.0, frame)


TYPES = [(BF, BF), (HF, HF), (SF, SF), (SF, BF), (SF, HF)]


@pytest.mark.parametrize("stream,block", TYPES)
@pytest.mark.parametrize("own_params", [False, True])
@pytest.mark.parametrize("dim", [128, 768, 2304])
def test_types(stream, block, own_params, dim):
    kw = dict(stream=stream, block=block, params=block if own_params else SF, post="rms",
              names=("gate", "scale", "shift", "weight", "bias", "post_weight"))
    plan, t, gr, gh = _case(45, dim, 20, **kw)
    _forward(plan, t, "layer", "rms", 1.0, 20)
    _backward(plan, t, gr, gh, "layer", "rms", 1.0, 20)


ALL = ("gate", "scale+shift", "weight", "bias", "post_weight")


@pytest.mark.parametrize("kind,post", itertools.product(["none", "layer", "rms"], repeat=2))
@pytest.mark.parametrize("given", range(32))
def test_every_set_of_parameters(kind, post, given):
    names = [p for i, p in enumerate(ALL) if given >> i & 1]
    if kind == "none" and set(names) & {"scale+shift", "weight", "bias"}:
        return
    if post == "none" and "post_weight" in names:
        return
    names = [q for p in names for q in p.split("+")]
    plan, t, gr, gh = _case(29, 264, 10, kind=kind, post=post, a=0.75, names=names, seed=given)
    _forward(plan, t, kind, post, 0.75, 10)
    _backward(plan, t, gr, gh, kind, post, 0.75, 10)


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("names", [(), ("weight",), ("scale", "shift"), ("weight", "bias", "scale",
                                                                          "shift")])
@pytest.mark.parametrize("stream,block", TYPES)
def test_without_a_block_before(kind, names, stream, block):
    plan, t, gr, gh = _case(37, 384, 8, stream=stream, block=block, kind=kind, with_y=False, names=names)
    _forward(plan, t, kind, "none", 1.0, 8, dtype=block)
    _backward(plan, t, gr, gh, kind, "none", 1.0, 8)


def test_strides_and_leading_dimensions():
    plan, t, gr, gh = _case(24, 256, 6)
    want = L.residual_norm(plan, **t)
    grads = L.residual_norm_backward(plan, gh, gr, want[0], t["y"], t["gate"], t["scale"], t["shift"])
    room = torch.zeros(24, 3, 256, device="cuda")
    room[:, 0], room[:, 2] = t["x"], t["y"]
    mods = torch.stack([t["gate"], t["scale"], t["shift"]], 1)      # [frames, 3, dim]
    gate, scale, shift = mods.unbind(1)
    got = L.residual_norm(plan, room[:, 0], room[:, 2], gate, scale, shift)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    got = L.residual_norm(plan, t["x"].view(4, 6, 256), t["y"].view(4, 6, 256), gate, scale, shift)
    assert got[0].shape == (4, 6, 256) and torch.equal(got[1].view(24, 256), want[1])
    again = L.residual_norm_backward(plan, gh.view(4, 6, 256), gr.view(4, 6, 256), got[0],
                                     t["y"].view(4, 6, 256), gate, scale, shift)
    for k, g in grads.items():
        assert torch.equal(again[k].reshape(g.shape), g)


def test_in_place():
    plan, t, gr, gh = _case(40, 1536, 16)
    want = L.residual_norm(plan, **t)
    params = {k: t[k] for k in ("gate", "scale", "shift")}
    x, y = t["x"].clone(), t["y"].clone()
    r, h = L.residual_norm(plan, x, y, r=x, h=y, **params)
    assert r is x and h is y and torch.equal(x, want[0]) and torch.equal(y, want[1])
    grads = L.residual_norm_backward(plan, gh, gr, want[0], t["y"], **params)
    a, b = gr.clone(), gh.clone()
    got = L.residual_norm_backward(plan, b, a, want[0], t["y"], grad_x=a, grad_y=b, **params)
    assert got["x"] is a and got["y"] is b
    assert all(torch.equal(got[k], grads[k]) for k in grads)


def test_rows_behind_the_last_stay():
    plan, t, gr, gh = _case(5, 256, 2)
    params = {k: t[k] for k in ("gate", "scale", "shift")}
    room = torch.full((4, 8, 256), 7.0, device="cuda")
    L.residual_norm(plan, t["x"], t["y"], r=room[0, :5], h=room[1, :5], **params)
    L.residual_norm_backward(plan, gh, gr, t["x"], t["y"], grad_x=room[2, :5], grad_y=room[3, :5],
                             **params)
    assert (room[:, 5:] == 7).all() and (room[:, :5] != 7).any()


def test_a_row_that_is_not_finite_stays_alone():
    for bad in (math.nan, math.inf):
        plan, t, gr, gh = _case(40, 128, 40)
        params = {k: t[k] for k in ("gate", "scale", "shift")}
        want = L.residual_norm(plan, **t)
        grads = L.residual_norm_backward(plan, gh, gr, t["x"], t["y"], **params)
        t["x"][13, 5] = bad
        got = L.residual_norm(plan, **t)
        again = L.residual_norm_backward(plan, gh, gr, t["x"], t["y"], **params)
        rest = torch.arange(40, device="cuda") != 13
        for a, b in ((got[0], want[0]), (got[1], want[1]), (again["x"], grads["x"]),
                     (again["y"], grads["y"])):
            assert torch.equal(a[rest], b[rest])
        assert torch.isnan(got[1][13]).any()


def test_constant_rows_and_large_means():
    """Rows of one value (variance zero: eps alone), and a mean 4096 times the deviation:
    the deviations are taken before they are squared."""
    plan, t, _, _ = _case(4, 512, 4)
    t["x"][:] = 3.0
    t["y"][:] = 0.0
    r, h = L.residual_norm(plan, **t)
    assert torch.equal(h, t["shift"].expand(4, 512))
    plan, t, _, _ = _case(4, 512, 4, names=())
    t["x"] = t["x"] + 4096.0
    _, h = L.residual_norm(plan, **t)
    with torch.no_grad():
        want = _formula(_wide(t), "layer", "none", 1.0, 4)[1]
    # r is rounded to fp32 after the addition of y: half a step of 4096 is 2^-12, and so the
    # mean is off by as much (its sum of 512 by their roundings, 512 * 2^-12 * 2^-1 / 512)
    assert ((h.double() - want).abs() <= 4 * 2.0 ** -12 * (1 + want.abs())).all()


def test_the_same_every_time():
    plan, t, gr, gh = _case(3000, 264, 700, names=("gate", "scale", "shift", "weight"), post="none")
    params = {k: v for k, v in t.items() if k not in ("x", "y")}
    first = L.residual_norm_backward(plan, gh, gr, t["x"], t["y"], **params)
    for _ in range(3):
        again = L.residual_norm_backward(plan, gh, gr, t["x"], t["y"], **params)
        assert all(torch.equal(first[k], again[k]) for k in first)


def test_rows_past_32_bits():
    """270,000 rows of 8,192 columns, 2.2e9 elements a tensor: rows at both ends and between as
    in calls of their own, and the sums over all rows of whole numbers, which are exact."""
    n, dim = 270000, 8192
    g = torch.Generator(device="cuda").manual_seed(5)
    x, y = (torch.randn(n, dim, dtype=BF, device="cuda", generator=g) for _ in range(2))
    gh = torch.randint(-2, 3, (n, dim), dtype=torch.int8, device="cuda", generator=g).to(BF)
    params = {k: torch.randn(1, dim, device="cuda", generator=g) for k in ("gate", "scale", "shift")}
    plan = L.ResidualNorm(dim, eps=EPS)
    r, h = L.residual_norm(plan, x, y, **params)
    grads = L.residual_norm_backward(plan, gh, None, r, y, **params)
    for at in (slice(0, 3), slice(134000, 134005), slice(n - 7, n)):
        few = L.residual_norm(plan, x[at], y[at], **params)
        assert torch.equal(r[at], few[0]) and torch.equal(h[at], few[1])
        few = L.residual_norm_backward(plan, gh[at], None, r[at], y[at], **params)
        assert torch.equal(grads["x"][at], few["x"]) and torch.equal(grads["y"][at], few["y"])
    total = torch.zeros(dim, dtype=torch.float64, device="cuda")
    for i in range(0, n, 10000):
        total += gh[i: i + 10000].double().sum(0)
    assert torch.equal(grads["shift"][0].double(), total)


def test_wanted():
    plan, t, gr, gh = _case(60, 256, 16)
    params = {k: t[k] for k in ("gate", "scale", "shift")}
    every = L.residual_norm_backward(plan, gh, gr, t["x"], t["y"], **params)
    for wanted in (["x"], ["y"], ["gate"], ["scale", "y"]):
        got = L.residual_norm_backward(plan, gh, gr, t["x"], t["y"], wanted=wanted, **params)
        assert set(got) == set(wanted) and all(torch.equal(got[k], every[k]) for k in wanted)
    assert torch.equal(
        L.residual_norm_backward(plan, gh, torch.zeros_like(gr), t["x"], t["y"], **params)["x"],
        L.residual_norm_backward(plan, gh, None, t["x"], t["y"], **params)["x"])
    with pytest.raises(ValueError):
        L.residual_norm_backward(plan, gh, gr, t["x"], t["y"], wanted=["weight"], **params)


# ------------------------------------------------------------------ autograd

@pytest.mark.parametrize("kind,post,with_y", [("layer", "none", True), ("rms", "rms", True),
                                              ("none", "layer", True), ("layer", "none", False)])
def test_autograd(kind, post, with_y):
    names = ["gate"] * with_y + (["scale", "shift", "weight"] if kind != "none" else [])
    plan, t, gr, gh = _case(50, 264, 20, kind=kind, post=post, with_y=with_y, names=names)
    params = {k: v for k, v in t.items() if k not in ("x", "y")}
    leaves = {k: v.clone().requires_grad_() for k, v in t.items()}
    got = L.residual_norm(plan, **leaves)
    want = L.residual_norm(plan, **t)
    if kind == "none" or not with_y:
        assert torch.equal(got, want)
        got.backward(gr if kind == "none" else gh)
        at = want if kind == "none" else t["x"]
        grads = L.residual_norm_backward(plan, None if kind == "none" else gh,
                                         gr if kind == "none" else None, at, t.get("y"), **params)
    else:
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        torch.autograd.backward(got, (gr, gh))
        grads = L.residual_norm_backward(plan, gh, gr, want[0], t["y"], **params)
    for k, leaf in leaves.items():
        assert torch.equal(leaf.grad, grads[k]), k


def test_autograd_of_one_output_alone():
    plan, t, gr, gh = _case(30, 128, 10)
    params = {k: t[k] for k in ("gate", "scale", "shift")}
    r, h = L.residual_norm(plan, **t)
    for which in (0, 1):
        leaves = {k: v.clone().requires_grad_() for k, v in t.items()}
        out = L.residual_norm(plan, **leaves)[which]
        out.backward((gr, gh)[which])
        zero = torch.zeros_like(gr)
        want = L.residual_norm_backward(plan, zero if which == 0 else gh, gr if which == 0 else None,
                                        r, t["y"], **params)
        for k, leaf in leaves.items():
            assert torch.equal(leaf.grad, want[k]), k
    x = t["x"].clone().requires_grad_()
    sum(o.sum() for o in L.residual_norm(plan, x, t["y"], **params)).backward()    # expanded scalars
    ones = torch.ones_like(gr)
    assert torch.equal(x.grad, L.residual_norm_backward(plan, ones, ones, r, t["y"], **params)["x"])
    with pytest.raises(ValueError):
        L.residual_norm(plan, x, t["y"], r=torch.empty_like(t["x"]), **params)


def test_captured():
    plan, t, gr, gh = _case(500, 512, 130, names=("gate", "scale", "shift", "weight"))
    params = {k: v for k, v in t.items() if k not in ("x", "y")}

    def step():
        leaves = {k: v.detach().requires_grad_() for k, v in t.items()}
        r, h = L.residual_norm(plan, **leaves)
        grads = torch.autograd.grad((r, h), list(leaves.values()), (gr, gh))
        return r.detach(), h.detach(), *grads

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
        _, fresh, _, _ = _case(500, 512, 130, names=("gate", "scale", "shift", "weight"), seed=50 + s)
        for k in t:
            t[k].copy_(fresh[k])
        for x in got:
            x.fill_(0.0)
        graph.replay()
        torch.cuda.synchronize()
        r, h = L.residual_norm(plan, **fresh)
        fp = {k: fresh[k] for k in params}
        want = L.residual_norm_backward(plan, gh, gr, r, fresh["y"], **fp)
        for x, w in zip(got, (r, h, *(want[k] for k in t))):
            assert torch.equal(x, w)


def test_on_another_stream():
    plan, t, gr, gh = _case(2000, 512, 700)
    params = {k: t[k] for k in ("gate", "scale", "shift")}
    want = L.residual_norm(plan, **t)
    grads = L.residual_norm_backward(plan, gh, gr, want[0], t["y"], **params)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    r, h = L.residual_norm(plan, **t, stream=s)
    got = L.residual_norm_backward(plan, gh, gr, r, t["y"], **params, stream=s)
    torch.cuda.synchronize()
    assert torch.equal(r, want[0]) and torch.equal(h, want[1])
    assert all(torch.equal(got[k], grads[k]) for k in grads)
