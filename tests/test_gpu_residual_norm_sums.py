"""The residual step's gradients where every number on the way is whole and fp32 holds it
(oracle/train.py, whole_step): each is exact, so a row that is left out or counted twice shows
at any number of rows."""
import functools

import pytest
import torch

import paper_2605_31057_amd as L
from oracle import train as OT
from tests import whole_cases as WHOLE

pytestmark = pytest.mark.gpu
BF, HF, SF = torch.bfloat16, torch.float16, torch.float32
KIND = {"none": L.NORM_NONE, "layer": L.NORM_LAYER, "rms": L.NORM_RMS}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    L.lib()


@functools.lru_cache(maxsize=1)
def _case(n, dim, frame, post, names, with_y, seed):
    wide, gr, gh = OT.whole_step(n, dim, frame, post, names, with_y, seed)
    return {k: x.cuda() for k, x in wide.items()}, gr.cuda(), gh.cuda()


def _exact(n, dim, frame, names, kind="layer", post="none", a=1.0, with_y=True, stream=SF, block=SF,
           params=SF, wanted=None, seed=0):
    wide, gr, gh = _case(n, dim, frame, post, tuple(names), with_y, seed)
    want = OT.whole_gradients(wide, gr, gh, kind, a, frame)
    types = {"x": stream, "y": block}
    t = {k: x.to(types.get(k, params)) for k, x in wide.items()}
    plan = L.ResidualNorm(dim, norm=KIND[kind], post=KIND[post], eps=0.0, residual=a, frame_tokens=frame)
    rest = {k: x for k, x in t.items() if k not in ("x", "y")}
    got = L.residual_norm_backward(plan, None if kind == "none" else gh.to(block), gr.to(stream), t["x"],
                                   t.get("y"), wanted=wanted, **rest)
    assert set(got) == set(want if wanted is None else wanted)
    for k, x in got.items():
        # one rounding, of a number that fp32 holds, to the result's type
        assert torch.equal(x, want[k].to(torch.float32).to(x.dtype)), (k, float(
            (x.double() - want[k]).abs().max()))


@pytest.mark.parametrize("n,dim,frame", WHOLE.SHAPES)
@pytest.mark.parametrize("names", WHOLE.NAMES)
def test_sums(n, dim, frame, names):
    post = "rms" if "post_weight" in names else "none"
    _exact(n, dim, frame, names, post=post, seed=n)
    # each alone, beside none of the others
    for k in names:
        _exact(n, dim, frame, names, post=post, wanted=[k], seed=n)


@pytest.mark.parametrize("stream,block", [(BF, BF), (HF, HF), (SF, BF), (SF, HF)])
@pytest.mark.parametrize("n,dim,frame", [(2000, 128, 700), (300, 1536, 7), (90, 5120, 0), (260, 512, 1),
                                         (40, 9000, 13), (500, 256, 0)])
def test_sums_of_types(n, dim, frame, stream, block):
    _exact(n, dim, frame, WHOLE.ALL, post="rms", stream=stream, block=block, params=block, seed=dim)


@pytest.mark.parametrize("kind", ["none", "layer", "rms"])
@pytest.mark.parametrize("post", ["none", "layer", "rms"])
@pytest.mark.parametrize("n,dim,frame", [(900, 264, 0), (900, 264, 250), (300, 2048, 3)])
def test_sums_of_norms(n, dim, frame, kind, post):
    names = [k for k in WHOLE.ALL if (kind != "none" or k in ("gate", "post_weight")) and
             (post != "none" or k != "post_weight")]
    _exact(n, dim, frame, names, kind, post, a=0.5, seed=n)


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("n,dim,frame", [(203520, 128, 0), (5000, 640, 0), (900, 5120, 100), (64, 1536, 1)])
@pytest.mark.parametrize("names", [("weight",), ("scale", "shift", "weight", "bias")])
def test_sums_of_a_norm_alone(n, dim, frame, kind, names):
    _exact(n, dim, frame, names, kind, with_y=False, seed=n)


@pytest.mark.parametrize("dim", WHOLE.WIDTHS)
@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("post", ["none", "layer", "rms"])
def test_rows(dim, kind, post):
    """What a row's means enter, in the 2-norm of each row (OT.ROW_NORM)."""
    if dim == 8 and "layer" in (kind, post):
        return       # eight columns: a row whose deviations are small beside their mean
    t, gr, gh = OT.row_case(dim, post)
    w = {k: x.double().cuda() for k, x in t.items()}
    plan = L.ResidualNorm(dim, norm=KIND[kind], post=KIND[post], eps=1e-5, frame_tokens=25)
    t = {k: x.cuda() for k, x in t.items()}
    gr, gh = gr.cuda(), gh.cuda()
    got = dict(zip("rh", L.residual_norm(plan, **t)))
    rest = {k: x for k, x in t.items() if k not in ("x", "y")}
    got.update(L.residual_norm_backward(plan, gh, gr, t["x"], t["y"], wanted=["x", "y"], **rest))
    want = OT.row_results(w, gr.double(), gh.double(), kind, post, 1e-5, 25)
    for k in want:
        off = (got[k].double() - want[k]).norm(dim=-1) / want[k].norm(dim=-1)
        assert off.max() <= OT.ROW_NORM[k], (k, float(off.max()))
