"""``rope`` under autograd: its gradient is ``rope_backward``, whatever the gradient's
layout, in place, into a buffer, on another stream, twice; without a graph nothing is
recorded."""
import pytest
import torch

import paper_2605_31057_amd as L

pytestmark = pytest.mark.gpu

BF, HF, SF = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    L.lib()


def _x(seed=1, dtype=SF, nhd=False, H=3, n=50):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((n, H, 128) if nhd else (H, n, 128), generator=g).to(dtype).cuda()
    return x.transpose(0, 1) if nhd else x


R = dict(start=11)


def _rope(halves=False):
    return L.Rope(3, 4, 5, layout=L.ROPE_HALVES if halves else L.ROPE_PAIRS)


@pytest.mark.parametrize("dtype", [BF, HF, SF])
@pytest.mark.parametrize("nhd", [False, True])
@pytest.mark.parametrize("halves", [False, True])
def test_gradient(dtype, nhd, halves):
    r = _rope(halves)
    x, w = _x(1, dtype, nhd), _x(2, dtype)
    want = L.rope(x, r, **R)
    x.requires_grad_()
    y = L.rope(x, r, **R)
    assert torch.equal(y, want)
    y.backward(w)
    assert torch.equal(x.grad, L.rope_backward(w, r, **R))


def test_gradients_that_are_expanded_or_not_aligned():
    r = _rope()
    ones = torch.ones(3, 50, 128, device="cuda")
    odd = torch.ones(3 * 50 * 128 + 1, device="cuda")[1:].view(3, 50, 128)
    for grad in (ones, ones[:1, :1].expand(3, 50, 128), ones[:, :, :1].expand(3, 50, 128), odd,
                 ones.transpose(1, 2).contiguous().transpose(1, 2)):
        x = _x().requires_grad_()
        L.rope(x, r, **R).backward(grad)
        assert torch.equal(x.grad, L.rope_backward(ones, r, **R))
    x = _x().requires_grad_()
    L.rope(x, r, **R).sum().backward()       # an expanded scalar
    assert torch.equal(x.grad, L.rope_backward(ones, r, **R))


def test_second_gradient():
    """<v, d<w, rope(x)>/dx> is <rope(v), w>: the gradient of a gradient goes through."""
    r = _rope()
    x = _x(1).requires_grad_()
    w = _x(2).requires_grad_()
    v = _x(3)
    g, = torch.autograd.grad(L.rope(x, r, **R), x, w, create_graph=True)
    gw, = torch.autograd.grad(g, w, v)
    assert torch.equal(gw, L.rope(v, r, **R))
    w = _x(2).requires_grad_()
    L.rope_backward(w, r, **R).backward(v)
    assert torch.equal(w.grad, L.rope(v, r, **R))


def test_in_place_and_into_a_buffer():
    r = _rope()
    w = _x(2)
    want = L.rope_backward(w, r, **R)
    x = _x().requires_grad_()
    y = x * 1.0
    assert L.rope(y, r, out=y, **R) is y
    y.backward(w)
    assert torch.equal(x.grad, want)
    x = _x().requires_grad_()
    out = torch.empty_like(x)
    L.rope(x, r, out=out, **R)
    assert torch.equal(out, L.rope(x.detach(), r, **R))
    out.backward(w)
    assert torch.equal(x.grad, want)
    with pytest.raises(RuntimeError):        # a leaf
        L.rope(x, r, out=x, **R)
    # a buffer that had a graph loses it
    z = _x(4).requires_grad_()
    out = z * 2.0
    L.rope(_x(), r, out=out, **R)
    out.backward(w)
    assert z.grad is None or (z.grad == 0).all()


def test_a_saved_tensor_that_is_overwritten_is_noticed():
    r = _rope()
    for with_grad in (False, True):
        w = _x(5).requires_grad_()
        x = _x()
        if with_grad:
            x = x.requires_grad_() * 1.0
        y = (w * x).sum()                    # saves x
        L.rope(x, r, out=x, **R)
        with pytest.raises(RuntimeError):
            y.backward()


def test_without_a_graph():
    r = _rope()
    x = _x().requires_grad_()
    with torch.no_grad():
        assert not L.rope(x, r, **R).requires_grad
    with torch.inference_mode():
        y = _x()
        L.rope(y, r, out=y, **R)
    assert torch.equal(y, L.rope(_x(), r, **R))
    assert not L.rope(x.detach(), r, **R).requires_grad


def test_on_another_stream():
    r = _rope()
    x, w = _x().requires_grad_(), _x(2)
    want = L.rope_backward(w, r, **R)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    y = L.rope(x, r, stream=s, **R)
    torch.cuda.current_stream().wait_stream(s)
    y.backward(w)
    torch.cuda.synchronize()
    assert torch.equal(x.grad, want)


def test_a_training_step():
    """A projection, positions, a loss: the weights' gradient against the same step
    written with the rotation as a matrix of 64 bits."""
    r = _rope()
    g = torch.Generator().manual_seed(7)
    a = torch.randn(50, 64, generator=g).cuda()
    W = (torch.randn(64, 128, generator=g) / 8).cuda().requires_grad_()
    t = torch.randn(1, 50, 128, generator=g).cuda()
    (L.rope((a @ W)[None], r, **R) * t).sum().backward()
    eye = torch.eye(128, device="cuda")[:, None].expand(128, 50, 128).contiguous()
    M = L.rope(eye, r, **R).double().cpu()   # [element, token, rotated]
    a, t = a.double().cpu(), t[0].double().cpu()
    want = torch.einsum("nk,ine,ne->ki", a, M, t)
    # sums of 50 products, a rounding of 2^-24 each, and those of the rotation
    size = torch.einsum("nk,ine,ne->ki", a.abs(), M.abs(), t.abs())
    assert ((W.grad.cpu() - want).abs() <= 60 * 2.0 ** -24 * size).all()


def test_reads_and_attention_into_a_saved_tensor_are_noticed():
    c = L.KvCache(2, 128)
    k = torch.randn(2, 100, 128, device="cuda").bfloat16()
    L.kv_write(c, k, k)
    for write in (lambda t: L.attention_cache(k, c, out=t),
                  lambda t: L.kv_read(c, out=(t, torch.empty_like(t))),
                  lambda t: L.kv_read(c, out=(torch.empty_like(t), t))):
        t = torch.ones_like(k)
        w = torch.ones_like(k).requires_grad_()
        y = (w * t).sum()
        write(t)
        with pytest.raises(RuntimeError):
            y.backward()
    with torch.inference_mode():
        L.attention_cache(k, c, out=torch.empty_like(k))


def test_a_captured_gradient():
    """Forward and gradient captured into a graph, replayed with new inputs among eager
    calls."""
    r = _rope()
    x, w = _x(1).requires_grad_(), _x(2)

    def step():
        y = L.rope(x, r, **R)
        return y.detach(), torch.autograd.grad(y, x, w)[0]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(3):
            step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, g = step()
    for s in range(4):
        with torch.no_grad():
            x.copy_(_x(10 + s))
            w.copy_(_x(20 + s))
            y.fill_(0.0)
            g.fill_(0.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, L.rope(_x(10 + s), r, **R))
        assert torch.equal(g, L.rope_backward(_x(20 + s), r, **R))
