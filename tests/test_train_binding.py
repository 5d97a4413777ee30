"""The binding of the operators of training where it needs no GPU: the library is replaced by
calls that write nothing and succeed, tensors lie in host memory."""
import pytest
import torch

import paper_2605_31057_amd as L

BF = torch.bfloat16


class _Calls:
    def __getattr__(self, name):
        return lambda *args: b"" if name == "lvsa_status_str" else L.OK


@pytest.fixture
def no_library(monkeypatch):
    L._fast()          # what the calls keep of the library is of the real one
    monkeypatch.setattr(L, "lib", _Calls)
    monkeypatch.setattr(L, "_stream_ptr", lambda stream: None)
    monkeypatch.setattr(L, "_tensor", lambda t: L._Tensor(t.data_ptr(), *t.shape, *t.stride()[:2]))


def _qkv(n=128):
    return [torch.zeros(1, n, 128, dtype=BF) for _ in range(3)]


def _masks(n=128):
    row_ptr, words = torch.zeros(2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    return L.csr_mask(row_ptr, words, n, 128), L.exact_csr_mask(row_ptr, words, n, 128, 64)


WRITERS = {
    "attention": lambda out: L.attention(*_qkv(), _masks()[0], out=out),
    "attention_noalloc": lambda out: L.attention_noalloc(*_qkv(), _masks()[0], out),
    "attention_exact": lambda out: L.attention_exact(*_qkv(), _masks()[1], out=out),
    "dense_attention": lambda out: L.dense_attention(*_qkv(), out=out),
}


class _Saves(torch.autograd.Function):
    """Saves what it gives, as attention with gradients does."""

    @staticmethod
    def forward(ctx, x):
        out = x.clone()
        ctx.save_for_backward(out)
        return out

    @staticmethod
    def backward(ctx, grad):
        return grad * ctx.saved_tensors[0]


@pytest.mark.parametrize("name", WRITERS)
def test_a_write_into_a_given_output_is_noticed(no_library, name):
    x = torch.ones(1, 128, 128, dtype=BF, requires_grad=True)
    saved = _Saves.apply(x)
    with torch.no_grad():
        assert WRITERS[name](saved.detach()) is not None
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        saved.sum().backward()


@pytest.mark.parametrize("build", [L.build_mask_device, L.build_exact_mask_device])
def test_a_write_of_a_mask_is_noticed(no_library, build):
    row_ptr, col = (torch.zeros(n, dtype=torch.int32) for n in (6, 25))
    before = row_ptr._version, col._version
    build(8, 40, 64, 0, row_ptr, col)
    assert row_ptr._version > before[0] and col._version > before[1]


@pytest.mark.parametrize("name", WRITERS)
def test_outputs_made_without_versions(no_library, name):
    """Tensors of inference mode, which no graph can save, are written as ever, within the
    mode and past it."""
    with torch.inference_mode():
        out = torch.zeros(1, 128, 128, dtype=BF)
        WRITERS[name](out)
    with torch.no_grad():
        WRITERS[name](out)


def _differentiable():
    """Each differentiable call with its tensors, by name."""
    x, p = torch.zeros(4, 128), torch.zeros(1, 128)
    plan = L.ResidualNorm(128)
    (q, k, v), mask = _qkv(), _masks()[0]
    return {
        "attention": (lambda **t: L.attention(mask=mask, **t), dict(q=q, k=k, v=v, out=q.clone())),
        "dense_attention": (L.dense_attention, dict(q=q, k=k, v=v, out=q.clone())),
        "residual_norm": (lambda **t: L.residual_norm(plan, **t),
                          dict(x=x, y=x.clone(), gate=p, scale=p.clone(), shift=p.clone(),
                               weight=p[0].clone(), bias=p[0].clone())),
        "rope": (lambda **t: L.rope(r=None, **t), dict(x=q)),
        "rope_backward": (lambda **t: L.rope_backward(r=None, **t), dict(grad=q)),
    }


@pytest.mark.parametrize("call", _differentiable())
@pytest.mark.parametrize("recorded", [False, True])
def test_forward_mode_is_refused(call, recorded):
    """A tangent would be dropped without a word: no call has a forward-mode derivative."""
    fn, tensors = _differentiable()[call]
    if recorded:
        first = next(iter(tensors))
        tensors[first] = tensors[first].clone().requires_grad_()
    for name in tensors:
        with torch.autograd.forward_ad.dual_level():
            t = tensors[name]
            dual = torch.autograd.forward_ad.make_dual(t, torch.ones_like(t))
            with pytest.raises(NotImplementedError, match="forward-mode"):
                fn(**dict(tensors, **{name: dual}))


@pytest.mark.parametrize("call", ["attention", "dense_attention", "rope", "residual_norm"])
def test_forward_mode_of_a_function_is_refused(call):
    fn, tensors = _differentiable()[call]
    first = next(iter(tensors))
    rest = {k: t for k, t in tensors.items() if k != first}
    x = tensors[first]
    with pytest.raises(NotImplementedError, match="forward-mode"):
        torch.func.jvp(lambda t: fn(**{first: t}, **rest), (x,), (torch.ones_like(x),))


def test_tensors_without_tangents_are_taken_at_a_dual_level(no_library):
    with torch.autograd.forward_ad.dual_level(), torch.no_grad():
        L.attention(*_qkv(), _masks()[0])
        L.dense_attention(*_qkv())


@pytest.fixture
def no_kernels(monkeypatch):
    """Attention's graph without its kernels: an output of ones, gradients of ones."""
    def forward(q, k, v, mask, out, lse):
        out = torch.empty_like(q) if out is None else out
        with torch.no_grad():
            out.fill_(1.0)
        return out, torch.zeros(q.shape[:2])

    monkeypatch.setattr(L, "_launch_lse", forward)
    monkeypatch.setattr(L, "_launch_back",
                        lambda grad, q, k, v, *rest: tuple(torch.ones_like(t) for t in (q, k, v)))


def test_masks_of_inference_mode(no_kernels):
    """A mask's tensors that were made in inference mode, which a graph cannot save."""
    with torch.inference_mode():
        mask = _masks()[0]
    q, k, v = (t.requires_grad_() for t in _qkv())
    L.attention(q, k, v, mask).sum().backward()
    assert q.grad is not None


def test_an_output_used_again_lets_go_of_what_was_saved(no_kernels):
    """Calls into one tensor, one after the other: each overwrites what the one before gave, so
    the graph holds the last one's inputs alone, and its gradients are the last one's."""
    import gc
    import weakref
    w = torch.ones(1, 128, 128, dtype=BF, requires_grad=True)
    k, v = _qkv()[1:]
    buf, seen = torch.empty(1, 128, 128, dtype=BF), []
    for call in (lambda q: L.dense_attention(q, k, v, out=buf),
                 lambda q: L.attention(q, k, v, _masks()[0], out=buf)) * 3:
        q = w * 2
        seen.append(weakref.ref(q))
        assert call(q) is buf
        del q
        gc.collect()
    assert [s() is None for s in seen] == [True] * 5 + [False]
    buf.sum().backward()
    assert (w.grad == 2).all()


@pytest.mark.parametrize("recorded", [False, True])
def test_attention_takes_a_mask_with_rows_alone(no_kernels, no_library, recorded):
    """No mask, or one without rows, is refused with gradients as without: every key is
    dense_attention's (and attention_lse's) to take."""
    q, k, v = (t.requires_grad_(recorded) for t in _qkv())
    with pytest.raises(TypeError):
        L.attention(q, k, v, None)
    if recorded:       # without a graph the library itself refuses
        for rows, cols in ((None, None), (None, 4096), (4096, None)):
            with pytest.raises(L.LvsaError) as e:
                L.attention(q, k, v, L.BlockMask(128, 128, 1, 1, rows, cols))
            assert e.value.status == L.EINVAL
    assert L.dense_attention(q, k, v).requires_grad == recorded
