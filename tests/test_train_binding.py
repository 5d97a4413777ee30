"""The binding of the operators of training where it needs no GPU: the library is replaced by
calls that write nothing and succeed, tensors lie in host memory."""
import pytest
import torch

import paper_2605_31057_amd as L

BF = torch.bfloat16


class _Calls:
    def __getattr__(self, name):
        return lambda *args: L.OK


@pytest.fixture
def no_library(monkeypatch):
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
