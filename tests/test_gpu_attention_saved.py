"""What attention's graphs have saved: a later write into it is an error, never a wrong
gradient."""
import pytest
import torch

import paper_2605_31057_amd as L

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
T, P, B = 6, 80, 64
N = T * P
NB = -(-N // B)


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    L.lib()


def _inputs(seed):
    g = torch.Generator().manual_seed(seed)
    return [torch.randn(2, N, 128, generator=g).to(BF).cuda() for _ in range(3)]


def _masks():
    csr = L.build_mask(T, P, B, 0, L.Params(window=1, tper=3), exact=True).upload()
    return csr, csr.device_mask(), csr.exact_mask()


@pytest.mark.parametrize("first", ["attention", "dense_attention"])
@pytest.mark.parametrize("then", ["attention", "attention_noalloc", "attention_exact",
                                  "dense_attention"])
def test_a_second_call_into_a_saved_output(first, then):
    csr, blocks, exact = _masks()
    q, k, v = (t.requires_grad_() for t in _inputs(1))
    buf = torch.empty(2, N, 128, dtype=BF, device="cuda")
    y = (L.attention(q, k, v, blocks, out=buf) if first == "attention" else
         L.dense_attention(q, k, v, out=buf))
    call = {"attention": lambda *x: L.attention(*x, blocks, out=buf),
            "attention_noalloc": lambda *x: L.attention_noalloc(*x, blocks, buf),
            "attention_exact": lambda *x: L.attention_exact(*x, exact, out=buf),
            "dense_attention": lambda *x: L.dense_attention(*x, out=buf)}[then]
    with torch.no_grad():
        call(*_inputs(2))
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward(torch.ones_like(y))


def test_an_exact_mask_built_into_a_saved_ones_offsets():
    row_ptr = torch.empty(NB + 1, dtype=torch.int32, device="cuda")
    cols, words = (torch.empty(NB * NB, dtype=torch.int32, device="cuda") for _ in range(2))
    p = L.Params(window=1, tper=3)
    m = L.build_mask_device(T, P, B, 0, row_ptr, cols, p)
    q, k, v = (t.requires_grad_() for t in _inputs(1))
    y = L.attention(q, k, v, m)
    L.build_exact_mask_device(T, P, B, 1, row_ptr, words, p)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward(torch.ones_like(y))
