"""Tokens past the grid and pairs that no axis has are not rotated: their elements
come out as they went in, bit for bit, whatever stands next to them."""
import pytest
import torch

import paper_2605_31057_amd as L

pytestmark = pytest.mark.gpu

BF, HF, SF = torch.bfloat16, torch.float16, torch.float32
GRID, PAIRS = (2, 3, 5), (10, 9, 8)        # 30 tokens; 27 pairs turn, 37 do not


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    L.lib()


def _bits(x):
    return x.view(torch.int32 if x.dtype == SF else torch.int16)


def _case(dtype, halves):
    """Rows with NaN, infinities and zeros of both signs in pairs that do not turn:
    (x, True where an element does not turn)."""
    H, n = 2, 45                           # the last 15 tokens are past the grid
    g = torch.Generator().manual_seed(3)
    x = torch.randn(H, n, 128, generator=g).to(dtype)
    pair = torch.arange(128) % 64 if halves else torch.arange(128) // 2
    still = (pair >= sum(PAIRS))[None, :] | (torch.arange(n) >= 30)[:, None]
    odd = torch.tensor([float("nan"), float("inf"), -float("inf"), -0.0, 0.0]).to(dtype)
    pick = odd[torch.randint(0, 5, x.shape, generator=g)]
    x = torch.where(still & (torch.rand(x.shape, generator=g) < 0.3), pick, x)
    return x.cuda(), still.cuda().expand(x.shape)


def _rope(halves):
    return L.Rope(*GRID, pairs=PAIRS, layout=L.ROPE_HALVES if halves else L.ROPE_PAIRS)


@pytest.mark.parametrize("dtype", [BF, HF, SF])
@pytest.mark.parametrize("halves", [False, True])
def test_rotation_leaves_them(dtype, halves):
    x, still = _case(dtype, halves)
    r = _rope(halves)
    for f in (L.rope, L.rope_backward):
        y = f(x, r)
        assert torch.equal(_bits(y)[still], _bits(x)[still])
        assert torch.isfinite(y[~still]).all()


@pytest.mark.parametrize("dtype", [BF, HF, SF])
@pytest.mark.parametrize("halves", [False, True])
def test_the_cache_write_leaves_them(dtype, halves):
    """The same bytes as without positions: where no pair of a block turns, and for
    pairs that do not turn in a block whose scale the same element sets."""
    x, still = _case(dtype, halves)
    r = _rope(halves)
    text = x[:, 30:]
    a, b = L.KvCache(2, 64, 64), L.KvCache(2, 64, 64)
    L.kv_write(a, x[:, :30], x[:, :30], rope=r)
    L.kv_write(a, text, text, start=30, rope=r)
    L.kv_write(b, L.rope(x[:, :30].float(), r), x[:, :30].float())
    L.kv_write(b, text.float(), text.float(), start=30)
    ka, kb = (L.kv_read(c, dtype=SF)[0] for c in (a, b))
    assert torch.equal(a.k_scale[:, 0], b.k_scale[:, 0])
    assert torch.equal(torch.isnan(ka), torch.isnan(kb))
    assert torch.equal(torch.isnan(ka), ~torch.isfinite(x.float()))   # and no partner of one
    same = still & torch.isfinite(x)
    assert torch.equal(ka[same], kb[same])
