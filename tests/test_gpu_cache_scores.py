"""Scores of the attention over the 8-bit cache where the products of one channel
are far larger than the others: the sums over a row's 128 products are taken in 32
bits in every form (few query rows, tiles, with a mask)."""
import numpy as np
import pytest
import torch

import paper_2605_31057_amd as L
from oracle import cache as OC

pytestmark = pytest.mark.gpu

BF = torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    L.lib()


def _full_mask(N, B):
    nb = -(-N // B)
    rp = torch.arange(nb + 1, dtype=torch.int32, device="cuda") * nb
    ci = torch.arange(nb, dtype=torch.int32, device="cuda").repeat(nb)
    return L.csr_mask(rp.int().contiguous(), ci.int().contiguous(), N, B)


# queries: both sides of the line between few rows and tiles, whole tiles and more
QUERIES = [1, 16, 33, 64, 65, 100, 300]


@pytest.mark.parametrize("mask", [0, 64, 128])
@pytest.mark.parametrize("n", QUERIES)
@pytest.mark.parametrize("kind", ["shared", "cancelling"])
def test_scores_that_are_equal_give_equal_weights(kind, n, mask):
    """Every key's score is the same number, a sum of multiples of 1/16 below 2^16:
    any order of adding gives it exactly in 32 bits.  One channel's product is 2^14,
    or two cancel; the small ones are a permutation of the same values for each key.
    Equal weights are powers of two, so the output is the mean of v, a sum of whole
    numbers below 2^24 times a power of two divided by the keys' number: within the
    output's half step (2^-8 of the value) and one step of a division in 32 bits."""
    H, N = 2, 768
    g = torch.Generator().manual_seed(n)
    small = torch.cat([torch.arange(1, 8), -torch.arange(1, 8)]).repeat(9).double() / 16   # 126
    k = torch.stack([small[torch.randperm(126, generator=g)] for _ in range(H * N)])
    k = k.view(H, N, 126)
    # 2^14 from one channel, or 2^14 - 2^14 from two whose signs differ from key to key
    sign = torch.ones(H, N) if kind == "shared" else \
        torch.where(torch.rand(H, N, generator=g) < 0.5, -1.0, 1.0)
    other = 0.0 if kind == "shared" else -1.0
    k = torch.cat([128 * sign[..., None], k, 128 * sign[..., None] * other], -1)
    q = torch.ones(H, n, 128)
    q[..., 0] = q[..., 127] = 128.0
    v = torch.randint(-8, 9, (H, N, 128), generator=g).double()
    c = L.KvCache(H, N, 128)
    L.kv_write(c, k.to(BF).cuda(), v.to(BF).cuda())
    back = L.kv_read(c, dtype=torch.float32)
    assert torch.equal(back[0].double().cpu(), k.double())     # held as they are
    assert torch.equal(back[1].double().cpu(), v)
    got = L.attention_cache(q.to(BF).cuda(), c, mask=_full_mask(N, mask) if mask else None,
                            q_start=N - n)
    want = v.mean(1, keepdim=True).expand(H, n, 128)
    err = (got.double().cpu() - want).abs()
    assert (err <= want.abs() * (2.0 ** -8 + 2.0 ** -22)).all(), float(err.max())


@pytest.mark.parametrize("big", [8.0, 32.0, 128.0])
@pytest.mark.parametrize("n", [1, 64, 65, 300])
def test_one_large_channel(big, n):
    """Against 64 bits: a score is off by at most 127 roundings of partial sums, 2^-24
    of sum |q k| each; a weight by that and half a bf16 step (2^-8); the output by its
    own half step.  Sums over the keys in fp32, 2^-24 of sum p |v| a step."""
    H, N = 2, 900
    g = torch.Generator().manual_seed(int(big) + n)
    q, k, v = (torch.randn(H, m, 128, generator=g) for m in (n, N, N))
    q[..., 5] = big
    k[..., 5] = big
    q = q.to(BF).cuda()
    c = L.KvCache(H, N, 128)
    L.kv_write(c, k.to(BF).cuda(), v.to(BF).cuda())
    kk, vv = (x.double().cpu().numpy() for x in L.kv_read(c, dtype=torch.float32))
    wide = q.double().cpu().numpy()
    want, spread, size, _ = OC.attend(wide, kk, vv)
    products = np.stack([(np.abs(wide[h]) @ np.abs(kk[h]).T).max(1) for h in range(H)])
    w = 2.0 ** -8 * 1.02 + 127 * 2.0 ** -24 * products[..., None] / np.sqrt(128)
    tol = (np.abs(want) + w * spread) * 2.0 ** -8 + w * spread + size * N * 2.0 ** -23
    err = np.abs(L.attention_cache(q, c).double().cpu().numpy() - want)
    assert (err <= tol).all(), float((err / tol).max())


@pytest.mark.parametrize("n", [65, 300])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_a_query_that_is_not_finite_over_keys_of_one_sign(n, bad):
    """It becomes NaN, the others stay as they are, bit for bit."""
    N = 300
    c = L.KvCache(1, N, 64)
    g = torch.Generator().manual_seed(n)
    k, v = (torch.randn(1, N, 128, generator=g) for _ in range(2))
    k[..., 9] = -1.0
    L.kv_write(c, k.to(BF).cuda(), v.to(BF).cuda())
    q = torch.randn(1, n, 128, generator=g).to(BF).cuda()
    want = L.attention_cache(q, c)
    q[0, 1, 9] = bad
    got = L.attention_cache(q, c)
    assert torch.isnan(got[0, 1]).all()
    assert torch.equal(got[0, 2:], want[0, 2:]) and torch.equal(got[0, 0], want[0, 0])


@pytest.mark.parametrize("n", [1, 16, 17, 40, 64])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_the_same_with_few_rows(n, bad):
    """An infinity times keys of one sign gives scores of -inf alone: NaN, not the zeros
    of a query without keys, with and without a mask."""
    N = 300
    c = L.KvCache(1, N, 64)
    g = torch.Generator().manual_seed(n)
    k, v = (torch.randn(1, N, 128, generator=g) for _ in range(2))
    k[..., 9] = -1.0
    L.kv_write(c, k.to(BF).cuda(), v.to(BF).cuda())
    q = torch.randn(1, n, 128, generator=g).to(BF).cuda()
    for mask in (None, _full_mask(N, 64)):
        want = L.attention_cache(q, c, mask=mask, q_start=0)
        p = q.clone()
        p[0, n // 2, 9] = bad
        got = L.attention_cache(p, c, mask=mask, q_start=0)
        assert torch.isnan(got[0, n // 2]).all()
        others = [i for i in range(n) if i != n // 2]
        assert torch.equal(got[0, others], want[0, others])
    none = L.KvCache(1, 128)
    assert (L.attention_cache(p, none) == 0).all()       # no key at all: still zeros
