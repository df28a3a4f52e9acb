"""Attention over 4-bit pages at the ends of the ranges that the header gives: scaled scores up to
2^22, values whose magnitudes add up to 2^118."""

import math

import pytest
import torch

import packed_oracle as ref
from test_gpu_packed import BF16, F16, Case, binding  # noqa: F401

pytestmark = pytest.mark.gpu

ROWS = [(1, 4, 2), (20, 4, 2), (61, 8, 2)]


def _put(case, which, page, rows):
    """Rows of every sequence into the keys' (0) or values' (1) pages."""
    pool = case.pool[which].cpu()
    for b, x in enumerate(rows):
        ref.store(pool, page, [case.table[b][e // page] * page + e % page for e in range(len(x))], x)
        (case.k, case.v)[which][b] = ref.held(x)
    case.pool[which] = pool.cuda()


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("n,H,K", ROWS)
@pytest.mark.parametrize("length", [150, 3001])
def test_large_scores(binding, dtype, n, H, K, length):  # noqa: F811
    """Two scores, 3 * 2^20 and 2^21 or their negatives: the rows' weights are the same over the
    entries of the larger one and 0 over the others.

    A row's probabilities are one number, off by half a step u of 16 bits, the output by another:
    2 u of the mean, 1/8 more for the sums in fp32.  The reference of the exponents, 2^22.1 to
    base 2, is rounded twice by 1/4 at most, and so is the logarithm, whose half step is 1/8:
    0.35 + 0.13."""
    page = 16
    case = Case(binding, dtype, [length, 40], n, H, K, 64, page, tail=n + 3, tree=True, seed=n)
    case.mask[:, :, 0] = 1                             # (some entry of each score)
    case.mask[:, :, 1] = 1
    g = torch.Generator().manual_seed(n)

    def keys(*shape):
        x = torch.zeros(shape + (64,), dtype=dtype)
        x[..., 5] = torch.where(torch.rand(shape, generator=g) < 0.3, 1536.0, 1024.0).to(dtype)
        return x

    _put(case, 0, page, [keys(length, K), keys(40, K)])
    case.k_tail = keys(2, n + 3, K)
    case.k_tail[:, 0, :, 5], case.k_tail[:, 1, :, 5] = 1536.0, 1024.0
    sign = torch.where(torch.rand((2, n, H), generator=g) < 0.5, -1.0, 1.0)
    case.q = torch.zeros((2, n, H, 64), dtype=dtype)
    case.q[..., 5] = (2048.0 * sign).to(dtype)
    out, lse = case.call(scale=1.0, lse=True)
    out, lse = out.cpu(), lse.cpu()
    u = {BF16: 2.0 ** -8, F16: 2.0 ** -11}[dtype]
    for b in range(2):
        seen = ref.seen(n, n + 3, case.lens[b], 0, 0, case.mask[b], case.positions[b])
        for h in range(H):
            kh = h * K // H
            k = torch.cat([case.k[b][:, kh, 5], case.k_tail[b, :, kh, 5].double()])
            v = torch.cat([case.v[b][:, kh], case.v_tail[b, :, kh].double()])
            score = torch.where(seen, 2048.0 * sign[b, :, h, None].double() * k, -math.inf)
            top = score.amax(1, keepdim=True)
            w = (score == top).double()
            count = w.sum(1, keepdim=True)
            want, size = w @ v / count, w @ v.abs() / count
            off = (out[b, :, h].double() - want).abs()
            assert (off <= 2.125 * u * want.abs() + 2.0 ** -24 * len(v) * size + 2.0 ** -24).all(), (b, h)
            assert ((lse[b, :, h].double() - (top + count.log())[:, 0]).abs() <= 0.48).all(), (b, h)
    case.c.close()


@pytest.mark.parametrize("n,H,K", ROWS)
def test_large_values(binding, n, H, K):  # noqa: F811
    """Some 200 values around 2^108, whose sum is less than 2^118: finite, and right."""
    page = 16
    case = Case(binding, BF16, [130, 17], n, H, K, 64, page, tree=True, seed=n, spread=3.0)
    g = torch.Generator().manual_seed(n)
    _put(case, 1, page, [(torch.randn((m, K, 64), generator=g) * 2.0 ** 108).to(BF16)
                         for m in case.lens])
    case.v_tail = (case.v_tail.float() * 2.0 ** 108).to(BF16)
    for b, m in enumerate(case.lens):
        assert (case.v[b].abs().sum(0) + case.v_tail[b].double().abs().sum(0)).max() < 2.0 ** 118
    case.check()
    case.c.close()
