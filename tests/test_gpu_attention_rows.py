"""What one row's attention may depend on, and how far below its largest score a key still
counts."""

import math

import pytest
import torch

import cache_oracle as ref
from test_gpu_cache import BF16, F16, Setup, _i32, _tree_mask

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def binding():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2609_21827_amd import binding
    binding.load_library()
    return binding


@pytest.mark.parametrize("dtype,n,H,K,D", [
    (BF16, 3, 16, 4, 64), (F16, 16, 16, 8, 128), (BF16, 20, 16, 8, 128), (BF16, 31, 16, 4, 64),
    (F16, 61, 32, 8, 128), (BF16, 61, 32, 8, 128), (BF16, 20, 16, 8, 160), (F16, 61, 16, 8, 256)])
def test_large_keys_change_only_the_rows_that_attend_them(binding, dtype, n, H, K, D):
    """Finite keys so large that they take nearly all of a softmax, in drafted entries behind
    the first tiles: a row that masks them has the result that it has without, bit for bit,
    whatever rows share its wave."""
    B = 96
    s = Setup(binding, dtype, [300 + 7 * (b % 5) for b in range(B)], n, n, H, K, D, 16, seed=n + D)
    mask = _tree_mask(s.g, 1, n).expand(B, n, n).contiguous()
    clean = s.run(mask)
    odd = sorted({1, n // 2, n - 1})
    for b in range(B):
        for j in odd:
            e = s.lens[b] + j
            s.kc.flatten(0, 1)[int(s.table[b, e // 16]) * 16 + e % 16] *= 24
    out, lse = s.run(mask)
    masks = (mask[:, :, odd] == 0).all(2)
    assert masks.any() and not masks.all()
    assert torch.equal(out[masks], clean[0][masks])
    assert torch.equal(lse[masks], clean[1][masks])
    assert not torch.equal(out[~masks], clean[0][~masks])
    s.check((out, lse), mask, only={0, B - 1})
    s.cache.close()


@pytest.mark.parametrize("B,n,H,K,D", [(128, 1, 4, 4, 64), (128, 1, 16, 4, 128), (64, 12, 16, 4, 64),
                                       (64, 30, 16, 4, 64), (64, 61, 16, 4, 64),
                                       (64, 61, 16, 4, 128), (64, 20, 16, 4, 256)])
def test_keys_far_below_a_sink_keep_their_weight(binding, B, n, H, K, D):
    """One key with value 0 that takes nearly everything, and 2000 keys 11 to 17 below it: what
    these give is in the output with fp16's own accuracy.

    Bound: as the oracle's, but that a probability's rounding where fp16 has no more
    smaller steps, 2^-25 at most, is against a sum of at least 2^10 (the kernel's
    reference for fp16: the largest probability is held as 2^10 to 2^15) and not of 1."""
    L, page = 2000, 16
    g = torch.Generator().manual_seed(D + n)
    pages = L // page + -(-n // page) + 1
    kc = torch.zeros((pages * page, K, D))
    # q is 1 (0.9, 0.8) in every element, so a key of -x sqrt(D) / D has the score -x; all
    # keys of a head alike, so that roundings do not cancel
    kc[:L] = (-torch.tensor([11.3, 14.0, 16.5, 17.0]) * D ** -0.5)[None, :, None]
    vc = torch.randn((pages * page, K, D), generator=g) * 8 + 64
    kc[L // 2 + 1], vc[L // 2 + 1] = 0.0, 0.0
    kc[L:] = -30.0 * D ** -0.5                        # the rows' own
    kc, vc = kc.to(F16), vc.to(F16)
    q = torch.ones((1, n, H, D))
    q[:, 1::3], q[:, 2::3] = 0.9, 0.8
    q = q.to(F16)
    c = binding.Cache(batch=B, heads=H, kv_heads=K, head_dim=D, page_size=page, pages=pages,
                      table_width=pages, dtype=F16)
    table = torch.arange(pages).int().expand(B, pages).contiguous().cuda()
    out, lse = c.attention(q.expand(B, n, H, D).contiguous().cuda(), kc.view(pages, page, K, D).cuda(),
                           vc.view(pages, page, K, D).cuda(), table, _i32([L] * B), lse=True)
    assert c.device_error() == 0
    out, lse = out.cpu(), lse.cpu()
    rows = sorted({0, n // 2, n - 1})
    seen = torch.arange(L + n)[None, :] <= L + torch.tensor(rows)[:, None]
    for h in range(0, H, H // K):
        kv = h * K // H
        k, v = kc[:L + n, kv:kv + 1], vc[:L + n, kv:kv + 1]
        want, w_lse, tol, tol_lse = ref.attention(q[0, rows, h:h + 1], k, v, seen, D ** -0.5, F16)
        for i in range(len(rows)):
            size = v[seen[i]].double().abs().sum(0)
            tol[i] += ref.TINY[F16] * (2.0 ** -10 * size + 1) - ref.TINY[F16] * (size + 1)
        assert float((tol / want.abs()).max()) < 0.01
        for b in range(B):
            off = (out[b, rows, h:h + 1].double() - want).abs()
            assert (off <= tol).all(), (b, h, float((off / want.abs()).max()))
            off = (lse[b, rows, h:h + 1].double() - w_lse).abs()
            assert (off <= tol_lse).all(), (b, h, float(off.max()))
    c.close()


def test_a_row_of_low_scores_beside_rows_of_high_ones(binding):
    """Rows whose maxima rise at different tiles, in one wave: each within its bound."""
    for dtype in (BF16, F16):
        s = Setup(binding, dtype, [900] * 40, 16, 16, 16, 8, 64, 16, seed=9)
        s.q *= torch.linspace(0.01, 4, 16)[None, :, None, None].to(dtype)
        got = s.run()
        assert all(math.isfinite(float(t.float().abs().max())) for t in got)
        s.check(got, only={0, 39})
        s.cache.close()
