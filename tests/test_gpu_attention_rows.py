"""What one row's attention may depend on."""

import math

import pytest
import torch

from test_gpu_cache import BF16, F16, Setup, _tree_mask

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


def test_a_row_of_low_scores_beside_rows_of_high_ones(binding):
    """Rows whose maxima rise at different tiles, in one wave: each within its bound."""
    for dtype in (BF16, F16):
        s = Setup(binding, dtype, [900] * 40, 16, 16, 16, 8, 64, 16, seed=9)
        s.q *= torch.linspace(0.01, 4, 16)[None, :, None, None].to(dtype)
        got = s.run()
        assert all(math.isfinite(float(t.float().abs().max())) for t in got)
        s.check(got, only={0, 39})
        s.cache.close()
