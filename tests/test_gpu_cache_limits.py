"""Sums and launches at the ends of the ranges that the cache and scoring calls allow."""

import pytest
import torch

from test_gpu_cache import _i32, _plan_cache

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def binding():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2609_21827_amd import binding
    binding.load_library()
    return binding


def test_plan_of_more_missing_pages_than_32_bits_hold(binding):
    """4096 sequences that lack 2^19 + 1023 pages each: no sum of them reaches its pages, also
    where sums pass 2^31."""
    B, width = 4096, (1 << 19) + 1024
    table = torch.zeros((B, width), dtype=torch.int32, device="cuda")
    c = _plan_cache(binding, B, 1, 10, width)
    held = _i32([0] * B)
    free, count = _i32(list(range(10))), _i32([10])
    slots, positions, status = c.plan(_i32([width - 2] * B), held, table, free, count, 1)
    assert (status == 1).all()
    assert (slots == -1).all() and (positions == -1).all()
    assert (held == 0).all() and count.tolist() == [10] and free.tolist() == list(range(10))
    assert c.device_error() == 0
    # one that lacks none, behind them all, is served
    lens = _i32([width - 2] * (B - 1) + [0])
    _, _, status = c.plan(lens, held, table, free, count, 0)
    assert status.tolist() == [1] * (B - 1) + [0] and (held == 0).all()
    c.close()
