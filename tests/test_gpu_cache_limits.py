"""Sums and launches at the ends of the ranges that the cache and scoring calls allow."""

import ctypes

import pytest
import torch

from test_gpu_cache import BF16, _i32, _plan_cache

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


@pytest.mark.parametrize("K,rows", [(1, (1 << 26) - 4), (40, (1 << 25) + 8)])
def test_write_of_the_most_rows(binding, K, rows):
    """A wave a row as the launch's threads end, and several that would go past them."""
    D, page = 8, 4096
    pages = -(-rows // page)
    c = binding.Cache(batch=1, heads=K, kv_heads=K, head_dim=D, page_size=page, pages=pages,
                      table_width=1)
    k = torch.arange(rows, device="cuda", dtype=torch.int32).remainder_(251).to(BF16)
    k = k[:, None].expand(rows, K * D).contiguous()
    pool = torch.zeros((pages, page, K, D), dtype=BF16, device="cuda")
    slots = torch.arange(rows, device="cuda")
    # (keys and values alike, so one pool takes both)
    c.write(None, k.view(1, rows, K, D), k.view(1, rows, K, D), slots[None], pool, pool)
    assert c.device_error() == 0
    for a in range(0, rows, 1 << 22):
        assert torch.equal(pool.view(-1, K * D)[a:min(a + (1 << 22), rows)], k[a:a + (1 << 22)])
    assert not pool.view(-1, K * D)[rows:].any()
    c.close()


def test_scores_of_the_most_entries(binding):
    m = (1 << 24) - 1
    x = torch.tensor([[[0.0, 1.0, 2.0, 3.0]]], device="cuda")
    tokens = torch.arange(m, device="cuda", dtype=torch.int32).remainder_(4)[None]
    path = torch.zeros((1, m), dtype=torch.int32, device="cuda")
    s = binding.Scorer(4, torch.float32)
    few = [t.clone() for t in s.logprobs(x, tokens[:, :4].contiguous(),
                                         path=path[:, :4].contiguous(), top=1)]
    got = s.logprobs(x, tokens, path=path, top=1)
    for a, b in zip(got, few):
        assert torch.equal(a[:, :m - 3].reshape(-1, 4), b.reshape(1, 4).expand(m // 4, 4))
    s.close()


def test_calls_past_a_launch_are_refused(binding):
    """Only the C ABI can be asked for them without the memory."""
    lib = binding.load_library()
    c = _plan_cache(binding, 4, 16, 10, 4)
    s = binding.Scorer(8, torch.float32)
    some = torch.zeros(64, dtype=torch.int64, device="cuda")
    p = some.data_ptr()
    for n in (1 << 24, (1 << 24) + 5, 1 << 28, 1 << 29, -1):
        a = binding.WriteArgs(n, 0, 0, 0, None, p, p, None, 0, 8, 8, 0, p, None, None, None, None,
                              0.0, p, p)
        assert lib.rheo_cache_write(c._h, ctypes.byref(a), None) == binding.RHEO_EINVAL
        assert "n must be" in lib.rheo_last_error().decode()
    for B, m in ((1, 1 << 24), (1 << 12, 1 << 12), (1 << 15, 1 << 15)):
        assert lib.rheo_token_logprobs(s._h, p, B, 1, p, p, m, 0, 1.0, p, None, None, None, None,
                                       None) == binding.RHEO_EINVAL
        assert "2^24" in lib.rheo_last_error().decode()
    torch.cuda.synchronize()
    c.close(), s.close()
