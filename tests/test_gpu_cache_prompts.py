"""Rows of a prompt, thousands at once: plan, write and causal attention."""

import math
import random

import pytest
import torch

import cache_oracle as ref
from test_gpu_cache import BF16, F16, _i32, _plan_cache

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def binding():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2609_21827_amd import binding
    binding.load_library()
    return binding


@pytest.mark.parametrize("B,n,page,ragged", [(1, 8192, 64, False), (3, 5000, 16, True), (2, 4099, 1, True)])
def test_plan_of_prompts(binding, B, n, page, ragged):
    rng = random.Random(n)
    lens = [rng.randint(0, 700) for _ in range(B)]
    held = [-(-x // page) for x in lens]
    width = max(-(-(x + n) // page) for x in lens)
    pages = B * width
    ids = list(range(pages))
    rng.shuffle(ids)
    table = [[ids.pop() if p < held[b] else -1 for p in range(width)] for b in range(B)]
    count = [rng.choice([n, rng.randint(0, n)]) for _ in range(B)] if ragged else None
    depth = [[rng.randint(0, 99) for _ in range(n)] for _ in range(B)] if ragged else None
    c = _plan_cache(binding, B, page, pages, width)
    state = [_i32(lens), _i32(held), _i32(table), _i32(ids + [0] * (pages - len(ids))), _i32([len(ids)])]
    slots, positions, status = c.plan(*state, n, count=None if count is None else _i32(count),
                                      depth=None if depth is None else _i32(depth))
    want = ref.plan(page, width, pages, lens, held, table, ids, n, count, depth)
    assert slots.tolist() == want[0] and positions.tolist() == want[1]
    assert status.tolist() == want[2] and state[1].tolist() == want[3]
    assert state[2].tolist() == want[4] and state[3].tolist()[:len(want[5])] == want[5]
    assert c.device_error() == 0
    c.close()


@pytest.mark.parametrize("dtype,lens,n,count,H,K,D,page", [
    (BF16, [0], 2000, None, 8, 2, 128, 64), (F16, [0, 900], 2049, [2049, 700], 4, 4, 64, 16),
    (BF16, [5000], 1500, None, 4, 1, 80, 64), (F16, [77], 1100, None, 2, 2, 256, 32)])
def test_attention_of_prompts(binding, dtype, lens, n, count, H, K, D, page):
    """Written and attended in one go, row after row against the 64-bit form."""
    B = len(lens)
    g = torch.Generator().manual_seed(n)
    width = -(-(max(lens) + n) // page)
    pages = B * width
    table = torch.randperm(pages, generator=g).int().view(B, width)
    old = torch.randn((2, pages * page, K, D), generator=g).to(dtype)
    q = torch.randn((B, n, H, D), generator=g).to(dtype)
    k, v = (torch.randn((B, n, K, D), generator=g).to(dtype) for _ in range(2))
    e = torch.tensor(lens)[:, None] + torch.arange(n)
    slots = table.gather(1, (e // page).long()).long() * page + e % page
    rows = count or [n] * B
    slots[torch.arange(n)[None, :] >= torch.tensor(rows)[:, None]] = -1
    c = binding.Cache(batch=B, heads=H, kv_heads=K, head_dim=D, page_size=page, pages=pages,
                      table_width=width, dtype=dtype)
    kc, vc = (x.view(pages, page, K, D).cuda() for x in old)
    got_q = c.write(q.cuda(), k.cuda(), v.cuda(), slots.cuda(), kc, vc)
    out, lse = c.attention(got_q, kc, vc, table.cuda(), _i32(lens), lse=True,
                           count=None if count is None else _i32(count))
    assert c.device_error() == 0
    out, lse = out.cpu(), lse.cpu()
    for b in range(B):
        L = lens[b] + rows[b]
        at = torch.arange(L)
        place = table[b].long()[at // page] * page + at % page
        keys, values = (x.cpu().view(-1, K, D)[place] for x in (kc, vc))
        assert torch.equal(keys[lens[b]:], k[b, :rows[b]]) and torch.equal(values[lens[b]:], v[b, :rows[b]])
        some = sorted({0, 1, 63, 64, 255, 256, rows[b] // 2, rows[b] - 2, rows[b] - 1})
        seen = at[None, :] <= lens[b] + torch.tensor(some)[:, None]
        want, w_lse, tol, tol_lse = ref.attention(q[b, some], keys, values, seen, D ** -0.5, dtype)
        off = (out[b, some].double() - want).abs()
        assert (off <= tol).all(), (b, float((off - tol).max()))
        assert ((lse[b, some].double() - w_lse).abs() <= tol_lse).all()
        # (all rows: weighted means of values below 6, and finite sums)
        assert (out[b, :rows[b]].float().abs() < 6).all()
        assert all(math.isfinite(x) for x in lse[b, :rows[b]].flatten().tolist())
    c.close()
