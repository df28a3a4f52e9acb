"""Steps in which the free pages do not reach: a sequence that the plan did not serve keeps what
it has, and meets nothing of the pages that it once had and others hold now."""

import random

import pytest
import torch

from test_gpu_cache import BF16, F16, Setup, _i32, _tree_mask
from test_gpu_cache_use import Loop, _refused

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def binding():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2609_21827_amd import binding
    binding.load_library()
    return binding


def test_an_unserved_sequence_leaves_anothers_pages_alone(binding):
    B, n, K, D, page, width, depth = 2, 20, 2, 64, 16, 4, 3
    pages = 6
    c = binding.Cache(batch=B, heads=4, kv_heads=K, head_dim=D, page_size=page, pages=pages,
                      table_width=width)
    table = _i32([[0, 1, 9, 9], [2, 3, 4, 5]])
    held, free, free_count = _i32([2, 4]), _i32([0] * pages), _i32([0])
    lens = _i32([30, 31])
    state = (lens, held, table, free, free_count)
    c.plan(*state, 0)                                  # the second gives two pages back,
    slots, pos, status = c.plan(*state, n)             # the first takes them, none are left
    assert status.tolist() == [0, 1] and sorted(table[0, 2:].tolist()) == [4, 5]
    assert table[1].tolist() == [2, 3, 4, 5] and held.tolist() == [4, 2]
    g = torch.Generator().manual_seed(0)
    kc, vc = (torch.randn((pages, page, K, D), generator=g).to(BF16).cuda() for _ in range(2))
    q = torch.randn((B, n, 4, D), generator=g).to(BF16).cuda()
    k, v = (torch.randn((B, n, K, D), generator=g).to(BF16).cuda() for _ in range(2))
    out = torch.full_like(q, 7.0)
    c.write(q, k, v, slots, kc, vc, out=out)
    assert (out[1] == 7).all() and torch.equal(out[0], q[0])
    mask = _tree_mask(g, 1, n).expand(B, n, n).contiguous().cuda()
    want, w_lse = c.attention(q, kc, vc, table, lens, mask=mask, count=_i32([n, 0]), lse=True)
    got, lse = torch.full_like(q, 9.0), torch.full((B, n, 4), 9.0, device="cuda")
    c.attention(q, kc, vc, table, lens, mask=mask, status=status, out=got, lse=lse)
    assert torch.equal(got[0], want[0]) and torch.equal(lse[0], w_lse[0])
    assert (got[1] == 9).all() and (lse[1] == 9).all()
    # the second's walk accepts nodes 3, 5, 8: entries that would move inside the first's pages
    parent = [-1, 0, 0, 0, 1, 3, 2, 2, 5] + [0] * 11
    par, tok = _i32([parent] * 2), _i32([list(range(100, 120))] * 2)
    acc, took = _i32([[103, 105, 108]] * 2), _i32([0, 3])
    k0, v0 = kc.clone(), vc.clone()
    path, new = c.commit(par, tok, acc, took, lens, table, kc[None], vc[None], status=status)
    assert torch.equal(kc, k0) and torch.equal(vc, v0)
    assert path.tolist() == [[0, -1, -1, -1], [-1] * 4] and new.tolist() == [31, 31]
    # in place; bad data of a sequence that is left out is not looked at
    c.commit(par, tok, acc, _i32([0, 99]), lens, table, kc[None], vc[None], status=status,
             out=(path, lens))
    assert lens.tolist() == [31, 31] and torch.equal(kc, k0)
    assert c.device_error() == 0
    for bad in (status.long(), status[:1], status.cpu()):
        _refused(binding, lambda: c.attention(q, kc, vc, table, lens, mask=mask, status=bad))
        _refused(binding, lambda: c.commit(par, tok, acc, took, lens, table, kc[None], vc[None],
                                           status=bad))
    c.close()


@pytest.mark.parametrize("dtype,lens,n,H,K,D", [
    (BF16, [900, 33, 0, 700], 61, 8, 2, 128), (F16, [300] * 70, 31, 32, 8, 64),
    (BF16, [200] * 40, 61, 32, 8, 128), (BF16, [5000, 60], 1, 8, 2, 128), (F16, [90], 5, 4, 4, 256)])
def test_status_is_a_count_of_zero(binding, dtype, lens, n, H, K, D):
    """Whole items, cut ones and joined ones, with a count beside it and without."""
    B = len(lens)
    s = Setup(binding, dtype, lens, n, n, H, K, D, 16, seed=n)
    mask = _tree_mask(s.g, 1, n).expand(B, n, n).contiguous()
    status = [1 if b % 3 == 1 else 2 if b % 7 == 5 else 0 for b in range(B)]
    for count in (None, [n - (b % 2) for b in range(B)]):
        left = [0 if status[b] else (n if count is None else count[b]) for b in range(B)]
        want = s.run(mask, left)
        got = s.run(mask, count, status=_i32(status))
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        got = s.run(mask, count, status=_i32([0] * B))
        s.check(got, mask, count, only={0, B - 1})
    s.run(mask, [-5 if x else n for x in status], status=_i32(status))
    s.cache.close()


def test_steps_with_too_few_pages(binding):
    """Twenty steps of five sequences that want more pages than there are: what each holds is
    what its own served steps have put there, whatever the others do."""
    loop = Loop(binding, B=5, n=20, depth=5, seed=3)
    B, page, layers = loop.B, loop.page, loop.layers
    loop.free_count.fill_(13)
    loop.free[13:] = -1
    rng = random.Random(8)
    kept = [[] for _ in range(B)]                      # each entry's keys and values, all layers
    seen = set()
    for step in range(20):
        loop.feed(step)
        state = (loop.lens, loop.held, loop.table, loop.free, loop.free_count)
        slots, pos, status = loop.cache.plan(*state, loop.n, depth=loop.depths)
        seen.update(status.tolist())
        for i in range(layers):
            q, k, v = loop.qkv[i].split([loop.H * loop.D, loop.K * loop.D, loop.K * loop.D], dim=2)
            q = loop.cache.write(q.unflatten(2, (loop.H, loop.D)), k.unflatten(2, (loop.K, loop.D)),
                                 v.unflatten(2, (loop.K, loop.D)), slots, loop.kc[i], loop.vc[i],
                                 positions=pos, rotation=loop.rot)
            loop.cache.attention(q, loop.kc[i], loop.vc[i], loop.table, loop.lens, mask=loop.mask,
                                 status=status)
        new = {}
        for b in range(B):
            if status[b] == 0:
                new[b] = [(loop.kc.flatten(1, 2)[:, s].clone(), loop.vc.flatten(1, 2)[:, s].clone())
                          for s in slots[b].tolist()]
        path, _ = loop.cache.commit(
            loop.parent, loop.token, loop.accepted, loop.accept_len, loop.lens, loop.table, loop.kc,
            loop.vc, status=status,
            out=(torch.empty((B, loop.depth + 1), dtype=torch.int32, device="cuda"), loop.lens))
        logp = loop.scorer.logprobs(loop.logits, loop.emitted, path=path)[0]
        for b in range(B):
            nodes = [x for x in path[b].tolist() if x >= 0]
            assert bool(nodes) == (status[b] == 0)
            if not nodes:
                assert (logp[b] == 0).all()
            kept[b] += [new[b][x] for x in nodes]
        ended = rng.randrange(B) if step % 4 == 3 else None
        if ended is not None:
            loop.lens[ended], kept[ended] = 0, []
        loop.cache.plan(*state, 0)
        lens, held, table = loop.lens.tolist(), loop.held.tolist(), loop.table.tolist()
        assert lens == [len(x) for x in kept]
        named = [p for b in range(B) for p in table[b][:held[b]]] + \
            loop.free[:int(loop.free_count)].tolist()
        assert len(named) == 13 and len(set(named)) == 13
        for b in range(B):
            for e, (k, v) in enumerate(kept[b]):
                s = table[b][e // page] * page + e % page
                assert torch.equal(loop.kc.flatten(1, 2)[:, s], k), (step, b, e)
                assert torch.equal(loop.vc.flatten(1, 2)[:, s], v), (step, b, e)
    assert seen >= {0, 1}
    assert loop.cache.device_error() == 0
    loop.close()
