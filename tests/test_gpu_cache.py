"""The cache operators (plan, write, tree attention, commit) against plain 64-bit forms."""

import math
import random

import pytest
import torch

import cache_oracle as ref

pytestmark = pytest.mark.gpu

BF16, F16 = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def binding():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2609_21827_amd import binding
    binding.load_library()
    return binding


def _i32(rows):
    return torch.tensor(rows, dtype=torch.int32, device="cuda")


# -- plan -------------------------------------------------------------------------


def _plan_cache(binding, B, page, pages, width):
    return binding.Cache(batch=B, heads=1, kv_heads=1, head_dim=8, page_size=page, pages=pages,
                         table_width=width)


PLANS = [
    # B, page, width, spare pages, n, most tokens
    (1, 64, 8, 3, 61, 400), (1, 1, 90, 40, 7, 80), (3, 16, 9, 0, 1, 100), (7, 16, 12, 5, 81, 90),
    (64, 16, 20, 60, 33, 250), (257, 8, 9, 300, 20, 40), (700, 4, 30, 500, 9, 100),
    (5, 4096, 2, 4, 300, 8000), (40, 32, 4, 10, 0, 120), (1500, 2, 6, 40, 5, 10),
]


@pytest.mark.parametrize("B,page,width,spare,n,most", PLANS)
def test_plan_matches_the_plain_form_over_steps(binding, B, page, width, spare, n, most):
    """Steps of growth, shrinkage, finished sequences, short pools and short tables, each
    from the state the last one left."""
    rng = random.Random(B * 31 + page)
    lens = [rng.randint(0, most) for _ in range(B)]
    held = [min(width, -(-x // page)) for x in lens]
    used = sum(held)
    pages = used + spare + 1
    ids = list(range(pages))
    rng.shuffle(ids)
    table = [[rng.randint(-5, pages + 5) for _ in range(width)] for _ in range(B)]
    for b in range(B):
        for p in range(held[b]):
            table[b][p] = ids.pop()
    free = ids
    c = _plan_cache(binding, B, page, pages, width)
    d_held, d_table = _i32(held), _i32(table)
    d_free = _i32(free + [12345] * (pages - len(free)))
    d_count = _i32([len(free)])
    for step in range(4):
        count = [rng.choice([n, rng.randint(0, n)]) for _ in range(B)] if step % 2 else None
        depth = [[rng.randint(0, 9) for _ in range(n)] for _ in range(B)] if step != 2 else None
        want = ref.plan(page, width, pages, lens, held, table, free, n, count, depth)
        slots, positions, status = c.plan(
            _i32(lens), d_held, d_table, d_free, d_count, n,
            count=None if count is None else _i32(count),
            depth=None if depth is None or n == 0 else _i32(depth))
        w_slots, w_pos, w_status, held, table, free = want
        assert status.tolist() == w_status, step
        assert d_held.tolist() == held
        assert d_count.tolist() == [len(free)]
        assert d_free.tolist()[:len(free)] == free
        assert d_table.tolist() == table            # (places past held as they were, too)
        if n:
            assert slots.tolist() == w_slots and positions.tolist() == w_pos
        assert c.device_error() == 0
        lens = [0 if rng.random() < 0.2 else max(0, min(x + rng.randint(-30, 20), held[b] * page))
                for b, x in enumerate(lens)]
    c.close()


def test_plan_returns_what_it_took(binding):
    """Rows planned and dropped again: tables, free list and counts end as they began."""
    B, page, width = 300, 16, 40
    rng = random.Random(5)
    lens = [rng.randint(0, 500) for _ in range(B)]
    held = [-(-x // page) for x in lens]
    pages = sum(held) + 5 * B
    ids = torch.randperm(pages, generator=torch.Generator().manual_seed(1)).int().cuda()
    table = torch.zeros((B, width), dtype=torch.int32, device="cuda")
    at = 0
    for b in range(B):
        table[b, :held[b]] = ids[at:at + held[b]]
        at += held[b]
    free = torch.cat([ids[at:], ids[:at]])
    state = [_i32(held), table, free, _i32([pages - at])]
    before = [t.clone() for t in state]
    c = _plan_cache(binding, B, page, pages, width)
    c.plan(_i32(lens), *state, 61)
    assert not torch.equal(state[0], before[0])
    c.plan(_i32(lens), *state, 0)
    for x, y, k in zip(state, before, ("held", "table", "free", "count")):
        if k == "table":
            x = torch.where(torch.arange(width, device="cuda") < before[0][:, None], x, 0)
        assert torch.equal(x, y), k
    c.close()


@pytest.mark.parametrize("kw", [dict(lens=[-1, 5]), dict(held=[9, 0]), dict(held=[0, -1]),
                                dict(count=[5, -1]), dict(count=[4, 0]), dict(free_count=[-1]),
                                dict(free_count=[11])])
def test_plan_flags_bad_data(binding, kw):
    base = dict(lens=[3, 5], held=[1, 1], count=[3, 3], free_count=[6])
    base.update(kw)
    c = _plan_cache(binding, 2, 16, 10, 4)
    table = _i32([[0, 1, 2, 3], [4, 5, 6, 7]])
    slots, positions, status = c.plan(_i32(base["lens"]), _i32(base["held"]), table,
                                      _i32(list(range(10))), _i32(base["free_count"]), 3,
                                      count=_i32(base["count"]))
    assert c.device_error() & 1
    assert ((slots >= -1) & (slots < 160)).all()
    c.close()


# -- write ------------------------------------------------------------------------

WRITES = [
    # dtype, B, n, H, K, D, page, rot, pairs, norm, fused
    (BF16, 1, 1, 4, 2, 128, 16, 128, False, True, True),
    (BF16, 2, 61, 32, 8, 128, 64, 128, False, True, True),
    (F16, 3, 17, 5, 5, 128, 16, 64, False, False, False),
    (F16, 2, 9, 8, 1, 64, 1, 64, True, True, True),
    (BF16, 1, 33, 7, 7, 80, 32, 80, False, True, False),
    (F16, 2, 5, 6, 3, 80, 16, 40, False, True, True),
    (BF16, 2, 5, 6, 3, 112, 16, 56, True, True, True),
    (BF16, 2, 5, 6, 3, 112, 16, 56, False, False, True),
    (F16, 1, 11, 4, 4, 160, 8, 80, False, True, True),
    (BF16, 3, 7, 16, 2, 256, 256, 256, False, True, True),
    (BF16, 3, 7, 2, 2, 256, 4, 2, False, True, True),
    (F16, 1, 3, 3, 1, 8, 2, 8, False, True, False),
    (BF16, 1, 3, 3, 1, 16, 2, 6, False, True, True),
    (F16, 1, 700, 4, 1, 24, 64, 0, False, True, True),
    (BF16, 5, 900, 4, 4, 64, 64, 0, True, False, True),
]


def _rows(g, B, n, H, K, D, dtype, fused):
    if fused:
        x = torch.randn((B, n, (H + 2 * K) * D), generator=g).to(dtype).cuda()
        q, k, v = x.split([H * D, K * D, K * D], dim=2)
        return q.unflatten(2, (H, D)), k.unflatten(2, (K, D)), v.unflatten(2, (K, D))
    return tuple(torch.randn((B, n, h, D), generator=g).to(dtype).cuda() for h in (H, K, K))


def _table(r, most, g):
    a = torch.arange(most, dtype=torch.float64)[:, None] * \
        10000.0 ** (-torch.arange(r // 2, dtype=torch.float64) / max(1, r // 2))
    return torch.cat([a.cos(), a.sin()], 1).float()


@pytest.mark.parametrize("dtype,B,n,H,K,D,page,rot,pairs,norm,fused", WRITES)
@pytest.mark.parametrize("in_place", [False, True])
def test_write_matches_the_plain_form(binding, dtype, B, n, H, K, D, page, rot, pairs, norm, fused,
                                      in_place):
    g = torch.Generator().manual_seed(n * D + rot)
    q, k, v = _rows(g, B, n, H, K, D, dtype, fused)
    pages = -(-B * n // page) + 3
    order = torch.randperm(pages * page, generator=g)[:B * n].view(B, n)
    order[torch.rand((B, n), generator=g) < 0.1] = -1
    positions = torch.randint(0, 500, (B, n), generator=g)
    rotation = _table(rot, 500, g) if rot else None
    qw, kw = ((1 + 0.3 * torch.randn((2, D), generator=g)).to(dtype) if norm else (None, None))
    kc, vc = (torch.randn((pages, page, K, D), generator=g).to(dtype) for _ in range(2))
    c = binding.Cache(batch=B, heads=H, kv_heads=K, head_dim=D, page_size=page, pages=pages,
                      table_width=1, dtype=dtype)
    d_kc, d_vc = kc.cuda(), vc.cuda()
    q0, k0, v0 = (t.cpu() for t in (q, k, v))
    out = q if in_place else torch.full((B, n, H, D), 7.0, dtype=dtype, device="cuda")
    got = c.write(q, k, v, order.cuda(), d_kc, d_vc,
                  positions=positions.int().cuda() if rot else None,
                  rotation=None if rotation is None else rotation.cuda(), interleaved=pairs,
                  q_weight=None if qw is None else qw.cuda(),
                  k_weight=None if kw is None else kw.cuda(), eps=1e-5, out=out)
    assert got is out and c.device_error() == 0
    live = order.flatten() >= 0
    at = order.flatten()[live]
    u = ref.U[dtype]
    pos = positions.flatten()
    for x, w, y in ((q0, qw, out), (k0, kw, d_kc)):
        want, size = ref.write_heads(x.flatten(0, 1), w, 1e-5, rotation, pos, pairs)
        tol = u * want.abs() * 1.001 + ref.U32 * size * 1.001 + ref.TINY[dtype] * 1.001
        y = y.cpu().double()
        if y.shape == (pages, page, K, D):
            flat = y.flatten(0, 1)
            assert ((flat[at] - want[live]).abs() <= tol[live]).all()
            rest = torch.ones(pages * page, dtype=torch.bool)
            rest[at] = False
            assert torch.equal(flat[rest], kc.double().flatten(0, 1)[rest])
        else:
            y = y.flatten(0, 1)
            assert ((y[live] - want[live]).abs() <= tol[live]).all()
            left = x.double().flatten(0, 1)[~live] if in_place else \
                torch.full_like(y[~live], 7.0)
            assert torch.equal(y[~live], left)
    want_v = vc.flatten(0, 1).clone()
    want_v[at] = v0.flatten(0, 1)[live]
    assert torch.equal(d_vc.cpu().flatten(0, 1), want_v)
    c.close()


def test_write_keys_alone_and_pages_apart(binding):
    """No q; pages with keys and values side by side (a page stride of its own)."""
    B, n, K, D, page, pages = 2, 10, 2, 64, 8, 5
    g = torch.Generator().manual_seed(3)
    _, k, v = _rows(g, B, n, 2, K, D, BF16, False)
    both = torch.zeros((pages, 2, page, K, D), dtype=BF16, device="cuda")
    c = binding.Cache(batch=B, heads=4, kv_heads=K, head_dim=D, page_size=page, pages=pages,
                      table_width=1, page_stride=2 * page * K * D)
    slots = torch.randperm(pages * page, generator=g)[:B * n].view(B, n).cuda()
    assert c.write(None, k, v, slots, both[:, 0], both[:, 1]) is None
    want = torch.zeros((2, pages * page, K, D), dtype=BF16, device="cuda")
    want[0, slots.flatten()] = k.flatten(0, 1)
    want[1, slots.flatten()] = v.flatten(0, 1)
    assert torch.equal(both, want.view(2, pages, page, K, D).transpose(0, 1))
    c.close()


def test_write_flags_bad_slots_and_positions(binding):
    B, n, K, D, page, pages = 1, 3, 1, 64, 8, 2
    k = torch.ones((B, n, K, D), dtype=BF16, device="cuda")
    kc, vc = (torch.zeros((pages, page, K, D), dtype=BF16, device="cuda") for _ in range(2))
    rot = torch.ones((4, D), device="cuda")
    for slots, pos, bit in (([[0, 16, 1]], [[0, 1, 2]], 2), ([[0, 1 << 40, 1]], [[0, 1, 2]], 2),
                            ([[0, 3, 1]], [[0, 4, 2]], 4), ([[0, 3, 1]], [[0, -1, 2]], 4)):
        c = binding.Cache(batch=B, heads=1, kv_heads=K, head_dim=D, page_size=page, pages=pages,
                          table_width=1)
        kc.zero_()
        c.write(None, k, k, torch.tensor(slots, device="cuda"), kc, vc, positions=_i32(pos),
                rotation=rot)
        assert c.device_error() == bit
        assert kc.flatten(0, 1).abs().sum((1, 2)).nonzero()[:, 0].tolist() == [0, 1]
        c.close()


# -- attention ----------------------------------------------------------------------


class Setup:
    """A cache with random pages and sequences of given lengths."""

    def __init__(self, binding, dtype, lens, n, tail, H, K, D, page, seed=0, apart=False, spread=1.0):
        g = torch.Generator().manual_seed(seed)
        self.g, self.dtype, self.lens, self.n, self.tail = g, dtype, lens, n, tail
        self.H, self.K, self.D, self.page = H, K, D, page
        B = len(lens)
        self.B, self.width = B, max(1, -(-(max(lens) + tail) // page)) + 1
        needs = [-(-(x + tail) // page) for x in lens]
        self.pages = sum(needs) + 1
        ids = torch.randperm(self.pages, generator=g)
        self.table = torch.full((B, self.width), -7, dtype=torch.int32)
        at = 0
        for b in range(B):
            self.table[b, :needs[b]] = ids[at:at + needs[b]]
            at += needs[b]
        self.kc, self.vc = (torch.randn((self.pages, page, K, D), generator=g).to(dtype)
                            for _ in range(2))
        self.q = (torch.randn((B, n, H, D), generator=g) * spread).to(dtype)
        self.cache = binding.Cache(batch=B, heads=H, kv_heads=K, head_dim=D, page_size=page,
                                   pages=self.pages, table_width=self.width, dtype=dtype,
                                   page_stride=2 * page * K * D if apart else 0)
        self.apart = apart

    def entries(self, cache, b, L):
        e = torch.arange(L)
        return cache.flatten(0, 1)[self.table[b].long()[e // self.page] * self.page + e % self.page]

    def pages_on_gpu(self):
        if not self.apart:
            return self.kc.cuda(), self.vc.cuda()
        both = torch.stack([self.kc, self.vc], 1).cuda()
        return both[:, 0], both[:, 1]

    def run(self, mask=None, count=None, scale=None, fused=False, **kw):
        q = self.q.cuda()
        if fused:                                    # rows of a wider matrix
            wide = torch.zeros((self.B, self.n, self.H * self.D + 64), dtype=self.dtype, device="cuda")
            wide[..., :self.H * self.D] = q.flatten(2)
            q = wide[..., :self.H * self.D].unflatten(2, (self.H, self.D))
        out = torch.full((self.B, self.n, self.H, self.D), 9.0, dtype=self.dtype, device="cuda")
        lse = torch.full((self.B, self.n, self.H), 9.0, device="cuda")
        kc, vc = self.pages_on_gpu()
        self.cache.attention(q, kc, vc, self.table.cuda(), _i32(self.lens),
                             mask=None if mask is None else mask.cuda(), tail=self.tail,
                             count=None if count is None else _i32(count), scale=scale, out=out,
                             lse=lse, **kw)
        assert self.cache.device_error() == 0
        return out.cpu(), lse.cpu()

    def check(self, got, mask=None, count=None, scale=None, only=None):
        scale = self.D ** -0.5 if scale is None else scale
        count = [self.n] * self.B if count is None else count
        out, lse = got
        for b in only or range(self.B):
            rows, tail = count[b], self.tail - (self.n - count[b])
            assert (out[b, rows:] == 9).all() and (lse[b, rows:] == 9).all()
            if not rows:
                continue
            tail = max(tail, 0)
            L = self.lens[b] + tail
            seen = torch.ones((rows, L), dtype=torch.bool)
            if mask is not None:
                seen[:, self.lens[b]:] = mask[b, :rows, :tail] != 0
            else:
                i, j = torch.arange(rows)[:, None], torch.arange(tail)[None, :]
                seen[:, self.lens[b]:] = j <= i + self.tail - self.n
            want, w_lse, tol, tol_lse = ref.attention(
                self.q[b, :rows], self.entries(self.kc, b, L), self.entries(self.vc, b, L), seen,
                scale, self.dtype)
            off = (out[b, :rows].double() - want).abs()
            assert (off <= tol).all(), (b, float((off - tol).max()), float(off.max()))
            none = w_lse == -math.inf
            assert (lse[b, :rows][none] == -math.inf).all()
            off = (lse[b, :rows].double() - w_lse).abs()[~none]
            assert (off <= tol_lse[~none]).all(), (b, float(off.max()))


def _tree_mask(g, B, n):
    mask = torch.zeros((B, n, n), dtype=torch.uint8)
    for b in range(B):
        for i in range(n):
            if i:
                mask[b, i] = mask[b, int(torch.randint(0, i, (1,), generator=g))]
            mask[b, i, i] = 1
    return mask


ATTENTION = [
    # dtype, lens, n, H, K, D, page
    (BF16, [0], 1, 1, 1, 128, 16), (BF16, [1], 1, 4, 1, 64, 16), (F16, [517], 1, 32, 8, 128, 64),
    (BF16, [33, 0, 700, 129], 1, 8, 2, 128, 16), (F16, [31, 32, 33, 127, 128, 129], 1, 7, 1, 80, 1),
    (BF16, [1000, 5], 13, 4, 2, 128, 16), (F16, [64, 300], 16, 8, 8, 64, 32),
    (BF16, [250, 77], 61, 4, 4, 128, 64), (F16, [130], 61, 8, 4, 112, 16),
    (BF16, [500, 3, 0], 61, 8, 2, 128, 64), (F16, [1029], 81, 12, 4, 64, 128),
    (BF16, [90], 100, 10, 2, 160, 16), (BF16, [260, 11], 61, 5, 5, 256, 16),
    (F16, [100], 40, 8, 1, 256, 8), (BF16, [7, 200], 3, 8, 2, 200, 4), (F16, [70], 5, 3, 3, 8, 2),
    (BF16, [40], 20, 6, 2, 24, 4096), (BF16, [2100], 61, 4, 1, 128, 256),
]


@pytest.mark.parametrize("dtype,lens,n,H,K,D,page", ATTENTION)
@pytest.mark.parametrize("kind", ["causal", "tree", "ragged", "sparse"])
def test_attention_matches_the_plain_form(binding, dtype, lens, n, H, K, D, page, kind):
    s = Setup(binding, dtype, lens, n, n, H, K, D, page, seed=n + D)
    mask = count = None
    if kind in ("tree", "ragged"):
        mask = _tree_mask(s.g, s.B, n)
    if kind == "ragged":
        count = [int(x) for x in torch.randint(0, n + 1, (s.B,), generator=s.g)]
    if kind == "sparse":                              # any mask, some rows naming nothing
        mask = (torch.rand((s.B, n, n), generator=s.g) < 0.2).to(torch.uint8) * 255
        mask[:, ::3] = 0
    s.check(s.run(mask, count), mask, count)
    s.cache.close()


@pytest.mark.parametrize("dtype,lens,n,tail,H,K,D,page", [
    (BF16, [100, 0], 4, 20, 8, 2, 128, 16), (F16, [65], 8, 9, 4, 4, 64, 16),
    (BF16, [3], 1, 200, 4, 1, 128, 32)])
@pytest.mark.parametrize("masked", [False, True])
def test_attention_of_some_of_the_entries_rows(binding, dtype, lens, n, tail, H, K, D, page, masked):
    """A draft level: its rows behind the entries of the levels before it."""
    s = Setup(binding, dtype, lens, n, tail, H, K, D, page, seed=tail)
    mask = (torch.rand((s.B, n, tail), generator=s.g) < 0.4).to(torch.uint8) if masked else None
    s.check(s.run(mask), mask)
    count = [max(0, n - 2)] * s.B
    s.check(s.run(mask, count), mask, count)
    s.cache.close()


def test_attention_with_fewer_entries_than_rows(binding):
    """tail < n (with a mask): the rows look at a few entries behind the prefix, or none."""
    for tail in (0, 3):
        s = Setup(binding, BF16, [40, 0], 6, tail, 4, 2, 64, 16, seed=tail)
        mask = torch.ones((2, 6, tail), dtype=torch.uint8)
        s.check(s.run(mask), mask)
        s.cache.close()


def test_attention_strides_and_scale(binding):
    s = Setup(binding, BF16, [90, 300], 61, 61, 8, 2, 128, 16, apart=True)
    mask = _tree_mask(s.g, 2, 61)
    s.check(s.run(mask, scale=0.3, fused=True), mask, scale=0.3)
    s.cache.close()


@pytest.mark.parametrize("n,H,K", [(1, 8, 8), (61, 4, 1), (61, 1, 1), (30, 4, 2)])
def test_attention_of_a_long_sequence(binding, n, H, K):
    """Items cut into many stretches, joined again; scores that grow along the cache."""
    s = Setup(binding, BF16, [9000], n, n, H, K, 64, 16, seed=n, spread=2.0)
    mask = _tree_mask(s.g, 1, n)
    s.check(s.run(mask), mask)
    s.cache.close()


@pytest.mark.parametrize("n", [300, 700])
def test_attention_of_many_rows(binding, n):
    """More rows than a workgroup holds, causal and under a mask."""
    s = Setup(binding, F16, [50, 0], n, n, 2, 1, 64, 64, seed=n)
    s.check(s.run())
    mask = (torch.rand((2, n, n), generator=s.g) < 0.05).to(torch.uint8)
    count = [n - 1, 77]
    s.check(s.run(mask, count), mask, count)
    s.cache.close()


@pytest.mark.parametrize("B,n,H,K,D,lens", [
    (70, 31, 16, 4, 64, "even"), (40, 61, 32, 8, 128, "even"), (40, 61, 32, 8, 128, "uneven"),
    (256, 61, 4, 1, 64, "even"), (257, 61, 4, 1, 64, "even"), (90, 31, 32, 8, 64, "ragged"),
    (70, 31, 16, 4, 160, "same")])
def test_attention_of_many_sequences(binding, B, n, H, K, D, lens):
    """More items than workgroups: given out whole where lengths even out, else in
    stretches; sequences without rows among them."""
    rng = random.Random(B + n)
    lengths = [{"even": rng.randint(20, 300), "ragged": rng.randint(0, 90), "same": 77,
                "uneven": 1500 if b == 3 else 10}[lens] for b in range(B)]
    s = Setup(binding, BF16, lengths, n, n, H, K, D, 16, seed=B)
    mask = _tree_mask(s.g, 1, n).expand(B, n, n).contiguous()
    count = [rng.choice([0, 1, n, n]) for _ in range(B)] if lens == "ragged" else None
    got = s.run(mask, count)
    longest = max(range(B), key=lambda b: lengths[b])
    only = {0, B - 1, longest, rng.randrange(B)}
    s.check(got, mask, count, only=only)
    # the others, against a run in the reversed order, which is given out otherwise: each is off
    # the exact result by at most 2^-8 |o| + (2^-8 + small) sum p |v| with |v| below 6 here, so
    # the two by twice that
    back = list(reversed(range(B)))
    t = Setup(binding, BF16, lengths, n, n, H, K, D, 16, seed=B)
    t.lens, t.q, t.table = [lengths[b] for b in back], s.q[back], s.table[back]
    again = t.run(mask, None if count is None else [count[b] for b in back])
    off = (again[0][back].float() - got[0].float()).abs()
    assert float(s.vc.float().abs().max()) < 6
    assert (off <= 2 * 2.0 ** -8 * (got[0].float().abs() + 1.1 * 6)).all()
    s.cache.close(), t.cache.close()


@pytest.mark.parametrize("dtype,n,H,K,D", [(BF16, 61, 8, 2, 128), (F16, 61, 4, 4, 128),
                                           (BF16, 4, 4, 2, 64), (F16, 61, 2, 1, 256),
                                           (BF16, 61, 2, 2, 64)])
def test_what_is_not_attended_has_no_effect(binding, dtype, n, H, K, D):
    """NaN and infinities in entries that some rows mask, in entries that all do, behind the
    last entry of each sequence and in pages of nobody: rows that do not attend them get
    the result that they get without, bit for bit; rows that do get NaN or inf."""
    s = Setup(binding, dtype, [70, 0, 127], n, n, H, K, D, 16, seed=1)
    mask = _tree_mask(s.g, 3, n)
    mask[:, :, n - 2] = 0                             # nobody's, not even its own
    count = [n, n - 1, max(1, n // 2)]
    clean = s.run(mask, count)
    s.check(clean, mask, count)
    named = torch.zeros(s.pages * s.page, dtype=torch.bool)
    rng = random.Random(2)
    odd = {}
    for b in range(3):
        e = torch.arange(s.lens[b] + count[b])
        at = s.table[b].long()[e // s.page] * s.page + e % s.page
        named[at] = True
        odd[b] = rng.randrange(1, count[b]) if count[b] > 2 else 1
        for j in {odd[b], n - 2}:
            if j >= count[b]:
                continue
            slot = int(at[s.lens[b] + j])
            for cache, value in ((s.kc, math.nan), (s.vc, math.inf)):
                cache.flatten(0, 1)[slot, :, ::3] = value
                cache.flatten(0, 1)[slot, :, 1] = -math.inf
    for cache in (s.kc, s.vc):
        cache.flatten(0, 1)[~named] = math.nan
    out, lse = s.run(mask, count)
    for b in range(3):
        for i in range(count[b]):
            if not mask[b, i, odd[b]] or odd[b] >= count[b]:
                assert torch.equal(out[b, i], clean[0][b, i]), (b, i)
                assert torch.equal(lse[b, i], clean[1][b, i])
            else:
                assert not torch.isfinite(lse[b, i].float()).any()
    s.cache.close()


def test_infinite_values_reach_the_rows_that_attend_them(binding):
    """An infinite value (with an ordinary key) of a drafted entry: its rows' elements are
    infinite, every other element is as without it."""
    s = Setup(binding, BF16, [37], 20, 20, 4, 2, 128, 16, seed=4)
    mask = _tree_mask(s.g, 1, 20)
    clean = s.run(mask)
    e = 37 + 5
    slot = int(s.table[0, e // 16]) * 16 + e % 16
    s.vc.flatten(0, 1)[slot, 1, 17] = math.inf
    s.vc.flatten(0, 1)[slot, 1, 90] = -math.inf
    out, lse = s.run(mask)
    assert torch.equal(lse, clean[1])
    want, w_lse, tol, _ = ref.attention(s.q[0], s.entries(s.kc, 0, 57), s.entries(s.vc, 0, 57),
                                        torch.cat([torch.ones((20, 37)).bool(), mask[0] != 0], 1),
                                        128 ** -0.5, BF16)
    for i in range(20):
        if mask[0, i, 5]:
            assert (out[0, i, 2:, 17] == math.inf).all() and (out[0, i, 2:, 90] == -math.inf).all()
            fine = torch.isfinite(want[i])
            off = (out[0, i].double() - want[i]).abs()
            assert (off[fine] <= tol[i][fine]).all()
        else:
            assert torch.equal(out[0, i], clean[0][0, i])
    s.cache.close()


@pytest.mark.parametrize("n,H,K", [(20, 4, 2), (1, 4, 1), (61, 4, 1)])
def test_infinite_values_of_the_prefix_reach_all_rows(binding, n, H, K):
    """In the tile that the drafted entries begin in, in one before it, next to the last."""
    s = Setup(binding, F16, [337], n, n, H, K, 64, 16, seed=4)
    mask = _tree_mask(s.g, 1, n)
    clean = s.run(mask)
    for e, d in ((3, 5), (336, 17), (330, 40)):
        s.vc.flatten(0, 1)[int(s.table[0, e // 16]) * 16 + e % 16, :, d] = math.inf
    out, lse = s.run(mask)
    assert torch.equal(lse, clean[1])
    for d in range(64):
        if d in (5, 17, 40):
            assert (out[..., d] == math.inf).all()
        else:
            assert torch.equal(out[..., d], clean[0][..., d])
    s.cache.close()


def test_attention_flags_pages_outside_the_pool(binding):
    s = Setup(binding, BF16, [70], 3, 3, 4, 2, 64, 16)
    for bad in (-1, s.pages, 1 << 30):
        c = binding.Cache(batch=1, heads=4, kv_heads=2, head_dim=64, page_size=16, pages=s.pages,
                          table_width=s.width)
        table = s.table.clone()
        table[0, 1] = bad
        c.attention(s.q.cuda(), s.kc.cuda(), s.vc.cuda(), table.cuda(), _i32([70]))
        assert c.device_error() == 8
        c.close()
    for lens in (-1, s.width * 16 - 2, 2 ** 31 - 1):
        c = binding.Cache(batch=1, heads=4, kv_heads=2, head_dim=64, page_size=16, pages=s.pages,
                          table_width=s.width)
        c.attention(s.q.cuda(), s.kc.cuda(), s.vc.cuda(), s.table.clamp(min=0).cuda(), _i32([lens]))
        assert c.device_error() == 32
        c.close()
    for count in (-1, 4):
        c = binding.Cache(batch=1, heads=4, kv_heads=2, head_dim=64, page_size=16, pages=s.pages,
                          table_width=s.width)
        c.attention(s.q.cuda(), s.kc.cuda(), s.vc.cuda(), s.table.cuda(), _i32([70]),
                    count=_i32([count]))
        assert c.device_error() == 1
        c.close()
    s.cache.close()


# -- commit -------------------------------------------------------------------------


def _drafted(rng, n, depth):
    parent, token, level = [-1], [-1], [0]
    for i in range(1, n):
        p = rng.choice([j for j in range(i) if level[j] < depth])
        parent.append(p), level.append(level[p] + 1)
        taken = {token[j] for j in range(1, i) if parent[j] == p}
        token.append(rng.choice([t for t in range(n + 3) if t not in taken]))
    return parent, token


def _walk(rng, parent, token, most):
    path = [0]
    while len(path) <= most:
        kids = [i for i in range(len(parent)) if parent[i] == path[-1]]
        if not kids or rng.random() < 0.15:
            break
        path.append(rng.choice(kids))
    return path


@pytest.mark.parametrize("B,n,depth,layers,K,D,page,in_place,apart", [
    (1, 61, 7, 3, 8, 128, 64, True, False), (5, 20, 15, 2, 2, 64, 16, False, True),
    (9, 81, 8, 1, 1, 80, 1, True, False), (3, 2, 1, 4, 4, 256, 8, False, False),
    (40, 40, 6, 2, 5, 128, 32, True, False), (2, 1, 3, 1, 1, 8, 16, False, False),
    (1, 500, 15, 2, 1, 64, 16, True, True)])
def test_commit_moves_the_accepted_path(binding, B, n, depth, layers, K, D, page, in_place, apart):
    rng = random.Random(n * depth)
    g = torch.Generator().manual_seed(n)
    lens = [rng.randint(0, 60) for _ in range(B)]
    width = max(-(-(x + n) // page) for x in lens)
    pages = B * width
    table = torch.randperm(pages, generator=g).view(B, width)
    trees = [_drafted(rng, n, depth) for _ in range(B)]
    paths = [_walk(rng, *t, depth) for t in trees]
    took = [len(p) - 1 for p in paths]
    if B > 2:
        took[1] = -1                                  # a failed walk
    accepted = [[trees[b][1][x] for x in p[1:]] + [-1] * (depth - len(p) + 1)
                for b, p in enumerate(paths)]
    shape = (layers, pages, page, K, D)
    kc, vc = torch.randn(shape, generator=g).to(BF16), torch.randn(shape, generator=g).to(BF16)
    c = binding.Cache(batch=B, heads=K, kv_heads=K, head_dim=D, page_size=page, pages=pages,
                      table_width=width, layers=layers,
                      page_stride=2 * page * K * D if apart else 0,
                      layer_stride=2 * pages * page * K * D if apart else 0)
    if apart:
        both = torch.stack([kc, vc], 2).cuda()
        d_kc, d_vc = both[:, :, 0], both[:, :, 1]
    else:
        d_kc, d_vc = kc.cuda(), vc.cuda()
    d_lens = _i32(lens)
    new = d_lens if in_place else torch.zeros_like(d_lens)
    path = torch.full((B, depth + 1), 99, dtype=torch.int32, device="cuda")
    c.commit(_i32([t[0] for t in trees]), _i32([t[1] for t in trees]), _i32(accepted),
             _i32(took), d_lens, table.int().cuda(), d_kc, d_vc, out=(path, new))
    assert c.device_error() == 0
    assert new.tolist() == [x + 1 + k if k >= 0 else x for x, k in zip(lens, took)]
    for b in range(B):
        want = [-1] * (depth + 1)
        if took[b] >= 0:
            want[:len(paths[b])] = paths[b]
            for cache in (kc, vc):
                flat = cache.flatten(1, 2)
                slot = [int(table[b, (lens[b] + e) // page]) * page + (lens[b] + e) % page
                        for e in range(n)]
                flat[:, [slot[j] for j in range(len(paths[b]))]] = \
                    flat[:, [slot[j] for j in paths[b]]].clone()
        assert path[b].tolist() == want
    assert torch.equal(d_kc.cpu(), kc) and torch.equal(d_vc.cpu(), vc)
    c.close()


@pytest.mark.parametrize("kw,bit", [
    (dict(accepted=[[9, -1]], took=[1]), 16), (dict(accepted=[[5, 5]], took=[2]), 16),
    (dict(took=[3]), 16), (dict(lens=[-1]), 32), (dict(lens=[127]), 32), (dict(lens=[126]), 32),
    (dict(lens=[2 ** 31 - 1]), 32), (dict(table=[[0, -1, 1, 2]]), 8), (dict(table=[[0, 4, 1, 2]]), 8)])
def test_commit_flags_bad_data(binding, kw, bit):
    base = dict(lens=[33], accepted=[[5, 6]], took=[2], table=[[0, 1, 2, 3]])
    base.update(kw)
    kc = torch.randn((1, 4, 32, 1, 64), device="cuda").to(BF16)
    vc = kc.clone()
    k0 = kc.clone()
    c = binding.Cache(batch=1, heads=1, kv_heads=1, head_dim=64, page_size=32, pages=4,
                      table_width=4)
    path, new = c.commit(_i32([[-1, 0, 0, 2]]), _i32([[-1, 4, 5, 6]]), _i32(base["accepted"]),
                         _i32(base["took"]), _i32(base["lens"]), _i32(base["table"]), kc, vc)
    assert c.device_error() == bit
    assert path.tolist() == [[-1, -1, -1]] and new.tolist() == base["lens"]
    assert torch.equal(kc, k0) and torch.equal(vc, k0)
    c.close()


@pytest.mark.parametrize("parent,accepted", [([-1, 2, 0, 1], [5, 4]), ([-1, 3, 0, 0], [6, 4])])
def test_commit_of_children_ahead_of_their_parents_is_flagged(binding, parent, accepted):
    """No tree has them, and moves along such a path would read what they have written."""
    kc = torch.randn((1, 4, 32, 1, 64), device="cuda").to(BF16)
    vc, k0 = kc.clone(), kc.clone()
    c = binding.Cache(batch=1, heads=1, kv_heads=1, head_dim=64, page_size=32, pages=4,
                      table_width=4)
    path, new = c.commit(_i32([parent]), _i32([[-1, 4, 5, 6]]), _i32([accepted]), _i32([2]),
                         _i32([33]), _i32([[0, 1, 2, 3]]), kc, vc)
    assert c.device_error() == 16
    assert path.tolist() == [[-1, -1, -1]] and new.tolist() == [33]
    assert torch.equal(kc, k0) and torch.equal(vc, k0)
    c.close()
