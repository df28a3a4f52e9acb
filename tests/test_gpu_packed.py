"""The operators of the 4-bit cache (append, read, attention, commit) against plain 64-bit
forms."""

import math
import random

import pytest
import torch

import cache_oracle
import packed_oracle as ref

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


def _bytes(shape, seed):
    return torch.randint(0, 256, shape, dtype=torch.uint8, generator=torch.Generator().manual_seed(seed))


def _normal(shape, dtype, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale).to(dtype)


def _values(shape, dtype, seed):
    """Normal values, whole blocks scaled up and down over the type's range, zeros, ties."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(shape, generator=g, dtype=torch.float64)
    low, high = (-130, 126) if dtype == BF16 else (-26, 15)
    pick = torch.rand(shape[:-1], generator=g)
    power = torch.randint(low, high, shape[:-1], generator=g).double()
    x = x * 2.0 ** torch.where(pick < 0.3, power, torch.zeros_like(power))[..., None]
    half = torch.randint(-28, 29, shape, generator=g).double() / 4    # codes and their borders
    x = torch.where((pick > 0.6)[..., None], half, x)
    x = torch.where((pick > 0.95)[..., None], torch.zeros_like(x), x)
    most = torch.finfo(dtype).max
    return x.clamp(-most, most).to(dtype)


# -- append and read ----------------------------------------------------------------

ROWS = [
    # dtype, B, n, K, D, page, layers (None: pages without that dimension)
    (BF16, 1, 1, 1, 8, 16, None), (BF16, 1, 1, 8, 128, 64, None), (F16, 3, 7, 2, 64, 16, None),
    (BF16, 2, 33, 5, 80, 32, 2), (F16, 1, 61, 3, 112, 16, 3), (BF16, 4, 9, 1, 256, 4096, None),
    (F16, 2, 20, 4, 160, 64, 1), (BF16, 1, 130, 2, 200, 128, None), (F16, 5, 11, 2, 24, 16, 2),
    (BF16, 2, 5, 40, 32, 16, None), (F16, 1, 3, 1, 232, 16, None), (BF16, 1, 700, 2, 96, 64, None),
]


def _cache(binding, B, K, D, page, pages, dtype, layers=1, H=None, width=1):
    return binding.PackedCache(batch=B, heads=H or K, kv_heads=K, head_dim=D, page_size=page,
                               pages=pages, table_width=width, layers=layers, dtype=dtype)


def _row_slots(B, n, pages, page, seed, skip=0.15):
    rng = random.Random(seed)
    s = rng.sample(range(pages * page), B * n)
    return torch.tensor([-1 if rng.random() < skip else x for x in s]).view(B, n)


@pytest.mark.parametrize("dtype,B,n,K,D,page,layers", ROWS)
def test_rows_are_packed_and_read_back(binding, dtype, B, n, K, D, page, layers):
    """Bytes equal to the plain form's, those of other entries left alone; values read back
    equal, rows without a slot left alone."""
    pages = -(-B * n // page) + 2
    many = (layers,) if layers is not None else ()
    slots = _row_slots(B, n, pages, page, B * 100 + n)
    shape = many + (B, n, K, D)
    k, v = _values(shape, dtype, 1), _values(shape, dtype, 2)
    size = many + (pages, K, ref.page_bytes(D, page))
    # (exponents of every page in range, as the library keeps them)
    kp, vp = _bytes(size, 3), _bytes(size, 4)
    c = _cache(binding, B, K, D, page, pages, dtype, layers or 1)
    assert c.page_bytes == ref.page_bytes(D, page)
    dk, dv = kp.cuda(), vp.cuda()
    c.append(k.cuda(), v.cuda(), slots.cuda(), dk, dv)
    for x, pool in ((k, kp), (v, vp)):
        for i in range(layers or 1):
            one, rows = (pool[i], x[i]) if many else (pool, x)
            ref.store(one, page, slots.flatten().tolist(), rows.flatten(0, 1))
    assert torch.equal(dk.cpu(), kp) and torch.equal(dv.cpu(), vp)
    assert c.device_error() == 0
    was = [_normal(shape, dtype, s) for s in (5, 6)]
    out = c.read(slots.cuda(), dk, dv, out=tuple(x.cuda() for x in was))
    live = (slots >= 0).flatten()
    for x, pool, y, old in zip((k, v), (kp, vp), out, was):
        for i in range(layers or 1):
            one, got, before = (pool[i], y[i], old[i]) if many else (pool, y, old)
            got, before = got.cpu().flatten(0, 1), before.flatten(0, 1)
            want = ref.load(one, page, slots.flatten().clamp(min=0), D)
            assert torch.equal(got[live].double(), want[live])
            assert torch.equal(got[~live], before[~live])
    # the values are those of the rows, off by half a step of the block's codes at most: 1/4
    # of its power of two to 1 (and the last eighth, 7 held as 6); the power is at most
    # a quarter of the largest magnitude, and 2^-125 (bf16), 2^-23 (fp16) at least
    got = ref.held(k)
    blocks = torch.nn.functional.pad((got - k.double()).abs(), (0, -D % 32)).unflatten(-1, (-1, 32))
    most = torch.nn.functional.pad(k.double().abs(), (0, -D % 32)).unflatten(-1, (-1, 32)).amax(-1)
    small = 2.0 ** ref.LOW[dtype]
    inside = most <= 6 * 2.0 ** ref.HIGH[dtype]
    assert (blocks.amax(-1) <= (most / 4).clamp(min=small))[inside].all()
    new = c.read(slots.cuda(), dk, dv)
    assert all((y.flatten(-4, -3)[..., (~live).cuda(), :, :] == 0).all() for y in new)
    c.close()


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_every_16_bit_value_is_packed_as_by_the_plain_form(binding, dtype):
    """All 65536 patterns, finite or not, each the largest of a block and beside others."""
    x = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(dtype).view(1024, 2, 32)
    g = torch.Generator().manual_seed(9)
    order = torch.randperm(65536, generator=g)
    y = torch.zeros((65536, 32), dtype=dtype)
    y[:, 0] = x.flatten()[order]
    finite = torch.isfinite(y[:, 0])
    near = (y[:, :1].float() * torch.rand((65536, 31), generator=g)).to(dtype)
    y[:, 1:] = torch.where(finite[:, None], near, torch.ones_like(near))
    rows = torch.cat([x.reshape(2048, 1, 1, 32), y.view(65536, 1, 1, 32)]).view(1, -1, 1, 32)
    n, page = rows.shape[1], 4096
    pages = -(-n // page)
    c = _cache(binding, 1, 1, 32, page, pages, dtype)
    pool = [torch.zeros((pages, 1, ref.page_bytes(32, page)), dtype=torch.uint8, device="cuda")
            for _ in range(2)]
    slots = torch.arange(n, device="cuda").view(1, n)
    c.append(rows.cuda(), rows.cuda(), slots, *pool)
    code, e = ref.pack(rows[0, :, 0])
    codes = pool[0][:, 0, :16 * page].reshape(-1, 16).cpu()[:n]
    got = torch.stack([codes % 16, codes // 16], -1).flatten(-2).long()
    bad = (got != code).any(-1)
    assert not bad.any(), (rows[0, bad][:2], got[bad][:2], code[bad][:2])
    assert torch.equal(pool[0][:, 0, 16 * page:].flatten().cpu()[:n].long() - 127, e[:, 0])
    assert torch.equal(pool[0], pool[1])
    assert c.device_error() == 64                      # there were infinities and NaN
    k, _ = c.read(slots, *pool)
    assert torch.equal(k[0, :, 0].cpu().double(), ref.value(code, e, 32))
    assert torch.isfinite(k).all()
    c.close()


def test_rows_and_pages_with_gaps(binding):
    """k inside a projection's output, pages and layers with room between them."""
    B, n, K, D, page, pages, layers = 2, 13, 3, 64, 32, 4, 2
    c = _cache(binding, B, K, D, page, pages, BF16, layers)
    qkv = _normal((layers, B, n, 12, D), BF16, 1).cuda()
    k, v = qkv[..., 3:6, :], qkv[..., 6:9, :]
    store = torch.zeros((layers, pages + 1, K + 2, c.page_bytes), dtype=torch.uint8, device="cuda")
    kp, vp = store[:, :pages, :K], torch.zeros_like(store)[:, :pages, :K]
    slots = _row_slots(B, n, pages, page, 3).cuda()
    c.append(k, v, slots, kp, vp)
    assert (store[:, pages] == 0).all() and (store[:, :, K:] == 0).all()
    dense = [torch.zeros((layers, pages, K, c.page_bytes), dtype=torch.uint8, device="cuda")
             for _ in range(2)]
    c.append(k.contiguous(), v.contiguous(), slots, *dense)
    assert torch.equal(kp, dense[0]) and torch.equal(vp, dense[1])
    out = torch.zeros((layers, B, n, 5, D), dtype=BF16, device="cuda")
    two = torch.zeros((layers, B, n, 5, D), dtype=BF16, device="cuda")
    c.read(slots, kp, vp, out=(out[..., 1:4, :], two[..., :3, :]))
    want = c.read(slots, *dense)
    assert torch.equal(out[..., 1:4, :], want[0]) and torch.equal(two[..., :3, :], want[1])
    assert (out[..., 0, :] == 0).all() and (out[..., 4, :] == 0).all()
    c.close()


@pytest.mark.parametrize("call", ["append", "read"])
def test_slots_out_of_range_set_the_flag(binding, call):
    B, n, K, D, page, pages = 1, 4, 2, 32, 16, 3
    c = _cache(binding, B, K, D, page, pages, F16)
    room = torch.zeros((pages + 4, K, c.page_bytes), dtype=torch.uint8, device="cuda")
    kp, vp = room[2:2 + pages], room[2:2 + pages].clone()
    slots = torch.tensor([[47, 48, 2 ** 40, -3]], device="cuda")
    k = torch.ones((B, n, K, D), dtype=F16, device="cuda")
    if call == "append":
        c.append(k, k, slots, kp, vp)
        assert (room[:2] == 0).all() and (room[2 + pages:] == 0).all() and (kp[2] != 0).any()
    else:
        out, _ = c.read(slots, kp, vp, out=(k.clone(), k.clone()))
        assert torch.equal(out[0, 1:], k[0, 1:]) and (out[0, 0] == 0).all()
    assert c.device_error() == 2
    c.close()


def test_offsets_past_32_bits(binding):
    """A pool of more than 4 GiB, its last page read and written."""
    K, D, page = 8, 256, 4096
    pages = 1 << 31
    pages = pages // (page * 8 * 17 * K) * 2 + 4       # some 4.5 GiB of each
    c = _cache(binding, 1, K, D, page, pages, BF16, width=pages)
    assert pages * K * c.page_bytes > 1 << 32
    kp = torch.zeros((pages, K, c.page_bytes), dtype=torch.uint8, device="cuda")
    vp = torch.zeros_like(kp)
    n = 3
    k, v = _normal((1, n, K, D), BF16, 1), _normal((1, n, K, D), BF16, 2)
    slots = torch.tensor([[pages * page - 1, (pages - 1) * page, 5]], device="cuda")
    c.append(k.cuda(), v.cuda(), slots, kp, vp)
    got = c.read(slots, kp, vp)
    for x, y in zip((k, v), got):
        assert torch.equal(y.cpu().double(), ref.held(x))
    # attended, too: the last page as the sequence's first
    q = _normal((1, 1, K, D), BF16, 3)
    table = torch.zeros((1, pages), dtype=torch.int32, device="cuda")
    table[0, 0] = pages - 1
    out = c.attention(q.cuda(), kp, vp, table, _i32([1])).cpu()
    assert torch.equal(out[0, 0].double(), ref.held(v)[0, 1])
    c.close()


# -- attention ----------------------------------------------------------------------


class Case:
    """A cache of packed entries, a tail, and what each row attends."""

    def __init__(self, binding, dtype, lens, n, H, K, D, page, tail=None, window=0, sinks=0,
                 tree=False, count=None, positions=True, seed=0, spread=1.0, spare=0):
        B = len(lens)
        self.tail = n if tail is None else tail
        self.B, self.n, self.H, self.K, self.D, self.dtype = B, n, H, K, D, dtype
        self.lens, self.window, self.sinks, self.count = lens, window, sinks, count
        rng = random.Random(seed)
        width = max(1, max(-(-x // page) for x in lens)) + spare
        needs = [-(-x // page) for x in lens]
        pages = sum(needs) + 3
        ids = rng.sample(range(pages), pages)
        # places that hold no entry name pages outside the pool
        self.table = [[ids.pop() if p < m else rng.choice([-1, pages + 7, 1 << 30])
                       for p in range(width)] for m in needs]
        self.c = _cache(binding, B, K, D, page, pages, dtype, H=H, width=width)
        self.pool, self.k, self.v = [], [], []
        for which in range(2):
            pool = _bytes((pages, K, self.c.page_bytes), seed + which)     # any bytes
            rows = []
            for b in range(B):
                x = _normal((lens[b], K, D), dtype, seed * 7 + 2 * b + which, spread)
                slots = [self.table[b][e // page] * page + e % page for e in range(lens[b])]
                ref.store(pool, page, slots, x)
                rows.append(ref.held(x))
            self.pool.append(pool.cuda())
            (self.k, self.v)[which].extend(rows)
        self.q = _normal((B, n, H, D), dtype, seed + 11, 1.5)
        self.k_tail = _normal((B, self.tail, K, D), dtype, seed + 12, spread)
        self.v_tail = _normal((B, self.tail, K, D), dtype, seed + 13)
        self.mask = self.positions = None
        if tree:
            self.mask = torch.zeros((B, n, self.tail), dtype=torch.uint8)
            self.positions = torch.zeros((B, n), dtype=torch.int32)
            for b in range(B):
                for i in range(n):
                    j = i + self.tail - n
                    if i and j >= 0:
                        p = rng.randrange(i)
                        self.mask[b, i] = self.mask[b, p]
                        self.positions[b, i] = self.positions[b, p] + 1
                    if j >= 0:
                        self.mask[b, i, j] = rng.choice([1, 255])
                self.positions[b] += lens[b]
            if not positions:
                self.positions = None

    def call(self, **kw):
        up = lambda t: None if t is None else t.cuda()  # noqa: E731
        args = dict(mask=up(self.mask), window=self.window, sinks=self.sinks,
                    positions=up(self.positions),
                    count=None if self.count is None else _i32(self.count))
        if self.tail:
            args.update(k_tail=up(self.k_tail), v_tail=up(self.v_tail))
        args.update(kw)
        return self.c.attention(up(self.q), *self.pool, _i32(self.table), _i32(self.lens), **args)

    def want(self, b):
        count = None if self.count is None else self.count[b]
        seen = ref.seen(self.n, self.tail, self.lens[b], self.window, self.sinks,
                        None if self.mask is None else self.mask[b],
                        None if self.positions is None else self.positions[b], count)
        there = seen.shape[1] - self.lens[b]
        k = torch.cat([self.k[b], self.k_tail[b, :there].double()])
        v = torch.cat([self.v[b], self.v_tail[b, :there].double()])
        return cache_oracle.attention(self.q[b], k, v, seen, self.D ** -0.5, self.dtype)

    def check(self):
        out0 = _normal((self.B, self.n, self.H, self.D), self.dtype, 77)
        lse0 = _normal((self.B, self.n, self.H), torch.float32, 78)
        out, lse = self.call(out=out0.cuda(), lse=lse0.cuda())
        out, lse = out.cpu(), lse.cpu()
        assert self.c.device_error() == 0
        for b in range(self.B):
            rows = self.n if self.count is None else self.count[b]
            w, w_lse, tol, tol_lse = self.want(b)
            assert torch.equal(out[b, rows:], out0[b, rows:])
            assert torch.equal(lse[b, rows:], lse0[b, rows:])
            off = (out[b].double() - w).abs()[:rows]
            assert (off <= tol[:rows]).all(), (b, float((off / tol[:rows]).max()))
            none = torch.isinf(w_lse[:rows])
            assert (lse[b, :rows][none] == -math.inf).all() and (out[b, :rows][none] == 0).all()
            off = (lse[b].double() - w_lse).abs()[:rows][~none]
            assert (off <= tol_lse[:rows][~none]).all(), (b, float((off / tol_lse[:rows][~none]).max()))
        return out


ATTENTION = [
    # dtype, lens, n, H, K, D, page, more
    (BF16, [1], 1, 1, 1, 8, 16, {}),
    (BF16, [0], 1, 4, 2, 128, 16, {}),
    (F16, [517], 1, 32, 8, 128, 64, {}),
    (BF16, [16, 17, 31, 32, 33], 1, 8, 2, 64, 16, {}),
    (BF16, [300, 0, 129], 5, 8, 2, 128, 32, dict(tree=True)),
    (F16, [200, 131], 61, 8, 2, 128, 64, dict(tree=True)),
    (BF16, [511], 61, 32, 8, 128, 16, dict(tree=True)),
    (BF16, [700, 3], 33, 4, 1, 64, 16, {}),
    (F16, [250, 90], 9, 7, 1, 80, 16, dict(tree=True)),
    (BF16, [120, 77], 12, 6, 3, 112, 32, {}),
    (F16, [260], 17, 5, 5, 160, 64, dict(tree=True)),
    (BF16, [150, 40], 23, 12, 2, 256, 16, dict(tree=True)),
    (F16, [99], 70, 8, 1, 256, 128, {}),
    (BF16, [130], 10, 2, 1, 24, 16, {}),
    (F16, [170], 3, 4, 2, 200, 16, dict(tree=True)),
    (BF16, [95], 40, 4, 2, 224, 32, {}),
    (F16, [64], 8, 2, 2, 32, 16, dict(tail=20)),
    (BF16, [64, 200], 8, 4, 2, 96, 16, dict(tail=37, tree=True)),
    (BF16, [80, 300], 1, 8, 2, 128, 16, dict(tail=0)),
    (F16, [80, 33], 40, 4, 2, 64, 16, dict(tail=0)),
    (BF16, [300], 20, 4, 2, 128, 16, dict(tail=7)),
    (BF16, [300, 20, 0, 77], 9, 8, 2, 128, 16, dict(tree=True, count=[9, 0, 4, 1])),
    (F16, [300, 20, 0, 77], 9, 8, 2, 64, 16, dict(count=[3, 9, 2, 0], tail=14)),
    (BF16, [1000], 1, 8, 2, 128, 16, dict(window=100, sinks=4)),
    (BF16, [1000], 1, 8, 2, 128, 16, dict(window=1)),
    (F16, [900, 15, 64], 1, 28, 4, 128, 64, dict(window=64, sinks=20)),
    (BF16, [600, 40], 30, 8, 2, 128, 16, dict(window=33, sinks=3)),
    (BF16, [600, 40], 30, 8, 2, 128, 16, dict(window=7, sinks=50)),
    (F16, [640, 90], 61, 16, 4, 64, 32, dict(window=128, sinks=17, tree=True)),
    (BF16, [640, 90], 21, 16, 4, 80, 16, dict(window=70, tree=True, positions=False)),
    (BF16, [0, 5], 200, 4, 1, 64, 16, dict(window=40, sinks=9)),
    (BF16, [300], 20, 4, 2, 128, 16, dict(tail=7, window=16, sinks=2)),
    (F16, [256], 40, 2, 1, 160, 16, dict(tail=0, window=50, sinks=300)),
    (BF16, [200, 130], 9, 8, 2, 128, 16, dict(window=1 << 30, sinks=1 << 30, tree=True)),
    (BF16, [230], 130, 4, 2, 96, 16, dict(window=64)),
    (BF16, [30, 1, 9] * 30, 2, 4, 2, 64, 16, dict(tree=True)),
]


@pytest.mark.parametrize("dtype,lens,n,H,K,D,page,more", ATTENTION)
def test_attention_matches_the_plain_form(binding, dtype, lens, n, H, K, D, page, more):
    case = Case(binding, dtype, lens, n, H, K, D, page, seed=len(lens) * 1000 + n + D, **more)
    case.check()
    case.c.close()


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("n,H,K,D", [(1, 4, 1, 128), (61, 4, 1, 128), (20, 2, 1, 80)])
def test_attention_cut_over_many_workgroups(binding, dtype, n, H, K, D):
    """One long sequence, whose results come from many parts."""
    case = Case(binding, dtype, [20011], n, H, K, D, 64, seed=5, tree=n > 1)
    case.check()
    case.c.close()


def test_attention_of_peaked_scores(binding):
    """Scores far apart: the running maximum rises often, and most weights vanish."""
    for dtype in (BF16, F16):
        case = Case(binding, dtype, [400, 90], 9, 8, 2, 128, 16, seed=6, spread=6.0, tree=True)
        case.check()
        case.c.close()


def test_rows_that_attend_nothing(binding):
    """Masks that name nothing over no pages, causal rows before the first entry."""
    case = Case(binding, BF16, [0, 40], 6, 4, 2, 64, 16, tree=True, seed=2)
    case.mask[0] = 0
    out = case.check()
    assert (out[0] == 0).all()
    case.c.close()
    case = Case(binding, F16, [2, 0], 6, 4, 2, 64, 16, tail=0, seed=2)
    out = case.check()
    assert (out[0, :4] == 0).all() and (out[1] == 0).all()
    case.c.close()


# -- commit -------------------------------------------------------------------------

COMMITS = [
    # dtype, B, n, depth, K, D, page, layers
    (BF16, 1, 61, 7, 8, 128, 64, 3), (F16, 3, 20, 5, 2, 80, 16, 2), (BF16, 40, 9, 3, 1, 64, 16, 1),
    (F16, 2, 200, 15, 3, 24, 32, 2), (BF16, 1, 1, 1, 2, 256, 16, 4), (BF16, 600, 5, 4, 1, 32, 16, 5),
]


def _tree(rng, n, depth_most):
    parent, depth = [-1], [0]
    for i in range(1, n):
        p = rng.randrange(i)
        while depth[p] >= depth_most:
            p = rng.randrange(i)
        parent.append(p)
        depth.append(depth[p] + 1)
    return parent, [-1] + rng.sample(range(10000), n - 1)


def _accepted(rng, parent, token, depth):
    """An accepted path and its tokens."""
    path = [0]
    for _ in range(rng.randint(0, depth)):
        children = [i for i, p in enumerate(parent) if p == path[-1]]
        if not children:
            break
        path.append(rng.choice(children))
    return path, [token[i] for i in path[1:]]


@pytest.mark.parametrize("dtype,B,n,depth,K,D,page,layers", COMMITS)
def test_commit_packs_the_accepted_rows(binding, dtype, B, n, depth, K, D, page, layers):
    """Entries and lengths of the accepted paths in every layer, bytes equal; what fails or
    was not served stays as it was."""
    rng = random.Random(B * 10 + n)
    width = 3 + depth // page
    pages = B * width
    ids = rng.sample(range(pages), pages)
    table = [[ids.pop() for _ in range(width)] for _ in range(B)]
    lens = [rng.randint(0, 2 * page) for _ in range(B)]
    trees = [_tree(rng, n, depth) for _ in range(B)]
    paths = [_accepted(rng, p, t, depth) for p, t in trees]
    took = [len(p) - 1 for p, _ in paths]
    status, fails = [0] * B, set()
    for b in range(1, B):
        if rng.random() < 0.2:                         # not served; or a walk that failed
            fails.add(b)
            if b % 2:
                status[b] = rng.choice([1, 2])
            else:
                took[b] = -1
    acc = [t + [-1] * (depth - len(t)) for _, t in paths]
    shape = (layers, B, n, K, D)
    k, v = _values(shape, dtype, 1), _values(shape, dtype, 2)
    size = (layers, pages, K, ref.page_bytes(D, page))
    kp, vp = _bytes(size, 3), _bytes(size, 4)
    c = _cache(binding, B, K, D, page, pages, dtype, layers, width=width)
    dk, dv, d_lens = kp.cuda(), vp.cuda(), _i32(lens)
    path, new = c.commit(_i32([p for p, _ in trees]), _i32([t for _, t in trees]), _i32(acc),
                         _i32(took), d_lens, _i32(table), k.cuda(), v.cuda(), dk, dv,
                         out=(None, d_lens), status=_i32(status))
    assert new is d_lens and c.device_error() == 0
    for b in range(B):
        good = b not in fails
        want = paths[b][0] if good else []
        assert path[b].tolist() == want + [-1] * (depth + 1 - len(want))
        assert int(new[b]) == lens[b] + len(want)
        slots = [table[b][(lens[b] + j) // page] * page + (lens[b] + j) % page
                 for j in range(len(want))]
        for x, pool in ((k, kp), (v, vp)):
            for i in range(layers):
                ref.store(pool[i], page, slots, x[i, b, want])
    assert torch.equal(dk.cpu(), kp) and torch.equal(dv.cpu(), vp)
    c.close()


@pytest.mark.parametrize("kw,bit", [(dict(accepted=[[7, -1]], took=[1]), 16),
                                    (dict(accepted=[[5, 9]], took=[3]), 16),
                                    (dict(lens=[-1]), 32), (dict(lens=[47]), 32),
                                    (dict(table=[[0, 9, 1]], lens=[15]), 8),
                                    (dict(table=[[0, -1, 1]], lens=[16]), 8)])
def test_commit_flags_bad_data(binding, kw, bit):
    """A sequence that sets an error bit keeps its entries and its length."""
    a = dict(accepted=[[5, 6]], took=[2], lens=[3], table=[[0, 1, 2]])
    a.update(kw)
    c = _cache(binding, 1, 1, 32, 16, 3, BF16, width=3)
    room = torch.zeros((12, 1, c.page_bytes), dtype=torch.uint8, device="cuda")
    pool = room[4:7], room[4:7].clone()
    k = torch.ones((1, 1, 4, 1, 32), dtype=BF16, device="cuda")
    path, new = c.commit(_i32([[-1, 0, 1, 2]]), _i32([[-1, 5, 6, 7]]), _i32(a["accepted"]),
                         _i32(a["took"]), _i32(a["lens"]), _i32(a["table"]), k, k,
                         *(x[None] for x in pool))
    assert c.device_error() == bit
    assert path.tolist() == [[-1] * 3] and new.tolist() == a["lens"]
    assert (room == 0).all()
    c.close()


def test_commit_of_values_that_are_not_finite(binding):
    """They are held as the format says, and flagged."""
    c = _cache(binding, 1, 1, 32, 16, 1, F16)
    x = torch.ones((1, 1, 1, 1, 32), dtype=F16)
    x[..., 3], x[..., 4], x[..., 5] = math.inf, -math.inf, math.nan
    pool = [torch.zeros((1, 1, 1, c.page_bytes), dtype=torch.uint8, device="cuda") for _ in range(2)]
    c.commit(_i32([[-1]]), _i32([[-1]]), _i32([[-1]]), _i32([0]), _i32([0]), _i32([[0]]), x.cuda(),
             torch.ones_like(x).cuda(), *pool)
    assert c.device_error() == 64
    k, v = c.read(torch.zeros((1, 1), dtype=torch.int64, device="cuda"), pool[0][0], pool[1][0])
    want = [1, 1, 1, 1.5, -1.5, 0] + [1] * 26          # (1 = 4 times 1/4, whose most is 6)
    assert k.flatten().tolist() == want and (v == 1).all()
    c.close()
