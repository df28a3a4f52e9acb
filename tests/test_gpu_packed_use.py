"""The 4-bit cache as it is used: values that are not finite, strides, streams, graphs, bad
data, refusals, many sequences, and whole decoding steps."""

import math
import random

import pytest
import torch

import packed_oracle as ref
from test_gpu_packed import BF16, F16, Case, _bytes, _cache, _i32, _normal, _tree, binding  # noqa: F401

pytestmark = pytest.mark.gpu

# shapes that take each way through the attention: few rows, up to 64, 128, more
ROWS = [(1, 4, 2), (3, 8, 2), (12, 8, 2), (25, 8, 2), (61, 8, 2), (80, 4, 1)]


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("n,H,K", ROWS)
@pytest.mark.parametrize("D", [64, 160])
def test_values_that_are_not_attended_have_no_effect(binding, dtype, n, H, K, D):  # noqa: F811
    """NaN, infinities and large numbers in masked entries of the tail, behind the rows that
    are there and in rows of no query: bit for bit the same."""
    case = Case(binding, dtype, [70, 33], n, H, K, D, 16, tail=n + 5, tree=True, seed=n,
                count=[n, max(n - 2, 0)])
    case.mask[:, :, 1] = 0
    case.mask[:, :, 4] = 0
    out, lse = case.call(lse=True)
    want = out.clone(), lse.clone()
    for bad in (math.nan, math.inf, -math.inf, torch.finfo(dtype).max):
        case.k_tail[:, 1] = bad
        case.v_tail[:, 4] = bad
        case.v_tail[:, 1, :, ::3] = bad
        case.k_tail[1, n + 3:], case.v_tail[1, n + 3:] = bad, bad
        case.q[1, max(n - 2, 0):] = bad
        out, lse = case.call(lse=True, out=want[0].clone())
        live = slice(0, max(n - 2, 0))
        assert torch.equal(out[0], want[0][0]) and torch.equal(out[1, live], want[0][1, live])
        assert torch.equal(lse[0], want[1][0]) and torch.equal(lse[1, live], want[1][1, live])
    case.c.close()


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("n,H,K", ROWS)
def test_values_that_are_attended_act_on_their_rows_alone(binding, dtype, n, H, K):  # noqa: F811
    """An infinite and a NaN value of the tail: where a row attends it, its element is that; the
    rest is the same, bit for bit.  Cut over workgroups, too."""
    for length, window in ((40, 0), (3000, 0), (3000, 128)):
        case = Case(binding, dtype, [length], n, H, K, 64, 16, tree=True, seed=n + 7, window=window)
        want = case.call().clone().cpu()
        j = n // 2
        case.v_tail[0, j, :, 5], case.v_tail[0, j, :, 6] = math.inf, math.nan
        case.v_tail[0, j, :, 63] = -math.inf
        out = case.call().cpu()
        sees = case.mask[0, :, j] != 0
        assert sees.any() and torch.equal(out[0, ~sees], want[0, ~sees])
        same = [d for d in range(64) if d not in (5, 6, 63)]
        assert torch.equal(out[0][..., same], _without(case, j).cpu()[0][..., same])
        assert (out[0, sees][..., 5] == math.inf).all() and (out[0, sees][..., 63] == -math.inf).all()
        assert torch.isnan(out[0, sees][..., 6]).all()
        case.c.close()


def _without(case, j):
    """The output with the values that are not finite as zeros."""
    keep = case.v_tail.clone()
    case.v_tail[~torch.isfinite(case.v_tail)] = 0
    out = case.call()
    case.v_tail = keep
    return out


def test_a_causal_tail_with_values_that_are_not_finite(binding):  # noqa: F811
    """Without a mask rows before the entry do not attend it; those a window later neither."""
    case = Case(binding, BF16, [90], 50, 4, 2, 64, 16, window=8, seed=3)
    want = case.call().cpu()
    case.v_tail[0, 20, :, 3] = math.nan
    out = case.call().cpu()
    sees = torch.zeros(50, dtype=torch.bool)
    sees[20:28] = True
    assert torch.isnan(out[0, sees][..., 3]).all()
    assert torch.equal(out[0, ~sees], want[0, ~sees])
    case.c.close()


def test_queries_that_are_not_finite_act_on_their_rows_alone(binding):  # noqa: F811
    for n in (3, 61):
        case = Case(binding, F16, [100], n, 8, 2, 128, 16, tree=True, seed=4)
        want = case.call().cpu()
        case.q[0, 1, 3, 7] = math.nan
        out = case.call().cpu()
        assert torch.isnan(out[0, 1, 3]).all()
        out[0, 1, 3] = want[0, 1, 3]
        assert torch.equal(out, want)
        case.c.close()


def test_rows_with_gaps(binding):  # noqa: F811
    """q inside a projection's output, out and the tail inside larger ones."""
    for n in (1, 20, 61):
        case = Case(binding, BF16, [77, 30], n, 8, 2, 64, 16, tree=True, seed=8)
        want = case.call()
        wide = torch.randn((2, n, 14, 64), device="cuda").to(BF16)
        wide[..., 2:10, :] = case.q.cuda()
        tail = torch.full((2, n, 6, 64), math.nan, dtype=BF16, device="cuda")
        tail[..., 1:3, :], tail[..., 3:5, :] = case.k_tail.cuda(), case.v_tail.cuda()
        room = torch.zeros((2, n, 9, 64), dtype=BF16, device="cuda")
        out = case.c.attention(wide[..., 2:10, :], *case.pool, _i32(case.table), _i32(case.lens),
                               tail[..., 1:3, :], tail[..., 3:5, :], mask=case.mask.cuda(),
                               out=room[..., :8, :])
        assert torch.equal(out, want) and (room[..., 8, :] == 0).all()
        case.c.close()


@pytest.mark.parametrize("B,n,H,K,D,window", [(64, 20, 32, 4, 32, 0), (300, 9, 4, 1, 64, 0),
                                              (70, 1, 8, 8, 32, 20), (40, 40, 12, 6, 64, 50),
                                              (4096, 1, 1, 1, 16, 0)])
def test_many_sequences_of_all_lengths(binding, B, n, H, K, D, window):  # noqa: F811
    """Items dealt out whole and items cut; some sequences have no rows, some no entries."""
    rng = random.Random(B)
    lens = [rng.choice([0, rng.randint(1, 200)]) for _ in range(B)]
    count = [rng.choice([n, n, rng.randint(0, n)]) for _ in range(B)]
    case = Case(binding, BF16, lens, n, H, K, D, 16, tree=n > 1, seed=B, window=window, sinks=3,
                count=count)
    out, lse = case.call(lse=torch.full((B, n, H), 7.0, device="cuda"),
                         out=torch.full((B, n, H, D), 5.0, dtype=BF16, device="cuda"))
    again, _ = case.call(lse=True, out=torch.full((B, n, H, D), 5.0, dtype=BF16, device="cuda"))
    assert torch.equal(out, again)
    out, lse = out.cpu(), lse.cpu()
    for b in rng.sample(range(B), 12):
        want, w_lse, tol, tol_lse = case.want(b)
        k = count[b]
        assert (out[b, k:] == 5).all() and (lse[b, k:] == 7).all()
        assert ((out[b].double() - want).abs() <= tol)[:k].all(), b
        none = torch.isinf(w_lse[:k])
        assert (lse[b, :k][none] == -math.inf).all()
        assert ((lse[b].double() - w_lse).abs() <= tol_lse)[:k][~none].all(), b
    assert case.c.device_error() == 0
    case.c.close()


def test_a_long_prompt(binding):  # noqa: F811
    """1500 causal rows on 700 entries, all and in a window: against 64 bits on the GPU.

    Off by the output's rounding, 2^-9 |o|, and each probability's, 2^-9 of sum p |v|, with
    1/8 more for fp32 sums of scores and of up to 2200 terms (2^-24 times some thousands)."""
    n, length, H, K, D = 1500, 700, 4, 2, 64
    for window, sinks in ((0, 0), (300, 5)):
        case = Case(binding, BF16, [length], n, H, K, D, 64, seed=12, window=window, sinks=sinks)
        out, lse = case.call(lse=True)
        k = torch.cat([case.k[0], case.k_tail[0].double()]).cuda()
        v = torch.cat([case.v[0], case.v_tail[0].double()]).cuda()
        e = torch.arange(length + n, device="cuda")[None, :]
        at = length + torch.arange(n, device="cuda")[:, None]
        seen = e <= at
        if window:
            seen &= (e > at - window) | (e < sinks)
        for h in range(H):
            x = case.q[0, :, h].cuda().double() @ k[:, h // 2].t() / 8
            x = torch.where(seen, x, -math.inf)
            p = x.softmax(1)
            want, size = p @ v[:, h // 2], p @ v[:, h // 2].abs()
            assert ((out[0, :, h].double() - want).abs() <= 2.0 ** -8 * 1.125 * size).all()
            assert ((lse[0, :, h].double() - x.logsumexp(1)).abs() <= 2.0 ** -24 * 4000).all()
        case.c.close()


# -- bad data -----------------------------------------------------------------------


@pytest.mark.parametrize("n,H,K", [(1, 2, 1), (20, 4, 1), (61, 8, 2)])
def test_attention_flags_bad_data(binding, n, H, K):  # noqa: F811
    """Lengths, counts and pages out of range set their bit; no memory outside the pool is
    read (there is none mapped far from it), sequences without fault are right."""
    for what, bit in (("len", 32), ("long", 32), ("count", 1), ("low", 1), ("page", 8), ("far", 8)):
        case = Case(binding, BF16, [40, 50], n, H, K, 64, 16, tree=n > 1, seed=n)
        want = case.call().cpu()
        if what == "len":
            case.lens = [40, -3]
        elif what == "long":
            case.lens = [40, 1000]
        elif what in ("count", "low"):
            case.count = [n, n + 1 if what == "count" else -1]
        else:
            case.table[1][1] = -1 if what == "page" else 2 ** 31 - 1
        if what == "long":
            # (the length is taken as what the table's row holds: all of it named)
            case.table = [[p if 0 <= p < case.c.pages else 0 for p in r] for r in case.table]
        out = case.call().cpu()
        assert case.c.device_error() == bit, what
        assert torch.equal(out[0], want[0]), what
        case.c.close()


def test_an_unserved_sequence_is_left_out(binding):  # noqa: F811
    case = Case(binding, BF16, [40, 50, 60], 9, 4, 2, 64, 16, tree=True, seed=1)
    want = case.call()
    out = torch.full_like(want, 3.0)
    case.call(out=out, status=_i32([0, 2, 0]))
    assert torch.equal(out[0], want[0]) and torch.equal(out[2], want[2]) and (out[1] == 3).all()
    case.c.close()


def _refused(binding, call, match=None):  # noqa: F811
    with pytest.raises(binding.RheoError, match=match) as e:
        call()
    assert e.value.code == binding.RHEO_EINVAL


def test_refusals(binding):  # noqa: F811
    B, n, H, K, D, page = 2, 5, 4, 2, 64, 16
    case = Case(binding, BF16, [20, 30], n, H, K, D, page, tree=True)
    c, pool = case.c, case.pool
    q, kt, vt = case.q.cuda(), case.k_tail.cuda(), case.v_tail.cuda()
    table, lens, mask = _i32(case.table), _i32(case.lens), case.mask.cuda()
    at = lambda **kw: c.attention(**{**dict(q=q, k_pages=pool[0], v_pages=pool[1], table=table,  # noqa: E731
                                            lens=lens, k_tail=kt, v_tail=vt, mask=mask), **kw})
    at()
    for kw in (dict(q=q.half()), dict(q=q[:1]), dict(k_pages=pool[0][1:]), dict(v_pages=pool[1].int()),
               dict(k_pages=pool[0].transpose(1, 2)), dict(k_tail=None), dict(v_tail=vt[:, 1:]),
               dict(mask=mask.bool()), dict(mask=mask[..., 1:]), dict(table=table.long()),
               dict(lens=lens[:1]), dict(scale=0.0), dict(scale=math.nan), dict(scale=2.0 ** 101),
               dict(window=-1), dict(sinks=-1), dict(out=q), dict(positions=lens),
               dict(count=_i32([1])), dict(lse=torch.zeros(3, device="cuda")),
               dict(status=_i32([0, 0]).long()), dict(k_tail=kt.cpu()),
               dict(v_tail=torch.zeros((B, n, 2 * K, D), dtype=BF16, device="cuda")[:, :, :K])):
        _refused(binding, lambda: at(**kw))
    slots = torch.zeros((B, n), dtype=torch.int64, device="cuda")
    for args in ((kt.half(), vt, slots, *pool), (kt, vt[:, :3], slots, *pool), (kt, vt, slots.int(), *pool),
                 (kt, vt, slots, pool[0], pool[1][:2]), (kt[None], vt[None], slots, *pool),
                 (kt, vt, slots, *(p[None] for p in pool)), (kt, vt, slots[:1], *pool)):
        _refused(binding, lambda: c.append(*args))
    _refused(binding, lambda: c.read(slots, *pool, out=(kt, vt[:, :3])))
    two = [torch.zeros((2, *pool[0].shape), dtype=torch.uint8, device="cuda") for _ in range(2)]
    _refused(binding, lambda: c.read(slots, *two), "layers")       # (the handle has one)
    _refused(binding, lambda: c.write(q, kt, vt, slots, kt, vt))
    tree = [_i32([[-1, 0, 0, 1, 1]] * B), _i32([[-1, 2, 3, 4, 5]] * B), _i32([[2]] * B), _i32([1] * B)]
    one = [p[None] for p in pool]
    c.commit(*tree, _i32([3, 4]), table, kt[None], vt[None], *one)
    _refused(binding, lambda: c.commit(*tree, _i32([3, 4]), table, kt, vt, *one))
    _refused(binding, lambda: c.commit(*tree, _i32([3, 4]), table, kt[None], vt[None], *pool))
    _refused(binding, lambda: c.commit(tree[0], tree[1], _i32([[2] * 16] * B), tree[3], _i32([3, 4]),
                                       table, kt[None], vt[None], *one), "depth")
    both = torch.zeros(B + 1, dtype=torch.int32, device="cuda")
    _refused(binding, lambda: c.commit(*tree, both[:B], table, kt[None], vt[None], *one,
                                       out=(None, both[1:])), "overlaps")
    # nothing to do
    empty = torch.zeros((B, 0, H, D), dtype=BF16, device="cuda")
    assert at(q=empty, mask=torch.zeros((B, 0, n), dtype=torch.uint8, device="cuda")).shape == empty.shape
    c.append(kt[:, :0], vt[:, :0], slots[:, :0], *pool)
    assert c.device_error() == 0
    c.close()


# -- streams and graphs ---------------------------------------------------------------


def test_calls_on_another_stream(binding):  # noqa: F811
    """Inputs made on a stream, calls on it, outputs theirs: read where they were asked for."""
    case = Case(binding, BF16, [500, 90], 20, 8, 2, 128, 16, tree=True, seed=6)
    want, want_lse = case.call(lse=True)
    slots = torch.arange(40, device="cuda").view(2, 20)
    c = case.c
    s = torch.cuda.Stream()
    for _ in range(3):
        with torch.cuda.stream(s):
            torch.cuda._sleep(20_000_000)
            args = [t.cuda(non_blocking=True) for t in (case.q, case.k_tail, case.v_tail, case.mask)]
            table, lens = _i32(case.table), _i32(case.lens)
            new = [torch.zeros_like(p) for p in case.pool]
        out, lse = c.attention(args[0], *case.pool, table, lens, args[1], args[2], mask=args[3],
                               lse=True, stream=s)
        c.append(args[1], args[2], slots, *new, stream=s)
        k, v = c.read(slots, *new, stream=s)
        del args, new
        torch.cuda.current_stream().wait_stream(s)
        assert torch.equal(out, want) and torch.equal(lse, want_lse)
        assert torch.equal(k.cpu().double(), ref.held(case.k_tail))
        assert torch.equal(v.cpu().double(), ref.held(case.v_tail))
    c.close()


@pytest.mark.parametrize("n,H,K,D", [(1, 8, 2, 128), (9, 8, 2, 80), (61, 8, 2, 64)])
def test_a_step_captured_and_replayed(binding, n, H, K, D):  # noqa: F811
    """Plan, write into the tail, attention, commit and read captured once and replayed on new
    inputs and lengths, with eager work between, against eager results."""
    B, page, layers, depth, width = 3, 16, 2, 4, 20
    pages = B * width
    rng = random.Random(n)
    c = _cache(binding, B, K, D, page, pages, BF16, layers, H=H, width=width)
    tail = binding.Cache(batch=B, heads=H, kv_heads=K, head_dim=D, page_size=1, pages=B * n,
                         table_width=1)
    at = torch.arange(B * n, device="cuda").view(B, n)
    half = D // 2
    angle = torch.arange(400, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(half) / half)
    rotation = torch.cat([angle.cos(), angle.sin()], 1).float().cuda()

    def inputs(seed):
        trees = [_tree(rng, n, depth) for _ in range(B)]
        mask = torch.zeros((B, n, n), dtype=torch.uint8)
        deep = torch.zeros((B, n), dtype=torch.int32)
        for b in range(B):
            for i in range(n):
                p = trees[b][0][i]
                if i:
                    mask[b, i] = mask[b, p]
                    deep[b, i] = deep[b, p] + 1
                mask[b, i, i] = 1
        took = [0 if n == 1 else 1] * B
        acc = [[t[1][1] if n > 1 else -1] + [-1] * (depth - 1) for t in trees]
        return dict(qkv=_normal((layers, B, n, H + 2 * K, D), BF16, seed), mask=mask, deep=deep,
                    parent=torch.tensor([t[0] for t in trees], dtype=torch.int32),
                    token=torch.tensor([t[1] for t in trees], dtype=torch.int32),
                    acc=torch.tensor(acc, dtype=torch.int32),
                    took=torch.tensor(took, dtype=torch.int32))

    ids = torch.randperm(pages, generator=torch.Generator().manual_seed(1)).int()

    def state():
        held = [-(-x // page) for x in (100, 37, 0)]
        table = torch.zeros((B, width), dtype=torch.int32)
        free = ids.tolist()
        for b in range(B):
            for p in range(held[b]):
                table[b, p] = free.pop()
        free_list = torch.zeros(pages, dtype=torch.int32)
        free_list[:len(free)] = torch.tensor(free, dtype=torch.int32)
        d = dict(lens=_i32([100, 37, 0]), held=_i32(held), table=table.cuda(),
                 free_list=free_list.cuda(), free_count=_i32([len(free)]))
        pool = [_bytes((layers, pages, K, c.page_bytes), s).clamp(110, 130).cuda() for s in (3, 4)]
        d.update(kp=pool[0], vp=pool[1],
                 kt=torch.zeros((layers, B, n, K, D), dtype=BF16, device="cuda"),
                 vt=torch.zeros((layers, B, n, K, D), dtype=BF16, device="cuda"))
        return d

    def step(x, d):
        slots, _, status = c.plan(d["lens"], d["held"], d["table"], d["free_list"], d["free_count"],
                                  depth + 1)
        positions = (d["lens"][:, None] + x["deep"]).to(torch.int32)
        outs = []
        for layer in range(layers):
            q, k, v = x["qkv"][layer].split([H, K, K], 2)
            q = tail.write(q, k, v, at, d["kt"][layer].view(B * n, 1, K, D),
                           d["vt"][layer].view(B * n, 1, K, D), positions=positions, rotation=rotation)
            outs.append(c.attention(q, d["kp"][layer], d["vp"][layer], d["table"], d["lens"],
                                    d["kt"][layer], d["vt"][layer], mask=x["mask"], window=64, sinks=4,
                                    positions=positions, status=status))
        path, _ = c.commit(x["parent"], x["token"], x["acc"], x["took"], d["lens"], d["table"],
                           d["kt"], d["vt"], d["kp"], d["vp"], out=(None, d["lens"]), status=status)
        return (*outs, path, *c.read(slots, d["kp"], d["vp"]))

    steps = [{k: v.cuda() for k, v in inputs(s).items()} for s in range(4)]
    eager, d = [], state()
    for x in steps:
        eager.append([t.clone() for t in step(x, d)])
    final = {k: t.clone() for k, t in d.items()}
    hold = {k: t.clone() for k, t in steps[0].items()}
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        step(hold, state())
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    d = state()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = step(hold, d)
    for i, x in enumerate(steps):
        for k, t in x.items():
            hold[k].copy_(t)
        g.replay()
        torch.cuda.synchronize()
        for y, w in zip(out, eager[i]):
            assert torch.equal(y, w), i
        (torch.randn(1000, device="cuda") @ torch.randn(1000, device="cuda")).item()
    for k, t in d.items():
        assert torch.equal(t, final[k]), k
    assert c.device_error() == 0 and tail.device_error() == 0
    c.close()
    tail.close()


# -- whole steps ----------------------------------------------------------------------


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_decoding_steps_over_a_4_bit_cache(binding, dtype):  # noqa: F811
    """A prompt in two pieces, appended, then drafted trees, committed: what a later step attends
    to is what the earlier ones kept, sequence by sequence, with fewer pages than all ask
    for."""
    B, H, K, D, page, width, depth, n = 3, 4, 2, 64, 16, 12, 3, 10
    pages = 14
    c = _cache(binding, B, K, D, page, pages, dtype, H=H, width=width)
    rng = random.Random(3)
    lens, held = _i32([0] * B), _i32([0] * B)
    table = torch.zeros((B, width), dtype=torch.int32, device="cuda")
    free_list, free_count = _i32(rng.sample(range(pages), pages)), _i32([pages])
    pool = [_bytes((pages, K, c.page_bytes), s).cuda() for s in (1, 2)]
    kept = [[], []]                                    # rows in 64 bits, sequence by sequence
    kept = [[torch.zeros((0, K, D), dtype=torch.float64) for _ in range(B)] for _ in range(2)]

    def check(q, out, kt, vt, seen, served):
        for b in range(B):
            if not served[b]:
                continue
            k = torch.cat([kept[0][b], kt[b].double()])
            v = torch.cat([kept[1][b], vt[b].double()])
            for h in range(H):
                x = q[b, :, h].double() @ k[:, h // 2].t() / 8
                s = torch.cat([torch.ones((len(x), len(kept[0][b])), dtype=torch.bool), seen[b]], 1)
                p = torch.where(s, x, -math.inf).softmax(1)
                want, size = p @ v[:, h // 2], p @ v[:, h // 2].abs()
                # two roundings to 16 bits (half a step each), and 1/8 more for fp32 sums
                u = {BF16: 2.0 ** -8, F16: 2.0 ** -11}[dtype]
                assert ((out[b, :, h].cpu().double() - want).abs() <= u * 1.125 * (size + want.abs())).all()

    for piece in (33, 20):                             # the prompt
        count = [piece, piece - 5, piece]
        slots, _, status = c.plan(lens, held, table, free_list, free_count, piece, count=_i32(count))
        assert status.tolist() == [0, 0, 0]
        q, kt, vt = (_normal((B, piece, x, D), dtype, piece + x) for x in (H, K, K))
        vt = vt + 1
        out = c.attention(q.cuda(), *pool, table, lens, kt.cuda(), vt.cuda(), count=_i32(count))
        causal = torch.ones((piece, piece), dtype=torch.bool).tril()
        for b in range(B):
            m = count[b]
            check(q[:, :m], out[:, :m], kt[:, :m], vt[:, :m], [causal[:m, :m]] * B,
                  [x == b for x in range(B)])
            for which, t in ((0, kt), (1, vt)):
                kept[which][b] = torch.cat([kept[which][b], ref.held(t[b, :m])])
        c.append(kt.cuda(), vt.cuda(), slots, *pool)
        lens += _i32(count)
    refused = 0
    for step in range(40):
        slots, _, status = c.plan(lens, held, table, free_list, free_count, depth + 1)
        served = [s == 0 for s in status.tolist()]
        refused += served.count(False)
        q, kt, vt = (_normal((B, n, x, D), dtype, step * 100 + x) for x in (H, K, K))
        trees = [_tree(rng, n, depth) for _ in range(B)]
        mask = torch.zeros((B, n, n), dtype=torch.uint8)
        paths = []
        for b in range(B):
            for i in range(n):
                if i:
                    mask[b, i] = mask[b, trees[b][0][i]]
                mask[b, i, i] = 1
            path = [0]
            while len(path) <= depth and rng.random() < 0.8:
                below = [i for i in range(n) if trees[b][0][i] == path[-1]]
                if not below:
                    break
                path.append(rng.choice(below))
            paths.append(path)
        out = c.attention(q.cuda(), *pool, table, lens, kt.cuda(), vt.cuda(), mask=mask.cuda(),
                          status=status)
        check(q, out, kt, vt, mask != 0, served)
        acc = [[trees[b][1][i] for i in paths[b][1:]] + [-1] * (depth + 1 - len(paths[b])) for b in range(B)]
        got, _ = c.commit(_i32([t[0] for t in trees]), _i32([t[1] for t in trees]), _i32(acc),
                          _i32([len(p) - 1 for p in paths]), lens, table, kt[None].cuda(),
                          vt[None].cuda(), *(p[None] for p in pool), out=(None, lens), status=status)
        for b in range(B):
            path = paths[b] if served[b] else []
            assert got[b].tolist() == path + [-1] * (depth + 1 - len(path))
            for which, t in ((0, kt), (1, vt)):
                if path:
                    kept[which][b] = torch.cat([kept[which][b], ref.held(t[b, path])])
            assert int(lens[b]) == len(kept[0][b])
        if step % 10 == 9:                             # a sequence is over; another begins
            b = step // 10 % B
            lens[b] = 0
            kept[0][b], kept[1][b] = kept[0][b][:0], kept[1][b][:0]
        c.plan(lens, held, table, free_list, free_count, 0)
    assert refused > 0 and c.device_error() == 0
    c.close()
