"""The cache operators as a serving loop uses them: refusals, graphs, streams, handles side
by side, and whole decoding steps together with the tree's own calls."""

import ctypes
import math

import pytest
import torch

import cache_oracle as ref
from test_gpu_cache import BF16, F16, Setup, _drafted, _i32, _tree_mask

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def binding():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2609_21827_amd import binding
    binding.load_library()
    return binding


# -- refusals -----------------------------------------------------------------------


def _refused(binding, call):
    with pytest.raises(binding.RheoError) as e:
        call()
    assert e.value.code == binding.RHEO_EINVAL and str(e.value)


def test_wrong_tensors_are_refused(binding):
    s = Setup(binding, BF16, [40, 9], 5, 5, 4, 2, 64, 16)
    c, q = s.cache, s.q.cuda()
    kc, vc = s.pages_on_gpu()
    table, lens = s.table.cuda(), _i32(s.lens)
    mask = _tree_mask(s.g, 2, 5).cuda()
    good = dict(q=q, k_cache=kc, v_cache=vc, table=table, lens=lens, mask=mask)
    c.attention(**good)
    for bad in (dict(q=q.float()), dict(q=q.cpu()), dict(q=q[:1]), dict(q=q.transpose(0, 1)),
                dict(q=q.transpose(1, 2).contiguous().transpose(1, 2)), dict(k_cache=kc[1:]),
                dict(k_cache=kc.to(F16)), dict(v_cache=vc.transpose(1, 2)), dict(table=table.long()),
                dict(table=table[:, 1:]), dict(table=table.t().contiguous().t()),
                dict(lens=lens.cpu()), dict(mask=mask.bool()), dict(mask=mask[:, :4]),
                dict(mask=mask, tail=6), dict(mask=None, tail=4), dict(mask=None, tail=-1),
                dict(scale=0.0), dict(scale=-1.0), dict(scale=math.inf), dict(scale=math.nan),
                dict(out=q), dict(out=q.float()), dict(lse=torch.zeros(2, 5, 4).cuda().half()),
                dict(count=lens.long()), dict(tail=1 << 25, mask=None)):
        _refused(binding, lambda: c.attention(**{**good, **bad}))
    k = torch.zeros((2, 5, 2, 64), dtype=BF16, device="cuda")
    slots = torch.arange(10, device="cuda").view(2, 5)
    rot, pos = torch.zeros((50, 64), device="cuda"), torch.zeros((2, 5), dtype=torch.int32, device="cuda")
    w = dict(q=q, k=k, v=k, slots=slots, k_cache=kc, v_cache=vc, positions=pos, rotation=rot)
    c.write(**w)
    for bad in (dict(slots=slots.int()), dict(slots=slots[:, :4]), dict(rotation=rot.double()),
                dict(rotation=torch.zeros((50, 66), device="cuda")), dict(rotation=rot[:, :63].contiguous()),
                dict(rotation=rot[:0]), dict(rotation=rot[0]), dict(positions=None),
                dict(positions=pos.long()), dict(k=k.expand(2, 5, 2, 64)[:, :, :1]),
                dict(v=k.float()), dict(q_weight=torch.ones(64, device="cuda")),
                dict(q_weight=torch.ones(63, dtype=BF16, device="cuda")), dict(eps=-1.0),
                dict(eps=math.nan), dict(interleaved=2), dict(q=None, out=q),
                dict(out=torch.zeros((2, 5, 4, 64), device="cuda"))):
        _refused(binding, lambda: c.write(**{**w, **bad}))
    par = torch.zeros((2, 5), dtype=torch.int32, device="cuda")
    one = torch.zeros(2, dtype=torch.int32, device="cuda")
    m = dict(parent=par, token=par, accepted=par[:, :3].contiguous(), accept_len=one, lens=lens,
             table=table, k_cache=kc[None], v_cache=vc[None])
    c.commit(**m)
    for bad in (dict(token=par[:, :4]), dict(accepted=par.long()), dict(k_cache=kc),
                dict(accepted=torch.zeros((2, 16), dtype=torch.int32, device="cuda")),
                dict(accept_len=one.long()), dict(out=(par, one))):
        _refused(binding, lambda: c.commit(**{**m, **bad}))
    held, free, cnt = one.clone(), torch.zeros(s.pages, dtype=torch.int32, device="cuda"), one[:1]
    c.plan(lens, held.clone(), table.clone(), free.clone(), cnt.clone(), 2)
    for bad in ((lens.long(), held, table, free, cnt, 2), (lens, held, table, free[1:], cnt, 2),
                (lens, held, table, free, one, 2), (lens, held, table, free, cnt, 1 << 30)):
        _refused(binding, lambda: c.plan(*bad, out=None if bad[-1] == 2 else
                                         (torch.zeros((2, 0)).long().cuda(), par, one)))
    s.cache.close()
    for bad in (dict(dtype=torch.float32), dict(device="cpu"), dict(dtype=torch.int8)):
        _refused(binding, lambda: binding.Cache(**{**dict(
            batch=1, heads=1, kv_heads=1, head_dim=64, page_size=16, pages=1, table_width=1), **bad}))


def test_wrong_scoring_calls_are_refused(binding):
    s = binding.Scorer(100, torch.float32, 104)
    x = torch.zeros((2, 3, 104), device="cuda")
    t = torch.zeros((2, 3), dtype=torch.int32, device="cuda")
    s.logprobs(x, t)
    for args, kw in (((x.half(), t), {}), ((x[0], t), {}), ((x[..., :100], t), {}), ((x, t.long()), {}),
                     ((x, t[:1]), {}), ((x, t), dict(top=33)), ((x, t), dict(top=-1)),
                     ((x, t), dict(T=0.0)), ((x, t), dict(T=math.nan)), ((x, t), dict(T=1e-45)),
                     ((x, t), dict(path=t[:, :2])), ((x[:, :2].contiguous(), t), {}),
                     ((x, t), dict(out=(t, t, t, t, t)))):
        _refused(binding, lambda: s.logprobs(*args, **kw))
    s.close()
    small = binding.Scorer(3, torch.float32, 4)
    _refused(binding, lambda: small.logprobs(torch.zeros((1, 1, 4), device="cuda"),
                                             t[:1, :1].contiguous(), top=4))
    small.close()


def test_unaligned_and_overlapping_arguments_are_refused(binding):
    """What only the C ABI can be given."""
    lib = binding.load_library()
    s = Setup(binding, BF16, [40], 3, 3, 4, 2, 64, 16)
    q, out = s.q.cuda(), torch.zeros((1, 3, 4, 64), dtype=BF16, device="cuda")
    kc, vc = s.pages_on_gpu()
    table, lens = s.table.cuda(), _i32(s.lens)

    def args(**kw):
        a = binding.AttentionArgs(3, 3, q.data_ptr(), 256, 256, kc.data_ptr(), vc.data_ptr(),
                                  table.data_ptr(), lens.data_ptr(), None, None, 1.0,
                                  out.data_ptr(), None)
        for k, v in kw.items():
            setattr(a, k, v)
        return lib.rheo_tree_attention(s.cache._h, ctypes.byref(a), None)

    assert args() == binding.RHEO_OK
    torch.cuda.synchronize()
    for bad in (dict(q=q.data_ptr() + 2), dict(q=None), dict(q_stride=255), dict(q_stride=252),
                dict(q_stride=257), dict(out_stride=1 << 32), dict(k_cache=kc.data_ptr() + 8),
                dict(lens=lens.data_ptr() + 2), dict(table=None), dict(out=None), dict(n=-1),
                dict(n=1 << 30), dict(lse=out.data_ptr() + 1)):
        assert args(**bad) == binding.RHEO_EINVAL, bad
    two = torch.zeros(8, dtype=torch.int32, device="cuda")
    c2 = binding.Cache(batch=2, heads=2, kv_heads=2, head_dim=64, page_size=16, pages=s.pages,
                       table_width=1)
    p = two.data_ptr()
    assert lib.rheo_cache_commit(c2._h, 1, 1, p, p, p, p, p, p, kc.data_ptr(), vc.data_ptr(),
                                 p, p + 4, None) == binding.RHEO_EINVAL
    s.cache.close()
    c2.close()


def test_calls_without_rows_do_nothing(binding):
    s = Setup(binding, BF16, [40], 1, 1, 4, 2, 64, 16)
    kc, vc = s.pages_on_gpu()
    q = torch.zeros((1, 0, 4, 64), dtype=BF16, device="cuda")
    assert s.cache.attention(q, kc, vc, s.table.cuda(), _i32([40])).shape == (1, 0, 4, 64)
    k = torch.zeros((1, 0, 2, 64), dtype=BF16, device="cuda")
    assert s.cache.write(q, k, k, torch.zeros((1, 0)).long().cuda(), kc, vc).shape == (1, 0, 4, 64)
    x = binding.Scorer(100, BF16, 104)
    got = x.logprobs(torch.zeros((2, 0, 104), dtype=BF16, device="cuda"),
                     torch.zeros((2, 0), dtype=torch.int32, device="cuda"), top=3)
    assert [tuple(t.shape) for t in got] == [(2, 0)] * 3 + [(2, 0, 3)] * 2
    got = x.logprobs(torch.zeros((0, 4, 104), dtype=BF16, device="cuda"),
                     torch.zeros((0, 4), dtype=torch.int32, device="cuda"))
    assert got[0].shape == (0, 4)
    x.close()
    s.cache.close()


# -- a step's calls -------------------------------------------------------------------


class Loop:
    """Layers of attention over one paged cache, driven step by step; everything lives in
    buffers of fixed place, so that a step may be captured."""

    def __init__(self, binding, B=3, n=20, H=4, K=2, D=64, page=16, layers=2, V=500, depth=5, seed=0):
        g = torch.Generator().manual_seed(seed)
        self.B, self.n, self.H, self.K, self.D, self.layers, self.V = B, n, H, K, D, layers, V
        self.depth, self.page, self.width = depth, page, 12
        self.pages = B * self.width
        self.cache = binding.Cache(batch=B, heads=H, kv_heads=K, head_dim=D, page_size=page,
                                   pages=self.pages, table_width=self.width, layers=layers)
        self.scorer = binding.Scorer(V, BF16, 504)
        shape = (layers, self.pages, page, K, D)
        self.kc, self.vc = (torch.zeros(shape, dtype=BF16, device="cuda") for _ in range(2))
        self.table = torch.zeros((B, self.width), dtype=torch.int32, device="cuda")
        self.lens, self.held = _i32([0] * B), _i32([0] * B)
        self.free = torch.randperm(self.pages, generator=g).int().cuda()
        self.free_count = _i32([self.pages])
        self.rot = torch.randn((400, D), generator=g).cuda()
        self.qw, self.kw = (torch.rand(D, generator=g).to(BF16).cuda() for _ in range(2))
        self.g = g
        i32 = dict(dtype=torch.int32, device="cuda")
        self.qkv = torch.zeros((layers, B, n, (H + 2 * K) * D), dtype=BF16, device="cuda")
        self.mask = torch.zeros((B, n, n), dtype=torch.uint8, device="cuda")
        self.depths, self.parent, self.token = (torch.zeros((B, n), **i32) for _ in range(3))
        self.accepted = torch.zeros((B, depth), **i32)
        self.accept_len = torch.zeros(B, **i32)
        self.logits = torch.zeros((B, n, 504), dtype=BF16, device="cuda")
        self.emitted = torch.zeros((B, depth + 1), **i32)

    def feed(self, seed):
        """The next step's inputs, into the fixed buffers."""
        import random
        rng, g = random.Random(seed), torch.Generator().manual_seed(seed)
        trees = [_drafted(rng, self.n, self.depth) for _ in range(self.B)]
        mask, depths, acc, took, emitted = [], [], [], [], []
        for parent, token in trees:
            m = torch.zeros((self.n, self.n), dtype=torch.uint8)
            d = []
            for i in range(self.n):
                if i:
                    m[i] = m[parent[i]]
                m[i, i] = 1
                d.append(int(m[i].sum()) - 1)
            path, row = [0], []
            while rng.random() < 0.8:
                kids = [i for i in range(self.n) if parent[i] == path[-1]]
                if not kids:
                    break
                path.append(rng.choice(kids))
                row.append(token[path[-1]])
            mask.append(m), depths.append(d)
            took.append(len(row))
            emitted.append(row + [rng.randrange(self.V)] + [-1] * (self.depth - len(row)))
            acc.append(row + [-1] * (self.depth - len(row)))
        self.mask.copy_(torch.stack(mask))
        for t, rows in ((self.depths, depths), (self.parent, [x[0] for x in trees]),
                        (self.token, [x[1] for x in trees]), (self.accepted, acc),
                        (self.accept_len, took), (self.emitted, emitted)):
            t.copy_(torch.tensor(rows, dtype=torch.int32))
        self.qkv.copy_(torch.randn(self.qkv.shape, generator=g).to(BF16))
        self.logits.copy_((torch.randn(self.logits.shape, generator=g) * 3).to(BF16))

    def state(self):
        return [self.kc, self.vc, self.table, self.lens, self.held, self.free, self.free_count]

    def step(self, stream=None):
        H, K, D = self.H, self.K, self.D
        c, kw = self.cache, dict(stream=stream)
        out = []
        state = (self.lens, self.held, self.table, self.free, self.free_count)
        slots, pos, status = c.plan(*state, self.n, depth=self.depths, **kw)
        for i in range(self.layers):
            q, k, v = self.qkv[i].split([H * D, K * D, K * D], dim=2)
            q = c.write(q.unflatten(2, (H, D)), k.unflatten(2, (K, D)), v.unflatten(2, (K, D)),
                        slots, self.kc[i], self.vc[i], positions=pos, rotation=self.rot,
                        q_weight=self.qw, k_weight=self.kw, **kw)
            out += c.attention(q, self.kc[i], self.vc[i], self.table, self.lens, mask=self.mask,
                               lse=True, **kw)
        path, _ = c.commit(self.parent, self.token, self.accepted, self.accept_len, self.lens,
                           self.table, self.kc, self.vc, **kw,
                           out=(torch.empty((self.B, self.depth + 1), dtype=torch.int32,
                                            device="cuda"), self.lens))
        scores = self.scorer.logprobs(self.logits, self.emitted, path=path, top=4, **kw)
        c.plan(*state, 0, **kw)
        return [slots, pos, status, path] + out + list(scores)

    def close(self):
        self.cache.close()
        self.scorer.close()


def _same(xs, ys):
    for i, (x, y) in enumerate(zip(xs, ys)):
        assert torch.equal(x, y), i


def test_steps_on_the_default_and_another_stream(binding):
    a, b = Loop(binding), Loop(binding)
    side = torch.cuda.Stream()
    for seed in range(4):
        a.feed(seed), b.feed(seed)
        want = a.step()
        side.wait_stream(torch.cuda.current_stream())
        got = b.step(stream=side)
        torch.cuda.current_stream().wait_stream(side)
        _same(got, want)
        _same(b.state(), a.state())
    assert a.cache.device_error() == 0 and b.cache.device_error() == 0
    a.close(), b.close()


def test_a_captured_step_replays(binding):
    """The same step captured once and replayed on new inputs, with eager steps of
    another loop and synchronisations between; against eager results each time."""
    a, b = Loop(binding), Loop(binding)
    a.feed(100), b.feed(100)
    _same(b.step(), a.step())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        before = [t.clone() for t in b.state()]
        b.step()                                       # warm-up of the allocator
        for t, x in zip(b.state(), before):
            t.copy_(x)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = b.step()
    for seed in range(5):
        a.feed(seed), b.feed(seed)
        want = a.step()
        graph.replay()
        torch.cuda.synchronize()
        _same(got, want)
        _same(b.state(), a.state())
    assert b.cache.device_error() == 0
    a.close(), b.close()


def test_handles_side_by_side_on_two_streams(binding):
    """Two handles at work at once do not share workspaces."""
    s = [Setup(binding, BF16, [3000, 700], 61, 61, 8, 2, 128, 16, seed=k) for k in (1, 2)]
    mask = [_tree_mask(x.g, 2, 61).cuda() for x in s]
    args = [(x.q.cuda(), *x.pages_on_gpu(), x.table.cuda(), _i32(x.lens)) for x in s]
    want = [x.cache.attention(*a, mask=m).clone() for x, a, m in zip(s, args, mask)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in s]
    got = [[], []]
    for _ in range(10):
        for k in (0, 1):
            with torch.cuda.stream(streams[k]):
                got[k].append(s[k].cache.attention(*args[k], mask=mask[k]))
    torch.cuda.synchronize()
    for k in (0, 1):
        for x in got[k]:
            assert torch.equal(x, want[k])
        s[k].cache.close()


def test_results_do_not_depend_on_earlier_calls(binding):
    """A call after others of other sizes on the same handle: nothing of theirs is left, nor of
    one with a length past the pages that a sequence holds, which sets its error bit (the
    third's 70 entries: its row of the table names four pages of 16, then -7)."""
    s = Setup(binding, BF16, [900, 33, 0], 61, 61, 8, 2, 128, 16)
    mask = _tree_mask(s.g, 3, 61).cuda()
    a = (s.q.cuda(), *s.pages_on_gpu(), s.table.cuda(), _i32(s.lens))
    want = s.cache.attention(*a, mask=mask).clone()
    one = s.q.cuda()[:, :1].contiguous()
    for q, lens in ((one, [0, 0, 5]), (one, [900, 50, 70]), (a[0], [0, 0, 0])):
        s.cache.attention(q, *a[1:4], _i32(lens), mask=None)
        assert torch.equal(s.cache.attention(*a, mask=mask), want)
    assert s.cache.device_error() == 8
    s.cache.close()


def test_entries_past_32_bits_of_offset(binding):
    """A pool of 5 GiB of keys: pages at its end, behind 2^32 bytes and 2^31 elements, written,
    attended and moved as the same entries of a small pool are."""
    B, n, H, K, D, page, depth = 1, 20, 8, 8, 128, 64, 5
    far, near = 41000, 4
    g = torch.Generator().manual_seed(0)
    q, k, v = ((torch.randn((B, n, h, D), generator=g)).to(BF16).cuda() for h in (H, K, K))
    old = [torch.randn((near, page, K, D), generator=g).to(BF16).cuda() for _ in range(2)]
    mask = _tree_mask(g, B, n).cuda()
    parent = _i32([[-1] + [i - 1 for i in range(1, n)]])
    token = _i32([[-1] + list(range(1, n))])
    lens, took = _i32([3 * page - 7]), _i32([3])
    accepted = _i32([[1, 2, 3, -1, -1]])
    parent[0, 1:4] = torch.tensor([0, 4, 9], dtype=torch.int32)      # 0 -> 4 -> 9 -> 15
    parent[0, 4], parent[0, 9], parent[0, 15] = 0, 4, 9
    token[0, 4], token[0, 9], token[0, 15] = 101, 102, 103
    accepted[0, :3] = torch.tensor([101, 102, 103], dtype=torch.int32)
    got = []
    for pages, first in ((near, 0), (far, far - near)):
        c = binding.Cache(batch=B, heads=H, kv_heads=K, head_dim=D, page_size=page, pages=pages,
                          table_width=near)
        pools = [torch.empty((1, pages, page, K, D), dtype=BF16, device="cuda") for _ in range(2)]
        for pool, x in zip(pools, old):
            pool[0, first:] = x
        table = _i32([[first + i for i in (2, 0, 3, 1)]])
        e = torch.arange(n, device="cuda") + int(lens)
        slots = (table[0].long()[e // page] * page + e % page)[None]
        c.write(q, k, v, slots, pools[0][0], pools[1][0])
        out, lse = c.attention(q, pools[0][0], pools[1][0], table, lens, mask=mask, lse=True)
        path, new = c.commit(parent, token, accepted, took, lens, table, *pools)
        assert c.device_error() == 0
        got.append([out, lse, path, new] + [pool[0, first:].clone() for pool in pools])
        c.close()
        del pools
    assert got[0][2].tolist() == [[0, 4, 9, 15, -1, -1]]
    _same(*got)


# -- whole decoding steps -----------------------------------------------------------------


def test_decoding_steps_with_a_model(binding):
    """Trees built from a model's logits, scored in one pass over the cache, verified,
    committed; step after step.  The target rows are those of the model run token
    by token over every node's path with a dense cache of its own, and what is in the pages
    after a commit is what that run holds."""
    torch.manual_seed(0)
    B, H, K, D, layers, V, depth, R, page, T = 2, 4, 2, 64, 2, 320, 3, 12, 16, 1.0
    E = H * D
    emb = torch.randn(V, E, device="cuda") * 0.5
    w_in = [torch.randn(E, (H + 2 * K) * D, device="cuda") / E ** 0.5 for _ in range(layers)]
    w_out = [torch.randn(H * D, E, device="cuda") / E ** 0.5 for _ in range(layers)]
    head = torch.randn(E, V, device="cuda") * 4 / E ** 0.5
    half = D // 2
    ang = torch.arange(300, dtype=torch.float64)[:, None] * 100.0 ** (-torch.arange(half) / half)
    rot = torch.cat([ang.cos(), ang.sin()], 1).float().cuda()
    width = 8
    cache = binding.Cache(batch=B, heads=H, kv_heads=K, head_dim=D, page_size=page,
                          pages=B * width, table_width=width, layers=layers)
    kc, vc = (torch.zeros((layers, B * width, page, K, D), dtype=BF16, device="cuda")
              for _ in range(2))
    table = torch.zeros((B, width), dtype=torch.int32, device="cuda")
    lens, held = _i32([0] * B), _i32([0] * B)
    free, free_count = torch.randperm(B * width).int().cuda(), _i32([B * width])

    def forward(tokens, mask, depths):
        """The model on rows of tokens [B, n] behind the cache; bf16 logits [B, n, V]."""
        n = tokens.shape[1]
        state = (lens, held, table, free, free_count)
        slots, pos, status = cache.plan(*state, n, depth=depths)
        assert (status == 0).all()
        x = emb[tokens.long()]
        for i in range(layers):
            q, k, v = (x @ w_in[i]).to(BF16).split([H * D, K * D, K * D], dim=2)
            q = cache.write(q.unflatten(2, (H, D)), k.unflatten(2, (K, D)), v.unflatten(2, (K, D)),
                            slots, kc[i], vc[i], positions=pos, rotation=rot)
            x = x + cache.attention(q, kc[i], vc[i], table, lens, mask=mask).flatten(2).float() @ w_out[i]
        return (x @ head).to(BF16)

    def dense(tokens):
        """64-bit logits after every token of one sequence, and each layer's keys and values."""
        n = len(tokens)
        x = emb[torch.tensor(tokens, device="cuda")].double()
        kv = []
        for i in range(layers):
            q, k, v = (x @ w_in[i].double()).split([H * D, K * D, K * D], dim=1)
            pos = torch.arange(n)
            q = ref.write_heads(q.cpu().view(n, H, D), None, 0, rot.cpu(), pos, False)[0].cuda()
            k = ref.write_heads(k.cpu().view(n, K, D), None, 0, rot.cpu(), pos, False)[0].cuda()
            v = v.view(n, K, D)
            kv.append((k, v))
            s = torch.einsum("ihd,jhd->hij", q, k.repeat_interleave(H // K, 1)) * D ** -0.5
            s.masked_fill_(torch.ones(n, n, device="cuda").triu(1) > 0, -math.inf)
            o = torch.einsum("hij,jhd->ihd", s.softmax(2), v.repeat_interleave(H // K, 1))
            x = x + o.reshape(n, E) @ w_out[i].double()
        return x @ head.double(), kv

    tree = binding.Tree(batch=B, vocab=V, pool=4, leads=1, depth=depth, support=64, dtype=BF16)
    scorer = binding.Scorer(V, BF16)
    done = [[int(t) for t in torch.randint(0, V, (9,))] for _ in range(B)]
    prompt = torch.tensor([d[:-1] for d in done], dtype=torch.int32, device="cuda")
    forward(prompt, None, None)                        # causal, into the cache
    lens += 8
    # roundings to bf16: the projections' outputs, the keys' and queries' after the rotation, the
    # probabilities, the attention's output, each 2^-8 of it at most and a layer's
    # results passing through the next; and the logits'
    bound = (5 * layers + 1) * 2.0 ** -8
    accepted_any = 0
    for step in range(4):
        key = 1000 + step
        tree.begin_step()
        rows = [[d] for d in done]                     # each frontier node's tokens so far
        for level in range(depth):
            logits = torch.stack([torch.stack([dense(r)[0][-1] for r in rows_b])
                                  for rows_b in rows]).to(BF16)
            tree.expand_level(logits.contiguous(), T, key)
            if level + 1 < depth:
                par, tok = (t.cpu().tolist() for t in tree.frontier())
                rows = [[rows[b][par[b][j]] + [tok[b][j]] for j in range(len(par[b]))]
                        for b in range(B)]
        tree.prune(R)
        parent, token = tree.pruned_view()
        mask, depths = tree.tree_mask()
        rows_in = token.clone()
        rows_in[:, 0] = _i32([d[-1] for d in done])
        target = forward(rows_in, mask, depths)
        for b in range(B):
            for i in range(R + 1):
                path = [j for j in range(1, R + 1) if mask[b, i, j]]
                want = dense(done[b] + [int(token[b, j]) for j in path])[0][-1]
                off = (target[b, i].double() - want).norm() / want.norm()
                assert off <= bound, (step, b, i, float(off))
        acc, alen, final = tree.verify(target, T, key)
        assert (alen >= 0).all()
        accepted_any += int(alen.sum())
        emitted = torch.cat([acc, torch.full((B, 1), -1, dtype=torch.int32, device="cuda")], 1)
        emitted[torch.arange(B), alen.long()] = final
        path, _ = cache.commit(parent, token, acc, alen, lens, table, kc, vc,
                               out=(torch.empty((B, depth + 1), dtype=torch.int32, device="cuda"),
                                    lens))
        logp = scorer.logprobs(target, emitted, path=path, top=3)[0]
        for b in range(B):
            took = int(alen[b])
            nodes = path[b].tolist()
            assert nodes[0] == 0 and nodes[took + 1:] == [-1] * (depth - took)
            assert [int(token[b, j]) for j in nodes[1:took + 1]] == acc[b, :took].tolist()
            for j in range(took + 1):
                w = target[b, nodes[j]].double().log_softmax(0)[emitted[b, j].long()]
                assert abs(float(logp[b, j]) - float(w)) <= 2.0 ** -24 * (200 + 20 * abs(float(w)))
            done[b] += emitted[b, :took + 1].tolist()
            assert int(lens[b]) == len(done[b]) - 1
            _, kv = dense(done[b][:-1])
            e = torch.arange(int(lens[b]), device="cuda")
            for i in range(layers):
                for pages, want in ((kc[i], kv[i][0]), (vc[i], kv[i][1])):
                    got = pages.flatten(0, 1)[table[b].long()[e // page] * page + e % page].double()
                    assert (got - want).norm() / want.norm() <= bound
        cache.plan(lens, held, table, free, free_count, 0)
        assert held.tolist() == [-(-int(x) // page) for x in lens]
    assert accepted_any > 0
    assert cache.device_error() == 0 and tree.device_error() == 0
    tree.close(), cache.close(), scorer.close()


def test_smallest_scale_and_scales_out_of_range(binding):
    """2^-100: all weights are the same.  A scale so small that 8 / scale is infinite would
    leave the running maximum where it began, and is refused."""
    s = Setup(binding, BF16, [40], 3, 3, 4, 2, 64, 16)
    q = s.q.cuda()
    kc, vc = s.pages_on_gpu()
    table, lens = s.table.cuda(), _i32(s.lens)
    _, lse = s.cache.attention(q, kc, vc, table, lens, scale=2.0 ** -100, lse=True)
    want = torch.tensor([41.0, 42.0, 43.0]).double().log()
    # 43 terms of 1 are exact; their logarithm and its sum with 0: some roundings
    assert ((lse.cpu().double() - want[None, :, None]).abs() <= 8 * 2.0 ** -24 * 4).all()
    for bad in (2.0 ** -101, 1e-38, 2.0 ** 101, 3e38, 0.0, -1.0, float("inf"), float("nan")):
        with pytest.raises(binding.RheoError):
            s.cache.attention(q, kc, vc, table, lens, scale=bad)
    s.cache.close()
