"""The cache and scoring operators whose speed counts: cases, inputs, plain forms.

Around a drafted tree a serving loop makes room in its paged key/value cache
(plan), stores the rows' keys and values there (write), attends from every row to
the prefix and to its ancestors (attention), moves the accepted path's entries
together (commit) and reports log probabilities (logprobs).  Each case is one
pass through one of them.  ``run`` computes it with elementary torch operations,
or, where ``own`` is true, with the calls of ``paper_2609_21827_amd.binding``.
"""

import math
import random

import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}

# Heads: "heads" query heads share "kv_heads" key/value heads of "dim" elements.
_BASE = {
    "plan": dict(op="plan", B=1, n=61, page=64, ctx=2000, spare=1.0, ragged=False),
    "write": dict(op="write", B=1, n=61, page=64, heads=32, kv_heads=8, dim=128, dtype="bf16",
                  norm=True, rot=128, pairs=False, ragged=False),
    "attention": dict(op="attention", B=1, n=61, page=64, heads=32, kv_heads=8, dim=128,
                      dtype="bf16", ctx=2000, tree=True, ragged=False),
    "commit": dict(op="commit", B=1, n=61, depth=7, page=64, layers=32, kv_heads=8, dim=128,
                   dtype="bf16", ctx=2000),
    "logprobs": dict(op="logprobs", B=1, n=61, m=8, V=128256, dtype="bf16", top=5, T=1.0),
}


def _case(op, **kw):
    c = dict(_BASE[op])
    c.update(kw)
    return c


def listed():
    return [
        # one conversation: room for the next tree, every step
        _case("plan", name="plan_b1"),
        # a full server: many sequences of all lengths, small pages, a pool that
        # does not hold what all of them ask for
        _case("plan", name="plan_b1024", B=1024, n=81, page=16, ctx=30000, spare=0.9, ragged=True),
        # the tree's rows of one conversation in one layer
        _case("write", name="write_b1"),
        # the largest batch: as many key heads as query heads, half of each head
        # rotated in neighbouring pairs, some rows of each sequence empty
        _case("write", name="write_b128_mha", B=128, n=81, page=16, heads=40, kv_heads=40,
              dtype="f16", norm=False, rot=64, pairs=True, ragged=True),
        # one token of one short conversation
        _case("attention", name="attn_b1_n1", n=1, ctx=517, tree=False),
        # the headline serving batch: a tree of 60 drafted tokens each
        _case("attention", name="attn_b64_tree", B=64, ctx=4096),
        # one tree over a very long context
        _case("attention", name="attn_b1_long", ctx=131011),
        # plain decoding of many sequences, seven query heads to a key head
        _case("attention", name="attn_b128_n1", B=128, n=1, page=16, heads=28, kv_heads=4,
              dtype="f16", ctx=8191, tree=False),
        # the accepted path of one conversation, all layers
        _case("commit", name="commit_b1"),
        # the same for the largest batch
        _case("commit", name="commit_b128", B=128, n=81, depth=8, page=16, ctx=6000),
        # what one conversation's step emitted, fp32 logits, a small vocabulary
        _case("logprobs", name="logp_b1", m=7, V=32000, dtype="f32"),
        # the largest batch and vocabulary, twenty alternatives each
        _case("logprobs", name="logp_b128", B=128, n=81, m=9, V=151936, top=20, T=0.8),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


_HEADS = [(32, 8), (32, 8), (40, 40), (28, 4), (64, 8), (16, 16), (8, 1), (10, 2), (5, 5), (20, 4)]
_DIMS = [128, 128, 128, 64, 64, 80, 112, 160, 256]
_most = {}


def draw(rng):
    """A case of the same ranges.  No dearer than the largest listed one of its operator."""
    op = rng.choice(["plan", "write", "attention", "attention", "attention", "commit", "logprobs"])
    c = _case(op)
    c["B"] = _log_int(rng, 1, 1024 if op == "plan" else 128)
    c["n"] = rng.choice([1, rng.randint(2, 80), rng.randint(20, 80), rng.randint(20, 80)])
    if op != "logprobs":
        c["page"] = rng.choice([16, 32, 64, 64, 128, 256])
    if op in ("write", "attention", "commit"):
        heads, c["kv_heads"] = rng.choice(_HEADS)
        if op != "commit":
            c["heads"] = heads
        c["dim"] = rng.choice(_DIMS)
        c["dtype"] = rng.choice(["bf16", "bf16", "f16"])
    if op in ("plan", "write", "attention"):
        c["ragged"] = rng.random() < 0.7
    if op == "plan":
        c["ctx"] = _log_int(rng, 1, 30000)
        c["spare"] = rng.choice([1.0, 1.0, 0.8])
    elif op == "write":
        c["n"] = rng.choice([c["n"], _log_int(rng, 1, 4000)])
        c["norm"] = rng.random() < 0.6
        c["rot"] = rng.choice([c["dim"], c["dim"], c["dim"] // 2, 0])
        c["pairs"] = rng.random() < 0.4
    elif op == "attention":
        c["ctx"] = _log_int(rng, 1, 131000)
        c["tree"] = c["n"] > 1 and rng.random() < 0.8
        if c["n"] > 1 and not c["tree"]:
            c["n"] = _log_int(rng, 2, 2000)
    elif op == "commit":
        c["n"] = max(c["n"], 17)
        c["depth"] = rng.randint(1, 8)
        c["layers"] = rng.choice([1, 16, 32])
        c["ctx"] = _log_int(rng, 1, 6000)
    else:
        c["m"] = min(c["n"], rng.randint(1, 9))
        c["V"] = _log_int(rng, 1000, 262143)
        c["dtype"] = rng.choice(["bf16", "bf16", "f16", "f32"])
        c["top"] = rng.choice([0, 1, 5, 20, 32])
        c["T"] = rng.choice([0.6, 0.8, 1.0, 1.5])
    if op not in _most:
        every = [work(x) for x in listed() if x["op"] == op]
        _most[op] = {k: max(w[k] for w in every) for k in ("bytes", "flops")}
    size = "ctx" if op == "attention" else "n" if op == "write" else "B"
    for key in [size, "B", "n"]:
        while c[key] > 1 and any(work(c)[k] > _most[op][k] for k in _most[op]):
            c[key] = max(1, int(c[key] * 0.8))
    if op == "attention" and c["n"] == 1:
        c["tree"] = False
    if op == "logprobs":
        c["m"] = min(c["m"], c["n"])
    return c


# -- sizes that follow from a case alone ---------------------------------------


def _lens(c):
    """Tokens in the cache of each sequence before the pass."""
    if c["B"] == 1:
        return [c["ctx"]]
    rng = random.Random(c["B"] * 7919 + c["ctx"])
    return [max(1, int(c["ctx"] * rng.uniform(0.25, 1.0))) for _ in range(c["B"])]


def _counts(c):
    """Rows of each sequence: all of them, or (ragged) some, in a few sequences none."""
    if not c["ragged"] or c["n"] == 1:
        return [c["n"]] * c["B"]
    rng = random.Random(c["B"] * 104729 + c["n"])
    return [0 if b and rng.random() < 0.05 else rng.randint(1, c["n"]) for b in range(c["B"])]


def _accept(c):
    """Tokens accepted in each sequence."""
    rng = random.Random(c["B"] * 1299709 + c["n"])
    most = min(c["depth"] if c["op"] == "commit" else c["m"] - 1, (c["n"] - 1) // 2)
    return [rng.randint(0, most) for _ in range(c["B"])]


def _esz(c):
    return 4 if c["dtype"] == "f32" else 2


def _stride(c):
    unit = 16 // _esz(c)
    return (c["V"] + unit - 1) // unit * unit


def _up(a, b):
    return -(-a // b)


# -- inputs ---------------------------------------------------------------------


def _ints(rows, dtype=torch.int32):
    return torch.tensor(rows, dtype=dtype, device="cuda")


def _normal(g, shape, c):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(_TYPES[c["dtype"]])


def _pages(g, needs, width):
    """A block table [B, width] over a pool in random order, and the pool's size."""
    total = sum(needs)
    order = torch.randperm(total, generator=g, device="cuda").to(torch.int32)
    first = torch.tensor([0] + needs, device="cuda").cumsum(0)
    place = first[:-1, None] + torch.arange(width, device="cuda")
    held = torch.arange(width, device="cuda") < _ints(needs)[:, None]
    return torch.where(held, order[place.clamp(max=total - 1)], 0).to(torch.int32), total


def _tree(g, B, n, depth_most):
    """Parents [B, n] of random trees, every parent before its children, and depths."""
    parent = torch.full((B, n), -1, dtype=torch.int64, device="cuda")
    depth = torch.zeros((B, n), dtype=torch.int64, device="cuda")
    u = torch.rand((B, n), generator=g, device="cuda")
    b = torch.arange(B, device="cuda")
    for i in range(1, n):
        p = (u[:, i] * u[:, i] * i).long().clamp(max=i - 1)
        p = torch.where(depth[b, p] >= depth_most, 0, p)
        parent[:, i] = p
        depth[:, i] = depth[b, p] + 1
    return parent, depth


def _prepare_plan(c, g):
    B, n, page = c["B"], c["n"], c["page"]
    lens, counts = _lens(c), _counts(c)
    held = [_up(x, page) for x in lens]
    width = max(_up(x + n, page) for x in lens)
    more = sum(_up(x + k, page) - h for x, k, h in zip(lens, counts, held))
    table, used = _pages(g, held, width)
    free = torch.randperm(more, generator=g, device="cuda").to(torch.int32) + used
    free = free[:int(c["spare"] * more)]               # the pool's other pages, some taken
    free_list = torch.zeros(used + more, dtype=torch.int32, device="cuda")
    free_list[:free.numel()] = free
    return dict(lens=_ints(lens), count=_ints(counts), held=_ints(held), table=table,
                free_list=free_list, free_count=_ints([free.numel()]),
                depth=_tree(g, B, n, 8)[1].to(torch.int32), pages=used + more, width=width)


def _prepare_write(c, g):
    B, n, page, H, K, D = c["B"], c["n"], c["page"], c["heads"], c["kv_heads"], c["dim"]
    counts = _ints(_counts(c))
    pages = _up(B * n, page) + 1
    place = torch.randperm(pages, generator=g, device="cuda")
    at = torch.arange(B * n, device="cuda") + 3        # rows begin inside a page
    at = at % (pages * page)
    slots = (place[at // page] * page + at % page).view(B, n)
    slots = torch.where(torch.arange(n, device="cuda") < counts[:, None], slots, -1)
    most = 40960
    positions = torch.randint(0, most - n, (B, 1), generator=g, device="cuda") + \
        torch.arange(n, device="cuda")
    qkv = _normal(g, (B, n, (H + 2 * K) * D), c)       # one projection's output
    q, k, v = qkv.split([H * D, K * D, K * D], dim=2)
    s = dict(q=q.unflatten(2, (H, D)), k=k.unflatten(2, (K, D)), v=v.unflatten(2, (K, D)),
             slots=slots, spare=place[-1] * page + page - 1,   # a slot of no row
             positions=positions.to(torch.int32), rotation=None,
             q_weight=None, k_weight=None, pages=pages, width=1,
             k_cache=_normal(g, (pages, page, K, D), c), v_cache=_normal(g, (pages, page, K, D), c),
             out=torch.zeros((B, n, H, D), dtype=_TYPES[c["dtype"]], device="cuda"))
    if c["rot"]:
        half = c["rot"] // 2
        rate = 500000.0 ** (-torch.arange(half, dtype=torch.float64, device="cuda") / half)
        angle = torch.arange(most, dtype=torch.float64, device="cuda")[:, None] * rate
        s["rotation"] = torch.cat([angle.cos(), angle.sin()], 1).float()
    if c["norm"]:
        s["q_weight"] = (1 + 0.2 * torch.randn(D, generator=g, device="cuda")).to(_TYPES[c["dtype"]])
        s["k_weight"] = (1 + 0.2 * torch.randn(D, generator=g, device="cuda")).to(_TYPES[c["dtype"]])
    return s


def _prepare_attention(c, g):
    B, n, page, K, D = c["B"], c["n"], c["page"], c["kv_heads"], c["dim"]
    lens, counts = _lens(c), _counts(c)
    needs = [_up(x + k, page) for x, k in zip(lens, counts)]
    width = max(_up(x + n, page) for x in lens)
    table, pages = _pages(g, needs, width)
    s = dict(q=_normal(g, (B, n, c["heads"], D), c) * 1.5, table=table, lens=_ints(lens),
             count=_ints(counts) if c["ragged"] else None, mask=None, pages=pages, width=width,
             k_cache=_normal(g, (pages, page, K, D), c), v_cache=_normal(g, (pages, page, K, D), c),
             out=torch.zeros((B, n, c["heads"], D), dtype=_TYPES[c["dtype"]], device="cuda"),
             lse=torch.zeros((B, n, c["heads"]), dtype=torch.float32, device="cuda"))
    if c["tree"]:
        parent, _ = _tree(g, B, n, 8)
        mask = torch.zeros((B, n, n), dtype=torch.uint8, device="cuda")
        b = torch.arange(B, device="cuda")
        for i in range(n):
            if i:
                mask[:, i] = mask[b, parent[:, i]]
            mask[:, i, i] = 1
        s["mask"] = mask
    return s


def _prepare_commit(c, g):
    B, n, page, K, D, depth = c["B"], c["n"], c["page"], c["kv_heads"], c["dim"], c["depth"]
    lens, took = _lens(c), _accept(c)
    # the pages of the drafted rows; what lies before them is not touched, so all
    # of it stands on the pool's page 0
    first = [x // page for x in lens]
    last = [_up(x + n, page) for x in lens]
    width = max(last)
    place = torch.arange(width, device="cuda")[None, :] - _ints(first)[:, None]
    new, pages = _pages(g, [b - a for a, b in zip(first, last)], max(b - a for a, b in zip(first, last)))
    at = place.clamp(0, new.shape[1] - 1).long()
    table = torch.where(place >= 0, new.gather(1, at) + 1, 0).to(torch.int32)
    pages += 1
    # an accepted path whose nodes rank behind the path's length, each a child of
    # the one before, so that a pass can be repeated on the same entries
    parent, _ = _tree(g, B, n, depth)
    token = torch.stack([torch.randperm(50000, generator=g, device="cuda")[:n] for _ in range(B)])
    order = torch.rand((B, n), generator=g, device="cuda")
    behind = _ints([x + 1 for x in took])[:, None]
    ranks = torch.arange(n, device="cuda")
    order = torch.where(ranks >= behind, order, 2.0)
    chosen = order.argsort(1)[:, :max(1, max(took))]
    chosen = torch.where(torch.arange(chosen.shape[1], device="cuda") < behind - 1, chosen, n).sort(1)[0]
    accepted = torch.full((B, depth), -1, dtype=torch.int32, device="cuda")
    b = torch.arange(B, device="cuda")
    before = torch.zeros(B, dtype=torch.int64, device="cuda")
    for j in range(max(took)):
        node = chosen[:, j]
        live = node < n
        node = node.clamp(max=n - 1)
        parent[b, node] = torch.where(live, before, parent[b, node])
        accepted[:, j] = torch.where(live, token[b, node], -1).to(torch.int32)
        before = torch.where(live, node, before)
    token[:, 0] = -1
    shape = (c["layers"], pages, page, K, D)
    return dict(parent=parent.to(torch.int32), token=token.to(torch.int32), accepted=accepted,
                accept_len=_ints(took), lens=_ints(lens), table=table, pages=pages, width=width,
                k_cache=_normal(g, shape, c), v_cache=_normal(g, shape, c),
                path=torch.zeros((B, depth + 1), dtype=torch.int32, device="cuda"),
                new_lens=torch.zeros(B, dtype=torch.int32, device="cuda"))


def _prepare_logprobs(c, g):
    B, n, m, V, top = c["B"], c["n"], c["m"], c["V"], c["top"]
    logits = torch.zeros((B, n, _stride(c)), dtype=_TYPES[c["dtype"]], device="cuda")
    base = -1.1 * torch.log1p(torch.arange(V, dtype=torch.float32, device="cuda"))
    for b in range(B):                                 # a Zipf prior in an order of its own, and noise
        x = torch.randn((n, V), generator=g, device="cuda")
        logits[b, :, :V] = x.mul_(1.5).add_(base[torch.randperm(V, generator=g, device="cuda")])
    rows = _ints([x + 1 for x in _accept(c)])[:, None]  # the accepted tokens and the final one
    live = torch.arange(m, device="cuda") < rows
    path = torch.rand((B, n), generator=g, device="cuda").argsort(1)[:, :m].sort(1)[0]
    # tokens of the first five, or any
    best = logits[torch.arange(B, device="cuda")[:, None], path][:, :, :V].float().topk(5, dim=2)[1]
    pick = torch.randint(0, 5, (B, m, 1), generator=g, device="cuda")
    anyone = torch.randint(0, V, (B, m), generator=g, device="cuda")
    token = torch.where(torch.rand((B, m), generator=g, device="cuda") < 0.8,
                        best.gather(2, pick)[:, :, 0], anyone)
    f32, i32 = dict(dtype=torch.float32, device="cuda"), dict(dtype=torch.int32, device="cuda")
    return dict(logits=logits, path=torch.where(live, path, -1).to(torch.int32),
                tokens=torch.where(live, token, -1).to(torch.int32),
                out=(torch.zeros((B, m), **f32), torch.zeros((B, m), **f32),
                     torch.zeros((B, m), **i32), torch.zeros((B, m, top), **i32),
                     torch.zeros((B, m, top), **f32)))


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    state = globals()["_prepare_" + case["op"]](case, g)
    state["case"] = case
    if own:                                            # the handle that a program keeps
        state["handle"] = _handle(case, state)
    return state


def _handle(c, s):
    from paper_2609_21827_amd.binding import Cache, Scorer
    if c["op"] == "logprobs":
        return Scorer(vocab=c["V"], dtype=_TYPES[c["dtype"]], row_stride=_stride(c))
    return Cache(batch=c["B"], heads=c.get("heads", c.get("kv_heads", 1)),
                 kv_heads=c.get("kv_heads", 1), head_dim=c.get("dim", 128), page_size=c["page"],
                 pages=s["pages"], table_width=s["width"], layers=c.get("layers", 1),
                 dtype=_TYPES[c.get("dtype", "bf16")])


# -- one pass ---------------------------------------------------------------------


def run(state):
    return globals()[("_own_" if own else "_plain_") + state["case"]["op"]](state["case"], state)


def _own_plan(c, s):
    args = (s["lens"], s["held"], s["table"], s["free_list"], s["free_count"])
    slots, positions, status = s["handle"].plan(*args, c["n"], count=s["count"], depth=s["depth"])
    # the step over, nothing kept: what the drafted rows took goes back
    _, _, after = s["handle"].plan(*args, 0)
    return dict(slots=slots, positions=positions, status=status, after=after, table=s["table"],
                held=s["held"], free_list=s["free_list"], free_count=s["free_count"])


def _plain_plan(c, s):
    slots, positions, status = _plan_once(c, s, c["n"], s["count"].long(), s["depth"])
    after = _plan_once(c, s, 0, torch.zeros_like(s["lens"]).long(), None)[2]
    return dict(slots=slots, positions=positions, status=status, after=after, table=s["table"],
                held=s["held"], free_list=s["free_list"], free_count=s["free_count"])


def _plan_once(c, s, n, count, depth):
    page, table, width = c["page"], s["table"], s["width"]
    lens, held, have = s["lens"].long(), s["held"].long(), s["free_count"].long()
    need = (lens + count + page - 1) // page
    fits = need <= width
    take = torch.where(fits, (need - held).clamp(min=0), 0)
    give = torch.where(fits, (held - need).clamp(min=0), 0)
    freed, asked = give.cumsum(0), take.cumsum(0)
    room = have + freed[-1]
    served = fits & ((take == 0) | (asked <= room))
    take = torch.where(served, take, 0)
    place = torch.arange(width, device="cuda")[None, :]
    # the stack after the released pages, pushed from the last to the first
    total = freed[-1]
    size = s["free_list"].numel()
    ordinal = (freed - give)[:, None] + place - need[:, None]
    released = (place >= need[:, None]) & (place < held[:, None]) & fits[:, None]
    stack = torch.cat([s["free_list"], s["free_list"].new_zeros(1)])
    stack.scatter_(0, torch.where(released, have + total - 1 - ordinal, size).clamp(max=size).flatten(),
                   table.flatten())
    first = take.cumsum(0) - take
    top = room - 1 - first[:, None] - (place - held[:, None])
    new = (place >= held[:, None]) & (place < (held + take)[:, None])
    table.copy_(torch.where(new, stack[top.clamp(0, size)], table))
    left = room - take.sum()
    at = torch.arange(size, device="cuda")
    s["free_list"].copy_(torch.where((at >= have) & (at < left), stack[:size], s["free_list"]))
    s["free_count"].copy_(left)
    s["held"].copy_(torch.where(served, need, held))
    i = torch.arange(n, device="cuda")[None, :]
    live = (i < count[:, None]) & served[:, None]
    pos = lens[:, None] + i
    pg = table.gather(1, (pos // page).clamp(max=width - 1)).long()
    slots = torch.where(live, pg * page + pos % page, -1)
    positions = lens[:, None] + (i if depth is None else depth.long())
    status = torch.where(fits, torch.where(served, 0, 1), 2)
    return slots, torch.where(live, positions, -1).to(torch.int32), status.to(torch.int32)


def _own_write(c, s):
    out = s["handle"].write(s["q"], s["k"], s["v"], s["slots"], s["k_cache"], s["v_cache"],
                            positions=s["positions"], rotation=s["rotation"],
                            interleaved=c["pairs"], q_weight=s["q_weight"], k_weight=s["k_weight"],
                            eps=1e-6, out=s["out"])
    return dict(q=out, k_cache=s["k_cache"], v_cache=s["v_cache"])


def _plain_write(c, s):
    live = s["slots"] >= 0
    q = _rotated(c, s, _normed(s["q"].float(), s["q_weight"]))
    k = _rotated(c, s, _normed(s["k"].float(), s["k_weight"]))
    s["out"].copy_(torch.where(live[:, :, None, None], q.to(s["out"].dtype), s["out"]))
    # rows without a slot write the spare slot as it is
    at = torch.where(live, s["slots"], s["spare"])
    for cache, x in ((s["k_cache"], k), (s["v_cache"], s["v"])):
        flat = cache.flatten(0, 1)
        flat[at] = torch.where(live[:, :, None, None], x.to(cache.dtype), flat[s["spare"]])
    return dict(q=s["out"], k_cache=s["k_cache"], v_cache=s["v_cache"])


def _normed(x, w):
    if w is None:
        return x
    return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * w.float()


def _rotated(c, s, x):
    r = c["rot"]
    if not r:
        return x
    row = s["rotation"][s["positions"].long()]
    cos, sin = row[:, :, None, :r // 2], row[:, :, None, r // 2:]
    y = x.clone()
    one, two = (slice(0, r, 2), slice(1, r, 2)) if c["pairs"] else (slice(0, r // 2), slice(r // 2, r))
    a, b = x[..., one], x[..., two]
    y[..., one] = a * cos - b * sin
    y[..., two] = b * cos + a * sin
    return y


def _own_attention(c, s):
    out, lse = s["handle"].attention(s["q"], s["k_cache"], s["v_cache"], s["table"], s["lens"],
                                     mask=s["mask"], count=s["count"], out=s["out"], lse=s["lse"])
    return dict(out=out, lse=lse)


def _plain_attention(c, s):
    B, n, H, K, D, page = c["B"], c["n"], c["heads"], c["kv_heads"], c["dim"], c["page"]
    L = s["width"] * page
    k = s["k_cache"][s["table"].long()].view(B, L, K, D).permute(0, 2, 3, 1).float().contiguous()
    v = s["v_cache"][s["table"].long()].view(B, L, K, D).permute(0, 2, 1, 3).float().contiguous()
    q = s["q"].float().view(B, n, K, H // K, D).permute(0, 2, 1, 3, 4).reshape(B, K, -1, D)
    score = torch.matmul(q, k).mul_(D ** -0.5).view(B, K, n, H // K, L)
    count = s["count"] if s["count"] is not None else torch.full_like(s["lens"], n)
    j = torch.arange(L, device="cuda")[None, None, :] - s["lens"][:, None, None]
    i = torch.arange(n, device="cuda")[None, :, None]
    if s["mask"] is not None:
        seen = s["mask"].gather(2, j.clamp(0, n - 1).expand(B, n, L).long()) != 0
    else:
        seen = j <= i
    seen = (j < 0) | (seen & (j < count[:, None, None]))
    score.masked_fill_(~seen[:, None, :, None, :], -math.inf)
    top = score.amax(-1, keepdim=True)
    p = score.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p.view(B, K, -1, L), v).view(B, K, n, H // K, D)
    out = torch.where(total > 0, out / total, 0.0).permute(0, 2, 1, 3, 4).reshape(B, n, H, D)
    lse = (top + total.log())[..., 0].permute(0, 2, 1, 3).reshape(B, n, H)
    live = i < count[:, None, None]
    s["out"].copy_(torch.where(live[..., None], out.to(s["out"].dtype), s["out"]))
    s["lse"].copy_(torch.where(live, lse, s["lse"]))
    return dict(out=s["out"], lse=s["lse"])


def _own_commit(c, s):
    path, lens = s["handle"].commit(s["parent"], s["token"], s["accepted"], s["accept_len"],
                                    s["lens"], s["table"], s["k_cache"], s["v_cache"],
                                    out=(s["path"], s["new_lens"]))
    return dict(path=path, lens=lens, k_cache=s["k_cache"], v_cache=s["v_cache"])


def _plain_commit(c, s):
    B, page = c["B"], c["page"]
    node = torch.zeros(B, dtype=torch.int64, device="cuda")
    path = [node]
    for j in range(c["depth"]):                        # one level of the tree after another
        hit = (s["parent"] == node[:, None]) & (s["token"] == s["accepted"][:, j:j + 1])
        node = hit.to(torch.int32).argmax(1)
        path.append(node)
    path = torch.stack(path, 1)
    j = torch.arange(c["depth"] + 1, device="cuda")
    live = j[None, :] <= s["accept_len"][:, None]
    lens = s["lens"].long()[:, None]
    # entries past the end of the path copy the root onto itself
    src = lens + torch.where(live, path, 0)
    dst = lens + torch.where(live, j[None, :], 0)
    src = (s["table"].gather(1, src // page).long() * page + src % page).flatten()
    dst = (s["table"].gather(1, dst // page).long() * page + dst % page).flatten()
    for cache in (s["k_cache"], s["v_cache"]):
        flat = cache.flatten(1, 2)
        flat[:, dst] = flat[:, src]
    s["path"].copy_(torch.where(live, path, -1))
    s["new_lens"].copy_(s["lens"] + 1 + s["accept_len"])
    return dict(path=s["path"], lens=s["new_lens"], k_cache=s["k_cache"], v_cache=s["v_cache"])


def _own_logprobs(c, s):
    got = s["handle"].logprobs(s["logits"], s["tokens"], path=s["path"], top=c["top"], T=c["T"],
                               out=s["out"])
    return dict(zip(("logprob", "entropy", "rank", "top_token", "top_logprob"), got))


def _plain_logprobs(c, s):
    B, V, top, T = c["B"], c["V"], c["top"], c["T"]
    live = (s["path"] >= 0) & (s["tokens"] >= 0)
    b = torch.arange(B, device="cuda")[:, None]
    x = s["logits"][b, s["path"].clamp(min=0).long()][:, :, :V].float() + 0.0
    token = s["tokens"].clamp(min=0).long()[:, :, None]
    # one whole number orders by value, then by the lower id
    bits = x.view(torch.int32)
    key = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long() * 2 ** 32
    key += 2 ** 32 - 1 - torch.arange(V, device="cuda")
    rank = (key > key.gather(2, token)).sum(2)
    ids = key.topk(top, dim=2)[1]
    x = (x - x.amax(2, keepdim=True)) / T
    e = x.exp()
    z = e.sum(2)
    log_z = z.log()
    entropy = log_z - (e * torch.where(e > 0, x, 0.0)).sum(2) / z
    got = (x.gather(2, token)[:, :, 0] - log_z, entropy, rank, ids,
           x.gather(2, ids) - log_z[:, :, None])
    for buf, y in zip(s["out"], got):
        keep = live if y.dim() == 2 else live[:, :, None]
        buf.copy_(torch.where(keep, y.to(buf.dtype), buf))
    return dict(zip(("logprob", "entropy", "rank", "top_token", "top_logprob"), s["out"]))


# -- what a pass cannot do without ---------------------------------------------------


def work(case):
    c = case
    B, n = c["B"], c["n"]
    if c["op"] == "plan":
        rows = sum(_counts(c))
        pages = sum(_up(x + k, c["page"]) - _up(x, c["page"]) for x, k in zip(_lens(c), _counts(c)))
        return dict(bytes=4 * rows + 12 * B * n + 24 * B + 16 * pages, flops=4 * B * n)
    if c["op"] == "write":
        rows, H, K, D = sum(_counts(c)), c["heads"], c["kv_heads"], c["dim"]
        each = 2 * (H + 2 * K) * D * _esz(c) + 12 + 4 * c["rot"]
        return dict(bytes=rows * each, flops=rows * (H + K) * D * 6)
    if c["op"] == "attention":
        H, K, D, counts = c["heads"], c["kv_heads"], c["dim"], _counts(c)
        entries = sum(x + k for x, k in zip(_lens(c), counts) if k)
        rows = sum(counts)
        if c["tree"]:
            seen = sum(k * (x + k) for x, k in zip(_lens(c), counts))
        else:
            seen = sum(k * x + k * (k + 1) // 2 for x, k in zip(_lens(c), counts))
        moved = entries * K * D * 2 * _esz(c) + rows * H * (2 * D * _esz(c) + 4)
        moved += sum(k * k for k in counts) if c["tree"] else 0
        return dict(bytes=moved, flops=4 * seen * H * D)
    if c["op"] == "commit":
        moved = sum(_accept(c)) * c["layers"] * c["kv_heads"] * c["dim"] * 2 * _esz(c)
        return dict(bytes=2 * moved + B * n * 8 + B * (8 * c["depth"] + 16), flops=B * n)
    rows = sum(x + 1 for x in _accept(c))
    return dict(bytes=rows * (c["V"] * _esz(c) + 20 + 8 * c["top"]), flops=rows * c["V"] * 4)


# -- the definitions in 64 bits --------------------------------------------------------


def exact(case, seed):
    c = case
    if c["op"] in ("plan", "commit"):
        return None                                    # whole numbers, and copies
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    s = globals()["_prepare_" + c["op"]](c, g)
    return globals()["_exact_" + c["op"]](c, s)


def _exact_write(c, s):
    D, r = c["dim"], c["rot"]
    half = r // 2
    first = torch.arange(half, device="cuda")
    first, second = (2 * first, 2 * first + 1) if c["pairs"] else (first, first + half)

    def turned(x, w):
        x = x.double()
        if w is not None:
            x = x / (x.square().sum(-1, keepdim=True) / D + 1e-6).sqrt() * w.double()
        if r:
            row = s["rotation"].double()[s["positions"].long()].unsqueeze(2)
            z = torch.complex(x[..., first], x[..., second]) * torch.complex(row[..., :half], row[..., half:])
            x = x.clone()
            x[..., first], x[..., second] = z.real, z.imag
        return x

    out, kc, vc = s["out"].double(), s["k_cache"].double(), s["v_cache"].double()
    live = s["slots"] >= 0
    out[live] = turned(s["q"], s["q_weight"])[live]
    at = s["slots"][live]
    kc.flatten(0, 1)[at] = turned(s["k"], s["k_weight"])[live]
    vc.flatten(0, 1)[at] = s["v"].double()[live]
    return dict(q=out, k_cache=kc, v_cache=vc)


def _exact_attention(c, s):
    B, n, H, K, D, page = c["B"], c["n"], c["heads"], c["kv_heads"], c["dim"], c["page"]
    out, lse = s["out"].double(), s["lse"].double()
    for b, (ctx, rows) in enumerate(zip(_lens(c), _counts(c))):
        if not rows:
            continue
        L = ctx + rows
        at = torch.arange(L, device="cuda")
        slot = s["table"][b].long()[at // page] * page + at % page
        k = s["k_cache"].flatten(0, 1)[slot].double()
        v = s["v_cache"].flatten(0, 1)[slot].double()
        seen = torch.ones((rows, L), dtype=torch.bool, device="cuda")
        if c["tree"]:
            seen[:, ctx:] = s["mask"][b, :rows, :rows] > 0
        else:
            seen[:, ctx:] = torch.ones((rows, rows), device="cuda").tril() > 0
        for h in range(H):
            x = s["q"][b, :rows, h].double() @ k[:, h * K // H].t() / math.sqrt(D)
            x = torch.where(seen, x, -math.inf)
            lse[b, :rows, h] = x.logsumexp(1)
            out[b, :rows, h] = x.softmax(1) @ v[:, h * K // H]
    return dict(out=out, lse=lse)


def _exact_logprobs(c, s):
    V, T = c["V"], c["T"]
    out = [x.double() for x in s["out"]]
    for b, rows in enumerate(x + 1 for x in _accept(c)):
        x = s["logits"][b, s["path"][b, :rows].long(), :V].double()
        best = x.sort(dim=1, descending=True, stable=True)[0][:, :c["top"]]
        log_z = (x / T).logsumexp(1, keepdim=True)
        logp = x / T - log_z
        out[0][b, :rows] = logp.gather(1, s["tokens"][b, :rows, None].long())[:, 0]
        out[1][b, :rows] = -(logp.exp() * logp).sum(1)
        out[4][b, :rows] = best / T - log_z
    return dict(logprob=out[0], entropy=out[1], rank=None, top_token=None, top_logprob=out[4])
