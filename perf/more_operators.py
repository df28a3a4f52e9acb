"""The operators of the 4-bit cache whose speed counts: cases, inputs, plain forms.

Where a server's contexts do not fit its memory in 16 bits, their entries are held in
4 (blocks of 32 elements with a power of two each): prompts and single tokens are
rounded into pages (append), a verified tree's accepted path in all layers (commit);
a step's rows attend to the pages and to the step's own keys and values, which are
still in 16 bits (attention), over all of the prefix or over a window and the first
entries; entries go back to 16 bits where a sequence moves on (read).  Each case is
one pass through one of them, after append and commit with what they stored read back.
``run`` computes it with elementary torch operations, or, where ``own`` is true, with
the calls of ``paper_2609_21827_amd.binding``.
"""

import math
import random

import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
# the exponents of a block's power of two that keep every value exact in the type
_LOW = {"bf16": -125, "f16": -23}
_HIGH = {"bf16": 125, "f16": 13}

# Heads: "heads" query heads share "kv_heads" key/value heads of "dim" elements.
_BASE = {
    "append": dict(op="append", B=1, n=1, page=64, kv_heads=8, dim=128, dtype="bf16",
                   ragged=False),
    "read": dict(op="read", B=1, n=500, page=64, kv_heads=8, dim=128, dtype="bf16", layers=1,
                 ragged=False),
    "commit": dict(op="commit", B=1, n=61, depth=7, page=64, layers=32, kv_heads=8, dim=128,
                   dtype="bf16", ctx=2000),
    "attention": dict(op="attention", B=1, n=61, page=64, heads=32, kv_heads=8, dim=128,
                      dtype="bf16", ctx=2000, window=0, sinks=0, tree=True, ragged=False),
}


def _case(op, **kw):
    c = dict(_BASE[op])
    c.update(kw)
    return c


def listed():
    return [
        # one token of one conversation, one layer: every step of plain decoding
        _case("append", name="append_b1_n1"),
        # a batch of prompts of all lengths, as many key heads as query heads
        _case("append", name="append_prompts", B=16, n=1999, page=16, kv_heads=40, dim=80,
              dtype="f16", ragged=True),
        # one conversation's layer, back in 16 bits
        _case("read", name="read_b1", n=517, dim=64, dtype="f16"),
        # long conversations, several layers at a time
        _case("read", name="read_b8_long", B=8, n=8190, layers=4, ragged=True),
        # the accepted path of one conversation, all layers
        _case("commit", name="commit4_b1"),
        # the same for the largest batch
        _case("commit", name="commit4_b128", B=128, n=81, depth=8, page=16, ctx=6000),
        # one token of one short conversation
        _case("attention", name="attn4_b1_n1", n=1, ctx=517, tree=False),
        # plain decoding of many long conversations, seven query heads to a key head
        _case("attention", name="attn4_b128_n1", B=128, n=1, page=16, heads=28, kv_heads=4,
              dtype="f16", ctx=8191, tree=False),
        # the headline serving batch: a tree of 60 drafted tokens each
        _case("attention", name="attn4_b64_tree", B=64, ctx=4096),
        # one tree over a very long context
        _case("attention", name="attn4_b1_long", ctx=131011),
        # trees in a windowed layer of a model: the last 1024 entries and the first four
        _case("attention", name="attn4_b32_window", B=32, heads=64, ctx=20000, window=1024,
              sinks=4, ragged=True),
        # a piece of a long prompt in a windowed layer, behind pieces that are packed already
        _case("attention", name="attn4_prompt_window", B=2, n=1500, ctx=6001, window=2048,
              sinks=16, tree=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


_HEADS = [(32, 8), (32, 8), (40, 40), (28, 4), (64, 8), (16, 16), (8, 1), (10, 2), (5, 5), (20, 4)]
_DIMS = [128, 128, 128, 64, 64, 80, 112, 160, 256]
_most = {}


def draw(rng):
    """A case of the same ranges.  No dearer than the largest listed one of its operator."""
    op = rng.choice(["append", "read", "commit", "attention", "attention", "attention"])
    c = _case(op)
    c["B"] = _log_int(rng, 1, 128)
    c["page"] = rng.choice([16, 32, 64, 64, 128, 256])
    heads, c["kv_heads"] = rng.choice(_HEADS)
    c["dim"] = rng.choice(_DIMS)
    c["dtype"] = rng.choice(["bf16", "bf16", "f16"])
    if op != "commit":
        c["ragged"] = rng.random() < 0.6
    if op == "append":
        c["n"] = rng.choice([1, _log_int(rng, 2, 100), _log_int(rng, 100, 8000)])
    elif op == "read":
        c["n"] = _log_int(rng, 1, 30000)
        c["layers"] = rng.choice([1, 1, 4, 16])
    elif op == "commit":
        c["n"] = rng.randint(17, 80)
        c["depth"] = rng.randint(1, 8)
        c["layers"] = rng.choice([1, 16, 32])
        c["ctx"] = _log_int(rng, 1, 6000)
    else:
        c["heads"] = heads
        c["n"] = rng.choice([1, rng.randint(2, 80), rng.randint(20, 80), rng.randint(20, 80)])
        c["ctx"] = _log_int(rng, 1, 131000)
        c["tree"] = c["n"] > 1 and rng.random() < 0.8
        if c["n"] > 1 and not c["tree"]:
            c["n"] = _log_int(rng, 2, 2000)
        if rng.random() < 0.5:
            c["window"] = _log_int(rng, 16, 8000)
            c["sinks"] = rng.choice([0, 1, 4, 128])
    if op not in _most:
        every = [work(x) for x in listed() if x["op"] == op]
        _most[op] = {k: max(w[k] for w in every) for k in ("bytes", "flops")}
    size = {"append": "n", "read": "n", "commit": "B", "attention": "ctx"}[op]
    # (the pages of a windowed layer's whole prefix are there, too)
    costs = [c, dict(c, window=0)] if op == "attention" else [c]
    for key in [size, "B", "n"]:
        while c[key] > 1 and any(work(dict(x, **{key: c[key]}))[k] > _most[op][k]
                                 for x in costs for k in _most[op]):
            c[key] = max(1, int(c[key] * 0.8))
        costs = [dict(x, **{key: c[key]}) for x in costs]
    if op == "attention" and c["n"] == 1:
        c["tree"] = False
    return c


# -- sizes that follow from a case alone ---------------------------------------


def _lens(c):
    """Entries in the pages of each sequence before the pass."""
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
    return [rng.randint(0, min(c["depth"], (c["n"] - 1) // 2)) for _ in range(c["B"])]


def _up(a, b):
    return -(-a // b)


def _blocks(c):
    return _up(c["dim"], 32)


def _page_bytes(c):
    """Bytes of one head's page: 16 and a scale for every block of 32 elements."""
    return c["page"] * _blocks(c) * 17


# -- inputs ---------------------------------------------------------------------


def _ints(rows, dtype=torch.int32):
    return torch.tensor(rows, dtype=dtype, device="cuda")


def _normal(g, shape, c):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(_TYPES[c["dtype"]])


def _keys(g, shape, c):
    """Keys as models have them: some channels are ten times as large as others."""
    wide = torch.rand((shape[-2], shape[-1]), generator=g, device="cuda") < 0.05
    x = torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)
    return x.mul_(torch.where(wide, 4.0, 0.4)).to(_TYPES[c["dtype"]])


def _table(g, needs, width):
    """A block table [B, width] over a pool in random order, and the pool's size."""
    total = sum(needs)
    order = torch.randperm(total, generator=g, device="cuda").to(torch.int32)
    first = torch.tensor([0] + needs, device="cuda").cumsum(0)
    place = first[:-1, None] + torch.arange(width, device="cuda")
    held = torch.arange(width, device="cuda") < _ints(needs)[:, None]
    return torch.where(held, order[place.clamp(max=total - 1)], 0).to(torch.int32), total


def _filled(g, c, layers, pages):
    """Pages [layers, pages, kv_heads, page bytes] of packed normal entries."""
    shape = (pages * c["page"], c["kv_heads"], c["dim"])
    out = []
    for make in (_keys, _normal):
        pool = torch.empty((layers, pages, c["kv_heads"], _page_bytes(c)), dtype=torch.uint8,
                           device="cuda")
        for layer in range(layers):
            for p in range(0, pages, 4096):
                some = min(4096, pages - p)
                x = make(g, (some * c["page"],) + shape[1:], c)
                _store(c, pool[layer, p:p + some], torch.arange(some * c["page"], device="cuda"),
                       *_packed(c, x))
        out.append(pool)
    return out


def _rows_of(g, c):
    """(slots [B, n], pages): where the rows of each sequence stand, -1 for those not there."""
    B, n, page = c["B"], c["n"], c["page"]
    pages = _up(B * n + 3, page) + 1
    place = torch.randperm(pages, generator=g, device="cuda")
    at = torch.arange(B * n, device="cuda") + 3        # rows begin inside a page
    slots = (place[at // page] * page + at % page).view(B, n)
    return torch.where(torch.arange(n, device="cuda") < _ints(_counts(c))[:, None], slots, -1), pages


def _outputs(c, shape):
    return tuple(torch.zeros(shape + (c["kv_heads"], c["dim"]), dtype=_TYPES[c["dtype"]],
                             device="cuda") for _ in range(2))


def _prepare_append(c, g):
    B, n, K, D = c["B"], c["n"], c["kv_heads"], c["dim"]
    slots, pages = _rows_of(g, c)
    kp, vp = (x[0] for x in _filled(g, c, 1, pages))
    return dict(k=_keys(g, (B, n, K, D), c), v=_normal(g, (B, n, K, D), c), slots=slots,
                pages=pages, width=1, k_pages=kp, v_pages=vp, out=_outputs(c, (B, n)))


def _prepare_read(c, g):
    B, n = c["B"], c["n"]
    slots, pages = _rows_of(g, c)
    kp, vp = _filled(g, c, c["layers"], pages)
    return dict(slots=slots, pages=pages, width=1, k_pages=kp, v_pages=vp,
                out=_outputs(c, (c["layers"], B, n)))


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


def _prepare_commit(c, g):
    B, n, page, K, D, depth = c["B"], c["n"], c["page"], c["kv_heads"], c["dim"], c["depth"]
    lens, took = _lens(c), _accept(c)
    # the pages that a path may reach; what lies before them is not touched, so all of
    # it stands on the pool's page 0
    first = [x // page for x in lens]
    last = [_up(x + depth + 1, page) for x in lens]
    width = max(last)
    new, pages = _table(g, [b - a for a, b in zip(first, last)],
                        max(b - a for a, b in zip(first, last)))
    place = torch.arange(width, device="cuda")[None, :] - _ints(first)[:, None]
    at = place.clamp(0, new.shape[1] - 1).long()
    table = torch.where(place >= 0, new.gather(1, at) + 1, 0).to(torch.int32)
    pages += 1
    # an accepted path: nodes in rising order, each a child of the one before
    parent, _ = _tree(g, B, n, depth)
    token = torch.stack([torch.randperm(50000, generator=g, device="cuda")[:n] for _ in range(B)])
    order = torch.rand((B, n), generator=g, device="cuda")
    order[:, 0] = 2.0
    chosen = order.argsort(1)[:, :max(1, max(took))]
    live = torch.arange(chosen.shape[1], device="cuda") < _ints(took)[:, None]
    chosen = torch.where(live, chosen, n).sort(1)[0]
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
    # the slots of the entries behind each prefix, as the plan of the step gave them
    e = _ints(lens).long()[:, None] + torch.arange(depth + 1, device="cuda")
    slots = table.gather(1, e // page).long() * page + e % page
    kp, vp = _filled(g, c, c["layers"], pages)
    shape = (c["layers"], B, n, K, D)
    return dict(parent=parent.to(torch.int32), token=token.to(torch.int32), accepted=accepted,
                accept_len=_ints(took), lens=_ints(lens), table=table, pages=pages, width=width,
                k_pages=kp, v_pages=vp, k=_keys(g, shape, c), v=_normal(g, shape, c), slots=slots,
                path=torch.zeros((B, depth + 1), dtype=torch.int32, device="cuda"),
                new_lens=torch.zeros(B, dtype=torch.int32, device="cuda"),
                out=_outputs(c, (c["layers"], B, depth + 1)))


def _prepare_attention(c, g):
    B, n, K, D = c["B"], c["n"], c["kv_heads"], c["dim"]
    lens, counts = _lens(c), _counts(c)
    needs = [_up(x, c["page"]) for x in lens]
    table, pages = _table(g, needs, max(needs))
    kp, vp = (x[0] for x in _filled(g, c, 1, pages))
    s = dict(q=_normal(g, (B, n, c["heads"], D), c) * 1.5, table=table, lens=_ints(lens),
             count=_ints(counts) if c["ragged"] else None, mask=None, positions=None, pages=pages,
             width=max(needs), k_pages=kp, v_pages=vp, k_tail=_keys(g, (B, n, K, D), c),
             v_tail=_normal(g, (B, n, K, D), c),
             out=torch.zeros((B, n, c["heads"], D), dtype=_TYPES[c["dtype"]], device="cuda"),
             lse=torch.zeros((B, n, c["heads"]), dtype=torch.float32, device="cuda"))
    if c["tree"]:
        parent, depth = _tree(g, B, n, 8)
        mask = torch.zeros((B, n, n), dtype=torch.uint8, device="cuda")
        b = torch.arange(B, device="cuda")
        for i in range(n):
            if i:
                mask[:, i] = mask[b, parent[:, i]]
            mask[:, i, i] = 1
        s["mask"] = mask
        s["positions"] = (s["lens"][:, None] + depth).to(torch.int32)
    return s


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    state = globals()["_prepare_" + case["op"]](case, g)
    state["case"] = case
    if own:                                            # the handle that a program keeps
        from paper_2609_21827_amd.binding import PackedCache
        c = case
        state["handle"] = PackedCache(
            batch=c["B"], heads=c.get("heads", c["kv_heads"]), kv_heads=c["kv_heads"],
            head_dim=c["dim"], page_size=c["page"], pages=state["pages"],
            table_width=state["width"], layers=c.get("layers", 1), dtype=_TYPES[c["dtype"]])
    return state


# -- the format -------------------------------------------------------------------


def _packed(c, x):
    """Codes [..., 16 blocks] and scales [..., blocks] of rows x [..., dim], as bytes."""
    D, nb = c["dim"], _blocks(c)
    x = x.float()
    if 32 * nb > D:
        x = torch.cat([x, x.new_zeros(x.shape[:-1] + (32 * nb - D,))], -1)
    x = x.unflatten(-1, (nb, 32))
    m, e = torch.frexp(x.abs().amax(-1))               # the largest: m 2^e, m in [1/2, 1)
    e = torch.where(m < 0.875, e - 3, e - 2).clamp(_LOW[c["dtype"]], _HIGH[c["dtype"]])
    e = torch.where(m == 0, _LOW[c["dtype"]], e)
    a = torch.ldexp(torch.ldexp(x.abs(), -(e // 2)[..., None]), -(e - e // 2)[..., None])
    # eight magnitudes; where two are as near, the even code
    code = (a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + \
        (a >= 3.5) + (a > 5.0)
    code = code + 8 * torch.signbit(x).to(torch.uint8)
    code = code.flatten(-2)
    return code[..., 0::2] + 16 * code[..., 1::2], (e + 127).to(torch.uint8)


def _parts(c, pool):
    """A pool's codes [..., pages, heads, page, bytes] and scales [..., blocks, page]."""
    n = c["page"] * 16 * _blocks(c)
    return (pool[..., :n].unflatten(-1, (c["page"], -1)),
            pool[..., n:].unflatten(-1, (_blocks(c), c["page"])))


def _store(c, pool, slots, codes, scales):
    """Rows' codes and scales [rows, ..., heads, bytes] into their slots of pages
    [..., pages, heads, page bytes]."""
    p, i = slots // c["page"], slots % c["page"]
    all_codes, all_scales = _parts(c, pool)
    all_codes[..., p, :, i, :] = codes
    all_scales[..., p, :, :, i] = scales


def _values(c, codes, scales):
    """What codes [..., bytes] and scales [..., blocks] stand for, in 32 bits."""
    code = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).long()
    size = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], device="cuda")
    x = torch.cat([size, -size])[code].unflatten(-1, (_blocks(c), 32))
    e = scales.int() - 127
    x = torch.ldexp(torch.ldexp(x, (e // 2)[..., None]), (e - e // 2)[..., None])
    return x.flatten(-2)[..., :c["dim"]]


def _load(c, pool, slots):
    """Entries [slots ..., (layers,) heads, dim] of pages [(layers,) pages, ...]."""
    p, i = slots // c["page"], slots % c["page"]
    codes, scales = _parts(c, pool)
    return _values(c, codes[..., p, :, i, :], scales[..., p, :, :, i])


# -- one pass ---------------------------------------------------------------------


def run(state):
    return globals()[("_own_" if own else "_plain_") + state["case"]["op"]](state["case"], state)


def _own_append(c, s):
    s["handle"].append(s["k"], s["v"], s["slots"], s["k_pages"], s["v_pages"])
    k, v = s["handle"].read(s["slots"], s["k_pages"], s["v_pages"], out=s["out"])
    return dict(k=k, v=v)


def _plain_append(c, s):
    live = s["slots"] >= 0
    at = s["slots"][live]
    for x, pool in ((s["k"], s["k_pages"]), (s["v"], s["v_pages"])):
        _store(c, pool, at, *_packed(c, x[live]))
    for out, pool in zip(s["out"], (s["k_pages"], s["v_pages"])):
        out[live] = _load(c, pool, at).to(out.dtype)
    return dict(k=s["out"][0], v=s["out"][1])


def _own_read(c, s):
    k, v = s["handle"].read(s["slots"], s["k_pages"], s["v_pages"], out=s["out"])
    return dict(k=k, v=v)


def _plain_read(c, s):
    live = s["slots"] >= 0
    at = s["slots"][live]
    for out, pool in zip(s["out"], (s["k_pages"], s["v_pages"])):
        out[:, live] = _load(c, pool, at).to(out.dtype).transpose(0, 1)
    return dict(k=s["out"][0], v=s["out"][1])


def _own_commit(c, s):
    path, lens = s["handle"].commit(s["parent"], s["token"], s["accepted"], s["accept_len"],
                                    s["lens"], s["table"], s["k"], s["v"], s["k_pages"],
                                    s["v_pages"], out=(s["path"], s["new_lens"]))
    k, v = s["handle"].read(s["slots"], s["k_pages"], s["v_pages"], out=s["out"])
    return dict(path=path, lens=lens, k=k, v=v)


def _plain_commit(c, s):
    B = c["B"]
    node = torch.zeros(B, dtype=torch.int64, device="cuda")
    path = [node]
    for j in range(c["depth"]):                        # one level of the tree after another
        hit = (s["parent"] == node[:, None]) & (s["token"] == s["accepted"][:, j:j + 1])
        node = hit.to(torch.int32).argmax(1)
        path.append(node)
    path = torch.stack(path, 1)
    live = torch.arange(c["depth"] + 1, device="cuda")[None, :] <= s["accept_len"][:, None]
    b, j = live.nonzero(as_tuple=True)
    at, rows = s["slots"][b, j], path[b, j]
    for x, pool, out in ((s["k"], s["k_pages"], s["out"][0]), (s["v"], s["v_pages"], s["out"][1])):
        _store(c, pool, at, *_packed(c, x[:, b, rows].transpose(0, 1)))
        out.copy_(_load(c, pool, s["slots"]).permute(2, 0, 1, 3, 4))
    s["path"].copy_(torch.where(live, path, -1))
    s["new_lens"].copy_(s["lens"] + 1 + s["accept_len"])
    return dict(path=s["path"], lens=s["new_lens"], k=s["out"][0], v=s["out"][1])


def _own_attention(c, s):
    out, lse = s["handle"].attention(
        s["q"], s["k_pages"], s["v_pages"], s["table"], s["lens"], s["k_tail"], s["v_tail"],
        mask=s["mask"], window=c["window"], sinks=c["sinks"], positions=s["positions"],
        count=s["count"], out=s["out"], lse=s["lse"])
    return dict(out=out, lse=lse)


def _plain_attention(c, s):
    B, n, H, K, D, page = c["B"], c["n"], c["heads"], c["kv_heads"], c["dim"], c["page"]
    w, sinks, lens = c["window"], c["sinks"], s["lens"][:, None]
    # the prefix's entries that come into question: all, or the first and the last ones
    e = torch.arange(s["width"] * page, device="cuda")[None, :].expand(B, -1)
    if w and sinks + w < e.shape[1]:
        e = e[:, :sinks + w]
        e = torch.where(e < sinks, e, e - sinks + (lens - w).clamp(min=sinks))
    L = e.shape[1]
    there = (e < lens)[:, None, :]
    slot = s["table"].gather(1, (e // page).clamp(max=s["width"] - 1)).long() * page + e % page

    def entries(pool, tail):                           # [B, K, L + n, D]
        return torch.cat([_load(c, pool, slot), tail.float()], 1).transpose(1, 2)

    k = entries(s["k_pages"], s["k_tail"]).transpose(2, 3).contiguous()
    q = s["q"].float().view(B, n, K, H // K, D).permute(0, 2, 1, 3, 4).reshape(B, K, -1, D)
    score = torch.matmul(q, k).mul_(D ** -0.5).view(B, K, n, H // K, L + n)
    del k
    count = s["count"] if s["count"] is not None else torch.full_like(s["lens"], n)
    i = torch.arange(n, device="cuda")
    at = s["positions"] if c["tree"] else lens + i
    if w:
        there = there & ((e[:, None, :] > at[:, :, None] - w) | (e[:, None, :] < sinks))
    if c["tree"]:
        tail = s["mask"] != 0
    else:
        tail = (i[None, :] <= i[:, None])[None]
        if w:
            tail = tail & ((i[None, :] > i[:, None] - w)[None] | (lens + i < sinks)[:, None, :])
    tail = tail & (i < count[:, None])[:, None, :]
    seen = torch.cat([there.expand(B, n, L), tail.expand(B, n, n)], 2)
    score.masked_fill_(~seen[:, None, :, None, :], -math.inf)
    top = score.amax(-1, keepdim=True)
    p = score.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p.view(B, K, -1, L + n), entries(s["v_pages"], s["v_tail"]).contiguous())
    out = out.view(B, K, n, H // K, D)
    out = torch.where(total > 0, out / total, 0.0).permute(0, 2, 1, 3, 4).reshape(B, n, H, D)
    lse = (top + total.log())[..., 0].permute(0, 2, 1, 3).reshape(B, n, H)
    live = (i < count[:, None])[:, :, None]
    s["out"].copy_(torch.where(live[..., None], out.to(s["out"].dtype), s["out"]))
    s["lse"].copy_(torch.where(live, lse, s["lse"]))
    return dict(out=s["out"], lse=s["lse"])


# -- what a pass cannot do without ---------------------------------------------------


def _reach(c, ctx, rows):
    """(prefix entries that some row attends, (row, entry) pairs) of one sequence.  A tree's
    rows count as all of them at the prefix's end, and as attending the whole tree."""
    w, sinks = c["window"], c["sinks"]
    if not rows:
        return 0, 0
    if not w:
        pairs = rows * (ctx + rows) if c["tree"] else rows * ctx + rows * (rows + 1) // 2
        return ctx, pairs
    seen = ctx - max(0, min(ctx, ctx - w + 1) - sinks) if ctx > sinks else ctx
    if c["tree"]:
        return seen, rows * (seen + rows)
    pairs = 0
    for i in range(rows):
        last = ctx + i
        far = max(0, last - w + 1)
        pairs += last + 1 - far + min(sinks, far)
    return seen, pairs


def work(case):
    c = case
    B, n, K, D, nb = c["B"], c["n"], c["kv_heads"], c["dim"], _blocks(c)
    wide, packed = 2 * K * D * 2, 2 * K * nb * 17      # bytes of an entry, keys and values
    if c["op"] == "append":
        rows = sum(_counts(c))
        return dict(bytes=rows * (wide + packed + 8 + packed + wide), flops=rows * 2 * K * D * 4)
    if c["op"] == "read":
        rows = sum(_counts(c))
        return dict(bytes=rows * (c["layers"] * (wide + packed) + 8),
                    flops=rows * c["layers"] * 2 * K * D)
    if c["op"] == "commit":
        rows = sum(x + 1 for x in _accept(c))
        back = B * (c["depth"] + 1)
        moved = (rows * (wide + packed) + back * (wide + packed)) * c["layers"]
        return dict(bytes=moved + B * n * 8 + B * (8 * c["depth"] + 16) + 8 * back,
                    flops=(rows * 4 + back) * c["layers"] * 2 * K * D)
    H, counts = c["heads"], _counts(c)
    reach = [_reach(c, x, k) for x, k in zip(_lens(c), counts)]
    moved = sum(x for x, _ in reach) * packed + sum(counts) * (wide + H * (2 * D * 2 + 4))
    moved += sum(k * k for k in counts) if c["tree"] else 0
    return dict(bytes=moved, flops=4 * sum(p for _, p in reach) * H * D)


# -- the definitions in 64 bits --------------------------------------------------------


def exact(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    s = globals()["_prepare_" + case["op"]](case, g)
    return globals()["_exact_" + case["op"]](case, s)


_LEVELS = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _held(c, x):
    """Rows x [..., dim] as 4 bits hold them: each block's power of two from its largest
    element, each element the nearest multiple."""
    x = x.double()
    y = torch.zeros_like(x)
    for d in range(0, c["dim"], 32):
        z = x[..., d:d + 32]
        top = z.abs().amax(-1, keepdim=True)
        power = torch.floor(torch.log2(torch.where(top > 0, top, 1.0)))
        power += (torch.exp2(power) > top).double() * -1 + (torch.exp2(power + 1) <= top)
        step = torch.where(top >= 1.75 * torch.exp2(power), power - 1, power - 2)
        unit = torch.exp2(step.clamp(_LOW[c["dtype"]], _HIGH[c["dtype"]]))
        a = z.abs() / unit
        near = torch.where(a < 2, (a * 2).round() / 2,                # (round: ties to even)
                           torch.where(a < 4, a.round(), (a / 2).round() * 2).clamp(max=6))
        y[..., d:d + 32] = torch.sign(z) * near * unit
    return y


def _meant(c, pool, slot):
    """Entries [slots, heads, dim] of pages, in 64 bits."""
    level = torch.tensor(_LEVELS + [-x for x in _LEVELS], dtype=torch.float64, device="cuda")
    page, nb = c["page"], _blocks(c)
    head = pool[slot // page]                          # [slots, heads, page bytes]
    at = (slot % page)[:, None, None]
    byte = (at * (16 * nb) + torch.arange(16 * nb, device="cuda")).expand(-1, head.shape[1], -1)
    codes = head.gather(2, byte).long()
    place = page * 16 * nb + torch.arange(nb, device="cuda") * page + at
    power = torch.exp2(head.gather(2, place.expand(-1, head.shape[1], -1)).double() - 127)
    x = level[torch.stack([codes % 16, codes // 16], 3).flatten(2)]
    return (x * power.repeat_interleave(32, 2))[..., :c["dim"]]


def _exact_append(c, s):
    live = (s["slots"] >= 0)[..., None, None]
    return dict(k=torch.where(live, _held(c, s["k"]), 0.0), v=torch.where(live, _held(c, s["v"]), 0.0))


def _exact_read(c, s):
    got = []
    for pool, out in zip((s["k_pages"], s["v_pages"]), s["out"]):
        x = out.double()
        for layer in range(c["layers"]):
            for b, rows in enumerate(_counts(c)):
                for i in range(0, rows, 4096):
                    at = s["slots"][b, i:min(rows, i + 4096)]
                    x[layer, b, i:i + len(at)] = _meant(c, pool[layer], at)
        got.append(x)
    return dict(k=got[0], v=got[1])


def _exact_commit(c, s):
    got = []
    lens, took = _lens(c), _accept(c)
    for pool, rows in ((s["k_pages"], s["k"]), (s["v_pages"], s["v"])):
        flat = s["slots"].flatten()
        x = torch.stack([_meant(c, pool[layer], flat) for layer in range(c["layers"])])
        x = x.unflatten(1, s["slots"].shape)
        for b, m in enumerate(took):
            parent, token = s["parent"][b].tolist(), s["token"][b].tolist()
            path = [0]
            for t in s["accepted"][b, :m].tolist():
                path.append([i for i in range(c["n"]) if parent[i] == path[-1] and token[i] == t][0])
            x[:, b, :m + 1] = _held(c, rows[:, b, path])
        got.append(x)
    return dict(path=None, lens=None, k=got[0], v=got[1])


def _exact_attention(c, s):
    H, K, D, page = c["heads"], c["kv_heads"], c["dim"], c["page"]
    out, lse = s["out"].double(), s["lse"].double()
    for b, (ctx, rows) in enumerate(zip(_lens(c), _counts(c))):
        if not rows:
            continue
        at = torch.arange(ctx, device="cuda")
        slot = s["table"][b].long()[at // page] * page + at % page
        k, v = (torch.cat([_meant(c, pool, slot), tail[b, :rows].double()])
                for pool, tail in ((s["k_pages"], s["k_tail"]), (s["v_pages"], s["v_tail"])))
        seen = torch.ones((rows, ctx + rows), dtype=torch.bool, device="cuda")
        entry = torch.arange(ctx + rows, device="cuda")[None, :]
        where = torch.arange(rows, device="cuda")[:, None] + ctx
        if c["tree"]:
            seen[:, ctx:] = s["mask"][b, :rows, :rows] > 0
            where = s["positions"][b, :rows, None]
        else:
            seen &= entry <= where
        if c["window"]:
            out_of = (where - entry >= c["window"]) & (entry >= c["sinks"])
            if c["tree"]:
                out_of &= entry < ctx
            seen &= ~out_of
        for h in range(H):
            x = s["q"][b, :rows, h].double() @ k[:, h * K // H].t() / math.sqrt(D)
            x = torch.where(seen, x, -math.inf)
            lse[b, :rows, h] = x.logsumexp(1)
            out[b, :rows, h] = x.softmax(1) @ v[:, h * K // H]
    return dict(out=out, lse=lse)
