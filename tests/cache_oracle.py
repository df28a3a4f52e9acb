"""Plain 64-bit forms of the cache and scoring operators, and bounds on what a correctly
rounding implementation may be off by.  Test infrastructure; CPU tensors throughout."""

import math

import torch

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
U32 = 2.0 ** -24
# half a step below the smallest normal number
TINY = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}


def plan(page, width, pages, lens, held, table, free, n, count=None, depth=None):
    """Python lists in, copies out: (slots, positions, status, held, table, free)."""
    B = len(lens)
    count = [n] * B if count is None else count
    held, table, free = list(held), [list(r) for r in table], list(free)
    need = [-(-(x + k) // page) for x, k in zip(lens, count)]
    fits = [k <= width for k in need]
    for b in reversed(range(B)):                       # returned pages, the last one first
        if fits[b]:
            for p in reversed(range(need[b], held[b])):
                free.append(table[b][p])
            held[b] = min(held[b], need[b])
    room, asked, status = len(free), 0, [0] * B
    for b in range(B):
        if not fits[b]:
            status[b] = 2
            continue
        lacks = max(0, need[b] - held[b])
        asked += lacks
        if lacks and asked > room:
            status[b] = 1
            continue
        for p in range(held[b], need[b]):
            table[b][p] = free.pop()
        held[b] = need[b]
    slots, positions = [], []
    for b in range(B):
        row, pos = [], []
        for i in range(n):
            if status[b] or i >= count[b]:
                row.append(-1), pos.append(-1)
                continue
            e = lens[b] + i
            row.append(table[b][e // page] * page + e % page)
            pos.append(lens[b] + (i if depth is None else depth[b][i]))
        slots.append(row), positions.append(pos)
    return slots, positions, status, held, table, free


def write_heads(x, weight, eps, rotation, positions, interleaved):
    """(values, bound scale) of heads x [N, heads, D] in 64 bits; the scale is what fp32
    roundings inside are relative to."""
    x = x.double()
    D = x.shape[-1]
    if weight is not None:
        x = x / (x.square().mean(-1, keepdim=True) + eps).sqrt() * weight.double()
    size = x.abs()
    if rotation is not None:
        r = rotation.shape[1]
        row = rotation.double()[positions][:, None, :]
        c, s = row[..., :r // 2], row[..., r // 2:]
        j = torch.arange(r // 2)
        a, b = (2 * j, 2 * j + 1) if interleaved else (j, j + r // 2)
        y, size = x.clone(), size.clone()
        y[..., a] = x[..., a] * c - x[..., b] * s
        y[..., b] = x[..., b] * c + x[..., a] * s
        both = (x[..., a] * c).abs() + (x[..., b] * s).abs()
        other = (x[..., b] * c).abs() + (x[..., a] * s).abs()
        size[..., a], size[..., b] = both, other
        x = y
    return x, size * (D + 16)


def attention(q, k, v, seen, scale, dtype):
    """One sequence: q [n, H, D], k and v [L, K, D], seen [n, L] bool.  Returns out, lse and
    their bounds.

    Off by: the output's rounding, u |o|; each probability's rounding to dtype, u of it
    (and half a smallest step, over a sum that is at least 1); scores in fp32 from exact
    products (D additions and the scaling), whose error is the exponent's; the
    exponential and its argument; sums of L terms in fp32.  Rescaling adds two roundings a
    tile of 32 entries."""
    n, H, D = q.shape
    L, K = k.shape[0], k.shape[1]
    out = torch.zeros((n, H, D), dtype=torch.float64)
    lse = torch.full((n, H), -math.inf, dtype=torch.float64)
    tol, tol_lse = torch.zeros_like(out), torch.zeros_like(lse)
    u = U[dtype]
    for h in range(H):
        kk, vv = k[:, h * K // H].double(), v[:, h * K // H].double()
        qq = q[:, h].double()
        for i in range(n):
            at = seen[i].nonzero()[:, 0]
            if not len(at):
                continue
            x = (kk[at] @ qq[i]) * scale
            big = float((kk[at].abs() @ qq[i].abs()).max()) * scale
            lse[i, h] = x.logsumexp(0)
            p = x.softmax(0)
            out[i, h] = p @ vv[at]
            size = p @ vv[at].abs()
            e32 = U32 * (2 * D * big + 4 * big + 16 + len(at) + L / 16)
            tol[i, h] = u * out[i, h].abs() * 1.01 + (u + 2 * e32) * size * 1.01 + 1e-30
            if dtype == torch.float16:
                tol[i, h] += TINY[dtype] * (vv[at].abs().sum(0) + 1)
            tol_lse[i, h] = 2 * e32 + 4 * U32 * abs(float(lse[i, h]))
    return out, lse, tol, tol_lse


def path_of(parent, token, accepted):
    """Pruned indices of the root and the accepted tokens; None if one is no child."""
    path = [0]
    for t in accepted:
        hit = [i for i in range(len(parent)) if parent[i] == path[-1] and token[i] == t]
        if not hit:
            return None
        path.append(hit[0])
    return path


def logprobs(row, token, top, T):
    """(logprob, entropy, rank, ids, logps, bounds of logprob, entropy, logps) of one row."""
    x = row.double()
    V = len(x)
    logp = x / T - (x / T).logsumexp(0)
    p = logp.exp()
    plogp = torch.where(p > 0, p * logp, torch.zeros_like(p))
    order = torch.sort(x, descending=True, stable=True)[1]
    rank = int((order == token).nonzero()[0, 0])
    ids = order[:top]
    # fp32: a thread of 256 adds at most V / 256 terms and 16, a block's and the
    # segments' results are joined in 16 more steps; an exponent is off by a few
    # roundings of itself, which weigh as much as the terms do
    adds = V // 256 + 32
    spread = float((p * torch.where(p > 0, (x - x.max()).abs() / T, torch.zeros_like(p))).sum())
    base = U32 * (adds + 8 * spread + 16)
    bound = lambda y: base + 8 * U32 * (y.abs() + float(-logp.max()))  # noqa: E731
    return (logp[token], -plogp.sum(), rank, ids, logp[ids], bound(logp[token]),
            base * (2 + spread) + 8 * U32 * float(-plogp.sum()), bound(logp[ids]))
