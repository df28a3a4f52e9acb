"""The 4-bit format in 64 bits, element by element.  Test infrastructure; CPU tensors."""


import torch

LEVELS = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
LOW = {torch.bfloat16: -125, torch.float16: -23}
HIGH = {torch.bfloat16: 125, torch.float16: 13}


def page_bytes(D, page):
    return page * -(-D // 32) * 17


def pack(x):
    """(codes [..., D'] int64, exponents [..., blocks] int64) of rows x [..., D] of a 16-bit
    type, D' = 32 blocks."""
    low, high, D = LOW[x.dtype], HIGH[x.dtype], x.shape[-1]
    nb = -(-D // 32)
    x = x.double()
    x = torch.cat([x, x.new_zeros(x.shape[:-1] + (32 * nb - D,))], -1).unflatten(-1, (nb, 32))
    finite = torch.isfinite(x)
    a = torch.where(finite, x.abs(), torch.zeros_like(x))
    m, e = torch.frexp(a.amax(-1))                     # m in [1/2, 1): the largest is 2 m 2^(e - 1)
    e = torch.where(2 * m < 1.75, e - 3, e - 2).clamp(low, high)
    e = torch.where(m == 0, torch.full_like(e, low), e)
    a = a / 2.0 ** e.double()[..., None]
    level = torch.tensor(LEVELS, dtype=torch.float64)
    far = (a[..., None] - level).abs()
    least = far.amin(-1, keepdim=True)
    # of two levels as near, the one of the even code
    near = (far == least)
    even = near & (torch.arange(8) % 2 == 0)
    code = torch.where(even.any(-1), even.to(torch.uint8).argmax(-1), near.to(torch.uint8).argmax(-1))
    code = torch.where(torch.isinf(x), torch.full_like(code, 7), code)
    code = code + 8 * (torch.signbit(x) & ~torch.isnan(x)).long()
    return code.flatten(-2), e.long()


def value(code, e, D):
    """What codes and exponents stand for, in 64 bits."""
    level = torch.tensor(LEVELS + [-x for x in LEVELS], dtype=torch.float64)
    x = level[code].unflatten(-1, (-1, 32)) * 2.0 ** e.double()[..., None]
    return x.flatten(-2)[..., :D]


def held(x):
    """Rows as 4 bits hold them, in 64 bits."""
    return value(*pack(x), x.shape[-1])


def store(pages, page, slots, x):
    """Rows x [rows, K, D] into slots of one layer's pages [pages, K, page bytes] uint8."""
    code, e = pack(x)
    nb = e.shape[-1]
    for i, s in enumerate(slots):
        if s < 0:
            continue
        p, at = s // page, s % page
        byte = (code[i, :, 0::2] + 16 * code[i, :, 1::2]).to(torch.uint8)
        pages[p, :, at * 16 * nb:(at + 1) * 16 * nb] = byte
        for b in range(nb):
            pages[p, :, page * 16 * nb + b * page + at] = (e[i, :, b] + 127).to(torch.uint8)


def load(pages, page, slots, D):
    """Entries [len(slots), K, D] of one layer's pages, in 64 bits."""
    nb = -(-D // 32)
    s = torch.as_tensor(slots, dtype=torch.int64)
    head = pages[s // page]
    at = (s % page)[:, None, None]
    byte = head.gather(2, (at * 16 * nb + torch.arange(16 * nb)).expand(-1, head.shape[1], -1)).long()
    e = head.gather(2, (page * 16 * nb + torch.arange(nb) * page + at).expand(-1, head.shape[1], -1))
    return value(torch.stack([byte % 16, byte // 16], -1).flatten(-2), e.long() - 127, D)


def seen(n, tail, length, window, sinks, mask=None, positions=None, count=None):
    """[n, length + tail'] bool: what each row of a sequence attends, tail' the tail's rows
    that are there; rows past count attend nothing."""
    count = n if count is None else count
    there = max(tail - (n - count), 0)
    s = torch.zeros((n, length + there), dtype=torch.bool)
    for i in range(count):
        at = length + tail - n + i
        if mask is not None:
            at = length if positions is None else max(int(positions[i]), length)
        for e in range(length + there):
            near = not window or e > at - window or e < sinks
            if mask is None:
                s[i, e] = e <= at and near
            elif e < length:
                s[i, e] = near
            else:
                s[i, e] = bool(mask[i, e - length])
    return s
