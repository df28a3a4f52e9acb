"""Pages whose keys and values come from different stores: strides of dimensions of one element
say nothing."""

import pytest
import torch

from test_gpu_packed import BF16, _cache, _i32, _normal, binding  # noqa: F401

pytestmark = pytest.mark.gpu


def _store(c, layers, pages, K, other):
    """Zeros [layers, pages, K, page_bytes] (None: without layers); `other`: with strides of
    their own for dimensions of one element, as a part of a larger store has them."""
    shape = ([] if layers is None else [layers]) + [pages, K, c.page_bytes]
    x = torch.zeros(shape, dtype=torch.uint8, device="cuda")
    strides = [7 * s if other and n == 1 else s for n, s in zip(shape, x.stride())]
    return x.as_strided(shape, strides)


@pytest.mark.parametrize("layers,pages,K", [(None, 1, 2), (None, 3, 1), (None, 1, 1), (1, 3, 2),
                                            (1, 1, 1), (2, 1, 2), (2, 3, 1)])
def test_one_layer_page_or_head_of_a_larger_store(binding, layers, pages, K):  # noqa: F811
    """append, read, attention and commit, against pages of the same store."""
    D, page, n, L = 64, 16, 5, layers or 1
    c = _cache(binding, 1, K, D, page, pages, BF16, L, width=pages)
    pools = [[_store(c, layers, pages, K, x) for x in two] for two in ((True, False), (False, False))]
    assert pools[0][0].stride() != pools[0][1].stride()
    k, v = (_normal((L, 1, n, K, D), BF16, s).cuda() for s in (1, 2))
    slots = (torch.arange(n, device="cuda") + 2)[None]
    table, lens = _i32([list(range(pages))]), _i32([n + 2])
    q = _normal((1, 1, K, D), BF16, 3).cuda()
    got = []
    for pool in pools:
        c.append(*((k, v) if layers else (k[0], v[0])), slots, *pool)
        one = [x[0] if layers else x for x in pool]
        out = [*c.read(slots, *pool), c.attention(q, *one, table, lens)]
        c.commit(_i32([[-1, 0, 1, 2, 3]]), _i32([[-1, 5, 6, 7, 8]]), _i32([[5, 6]]), _i32([2]), lens,
                 table, k, v, *(x if layers else x[None] for x in pool))
        got.append([*out, *pool])
    for x, y in zip(*got):
        assert torch.equal(x, y) and (x != 0).any()
    assert c.device_error() == 0
    c.close()


def test_strides_that_differ_are_refused(binding):  # noqa: F811
    """Of pages, of layers, with more than one of them; bytes that are not dense."""
    c = _cache(binding, 1, 2, 64, 16, 3, BF16, 2, width=3)
    dense = torch.zeros((2, 3, 2, c.page_bytes), dtype=torch.uint8, device="cuda")
    wide = torch.zeros((2, 3, 3, c.page_bytes), dtype=torch.uint8, device="cuda")[:, :, :2]
    tall = torch.zeros((2, 4, 2, c.page_bytes), dtype=torch.uint8, device="cuda")[:, :3]
    bytes2 = torch.zeros((2, 3, 2, 2 * c.page_bytes), dtype=torch.uint8, device="cuda")[..., ::2]
    heads = torch.zeros((2, 3, 4, c.page_bytes), dtype=torch.uint8, device="cuda")[:, :, ::2]
    slots = torch.zeros((1, 1), dtype=torch.int64, device="cuda")
    c.read(slots, dense, dense)
    c.read(slots, wide, wide)
    for pool in ((dense, wide), (wide, dense), (dense, tall), (tall, wide), (dense, bytes2),
                 (bytes2, bytes2), (heads, heads), (dense, heads)):
        with pytest.raises(binding.RheoError):
            c.read(slots, *pool)
    one = [dense[0], tall[0]]
    c.read(slots, *one)                                # (a layer's pages are alike in both)
    c.close()
