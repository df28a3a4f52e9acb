"""Pages that a window has left behind: they are not read, so that the table may hold anything in
their place and others may have them."""

import random

import pytest
import torch

import packed_oracle as ref
from test_gpu_packed import BF16, F16, Case, binding  # noqa: F401

pytestmark = pytest.mark.gpu


def _hidden(case, page):
    """The pages (b, place in the table) of which no row attends an entry: with a mask, no row
    at position lens."""
    found = []
    for b, length in enumerate(case.lens):
        if case.mask is not None:
            seen = ref.seen(1, 0, length, case.window, case.sinks, mask=torch.zeros((1, 0)))
        else:
            count = None if case.count is None else case.count[b]
            seen = ref.seen(case.n, case.tail, length, case.window, case.sinks, count=count)
        seen = seen[:, :length].any(0)
        found += [(b, p) for p in range(-(-length // page))
                  if not seen[p * page:(p + 1) * page].any()]
    return found


def _check(case, page, rng, most=None):
    """The same, bit for bit, with the hidden pages' bytes, then their numbers, replaced; and
    the plain form's."""
    out = case.check()
    hidden = _hidden(case, page)
    assert most is None or len(hidden) >= most
    for b, p in hidden:
        for pool in case.pool:                         # NaN, wherever it would count
            pool[case.table[b][p]] = 255
    assert torch.equal(case.check(), out)
    for b, p in hidden:
        case.table[b][p] = rng.choice([-1, case.c.pages, case.c.pages + 7, 1 << 30, -(1 << 31)])
    assert torch.equal(case.check(), out)              # (no error flag, either)
    case.c.close()


HIDDEN = [
    # dtype, lens, n, H, K, D, page, at least that many hidden pages, more
    # the window begins behind the pages' end, the first entries' tile holds the last page
    (BF16, [97], 4, 2, 1, 64, 16, 5, dict(tail=8, window=2, sinks=20)),
    (BF16, [17], 1, 4, 2, 64, 16, 1, dict(tail=5, window=2, sinks=4)),
    (F16, [146], 3, 4, 2, 128, 16, 8, dict(tail=0, window=1, sinks=20, tree=True)),
    (BF16, [127, 113], 1, 8, 1, 80, 16, 6, dict(tail=15, window=2, sinks=33)),
    # behind nearly all of the pages, with and without first entries
    (BF16, [1000], 1, 8, 2, 128, 16, 50, dict(window=100, sinks=4)),
    (F16, [1000, 333, 31], 1, 8, 2, 64, 32, 30, dict(window=65)),
    (BF16, [700, 20, 0], 3, 8, 2, 96, 16, 40, dict(window=17, sinks=1, tree=True)),
    (F16, [700], 20, 4, 2, 128, 16, 30, dict(window=33, sinks=3)),
    (BF16, [513, 90], 20, 8, 2, 64, 64, 5, dict(window=60, sinks=65, tree=True)),
    (BF16, [640, 100], 61, 8, 2, 128, 16, 30, dict(window=40, sinks=17, tree=True)),
    (F16, [640, 100], 61, 8, 2, 64, 32, 18, dict(window=7, tail=90)),
    (BF16, [800], 24, 4, 2, 256, 16, 35, dict(window=90, sinks=20)),
    (BF16, [900, 60], 150, 4, 1, 64, 16, 40, dict(window=50, sinks=5)),
    (F16, [900], 300, 2, 1, 128, 64, 7, dict(window=120, tail=0)),
    # rows among the pages' last entries, rows that are not there
    (BF16, [400], 9, 2, 2, 64, 16, 20, dict(window=20, tail=0, sinks=40)),
    (F16, [400, 300, 200], 9, 4, 2, 64, 16, 30, dict(window=20, count=[9, 0, 4])),
    (BF16, [400, 300, 200], 40, 4, 2, 64, 16, 30, dict(window=20, sinks=70, count=[40, 1, 0])),
]


@pytest.mark.parametrize("dtype,lens,n,H,K,D,page,most,more", HIDDEN)
def test_pages_left_behind_are_not_read(binding, dtype, lens, n, H, K, D, page, most, more):  # noqa: F811
    case = Case(binding, dtype, lens, n, H, K, D, page, seed=n + D, **more)
    _check(case, page, random.Random(n), most)


@pytest.mark.parametrize("seed", range(40))
def test_pages_left_behind_at_any_place(binding, seed):  # noqa: F811
    """Lengths, tails, windows and first entries around each other's borders."""
    rng = random.Random(seed)
    n, H, K = rng.choice([(1, 2, 1), (1, 8, 1), (3, 4, 2), (4, 4, 1), (20, 2, 1), (61, 4, 2)])
    page = rng.choice([16, 16, 32])
    case = Case(binding, rng.choice([BF16, F16]), [rng.randint(0, 200) for _ in range(3)], n, H, K, 64,
                page, tail=rng.choice([n, 0, n + rng.randint(0, 40)]),
                window=rng.choice([1, 2, rng.randint(1, 40)]), sinks=rng.choice([0, rng.randint(1, 60)]),
                tree=rng.random() < 0.4, seed=seed)
    _check(case, page, rng)
