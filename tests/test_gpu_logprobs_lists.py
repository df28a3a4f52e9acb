"""rheo_token_logprobs on rows whose later chunks have more candidates than the list holds: whole
rows of many chunks a block, as batches have them."""

import math

import pytest
import torch

import cache_oracle as ref

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(scope="module")
def binding():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2609_21827_amd import binding
    binding.load_library()
    return binding


def _rows(g, V):
    """Rows whose chunks of 4096 overflow in every place: the first, a later one, the last,
    several; between chunks that do not."""
    chunk = 4096
    normal = torch.randn(V, generator=g)
    rows = [torch.zeros(V), torch.where(torch.rand(V, generator=g) < 0.5, 0.0, -0.0),
            torch.randint(0, 3, (V,), generator=g).float(), torch.linspace(-5, 5, V),
            torch.linspace(5, -5, V), normal]
    for places in ((1,), (2, 3), (0, 2), (1, 3), (V // chunk,), (0, 1, 2, 3, 4)):
        x = normal.clone()
        for i, p in enumerate(places):                 # a chunk of equal values above all before
            x[p * chunk:(p + 1) * chunk] = 10.0 + i
        rows.append(x)
        y = x.clone()                                  # of two values, shuffled
        for p in places:
            part = y[p * chunk:(p + 1) * chunk]
            part[torch.rand(len(part), generator=g) < 0.4] += 0.5
        rows.append(y)
    steps = torch.arange(V).div(chunk, rounding_mode="floor").float()
    rows += [steps, -steps, steps + 0.1 * normal]      # every chunk above, below the last
    for keep in (1, 7, V // 2):
        x = torch.full((V,), -math.inf)
        at = torch.randperm(V, generator=g)[:keep]
        x[at] = torch.randn(keep, generator=g)
        rows.append(x)
    late = torch.full((V,), -math.inf)                 # -inf, then a chunk of equals
    late[2 * chunk:3 * chunk] = 1.0
    rows.append(late)
    return rows


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("V", [20000, 20480, 8193])
@pytest.mark.parametrize("top", [1, 20, 32])
def test_lists_that_overflow_behind_the_first_chunk(binding, dtype, V, top):
    g = torch.Generator().manual_seed(V + top)
    x = torch.stack(_rows(g, V)).to(dtype)
    n = len(x)
    x = torch.nn.functional.pad(x, (0, -V % 8))
    # more entries than rows are split for: the rows again and again, other tokens each time
    m = n * (2500 // n + 1)
    path = torch.arange(m).remainder(n)
    tokens = torch.randint(0, V, (m,), generator=g)
    tokens[:n] = x[:, :V].float().argmax(1)
    tokens[n:2 * n], tokens[2 * n:3 * n] = 0, V - 1
    s = binding.Scorer(V, dtype, x.shape[1])
    got = s.logprobs(x[None].cuda(), tokens[None].int().cuda(), path=path[None].int().cuda(), top=top)
    logp, ent, rank, ids, lps = (t[0].cpu() for t in got)
    s.close()
    for line in range(n):
        row = x[line, :V].double()
        want = ref.logprobs(x[line, :V], int(tokens[line]), top, 1.0)
        at = path == line
        all_logp = row - row.logsumexp(0)
        order = torch.sort(row, descending=True, stable=True)[1]
        place = torch.empty_like(order)
        place[order] = torch.arange(V)
        t = tokens[at]
        assert torch.equal(rank[at].long(), place[t]), line
        assert (ids[at] == want[3].int()).all(), line
        for mine, exact, tol in ((logp[at], all_logp[t], None), (ent[at], want[1].expand(len(t)), want[6]),
                                 (lps[at], want[4].expand(len(t), top), want[7])):
            fine = torch.isfinite(exact)
            assert torch.equal(mine.double()[~fine], exact[~fine]), line
            if tol is None:                            # the oracle's bound, of each token's value
                tol = want[5] + 8 * ref.U32 * exact.abs()
            off = (mine.double() - exact).abs()
            assert (off[fine] <= (tol * torch.ones_like(exact))[fine]).all(), (line, float(off[fine].max()))


def test_lists_that_overflow_in_segments_of_several_chunks(binding):
    """Fewer entries, rows cut into parts of more than one chunk each."""
    V, top = 20 * 4096 + 77, 20
    g = torch.Generator().manual_seed(1)
    steps = torch.arange(V).div(4096, rounding_mode="floor").float()
    rows = torch.stack([steps, torch.zeros(V), torch.randn(V, generator=g) + steps, -steps])
    x = torch.nn.functional.pad(rows.to(BF16), (0, -V % 8))
    m = 300                                            # 2400 / 300: eight parts of three chunks
    path = torch.arange(m).remainder(4)
    tokens = torch.randint(0, V, (m,), generator=g)
    s = binding.Scorer(V, BF16, x.shape[1])
    got = s.logprobs(x[None].cuda(), tokens[None].int().cuda(), path=path[None].int().cuda(), top=top)
    s.close()
    rank, ids = got[2][0].cpu(), got[3][0].cpu()
    for line in range(4):
        order = torch.sort(x[line, :V].double(), descending=True, stable=True)[1]
        place = torch.empty_like(order)
        place[order] = torch.arange(V)
        at = path == line
        assert torch.equal(rank[at].long(), place[tokens[at]])
        assert (ids[at] == order[:top].int()).all()
