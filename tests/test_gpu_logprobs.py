"""rheo_token_logprobs against a plain 64-bit form."""

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


def _check(binding, logits, V, path, tokens, top, T):
    """Runs and compares every entry; logits [B, n, stride] on the CPU."""
    B, n, stride = logits.shape
    m = tokens.shape[1]
    s = binding.Scorer(V, logits.dtype, stride)
    out = (torch.full((B, m), 7.0), torch.full((B, m), 7.0), torch.full((B, m), 7).int(),
           torch.full((B, m, top), 7).int(), torch.full((B, m, top), 7.0))
    out = tuple(t.cuda() for t in out)
    s.logprobs(logits.cuda(), tokens.int().cuda(), path=None if path is None else path.int().cuda(),
               top=top, T=T, out=out)
    logp, ent, rank, ids, lps = (t.cpu() for t in out)
    for b in range(B):
        for j in range(m):
            line = j if path is None else int(path[b, j])
            t = int(tokens[b, j])
            if not (0 <= line < n and 0 <= t < V):
                assert logp[b, j] == 7 and ent[b, j] == 7 and rank[b, j] == 7
                assert (ids[b, j] == 7).all() and (lps[b, j] == 7).all()
                continue
            w = ref.logprobs(logits[b, line, :V], t, top, T)
            assert int(rank[b, j]) == w[2], (b, j)
            assert ids[b, j].tolist() == w[3].tolist(), (b, j)
            for got, want, tol in ((logp[b, j], w[0], w[5]), (ent[b, j], w[1], w[6]),
                                   (lps[b, j], w[4], w[7])):
                got, want = got.double(), want.double()
                fine = torch.isfinite(want)
                assert torch.equal(got[~fine], want[~fine]), (b, j)
                assert ((got - want).abs()[fine] <= (tol * torch.ones_like(want))[fine]).all(), \
                    (b, j, float((got - want).abs()[fine].max()), tol)
    s.close()


def _rows(g, B, n, V, dtype, spread=3.0):
    stride = -(-V // 8) * 8
    x = torch.full((B, n, stride), 1e4)
    x[..., :V] = torch.randn((B, n, V), generator=g) * spread
    return x.to(dtype)


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("V", [2, 3, 31, 100, 1000, 8191, 8192, 8193, 32000, 50001])
@pytest.mark.parametrize("top", [0, 1, 20, 32])
def test_logprobs_match_the_plain_form(binding, dtype, V, top):
    g = torch.Generator().manual_seed(V + top)
    B, n, m = 2, 5, 4
    x = _rows(g, B, n, V, dtype)
    tokens = torch.randint(0, V, (B, m), generator=g)
    tokens[0, 0] = int(x[0, 1, :V].float().argmax())
    tokens[1, 1] = V - 1
    path = torch.tensor([[1, 4, 0, 1], [-1, 3, 2, 5]])
    _check(binding, x, V, path, tokens, min(top, V), 0.7)
    _check(binding, x, V, None, tokens, min(top, V), 1.0)


def test_logprobs_of_large_vocabularies(binding):
    for V, dtype, T in ((262143, BF16, 1.0), (151936, F32, 0.8), (1 << 20, F16, 2.0)):
        g = torch.Generator().manual_seed(V)
        x = _rows(g, 1, 2, V, dtype)
        _check(binding, x, V, None, torch.randint(0, V, (1, 2), generator=g), 20, T)


def test_logprobs_of_many_entries(binding):
    """More entries than rows are split for."""
    g = torch.Generator().manual_seed(1)
    x = _rows(g, 40, 3, 9000, BF16)
    path = torch.randint(-1, 3, (40, 60), generator=g)
    _check(binding, x, 9000, path, torch.randint(0, 9000, (40, 60), generator=g), 5, 1.0)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("V", [100, 20000])
def test_logprobs_of_ties_masks_and_orders(binding, dtype, V):
    """Equal logits, signed zeros, few values, rows that rise or fall, masked tokens (fewer
    left than alternatives; one; the given token among them)."""
    g = torch.Generator().manual_seed(V)
    rows = [torch.zeros(V), torch.where(torch.rand(V, generator=g) < 0.5, 0.0, -0.0),
            torch.randint(0, 3, (V,), generator=g).float(), torch.linspace(-5, 5, V),
            torch.linspace(5, -5, V), torch.randn(V, generator=g) * 40]
    for keep in (1, 7, V // 2):
        x = torch.full((V,), -math.inf)
        at = torch.randperm(V, generator=g)[:keep]
        x[at] = torch.randn(keep, generator=g)
        rows.append(x)
    peak = torch.full((V,), -30.0)
    peak[V // 3] = 20.0
    rows.append(peak)
    x = torch.stack(rows)[None].to(dtype)
    x = torch.nn.functional.pad(x, (0, -V % 8))
    n = x.shape[1]
    for tokens in (torch.randint(0, V, (1, n), generator=g), torch.zeros((1, n)).long(),
                   x[..., :V].float().argmax(2)):
        _check(binding, x, V, None, tokens, 32, 1.0)


def test_rows_without_a_finite_logit_are_nan(binding):
    x = torch.full((1, 2, 1000), -math.inf, dtype=BF16, device="cuda")
    s = binding.Scorer(1000, BF16)
    logp, ent, rank, ids, lps = s.logprobs(x, torch.tensor([[3, 900]], device="cuda").int(), top=4)
    assert logp.isnan().all() and ent.isnan().all() and lps.isnan().all()
    assert rank.tolist() == [[3, 900]] and ids.tolist() == [[[0, 1, 2, 3]] * 2]
    s.close()


def test_one_sure_token(binding):
    """All mass on one token: log probability and entropy 0, not a rounding below."""
    x = torch.full((1, 1, 5000), -math.inf, device="cuda")
    x[0, 0, 77] = 3.0
    s = binding.Scorer(5000, F32)
    logp, ent, rank, ids, lps = s.logprobs(x, torch.tensor([[77]], device="cuda").int(), top=2)
    assert logp.item() == 0 and ent.item() == 0 and rank.item() == 0
    assert ids.tolist() == [[[77, 0]]] and lps[0, 0].tolist() == [0.0, -math.inf]
    s.close()


def test_a_new_scorer_used_at_once_on_another_stream(binding):
    """Its workspace is filled behind work of the default stream, which the other stream
    does not wait for: creation has to."""
    g = torch.Generator().manual_seed(3)
    x = _rows(g, 1, 2, 50000, BF16).cuda()
    tokens = torch.tensor([[11, 49999]], dtype=torch.int32, device="cuda")
    old = binding.Scorer(50000, BF16)
    want = old.logprobs(x, tokens, top=20)
    big = torch.ones((4096, 4096), device="cuda")
    side = torch.cuda.Stream()
    out = tuple(torch.zeros_like(t) for t in want)
    torch.cuda.synchronize()
    for _ in range(10):
        big = big @ big * 2.0 ** -12
    s = binding.Scorer(50000, BF16)
    s.logprobs(x, tokens, top=20, out=out, stream=side)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, want))
    s.close()
    old.close()
