"""Outputs that a call makes itself, on a stream other than torch's current one: nothing that
the current stream has still to do lands in them, and nothing that it has still to read of
them is written over."""

import pytest
import torch

from test_gpu_cache import BF16, Setup, _i32, _tree_mask
from test_gpu_cache_use import Loop

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def binding():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2609_21827_amd import binding
    binding.load_library()
    return binding


def _busy():
    """Some 20 ms of work on the current stream."""
    x = torch.ones((4096, 4096), device="cuda")
    for _ in range(10):
        x = x @ x * 2.0 ** -12


def _calls(binding):
    """name -> (call taking stream=, seed) that returns tensors made by the call; and the
    handles."""
    s = Setup(binding, BF16, [300, 40], 20, 20, 8, 2, 64, 16)
    g = torch.Generator().manual_seed(5)
    kc, vc = s.pages_on_gpu()
    table, lens, mask = s.table.cuda(), _i32(s.lens), _tree_mask(s.g, 2, 20).cuda()
    qs = [torch.randn((2, 20, 8, 64), generator=g).to(BF16).cuda() for _ in range(2)]
    k = torch.randn((2, 20, 2, 64), generator=g).to(BF16).cuda()
    slots = torch.full((2, 20), -1, dtype=torch.int64, device="cuda")
    slots[0] = torch.arange(20)
    spare = [torch.zeros_like(kc), torch.zeros_like(vc)]
    par = _i32([[i - 1 for i in range(20)]] * 2)
    tok = _i32([[-1] + list(range(19))] * 2)
    acc, took = _i32([[0, 1, 2, -1]] * 2), [_i32([3, 1]), _i32([0, 2])]
    scorer = binding.Scorer(1000, BF16)
    logits = torch.randn((2, 4, 1000), generator=g).to(BF16).cuda()
    tokens = [torch.randint(0, 1000, (2, 4), generator=g).int().cuda() for _ in range(2)]
    free = _i32(list(range(s.pages)))

    def plan(seed, stream):
        # (two pages go back and some come: the state is each call's own, made beforehand)
        return s.cache.plan(*states.pop(), 20 - seed, stream=stream)

    states = [[_i32([30, 20]), _i32([2, 2]), table.clamp(min=0), free.clone(), _i32([5])]
              for _ in range(8)]
    calls = {
        "plan": plan,
        "write": lambda seed, stream: (s.cache.write(qs[seed], k, k, slots, *spare, stream=stream)[:1],),
        "attention": lambda seed, stream: s.cache.attention(qs[seed], kc, vc, table, lens, mask=mask,
                                                            lse=True, stream=stream),
        "commit": lambda seed, stream: s.cache.commit(par, tok, acc, took[seed], lens, table,
                                                      spare[0][None], spare[1][None], stream=stream),
        "logprobs": lambda seed, stream: scorer.logprobs(logits, tokens[seed], top=5, stream=stream),
    }
    return calls, (s.cache, scorer)


NAMES = ["plan", "write", "attention", "commit", "logprobs"]


@pytest.mark.parametrize("name", NAMES)
def test_pending_work_of_the_current_stream_does_not_land_in_them(binding, name):
    """Memory that the current stream has still to write, given back and handed out again, and
    fills that a call enqueues itself."""
    calls, handles = _calls(binding)
    want = [t.clone() for t in calls[name](0, None)]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    old = [torch.empty_like(t) for t in want for _ in range(40)]
    _busy()
    for t in old:
        t.fill_(1)
    del old, t
    got = calls[name](0, side)
    torch.cuda.synchronize()
    for x, y in zip(got, want):
        assert torch.equal(x, y)
    for h in handles:
        h.close()


@pytest.mark.parametrize("name", NAMES)
def test_they_are_not_handed_out_again_while_the_current_stream_reads_them(binding, name):
    calls, handles = _calls(binding)
    want = [t.clone() for t in calls[name](0, None)]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = calls[name](0, side)
    torch.cuda.current_stream().wait_stream(side)
    _busy()
    copies = [t.clone() for t in got]                  # behind the work
    del got
    again = [calls[name](1, side) for _ in range(3)]   # (their own inputs are long there)
    torch.cuda.synchronize()
    for x, y in zip(copies, want):
        assert torch.equal(x, y)
    assert len(again) == 3
    for h in handles:
        h.close()


def test_streams_of_other_libraries(binding):
    """A stream known by its address alone."""
    calls, handles = _calls(binding)
    side = torch.cuda.Stream()
    for name in NAMES:
        want = [t.clone() for t in calls[name](0, None)]
        torch.cuda.synchronize()
        got = calls[name](0, torch.cuda.ExternalStream(side.cuda_stream))
        torch.cuda.synchronize()
        for x, y in zip(got, want):
            assert torch.equal(x, y)
    for h in handles:
        h.close()


def _tree(binding, levels):
    tree = binding.Tree(batch=2, vocab=320, pool=4, leads=1, depth=3, support=64, dtype=BF16)
    g = torch.Generator().manual_seed(0)
    tree.begin_step()
    for level in range(levels):
        rows = tree.NE if level else 1
        tree.expand_level(torch.randn((2, rows, 320), generator=g).to(BF16).cuda(), 1.0, 5)
    return tree, torch.randn((2, 9, 320), generator=g).to(BF16).cuda()


@pytest.mark.parametrize("name", ["frontier", "read_nodes", "pruned_view", "tree_mask", "verify"])
def test_outputs_of_a_trees_calls(binding, name):
    """As the first test above, for the calls of the tree that make their outputs."""
    levels = 2 if name == "frontier" else 3            # (the last level has none behind it)
    (a, target), (b, _) = _tree(binding, levels), _tree(binding, levels)
    side = torch.cuda.Stream()

    def call(tree, stream):
        if name in ("pruned_view", "tree_mask", "verify"):
            tree.prune(8, stream=stream)
        got = tree.verify(target, 1.0, 5, stream=stream) if name == "verify" else \
            getattr(tree, name)(stream=stream)
        return list(got.values()) if isinstance(got, dict) else list(got)

    want = [t.clone() for t in call(a, None)]
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    old = [torch.empty_like(t) for t in want for _ in range(40)]
    _busy()
    for t in old:
        t.fill_(1)
    del old, t
    got = call(b, side)
    torch.cuda.synchronize()
    for x, y in zip(got, want):
        assert torch.equal(x, y)
    a.close(), b.close()


def test_a_step_captured_on_a_forked_stream_replays(binding):
    """The calls go to a stream that a capture forks to and joins again, with outputs of their
    own: replays, with eager steps of another loop between them, give what eager steps give."""
    a, b = Loop(binding), Loop(binding)
    side, capture = torch.cuda.Stream(), torch.cuda.Stream()
    a.feed(100), b.feed(100)
    want = a.step()
    side.wait_stream(torch.cuda.current_stream())
    got = b.step(stream=side)
    torch.cuda.synchronize()
    for x, y in zip(got, want):
        assert torch.equal(x, y)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=capture):
        side.wait_stream(capture)
        got = b.step(stream=side)
        capture.wait_stream(side)
    for seed in range(4):
        a.feed(seed), b.feed(seed)
        want = a.step()
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(got + b.state(), want + a.state()):
            assert torch.equal(x, y)
    assert a.cache.device_error() == 0 and b.cache.device_error() == 0
    a.close(), b.close()
