"""Attention over 4-bit pages where windows and positions are as large as their type holds."""

import pytest
import torch

from test_gpu_packed import BF16, F16, Case, binding  # noqa: F401

pytestmark = pytest.mark.gpu

LARGEST = 2 ** 31 - 1


# rows of a key head: 5 (registers), 20 to 250 (LDS), more than one block
@pytest.mark.parametrize("n,H", [(5, 1), (20, 2), (50, 2), (61, 4), (300, 1)])
@pytest.mark.parametrize("tail", [0, 3])
@pytest.mark.parametrize("window", [LARGEST, LARGEST - 1, 2 ** 30 + 7])
def test_a_window_longer_than_any_sequence(binding, n, H, tail, window):  # noqa: F811
    """Hides nothing, also where rows stand before the first entry."""
    case = Case(binding, BF16, [n // 3, 0, n + 70, 4], n, H, 1, 64, 16, tail=tail, window=window)
    out = case.check()
    case.window = 0
    assert torch.equal(out, case.check())
    case.c.close()


@pytest.mark.parametrize("n,H", [(5, 1), (20, 2), (61, 4)])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 3), (40, 0), (LARGEST - 1, 0), (LARGEST, 1)])
def test_positions_far_beyond_the_entries(binding, n, H, window, sinks):  # noqa: F811
    case = Case(binding, F16, [300, 64, 0], n, H, 1, 64, 16, window=window, sinks=sinks, tree=True)
    # (rows of one sequence that are near, far, and as far as a position can be)
    case.positions[0, 1:] = LARGEST
    case.positions[1, 2:] = 2 ** 30
    case.positions[1, -1] = LARGEST - 5
    case.check()
    case.c.close()


def test_windows_that_32_bits_do_not_hold_are_refused(binding):  # noqa: F811
    case = Case(binding, BF16, [20], 2, 2, 1, 64, 16)
    for more in (dict(window=2 ** 31), dict(window=2 ** 32 + 5), dict(window=-1), dict(sinks=-1),
                 dict(window=4, sinks=2 ** 32 + 1)):
        with pytest.raises(binding.RheoError):
            case.call(**more)
    case.c.close()


def test_calls_without_rows(binding):  # noqa: F811
    """Nothing is read or written, whatever the addresses."""
    case = Case(binding, BF16, [20, 5], 2, 2, 1, 64, 16)
    c, (kp, vp) = case.c, case.pool
    was = kp.clone(), vp.clone()
    none = torch.empty((2, 0, 1, 64), dtype=BF16, device="cuda")
    slots = torch.empty((2, 0), dtype=torch.int64, device="cuda")
    c.append(none, none, slots, kp, vp)
    assert [x.shape for x in c.read(slots, kp, vp)] == [none.shape] * 2
    assert torch.equal(kp, was[0]) and torch.equal(vp, was[1])
    case.q = torch.empty((2, 0, 2, 64), dtype=BF16)
    out, lse = case.call(lse=True)
    assert out.shape == (2, 0, 2, 64) and lse.shape == (2, 0, 2)
    assert c.device_error() == 0
    c.close()


@pytest.mark.parametrize("n,H", [(1, 4), (61, 4)])
def test_two_caches_at_once_on_two_streams(binding, n, H):  # noqa: F811
    """Each handle has partial results of its own."""
    cases = [Case(binding, BF16, [900 + 50 * s, 1300], n, H, 1, 128, 16, seed=s) for s in (1, 2)]
    alone = [case.call() for case in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    args = []
    for case in cases:
        args.append(dict(k_tail=case.k_tail.cuda(), v_tail=case.v_tail.cuda()))
    q = [case.q.cuda() for case in cases]
    table = [torch.tensor(case.table, dtype=torch.int32, device="cuda") for case in cases]
    lens = [torch.tensor(case.lens, dtype=torch.int32, device="cuda") for case in cases]
    torch.cuda.synchronize()
    outs = [[], []]
    for _ in range(20):
        for i, case in enumerate(cases):
            outs[i].append(case.c.attention(q[i], *case.pool, table[i], lens[i], stream=streams[i],
                                            **args[i]))
    torch.cuda.synchronize()
    for want, got in zip(alone, outs):
        assert all(torch.equal(want, x) for x in got)
    for case in cases:
        case.c.close()
