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
