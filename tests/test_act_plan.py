"""CPU tests: how a weight gradient is cut, and that its workspace holds what the cut writes."""
import ctypes
import random

import pytest

import paper_2608_22322_amd as al
from tests.act_util import wgrad_plan


def _up(n, to):
    return -(-n // to) * to


def _bytes(dtype, tokens, out, cols):
    n = ctypes.c_size_t(0)
    assert al.lib().al_linear_wgrad_workspace_bytes(dtype, tokens, out, cols, ctypes.byref(n)) == 0
    return n.value


def _sizes():
    rng = random.Random(5)
    yield from [(0, 5, 7), (1, 1, 1), (100, 40, 0), (8192, 2048, 2048), (1, 128, 1 << 26), (277, 196, 4168), (20001, 1100, 700)]
    for _ in range(2000):
        yield tuple(int(2 ** rng.uniform(0, top)) for top in (16, 13, 13))


@pytest.mark.parametrize("dtype", [0, 1])
def test_workspaces_hold_the_plan(dtype):
    """Partial products in the plan's tiles and in 64-wide ones with the same splits (rows far apart), behind them dy's sums."""
    seen = set()
    for tokens, out, cols in _sizes():
        tile, splits, slabs, beside = wgrad_plan(dtype, tokens, out, cols)
        assert tile in (64, 128, 256) and splits >= 1 and slabs >= 1 and (tile == 64 or min(out, cols) >= tile)
        assert not beside or (splits > 1 and slabs % 8 == 0)  # a joining lane adds eight slabs at a time
        part = splits * _up(out, tile) * _up(cols, tile) * 4 if splits > 1 else 0
        edge = splits * _up(out, 64) * _up(cols, 64) * 4 if splits > 1 else 0
        assert edge <= part
        assert _bytes(dtype, tokens, out, cols) == _up(part, 256) + _up((slabs + 1) * out * 4, 256)
        seen.add((tile, splits > 1))
    assert len(seen) == 6


def test_refusals():
    plan, f = (ctypes.c_int32 * 4)(), al.lib().al_diag_wgrad_plan
    assert f(1, 64, 100, 100, None) == 1 and f(2, 64, 100, 100, plan) == 1 and f(1, -1, 100, 100, plan) == 1
    assert f(1, 64, 1 << 22, 100, plan) == 4 and f(1, 64, 100, 1 << 29, plan) == 4
