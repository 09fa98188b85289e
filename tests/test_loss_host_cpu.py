"""Host side of the output layer's losses beside test_loss_cpu.py: hooks, sizes of the largest calls, refusals (no GPU needed)."""
import ctypes as C

import pytest

import paper_2505_13765_b200 as pkg
from paper_2505_13765_b200 import binding as bd
from test_loss_cpu import layer, lib, size  # noqa: F401


def test_stall_hook_round_trip(lib):  # noqa: F811
    assert pkg.wind_debug_stall_loss(9) == 0 and pkg.wind_debug_stall_loss(10) == 9 and pkg.wind_debug_stall_loss(0) == 0
