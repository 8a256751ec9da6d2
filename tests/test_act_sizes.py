"""CPU tests: what the activation operators' size queries answer, and refuse."""
import ctypes

import pytest
import torch

import paper_2608_22322_amd as al
from paper_2608_22322_amd import activations as act


def test_code_bytes():
    assert act.code_bytes(3, 100, 64) == 3 * (128 + 2) and act.code_bytes(0, 100) == 0


@pytest.mark.parametrize("rows,cols,block", [(3, 100, 48), (-1, 100, 64), (3, -1, 64), (3, 1 << 31, 64)])
def test_sizes_of_no_code_are_refused(rows, cols, block):
    """The library answers -1 twice: no number of bytes."""
    with pytest.raises(ValueError):
        act.code_bytes(rows, cols, block)


def test_workspaces_of_other_types_are_refused():
    with pytest.raises(ValueError):
        act.norm_backward_workspace_bytes(act.RMS, 4, 100, dtype=torch.float16)


def test_size_queries_and_calls_agree_on_the_widest_row():
    """2^31 - 8193 columns: asked for as a size, then as (empty) work."""
    L, most = al.lib(), (1 << 31) - 8193
    assert L.al_act_code_bytes(1, most, 128) == (most + 127) // 128 * 128 and L.al_act_exp_bytes(1, most, 128) == (most + 127) // 128
    assert L.al_act_code_bytes(1, most + 1, 128) == -1 and L.al_act_exp_bytes(1, most + 1, 128) == -1
    n = ctypes.c_size_t(0)
    assert L.al_norm_backward_workspace_bytes(1, 1, 1, most, ctypes.byref(n)) == 0
    assert L.al_norm_backward_workspace_bytes(1, 1, 1, most + 1, ctypes.byref(n)) == 4
    assert L.al_act_quantize(1, None, most, 0, most, 64, None, None, None) == 0
    assert L.al_act_quantize(1, None, most, 0, most + 1, 64, None, None, None) == 4


def test_what_a_block_keeps():
    """Bytes between the passes of the MLP block, by hand: 2048 tokens at 2048 / 5632."""
    from types import SimpleNamespace

    from paper_2608_22322_amd.mlp import SwigluMLP

    net = object.__new__(SwigluMLP)
    net.hidden, net.ffn, net.tokens = 2048, 5632, 2048
    net.xhat, net.gate_code, net.up_code = (SimpleNamespace(nbytes=lambda c=c: act.code_bytes(2048, c, 64)) for c in (2048, 5632, 5632))
    assert net.saved_bytes() == 2048 * (2048 + 2 * 5632) * 65 // 64 + 4 * 2048
    assert net.bf16_bytes(recompute=True) == 2 * 2048 * (2048 + 2 * 5632) + 4 * 2048  # x, gate, up
    assert net.bf16_bytes() == 2 * 2048 * (2 * 2048 + 3 * 5632) + 4 * 2048  # and n, h
    assert 0.5 < net.saved_bytes() / net.bf16_bytes(recompute=True) < 0.51
