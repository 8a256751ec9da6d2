"""CPU tests: what the activation operators' size queries answer, and refuse."""
import pytest
import torch

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
