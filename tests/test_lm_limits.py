"""CPU tests: the largest sizes that the head's loss accepts are launched whole."""
import ctypes

import pytest

import paper_2608_22322_amd as al


def _bytes(tokens, hidden, vocab):
    n = ctypes.c_size_t(0)
    assert al.lib().al_linear_xent_workspace_bytes(tokens, hidden, vocab, hidden, 0, 0, 0, 0, ctypes.byref(n)) == 0
    return n.value


@pytest.mark.parametrize("tokens,hidden,vocab", [(16384, 64, 1 << 24), (16257, 64, (1 << 24) - 127), (16384, 8, 1 << 24), (16320, 8, 16777152), (16384, 128, 1 << 24),
                                                 (16384, 1024, 1 << 24), (16256, 64, 1 << 24), (8192, 8, 1 << 24)])
def test_the_statistics_grid_stays_below_32_bits(tokens, hidden, vocab):
    """A pass of the statistics takes block tokens by the vocabulary, in tiles of 128 x 128 by 256 threads or 256 x 256 by 512, and leaves 8 bytes for every 64 columns of a token
    and 4 for its target's logit behind a padded copy of h: what the workspace holds says how many tokens a pass takes."""
    tp, dp = -(-tokens // 64) * 64, -(-hidden // 64) * 64
    a_token = -(-vocab // 64) * 8 + 4
    block = (_bytes(tokens, hidden, vocab) - 2 * tp * dp) // a_token
    assert 64 <= block <= 16384
    blocks = {b: -(-block // b) * -(-vocab // b) for b in (128, 256)}
    # (wider tiles are half the threads: what the narrower of them would take bounds both, and 256-wide ones are taken from 65 features on)
    assert (blocks[128] * 256 if dp == 64 else blocks[256] * 512) < 1 << 32
