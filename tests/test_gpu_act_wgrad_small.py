"""The weight gradient of the smallest dy: exact down to bits of 2^-133 (bf16's smallest number), which is below the normal numbers."""
import numpy as np
import pytest
import torch

from tests.act_util import DT, to_code, wgrad_plan
from tests.test_gpu_act_wgrad import _run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,low", [("bf16", -133), ("bf16", -120), ("f32", -149), ("f32", -140), ("f32", -133), ("f32", -120)])
@pytest.mark.parametrize("tokens,out,cols,tile", [(40, 100, 128, 64), (33, 2731, 4200, 128)])
def test_smallest_numbers(tokens, out, cols, tile, dtype, low):
    assert wgrad_plan(0 if dtype == "f32" else 1, tokens, out, cols)[0] == tile
    rng = np.random.default_rng(3)
    v = np.ldexp((rng.integers(1 << 23, 1 << 24, out) if dtype == "f32" else rng.integers(1, 256, out)).astype(np.float64), low)
    dy = np.zeros((tokens, out), np.float32)
    dy[7] = v
    nb = -(-cols // 64)
    codes = np.zeros((tokens, nb * 64), np.int8)
    codes[:, :cols] = 1
    dw, _ = _run(torch.from_numpy(dy).cuda().to(DT[dtype]), to_code(codes, np.full((tokens, nb), 227, np.uint8), cols, 64), "f32")
    want = torch.from_numpy(np.ldexp(v, 100)).cuda()[:, None]
    off = (dw.double() - want).abs()
    assert bool((off < 2.0**-33).all()) if low < -133 else not bool(off.any())  # what is dropped: bits below 2^-133, times 2^100
