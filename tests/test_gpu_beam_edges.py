"""Beam selection and reordering at the ends of what the documentation allows."""
import math

import pytest
import torch

from paper_2410_18517_b200 import SharedKVCache
from paper_2410_18517_b200 import build as kbuild

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    kbuild.build()


DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_select_over_the_largest_vocabulary(dtype):
    """One row of 2^31 - 1 logits (the bound on n_beams * vocab): the last segment ends where 31 bits do."""
    cache = SharedKVCache(1, 1, 1, 64, 1, 1, "bf16")
    V = 2 ** 31 - 1
    x = torch.zeros(1, V, dtype=DT[dtype], device="cuda")
    best = {V - V % 2 ** 23: 6.0, V - 1: 5.0, V - 2: 4.0, 0: 3.0}
    for at, logit in best.items():
        x[0, at] = logit
    s, t, p = cache.beam_select(x, torch.zeros(1, device="cuda"), 1, 6)
    del x
    assert t[0].tolist() == list(best) + [1, 2] and p[0].tolist() == [0] * 6
    lse = math.log(V - 4 + sum(math.exp(v) for v in best.values()))
    want = torch.tensor([v - lse for v in best.values()] + [-lse] * 2, dtype=torch.float64)
    # sums of ones are exact up to 2^24; rescaled a few times per thread that holds one of the four: 2^-22 each, and the
    # score's own rounding (2^-24 of 21.5)
    assert float((s[0].cpu().double() - want).abs().max()) < 16 * 2.0 ** -22
    assert cache.device_status() == 0
