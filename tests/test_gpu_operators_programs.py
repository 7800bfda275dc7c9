"""Random programs of calls over one cache, queued without a wait (see operators_programs)."""
import random

import pytest
import torch

from operators_programs import Program
from paper_2410_18517_b200 import KVS_OPT_EARLY_START, KVS_OPT_FINISH_IN_KERNEL, KVS_OPT_KERNEL, KVS_OPT_MAX_CTAS
from paper_2410_18517_b200 import build as kbuild

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    kbuild.build()


def shape(seed, capacity):
    r = random.Random(seed)
    dtype = r.choice(("bf16", "bf16", "bf16", "f32"))
    G = r.choice((1, 2, 4, 8) if dtype == "f32" else range(1, 9))
    Hkv, D, B = r.choice((1, 2, 3, 4)), r.choice((64, 128)), r.choice((1, 2, 3, 5))
    share = [0]
    for l in range(1, r.choice((1, 2, 3))):
        share.append(r.choice((l, l, r.randrange(l))))
    options = [(KVS_OPT_MAX_CTAS, r.choice((0, 0, 0, 1, 3, 40)))]
    if seed % 5 == 3:
        options += [(KVS_OPT_EARLY_START, 0)]
    if seed % 5 == 4:
        options += [(KVS_OPT_FINISH_IN_KERNEL, 0)]
    if dtype == "bf16" and seed % 3 == 2:
        options += [(KVS_OPT_KERNEL, 2 if G in (3, 5, 6, 7) else r.choice((1, 2)))]
    return dtype, G * Hkv, Hkv, D, B, capacity, share, options


@pytest.mark.parametrize("seed", range(40))
def test_programs(seed):
    *args, options = shape(seed, (100, 300, 700, 2500)[seed % 4])
    Program(seed, *args, 30, options).run(torch.cuda.Stream() if seed % 2 else None)


@pytest.mark.parametrize("seed", range(100, 106))
def test_programs_over_long_caches(seed):
    """Kernels long enough that a call queued behind one really starts beside it."""
    *args, options = shape(seed, 12000)
    Program(seed, *args, 25, options, filled=9000 + 311 * (seed - 100)).run()


@pytest.mark.parametrize("seed", range(200, 216))
def test_recorded_programs(seed):
    *args, options = shape(seed, (100, 700, 2500)[seed % 3])
    Program(seed, *args, 30, options).run(graph=True)
