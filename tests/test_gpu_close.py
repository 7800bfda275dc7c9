"""A cache that is closed, or collected, while a graph is being recorded leaves the recording alone."""
import gc

import pytest
import torch

import paper_2410_18517_b200 as pkg
from paper_2410_18517_b200 import SharedKVCache
from paper_2410_18517_b200 import build as kbuild

pytestmark = pytest.mark.gpu


def test_caches_collected_during_a_recording():
    kbuild.build()
    cache = SharedKVCache(1, 4, 2, 64, 1, 20, "bf16")
    k = torch.ones(1, 5, 2, 64, dtype=torch.bfloat16, device="cuda")
    cache.append(0, k, k)
    q, out = k[:, :4, 0].contiguous(), torch.zeros(1, 4, 64, device="cuda")
    lost = [SharedKVCache(1, 4, 2, 64, 1, 20, "bf16"), SharedKVCache(1, 2, 2, 64, 1, 20, "f32")]
    lost.append(lost)                    # a cycle: only the collector ends these
    closed = SharedKVCache(1, 4, 2, 64, 1, 20, "bf16")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        del lost
        gc.collect()
        closed.close()
        cache.decode_attention(0, q, out)
    assert len(pkg._unfinished) >= 3
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, torch.ones_like(out)) and cache.device_status() == 0
    SharedKVCache(1, 4, 2, 64, 1, 20, "bf16").close()
    assert not pkg._unfinished
