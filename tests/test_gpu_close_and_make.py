"""The memory of a cache that was closed while a graph was being recorded is there for the next cache."""
import threading

import pytest
import torch

import paper_2410_18517_b200 as pkg
from paper_2410_18517_b200 import SharedKVCache
from paper_2410_18517_b200 import build as kbuild

pytestmark = pytest.mark.gpu


def closed_during_a_recording(n):
    kbuild.build()
    caches = [SharedKVCache(1, 4, 2, 64, 1, 5000, "bf16") for _ in range(n)]
    x, g = torch.zeros(1, device="cuda"), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        x += 1
        for c in caches:
            c.close()
        assert len(pkg._unfinished) == n
        pkg._finish()                            # still recording: nothing is done
        assert len(pkg._unfinished) == n
    g.replay()
    torch.cuda.synchronize()
    assert float(x) == 1
    return caches                                # (whose end would end the others)


def test_a_new_cache_takes_the_memory_of_one_closed_during_a_recording():
    SharedKVCache(1, 4, 2, 64, 1, 20, "bf16").close()
    closed = closed_during_a_recording(1)
    before = torch.cuda.memory_allocated()
    new = SharedKVCache(1, 4, 2, 64, 1, 20, "bf16")
    assert not pkg._unfinished
    assert torch.cuda.memory_allocated() <= before - closed[0].pool_bytes + new.pool_bytes
    k = torch.ones(1, 5, 2, 64, dtype=torch.bfloat16, device="cuda")
    new.append(0, k, k)
    assert torch.equal(new.decode_attention(0, k[:, :1].expand(-1, 2, -1, -1).reshape(1, 4, 64).contiguous()), torch.ones(1, 4, 64, device="cuda"))


def test_threads_that_make_caches_at_once_end_each_closed_one_once():
    closed, failed = closed_during_a_recording(40), []

    def make():
        try:
            SharedKVCache(1, 4, 2, 64, 1, 20, "bf16").close()
        except Exception as e:              # noqa: BLE001
            failed.append(e)

    threads = [threading.Thread(target=make) for _ in range(8)]
    for t in threads:
        t.start()
    for t in threads:
        t.join(60)
    assert not failed and not pkg._unfinished and len(closed) == 40
