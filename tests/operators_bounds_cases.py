"""Cases of the serving operators run against the bounds-checking build of the library (-DKVS_DEBUG_BOUNDS): run as a
script by tests/test_gpu_operators_bounds.py with KVS_LIBRARY pointing at it.  Every global offset that build checks
must fall in its buffer, and the pool lies between canaries (helpers.GuardedCache)."""
import sys

import numpy as np
import torch

import operators_reference as ref
import test_gpu_operators as t
from paper_2410_18517_b200 import KVS_OPT_MAX_CTAS, Rotary
from paper_2410_18517_b200 import binding as kb


def step(dtype, Hq, Hkv, D, B, n, n_t, ctas):
    cache, _, _ = t.filled(Hq, Hkv, D, B, n, dtype, extra=n_t + 3, max_batch=B + 1)
    cache.set_option(KVS_OPT_MAX_CTAS, ctas)
    x = t.normal(5, dtype, B, n_t, Hq + 2 * Hkv, D)
    pos = torch.arange(n, n + n_t).int().expand(B, n_t).contiguous().cuda()
    w = t.normal(6, dtype, D)
    q = cache.append_rotary(0, x[:, :, :Hq], x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:], pos, Rotary.from_theta(D), w, w)
    rng = np.random.default_rng(n)
    words = [ref.random_tree(rng, n_t) for _ in range(B)]
    out = cache.tree_attention(0, q, torch.tensor([ref.to_int64(r) for r in words]).cuda())
    t.check_tree(cache, 0, q, words, out)
    counts = [1 + (b * 3 + n) % n_t for b in range(B)]
    path = torch.arange(n_t).int().expand(B, n_t).contiguous().cuda()
    cache.accept_draft(path, counts, n_t)
    total = torch.zeros(B, Hkv, n + n_t + 3, device="cuda")
    q1 = q[:, 0].contiguous()
    out = cache.decode_attention_weights(0, q1, None, total)
    t.check_weights(cache, 0, q1, None, total, out, total.shape[2])
    keep = [[max(1, (n + c) // 2)] * Hkv for c in counts]
    kept = cache.evict_by_weight(0, total, keep, min(2, min(r[0] for r in keep)))
    after = torch.zeros_like(kept)
    t.check_weights(cache, 0, q1, kept, after, cache.decode_attention_weights(0, q1, kept, after), kept.shape[2])
    assert cache.device_status() == 0, cache.device_status()
    cache.check_canaries()


def main():
    for shape in (("bf16", 8, 2, 128, 2), ("bf16", 3, 3, 64, 3), ("bf16", 7, 1, 128, 1), ("bf16", 16, 2, 64, 2), ("f32", 8, 2, 64, 2), ("f32", 4, 4, 128, 1)):
        for n, n_t in ((1, 1), (63, 2), (64, 64), (125, 17), (700, 33)):
            for ctas in (0, 3):
                step(*shape, n, n_t, ctas)
    t.test_append_rotary_of_long_prompts(*t.ROT_LONG[0])
    t.test_append_rotary_of_long_prompts(*t.ROT_LONG[3])
    print("ALL OPERATOR BOUNDS CASES PASSED", kb.LIB_PATH)
    return 0


if __name__ == "__main__":
    sys.exit(main())
