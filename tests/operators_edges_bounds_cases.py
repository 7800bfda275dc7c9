"""More cases of the serving operators against the bounds-checking build (-DKVS_DEBUG_BOUNDS): selection by one block and by
a cluster, totals in several passes, tree attention of every split, prompts without positions.  Run as a script by
tests/test_gpu_operators_bounds_more.py with KVS_LIBRARY pointing at that build.  A check that fails leaves
KVS_ERR_BOUNDS in the status word of the cache that made the call."""
import sys

import test_gpu_operators as t
import test_gpu_operators_edges as e
from helpers import GuardedCache
from paper_2410_18517_b200 import SharedKVCache
from paper_2410_18517_b200 import binding as kb

closed = []


def checked(cls):
    class Checked(cls):
        def close(self):
            if getattr(self, "ctx", None):
                closed.append(self.device_status())
            super().close()

    return Checked


def main():
    t.GuardedCache, t.SharedKVCache = checked(GuardedCache), checked(SharedKVCache)
    kinds = {"f": t.filled.__defaults__}
    t.filled.__defaults__ = tuple(t.GuardedCache if x is GuardedCache else x for x in kinds["f"])
    for n in (1, 33, 1025, 5000, 60000):
        t.test_select_rows(n)
    for shape in ((1, 8, 16400), (1, 2, 70000), (1, 1, 262144), (10, 14, 33000)):
        t.test_select_long_units(*shape)
    t.test_select_on_ragged_units()
    t.test_select_more_units_than_one_launch_takes()
    t.test_weights_of_ragged_units()
    t.test_weights_under_graph_replay()
    for dtype, kernel in (("bf16", 1), ("bf16", 2), ("f32", 1)):
        for ctas in (0, 3):
            t.test_decode_attention_weights_any_split_and_kernel(dtype, kernel, ctas)
    e.test_weights_of_caches_whose_scores_take_several_passes("bf16", 64, 8, 64, 5, 70001, (70001, 1, 64, 33333, 69999, 5, 40960))
    e.test_weights_of_caches_whose_scores_take_several_passes("bf16", 40, 20, 64, 3, 150000, None)
    for dtype in ("bf16", "f32"):
        for ctas in (1, 2, 7, 50):
            t.test_tree_attention_any_split(dtype, ctas)
        t.test_tree_on_ragged_units_and_smaller_batch(dtype)
    for case in t.TREE:
        t.test_tree_attention_random_trees(*case)
    e.test_append_rotary_without_positions("bf16", 32, 8, 128, 1, 900, True)
    e.test_append_rotary_without_positions("bf16", 4, 2, 64, 2, 1000, True)
    t.test_append_rotary_of_long_prompts_in_place_on_sharing_layers_and_ragged_slots()
    assert len(closed) > 50 and not any(closed), closed
    print("ALL FURTHER BOUNDS CASES PASSED", kb.LIB_PATH, len(closed))
    return 0


if __name__ == "__main__":
    sys.exit(main())
