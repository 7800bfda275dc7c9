"""Cases of the 4-bit cache and of beam search run against the bounds-checking build of the library (-DKVS_DEBUG_BOUNDS): run as a
script by tests/test_gpu_pack4_bounds.py with KVS_LIBRARY pointing at it.  Every global offset that build checks must fall in
its buffer, and the pools lie between canaries (helpers.GuardedCache)."""
import sys

import test_gpu_beam as beam
import test_gpu_pack4 as pack
from paper_2410_18517_b200 import SharedKVCache
from paper_2410_18517_b200 import binding as kb


def main():
    for case in pack.STORE:
        pack.test_rows_bit_for_bit(*case, 0.5, 2.0)
    pack.test_rows_of_units_of_different_length()
    pack.test_rotary_append("bf16", 8, 2, 128, 2, 5, 40)
    pack.test_rotary_append("f32", 4, 4, 64, 3, 33, 64)
    for case in pack.ATTEND:
        pack.test_attention(*case)
    for dtype in ("bf16", "f32"):
        for ctas in (1, 3, 7):
            pack.test_attention_any_split(dtype, ctas)
        for n in (1, 17, 64):
            pack.test_rolled_back_rows_reach_nothing(dtype, n)
        pack.test_steps_shared_layers_and_host_buffers(dtype)
        pack.test_recorded_steps(dtype)
    for case in (("bf16", 8, 2, 128, 2, 300, 300), ("f32", 4, 2, 64, 2, 70, 33), ("bf16", 7, 1, 128, 1, 1000, 77)):
        pack.test_prompts(*case)
    ctx = SharedKVCache(1, 2, 2, 64, 300, 16, "bf16")
    for case in beam.SELECT:
        beam.test_select(ctx, *case)
    for dtype in ("bf16", "f32"):
        beam.test_select_ties(ctx, dtype, 5000)
        beam.test_select_sorted_logits(ctx, dtype, 70001)
        beam.test_select_masks_and_broken_rows(ctx, dtype, 9000)
        beam.test_select_strided_and_unaligned_rows(ctx, dtype)
    for parent, old, first in beam.REORDER:
        for fmt, dtype, D in (("plain", "bf16", 64), ("4bit", "bf16", 128), ("4bit", "f32", 64)):
            beam.test_reorder(parent, old, first, fmt, dtype, D)
    beam.test_reorder_many_sequences_and_long_rows()
    beam.test_reorder_slots_of_different_length()
    beam.test_reorder_then_steps()
    beam.test_beam_search_as_it_is_used("4bit", "bf16")
    print("ALL 4-BIT AND BEAM BOUNDS CASES PASSED", kb.LIB_PATH)
    return 0


if __name__ == "__main__":
    sys.exit(main())
