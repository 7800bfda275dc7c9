"""The serving operators' checks and tables that need no device: refusals before memory is bound, the Rotary table, and
the reference the GPU tests use against independent restatements."""
import ctypes
import math

import numpy as np
import pytest
import torch

import operators_reference as ref
from paper_2410_18517_b200 import Rotary
from paper_2410_18517_b200 import binding as kb
from paper_2410_18517_b200 import build as kbuild


@pytest.fixture(scope="module", autouse=True)
def _built():
    kbuild.build()


def refused(status, fn, *args):
    with pytest.raises(kb.KvsError) as e:
        fn(*args)
    assert e.value.status == status


def test_state_and_null_refusals():
    c = kb.kvs_create(2, 8, 2, 64, 2, 100, kb.KVS_BF16, 0.0, 0)
    rot = kb.kvs_rotary(0, 0, 1e-6, None)
    p = 1 << 20                                  # never read: the context has no memory
    refused(kb.KVS_ERR_STATE, kb.kvs_append_rotary, c, 0, rot, p, 512, p, 128, p, 128, None, None, None, p, 1, 1)
    refused(kb.KVS_ERR_STATE, kb.kvs_tree_attention, c, 0, p, p, None, 1, 1)
    refused(kb.KVS_ERR_STATE, kb.kvs_accept_draft, c, p, 1, [1], 1, 1)
    refused(kb.KVS_ERR_STATE, kb.kvs_decode_attention_weights, c, 0, p, p, None, p, 100, 1)
    refused(kb.KVS_ERR_STATE, kb.kvs_select_rows, c, 0, p, 100, [1, 1], 0, p, None, 1, 1)
    kb.kvs_destroy(c)
    for fn, args in ((kb.kvs_append_rotary, (0, rot, p, 512, p, 128, p, 128, None, None, None, p, 1, 1)), (kb.kvs_tree_attention, (0, p, p, None, 1, 1)),
                     (kb.kvs_accept_draft, (p, 1, [1], 1, 1)), (kb.kvs_decode_attention_weights, (0, p, p, None, p, 100, 1)),
                     (kb.kvs_select_rows, (0, p, 100, [1], 0, p, None, 1, 1))):
        refused(kb.KVS_ERR_INVALID_ARG, fn, None, *args)


def test_rotary_table():
    r = Rotary.from_theta(64, 500000.0, interleaved=True)
    s = r._struct(1e-5)
    assert s.rotary_dim == 64 and s.interleaved == 1 and abs(s.eps - 1e-5) < 1e-11
    assert [s.inv_freq[i] for i in range(32)] == [500000.0 ** (-2.0 * i / 64) for i in range(32)]
    assert r._struct(1e-5) is s and r._struct(1e-6) is not s
    assert ctypes.sizeof(kb.kvs_rotary) == 24


def test_workspace_serves_every_call():
    """The scratch of the calls that share the search reductions' bytes fits the workspace of small and of wide shapes."""
    for Hq, Hkv, D, B, n, dt in ((1, 1, 64, 1, 1, kb.KVS_F32), (64, 8, 128, 4, 300, kb.KVS_BF16), (8, 8, 64, 200, 9000, kb.KVS_BF16)):
        c = kb.kvs_create(1, Hq, Hkv, D, B, n, dt, 0.0, 0)
        _, ws = kb.kvs_required_bytes(c)
        rows = min(128, Hq // Hkv * 64)
        assert ws >= B * Hq * kb.kvs_row_stride(c) * 4 and ws >= 2 * 320 * rows * (D + 2) * 4
        kb.kvs_destroy(c)


def test_reference_attention_against_torch():
    g = torch.Generator().manual_seed(0)
    q, K, V = (torch.randn(*s, generator=g, dtype=torch.float64) for s in ((5, 2, 16), (9, 16), (9, 16)))
    sees = torch.rand(5, 9, generator=g) < 0.6
    sees[:, 0] = True
    out, p, _, _ = ref.attend(q, K, V, sees)
    want = torch.nn.functional.scaled_dot_product_attention(q.transpose(0, 1), K.expand(2, 9, 16), V.expand(2, 9, 16), attn_mask=sees)
    assert (out - want.transpose(0, 1)).abs().max() < 1e-12 and (p.sum(-1) - 1).abs().max() < 1e-12
    out, _, _, _ = ref.attend(q, K, V, torch.zeros(5, 9, dtype=torch.bool))
    assert not out.any()


def test_reference_rotation_is_relative():
    """Dot products of rotated vectors depend on the distance alone; norms do not change."""
    g = torch.Generator().manual_seed(1)
    x = torch.randn(1, 2, 1, 32, generator=g, dtype=torch.float64)
    freq = [100.0 ** (-i / 16) for i in range(16)]
    for inter in (False, True):
        dots = []
        for base in (0, 1000003):
            y, _ = ref.norm_rope(x, None, torch.tensor([[base, base + 7]]), freq, inter, 0.0)
            assert (y.norm(dim=-1) - x.norm(dim=-1)).abs().max() < 1e-9
            dots.append(float((y[0, 0, 0] * y[0, 1, 0]).sum()))
        assert abs(dots[0] - dots[1]) < 1e-8
    y, _ = ref.norm_rope(x, torch.ones(32), torch.zeros(1, 2), freq, False, 0.0)
    assert ((y * y).mean(-1) - 1).abs().max() < 1e-12


def test_reference_selection_and_trees():
    total = [3.0, float("nan"), 3.0, -0.0, 0.0, float("inf"), -1.0, 5.0]
    assert ref.select(total, 8, 3, 1) == [0, 5, 7] and ref.select(total, 8, 8, 0) == list(range(8))
    assert ref.select(total, 8, 5, 0) == [0, 2, 3, 5, 7] and ref.select(total, 8, 2, 2) == [6, 7]
    rng = np.random.default_rng(0)
    for n_t in (1, 5, 64):
        words = ref.random_tree(rng, n_t)
        for t, w in enumerate(words):
            assert w >> t & 1 and w < 2 << t
            for j in range(t):
                assert not (w >> j & 1) or words[j] & ~w == 0          # ancestors bring their own ancestors
        assert [x & (1 << 64) - 1 for x in ref.to_int64(words)] == words
    assert math.isclose(ref.weight_error(0.0, 1), 2 * 120 * ref.U + 2 * ref.EXP2 + 2 * ref.U)


def test_workspace_does_not_grow_with_the_scores_of_the_whole_cache():
    """The weighted decode works through a cache in passes of 64 MiB of scores: 32 sequences of 32768 rows and 32 q-heads would
    fill 128 MiB.  Beyond that a context needs the partial results, and 48 MiB and the partial sums of the search reductions."""
    def workspace(B, n, Hq=32, Hkv=8, D=128):
        c = kb.kvs_create(1, Hq, Hkv, D, B, n, kb.KVS_BF16, 0.0, 0)
        ws = kb.kvs_required_bytes(c)[1]
        kb.kvs_destroy(c)
        return ws

    assert workspace(32, 32768) < 80 << 20
    assert workspace(32, 32768) - workspace(32, 16384) < 1 << 20          # both at the limit
    assert workspace(1, 1 << 20, Hq=64, Hkv=8) < 80 << 20                 # 8 units of 32 MiB of scores


@pytest.mark.parametrize("source,limits", [
    ("kvs_kernels.cu", ["score_count"]), ("kvs_mma.cu", ["score_count"]), ("kvs_rotary.cu", ["plane_bytes", "a.tokens"]),
    ("kvs_tree.cu", ["plane_bytes", "plane_vecs", "tree_piece_rows", "kTreeMaxTokens"]), ("kvs_tree_tc.cu", ["plane_rows", "tree_piece_rows", "a.n_t * a.Hq"]),
    ("kvs_weights.cu", ["score_count", "a.units + a.NC", "total_stride", "keep_stride"]),
])
def test_bounds_build_checks_the_serving_kernels_buffers(source, limits):
    """Every buffer the serving kernels index (scores, totals, partial results, keep lists, rows) is the limit of a check."""
    import os
    import re

    with open(os.path.join(kbuild.CSRC, source)) as f:
        text = re.sub(r"\s+", " ", f.read())
    calls = [text[m.end(): m.end() + 220].split("status)")[0] for m in re.finditer(r"KVS_BOUNDS_OK\(", text)]
    for limit in limits:
        assert any(limit in c for c in calls), (source, limit)


@pytest.mark.parametrize("source", ["kvs_rotary.cu", "kvs_tree.cu", "kvs_tree_tc.cu", "kvs_weights.cu"])
def test_launch_rules_ask_for_the_device_s_sm_count(source):
    import os
    import re

    with open(os.path.join(kbuild.CSRC, source)) as f:
        code = re.sub(r"//[^\n]*", "", f.read())
    assert not re.search(r"\b148\b", code)
