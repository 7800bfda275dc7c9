"""4-bit caches and beam search: what needs no device - sizes, refusals before memory is bound, and the references the GPU tests
use against independent restatements."""
import math
from fractions import Fraction

import pytest
import torch

import pack4_reference as ref
from paper_2410_18517_b200 import binding as kb
from paper_2410_18517_b200 import build as kbuild


@pytest.fixture(scope="module", autouse=True)
def _built():
    kbuild.build()


def refused(status, fn, *args):
    with pytest.raises(kb.KvsError) as e:
        fn(*args)
    assert e.value.status == status


def test_format_sizes():
    for D, row in ((64, 48), (128, 80)):
        for dt in (kb.KVS_BF16, kb.KVS_F32):
            c = kb.kvs_create(3, 8, 2, D, 4, 130, dt, 0.0, 0)
            kb.kvs_set_share_map(c, [0, 0, 2])
            plain, ws = kb.kvs_required_bytes(c)
            kb.kvs_set_cache_format(c, kb.KVS_CACHE_4BIT)
            pool, ws4 = kb.kvs_required_bytes(c)
            assert pool == 2 * 2 * 4 * 2 * 256 * row and kb.kvs_plane_offset(c, 1, 1) == 3 * 4 * 2 * 256 * row
            assert ws4 >= 2 * 2 * 256 * D * (2 if dt == kb.KVS_BF16 else 4)       # a sequence's rows in the storage type
            kb.kvs_set_cache_format(c, kb.KVS_CACHE_4BIT)
            kb.kvs_set_cache_format(c, kb.KVS_CACHE_PLAIN)
            assert kb.kvs_required_bytes(c) == (plain, ws)
            kb.kvs_destroy(c)


def test_workspace_of_long_caches():
    """Rows in the storage type: 64 MiB, or one sequence where that is more."""
    def workspace(B, n, fmt):
        c = kb.kvs_create(1, 32, 8, 128, B, n, kb.KVS_BF16, 0.0, 0)
        kb.kvs_set_cache_format(c, fmt)
        ws = kb.kvs_required_bytes(c)[1]
        kb.kvs_destroy(c)
        return ws

    assert workspace(32, 8192, kb.KVS_CACHE_4BIT) < 80 << 20
    assert 134 << 20 < workspace(2, 34304, kb.KVS_CACHE_4BIT) < 150 << 20


def test_refusals_without_memory():
    c = kb.kvs_create(2, 8, 2, 64, 4, 100, kb.KVS_BF16, 0.0, 0)
    p = 1 << 20                                  # never read: the context has no memory
    refused(kb.KVS_ERR_INVALID_ARG, kb.kvs_set_cache_format, c, 2)
    refused(kb.KVS_ERR_INVALID_ARG, kb.kvs_set_cache_format, c, -1)
    refused(kb.KVS_ERR_STATE, kb.kvs_read_rows, c, 0, 0, 1, p, p, 1)
    refused(kb.KVS_ERR_STATE, kb.kvs_beam_select, c, p, kb.KVS_F32, 10, 10, p, 1, 2, 2, p + 64, p, p)
    refused(kb.KVS_ERR_STATE, kb.kvs_reorder, c, p, 0, 1)
    kb.kvs_destroy(c)
    refused(kb.KVS_ERR_INVALID_ARG, kb.kvs_set_cache_format, None, 1)
    refused(kb.KVS_ERR_INVALID_ARG, kb.kvs_read_rows, None, 0, 0, 1, p, p, 1)
    refused(kb.KVS_ERR_INVALID_ARG, kb.kvs_beam_select, None, p, kb.KVS_F32, 10, 10, p, 1, 2, 2, p + 64, p, p)
    refused(kb.KVS_ERR_INVALID_ARG, kb.kvs_reorder, None, p, 0, 1)
    refused(kb.KVS_ERR_INVALID_ARG, kb.kvs_cached_batch, None)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_reference_rows_against_rationals(dtype):
    g = torch.Generator().manual_seed(0)
    for spread, offset in ((1.0, 0.0), (0.01, 3.0), (100.0, -7.0), (1e-20, 0.0), (1.0, 1e4)):
        x = (torch.randn(5, 64, generator=g) * spread + offset).to(dtype)
        c, s, b = ref.pack(x)
        for r in range(5):
            for k in range(4):
                xs = [Fraction(float(v)) for v in x[r, 16 * k:16 * k + 16].float()]
                S, O = Fraction(float(s[r, k, 0])), Fraction(float(b[r, k, 0]))
                assert S * 15 * (1 + Fraction(1, 1 << 20)) >= max(xs) - min(xs)
                for i, v in enumerate(xs):
                    want = min(15, max(0, round((v - O) / S) - 16)) if S else 0      # round(): ties to even
                    assert int(c[r, k, i]) == want
        assert ((ref.values(x).double() - x.double()).abs() <= ref.error_bound(x)).all()


def test_reference_rows_of_special_groups():
    x = torch.zeros(6, 64)
    x[1] = 0.3                                   # constant
    x[2, 5] = math.nan
    x[3, 20] = math.inf
    x[4, 40], x[4, 41] = 3e38, -3e38             # the range overflows
    x[5, :16] = torch.arange(16) * 0.5           # a grid: 0.5 apart, exactly its own codes
    v = ref.values(x)
    assert not v[0].any() and (v[1] - x[1]).abs().max() <= ref.error_bound(x[1]).max()
    for r, k in ((2, 0), (3, 1), (4, 2)):
        broken = torch.zeros(64, dtype=torch.bool)
        broken[16 * k:16 * k + 16] = True
        assert torch.equal(torch.isnan(v[r]), broken)
    assert torch.equal(v[5], x[5])
    raw = ref.row_bytes(x.bfloat16())
    assert raw.shape == (6, 48) and raw[5, 16:24].tolist() == [0x10, 0x32, 0x54, 0x76, 0x98, 0xBA, 0xDC, 0xFE]
    assert raw[5, :4].view(torch.bfloat16).tolist() == [0.5, -8.0]


def test_reference_beams():
    x = torch.tensor([[1.0, 2.0, 2.0], [0.0, -math.inf, 5.0], [math.nan, 0.0, 0.0], [-math.inf] * 3])
    got = ref.beams(x, torch.tensor([0.0, -1.0, 0.0, 0.0]), 2, 7)
    lse = math.log(math.exp(1) + 2 * math.exp(2))
    want = sorted([(1 - lse, 0, 0), (2 - lse, 1, 0), (2 - lse, 2, 0), (-1 - math.log(1 + math.exp(5)), 0, 1),
                   (4 - math.log(1 + math.exp(5)), 2, 1)], key=lambda t: (-t[0], t[2], t[1]))
    assert [t[1:] for t in got[0]] == [t[1:] for t in want] + [(-1, 0)] * 2
    assert all(abs(a[0] - b[0]) < 1e-6 for a, b in zip(got[0], want)) and got[1] == [(-math.inf, -1, 2)] * 7


@pytest.mark.parametrize("source,limits", [
    ("kvs_pack4.cu", ["plane_bytes", "out_bytes", "a.units"]), ("kvs_pack4_mma.cu", ["plane_bytes", "a.units"]),
    ("kvs_beam.cu", ["sum_count", "list_count", "plane_bytes"]),
])
def test_bounds_build_checks_the_buffers(source, limits):
    """Every buffer the kernels index is the limit of a check, and launch rules ask for the device's SM count."""
    import os
    import re

    with open(os.path.join(kbuild.CSRC, source)) as f:
        text = f.read()
    calls = [m.group(1) for m in re.finditer(r"KVS_BOUNDS_OK\(((?:[^()]|\([^()]*\))*)\)", text)]
    for limit in limits:
        assert any(limit in c for c in calls), (source, limit)
    assert not re.search(r"\b148\b", re.sub(r"//[^\n]*", "", text))
