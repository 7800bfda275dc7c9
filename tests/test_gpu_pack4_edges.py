"""The 4-bit cache where its numbers are extreme."""
import math
import random
from fractions import Fraction

import pytest
import torch

import operators_reference as oref
import pack4_reference as ref
from paper_2410_18517_b200 import KVS_OPT_REPLAY, Rotary, SharedKVCache
from paper_2410_18517_b200 import binding as kb
from paper_2410_18517_b200 import build as kbuild

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    kbuild.build()


DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def stored(x, dtype):
    """The bytes of a 4-bit cache's K rows of x [tokens][D], and what reading them gives."""
    cache = SharedKVCache(1, 1, 1, x.shape[1], 1, x.shape[0], dtype, cache_format="4bit")
    rows = x.to(DT[dtype])[None, :, None].contiguous().cuda()
    cache.append(0, rows, rows)
    raw, (k, v) = cache.plane(0, 0)[0, 0, :x.shape[0]].cpu(), cache.read_rows(0)
    assert torch.equal(cache.plane(0, 1)[0, 0, :x.shape[0]].cpu(), raw) and torch.equal(v.view(torch.uint8), k.view(torch.uint8))
    assert cache.device_status() == 0
    return raw, k[0, :, 0].cpu()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
def test_groups_whose_range_is_near_the_largest_number(dtype, D):
    """x - b, up to 31 steps, passes the fp32 range long before s and b do (a range of 1.7e38): codes and bytes are the
    definition's up to where b overflows, and NaN from there on."""
    g = torch.Generator().manual_seed(D)
    scale = torch.logspace(36, 38.5, 200, dtype=torch.float64)[:, None]
    x = ((torch.rand(200, D, generator=g, dtype=torch.float64) * 2 - 1) * scale)
    x[100:] += scale[100:] * 0.5 * (torch.rand(100, 1, generator=g, dtype=torch.float64) - 0.5)
    x = x.clamp(-3.3e38, 3.3e38).to(DT[dtype])
    raw, values = stored(x, dtype)
    assert torch.equal(raw, ref.row_bytes(x))
    want = ref.values(x)
    assert bool(want.isnan().any()) and bool(((values == want) | (values.isnan() & want.isnan())).all())
    wide = x.float().unflatten(1, (4, -1))
    wide = (wide.amax(-1) - wide.amin(-1) > 1.7e38) & ~want.unflatten(1, (4, -1)).isnan().any(-1)
    assert int(wide.sum()) > 20                  # groups with values whose differences overflow


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_values_that_lie_on_sixteen_levels(dtype):
    """Grids of every bf16 significand, and values read from such a cache: stored (again) as the definition says, bit for bit."""
    steps = torch.arange(128).mul(2.0 ** -7).add(1.0).bfloat16().float()
    grids = (torch.arange(16).repeat(4)[None] * steps[:, None]).to(DT[dtype])
    for x in (grids, torch.randn(300, 64, generator=torch.Generator().manual_seed(3)).to(DT[dtype])):
        for _ in range(3):
            raw, values = stored(x, dtype)
            assert torch.equal(raw, ref.row_bytes(x)) and torch.equal(values, ref.values(x))
            x = values


@pytest.mark.parametrize("Hq,Hkv,D,n,T", [(8, 2, 128, 700, 700), (2, 2, 64, 1300, 5), (7, 1, 128, 150, 33)])
def test_prompts_and_single_tokens_are_as_exact_as_the_header_says(Hq, Hkv, D, n, T):
    """Weights of 2^-16 for prompts and 2^-24 for single tokens, over the values the cache stands for."""
    g = torch.Generator().manual_seed(n)
    cache = SharedKVCache(1, Hq, Hkv, D, 1, n, "bf16", cache_format="4bit")
    cache.append(0, *(torch.randn(1, n, Hkv, D, generator=g).bfloat16().cuda() for _ in range(2)))
    q = torch.randn(1, T, Hq, D, generator=g).bfloat16().cuda()
    prompt, single = cache.prefill_attention(0, q), cache.decode_attention(0, q[:, -1].contiguous())
    K, V = (x[0].cpu() for x in cache.read_rows(0))
    sees = torch.arange(n) <= torch.arange(n - T, n)[:, None]
    for h in range(Hq):
        o, _, mass, d = oref.attend(q[0, :, h:h + 1].cpu(), K[:, h // (Hq // Hkv)], V[:, h // (Hq // Hkv)], sees)
        rest = oref.weight_error(d, n) * mass + oref.U * o.abs()
        # (the tensor cores' sums over the keys may be cut off instead of rounded: 2^-23 for each product of 16 keys)
        assert ((prompt[0, :, h:h + 1].cpu().double() - o).abs() <= rest + (2.0 ** -16 + n / 16 * 2.0 ** -23) * mass).all()
        assert ((single[0, h].cpu().double() - o[-1, 0]).abs() <= rest[-1, 0] + 2.0 ** -24 * mass[-1, 0]).all()
    assert cache.device_status() == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("at", [-130, -110, -60, 0, 60, 123])
def test_ties_that_a_tiny_element_decides(dtype, at):
    """Elements that are next to nothing beside their group's step, where -b / s is a whole number and a half: their sign
    decides between two codes, though x - b is b in fp64 too.  Against rationals, steps of every size."""
    n, group = 400, 16
    r = random.Random(at)
    x = torch.zeros(n, 64, dtype=torch.float64)
    for t in range(n):
        for k in range(4):
            # hi - lo is 15 s up to rounding, lo such that b = lo - 16 s lies on a half step
            s = r.randint(128, 255) * 2.0 ** (at - 8)
            lo = -s * (r.randint(0, 14) + 0.5)
            x[t, 16 * k], x[t, 16 * k + 1] = lo, lo + 15 * s * (1 - 2.0 ** -6)
            for i in range(2, group):
                x[t, 16 * k + i] = r.choice((-1, 1)) * 2.0 ** max(-133, at - r.choice((20, 60, 100, 200)))
    x = x.to(DT[dtype])
    raw, _ = stored(x, dtype)
    head = raw[:, :16].clone().view(torch.bfloat16).view(n, 4, 2)
    codes = torch.stack((raw[:, 16:] & 15, raw[:, 16:] >> 4), -1).view(n, 4, group)
    ties = 0
    for t in range(n):
        for k in range(4):
            s, b = (Fraction(float(v)) for v in head[t, k])
            for i in range(group):
                q = (Fraction(float(x[t, group * k + i])) - b) / s
                ties += abs(q - (math.floor(q) + Fraction(1, 2))) < Fraction(1, 2 ** 18)
                assert int(codes[t, k, i]) == min(15, max(0, round(q) - 16)), (t, k, i, float(q))
    assert ties > 50


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rotary_steps_recorded_and_replayed_to_the_end(dtype):
    """Rotary append and attention over 4-bit rows, replayed until the slot is full: the rows of eager steps; one replay more
    stores nothing and says so."""
    Hq, Hkv, D, B, n, steps = 8, 2, 64, 3, 61, 5
    g = torch.Generator().manual_seed(0)
    new = lambda *s: torch.randn(*s, generator=g).to(DT[dtype]).cuda()  # noqa: E731
    eager, graph = (SharedKVCache(2, Hq, Hkv, D, B, n + steps, dtype, share_map=[0, 0], cache_format="4bit") for _ in range(2))
    k, v = new(B, n, Hkv, D), new(B, n, Hkv, D)
    for c in (eager, graph):
        c.append(0, k, v)
    graph.set_option(KVS_OPT_REPLAY, 1)
    rot, x = Rotary.from_theta(D), torch.zeros(B, 1, Hq + 2 * Hkv, D, dtype=DT[dtype], device="cuda")
    pos = torch.zeros(B, 1, dtype=torch.int32, device="cuda")

    def step(c, out):
        q = c.append_rotary(0, x[:, :, :Hq], x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:], pos, rot)
        for l in range(2):
            c.decode_attention(l, q[:, 0].contiguous(), out[l])

    got, want = (torch.zeros(2, B, Hq, D, device="cuda") for _ in range(2))
    rec = torch.cuda.CUDAGraph()
    with torch.cuda.graph(rec):
        step(graph, got)
        graph.replay_advance()
    for t in range(steps):
        x.copy_(new(*x.shape))
        pos.fill_(n + t)
        rec.replay()
        step(eager, want)
        # (tiles are dealt out for the recorded length: another order of the same fp32 sums of some 60 rows)
        assert float((got - want).abs().max()) <= 70 * 2.0 ** -24 * 4
    assert graph.device_status() == 0
    before = [graph.plane(0, kv).clone() for kv in range(2)]
    rec.replay()
    torch.cuda.synchronize()
    assert graph.device_status() == kb.KVS_ERR_CAPACITY
    assert all(torch.equal(graph.plane(0, kv), before[kv]) for kv in range(2))
    graph.clear_device_status()
    graph.replay_commit(steps)
    assert graph.seq_len(1) == n + steps
    assert all(torch.equal(a, b) for a, b in zip(eager.read_rows(0), graph.read_rows(1)))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rotary_tokens_behind_units_of_different_length(dtype):
    """After an eviction every unit of a 4-bit cache takes the new tokens behind its own rows, as a plain cache's do."""
    Hq, Hkv, D, B, n = 4, 2, 128, 3, 40
    g = torch.Generator().manual_seed(1)
    new = lambda *s: torch.randn(*s, generator=g).to(DT[dtype]).cuda()  # noqa: E731
    packed, plain = (SharedKVCache(1, Hq, Hkv, D, B, n + 6, dtype, cache_format=f) for f in ("4bit", "plain"))
    k, v = new(B, n, Hkv, D), new(B, n, Hkv, D)
    keep = torch.arange(n, dtype=torch.int32).expand(B, Hkv, n).contiguous().cuda()
    lens = [7, 40, 1, 23, 39, 16]
    x, rot = new(B, 3, Hq + 2 * Hkv, D), Rotary.from_theta(D)
    pos = torch.arange(n, n + 3, dtype=torch.int32).expand(B, 3).contiguous().cuda()
    for c in (packed, plain):
        c.append(0, k, v)
        c.evict(0, keep, lens)
        c.append_rotary(0, x[:, :, :Hq], x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:], pos, rot)
    assert packed.seq_len(0) == 43
    for a, b in zip(plain.read_rows(0), packed.read_rows(0)):
        for u, m in enumerate(lens):
            i, h = divmod(u, Hkv)
            assert packed.unit_len(0, i, h) == m + 3
            assert torch.equal(b[i, :m + 3, h].cpu(), ref.values(a[i, :m + 3, h].cpu())) and not b[i, m + 3:, h].any()
    assert packed.device_status() == 0
