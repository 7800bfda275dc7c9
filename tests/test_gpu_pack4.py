"""The 4-bit cache on the GPU: rows stored and read back bit for bit, attention over their values against float64, every call
that takes such a cache, and the refusals."""
import math

import pytest
import torch

import operators_reference as oref
import pack4_reference as ref
import synth_inputs as si
from helpers import GuardedCache
from paper_2410_18517_b200 import (KVS_OPT_EARLY_START, KVS_OPT_FINISH_IN_KERNEL, KVS_OPT_MAX_CTAS, KVS_OPT_REPLAY,
                                   KVS_OPT_WAIT_LIMIT_US, KvsError, Rotary, SharedKVCache)
from paper_2410_18517_b200 import binding as kb
from paper_2410_18517_b200 import build as kbuild

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    kbuild.build()


DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def normal(seed, dtype, *shape, offset=0.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) + offset).to(DT[dtype])


def cache4(Hq, Hkv, D, B, rows, dtype, L=1, share_map=None, cls=GuardedCache, in_use=None):
    cache = cls(L, Hq, Hkv, D, B, rows, dtype, share_map=share_map, cache_format="4bit")
    if isinstance(cache, GuardedCache):
        cache.paint(rows, in_use or B)
    return cache


def same(a, b):
    """Equal, NaN to NaN."""
    a, b = a.cpu(), b.cpu()
    return a.shape == b.shape and a.dtype == b.dtype and bool(((a == b) | (a.isnan() & b.isnan())).all())


def check_attention(cache, layer, q, out, lens=None):
    """out against float64 over the values the cache stands for.  The scores' products are exact in fp32 (bf16 by bf16; fp32
    storage: rounded), the weights enter as three bf16 terms (2^-24 of themselves) or in fp32."""
    B, Hq, D = q.shape
    Hkv = cache.shape[2]
    G = Hq // Hkv
    K, V = cache.read_rows(layer)
    for b in range(B):
        for h in range(Hkv):
            n = cache.unit_len(layer, b, h)
            o, _, mass, d = oref.attend(q[b, h * G:(h + 1) * G][None], K[b, :n, h], V[b, :n, h])
            bound = (oref.weight_error(d, n) + 2 * oref.U) * mass[0] + oref.U * o[0].abs() + 1e-30
            got = out[b, h * G:(h + 1) * G].double()
            assert torch.isfinite(got).all()
            assert ((got - o[0]).abs() <= bound).all(), (b, h, float(((got - o[0]).abs() / bound).max()))


# ----------------------------------------------------------------------------------------- storing and reading

STORE = [("bf16", 1, 64, 1, 1), ("bf16", 8, 128, 3, 1), ("bf16", 2, 128, 2, 301), ("bf16", 5, 64, 1, 77), ("f32", 2, 64, 3, 50),
         ("f32", 1, 128, 1, 1), ("f32", 3, 128, 2, 129), ("bf16", 1, 128, 33, 2), ("bf16", 8, 128, 1, 2500)]


@pytest.mark.parametrize("dtype,Hkv,D,B,n", STORE)
@pytest.mark.parametrize("offset,scale", [(0.0, 1.0), (3.0, 0.05), (-200.0, 30.0), (0.0, 1e-4)])
def test_rows_bit_for_bit(dtype, Hkv, D, B, n, offset, scale):
    cache = cache4(Hkv, Hkv, D, B + 1, n + 4, dtype, in_use=B)
    k, v = (normal(s, dtype, B, n, Hkv, D, offset=offset) * scale for s in (1, 2))
    k, v = k.to(DT[dtype]), v.to(DT[dtype])
    cache.append(0, k.cuda(), v.cuda())
    cache.append(0, k[:, :1].contiguous().cuda(), v[:, -1:].contiguous().cuda())
    for i, (x, more) in enumerate(((k, k[:, :1]), (v, v[:, -1:]))):
        raw = cache.plane(0, i)[:B, :, :n + 1].cpu()
        assert torch.equal(raw, ref.row_bytes(torch.cat((x, more), 1)).transpose(1, 2))
    ko, vo = cache.read_rows(0)
    assert torch.equal(ko.cpu(), ref.values(torch.cat((k, k[:, :1]), 1))) and torch.equal(vo.cpu(), ref.values(torch.cat((v, v[:, -1:]), 1)))
    assert ((ko[:, :n].cpu().double() - k.double()).abs() <= ref.error_bound(k)).all()
    first, count = n // 2, max(1, n // 3)
    kp, vp = cache.read_rows(0, first, count, batch=1)
    assert torch.equal(kp, ko[:1, first:first + count]) and torch.equal(vp, vo[:1, first:first + count])
    assert cache.device_status() == 0 and kb.kvs_cached_batch(cache.ctx) == B
    cache.check_canaries()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
def test_rows_of_special_values(dtype, D):
    """Constants, zeros of either sign, grids whose elements lie exactly between two codes, ranges that overflow, subnormal
    steps, infinities and NaN: the same bits as the reference, and broken groups do not touch their neighbours."""
    Q = D // 4
    x = normal(3, dtype, 1, 40, 1, D)
    big = 3e38
    x[0, 0] = 0
    x[0, 1] = -0.0
    x[0, 2] = 0.3
    x[0, 3, 0, :Q] = torch.arange(Q) % 16 * 0.5
    for i, step in enumerate((0.5, 0.25, 0.125)):       # s = 1: codes and every border between them
        x[0, 4 + i, 0] = (torch.arange(D) * step) % 15.5
        x[0, 4 + i, 0, 0::Q] = 0
        x[0, 4 + i, 0, 1::Q] = 15
    x[0, 7, 0, 1] = math.nan
    x[0, 8, 0, Q] = math.inf
    x[0, 9, 0, -1] = -math.inf
    x[0, 10, 0, 0], x[0, 10, 0, 1] = big, -big
    x[0, 11, 0, :Q] = big
    x[0, 12] *= 1e-38
    x[0, 13] *= 2e-40
    x[0, 14] = torch.arange(D).to(x.dtype) * 1e-45
    x[0, 15] *= 1e30
    x[0, 16] = torch.finfo(x.dtype).min
    x[0, 17, 0, ::2] = torch.finfo(x.dtype).min
    x[0, 18] = 7 + torch.arange(D) * 2.0 ** -5
    x[0, 19] = 1e4 + torch.arange(D) % 3
    x = x.to(DT[dtype])
    cache = cache4(1, 1, D, 1, 40, dtype)
    cache.append(0, x.cuda(), x.flip(1).contiguous().cuda())
    assert torch.equal(cache.plane(0, 0)[0, 0, :40].cpu(), ref.row_bytes(x)[0, :, 0])
    k, v = cache.read_rows(0)
    assert same(k, ref.values(x)) and same(v, ref.values(x).flip(1))


def test_reading_plain_caches():
    for dtype, D in (("bf16", 64), ("f32", 128)):
        cache = SharedKVCache(2, 4, 2, D, 3, 50, dtype, share_map=[0, 0])
        k, v = normal(1, dtype, 2, 41, 2, D).cuda(), normal(2, dtype, 2, 41, 2, D).cuda()
        k[0, 3, 1, 2] = math.nan
        cache.append(0, k, v)
        ko, vo = cache.read_rows(1, 1)
        assert same(ko, k[:, 1:]) and same(vo, v[:, 1:])


def test_rows_of_units_of_different_length():
    """Evicted 4-bit rows move as they are; appends go to every unit's own end; reading pads with zeros."""
    B, Hkv, D, n = 2, 3, 128, 70
    cache = cache4(Hkv, Hkv, D, B, n + 5, "bf16")
    k, v = normal(1, "bf16", B, n, Hkv, D), normal(2, "bf16", B, n, Hkv, D)
    cache.append(0, k.cuda(), v.cuda())
    lens = torch.tensor([[1, 70, 33], [17, 64, 2]])
    keep = torch.zeros(B, Hkv, n, dtype=torch.int32)
    g = torch.Generator().manual_seed(0)
    for b in range(B):
        for h in range(Hkv):
            keep[b, h, :lens[b, h]] = torch.randperm(n, generator=g)[:lens[b, h]].sort().values.int()
    cache.evict(0, keep.cuda(), lens)
    k1, v1 = normal(3, "bf16", B, 2, Hkv, D), normal(4, "bf16", B, 2, Hkv, D)
    cache.append(0, k1.cuda(), v1.cuda())
    ko, vo = cache.read_rows(0)
    assert ko.shape[1] == 72
    for b in range(B):
        for h in range(Hkv):
            m = int(lens[b, h])
            at = keep[b, h, :m].long()
            want = torch.cat((ref.values(k)[b, at, h], ref.values(k1)[b, :, h], torch.zeros(70 - m, D, dtype=torch.bfloat16)))
            assert torch.equal(ko[b, :, h].cpu(), want)
            assert torch.equal(vo[b, :m, h].cpu(), ref.values(v)[b, at, h]) and not vo[b, m + 2:, h].any()
    q = normal(5, "bf16", B, Hkv, D).cuda()
    check_attention(cache, 0, q, cache.decode_attention(0, q))
    assert cache.device_status() == 0
    cache.check_canaries()


@pytest.mark.parametrize("dtype,Hq,Hkv,D,B,n,max_seq", [("bf16", 8, 2, 128, 2, 5, 40), ("f32", 4, 4, 64, 3, 33, 64),
                                                      ("bf16", 8, 8, 128, 3, 9001, 9002)])
def test_rotary_append(dtype, Hq, Hkv, D, B, n, max_seq):
    """The rows a plain cache gets, packed; queries bit for bit; several passes over the scratch where the prompt is long."""
    x = normal(1, dtype, B, n, Hq + 2 * Hkv, D).cuda()
    pos = (torch.arange(n).int() * 3 + torch.arange(B).int()[:, None]).contiguous().cuda()
    w = (1 + 0.1 * normal(2, dtype, D)).to(DT[dtype]).cuda()
    plain = SharedKVCache(1, Hq, Hkv, D, B, max_seq, dtype)
    packed = cache4(Hq, Hkv, D, B, max_seq, dtype)
    rot = Rotary.from_theta(D)
    args = (0, x[:, :, :Hq], x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:], pos, rot, w, w)
    assert torch.equal(plain.append_rotary(*args), packed.append_rotary(*args))
    assert packed.seq_len(0) == n
    some = [0, n // 2, n - 1]
    for (a, b) in zip(plain.read_rows(0), packed.read_rows(0)):
        for b_ in range(B):
            assert torch.equal(b[b_, some].cpu(), ref.values(a[b_, some].cpu()))
    one = x[:, :1].contiguous()
    args = (0, one[:, :, :Hq], one[:, :, Hq:Hq + Hkv], one[:, :, Hq + Hkv:], pos[:, :1].contiguous(), rot, w, w)
    assert torch.equal(plain.append_rotary(*args), packed.append_rotary(*args))
    for (a, b) in zip(plain.read_rows(0, n), packed.read_rows(0, n)):
        assert torch.equal(b.cpu(), ref.values(a.cpu()))
    assert packed.device_status() == 0
    packed.check_canaries()


# ----------------------------------------------------------------------------------------------- attention

ATTEND = [
    # dtype, Hq, Hkv, D, B, n
    ("bf16", 1, 1, 128, 1, 1), ("bf16", 1, 1, 64, 1, 17), ("bf16", 4, 4, 128, 2, 63), ("bf16", 8, 4, 128, 1, 64), ("bf16", 6, 2, 64, 3, 65),
    ("bf16", 8, 2, 128, 2, 257), ("bf16", 5, 1, 128, 1, 700), ("bf16", 12, 2, 64, 2, 1031), ("bf16", 7, 1, 64, 40, 33), ("bf16", 16, 2, 128, 3, 2049),
    ("bf16", 32, 8, 128, 4, 5000), ("bf16", 40, 40, 128, 4, 900), ("bf16", 8, 1, 128, 1, 20011), ("bf16", 16, 16, 64, 20, 1500), ("bf16", 12, 4, 64, 1, 128),
    ("f32", 4, 4, 64, 2, 1), ("f32", 8, 2, 64, 2, 733), ("f32", 8, 1, 128, 1, 2000), ("f32", 4, 2, 128, 3, 64), ("f32", 2, 2, 128, 30, 65),
]


@pytest.mark.parametrize("dtype,Hq,Hkv,D,B,n", ATTEND)
def test_attention(dtype, Hq, Hkv, D, B, n):
    cache = cache4(Hq, Hkv, D, B + 1, n + 3, dtype, in_use=B)
    k, v = normal(1, dtype, B, n, Hkv, D, offset=0.5), normal(2, dtype, B, n, Hkv, D)
    cache.append(0, k.cuda(), v.cuda())
    q = normal(3, dtype, B, Hq, D).cuda()
    out = cache.decode_attention(0, q)
    check_attention(cache, 0, q, out)
    assert torch.equal(out, cache.decode_attention(0, q))              # the same bits every time
    # fewer sequences than are cached: the first ones
    less = cache.decode_attention(0, q[:1].contiguous())
    check_attention(cache, 0, q[:1], less)
    assert cache.device_status() == 0
    cache.check_canaries()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("ctas", [1, 2, 3, 5, 6, 7, 50])
def test_attention_any_split(dtype, ctas):
    """However the tiles are dealt out; finished in the kernel and by the combine step."""
    cache = cache4(8, 2, 128, 3, 1003, dtype)
    cache.append(0, normal(1, dtype, 3, 1000, 2, 128).cuda(), normal(2, dtype, 3, 1000, 2, 128).cuda())
    cache.set_option(KVS_OPT_MAX_CTAS, ctas)
    q = normal(3, dtype, 3, 8, 128).cuda()
    for finish in (1, 0):
        cache.set_option(KVS_OPT_FINISH_IN_KERNEL, finish)
        check_attention(cache, 0, q, cache.decode_attention(0, q))
    cache.check_canaries()


def test_many_units_and_the_hand_over():
    """As many units as blocks and more: units are cut between blocks and finished there."""
    for units_b, Hkv, G, D, n in ((40, 8, 4, 128, 1100), (160, 2, 1, 64, 600), (75, 4, 7, 128, 515)):
        cache = cache4(Hkv * G, Hkv, D, units_b, n, "bf16", cls=SharedKVCache)
        g = torch.Generator(device="cuda").manual_seed(1)
        k, v = (torch.randn(units_b, n, Hkv, D, device="cuda", generator=g).bfloat16() for _ in range(2))
        cache.append(0, k, v)
        q = torch.randn(units_b, Hkv * G, D, device="cuda", generator=g).bfloat16()
        out = cache.decode_attention(0, q)
        assert cache.last_launch()["kernel"] == 3
        cache.set_option(KVS_OPT_FINISH_IN_KERNEL, 0)
        again = cache.decode_attention(0, q)
        some = [0, units_b // 2, units_b - 1]
        K, V = cache.read_rows(0)
        for b in some:
            for h in range(Hkv):
                o, _, mass, d = oref.attend(q[b, h * G:(h + 1) * G][None], K[b, :, h], V[b, :, h])
                bound = (oref.weight_error(d, n) + 2 * oref.U) * mass[0] + oref.U * o[0].abs()
                assert ((out[b, h * G:(h + 1) * G].double() - o[0]).abs() <= bound).all()
        assert (out - again).abs().max() < 1e-5          # pieces merged in another order: sums of N(0, 1) shares
        assert cache.device_status() == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 15, 16, 17, 63, 64, 130])
def test_rolled_back_rows_reach_nothing(dtype, n):
    """Rows past a unit's end hold NaN and infinities (appended, then taken back)."""
    cache = cache4(8, 2, 64, 2, n + 90, dtype)
    junk = torch.full((2, 90, 2, 64), math.nan, dtype=DT[dtype])
    junk[:, ::2] = math.inf
    cache.append(0, normal(1, dtype, 2, n, 2, 64).cuda(), normal(2, dtype, 2, n, 2, 64).cuda())
    q = normal(3, dtype, 2, 8, 64).cuda()
    want = cache.decode_attention(0, q)
    cache.append(0, junk.cuda(), junk.cuda())
    cache.truncate(n)
    out = cache.decode_attention(0, q)
    check_attention(cache, 0, q, out)
    assert torch.equal(out, want)
    qp = normal(4, dtype, 2, n, 8, 64).cuda()
    assert torch.isfinite(cache.prefill_attention(0, qp)).all()
    cache.check_canaries()


def test_broken_rows_stay_in_their_unit_and_group():
    """A NaN in a cached key makes its unit's results NaN, one in a value only the group of columns it lies in."""
    cache = cache4(4, 4, 128, 2, 100, "bf16")
    k, v = normal(1, "bf16", 2, 100, 4, 128), normal(2, "bf16", 2, 100, 4, 128)
    k[0, 50, 1, 3] = math.nan
    v[1, 99, 2, 70] = math.inf
    cache.append(0, k.cuda(), v.cuda())
    out = cache.decode_attention(0, normal(3, "bf16", 2, 4, 128).cuda()).cpu()
    broken = torch.zeros(2, 4, 128, dtype=torch.bool)
    broken[0, 1] = True
    broken[1, 2, 64:96] = True
    assert torch.equal(out.isnan(), broken) and torch.isfinite(out[~broken]).all()


def test_large_scores_and_shares_that_cancel():
    """Scores far apart (one row takes all), and values of alternating sign whose shares nearly cancel."""
    n = 4000
    cache = cache4(2, 2, 128, 1, n, "bf16")
    k, v = normal(1, "bf16", 1, n, 2, 128), normal(2, "bf16", 1, n, 2, 128)
    k[:, :, 1] *= 30
    v[:, :, 0] = ((-1.0) ** torch.arange(n)[:, None] * 7 + 0.01 * torch.randn(n, 128, generator=torch.Generator().manual_seed(5))).bfloat16()
    cache.append(0, k.cuda(), v.cuda())
    q = normal(3, "bf16", 1, 2, 128).cuda()
    check_attention(cache, 0, q, cache.decode_attention(0, q))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_steps_shared_layers_and_host_buffers(dtype):
    """Decode steps over three layers, one of them sharing: kvs_decode_step, kvs_append + kvs_decode_attention, kvs_step_host and
    the static form give the same bits, with and without early starts."""
    L, Hq, Hkv, D, B, n, share = 3, 8, 2, 64, 2, 70, [0, 1, 0]
    caches = [cache4(Hq, Hkv, D, B, n + 4, dtype, L=L, share_map=share) for _ in range(4)]
    caches[3].set_option(KVS_OPT_EARLY_START, 0)
    for l in (0, 1):
        k, v = normal(10 + l, dtype, B, n, Hkv, D).cuda(), normal(20 + l, dtype, B, n, Hkv, D).cuda()
        for c in caches:
            c.append(l, k, v)
    status = torch.full((1,), 5, dtype=torch.int32, device="cuda")
    for t in range(4):
        q, k, v = (normal(100 * t + i, dtype, L, B, *s) for i, s in enumerate(((Hq, D), (1, Hkv, D), (1, Hkv, D))))
        outs = [[], [], [], []]
        for l in range(L):
            own = share[l] == l
            ql, kl, vl = q[l].cuda(), k[l].cuda() if own else None, v[l].cuda() if own else None
            outs[0].append(caches[0].decode_step(l, ql, kl, vl))
            for i in (1, 3):
                caches[i].append(l, kl, vl, B, 1)
                outs[i].append(caches[i].decode_attention(l, ql))
            check_attention(caches[0], l, ql, outs[0][-1])
            st = torch.empty_like(outs[1][-1])
            kb.kvs_decode_attention_static(caches[1].ctx, l, ql, st, B, torch.cuda.current_stream().cuda_stream, status)
            assert torch.equal(st, outs[1][-1]) and int(status) == 0
        out_host = torch.empty(L, B, Hq, D)
        caches[2].step_host(q, k, v, out_host)
        for l in range(L):
            assert torch.equal(outs[0][l], outs[1][l]) and torch.equal(outs[0][l], outs[3][l])
            assert torch.equal(outs[0][l].cpu(), out_host[l])
    assert caches[0].stats()["fused_appends"] == (8 if dtype == "bf16" else 0)      # two own layers, four steps
    for c in caches:
        assert c.device_status() == 0 and c.seq_len(2) == n + 4
        c.check_canaries()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_recorded_steps(dtype):
    """A recorded step replayed until the slot is full grows the same cache as eager steps; one more replay is refused on the
    device."""
    Hq, Hkv, D, B, n, steps = 8, 2, 128, 2, 60, 9
    eager, graph = (cache4(Hq, Hkv, D, B, n + steps, dtype) for _ in range(2))
    k, v = normal(1, dtype, B, n, Hkv, D).cuda(), normal(2, dtype, B, n, Hkv, D).cuda()
    for c in (eager, graph):
        c.append(0, k, v)
    graph.set_option(KVS_OPT_REPLAY, 1)
    q1, k1, v1 = (torch.zeros(*s, dtype=DT[dtype], device="cuda") for s in ((B, Hq, D), (B, 1, Hkv, D), (B, 1, Hkv, D)))
    out = torch.zeros(B, Hq, D, device="cuda")
    stream = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream):
        with torch.cuda.graph(g, stream=stream):
            graph.decode_step(0, q1, k1, v1, out)
            graph.replay_advance()
        for t in range(steps):
            for x, s in ((q1, 5), (k1, 6), (v1, 7)):
                x.copy_(normal(100 * t + s, dtype, *x.shape))
            g.replay()
            want = eager.decode_step(0, q1.clone(), k1.clone(), v1.clone())
            bound = 1e-5 if t else 0.0           # tiles are dealt out for the recorded length: another order of the same sums
            assert (out - want).abs().max() <= bound
        stream.synchronize()
        assert graph.device_status() == 0
        g.replay()                               # the slot is full: nothing is appended
        stream.synchronize()
        assert graph.device_status() == kb.KVS_ERR_CAPACITY
        graph.clear_device_status()
        graph.replay_commit(steps)
        assert graph.seq_len(0) == n + steps
        for a, b in zip(eager.read_rows(0), graph.read_rows(0)):
            assert torch.equal(a, b)
        stream.synchronize()
    eager.check_canaries()
    graph.check_canaries()


# -------------------------------------------------------------------------------------------------- prompts


@pytest.mark.parametrize("dtype,Hq,Hkv,D,B,n,T", [("bf16", 8, 2, 128, 2, 300, 300), ("bf16", 4, 4, 64, 3, 129, 1), ("bf16", 7, 1, 128, 1, 1000, 77),
                                                  ("f32", 4, 2, 64, 2, 70, 33), ("bf16", 8, 8, 128, 3, 9001, 5), ("bf16", 1, 1, 64, 1, 1, 1)])
def test_prompts(dtype, Hq, Hkv, D, B, n, T):
    """The bits of a plain cache that holds the values; several passes where the scratch holds fewer sequences."""
    packed = cache4(Hq, Hkv, D, B, n, dtype, cls=SharedKVCache)
    plain = SharedKVCache(1, Hq, Hkv, D, B, n, dtype)
    packed.append(0, normal(1, dtype, B, n, Hkv, D).cuda(), normal(2, dtype, B, n, Hkv, D).cuda())
    plain.append(0, *packed.read_rows(0))
    q = normal(3, dtype, B, T, Hq, D).cuda()
    assert torch.equal(packed.prefill_attention(0, q), plain.prefill_attention(0, q))
    q1 = q[:, -1].contiguous()
    a, b = packed.decode_attention(0, q1), plain.decode_attention(0, q1)
    # the plain cache's kernel holds the weights in two bf16 terms: 2^-16 of their share, and both kernels' fp32 sums
    assert (a - b).abs().max() <= (2.0 ** -16 + 2e-6) * max(1.0, float(plain.read_rows(0)[1].float().abs().max()))
    assert packed.device_status() == 0


# -------------------------------------------------------------------------------------------------- refusals


def refused(status, fn, *args):
    with pytest.raises(KvsError) as e:
        fn(*args)
    assert e.value.status == status


def test_refusals():
    c = cache4(4, 2, 64, 2, 20, "bf16")
    k = normal(1, "bf16", 2, 10, 2, 64).cuda()
    q = normal(2, "bf16", 2, 4, 64).cuda()
    ko, vo = torch.empty_like(k), torch.empty_like(k)
    refused(kb.KVS_ERR_STATE, c.decode_attention, 0, q)
    refused(kb.KVS_ERR_STATE, kb.kvs_read_rows, c.ctx, 0, 0, 1, ko, vo, 1)
    c.append(0, k, k)
    refused(kb.KVS_ERR_STATE, kb.kvs_set_cache_format, c.ctx, kb.KVS_CACHE_PLAIN)
    refused(kb.KVS_ERR_STATE, c.tree_attention, 0, q[:, None].contiguous())
    refused(kb.KVS_ERR_STATE, c.decode_attention_weights, 0, q, torch.zeros(2, 2, 20, device="cuda"))
    refused(kb.KVS_ERR_STATE, c.layer_distances)
    refused(kb.KVS_ERR_CAPACITY, c.append, 0, torch.zeros(2, 11, 2, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(2, 11, 2, 64, dtype=torch.bfloat16, device="cuda"))
    for args in ((1, 0, 1, ko, vo, 1), (0, -1, 1, ko, vo, 1), (0, 0, 0, ko, vo, 1), (0, 0, 11, ko, vo, 1), (0, 10, 1, ko, vo, 1), (0, 0, 1, ko, vo, 0),
                 (0, 0, 1, ko, vo, 3), (0, 0, 1, None, vo, 1), (0, 0, 1, ko, None, 1), (0, 0, 1, ko.data_ptr() + 2, vo, 1), (0, 2147483647, 2147483647, ko, vo, 1)):
        refused(kb.KVS_ERR_INVALID_ARG, kb.kvs_read_rows, c.ctx, *args)
    assert c.seq_len(0) == 10 and c.device_status() == 0
    c.reset()
    kb.kvs_set_cache_format(c.ctx, kb.KVS_CACHE_PLAIN)           # other sizes: the memory must be bound again
    refused(kb.KVS_ERR_STATE, c.append, 0, k, k)
    c.check_canaries = None


def test_a_stalled_copy_ends_with_an_error_status():
    c = cache4(8, 2, 128, 2, 700, "bf16")
    k = normal(1, "bf16", 2, 700, 2, 128).cuda()
    c.append(0, k, k)
    q = normal(2, "bf16", 2, 8, 128).cuda()
    want = c.decode_attention(0, q)
    c.set_option(KVS_OPT_WAIT_LIMIT_US, 2000)
    out = torch.empty_like(want)
    kb.kvs_selftest_stalled_copy(c.ctx, 0, q, out, 2, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert c.device_status() == kb.KVS_ERR_TIMEOUT
    c.clear_device_status()
    c.set_option(KVS_OPT_WAIT_LIMIT_US, 2000000)
    assert torch.equal(c.decode_attention(0, q), want) and c.device_status() == 0
    f = cache4(4, 4, 64, 1, 10, "f32")
    x = normal(1, "f32", 1, 10, 4, 64).cuda()
    f.append(0, x, x)
    refused(kb.KVS_ERR_STATE, kb.kvs_selftest_stalled_copy, f.ctx, 0, x[:, 0].contiguous(), torch.empty(1, 4, 64, device="cuda"), 1)


@pytest.mark.parametrize("Hq,Hkv,dtype", [(8, 8, "bf16"), (8, 2, "bf16"), (4, 4, "f32")])
def test_static_calls_twice_in_a_row(Hq, Hkv, dtype):
    """The form without a workspace: nothing the call before left in the built-in scratch is used, results as the other form's.

    It also loads kernels before tests/test_zz_no_alloc.py compares the device's free memory around the same calls: the
    driver loads a kernel's code at its first launch and takes 2 MiB when a chunk fills up, which that comparison cannot
    tell from an allocation.  With CUDA_MODULE_LOADING=EAGER that file passes without this test.
    """
    w = si.Workload(f"pack4_static_{Hq}_{Hkv}_{dtype}", L=3, Hq=Hq, Hkv=Hkv, D=128, B=4, context=2500, dtype=dtype, n_shared=1,
                    map_seed=0, steps=1, fixed_map=(0, 1, 0))
    cache = SharedKVCache(w.L, Hq, Hkv, w.D, w.B, w.context, dtype, share_map=w.share_map(), cache_format="4bit")
    for l in (0, 1):
        cache.append(l, *si.context_kv(w, l, device="cuda"))
    stream = torch.cuda.current_stream().cuda_stream
    status = torch.full((1,), -1, dtype=torch.int32, device="cuda")
    for call, layer in enumerate((2, 1)):
        q = si.step_qkv(w, call, layer, device="cuda")[0]
        ref_out = cache.decode_attention(layer, q)
        out = torch.full_like(ref_out, float("nan"))
        kb.kvs_decode_attention_static(cache.ctx, layer, q, out, w.B, stream, status)
        torch.cuda.synchronize()
        assert int(status.item()) == 0 and torch.equal(out, ref_out)
        assert (out - ref_out).abs().max().item() == 0 and ((out - ref_out).norm() / ref_out.norm()).item() == 0
        check_attention(cache, layer, q, out)
    out2 = torch.empty_like(ref_out)
    kb.kvs_decode_attention_static(cache.ctx, 1, q, out2, w.B, stream, None)
    assert torch.equal(out2, ref_out)
