"""Beam selection and the reordering of sequences on the GPU, against float64 and against plain indexing; a beam search with both
over a 4-bit cache; refusals."""
import math

import pytest
import torch

import pack4_reference as ref
from helpers import GuardedCache
from paper_2410_18517_b200 import KVS_OPT_REPLAY, KvsError, SharedKVCache
from paper_2410_18517_b200 import binding as kb
from paper_2410_18517_b200 import build as kbuild

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    kbuild.build()


DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def ctx():
    return SharedKVCache(1, 2, 2, 64, 300, 16, "bf16")


def check_select(ctx, x, scores, W, K):
    got = ctx.beam_select(x, scores, W, K)
    want = ref.beams(x, scores.cpu(), W, K)
    s, t, p = (a.cpu() for a in got)
    for r, row in enumerate(want):
        assert t[r].tolist() == [c[1] for c in row], r
        assert p[r].tolist() == [c[2] for c in row], r
        exact = torch.tensor([c[0] for c in row], dtype=torch.float64)
        # the sum of the exponentials: the hardware's exp2 (2^-22) and fp32 sums, at most 16 in a thread for every 4096 logits
        # of the row and 16 to merge the threads; the score is rounded to fp32
        bound = 2.0 ** -22 + (16 * (x.shape[1] // 4096 + 1) + 16) * 2.0 ** -24 + 2.0 ** -24 * exact.abs()
        real = torch.isfinite(exact)
        assert torch.equal(s[r][~real].double(), exact[~real]) and ((s[r].double() - exact).abs()[real] <= bound[real]).all()
    again = ctx.beam_select(x, scores, W, K)
    assert all(torch.equal(a, b) for a, b in zip(got, again))
    assert ctx.device_status() == 0
    return got


def logits_of(seed, dtype, rows, V, spread=2.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, V, generator=g) * spread + torch.rand(rows, V, generator=g) ** 64 * 10
    return x.to(DT[dtype]).cuda()


SELECT = [
    # dtype, R, W, V, K
    ("f32", 1, 1, 1, 1), ("bf16", 2, 3, 1, 5), ("f32", 1, 4, 15, 8), ("bf16", 3, 2, 17, 40), ("f32", 2, 5, 1000, 10), ("bf16", 1, 1, 4096, 64),
    ("f32", 1, 1, 4097, 64), ("bf16", 2, 8, 32000, 16), ("f32", 1, 64, 9001, 64), ("bf16", 5, 4, 50257, 8), ("f32", 1, 2, 200003, 3),
    ("bf16", 1, 33, 12345, 33), ("bf16", 60, 5, 700, 2), ("f32", 4, 16, 65537, 32), ("bf16", 1, 4, 131072, 64), ("f32", 16, 1, 8191, 1),
]


@pytest.mark.parametrize("dtype,R,W,V,K", SELECT)
def test_select(ctx, dtype, R, W, V, K):
    g = torch.Generator().manual_seed(V)
    scores = (-torch.rand(R * W, generator=g) * 10).cuda()
    check_select(ctx, logits_of(V + W, dtype, R * W, V), scores, W, K)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_select_strided_and_unaligned_rows(ctx, dtype):
    """Rows of a padded tensor, rows that start off 16 bytes: the same bits whichever way they are read."""
    R, W, V, K = 2, 3, 10007, 7
    x = logits_of(1, dtype, R * W, V)
    scores = -torch.arange(6.0).cuda()
    want = check_select(ctx, x, scores, W, K)
    for width, at in ((V + 9, 0), (V + 9, 3), (V + 5, 1), (10016, 8)):
        room = torch.full((R * W, width + 16), math.nan, dtype=DT[dtype], device="cuda")
        room[:, at:at + V] = x
        got = ctx.beam_select(room[:, at:at + V], scores, W, K)
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [100, 5000, 40000])
def test_select_ties(ctx, dtype, V):
    """Few distinct logits, identical beams, all logits equal: the lowest (beam, token) first; zeros of either sign are equal."""
    W, K = 4, 16
    g = torch.Generator().manual_seed(V)
    few = torch.randint(0, 3, (2 * W, V), generator=g).float()
    few[few == 0] = torch.where(torch.rand(int((few == 0).sum()), generator=g) < 0.5, 0.0, -0.0)
    zero = torch.zeros(2 * W)
    check_select(ctx, few.to(DT[dtype]).cuda(), zero.cuda(), W, K)
    same = few[:1].expand(2 * W, V).contiguous()
    check_select(ctx, same.to(DT[dtype]).cuda(), zero.cuda(), W, K)
    s, t, p = check_select(ctx, torch.full((2 * W, V), 0.25, dtype=DT[dtype], device="cuda"), zero.cuda(), W, K)
    assert t.tolist() == [list(range(K))] * 2 and p.tolist() == [[0] * K, [W] * K]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [300, 70001])
def test_select_sorted_logits(ctx, dtype, V):
    """Logits that rise or fall along the row, or gather in one stretch: the threshold has to keep up."""
    ramp = torch.linspace(-8, 8, V)
    rows = torch.stack((ramp, ramp.flip(0), torch.where(torch.arange(V) < 200, ramp.flip(0) + 3, -5.0), ramp.abs()))
    check_select(ctx, rows.to(DT[dtype]).cuda(), torch.zeros(4).cuda(), 1, 64)
    check_select(ctx, rows.to(DT[dtype]).cuda(), torch.tensor([0.0, -0.3, -0.1, -0.2]).cuda(), 4, 64)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [40, 9000])
def test_select_masks_and_broken_rows(ctx, dtype, V):
    """Masked tokens, rows masked throughout, the type's lowest value as a mask, NaN and infinities, beams that do not count,
    fewer candidates than places."""
    W, K = 6, 12
    x = logits_of(3, dtype, 3 * W, V).cpu()
    low = torch.finfo(DT[dtype]).min
    x[0, 5:] = -math.inf                        # few tokens left
    x[1] = -math.inf                            # none
    x[2, V // 2] = math.nan
    x[3, V - 1] = math.inf
    x[4, ::2] = low
    x[5] = low                                  # all masked by the lowest value: all alike
    x[W:2 * W] = -math.inf                      # a request without candidates ...
    x[2 * W:, 3:] = -math.inf                   # ... and one with three per beam, of which one counts
    scores = torch.linspace(-1, 0, 3 * W)
    scores[2 * W + 1:] = -math.inf
    scores[4] = -0.5
    s, t, p = check_select(ctx, x.cuda(), scores.cuda(), W, K)
    assert t[1].tolist() == [-1] * K and p[1].tolist() == [W] * K and bool((s[1] == -math.inf).all())
    assert t[2, 3:].tolist() == [-1] * (K - 3) and set(p[2].tolist()) == {2 * W}
    scores[0] = math.nan
    scores[4] = math.inf
    check_select(ctx, x.cuda(), scores.cuda(), W, K)
    x[W + 2, 7] = -3.0                          # one candidate: probability one
    s, t, p = check_select(ctx, x.cuda(), torch.zeros(3 * W).cuda(), W, K)
    assert (float(s[1, 0]), int(t[1, 0]), int(p[1, 0])) == (0.0, 7, W + 2) and t[1, 1:].tolist() == [-1] * (K - 1)


def test_select_beams_that_nearly_tie(ctx):
    """Beams with the same logits up to a shift, scores that make up for it within 1e-5."""
    V, W = 20000, 8
    base = logits_of(9, "f32", 1, V).cpu()
    shift = torch.arange(W).float() * 2.0
    x = (base + shift[:, None]).float()
    scores = torch.arange(W).flip(0).float() * 1e-5
    check_select(ctx, x.cuda(), scores.cuda(), W, 2 * W)


def test_select_peaked_rows(ctx):
    """One token with all the probability but 1e-6: its score is the small difference from zero."""
    x = torch.zeros(2, 1000)
    x[0, 7], x[1, 999] = 20.0, 60.0
    s, t, _ = check_select(ctx, x.cuda(), torch.zeros(2).cuda(), 1, 3)
    exact = -math.log1p(999 * math.exp(-20))
    assert abs(float(s[0, 0]) - exact) < 16 * 2.0 ** -24 and float(s[1, 0]) == 0.0      # 13 sums next to one


# ---------------------------------------------------------------------------------------------- reordering


def filled(fmt, dtype, L, Hkv, D, old, n, max_batch, share=None, extra=5):
    cache = GuardedCache(L, Hkv, Hkv, D, max_batch, n + extra, dtype, share_map=share, cache_format=fmt)
    cache.paint(n + extra, max_batch)
    for l in range(L):
        if share is None or share[l] == l:
            g = torch.Generator(device="cuda").manual_seed(l)
            k, v = (torch.randn(old, n, Hkv, D, device="cuda", generator=g).to(DT[dtype]) for _ in range(2))
            cache.append(l, k, v)
    return cache


def check_reorder(cache, parent, first, old, n):
    before = [cache.plane(s, kv).clone() for s in range(cache.num_slots()) for kv in range(2)]
    cache.reorder(torch.tensor(parent, dtype=torch.int32).cuda(), first)
    want_status = kb.KVS_OK
    for i, x in enumerate(before):
        want = x.clone()
        for b, p in enumerate(parent):
            if 0 <= p < old:
                want[b, :, first:n] = x[p, :, first:n]
            else:
                want_status = kb.KVS_ERR_INVALID_ARG
        got = cache.plane(i // 2, i % 2)
        assert torch.equal(got.view(torch.uint8), want.view(torch.uint8)), i
    assert cache.device_status() == want_status
    assert kb.kvs_cached_batch(cache.ctx) == len(parent)
    for big in cache._guarded:
        assert bool((big[:1024] == 0xA5).all()) and bool((big[-1024:] == 0xA5).all())


REORDER = [
    # parents, cached sequences, first row
    ([0, 1, 2, 3], 4, 0), ([1, 0, 3, 2], 4, 0), ([3, 0, 1, 2], 4, 7), ([2, 2, 2, 2], 4, 0), ([0, 0, 3, 1], 4, 33), ([1, 1, 0, 3], 4, 99),
    ([0] * 6, 1, 0), ([0, 0, 0, 1, 1, 1], 2, 0), ([1, 3], 4, 0), ([3], 4, 0), ([2, 0, 1], 4, 50), ([0, 9, -1, 2], 4, 0), ([3, 2, 1, 0], 4, 100),
    ([3, 2, 1, 0], 4, 250), ([5, 4, 3, 2, 1, 0], 6, 0),
]


@pytest.mark.parametrize("parent,old,first", REORDER)
@pytest.mark.parametrize("fmt,dtype,D", [("plain", "bf16", 64), ("4bit", "bf16", 128), ("4bit", "f32", 64), ("plain", "f32", 128)])
def test_reorder(parent, old, first, fmt, dtype, D):
    n = 100
    cache = filled(fmt, dtype, 3, 2, D, old, n, 6, share=[0, 1, 0])
    check_reorder(cache, parent, first, old, n)


def test_reorder_many_sequences_and_long_rows():
    g = torch.Generator().manual_seed(0)
    for old, new, n, Hkv, D, fmt in ((300, 300, 13, 1, 64, "4bit"), (37, 37, 2100, 2, 128, "plain"), (1100, 1100, 3, 1, 64, "plain"), (2, 64, 1500, 2, 128, "4bit"),
                                     (8, 8, 9000, 4, 128, "plain")):
        cache = filled(fmt, "bf16", 1, Hkv, D, old, n, max(old, new))
        check_reorder(cache, torch.randint(0, old, (new,), generator=g).tolist(), 0, old, n)
        check_reorder(cache, torch.randperm(new, generator=g).tolist(), 2, new, n)


def test_reorder_slots_of_different_length():
    """In the middle of a step one layer has its new row and the next has not; an empty slot."""
    cache = GuardedCache(3, 2, 2, 64, 4, 40, "bf16")
    cache.paint(40, 4)
    x = torch.randn(4, 21, 2, 64, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    cache.append(0, x, x)
    cache.append(1, x[:, :20].contiguous(), x[:, :20].contiguous())
    cache.reorder(torch.tensor([3, 3, 0, 1], dtype=torch.int32, device="cuda"))
    for layer, n in ((0, 21), (1, 20)):
        k, _ = cache.read_rows(layer)
        assert torch.equal(k, x[[3, 3, 0, 1], :n])
    assert cache.seq_len(2) == 0 and not cache.plane(2, 0)[:, :, :40].any()
    cache.check_canaries()


def test_reorder_then_steps():
    """The batch a reorder leaves is the one appends and attention go by, also right behind it on the stream."""
    cache = GuardedCache(1, 4, 2, 64, 6, 30, "bf16", cache_format="4bit")
    cache.paint(30, 6)
    x = torch.randn(2, 9, 2, 64, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    cache.append(0, x, x)
    cache.reorder(torch.tensor([0, 0, 0, 1, 1, 1], dtype=torch.int32, device="cuda"))
    q = torch.randn(6, 4, 64, generator=torch.Generator().manual_seed(2)).bfloat16().cuda()
    new = torch.randn(6, 1, 2, 64, generator=torch.Generator().manual_seed(3)).bfloat16().cuda()
    out = cache.decode_step(0, q, new, new)
    cache.reorder(torch.tensor([4, 1], dtype=torch.int32, device="cuda"), 9)
    two = cache.decode_attention(0, q[[4, 1]].contiguous())
    k, _ = cache.read_rows(0)
    want = torch.cat((x[[1, 0]], new[[4, 1]]), 1)
    # rows before first_row stay those of sequences 0 and 1, both of request 0
    assert torch.equal(k[:, 9:].cpu(), ref.values(want[:, 9:].cpu())) and torch.equal(k[:, :9].cpu(), ref.values(x[[0, 0], :9].cpu()))
    assert (two[1] - out[1]).abs().max() < 1e-5      # the same rows in another split
    with pytest.raises(KvsError):
        cache.append(0, new, new)                    # six sequences no more
    cache.append(0, new[:2].contiguous(), new[:2].contiguous())
    assert cache.seq_len(0) == 11 and cache.device_status() == 0
    cache.check_canaries()


def test_recorded_beam_steps():
    """A beam-search step - decode, select, reorder - recorded once and replayed: the cache of the eager steps."""
    B, Hq, Hkv, D, V, n, steps = 4, 4, 2, 64, 97, 12, 6
    g = torch.Generator(device="cuda").manual_seed(0)
    k0, v0 = (torch.randn(B, n, Hkv, D, device="cuda", generator=g).bfloat16() for _ in range(2))
    emb = torch.randn(V, Hq + 2 * Hkv, D, device="cuda", generator=g).bfloat16()
    head = torch.randn(Hq * D, V, device="cuda", generator=g)
    eager, graph = (GuardedCache(1, Hq, Hkv, D, B, n + steps, "bf16", cache_format="4bit") for _ in range(2))

    def start(cache):
        cache.paint(n + steps, B)
        cache.append(0, k0, v0)
        return dict(tokens=torch.arange(B, dtype=torch.int32, device="cuda"), scores=torch.zeros(B, device="cuda"), out=torch.zeros(B, Hq, D, device="cuda"))

    def step(cache, s):
        x = emb[s["tokens"].long()]
        cache.decode_step(0, x[:, :Hq].contiguous(), x[:, None, Hq:Hq + Hkv].contiguous(), x[:, None, Hq + Hkv:].contiguous(), s["out"])
        score, token, parent = cache.beam_select(s["out"].view(B, -1) @ head, s["scores"], B, B)
        cache.reorder(parent.view(-1))
        s["scores"].copy_(score.view(-1))
        s["tokens"].copy_(token.view(-1))

    se, sg = start(eager), start(graph)
    step(graph, dict(sg, tokens=sg["tokens"].clone(), scores=sg["scores"].clone()))      # library handles, outside the recording
    graph.reset()
    sg = start(graph)
    graph.set_option(KVS_OPT_REPLAY, 1)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    rec = torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream):
        with torch.cuda.graph(rec, stream=stream):
            step(graph, sg)
            graph.replay_advance()
        for t in range(steps):
            step(eager, se)
            rec.replay()
            assert torch.equal(se["tokens"], sg["tokens"]), t
        stream.synchronize()
        graph.replay_commit(steps)
        assert graph.device_status() == 0 and graph.seq_len(0) == n + steps
        for a, b in zip(eager.read_rows(0), graph.read_rows(0)):
            assert torch.equal(a, b)
        with pytest.raises(KvsError):
            graph.reorder(torch.zeros(2, dtype=torch.int32, device="cuda"))      # a recorded step keeps its batch
    torch.cuda.synchronize()
    eager.check_canaries()
    graph.check_canaries()


@pytest.mark.parametrize("fmt,dtype", [("4bit", "bf16"), ("plain", "bf16"), ("4bit", "f32")])
def test_beam_search_as_it_is_used(fmt, dtype):
    """Two requests of three beams over three layers, one sharing: prompts, fork, steps, one request dropped, more steps.  Every
    cached row is that of the beam's own history, every selection the reference's on the same logits."""
    L, Hq, Hkv, D, V, W, n, share = 3, 4, 2, 64, 61, 3, 10, [0, 1, 0]
    g = torch.Generator().manual_seed(5)
    emb = torch.randn(L, V, Hq + 2 * Hkv, D, generator=g).to(DT[dtype])
    head = torch.randn(Hq * D, V, generator=g).cuda()
    cache = GuardedCache(L, Hq, Hkv, D, 2 * W, n + 8, dtype, share_map=share, cache_format=fmt)
    cache.paint(n + 8, 2 * W)
    hist = torch.randint(0, V, (2, n), generator=g).tolist()             # every beam's tokens
    for l in (0, 1):
        x = emb[l][torch.tensor(hist)]
        cache.append(l, x[:, :, Hq:Hq + Hkv].contiguous().cuda(), x[:, :, Hq + Hkv:].contiguous().cuda())

    def step(scores, requests, K):
        rows = torch.tensor([h[-1] for h in hist])
        out = 0
        for l in range(L):
            x = emb[l][rows]
            own = share[l] == l
            k, v = (x[:, None, a:a + Hkv].contiguous().cuda() if own else None for a in (Hq, Hq + Hkv))
            out = out + cache.decode_step(l, x[:, :Hq].contiguous().cuda(), k, v)
        logits = out.view(len(hist), -1) @ head
        W_ = len(hist) // requests
        got = cache.beam_select(logits, scores, W_, K)
        for r, row in enumerate(ref.beams(logits, scores.cpu(), W_, K)):
            assert got[1][r].tolist() == [c[1] for c in row] and got[2][r].tolist() == [c[2] for c in row]
        return got

    def check():
        for l in range(L):
            x = emb[share[l]][torch.tensor([h[:-1] for h in hist])]      # the newest token is not cached yet
            for got, a in zip(cache.read_rows(l), (Hq, Hq + Hkv)):
                want = x[:, :, a:a + Hkv]
                assert torch.equal(got.cpu(), ref.values(want) if fmt == "4bit" else want)

    # the first step: one beam per request, forked by what it selects
    for h in hist:
        h.append(0)
    s, t, p = step(torch.zeros(2).cuda(), 2, W)
    cache.reorder(p.view(-1).contiguous())
    hist = [hist[b] + [tok] for b, tok in zip(p.view(-1).tolist(), t.view(-1).tolist())]
    check()
    for _ in range(3):
        s, t, p = step(s.view(-1).contiguous(), 2, W)
        cache.reorder(p.view(-1).contiguous(), n)                          # the prompts of a request's beams are the same
        hist = [hist[b] + [tok] for b, tok in zip(p.view(-1).tolist(), t.view(-1).tolist())]
        check()
    # request 0 is finished: the other closes up
    cache.reorder(torch.arange(W, 2 * W, dtype=torch.int32, device="cuda"))
    hist, s = hist[W:], s[1:].contiguous()
    check()
    for _ in range(2):
        s, t, p = step(s.view(-1).contiguous(), 1, W)
        cache.reorder(p.view(-1).contiguous(), n)
        hist = [hist[b] + [tok] for b, tok in zip(p.view(-1).tolist(), t.view(-1).tolist())]
        check()
    assert cache.device_status() == 0
    cache.check_canaries()


def refused(status, fn, *args):
    with pytest.raises(KvsError) as e:
        fn(*args)
    assert e.value.status == status


def test_refusals():
    c = SharedKVCache(1, 4, 2, 64, 4, 20, "bf16")
    x = torch.zeros(4, 100, device="cuda")
    s = torch.zeros(4, device="cuda")
    o, t, p = torch.empty(8, device="cuda"), torch.empty(8, dtype=torch.int32, device="cuda"), torch.empty(8, dtype=torch.int32, device="cuda")
    ok = (x, kb.KVS_F32, 100, 100, s, 2, 2, 4, o, t, p)
    kb.kvs_beam_select(c.ctx, *ok)
    for i, bad in ((0, None), (1, 2), (1, -1), (2, 99), (3, 0), (3, 101), (4, None), (5, 0), (5, 3), (6, 0), (6, 65), (7, 0), (7, 65), (8, None), (9, None),
                   (10, None), (0, x.data_ptr() + 1), (4, s.data_ptr() + 2), (8, s)):
        args = list(ok)
        args[i] = bad
        refused(kb.KVS_ERR_INVALID_ARG, kb.kvs_beam_select, c.ctx, *args)
    refused(kb.KVS_ERR_INVALID_ARG, kb.kvs_beam_select, c.ctx, x, kb.KVS_F32, 1 << 40, 2147483647, s, 2, 2, 4, o, t, p)
    par = torch.zeros(8, dtype=torch.int32, device="cuda")
    refused(kb.KVS_ERR_STATE, kb.kvs_reorder, c.ctx, par, 0, 2)
    k = torch.zeros(2, 5, 2, 64, dtype=torch.bfloat16, device="cuda")
    c.append(0, k, k)
    for args in ((None, 0, 2), (par, -1, 2), (par, 0, 0), (par, 0, 5), (par, 1, 3), (par.data_ptr() + 2, 0, 2)):
        refused(kb.KVS_ERR_INVALID_ARG, kb.kvs_reorder, c.ctx, *args)
    c.evict(0, torch.zeros(2, 2, 5, dtype=torch.int32, device="cuda"), [[1, 1], [1, 1]])
    refused(kb.KVS_ERR_STATE, kb.kvs_reorder, c.ctx, par, 0, 2)
    torch.cuda.synchronize()
    assert c.device_status() == 0
