"""The serving operators in calls that the header allows and their main tests do not make."""
import numpy as np
import pytest
import torch

import operators_reference as ref
import test_gpu_operators as t
from paper_2410_18517_b200 import KVS_OPT_REPLAY, KvsError, Rotary
from paper_2410_18517_b200 import build as kbuild

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    kbuild.build()


# ------------------------------------------------------------------------------------------ rotary append

@pytest.mark.parametrize("dtype,Hq,Hkv,D,B,n_new", [("bf16", 32, 8, 128, 1, 900), ("f32", 14, 7, 128, 3, 700), ("bf16", 32, 8, 128, 2, 3),
                                                    ("f32", 4, 2, 64, 1, 1), ("bf16", 4, 2, 64, 2, 1000)])
@pytest.mark.parametrize("norm", [True, False])
def test_append_rotary_without_positions(dtype, Hq, Hkv, D, B, n_new, norm):
    """Nothing is rotated (rotary_dim 0), so there are no positions: by both kernels, on a computing and a sharing layer."""
    cache, _, _ = t.filled(Hq, Hkv, D, B, 4, dtype, extra=n_new, L=2, share_map=[0, 0])
    q, k, v = (t.normal(3 + i, dtype, B, n_new, h, D) for i, h in enumerate((Hq, Hkv, Hkv)))
    qw, kw = (t.normal(8, dtype, D), t.normal(9, dtype, D)) if norm else (None, None)
    pos = torch.zeros(B, n_new, dtype=torch.int32, device="cuda")
    got = cache.append_rotary(0, q, k, v, None, Rotary([]), qw, kw)
    K, V = cache.plane(0, 0)[:B, :, 4:4 + n_new].transpose(1, 2), cache.plane(0, 1)[:B, :, 4:4 + n_new].transpose(1, 2)
    assert torch.equal(cache.append_rotary(1, q, None, None, None, Rotary([]), qw), got)
    if norm:
        t.check_rotary(got, q, qw, pos, [], False, 1e-6)
        t.check_rotary(K, k, kw, pos, [], False, 1e-6)
    else:
        assert torch.equal(got, q) and torch.equal(K, k)
    assert torch.equal(V, v) and cache.seq_len(0) == 4 + n_new
    assert cache.device_status() == 0
    cache.check_canaries()


# ----------------------------------------------------------------------------------------- tree attention

@pytest.mark.parametrize("Hq,Hkv,D,B,n,n_t", [(8, 2, 128, 2, 70, 7), (8, 8, 64, 2, 300, 30), (32, 8, 128, 1, 2100, 64), (5, 5, 128, 3, 9, 9),
                                              (8, 1, 128, 1, 9000, 33)])
def test_tree_weights_keep_sixteen_bits(Hq, Hkv, D, B, n, n_t):
    """The softmax weights reach the second product with both bf16 terms: beside the rounding of the result to its own
    type, an element is off by 2^-16 of the sum of |weight * value|, not by 2^-8 of it.  (hi = bf16(p) leaves a remainder of
    2^-8 p at most, of which lo = bf16(p - hi) keeps all but 2^-8: 2^-16 p.)"""
    cache, _, _ = t.filled(Hq, Hkv, D, B, n, "bf16")
    rng = np.random.default_rng(n)
    words = [ref.random_tree(rng, n_t) for _ in range(B)]
    q = t.normal(7, "bf16", B, n_t, Hq, D)
    out = cache.tree_attention(0, q, torch.tensor([ref.to_int64(w) for w in words]).cuda())
    G = Hq // Hkv
    for b in range(B):
        for h in range(Hkv):
            K, V = t.rows_of(cache, 0, b, h)
            o, _, mass, d = ref.attend(q[b, :, h * G:(h + 1) * G], K, V, ref.tree_sees(words[b], n, n_t).cuda())
            # (weight_error counts 2 n u for sums rounded to nearest; those of the tensor cores may be cut off: n 2^-23 more)
            rest = (ref.weight_error(d, n) + 2.0 ** -16 + n * 2.0 ** -23) * mass
            got = out[b, :, h * G:(h + 1) * G].double()
            bound = ref.half_step(q.dtype) * (o.abs() + rest) + rest + 1e-30
            assert ((got - o).abs() <= bound).all(), float(((got - o).abs() / bound).max())


# ------------------------------------------------------------------------------ rows left behind past the end

@pytest.mark.parametrize("dtype,Hq,Hkv,D,B,n,n_q", [("bf16", 8, 2, 128, 2, 73, 73), ("bf16", 2, 2, 64, 1, 1, 1), ("bf16", 4, 4, 128, 3, 130, 40),
                                                    ("bf16", 8, 1, 64, 1, 383, 383), ("bf16", 2, 1, 128, 2, 64, 20), ("f32", 4, 2, 64, 2, 73, 73)])
@pytest.mark.parametrize("how", ["truncate", "reset"])
def test_prefill_over_rows_left_behind(dtype, Hq, Hkv, D, B, n, n_q, how):
    """Rows of broken drafts (NaN) that were rolled back, or left by a sequence before, share the last tile with rows that
    prefill attention reads."""
    cache = t.GuardedCache(1, Hq, Hkv, D, B, n + 70, dtype)
    cache.paint(n + 70, B)
    k, v = t.normal(1, dtype, B, n, Hkv, D), t.normal(2, dtype, B, n, Hkv, D)
    bad = torch.full((B, 70, Hkv, D), float("nan"), dtype=t.DT[dtype], device="cuda")
    if how == "truncate":
        cache.append(0, k, v)
        cache.append(0, bad, bad)
        cache.truncate(n)
    else:
        nan = torch.full((B, n + 70, Hkv, D), float("nan"), dtype=t.DT[dtype], device="cuda")
        cache.append(0, nan, nan)
        cache.reset()
        cache.append(0, k, v)
    q = t.normal(3, dtype, B, n_q, Hq, D)
    out = cache.prefill_attention(0, q)
    again = cache.prefill_attention(0, q)
    assert torch.equal(out, again)
    G = Hq // Hkv
    causal = torch.arange(n)[None, :] <= (torch.arange(n_q) + n - n_q)[:, None]
    for b in range(B):
        for h in range(Hkv):
            o, _, mass, d = ref.attend(q[b, :, h * G:(h + 1) * G], k[b, :, h], v[b, :, h], causal.cuda())
            got = out[b, :, h * G:(h + 1) * G].double()
            assert ((got - o).abs() <= (ref.weight_error(d, n) + 2.0 ** -16 + n * 2.0 ** -23) * mass + 1e-30).all()
    # the other readers of the same rows
    one = q[:, -1].contiguous()
    want = out[:, -1]
    assert (cache.decode_attention(0, one) - want).abs().max() < 1e-4
    assert cache.device_status() == 0
    cache.check_canaries()


# ----------------------------------------------------------------------------------------- views of the pool

def test_every_view_of_a_plane_is_its_callers_own():
    cache, k, _ = t.filled(4, 2, 64, 3, 20, "bf16", L=2, max_batch=5)
    shape = (5, 2, 128, 64)
    first = cache.plane(1, 0)
    first.transpose_(1, 2).unsqueeze_(0)
    again = cache.plane(1, 0)
    assert again.shape == shape and again.is_contiguous() and again is not first
    for slot in (0, 1):
        assert torch.equal(cache.plane(slot, 0)[:3, :, :20].transpose(1, 2), k)
        for kv in (0, 1):
            x = cache.plane(slot, kv)
            assert x.shape == shape and x.data_ptr() == cache.pool.data_ptr() + (2 * slot + kv) * x.numel() * 2
    for slot, kv in ((2, 0), (-1, 1), (0, 2)):
        with pytest.raises(KvsError):
            cache.plane(slot, kv)
    old, cache.pool = cache.pool, torch.zeros_like(cache.pool)          # another pool: views of that one
    assert not cache.plane(0, 0).any()
    cache.pool = old
    assert torch.equal(cache.plane(0, 0)[:3, :, :20].transpose(1, 2), k)


# ------------------------------------------------------------------------------- weighted decode in several passes

@pytest.mark.parametrize("dtype,Hq,Hkv,D,B,n,lens", [("bf16", 64, 8, 64, 5, 70001, None), ("f32", 32, 16, 64, 5, 120000, None), ("bf16", 40, 20, 64, 3, 150000, None),
                                                     ("bf16", 64, 8, 64, 5, 70001, (70001, 1, 64, 33333, 69999, 5, 40960))])
def test_weights_of_caches_whose_scores_take_several_passes(dtype, Hq, Hkv, D, B, n, lens):
    cache = t.SharedKVCache(1, Hq, Hkv, D, B, n, dtype)
    g = torch.Generator("cuda").manual_seed(n)
    k, v = (torch.randn(B, n, Hkv, D, generator=g, device="cuda", dtype=t.DT[dtype]) for _ in range(2))
    cache.append(0, k, v)
    del k, v
    if lens:
        keep = torch.arange(n, dtype=torch.int32, device="cuda").expand(B, Hkv, n).contiguous()
        cache.evict(0, keep, [[lens[(b * Hkv + h) % len(lens)] for h in range(Hkv)] for b in range(B)])
    assert B * Hq * n * 4 > 64 << 20
    before_launches = cache.stats()["attention_launches"]
    q = t.normal(3, dtype, B, Hq, D)
    total = torch.rand(B, Hkv, n + 3, device="cuda", generator=g)
    new = torch.full_like(total, 9.0)
    out = cache.decode_attention_weights(0, q, total, new)
    assert cache.stats()["attention_launches"] - before_launches > 1
    t.check_weights(cache, 0, q, total, new, out, n + 3)
    assert (new[..., n:] == 9.0).all()
    again = total.clone()
    assert torch.equal(cache.decode_attention_weights(0, q, again), out)
    for b in range(B):
        for h in range(Hkv):
            m = cache.unit_len(0, b, h)
            assert torch.equal(again[b, h, :m], new[b, h, :m]) and torch.equal(again[b, h, m:], total[b, h, m:])
    assert (out - cache.decode_attention(0, q)).abs().max() < 2e-5
    assert cache.device_status() == 0


def test_weights_in_several_passes_under_graph_replay():
    """A recorded step reserves scores for the capacity: several passes although the rows are few."""
    B, Hq, Hkv, D, n0, steps = 4, 64, 8, 64, 100, 4
    results = []
    ks, vs, qs = (t.normal(30 + i, "bf16", steps, B, 1, h, D) for i, h in enumerate((Hkv, Hkv, Hq)))
    for graph in (False, True):
        cache, _, _ = t.filled(Hq, Hkv, D, B, n0, "bf16", extra=80000, cls=t.SharedKVCache)
        total = torch.zeros(B, Hkv, n0 + 80000, device="cuda")
        k, v, q, out = ks[0].clone(), vs[0].clone(), qs[0, :, 0].clone(), torch.empty(B, Hq, D, device="cuda")

        def step():
            cache.append(0, k, v)
            cache.decode_attention_weights(0, q, total, out=out)
            if graph:
                cache.replay_advance()

        if graph:
            cache.set_option(KVS_OPT_REPLAY, 1)
            before = cache.stats()["attention_launches"]
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                step()
            assert cache.stats()["attention_launches"] - before > 1
        outs = []
        for i in range(steps):
            k.copy_(ks[i]); v.copy_(vs[i]); q.copy_(qs[i, :, 0])
            g.replay() if graph else step()
            outs.append(out.clone())
        if graph:
            cache.replay_commit(steps)
        torch.cuda.synchronize()
        assert cache.seq_len(0) == n0 + steps and cache.device_status() == 0
        results.append((total, outs))
    assert (results[0][0] - results[1][0]).abs().max() < 1e-5
    for a, b in zip(results[0][1], results[1][1]):
        assert (a - b).abs().max() < 1e-5


# --------------------------------------------------------------------------------------- evictions recorded

@pytest.mark.parametrize("B,Hkv", [(2, 2), (60, 16)])
def test_a_recorded_eviction_keeps_its_counts(B, Hkv):
    """The counts of a recorded eviction are those of the call, whatever the caller's array holds when the graph runs."""
    Hq, D, n = Hkv, 64, 150
    counts = [[1 + (37 * b + 11 * h) % n for h in range(Hkv)] for b in range(B)]
    caches = [t.filled(Hq, Hkv, D, B, n, "bf16", extra=2)[0] for _ in range(2)]
    total = torch.rand(B, Hkv, n, generator=torch.Generator().manual_seed(1)).cuda()
    q = t.normal(5, "bf16", B, Hq, D)
    want = caches[0].evict_by_weight(0, total, counts, 1)
    outs = [torch.empty(B, Hq, D, device="cuda") for _ in range(2)]
    caches[0].decode_attention(0, q, outs[0])
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = caches[1].evict_by_weight(0, total, counts, 1)
        caches[1].decode_attention(0, q, outs[1])
    junk = [(1 << 30 | i) for i in range(4096)]
    arrays = [np.full(B * Hkv, 1 << 30, dtype=np.int32) for _ in range(64)]      # what was freed is used again
    g.replay()
    torch.cuda.synchronize()
    assert len(junk) == 4096 and len(arrays) == 64
    assert torch.equal(got, want) and torch.equal(outs[0], outs[1])
    for b in range(B):
        for h in range(Hkv):
            assert caches[1].unit_len(0, b, h) == counts[b][h]
    for i in range(2):
        assert torch.equal(caches[0].plane(0, i)[:, :, :n].view(torch.int16), caches[1].plane(0, i)[:, :, :n].view(torch.int16))
    for c in caches:
        assert c.device_status() == 0
        c.check_canaries()
