"""The serving operators around the cache (rotary append, tree attention, accepted drafts, attention weights, row
selection) against their definitions in float64, at the sizes and masks where they can go wrong, and their refusals."""
import ctypes

import numpy as np
import pytest
import torch

import operators_reference as ref
from helpers import GuardedCache
from paper_2410_18517_b200 import KVS_OPT_MAX_CTAS, KVS_OPT_REPLAY, KvsError, Rotary, SharedKVCache
from paper_2410_18517_b200 import binding as kb
from paper_2410_18517_b200 import build as kbuild

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    kbuild.build()


DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def normal(seed, dtype, *shape):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(*shape, generator=g).to(DT[dtype]).cuda()


def filled(Hq, Hkv, D, B, n, dtype, extra=0, L=1, seed=1, max_batch=None, share_map=None, cls=GuardedCache):
    cache = cls(L, Hq, Hkv, D, max_batch or B, n + extra, dtype, share_map=share_map)
    if isinstance(cache, GuardedCache):
        cache.paint(n + extra, B)
    k, v = normal(seed, dtype, B, n, Hkv, D), normal(seed + 1, dtype, B, n, Hkv, D)
    for l in range(L):
        if n and (share_map is None or share_map[l] == l):
            cache.append(l, k, v)
    return cache, k, v


def rows_of(cache, layer, b, h):
    """K, V rows of a unit as they stand in the pool."""
    s, n = cache.slot_of_layer(layer), cache.unit_len(layer, b, h)
    return cache.plane(s, 0)[b, h, :n], cache.plane(s, 1)[b, h, :n]


def check_tree(cache, layer, q, words, out):
    B, T, Hq, D = q.shape
    Hkv = cache.shape[2]
    G = Hq // Hkv
    bf16 = q.dtype == torch.bfloat16
    for b in range(B):
        for h in range(Hkv):
            K, V = rows_of(cache, layer, b, h)
            sees = ref.tree_sees(words[b], K.shape[0], T).cuda()
            o, _, mass, d = ref.attend(q[b, :, h * G:(h + 1) * G], K, V, sees)
            got = out[b, :, h * G:(h + 1) * G].double()
            bound = ref.half_step(q.dtype) * o.abs() + ref.weight_error(d, K.shape[0], bf16) * mass * (1 + 2 ** -7) + 1e-30
            assert torch.isfinite(got).all()
            bad = (got - o).abs() > bound
            assert not bad.any(), (b, h, float(((got - o).abs() / bound).max()))


# ------------------------------------------------------------------------------------------- tree attention

TREE = [
    # dtype, Hq, Hkv, D, B, n, n_t
    ("bf16", 4, 4, 128, 2, 1, 1), ("bf16", 8, 2, 128, 2, 5, 5), ("bf16", 8, 2, 128, 1, 64, 64), ("bf16", 8, 2, 128, 1, 65, 64),
    ("bf16", 8, 1, 128, 1, 700, 64), ("bf16", 8, 1, 64, 3, 129, 33), ("bf16", 7, 1, 128, 2, 300, 19), ("bf16", 10, 2, 64, 2, 191, 26),
    ("bf16", 6, 2, 128, 1, 4001, 43), ("bf16", 6, 1, 128, 1, 1000, 64), ("bf16", 2, 2, 64, 5, 63, 1), ("bf16", 2, 1, 128, 40, 127, 13),
    ("bf16", 32, 8, 128, 1, 2049, 17), ("bf16", 16, 16, 64, 20, 128, 2), ("bf16", 5, 5, 128, 1, 9000, 64),
    ("f32", 4, 4, 64, 2, 1, 1), ("f32", 4, 4, 64, 2, 135, 7), ("f32", 8, 2, 128, 1, 65, 64), ("f32", 8, 1, 128, 1, 2000, 64),
    ("f32", 4, 2, 64, 30, 191, 11), ("f32", 8, 8, 128, 1, 64, 3),
]


@pytest.mark.parametrize("dtype,Hq,Hkv,D,B,n,n_t", TREE)
def test_tree_attention_random_trees(dtype, Hq, Hkv, D, B, n, n_t):
    cache, _, _ = filled(Hq, Hkv, D, B, n, dtype, extra=3)
    rng = np.random.default_rng(n + n_t)
    words = [ref.random_tree(rng, n_t) for _ in range(B)]
    q = normal(7, dtype, B, n_t, Hq, D)
    mask = torch.tensor([ref.to_int64(w) for w in words], dtype=torch.int64).cuda()
    out = cache.tree_attention(0, q, mask)
    check_tree(cache, 0, q, words, out)
    assert torch.equal(out, cache.tree_attention(0, q, mask))          # the same bits every time
    chain = cache.tree_attention(0, q)
    check_tree(cache, 0, q, [ref.random_tree(rng, n_t, chain=True) for _ in range(B)], chain)
    assert cache.device_status() == 0
    cache.check_canaries()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("ctas", [1, 2, 3, 7, 50])
def test_tree_attention_any_split(dtype, ctas):
    """However the key tiles are dealt out, pieces of every kind included."""
    cache, _, _ = filled(8, 2, 128, 3, 1000, dtype)
    cache.set_option(KVS_OPT_MAX_CTAS, ctas)
    rng = np.random.default_rng(0)
    words = [ref.random_tree(rng, 40) for _ in range(3)]
    q = normal(8, dtype, 3, 40, 8, 128)
    out = cache.tree_attention(0, q, torch.tensor([ref.to_int64(w) for w in words]).cuda())
    check_tree(cache, 0, q, words, out)
    cache.check_canaries()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_tree_rows_that_see_nothing_are_zero(dtype):
    n_t = 9
    cache, _, _ = filled(4, 2, 64, 2, n_t, dtype)                       # no context at all
    words = [[0] * n_t, [0, 1, 0, 1 << 8, 0, 0, 1 << 5, 0, 0]]
    q = normal(3, dtype, 2, n_t, 4, 64)
    out = cache.tree_attention(0, q, torch.tensor(words).cuda())
    assert not out[0].any() and not out[1, 0].any() and out[1, 1].any()
    check_tree(cache, 0, q, words, out)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [6, 70, 131])
@pytest.mark.parametrize("junk", [float("nan"), float("inf"), -float("inf"), "lowest"])
def test_masked_drafts_may_hold_anything(dtype, n, junk):
    """Padding tokens (seen by nobody), and a broken token that some see and others do not; their queries too."""
    n_t, Hq, Hkv, D = 6, 4, 2, 64
    if junk == "lowest":
        junk = torch.finfo(DT[dtype]).min
    cache = GuardedCache(1, Hq, Hkv, D, 1, n + 5, dtype)
    cache.paint(n + 5, 1)
    k, v = normal(1, dtype, 1, n, Hkv, D), normal(2, dtype, 1, n, Hkv, D)
    k[:, -2:] = junk
    v[:, -2:] = junk
    v[:, n - n_t + 1, 1, 3] = junk                   # draft 1, kv-head 1, column 3
    cache.append(0, k, v)
    q = normal(3, dtype, 1, n_t, Hq, D)
    q[:, -1] = junk
    words = [1, 2, 4 | 1, 8, 8 | 4 | 1, 0]           # drafts 4 and 5 are seen by nobody, draft 1 by itself
    out = cache.tree_attention(0, q, torch.tensor([words]).cuda())
    clean = [0, 2, 3, 4]
    for h in range(Hkv):
        K, V = rows_of(cache, 0, 0, h)
        sees = ref.tree_sees(words, n, n_t).cuda()[clean]
        V = torch.where(sees.any(0)[:, None], V.double(), 0.0)
        o, _, mass, d = ref.attend(q[0, clean, 2 * h:2 * h + 2], torch.nan_to_num(K.double(), 0, 0, 0), V, sees)
        got = out[0, clean, 2 * h:2 * h + 2].double()
        assert torch.isfinite(got).all()
        bound = ref.half_step(q.dtype) * o.abs() + ref.weight_error(d, n, dtype == "bf16") * mass * (1 + 2 ** -7)
        assert ((got - o).abs() <= bound).all()
    # the broken value shows where it is seen, and only there
    broken = out[0, 1, 2:, 3].float()
    if abs(junk) == float("inf"):
        assert (broken == junk).all() or broken.isnan().all()
    elif junk != junk:
        assert broken.isnan().all()
    assert torch.isfinite(out[0, 1, :2].float()).all() and torch.isfinite(out[0, 1, 2:, :3].float()).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_stale_rows_behind_the_drafts(dtype):
    """Rows left behind by a longer, broken step lie in the same tile as the last draft."""
    cache, k, v = filled(4, 2, 128, 2, 40, dtype, extra=30)
    bad = torch.full((2, 20, 2, 128), float("nan"), dtype=DT[dtype], device="cuda")
    cache.append(0, bad, bad)
    cache.truncate(40)
    rng = np.random.default_rng(5)
    words = [ref.random_tree(rng, 5) for _ in range(2)]
    q = normal(9, dtype, 2, 5, 4, 128)
    check_tree(cache, 0, q, words, cache.tree_attention(0, q, torch.tensor(words).cuda()))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_tree_extreme_scores(dtype):
    """Scores that grow along the keys move the running maximum again and again; large ones saturate to one key."""
    n, n_t, D = 700, 12, 128
    cache = GuardedCache(1, 8, 2, D, 1, n, dtype)
    k, v = normal(1, dtype, 1, n, 2, D), normal(2, dtype, 1, n, 2, D)
    k = (k.float() * torch.linspace(0.05, 6, n, device="cuda")[None, :, None, None]).to(DT[dtype])
    cache.append(0, k, v)
    q = normal(3, dtype, 1, n_t, 8, D)
    words = [ref.random_tree(np.random.default_rng(1), n_t)]
    for scale in (1.0, 0.0, 4.0):
        qs = (q * scale).contiguous()
        check_tree(cache, 0, qs, words, cache.tree_attention(0, qs, torch.tensor(words).cuda()))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_tree_on_ragged_units_and_smaller_batch(dtype):
    B, Hkv, n, n_t = 3, 2, 200, 10
    cache, _, _ = filled(8, Hkv, 128, B, n, dtype, extra=60, max_batch=5)
    keep = torch.zeros(B, Hkv, n, dtype=torch.int32)
    counts = [[1, 64], [199, 63], [65, 130]]
    for b in range(B):
        for h in range(Hkv):
            rows = np.sort(np.random.default_rng(b * 2 + h).choice(n, counts[b][h], replace=False))
            keep[b, h, : len(rows)] = torch.from_numpy(rows)
    cache.evict(0, keep.cuda(), counts)
    cache.append(0, normal(4, dtype, B, n_t, Hkv, 128), normal(5, dtype, B, n_t, Hkv, 128))
    rng = np.random.default_rng(2)
    words = [ref.random_tree(rng, n_t) for _ in range(B)]
    mask = torch.tensor(words).cuda()
    q = normal(6, dtype, B, n_t, 8, 128)
    for batch in (3, 2, 1):
        out = cache.tree_attention(0, q[:batch].contiguous(), mask[:batch].contiguous())
        check_tree(cache, 0, q[:batch], words[:batch], out)
    for ctas in (1, 2, 5):
        cache.set_option(KVS_OPT_MAX_CTAS, ctas)
        check_tree(cache, 0, q, words, cache.tree_attention(0, q, mask))
    cache.check_canaries()


@pytest.mark.parametrize("Hq,Hkv,D,B,n,n_t", [(32, 32, 128, 8, 4112, 16), (32, 8, 128, 4, 8224, 32), (24, 8, 64, 3, 700, 20)])
def test_tree_many_calls_in_flight_give_the_same_bits(Hq, Hkv, D, B, n, n_t):
    """Two caches used in turn without a wait: the last tiles' clean-up must not meet a copy or a product in flight."""
    cases = []
    for i in range(2):
        cache, _, _ = filled(Hq, Hkv, D, B, n, "bf16", seed=10 * i + 1, cls=SharedKVCache)
        words = [ref.random_tree(np.random.default_rng(b + i), n_t) for b in range(B)]
        words = [[0 if t > 3 * b + 2 else w & ((8 << 3 * b) - 1) for t, w in enumerate(row)] for b, row in enumerate(words)]
        cases.append((cache, normal(5 + i, "bf16", B, n_t, Hq, D), torch.tensor([ref.to_int64(w) for w in words]).cuda()))
    first = [c.tree_attention(0, q, m) for c, q, m in cases]
    outs = [[c.tree_attention(0, q, m) for c, q, m in cases] for _ in range(40)]
    for pair in outs:
        for a, b in zip(pair, first):
            assert torch.equal(a, b)
    (cache, q, m), out = cases[0], first[0]
    check_tree(cache, 0, q[:1], m[:1].tolist(), out[:1])


def test_tree_bits_behind_the_last_draft_are_ignored_and_out_rows_stay():
    cache, _, _ = filled(8, 2, 128, 2, 90, "bf16")
    words = [ref.random_tree(np.random.default_rng(b), 11) for b in range(2)]
    q = normal(3, "bf16", 2, 11, 8, 128)
    clean = cache.tree_attention(0, q, torch.tensor(words).cuda())
    big = torch.full((4, 11, 8, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    noisy = torch.tensor([[w - (1 << 63) | 1 << 40 for w in row] for row in words]).cuda()
    cache.tree_attention(0, q, noisy, out=big[1:3])
    assert torch.equal(big[1:3], clean) and (big[0] == 7).all() and (big[3] == 7).all()


def test_tree_on_a_sharing_layer_and_with_a_scale():
    cache = SharedKVCache(3, 8, 2, 64, 2, 100, "bf16", share_map=[0, 1, 0], softmax_scale=0.05)
    k, v = normal(1, "bf16", 2, 90, 2, 64), normal(2, "bf16", 2, 90, 2, 64)
    cache.append(0, k, v)
    cache.append(1, v, k)
    q = normal(3, "bf16", 2, 8, 8, 64)
    words = [ref.random_tree(np.random.default_rng(b), 8) for b in range(2)]
    mask = torch.tensor(words).cuda()
    assert torch.equal(cache.tree_attention(0, q, mask), cache.tree_attention(2, q, mask))
    assert not torch.equal(cache.tree_attention(0, q, mask), cache.tree_attention(1, q, mask))
    out = cache.tree_attention(2, q, mask)
    want = torch.einsum("tgd,nd->tgn", q[0, :, :4].double(), k[0, :, 0].double()) * 0.05
    want = want.masked_fill(~ref.tree_sees(words[0], 90, 8).cuda()[:, None], float("-inf")).softmax(-1) @ v[0, :, 0].double()
    assert (out[0, :, :4].double() - want).abs().max() <= 2.0 ** -7 * v.abs().max().item()


def test_one_draft_is_a_decode_step():
    cache, _, _ = filled(32, 8, 128, 4, 777, "bf16")
    q = normal(3, "bf16", 4, 1, 32, 128)
    a, b = cache.tree_attention(0, q).double()[:, 0], cache.decode_attention(0, q[:, 0].contiguous()).double()
    assert (a - b).abs().max() <= 2.0 ** -7 * b.abs().max()


# ---------------------------------------------------------------------------------------- accepted drafts

@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 128)])
@pytest.mark.parametrize("counts", [[3, 3, 3], [0, 0, 0], [7, 7, 7], [1, 0, 5]])
def test_accept_draft(dtype, D, counts):
    B, Hkv, n, n_t = 3, 2, 61, 7
    cache, k, v = filled(4, Hkv, D, B, n, dtype, extra=n_t + 2, L=3, share_map=[0, 1, 0])
    dk, dv = normal(11, dtype, B, n_t, Hkv, D), normal(12, dtype, B, n_t, Hkv, D)
    cache.append(0, dk, dv)
    cache.append(1, dv, dk)
    rng = np.random.default_rng(3)
    path = torch.full((B, 9), -5, dtype=torch.int32)
    for b in range(B):
        path[b, : counts[b]] = torch.from_numpy(np.sort(rng.choice(n_t, counts[b], replace=False)).astype(np.int32))
    cache.accept_draft(path.cuda(), counts, n_t)
    for layer, (xk, xv) in ((0, (dk, dv)), (1, (dv, dk)), (2, (dk, dv))):
        for b in range(B):
            at = path[b, : counts[b]].long().cuda()
            for h in range(Hkv):
                assert cache.unit_len(layer, b, h) == n + counts[b]
                K, V = rows_of(cache, layer, b, h)
                assert torch.equal(K[:n], k[b, :, h]) and torch.equal(K[n:], xk[b, at, h])
                assert torch.equal(V[:n], v[b, :, h]) and torch.equal(V[n:], xv[b, at, h])
    assert cache.device_status() == 0
    # the slot is usable at once: a decode step and a step of drafts on top
    q = normal(13, dtype, B, 4, D)
    cache.append(0, dk[:, :1].contiguous(), dv[:, :1].contiguous())
    out = cache.decode_attention(0, q)
    for b in range(B):
        for h in range(Hkv):
            K, V = rows_of(cache, 0, b, h)
            assert K.shape[0] == n + counts[b] + 1 and torch.equal(K[-1], dk[b, 0, h])
            o, _, _, _ = ref.attend(q[b, None, 2 * h:2 * h + 2], K, V)
            assert (out[b, 2 * h:2 * h + 2].double() - o[0]).abs().max() < 2e-3
    cache.check_canaries()


def test_accept_everything_rejected_on_an_empty_context():
    cache, _, _ = filled(4, 2, 64, 2, 0, "bf16", extra=8)
    d = normal(1, "bf16", 2, 4, 2, 64)
    cache.append(0, d, d)
    cache.accept_draft(torch.zeros(2, 1, dtype=torch.int32).cuda(), [0, 0], 4)
    assert cache.seq_len(0) == 0
    cache.append(0, d[:1].contiguous(), d[:1].contiguous())        # even another batch may follow
    assert cache.seq_len(0) == 4


def test_accept_twice_on_ragged_slots():
    B, Hkv, n_t = 2, 2, 5
    cache, k, _ = filled(4, Hkv, 64, B, 30, "bf16", extra=20)
    want = [[k[b, :, h] for h in range(Hkv)] for b in range(B)]
    for step, counts in enumerate(([2, 4], [5, 1], [3, 3])):
        d = normal(20 + step, "bf16", B, n_t, Hkv, 64)
        cache.append(0, d, d)
        path = torch.stack([torch.sort(torch.randperm(n_t, generator=torch.Generator().manual_seed(step * 2 + b))).values for b in range(B)]).int()
        for b in range(B):
            path[b, : counts[b]] = torch.arange(n_t - counts[b], n_t)
        cache.accept_draft(path.cuda(), counts, n_t)
        for b in range(B):
            for h in range(Hkv):
                want[b][h] = torch.cat((want[b][h], d[b, n_t - counts[b]:, h]))
                K, V = rows_of(cache, 0, b, h)
                assert torch.equal(K, want[b][h])
    with pytest.raises(KvsError):
        cache.truncate(3)


def test_accept_reports_a_bad_path():
    cache, _, _ = filled(4, 2, 64, 1, 10, "bf16", extra=8)
    d = normal(1, "bf16", 1, 4, 2, 64)
    for path in ([2, 1, 3], [0, 1, 4], [0, 0, 2], [-1, 2, 3]):
        cache.truncate(10)
        cache.append(0, d, d)
        cache.accept_draft(torch.tensor([path], dtype=torch.int32).cuda(), [3], 4)
        assert cache.device_status() == kb.KVS_ERR_INVALID_ARG
        cache.clear_device_status()
        assert cache.device_status() == 0
    cache.check_canaries()


@pytest.mark.parametrize("how", ["accept", "truncate"])
@pytest.mark.parametrize("dtype,Hq", [("bf16", 8), ("bf16", 2), ("f32", 8)])
def test_broken_drafts_leave_no_trace(how, dtype, Hq):
    """Padding drafts whose rows are NaN, rejected or rolled back: the rows past the end share the last tile with rows that
    decode attention reads."""
    cache, _, _ = filled(Hq, 2, 128, 2, 70, dtype, extra=12)
    good = normal(5, dtype, 2, 3, 2, 128)
    bad = torch.full((2, 6, 2, 128), float("nan"), dtype=DT[dtype], device="cuda")
    rows = torch.cat((good, bad), 1)
    cache.append(0, rows, rows)
    if how == "accept":
        cache.accept_draft(torch.arange(3).int().expand(2, 3).contiguous().cuda(), [3, 3], 9)
        assert torch.isfinite(cache.plane(0, 0)[:2, :, :80].float()).all() and torch.isfinite(cache.plane(0, 1)[:2, :, :80].float()).all()
    else:
        cache.truncate(73)
    q = normal(6, dtype, 2, Hq, 128)
    total = torch.zeros(2, 2, 82, device="cuda")
    out = cache.decode_attention_weights(0, q, total)
    check_weights(cache, 0, q, torch.zeros_like(total), total, out, 82)
    assert torch.allclose(out, cache.decode_attention(0, q), rtol=0, atol=2e-5)
    check_tree(cache, 0, q[:, None].contiguous(), [[1]] * 2, cache.tree_attention(0, q[:, None].contiguous()))


# ------------------------------------------------------------------------------------------ rotary append

def check_rotary(got, x, w, pos, inv_freq, interleaved, eps):
    want, mag = ref.norm_rope(x, w, pos, inv_freq, interleaved, eps)
    # norm: the sum of squares and its root, the mean's and the weight's products (D + 8 roundings at most);
    # rotation: cos and sin are off by 2^-22 (the fp32 remainder of the turn, times pi, and the function)
    D = x.shape[-1]
    bound = ref.half_step(x.dtype) * want.abs() + ((D / 2 + 8) * ref.U + 2.0 ** -21) * mag * (1 + 2.0 ** -7) + 1e-37
    err = (got.double() - want).abs()
    assert (err <= bound).all(), float((err / bound).max())


ROT = [
    # dtype, Hq, Hkv, D, B, n0, n_new, rotary_dim, interleaved, norm, fused, first position
    ("bf16", 32, 8, 128, 3, 5, 1, 128, False, True, True, 5), ("bf16", 40, 40, 128, 2, 0, 33, 128, False, True, False, 0),
    ("bf16", 7, 1, 128, 2, 3, 17, 96, False, False, True, 1000000), ("bf16", 4, 2, 64, 1, 100, 130, 64, True, True, True, 2147483000),
    ("bf16", 6, 2, 64, 3, 9, 2, 16, True, False, False, -40), ("bf16", 2, 2, 64, 1, 0, 1, 0, False, True, False, 0),
    ("bf16", 5, 5, 64, 2, 1, 3, 32, False, True, True, 131071), ("f32", 4, 4, 64, 2, 128, 7, 64, False, True, True, 128),
    ("f32", 8, 1, 128, 1, 0, 65, 128, True, True, False, 999999), ("f32", 4, 2, 128, 3, 17, 1, 48, False, False, True, 4095),
]


@pytest.mark.parametrize("dtype,Hq,Hkv,D,B,n0,n_new,dim,inter,norm,fused,first", ROT)
def test_append_rotary(dtype, Hq, Hkv, D, B, n0, n_new, dim, inter, norm, fused, first):
    cache, k0, v0 = filled(Hq, Hkv, D, B, n0, dtype, extra=n_new + 1)
    if fused:
        x = normal(5, dtype, B, n_new, Hq + 2 * Hkv, D)
        q, k, v = x[:, :, :Hq], x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:]
    else:
        q, k, v = (normal(5 + i, dtype, B, n_new, h, D) for i, h in enumerate((Hq, Hkv, Hkv)))
    pos = (first + torch.arange(n_new)[None] + 3 * torch.arange(B)[:, None]).int().cuda()
    qw, kw = (normal(8, dtype, D), normal(9, dtype, D)) if norm else (None, None)
    freq = [10000.0 ** (-2 * i / dim) for i in range(dim // 2)]
    got = cache.append_rotary(0, q, k, v, pos, Rotary(freq, inter), qw, kw, eps=1e-5)
    check_rotary(got, q, qw, pos, freq, inter, 1e-5)
    assert cache.seq_len(0) == n0 + n_new
    K, V = cache.plane(0, 0)[:B, :, n0:n0 + n_new].transpose(1, 2), cache.plane(0, 1)[:B, :, n0:n0 + n_new].transpose(1, 2)
    check_rotary(K, k, kw, pos, freq, inter, 1e-5)
    assert torch.equal(V, v)
    if n0:
        assert torch.equal(cache.plane(0, 0)[:B, :, :n0].transpose(1, 2), k0)
    assert cache.device_status() == 0
    cache.check_canaries()


# long prompts: token rows of 8 KB and more, several hundred tokens
ROT_LONG = [
    ("bf16", 32, 8, 128, 2, 3, 1801, 128, False, True, True, 0), ("bf16", 40, 40, 128, 1, 1, 900, 128, True, True, False, 7),
    ("bf16", 49, 7, 64, 1, 0, 1333, 32, True, True, True, 0), ("f32", 14, 7, 128, 3, 5, 700, 96, False, False, True, 100000),
    ("f32", 8, 8, 128, 1, 0, 1000, 0, False, True, False, 0), ("bf16", 128, 16, 128, 1, 0, 907, 128, False, True, True, 0),
    ("bf16", 128, 128, 128, 1, 0, 901, 128, False, True, True, 0),
]


@pytest.mark.parametrize("dtype,Hq,Hkv,D,B,n0,n_new,dim,inter,norm,fused,first", ROT_LONG)
def test_append_rotary_of_long_prompts(dtype, Hq, Hkv, D, B, n0, n_new, dim, inter, norm, fused, first):
    test_append_rotary(dtype, Hq, Hkv, D, B, n0, n_new, dim, inter, norm, fused, first)


def test_append_rotary_of_long_prompts_in_place_on_sharing_layers_and_ragged_slots():
    B, n, Hq, Hkv, D = 2, 611, 32, 4, 128
    freq = [10000.0 ** (-i / 64) for i in range(64)]
    pos = (torch.arange(n)[None] + 11 * torch.arange(B)[:, None]).int().cuda()
    cache, k0, v0 = filled(Hq, Hkv, D, B, 20, "bf16", extra=n + 2, L=2, share_map=[0, 0])
    keep = torch.arange(20, dtype=torch.int32).expand(B, Hkv, 20).contiguous().cuda()
    kept = [[3, 20, 1, 9], [7, 11, 20, 2]]
    cache.evict(0, keep, kept)
    q, k, v = (normal(i, "bf16", B, n, h, D) for i, h in ((3, Hq), (4, Hkv), (5, Hkv)))
    w = normal(6, "bf16", D)
    x = q.clone()
    cache.append_rotary(0, x, k, v, pos, Rotary(freq), w, None, out=x)
    check_rotary(x, q, w, pos, freq, False, 1e-6)
    assert torch.equal(cache.append_rotary(1, q, None, None, pos, Rotary(freq), w), x)
    for b in range(B):
        for h in range(Hkv):
            K, V = rows_of(cache, 0, b, h)
            m = kept[b][h]
            assert K.shape[0] == m + n and torch.equal(V[m:], v[b, :, h]) and torch.equal(K[:m], k0[b, :m, h])
            check_rotary(K[None, m:, None], k[b:b + 1, :, h:h + 1], None, pos[b:b + 1], freq, False, 1e-6)
    assert cache.device_status() == 0
    cache.check_canaries()


def test_append_rotary_in_place_and_one_weight_only():
    cache, _, _ = filled(8, 2, 128, 2, 4, "bf16", extra=8)
    q, k, v = (normal(i, "bf16", 2, 3, h, 128) for i, h in ((1, 8), (2, 2), (3, 2)))
    pos = torch.arange(3).int().expand(2, 3).contiguous().cuda()
    rot = Rotary.from_theta(128)
    want = cache.append_rotary(0, q, k, v, pos, rot, None, normal(4, "bf16", 128))
    cache.truncate(4)
    x = q.clone()
    assert cache.append_rotary(0, x, k, v, pos, rot, None, normal(4, "bf16", 128), out=x) is x
    assert torch.equal(x, want)
    check_rotary(x, q, None, pos, [10000.0 ** (-i / 64) for i in range(64)], False, 1e-6)


def test_append_rotary_zero_rows_and_bits_of_v():
    """A zero head stays zero (the mean square is zero); the values of v, NaN included, are copied bit for bit."""
    cache, _, _ = filled(4, 4, 64, 1, 0, "bf16", extra=4)
    z = torch.zeros(1, 2, 4, 64, dtype=torch.bfloat16, device="cuda")
    v = torch.arange(512, dtype=torch.int32).add(0x7F00).to(torch.int16).cuda().view(torch.bfloat16).view(1, 2, 4, 64)
    pos = torch.tensor([[3, 9]], dtype=torch.int32).cuda()
    w = torch.ones(64, dtype=torch.bfloat16, device="cuda")
    q = cache.append_rotary(0, z, z, v, pos, Rotary.from_theta(64), w, w)
    assert not q.any() and not cache.plane(0, 0)[0, :, :2].any()
    assert torch.equal(cache.plane(0, 1)[0, :, :2].transpose(0, 1).view(torch.int16), v[0].view(torch.int16))


def test_append_rotary_on_sharing_layers_and_ragged_slots():
    cache = SharedKVCache(2, 8, 2, 64, 2, 50, "bf16", share_map=[0, 0])
    k, v = normal(1, "bf16", 2, 20, 2, 64), normal(2, "bf16", 2, 20, 2, 64)
    cache.append(0, k, v)
    keep = torch.arange(20, dtype=torch.int32).expand(2, 2, 20).contiguous().cuda()
    cache.evict(0, keep, [[3, 20], [7, 11]])
    q, k1, v1 = (normal(i, "bf16", 2, 4, h, 64) for i, h in ((3, 8), (4, 2), (5, 2)))
    pos = torch.arange(20, 24).int().expand(2, 4).contiguous().cuda()
    freq = [10000.0 ** (-i / 32) for i in range(32)]
    a = cache.append_rotary(0, q, k1, v1, pos, Rotary(freq))
    assert [cache.unit_len(0, b, h) for b in range(2) for h in range(2)] == [7, 24, 11, 15]
    b_ = cache.append_rotary(1, q, None, None, pos, Rotary(freq))
    assert torch.equal(a, b_) and cache.unit_len(1, 0, 0) == 7
    for b in range(2):
        for h in range(2):
            K, V = rows_of(cache, 0, b, h)
            check_rotary(K[None, -4:, None], k1[b:b + 1, :, h:h + 1], None, pos[b:b + 1], freq, False, 1e-6)
            assert torch.equal(V[-4:], v1[b, :, h])


# ----------------------------------------------------------------------------- attention weights and selection

WEIGHTS = [("bf16", 4, 4, 128, 2, 1), ("bf16", 8, 2, 128, 3, 65), ("bf16", 8, 1, 64, 1, 3001), ("bf16", 7, 1, 128, 2, 500),
           ("bf16", 40, 40, 128, 4, 257), ("bf16", 16, 8, 64, 20, 127), ("bf16", 32, 8, 128, 1, 5000), ("bf16", 32, 4, 128, 40, 1025),
           ("f32", 4, 4, 64, 2, 129), ("f32", 8, 1, 128, 1, 900), ("f32", 8, 2, 64, 1, 1), ("f32", 4, 2, 128, 90, 33)]


def check_weights(cache, layer, q, before, after, out, n_stride):
    B, Hq, D = q.shape
    Hkv = cache.shape[2]
    G = Hq // Hkv
    for b in range(B):
        for h in range(Hkv):
            K, V = rows_of(cache, layer, b, h)
            n = K.shape[0]
            o, p, mass, d = ref.attend(q[b, None, h * G:(h + 1) * G], K, V)
            rel = ref.weight_error(d, n)
            # the third bf16 term of a weight leaves 2^-24 of it, sums in the tensor cores truncate: 2^-23 a step
            got = out[b, h * G:(h + 1) * G].double()
            assert ((got - o[0]).abs() <= (rel + n * 2.0 ** -23) * mass[0] + 1e-30).all()
            w = p[0].sum(0)
            start = before[b, h, :n].double() if before is not None else 0.0
            want = start + w
            err = (after[b, h, :n].double() - want).abs()
            assert (err <= (rel + G * ref.U) * w + ref.U * want.abs() + 1e-30).all(), float((err / want).max())


@pytest.mark.parametrize("dtype,Hq,Hkv,D,B,n", WEIGHTS)
def test_decode_attention_weights(dtype, Hq, Hkv, D, B, n):
    cache, _, _ = filled(Hq, Hkv, D, B, n, dtype, extra=2)
    q = normal(3, dtype, B, Hq, D)
    total = torch.rand(B, Hkv, n + 5, generator=torch.Generator().manual_seed(1)).cuda()
    new = torch.full_like(total, 9.0)
    out = cache.decode_attention_weights(0, q, total, new)
    check_weights(cache, 0, q, total, new, out, n + 5)
    assert (new[..., n:] == 9.0).all()                                   # rows behind the last stay as they were
    assert torch.allclose(out, cache.decode_attention(0, q), rtol=0, atol=2e-5)
    again = total.clone()
    cache.decode_attention_weights(0, q, again)                          # in place, the same bits
    assert torch.equal(again[..., :n], new[..., :n]) and torch.equal(again[..., n:], total[..., n:])
    fresh = torch.empty_like(total)
    cache.decode_attention_weights(0, q, None, fresh)
    check_weights(cache, 0, q, None, fresh, out, n + 5)
    assert torch.allclose(fresh[..., :n].sum(-1), torch.full((B, Hkv), float(Hq // Hkv), device="cuda"), rtol=1e-5)
    assert cache.device_status() == 0
    cache.check_canaries()


@pytest.mark.parametrize("dtype,kernel", [("bf16", 1), ("bf16", 2), ("f32", 1)])
@pytest.mark.parametrize("ctas", [0, 1, 3, 20])
def test_decode_attention_weights_any_split_and_kernel(dtype, kernel, ctas):
    cache, _, _ = filled(8, 2, 128, 3, 1500, dtype)
    cache.set_option(1, kernel)
    cache.set_option(KVS_OPT_MAX_CTAS, ctas)
    q = normal(3, dtype, 3, 8, 128)
    total = torch.empty(3, 2, 1500, device="cuda")
    out = cache.decode_attention_weights(0, q, None, total)
    check_weights(cache, 0, q, None, total, out, 1500)


def test_weights_of_ragged_units():
    B, Hkv = 2, 2
    for dtype in ("bf16", "f32"):
        cache, _, _ = filled(8, Hkv, 64, B, 300, dtype, extra=4)
        keep = torch.arange(300, dtype=torch.int32).expand(B, Hkv, 300).contiguous().cuda()
        cache.evict(0, keep, [[1, 300], [140, 64]])
        q = normal(3, dtype, B, 8, 64)
        total = torch.full((B, Hkv, 300), 0.5, device="cuda")
        new = torch.full((B, Hkv, 300), -1.0, device="cuda")
        out = cache.decode_attention_weights(0, q, total, new)
        check_weights(cache, 0, q, total, new, out, 300)
        for b, h, n in ((0, 0, 1), (1, 0, 140), (1, 1, 64)):
            assert (new[b, h, n:] == -1.0).all()


def test_weights_under_graph_replay():
    """A recorded step (append, weights, advance) replayed: totals grow by one row per replay, like the eager steps."""
    B, Hq, Hkv, D, n0, steps = 2, 8, 2, 128, 61, 7
    ks, vs, qs = (normal(30 + i, "bf16", steps + 1, B, 1, h, D) for i, h in enumerate((Hkv, Hkv, Hq)))
    results = []
    for graph in (False, True):
        cache, _, _ = filled(Hq, Hkv, D, B, n0, "bf16", extra=steps + 2)
        cap = n0 + steps + 2
        total = torch.zeros(B, Hkv, cap, device="cuda")
        outs = []
        if not graph:
            for t in range(steps):
                cache.append(0, ks[t], vs[t])
                outs.append(cache.decode_attention_weights(0, qs[t, :, 0].contiguous(), total))
        else:
            cache.set_option(KVS_OPT_REPLAY, 1)
            k, v, q, out = ks[0].clone(), vs[0].clone(), qs[0, :, 0].clone(), torch.empty(B, Hq, D, device="cuda")
            s = torch.cuda.Stream()
            s.wait_stream(torch.cuda.current_stream())
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=s):
                cache.append(0, k, v)
                cache.decode_attention_weights(0, q, total, out=out)
                cache.replay_advance()
            for t in range(steps):
                k.copy_(ks[t]); v.copy_(vs[t]); q.copy_(qs[t, :, 0])
                g.replay()
                outs.append(out.clone())
            cache.replay_commit(steps)
        torch.cuda.synchronize()
        assert cache.seq_len(0) == n0 + steps and cache.device_status() == 0
        results.append((total, outs))
    assert (results[0][0] - results[1][0]).abs().max() < 1e-5
    for a, b in zip(results[0][1], results[1][1]):
        assert (a - b).abs().max() < 1e-5


@pytest.mark.parametrize("dtype,Hq,Hkv,D", [("bf16", 32, 8, 128), ("bf16", 24, 8, 64), ("bf16", 4, 4, 128), ("f32", 8, 2, 64)])
def test_weights_pass_does_not_drift_over_long_shares(dtype, Hq, Hkv, D):
    """16000 rows of a sequence in three blocks: thousands of steps into one accumulator."""
    n, B = 16000, 1
    cache, k, v = filled(Hq, Hkv, D, B, n, dtype, cls=SharedKVCache)
    cache.set_option(KVS_OPT_MAX_CTAS, 3)
    q = normal(9, dtype, B, Hq, D)
    total = torch.zeros(B, Hkv, n, device="cuda")
    out = cache.decode_attention_weights(0, q, total).double()
    s = torch.einsum("bhgd,bnhd->bhgn", q.double().view(B, Hkv, Hq // Hkv, D), k.double()) / D ** 0.5
    want = torch.einsum("bhgn,bnhd->bhgd", torch.softmax(s, -1), v.double()).reshape(out.shape)
    # A warp adds its quarter of the rows: N = 250 blocks of 16 (or 4000 rows one by one).  Rounded to nearest, independent, the
    # sums walk sqrt(N) 2^-25 <= 1.9e-6 of the result; cut off towards zero they drift by N 2^-25.
    assert (out - want).norm() <= 2e-6 * want.norm()


def test_rotary_append_under_graph_replay():
    B, Hq, Hkv, D, n0, steps = 2, 4, 2, 64, 10, 5
    x = normal(1, "bf16", steps, B, 1, Hq + 2 * Hkv, D)
    rot, w = Rotary.from_theta(D), normal(2, "bf16", D)
    planes = []
    for graph in (False, True):
        cache, _, _ = filled(Hq, Hkv, D, B, n0, "bf16", extra=steps)
        pos = torch.full((B, 1), n0, dtype=torch.int32, device="cuda")
        cur, out = x[0].clone(), torch.empty(B, 1, Hq, D, dtype=torch.bfloat16, device="cuda")
        att = torch.empty(B, Hq, D, device="cuda")

        def step():
            cache.append_rotary(0, cur[:, :, :Hq], cur[:, :, Hq:Hq + Hkv], cur[:, :, Hq + Hkv:], pos, rot, w, w, out=out)
            cache.decode_attention(0, out[:, 0], att)
            cache.replay_advance() if graph else None
            pos.add_(1)

        outs = []
        if graph:
            cache.set_option(KVS_OPT_REPLAY, 1)
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                step()
        for t in range(steps):
            cur.copy_(x[t])
            g.replay() if graph else step()
            outs.append((out.clone(), att.clone()))
        if graph:
            g.replay()                                   # one past the capacity: nothing is appended, and it is reported
            torch.cuda.synchronize()
            assert cache.device_status() == kb.KVS_ERR_CAPACITY
            cache.clear_device_status()
            cache.replay_commit(steps)
        torch.cuda.synchronize()
        cache.check_canaries()
        planes.append((cache.plane(0, 0).clone(), cache.plane(0, 1).clone(), outs))
    assert torch.equal(planes[0][0], planes[1][0]) and torch.equal(planes[0][1], planes[1][1])
    for (a, s), (b, t) in zip(planes[0][2], planes[1][2]):
        assert torch.equal(a, b) and (s - t).abs().max() < 1e-5


def _select_case(cache, total, n_keep, n_recent):
    B, Hkv = total.shape[:2]
    stride = max(max(r) for r in n_keep) + 3
    keep = torch.full((B, Hkv, stride), -7, dtype=torch.int32, device="cuda")
    kept = torch.full((B, Hkv, stride), -7.0, device="cuda")
    cache.select_rows(0, total, n_keep, n_recent, keep, kept)
    for b in range(B):
        for h in range(Hkv):
            n = cache.unit_len(0, b, h)
            want = ref.select(total[b, h].tolist(), n, n_keep[b][h], n_recent)
            assert keep[b, h, : len(want)].tolist() == want
            assert torch.equal(kept[b, h, : len(want)].view(torch.int32), total[b, h, want].view(torch.int32))
            assert (keep[b, h, len(want):] == -7).all() and (kept[b, h, len(want):] == -7).all()


@pytest.mark.parametrize("n", [1, 2, 31, 33, 1000, 1024, 1025, 5000, 60000])
def test_select_rows(n):
    cache = SharedKVCache(1, 2, 2, 64, 2, n, "bf16")
    z = torch.zeros(2, n, 2, 64, dtype=torch.bfloat16, device="cuda")
    cache.append(0, z, z)
    rng = np.random.default_rng(n)
    total = torch.from_numpy(rng.random((2, 2, n)).astype(np.float32))
    total[0, 1] = (total[0, 1] * 5).floor()                              # many equal
    total[1, 0] = total[1, 0].double().sub(0.5).mul(1e30).float()        # both signs
    total[1, 1] = 0.25                                                   # all equal
    total = total.cuda()
    for frac in (0.0, 0.3, 0.9, 1.0):
        for recent in sorted({0, min(n, 1), n // 3, n}):
            counts = [[min(n, max(1, recent, int(frac * n) - i - 2 * b)) for i in range(2)] for b in range(2)]
            if n > 10000 and (frac not in (0.3, 1.0) or recent not in (0, n // 3)):
                continue
            _select_case(cache, total, counts, recent)


@pytest.mark.parametrize("B,Hkv,n", [(1, 1, 8193), (1, 8, 16400), (1, 3, 40001), (4, 8, 20000), (8, 8, 9000), (16, 4, 33000), (1, 2, 70000),
                                     (1, 1, 262144), (1, 1, 262200), (10, 14, 33000), (19, 8, 2500), (40, 8, 2500)])
def test_select_long_units(B, Hkv, n):
    """Units shared by a cluster's blocks, and the sizes around them; equal rows that end in another block than they begin."""
    cache = SharedKVCache(1, Hkv, Hkv, 64, B, n, "bf16")
    z = torch.zeros(B, n, Hkv, 64, dtype=torch.bfloat16, device="cuda")
    cache.append(0, z, z)
    rng = np.random.default_rng(n)
    total = rng.random((B, Hkv, n), dtype=np.float32) ** 4
    total[0, 0, n // 7: n - n // 9] = 0.5                                # one run of equal totals over most of the unit
    total[-1, -1] = np.floor(total[-1, -1] * 3)
    total[-1, -1, ::11] = np.nan
    total = torch.from_numpy(total).cuda()
    for recent, frac in ((0, 0.5), (n // 5, 0.3), (17, 0.97), (n - 1, 1.0)):
        counts = [[max(1, recent, int(frac * n) - 13 * (b + i)) for i in range(Hkv)] for b in range(B)]
        check_selection_all(cache, total, counts, recent)
    # units of different lengths: some blocks of a cluster have no row
    keep = torch.arange(n, dtype=torch.int32, device="cuda").expand(B, Hkv, n).contiguous()
    lens = [[max(1, n - (b * Hkv + i) * n // (B * Hkv)) for i in range(Hkv)] for b in range(B)]
    lens[-1][-1] = 1 if B * Hkv > 1 else n
    cache.evict(0, keep, lens)
    check_selection_all(cache, total, [[(x + 1) // 2 for x in r] for r in lens], 0)
    check_selection_all(cache, total, lens, 1)


def check_selection_all(cache, total, counts, recent):
    """`_select_case` with the definition in numpy: a stable sort of the rows by falling total."""
    B, Hkv = total.shape[:2]
    stride = max(max(r) for r in counts) + 3
    keep = torch.full((B, Hkv, stride), -7, dtype=torch.int32, device="cuda")
    kept = torch.full((B, Hkv, stride), -7.0, device="cuda")
    cache.select_rows(0, total, counts, recent, keep, kept)
    got, got_kept, host = keep.cpu().numpy(), kept.cpu().numpy(), total.cpu().numpy()
    for b in range(B):
        for h in range(Hkv):
            n, c = cache.unit_len(0, b, h), counts[b][h]
            t = host[b, h, : n - recent]
            order = np.lexsort((np.arange(len(t)), -np.where(np.isnan(t), -np.inf, t), np.isnan(t)))
            rows = np.concatenate([np.sort(order[: c - recent]), np.arange(n - recent, n)])
            assert np.array_equal(got[b, h, :c], rows) and (got[b, h, c:] == -7).all() and (got_kept[b, h, c:] == -7).all()
            assert np.array_equal(got_kept[b, h, :c].view(np.int32), host[b, h, rows].view(np.int32))


def test_long_units_and_long_prompts_captured_on_a_side_stream():
    """The launches that long shapes take (clusters; a ring of tokens), recorded and replayed: the same bits as outside."""
    n, n_new, Hq, Hkv, D = 20000, 900, 32, 8, 128
    cache, _, _ = filled(Hq, Hkv, D, 1, n, "bf16", extra=n_new, cls=SharedKVCache)
    total = torch.rand(1, Hkv, n + n_new, generator=torch.Generator().manual_seed(3)).cuda()
    counts = [[700 * (h + 1) for h in range(Hkv)]]
    keep = [torch.zeros(1, Hkv, 700 * Hkv, dtype=torch.int32, device="cuda") for _ in range(2)]
    kept = [torch.zeros(1, Hkv, 700 * Hkv, device="cuda") for _ in range(2)]
    q, k, v = (normal(i, "bf16", 1, n_new, h, D) for i, h in ((1, Hq), (2, Hkv), (3, Hkv)))
    pos = torch.arange(n, n + n_new, dtype=torch.int32, device="cuda").view(1, n_new)
    rot, w = Rotary.from_theta(D), normal(4, "bf16", D)
    out = [torch.zeros_like(q) for _ in range(2)]

    def step(i):
        cache.select_rows(0, total, counts, 5, keep[i], kept[i])
        cache.append_rotary(0, q, k, v, pos, rot, w, w, out=out[i])

    step(0)
    rows = [cache.plane(0, i)[0, :, n:n + n_new].clone() for i in range(2)]
    cache.truncate(n)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(1)
    for i in range(2):
        cache.plane(0, i)[0, :, n:n + n_new] = 0
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(keep[0], keep[1]) and torch.equal(kept[0], kept[1]) and torch.equal(out[0], out[1])
    for i in range(2):
        assert torch.equal(rows[i], cache.plane(0, i)[0, :, n:n + n_new])
    assert cache.device_status() == 0


def test_select_odd_values():
    """Infinities, both zeros (equal), denormals and NaN (below everything)."""
    n = 64
    cache = SharedKVCache(1, 1, 1, 64, 1, n, "bf16")
    z = torch.zeros(1, n, 1, 64, dtype=torch.bfloat16, device="cuda")
    cache.append(0, z, z)
    vals = [0.0, -0.0, float("inf"), -float("inf"), float("nan"), 1e-45, -1e-45, 3.4e38, -3.4e38, 1.0]
    total = torch.tensor([vals[i * 7 % 10] for i in range(n)]).view(1, 1, n).cuda()
    for k in range(1, n + 1, 3):
        _select_case(cache, total, [[k]], 0)


def test_select_on_ragged_units():
    cache, _, _ = filled(4, 2, 64, 2, 300, "bf16", extra=9)
    keep = torch.arange(300, dtype=torch.int32).expand(2, 2, 300).contiguous().cuda()
    cache.evict(0, keep, [[1, 300], [33, 150]])
    total = torch.rand(2, 2, 309, generator=torch.Generator().manual_seed(2)).cuda()
    _select_case(cache, total, [[1, 40], [33, 7]], 1)
    _select_case(cache, total, [[1, 300], [2, 150]], 0)


def test_select_more_units_than_one_launch_takes():
    B, Hkv, n = 60, 16, 40                                               # 960 units
    cache = SharedKVCache(1, 16, 16, 64, B, n, "bf16")
    z = torch.zeros(B, n, Hkv, 64, dtype=torch.bfloat16, device="cuda")
    cache.append(0, z, z)
    total = torch.rand(B, Hkv, n, generator=torch.Generator().manual_seed(0)).cuda()
    _select_case(cache, total, [[1 + (b + h) % n for h in range(Hkv)] for b in range(B)], 1)


def test_evict_by_weight_keeps_what_the_selection_says():
    B, Hq, Hkv, D, n = 2, 8, 2, 128, 400
    cache, k, v = filled(Hq, Hkv, D, B, n, "bf16", extra=3)
    total = torch.zeros(B, Hkv, n + 3, device="cuda")
    for i in range(3):
        cache.decode_attention_weights(0, normal(40 + i, "bf16", B, Hq, D), total)
    counts = [[100, 37], [400, 64]]
    kept = cache.evict_by_weight(0, total, counts, 16, stride=n + 3)
    assert kept.shape == (B, Hkv, n + 3)
    for b in range(B):
        for h in range(Hkv):
            rows = ref.select(total[b, h].tolist(), n, counts[b][h], 16)
            K, V = rows_of(cache, 0, b, h)
            assert torch.equal(K, k[b, rows, h]) and torch.equal(V, v[b, rows, h])
            assert torch.equal(kept[b, h, : len(rows)], total[b, h, rows])
    # the totals go on from there, on units of different lengths
    q = normal(50, "bf16", B, Hq, D)
    after = kept.clone()
    out = cache.decode_attention_weights(0, q, kept, after)
    check_weights(cache, 0, q, kept, after, out, kept.shape[2])


# ------------------------------------------------------------------------------------------ used together

@pytest.mark.parametrize("dtype,Hq,Hkv,D", [("bf16", 32, 8, 128), ("f32", 4, 4, 64)])
def test_a_generation_loop(dtype, Hq, Hkv, D):
    """Prompt in, decode steps with totals, eviction, then two rounds of drafts: rotary append, tree attention, accepted
    path; two layers of which the second shares the first's cache.  Every output against the definition over the rows
    that should be there."""
    B, n = 2, 90
    cache = GuardedCache(2, Hq, Hkv, D, B, 200, dtype, share_map=[0, 0])
    cache.paint(200, B)
    rot, w = Rotary.from_theta(D, 500000.0), normal(1, dtype, D)

    def enter(T, seed, pos):
        x = normal(seed, dtype, B, T, Hq + 2 * Hkv, D)
        q = cache.append_rotary(0, x[:, :, :Hq], x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:], pos, rot, w, w)
        q1 = cache.append_rotary(1, x[:, :, :Hq], None, None, pos, rot, w, None)
        assert torch.equal(q, q1)
        return q

    enter(n, 2, torch.arange(n).int().expand(B, n).contiguous().cuda())
    total = torch.zeros(B, Hkv, 200, device="cuda")
    for t in range(3):
        q = enter(1, 3 + t, torch.full((B, 1), n + t, dtype=torch.int32, device="cuda"))[:, 0].contiguous()
        for layer in (0, 1):
            before = total.clone()
            out = cache.decode_attention_weights(layer, q, total)
            check_weights(cache, layer, q, before, total, out, 200)
    counts = [[40] * Hkv] * B
    cache.evict_by_weight(0, total, counts, 8)
    rng = np.random.default_rng(0)
    for r in range(2):
        T = 9
        words = [ref.random_tree(rng, T) for _ in range(B)]
        depth = torch.tensor([[bin(x).count("1") - 1 for x in row] for row in words]).int()
        q = enter(T, 20 + r, (depth + n + 3 + 4 * r).cuda().contiguous())
        mask = torch.tensor(words).cuda()
        check_tree(cache, 0, q, words, cache.tree_attention(0, q, mask))
        check_tree(cache, 1, q, words, cache.tree_attention(1, q, mask))
        paths = [[j for j in range(T) if row[-1] >> j & 1] for row in words]
        path = torch.zeros(B, T, dtype=torch.int32)
        for b, p in enumerate(paths):
            path[b, : len(p)] = torch.tensor(p)
        want = [[torch.cat((K[:-T], K[-T:][p])) for h in range(Hkv) for K in [rows_of(cache, 0, b, h)[0].clone()]] for b, p in enumerate(paths)]
        cache.accept_draft(path.cuda(), [len(p) for p in paths], T)
        for b in range(B):
            for h in range(Hkv):
                assert torch.equal(rows_of(cache, 1, b, h)[0], want[b][h])
    assert cache.device_status() == 0
    cache.check_canaries()


def test_on_another_stream_and_back_to_back():
    """Calls queued without a wait between them, on a stream of their own, give the bits of calls waited for."""
    cache, _, _ = filled(32, 8, 128, 2, 3000, "bf16", extra=40, cls=SharedKVCache)
    x = normal(3, "bf16", 2, 20, 48, 128)
    pos = torch.arange(20).int().expand(2, 20).contiguous().cuda()
    rot, w = Rotary.from_theta(128), normal(4, "bf16", 128)
    words = torch.tensor([ref.random_tree(np.random.default_rng(b), 20) for b in range(2)]).cuda()
    path = torch.arange(0, 20, 2).int().expand(2, 10).contiguous().cuda()
    total = torch.zeros(2, 8, 3040, device="cuda")

    def step(sync):
        outs = []
        cache.truncate(3000)
        q = cache.append_rotary(0, x[:, :, :32], x[:, :, 32:40], x[:, :, 40:], pos, rot, w, w)
        sync()
        outs.append(cache.tree_attention(0, q, words))
        sync()
        cache.accept_draft(path, [10, 10], 20)
        sync()
        t = torch.empty_like(total).fill_(0)
        outs.append(cache.decode_attention_weights(0, q[:, 0].contiguous(), total, t))
        sync()
        outs += [t, *cache.select_rows(0, t, [[500] * 8] * 2, 100)]
        sync()
        return outs

    want = step(torch.cuda.synchronize)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = [step(lambda: None) for _ in range(20)]
    torch.cuda.synchronize()
    for g in got:
        for a, b in zip(g, want):
            assert torch.equal(a, b)


def test_captured_and_replayed():
    """One verification step recorded as a graph (the lengths of its one recording) and replayed on new inputs."""
    cache, _, _ = filled(16, 4, 64, 2, 500, "bf16", extra=30, cls=SharedKVCache)
    x = normal(3, "bf16", 2, 12, 24, 64)
    pos = torch.arange(12).int().expand(2, 12).contiguous().cuda()
    rot = Rotary.from_theta(64)
    mask = torch.tensor([ref.random_tree(np.random.default_rng(b), 12) for b in range(2)]).cuda()
    out = torch.empty(2, 12, 16, 64, dtype=torch.bfloat16, device="cuda")

    def step():
        cache.truncate(500)
        q = cache.append_rotary(0, x[:, :, :16], x[:, :, 16:20], x[:, :, 20:], pos, rot)
        cache.tree_attention(0, q, mask, out)

    step()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for seed in (5, 6):
        x.copy_(normal(seed, "bf16", 2, 12, 24, 64))
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        got = out.clone()
        step()
        assert torch.equal(got, out)


# ---------------------------------------------------------------------------------------------- refusals

def refused(status, fn, *args):
    with pytest.raises(KvsError) as e:
        fn(*args)
    assert e.value.status == status


def test_refusals_leave_everything_as_it_was():
    cache, _, _ = filled(8, 2, 64, 2, 20, "bf16", extra=4, L=2, share_map=[0, 0], max_batch=3)
    c = cache.ctx
    A, S, C = kb.KVS_ERR_INVALID_ARG, kb.KVS_ERR_STATE, kb.KVS_ERR_CAPACITY
    buf = torch.zeros(1 << 20, dtype=torch.uint8, device="cuda")
    p = buf.data_ptr()
    pool = cache.pool.clone()

    t = kb.kvs_tree_attention
    r_ = p + 65536
    for args in ((2, p, r_, p, 2, 4), (-1, p, r_, p, 2, 4), (0, None, r_, p, 2, 4), (0, p, None, p, 2, 4), (0, p + 2, r_, p, 2, 4),
                 (0, p, r_ + 8, p, 2, 4), (0, p, r_, p + 4, 2, 4), (0, p, r_, p, 3, 4), (0, p, r_, p, 0, 4), (0, p, r_, p, 4, 4),
                 (0, p, p + 65536, p, 2, 0), (0, p, p + 65536, p, 2, 65), (0, p, p + 65536, p, 2, 21), (0, p, p, p, 2, 4)):
        refused(A, t, c, *args)

    f = kb.kvs_accept_draft
    for args in ((None, 4, [1, 1], 4, 2), (p, 0, [1, 1], 4, 2), (p + 2, 4, [1, 1], 4, 2), (p, 4, [1, 1], 0, 2), (p, 4, [1, 1], 65, 2),
                 (p, 4, [5, 1], 4, 2), (p, 4, [-1, 1], 4, 2), (p, 2, [3, 3], 4, 2), (p, 4, [1], 4, 1), (p, 4, [1, 1, 1], 4, 3),
                 (p, 20, [0, 1], 20, 2)):
        refused(A, f, c, *args)
    refused(S, f, c, p, 4, [1, 1], 21, 2)

    freq = (ctypes.c_double * 32)(*[0.5] * 32)

    def rot(dim=64, inter=0, eps=1e-6, arr=freq):
        return kb.kvs_rotary(dim, inter, eps, arr)

    def r(rt=None, layer=0, q=p, qs=512, k=p, ks=128, v=p, vs=128, pos=p, qw=None, kw=None, out=p + 65536, batch=2, n_new=1):
        kb.kvs_append_rotary(c, layer, rt or rot(), q, qs, k, ks, v, vs, pos, qw, kw, out, batch, n_new)

    for kw in (dict(rt=rot(8)), dict(rt=rot(80)), dict(rt=rot(-16)), dict(rt=rot(64, 2)), dict(rt=rot(eps=-1.0)), dict(rt=rot(eps=float("nan"))),
               dict(rt=rot(eps=float("inf"))), dict(rt=rot(arr=None)), dict(rt=rot(arr=(ctypes.c_double * 32)(*[float("inf")] * 32))),
               dict(layer=2), dict(q=None), dict(q=p + 8), dict(qs=504), dict(qs=513), dict(k=None), dict(k=p + 4), dict(ks=127), dict(ks=120),
               dict(v=None), dict(vs=132), dict(pos=None), dict(pos=p + 2), dict(qw=p + 2), dict(kw=p + 8), dict(out=None), dict(out=p + 8),
               dict(batch=1), dict(batch=4), dict(batch=0), dict(n_new=0), dict(q=p, out=p, qs=520)):
        refused(A, lambda: r(**kw))
    refused(C, lambda: r(n_new=5))
    r(layer=1, k=None, v=None, ks=0, vs=0)            # a sharing layer needs no k, v

    d = kb.kvs_decode_attention_weights
    o = p + 65536
    for args in ((2, p, o, None, o, 20, 2), (0, None, o, None, o, 20, 2), (0, p, None, None, o, 20, 2), (0, p, o, None, None, 20, 2),
                 (0, p, o, p + 2, o, 20, 2), (0, p, o, None, o + 2, 20, 2), (0, p, o, None, o, 19, 2), (0, p, o, None, o, 20, 3),
                 (0, p + 8, o, None, o, 20, 2)):
        refused(A, d, c, *args)

    s = kb.kvs_select_rows
    for args in ((2, p, 20, [1] * 4, 0, o, None, 20, 2), (0, None, 20, [1] * 4, 0, o, None, 20, 2), (0, p, 19, [1] * 4, 0, o, None, 20, 2),
                 (0, p, 20, [0, 1, 1, 1], 0, o, None, 20, 2), (0, p, 20, [21, 1, 1, 1], 0, o, None, 30, 2), (0, p, 20, [1] * 4, -1, o, None, 20, 2),
                 (0, p, 20, [1] * 4, 2, o, None, 20, 2), (0, p, 20, [9] * 4, 0, o, None, 8, 2), (0, p, 20, [1] * 4, 0, None, None, 20, 2),
                 (0, p, 20, [1] * 4, 0, o + 1, None, 20, 2), (0, p, 20, [1] * 4, 0, o, o + 2, 20, 2), (0, p + 2, 20, [1] * 4, 0, o, None, 20, 2),
                 (0, p, 20, [1] * 6, 0, o, None, 20, 3)):
        refused(A, s, c, *args)

    cache.set_option(KVS_OPT_REPLAY, 1)
    refused(S, t, c, 0, p, r_, p, 2, 4)
    refused(S, f, c, p, 4, [1, 1], 4, 2)
    refused(S, s, c, 0, p, 20, [1] * 4, 0, o, None, 20, 2)
    refused(A, d, c, 0, p, o, None, o, 20, 2)           # a recorded step needs totals for max_seq rows
    cache.set_option(KVS_OPT_REPLAY, 0)

    torch.cuda.synchronize()
    assert torch.equal(pool, cache.pool) and cache.seq_len(0) == 20 and cache.device_status() == 0


def test_tensors_of_another_device_are_refused():
    cache, _, _ = filled(8, 2, 64, 2, 20, "bf16", extra=4)
    q = normal(1, "bf16", 2, 1, 8, 64)
    kv = normal(2, "bf16", 2, 1, 2, 64)
    pos = torch.zeros(2, 1, dtype=torch.int32)
    total = torch.zeros(2, 2, 24)
    rot = Rotary.from_theta(64)
    for call in (lambda: cache.append_rotary(0, q, kv, kv, pos, rot), lambda: cache.append_rotary(0, q.cpu(), kv, kv, pos.cuda(), rot),
                 lambda: cache.append_rotary(0, q, kv, kv.cpu(), pos.cuda(), rot), lambda: cache.tree_attention(0, q.cpu()),
                 lambda: cache.tree_attention(0, q, torch.zeros(2, 1, dtype=torch.int64)), lambda: cache.accept_draft(pos, [1, 1], 1),
                 lambda: cache.decode_attention_weights(0, q[:, 0].contiguous(), total), lambda: cache.select_rows(0, total, [[1, 1]] * 2, 0)):
        with pytest.raises(AssertionError):
            call()
    assert cache.seq_len(0) == 20


def test_refusals_on_empty_slots():
    cache, _, _ = filled(8, 2, 64, 2, 0, "bf16", extra=4)
    p = torch.zeros(4096, dtype=torch.uint8, device="cuda").data_ptr()
    refused(kb.KVS_ERR_STATE, kb.kvs_tree_attention, cache.ctx, 0, p, p + 2048, None, 2, 1)
    refused(kb.KVS_ERR_STATE, kb.kvs_accept_draft, cache.ctx, p, 4, [1, 1], 1, 2)
    refused(kb.KVS_ERR_STATE, kb.kvs_decode_attention_weights, cache.ctx, 0, p, p, None, p, 4, 2)
    refused(kb.KVS_ERR_STATE, kb.kvs_select_rows, cache.ctx, 0, p, 4, [1] * 4, 0, p, None, 4, 2)
