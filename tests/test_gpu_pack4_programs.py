"""Random programs over 4-bit and plain caches with reordered sequences, queued without a wait, against a host model of every
sequence's rows; the calls recorded into graphs and on another stream."""
import random

import pytest
import torch

import operators_reference as oref
import pack4_reference as ref
from helpers import GuardedCache
from paper_2410_18517_b200 import KVS_OPT_EARLY_START, KVS_OPT_FINISH_IN_KERNEL, KVS_OPT_MAX_CTAS, SharedKVCache
from paper_2410_18517_b200 import build as kbuild

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    kbuild.build()


DT = {"bf16": torch.bfloat16, "f32": torch.float32}


class Model:
    """What every sequence of every layer's own cache holds: k, v [B][n][Hkv][D] on the CPU, as the cache stands for them."""

    def __init__(self, share, fmt):
        self.share, self.fmt = share, fmt
        self.rows = {l: None for l in range(len(share)) if share[l] == l}

    def held(self, x):
        return ref.values(x) if self.fmt == "4bit" else x

    def append(self, l, k, v):
        new = [self.held(k), self.held(v)]
        self.rows[l] = new if self.rows[l] is None else [torch.cat(p, 1) for p in zip(self.rows[l], new)]

    def reorder(self, parent, first):
        for l, kv in self.rows.items():
            if kv is not None:
                self.rows[l] = [torch.cat((x[:len(parent), :first] if first else x[parent][:, :0], x[parent][:, first:]), 1) for x in kv]

    def truncate(self, n):
        for l, kv in self.rows.items():
            if kv is not None:
                self.rows[l] = [x[:, :n] for x in kv]


def program(seed, fmt, dtype, stream=None, graph=False, long=False):
    r = random.Random(seed)
    g = torch.Generator().manual_seed(seed)
    G, Hkv, D = r.choice((1, 2, 4, 8) if dtype == "f32" else range(1, 9)), r.choice((1, 2, 3)), r.choice((64, 128))
    share = r.choice(([0], [0, 0], [0, 1, 0]))
    most, cap = r.choice((3, 6)), 6000 if long else r.choice((90, 400))
    cache = GuardedCache(len(share), G * Hkv, Hkv, D, most, cap, dtype, share_map=share, cache_format=fmt)
    cache.paint(cap, most)
    cache.set_option(KVS_OPT_MAX_CTAS, r.choice((0, 0, 3)))
    cache.set_option(KVS_OPT_EARLY_START, int(seed % 5 != 3))
    cache.set_option(KVS_OPT_FINISH_IN_KERNEL, int(seed % 5 != 4))
    model, calls, checks, B = Model(share, fmt), [], [], r.randint(1, most)
    own = [l for l in range(len(share)) if share[l] == l]

    def tensors(*shapes):
        return [torch.randn(s, generator=g).to(DT[dtype]) for s in shapes]

    def attend(l, q, out):
        K, V = (x.clone() for x in model.rows[share[l]])

        def check():
            for b in range(q.shape[0]):
                for h in range(Hkv):
                    o, _, mass, d = oref.attend(q[b, h * G:(h + 1) * G][None], K[b, :, h], V[b, :, h])
                    # (a plain bf16 cache: the weights in two bf16 terms, 2^-16 of themselves)
                    bound = (oref.weight_error(d, K.shape[1]) + 2.0 ** -16) * mass[0] + oref.U * o[0].abs() + 1e-30
                    assert ((out[b, h * G:(h + 1) * G].cpu().double() - o[0]).abs() <= bound).all(), ("attend", l, b, h)
        checks.append(check)

    def append(n):
        for l in own:
            k, v = tensors((B, n, Hkv, D), (B, n, Hkv, D))
            kd, vd = k.cuda(), v.cuda()
            calls.append(lambda l=l, kd=kd, vd=vd: cache.append(l, kd, vd))
            model.append(l, k, v)

    append(3000 if long else r.randint(1, 40))
    for _ in range(14):
        n = model.rows[own[0]][0].shape[1]
        what = r.choice(("append", "step", "step", "reorder", "reorder", "attend", "truncate", "read", "prompt"))
        if what == "append" and n + 20 < cap:
            append(r.randint(1, 20))
        elif what == "step" and n + 1 < cap:
            for l in range(len(share)):
                q, k, v = tensors((B, G * Hkv, D), (B, 1, Hkv, D), (B, 1, Hkv, D))
                out = torch.zeros(B, G * Hkv, D, device="cuda")
                mine = share[l] == l
                if mine:
                    model.append(l, k, v)
                qd, kd, vd = q.cuda(), k.cuda() if mine else None, v.cuda() if mine else None
                calls.append(lambda l=l, qd=qd, kd=kd, vd=vd, out=out: cache.decode_step(l, qd, kd, vd, out))
                attend(l, q, out)
        elif what == "attend":
            l = r.randrange(len(share))
            q, = tensors((B, G * Hkv, D))
            out = torch.zeros(B, G * Hkv, D, device="cuda")
            qd = q.cuda()
            calls.append(lambda l=l, qd=qd, out=out: cache.decode_attention(l, qd, out))
            attend(l, q, out)
        elif what == "reorder":
            new = r.randint(1, most)
            first = r.randint(0, n) if new <= B and r.random() < 0.5 else 0
            parent = [r.randrange(B) for _ in range(new)]
            pd = torch.tensor(parent, dtype=torch.int32, device="cuda")
            calls.append(lambda pd=pd, first=first: cache.reorder(pd, first))
            model.reorder(parent, first)
            B = new
        elif what == "truncate" and n > 2:
            to = r.randint(n // 2, n)
            calls.append(lambda to=to: cache.truncate(to))
            model.truncate(to)
        elif what == "read":
            first = r.randrange(n)
            count = r.randint(1, n - first)
            l = r.randrange(len(share))
            want = [x[:, first:first + count].clone() for x in model.rows[share[l]]]
            got = []
            calls.append(lambda l=l, first=first, count=count, got=got: got.extend(cache.read_rows(l, first, count)))
            checks.append(lambda want=want, got=got: [None for a, b in zip(want, got) if not torch.equal(a, b.cpu())] == [] or 1 / 0)
        elif what == "prompt":
            l, T = r.randrange(len(share)), r.randint(1, min(n, 9))
            q, = tensors((B, T, G * Hkv, D))
            out = torch.zeros(B, T, G * Hkv, D, device="cuda")
            qd = q.cuda()
            calls.append(lambda l=l, qd=qd, out=out: cache.prefill_attention(l, qd, out))
            K, V = (x.clone() for x in model.rows[share[l]])

            def check(q=q, K=K, V=V, out=out, n=n, T=T):
                sees = torch.arange(n) <= torch.arange(n - T, n)[:, None]
                for b in range(q.shape[0]):
                    o, _, mass, d = oref.attend(q[b, :, :G], K[b, :, 0], V[b, :, 0], sees)
                    bound = (oref.weight_error(d, n) + 2.0 ** -16) * mass + oref.U * o.abs() + 1e-30
                    assert ((out[b, :, :G].cpu().double() - o).abs() <= bound).all(), ("prompt", b)
            checks.append(check)
    torch.cuda.synchronize()
    if graph:
        rec = torch.cuda.CUDAGraph()
        with torch.cuda.graph(rec):
            for call in calls:
                call()
        rec.replay()
    else:
        with torch.cuda.stream(stream or torch.cuda.current_stream()):
            for call in calls:
                call()
    torch.cuda.synchronize()
    assert cache.device_status() == 0
    for check in checks:
        check()
    for l in own:
        if model.rows[l] is not None and model.rows[l][0].shape[1]:
            for a, b in zip(model.rows[l], cache.read_rows(l)):
                assert torch.equal(a, b.cpu()), ("rows", l)
    cache.check_canaries()


@pytest.mark.parametrize("fmt,dtype", [("4bit", "bf16"), ("4bit", "f32"), ("plain", "bf16")])
@pytest.mark.parametrize("seed", range(14))
def test_programs(seed, fmt, dtype):
    program(seed, fmt, dtype, torch.cuda.Stream() if seed % 2 else None)


@pytest.mark.parametrize("seed", range(100, 104))
def test_programs_over_long_caches(seed):
    """Kernels long enough that a call queued behind one really starts beside it."""
    program(seed, "4bit", "bf16", long=True)


@pytest.mark.parametrize("fmt,dtype", [("4bit", "bf16"), ("4bit", "f32"), ("plain", "bf16")])
@pytest.mark.parametrize("seed", range(200, 206))
def test_recorded_programs(seed, fmt, dtype):
    program(seed, fmt, dtype, graph=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_chain_drafts_over_a_4bit_cache(dtype):
    """Drafts are appended, verified as the newest chunk of a prompt, and partly accepted: their 4-bit rows move bit for bit."""
    B, Hkv, D, n, T = 3, 2, 64, 21, 6
    cache = GuardedCache(2, 4, Hkv, D, B, n + T, dtype, share_map=[0, 0], cache_format="4bit")
    cache.paint(n + T, B)
    g = torch.Generator().manual_seed(1)
    k, v = (torch.randn(B, n + T, Hkv, D, generator=g).to(DT[dtype]) for _ in range(2))
    cache.append(0, k.cuda(), v.cuda())
    assert torch.isfinite(cache.prefill_attention(1, torch.randn(B, T, 4, D, generator=g).to(DT[dtype]).cuda())).all()
    before = cache.plane(0, 0).clone()
    path = torch.tensor([[0, 2, 5], [1, 3, 4], [0, 1, 99]], dtype=torch.int32).cuda()
    cache.accept_draft(path, [3, 3, 2], T)
    for b, took in enumerate(([0, 2, 5], [1, 3, 4], [0, 1])):
        assert cache.unit_len(1, b, 0) == n + len(took)
        assert torch.equal(cache.plane(0, 0)[b, :, n:n + len(took)], before[b, :, [n + t for t in took]])
    kr, _ = cache.read_rows(0)
    assert torch.equal(kr[0, :n + 3].cpu(), ref.values(k)[0, list(range(n)) + [n, n + 2, n + 5]]) and not kr[2, n + 2:].any()
    assert cache.device_status() == 0
    cache.check_canaries()


def test_two_caches_and_a_selection_in_between():
    """Calls of two contexts interleaved on one stream; the selection's scratch is its own context's."""
    a, b = (SharedKVCache(1, 4, 2, 64, 4, 50, "bf16", cache_format="4bit") for _ in range(2))
    g = torch.Generator(device="cuda").manual_seed(0)
    k = torch.randn(4, 40, 2, 64, device="cuda", generator=g).bfloat16()
    q = torch.randn(4, 4, 64, device="cuda", generator=g).bfloat16()
    x = torch.randn(4, 5000, device="cuda", generator=g)
    a.append(0, k, k)
    b.append(0, -k, -k)
    outs = [(a.decode_attention(0, q), a.beam_select(x, x[:, 0].contiguous(), 2, 4), b.prefill_attention(0, q[:, None].contiguous()),
             b.beam_select(-x, x[:, 1].contiguous(), 4, 4), b.decode_attention(0, q), a.read_rows(0)[0]) for _ in range(5)]
    torch.cuda.synchronize()
    flat = [[t for o in run for t in (o if isinstance(o, tuple) else (o,))] for run in outs]
    for run in flat[1:]:
        assert all(torch.equal(s, t) for s, t in zip(run, flat[0]))
