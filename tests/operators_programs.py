"""Random programs over one cache: appends, rotary appends, decode, weighted decode, prefill, tree attention, accepted drafts,
roll-backs, selections and evictions in any legal order, queued without a wait between them, against a model that keeps
every unit's rows on the host.  What the calls return and what the pool holds at the end must be what the model says."""
import random

import torch

import operators_reference as ref
from paper_2410_18517_b200 import Rotary, SharedKVCache
from paper_2410_18517_b200 import binding as kb

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


class Program:
    def __init__(self, seed, dtype, Hq, Hkv, D, B, capacity, share_map, steps, options=(), filled=0):
        """`filled`: rows every slot starts with."""
        self.rng, self.gen = random.Random(seed), torch.Generator().manual_seed(seed)
        self.dtype, self.Hq, self.Hkv, self.D, self.B, self.cap, self.map = DT[dtype], Hq, Hkv, D, B, capacity, share_map
        self.cache = SharedKVCache(len(share_map), Hq, Hkv, D, B, capacity, dtype, share_map=share_map)
        self.side = SharedKVCache(1, Hq, Hkv, D, B, capacity, dtype)      # what a rotary append stores, taken by itself
        for o, v in options:
            self.cache.set_option(o, v)
        self.own = [l for l, s in enumerate(share_map) if s == l]
        empty = torch.zeros(0, D, dtype=self.dtype)
        self.rows = {l: [[[empty, empty] for _ in range(Hkv)] for _ in range(B)] for l in self.own}    # [b][h] -> K, V
        self.ragged = {l: False for l in self.own}
        self.calls, self.checks, self.log = [], [], []
        for l in self.own if filled else ():
            self.do_append(l, filled)
        for _ in range(steps):
            self.step()

    # ------------------------------------------------------------------ helpers
    def normal(self, *shape):
        return torch.randn(*shape, generator=self.gen).to(self.dtype)

    def source(self, layer):
        while self.map[layer] != layer:
            layer = self.map[layer]
        return layer

    def lens(self, l):
        return [self.rows[l][b][h][0].shape[0] for b in range(self.B) for h in range(self.Hkv)]

    def room(self, l):
        return self.cap - max(self.lens(l))

    def push(self, l, k, v):
        for b in range(self.B):
            for h in range(self.Hkv):
                r = self.rows[l][b][h]
                self.rows[l][b][h] = [torch.cat((r[0], k[b, :, h])), torch.cat((r[1], v[b, :, h]))]

    def expect_attention(self, l, q, out, sees, fp32_out, what):
        """q [B][T][Hq][D] host, out: the device tensor the call fills (same leading shape), sees(b, n) -> [T][n] or None."""
        snap = [[list(self.rows[l][b][h]) for h in range(self.Hkv)] for b in range(self.B)]
        G = self.Hq // self.Hkv

        def check():
            for b in range(self.B):
                for h in range(self.Hkv):
                    K, V = (x.cuda() for x in snap[b][h])
                    n = K.shape[0]
                    s = sees(b, n)
                    o, p, mass, d = ref.attend(q[b, :, h * G:(h + 1) * G].cuda(), K, V, None if s is None else s.cuda())
                    rest = (ref.weight_error(d, n) + 2.0 ** -16 + n * 2.0 ** -23) * mass + 1e-30
                    bound = rest if fp32_out else ref.half_step(self.dtype) * (o.abs() + rest) + rest
                    got = out[b].view(-1, self.Hq, self.D)[:, h * G:(h + 1) * G].double()
                    assert torch.isfinite(got).all(), (what, b, h, n, "not finite")
                    assert ((got - o).abs() <= bound).all(), (what, b, h, n, float(((got - o).abs() / bound).max()))
        self.checks.append(check)
        return snap

    # ------------------------------------------------------------------ steps
    def step(self):
        r = self.rng
        kinds = ["append", "rotary", "rotary", "decode", "step", "weights", "prefill", "tree", "draft", "draft", "truncate", "evict", "select", "static"]
        kind = r.choice(kinds)
        getattr(self, "do_" + kind)()

    def do_append(self, layer=None, n=None, junk_from=None):
        l = self.rng.choice(self.own) if layer is None else layer
        n = n or self.rng.choice((1, 1, 2, 5, 17, 40, 64, 130))
        if n > self.room(l):
            return
        k, v = self.normal(self.B, n, self.Hkv, self.D), self.normal(self.B, n, self.Hkv, self.D)
        if junk_from is not None:
            k[:, junk_from:] = float("nan")
            v[:, junk_from:] = float("nan")
        kd, vd = k.cuda(), v.cuda()
        self.log.append(("append", l, n))
        self.calls.append(lambda: self.cache.append(l, kd, vd))
        self.push(l, k, v)

    def do_rotary(self, layer=None, n=None, junk_from=None):
        layer = self.rng.randrange(len(self.map)) if layer is None else layer
        n = n or self.rng.choice((1, 1, 3, 20, 64))
        own = layer in self.own
        if own and n > self.room(layer):
            return
        x = self.normal(self.B, n, self.Hq + 2 * self.Hkv, self.D)
        if junk_from is not None:
            x[:, junk_from:] = float("nan")
        xd, w = x.cuda(), self.normal(self.D).cuda()
        Hq, Hkv = self.Hq, self.Hkv
        parts = xd[:, :, :Hq], xd[:, :, Hq:Hq + Hkv] if own else None, xd[:, :, Hq + Hkv:] if own else None
        pos = torch.randint(0, 100000, (self.B, n), generator=self.gen).int().cuda()
        rot = Rotary.from_theta(self.D)
        self.side.reset()
        want = self.side.append_rotary(0, xd[:, :, :Hq], xd[:, :, Hq:Hq + Hkv], xd[:, :, Hq + Hkv:], pos, rot, w, w).clone()
        k, v = (self.side.plane(0, i)[:, :, :n].transpose(1, 2).cpu() for i in range(2))
        out = torch.empty_like(want)
        self.log.append(("rotary", layer, n))
        self.calls.append(lambda: self.cache.append_rotary(layer, *parts, pos, rot, w, w, out=out))

        def check():
            assert torch.equal(out.view(torch.uint8), want.view(torch.uint8)), "rotary queries"
        self.checks.append(check)
        if own:
            self.push(layer, k, v)

    def pick(self):
        layers = [l for l in range(len(self.map)) if max(self.lens(self.source(l))) > 0]
        return self.rng.choice(layers) if layers else None

    def do_decode(self, static=False):
        layer = self.pick()
        if layer is None:
            return
        q = self.normal(self.B, 1, self.Hq, self.D)
        qd, out = q[:, 0].cuda().contiguous(), torch.empty(self.B, self.Hq, self.D, device="cuda")
        self.log.append(("static" if static else "decode", layer))
        if static:
            self.calls.append(lambda: kb.kvs_decode_attention_static(self.cache.ctx, layer, qd, out, self.B, self.cache._stream()))
        else:
            self.calls.append(lambda: self.cache.decode_attention(layer, qd, out))
        self.expect_attention(self.source(layer), q, out, lambda b, n: None, True, self.log[-1])

    def do_static(self):
        self.do_decode(static=True)

    def do_step(self):
        layer = self.rng.randrange(len(self.map))
        l, own = self.source(layer), layer in self.own
        if (own and self.room(l) < 1) or (not own and max(self.lens(l)) == 0):
            return
        q = self.normal(self.B, 1, self.Hq, self.D)
        k, v = self.normal(self.B, 1, self.Hkv, self.D), self.normal(self.B, 1, self.Hkv, self.D)
        qd, kd, vd = q[:, 0].cuda().contiguous(), k.cuda(), v.cuda()
        out = torch.empty(self.B, self.Hq, self.D, device="cuda")
        self.log.append(("step", layer))
        self.calls.append(lambda: self.cache.decode_step(layer, qd, kd if own else None, vd if own else None, out))
        if own:
            self.push(l, k, v)
        self.expect_attention(l, q, out, lambda b, n: None, True, self.log[-1])

    def do_weights(self):
        layer = self.pick()
        if layer is None:
            return
        l, stride = self.source(layer), self.cap + self.rng.choice((0, 1, 2))
        q = self.normal(self.B, 1, self.Hq, self.D)
        qd, out = q[:, 0].cuda().contiguous(), torch.empty(self.B, self.Hq, self.D, device="cuda")
        total = torch.rand(self.B, self.Hkv, stride, generator=self.gen)
        td, G = total.cuda(), self.Hq // self.Hkv
        self.log.append(("weights", layer))
        self.calls.append(lambda: self.cache.decode_attention_weights(layer, qd, td, out=out))
        snap = self.expect_attention(l, q, out, lambda b, n: None, True, self.log[-1])

        def check():
            for b in range(self.B):
                for h in range(self.Hkv):
                    K, V = (x.cuda() for x in snap[b][h])
                    n = K.shape[0]
                    _, p, _, d = ref.attend(q[b, :, h * G:(h + 1) * G].cuda(), K, V)
                    w, start = p[0].sum(0), total[b, h].cuda().double()
                    err = (td[b, h, :n].double() - start[:n] - w).abs()
                    assert (err <= (ref.weight_error(d, n) + G * ref.U) * w + ref.U * (start[:n] + w) + 1e-30).all(), ("totals", b, h, n)
                    assert torch.equal(td[b, h, n:].double(), start[n:])
        self.checks.append(check)

    def do_prefill(self):
        layer = self.pick()
        if layer is None or self.ragged[self.source(layer)]:
            return
        l = self.source(layer)
        n = self.lens(l)[0]
        T = self.rng.randint(1, max(1, min(n, 4_000_000 // n)))        # (the check holds T x n scores in float64)
        q = self.normal(self.B, T, self.Hq, self.D)
        qd, out = q.cuda(), torch.empty(self.B, T, self.Hq, self.D, device="cuda")
        self.log.append(("prefill", layer, n, T))
        self.calls.append(lambda: self.cache.prefill_attention(layer, qd, out))
        causal = torch.arange(n)[None, :] <= (torch.arange(T) + n - T)[:, None]
        self.expect_attention(l, q, out, lambda b, m: causal, True, self.log[-1])

    def tree(self, layer, T, junk_from=None):
        import numpy as np

        words = [ref.random_tree(np.random.default_rng(self.rng.randrange(1 << 30)), T) for _ in range(self.B)]
        if junk_from is not None:       # the tokens from there on are padding: nobody sees them, they see nothing
            words = [[w if t < junk_from else 0 for t, w in enumerate(row)] for row in words]
        q = self.normal(self.B, T, self.Hq, self.D)
        qd, out = q.cuda(), torch.empty(self.B, T, self.Hq, self.D, dtype=self.dtype, device="cuda")
        mask = torch.tensor([ref.to_int64(w) for w in words]).cuda()
        self.log.append(("tree", layer, T))
        self.calls.append(lambda: self.cache.tree_attention(layer, qd, mask, out))
        self.expect_attention(self.source(layer), q, out, lambda b, n: ref.tree_sees(words[b], n, T), False, self.log[-1])
        return words

    def do_tree(self):
        layer = self.pick()
        if layer is None:
            return
        least = min(self.lens(self.source(layer)))
        if least:
            self.tree(layer, self.rng.randint(1, min(64, least)))

    def do_draft(self):
        """Drafts into every slot, verified on some layers, then accepted, or rolled back."""
        T = self.rng.choice((1, 2, 7, 16, 33, 64))
        if any(self.room(l) < T for l in self.own):
            return
        before = {l: self.lens(l) for l in self.own}
        good = self.rng.randint(1, T)
        rotary = self.rng.random() < 0.5
        junk = good if good < T and self.rng.random() < 0.7 else None
        for l in self.own:
            (self.do_rotary if rotary else self.do_append)(l, T, junk)
        for layer in range(len(self.map)):
            if self.rng.random() < 0.7:
                self.tree(layer, T, junk)
        uniform = not any(self.ragged.values()) and len({x for l in self.own for x in before[l]}) == 1
        if uniform and (self.rng.random() < 0.4):
            base = before[self.own[0]][0]
            keep = self.rng.randint(0, good)
            self.truncate(base + keep)
            return
        same = self.rng.random() < 0.5
        counts = [self.rng.randint(0, good) for _ in range(self.B)]
        if same or any(x + c < 1 for l in self.own for i, x in enumerate(before[l]) for c in (counts[i // self.Hkv],)):
            counts = [max(counts)] * self.B
            if counts[0] == 0 and any(self.ragged[l] and min(before[l]) == 0 for l in self.own):
                counts = [good] * self.B
        path = torch.full((self.B, T), 99, dtype=torch.int32)
        for b, c in enumerate(counts):
            path[b, :c] = torch.tensor(sorted(self.rng.sample(range(good), c)), dtype=torch.int32)
        pd = path.cuda()
        self.log.append(("accept", T, tuple(counts)))
        self.calls.append(lambda: self.cache.accept_draft(pd, counts, T))
        for l in self.own:
            for b in range(self.B):
                at = path[b, :counts[b]].long()
                for h in range(self.Hkv):
                    n0 = self.rows[l][b][h][0].shape[0] - T
                    self.rows[l][b][h] = [torch.cat((x[:n0], x[n0:][at])) for x in self.rows[l][b][h]]
            if len(set(counts)) > 1:
                self.ragged[l] = True

    def truncate(self, n):
        self.log.append(("truncate", n))
        self.calls.append(lambda: self.cache.truncate(n))
        for l in self.own:
            for b in range(self.B):
                for h in range(self.Hkv):
                    self.rows[l][b][h] = [x[:n] for x in self.rows[l][b][h]]

    def do_truncate(self):
        if any(self.ragged.values()) or self.rng.random() < 0.5:
            return
        top = max(max(self.lens(l)) for l in self.own)
        if top:
            self.truncate(self.rng.randint(max(1, top // 2), top))

    def do_evict(self, by_weight=False):
        l = self.rng.choice(self.own)
        lens = self.lens(l)
        if min(lens) == 0 or self.rng.random() < 0.5:
            return
        lists = [sorted(self.rng.sample(range(n), self.rng.randint(max(1, n // 2), n))) for n in lens]
        stride = max(len(x) for x in lists)
        keep = torch.zeros(self.B, self.Hkv, stride, dtype=torch.int32)
        for u, x in enumerate(lists):
            keep[u // self.Hkv, u % self.Hkv, :len(x)] = torch.tensor(x, dtype=torch.int32)
        kd, counts = keep.cuda(), [len(x) for x in lists]
        self.log.append(("evict", l, tuple(counts)))
        self.calls.append(lambda: self.cache.evict(l, kd, counts))
        self.keep_rows(l, lists)

    def keep_rows(self, l, lists):
        for u, x in enumerate(lists):
            b, h = u // self.Hkv, u % self.Hkv
            self.rows[l][b][h] = [r[x] for r in self.rows[l][b][h]]
        self.ragged[l] = True

    def do_select(self):
        """The selection, and the eviction that takes its list from the device."""
        l = self.rng.choice(self.own)
        lens = self.lens(l)
        if min(lens) == 0 or self.rng.random() < 0.3:
            return
        total = (torch.rand(self.B, self.Hkv, max(lens) + 3, generator=self.gen) * self.rng.choice((4, 1000))).floor()
        recent = self.rng.randint(0, min(lens) // 2)
        counts = [self.rng.randint(max(1, recent, n // 2), n) for n in lens]
        td = total.cuda()
        keep = torch.zeros(self.B, self.Hkv, max(counts), dtype=torch.int32, device="cuda")
        kept = torch.zeros(self.B, self.Hkv, max(counts), device="cuda")
        lists = [ref.select(total[u // self.Hkv, u % self.Hkv].tolist(), lens[u], counts[u], recent) for u in range(len(lens))]
        self.log.append(("select", l, recent, tuple(counts)))
        self.calls.append(lambda: self.cache.select_rows(l, td, counts, recent, keep, kept))

        def check():
            for u, x in enumerate(lists):
                b, h = u // self.Hkv, u % self.Hkv
                assert keep[b, h, :len(x)].tolist() == x and torch.equal(kept[b, h, :len(x)].cpu(), total[b, h, x])
        self.checks.append(check)
        if self.rng.random() < 0.5:
            self.calls.append(lambda: self.cache.evict(l, keep, counts))
            self.keep_rows(l, lists)

    # ------------------------------------------------------------------ run
    def run(self, stream=None, graph=False):
        """`graph`: the calls are recorded, and run when the graph does."""
        torch.cuda.synchronize()
        if graph:
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                for call in self.calls:
                    call()
            g.replay()
        else:
            with torch.cuda.stream(stream or torch.cuda.current_stream()):
                for call in self.calls:
                    call()
        torch.cuda.synchronize()
        assert self.cache.device_status() == 0, (self.cache.device_status(), self.log)
        try:
            for check in self.checks:
                check()
            for l in self.own:
                s = self.cache.slot_of_layer(l)
                for b in range(self.B):
                    for h in range(self.Hkv):
                        n = self.rows[l][b][h][0].shape[0]
                        assert self.cache.unit_len(l, b, h) == n, ("length", l, b, h)
                        for i in range(2):
                            got = self.cache.plane(s, i)[b, h, :n].cpu()
                            assert torch.equal(got.view(torch.uint8), self.rows[l][b][h][i].contiguous().view(torch.uint8)), ("rows", l, b, h, i)
        except AssertionError as e:
            raise AssertionError(f"{e} after {self.log}") from e
