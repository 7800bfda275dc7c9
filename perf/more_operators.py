"""Cases of the operators for a cache held in 4 bits and for beam search over a cache: what is timed, on which inputs, and
what each computes.

Five kinds of pass (layouts as in include/kvs.h):

  pack     new tokens' keys and values enter a 4-bit cache; the values its rows stand for are read back
  attend   attention of one token per sequence over a 4-bit cache
  prompt   causal attention of a prompt (or its newest chunk) over a 4-bit cache
  select   beam search: the best continuations of every request's beams over the vocabulary
  reorder  beam search: the sequences of every cache slot take the rows of the beams they continue

A row of a 4-bit cache is cut into four groups of head_dim / 4 elements.  With lo and hi the group's smallest and largest
element (fp32 arithmetic):  s = (hi - lo) / 15 rounded up to bf16,  b = bf16(lo - 16 s),
code c = clamp(rint((x - b) / s) - 16, 0, 15)  (s = 0: c = 0),  value = s * (16 + c) + b, rounded once to the storage type.

With ``own`` false ``run`` computes a pass in elementary torch operations; with ``own`` true it makes the calls a program
makes of this package.  ``exact`` restates the definitions in float64.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # a decode step's tokens of a batch: launch latency is what counts
        dict(name="pack_decode_b32", kind="pack", dtype="bf16", B=32, n_ctx=700, n_new=1, Hkv=8, D=128),
        # a prompt chunk of four long sequences
        dict(name="pack_prompt_b4", kind="pack", dtype="bf16", B=4, n_ctx=0, n_new=4096, Hkv=8, D=128),
        # one user, a short odd context: latency
        dict(name="attend_b1_n1031", kind="attend", dtype="bf16", B=1, n=1031, Hq=32, Hkv=8, D=128, ragged=False),
        # the 13B shape, no grouped heads: one query row per cached row
        dict(name="attend_mha_b16_n8192", kind="attend", dtype="bf16", B=16, n=8192, Hq=40, Hkv=40, D=128, ragged=False),
        # grouped heads over long contexts
        dict(name="attend_gqa_b8_n32768", kind="attend", dtype="bf16", B=8, n=32768, Hq=32, Hkv=8, D=128, ragged=False),
        # fp32 storage, the units cut to lengths of their own by an eviction
        dict(name="attend_f32_ragged", kind="attend", dtype="f32", B=3, n=733, Hq=8, Hkv=2, D=64, ragged=True),
        # whole prompts
        dict(name="prompt_gqa_b2_t4096", kind="prompt", dtype="bf16", B=2, n=4096, T=4096, Hq=32, Hkv=8, D=128),
        # the newest chunk of longer prompts, odd sizes, no grouped heads
        dict(name="prompt_chunk_b3_t333", kind="prompt", dtype="bf16", B=3, n=1501, T=333, Hq=16, Hkv=16, D=64),
        # one request of four beams
        dict(name="select_r1_w4", kind="select", dtype="f32", R=1, W=4, V=32000, K=8, pad=0, first=False),
        # a batch of requests over a large vocabulary, rows of a padded logits tensor
        dict(name="select_r16_w8", kind="select", dtype="bf16", R=16, W=8, V=131071, K=16, pad=17, first=False),
        # four beams of a small model: three continue two others, only what was generated moves
        dict(name="reorder_r1_w4", kind="reorder", dtype="bf16", slots=3, R=1, W=4, moved=2, Hkv=8, D=64, n=517, first=480, fork=False),
        # the first step of a batch of requests: every prompt is copied to its beams
        dict(name="reorder_fork_r4_w8", kind="reorder", dtype="bf16", slots=4, R=4, W=8, moved=7, Hkv=8, D=128, n=1500, first=0, fork=True),
    ]


_HEADS_BF16 = [(32, 32, 128), (40, 40, 128), (32, 8, 128), (40, 8, 128), (28, 4, 128), (8, 1, 128),
               (16, 16, 64), (16, 8, 64), (24, 8, 64), (12, 2, 64)]
_HEADS_F32 = [(4, 4, 64), (8, 2, 64), (8, 1, 128), (4, 2, 128)]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    most = {}
    for c in listed():
        w = work(c)
        m = most.setdefault(c["kind"], [0.0, 0.0])
        m[0], m[1] = max(m[0], w["bytes"]), max(m[1], w["flops"])
    kind = rng.choice(["pack", "attend", "attend", "prompt", "select", "select", "reorder"])
    while True:
        dtype = "f32" if rng.random() < 0.2 else "bf16"
        Hq, Hkv, D = rng.choice(_HEADS_F32 if dtype == "f32" else _HEADS_BF16)
        c = dict(kind=kind, dtype=dtype)
        if kind == "pack":
            c.update(B=_log(rng, 1, 32), n_ctx=rng.choice([0, rng.randint(1, 300)]), n_new=1 if rng.random() < 0.25 else _log(rng, 1, 4096),
                     Hkv=Hkv, D=D)
        elif kind == "attend":
            c.update(B=_log(rng, 1, 32), n=_log(rng, 1, 2048 if dtype == "f32" else 32768), Hq=Hq, Hkv=Hkv, D=D, ragged=rng.random() < 0.2)
        elif kind == "prompt":
            n = _log(rng, 1, 512 if dtype == "f32" else 4096)
            c.update(B=_log(rng, 1, 8), n=n, T=n if rng.random() < 0.5 else _log(rng, 1, n), Hq=Hq, Hkv=Hkv, D=D)
        elif kind == "select":
            W = _log(rng, 1, 32)
            c.update(dtype="f32" if rng.random() < 0.4 else "bf16", R=_log(rng, 1, 16), W=W, V=_log(rng, 100, 131072),
                     K=rng.choice([W, 2 * W]), pad=rng.choice([0, rng.randint(1, 64)]), first=rng.random() < 0.2)
        else:
            W, n = _log(rng, 2, 16), _log(rng, 8, 4096)
            c.update(slots=_log(rng, 1, 8), R=_log(rng, 1, 8), W=W, moved=rng.randint(1, W - 1), Hkv=Hkv, D=D, n=n,
                     first=rng.choice([0, rng.randint(0, n - 1)]), fork=False)
        w = work(c)
        # a drawn case costs no more than the largest listed one of its kind; reordered caches stay within 2 GB
        if w["bytes"] <= most[kind][0] and w["flops"] <= most[kind][1]:
            if kind != "reorder" or 2 * c["slots"] * c["R"] * W * Hkv * n * D * (4 if dtype == "f32" else 2) <= 2 << 30:
                return c


def work(c):
    e = 4 if c["dtype"] == "f32" else 2
    kind = c["kind"]
    if kind == "select":
        # per logit: compare, subtract, exp, add
        return {"bytes": float(c["R"] * c["W"] * (c["V"] * e + 4) + 12 * c["R"] * c["K"]), "flops": 4.0 * c["R"] * c["W"] * c["V"]}
    D, Hkv = c["D"], c["Hkv"]
    packed = D // 2 + 16                     # bytes of a row of a 4-bit cache: the codes, four pairs of bf16
    if kind == "reorder":
        # sources that somebody else takes are read once, the sequences that change are written once
        seqs = c["R"] * (min(c["moved"], c["W"] - c["moved"]) + c["moved"])
        return {"bytes": 2.0 * c["slots"] * seqs * Hkv * (c["n"] - c["first"]) * D * e + 4 * c["R"] * c["W"], "flops": 0.0}
    if kind == "pack":
        rows = 2.0 * c["B"] * c["n_new"] * Hkv
        # the tokens in, the cache's rows written, their values out; per element: smallest, largest, subtract, scale, round, back
        return {"bytes": rows * (2 * D * e + packed), "flops": 6.0 * rows * D}
    B, n, Hq = c["B"], c["n"], c["Hq"]
    if kind == "attend":
        return {"bytes": 2.0 * B * Hkv * n * packed + B * Hq * D * (e + 4), "flops": 4.0 * B * Hq * n * D}
    T = c["T"]
    return {"bytes": 2.0 * B * Hkv * n * packed + B * T * Hq * D * (e + 4), "flops": 4.0 * B * Hq * D * T * (n - (T - 1) / 2)}


# ---------------------------------------------------------------------------------------------- inputs


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(g, dtype, *shape):
    return torch.randn(*shape, device="cuda", generator=g, dtype=torch.float32).to(DTYPES[dtype])


def _kv(g, c, n):
    """New tokens' k, v [B][n][Hkv][D]: keys have channels of different size and offset, as trained models' do."""
    Hkv, D = c["Hkv"], c["D"]
    out = []
    for spread in (True, False):
        x = torch.randn(c["B"], n, Hkv, D, device="cuda", generator=g)
        if spread:
            x *= torch.rand(Hkv, D, device="cuda", generator=g) * 1.5 + 0.25
            x += torch.randn(Hkv, D, device="cuda", generator=g)
        out.append(x.to(DTYPES[c["dtype"]]))
    return out


def _lengths(c, seed):
    """Ragged caches: how many rows every (sequence, kv-head) keeps, and which (ascending, padded with row 0)."""
    g = torch.Generator().manual_seed(seed)
    lens = torch.randint(1, c["n"] + 1, (c["B"], c["Hkv"]), generator=g)
    rows = torch.rand(c["B"], c["Hkv"], c["n"], generator=g).argsort(-1)
    real = torch.arange(c["n"]) < lens[..., None]
    rows = torch.where(real, rows, c["n"]).sort(-1).values
    return lens, torch.where(real, rows, 0).int().cuda()


def _parents(c, seed):
    """The sequence every sequence continues: of a request's beams some go on as they are and the others continue one of
    those (fork: all continue the first)."""
    R, W, moved = c["R"], c["W"], c["moved"]
    g = torch.Generator().manual_seed(seed)
    parent = torch.arange(R * W).view(R, W)
    for r in range(R):
        order = torch.arange(W - 1, -1, -1) if c["fork"] else torch.randperm(W, generator=g)
        gone, stay = order[:moved], order[moved:]
        parent[r, gone] = r * W + stay[torch.arange(moved) % (W - moved)]
    return parent.view(-1).int().cuda()


def prepare(c, seed):
    g = _gen(seed)
    s = dict(c)
    kind = c["kind"]
    if kind == "select":
        R, W, V = c["R"], c["W"], c["V"]
        # logits as language models give them: many small ones, a few likely tokens; 2 % of the vocabulary is masked
        x = torch.randn(R * W, V, device="cuda", generator=g) * 2
        x += torch.rand(R * W, V, device="cuda", generator=g).pow(64) * 12
        x.masked_fill_(torch.rand(V, device="cuda", generator=g) < 0.02, float("-inf"))
        room = torch.full((R * W, V + c["pad"]), float("nan"), device="cuda", dtype=DTYPES[c["dtype"]])
        room[:, :V] = x
        s["logits"] = room[:, :V]
        score = -torch.rand(R, W, device="cuda", generator=g).mul(20).sort(-1).values
        if c["first"]:                       # the first step: the beams are still the same, only one of them counts
            score[:, 1:] = float("-inf")
            score[:, 0] = 0
        s["scores"] = score.flatten()
        if own:
            from paper_2410_18517_b200 import SharedKVCache

            s["cache"] = SharedKVCache(1, 2, 2, 64, R * W, 16, "bf16")
        return s
    B = s.setdefault("B", c.get("R", 1) * c.get("W", 1))
    if kind == "reorder":
        s["parent"] = _parents(c, seed)
        planes = [_normal(g, c["dtype"], B, c["n"], c["Hkv"], c["D"]) for _ in range(2 * c["slots"])]
        if own:
            from paper_2410_18517_b200 import SharedKVCache

            s["cache"] = SharedKVCache(c["slots"], c["Hkv"], c["Hkv"], c["D"], B, c["n"], c["dtype"])
            for i in range(c["slots"]):
                s["cache"].append(i, planes[2 * i], planes[2 * i + 1])
        else:
            s["planes"] = [x.transpose(1, 2).contiguous() for x in planes]
        return s
    n_ctx = c["n_ctx"] if kind == "pack" else c["n"]
    k, v = _kv(g, dict(c, B=B), n_ctx)
    if kind == "pack":
        s["k"], s["v"] = _kv(g, c, c["n_new"])
    elif kind == "attend":
        s["q"] = _normal(g, c["dtype"], B, c["Hq"], c["D"])
    else:
        s["q"] = _normal(g, c["dtype"], B, c["T"], c["Hq"], c["D"])
    if c.get("ragged"):
        s["lens"], s["keep"] = _lengths(c, seed)
    if own:
        from paper_2410_18517_b200 import SharedKVCache

        cache = s["cache"] = SharedKVCache(1, c.get("Hq", c["Hkv"]), c["Hkv"], c["D"], B, n_ctx + c.get("n_new", 0), c["dtype"],
                                           cache_format="4bit")
        if n_ctx:
            cache.append(0, k, v)
        if c.get("ragged"):
            cache.evict(0, s["keep"], s["lens"])
    elif kind != "pack":
        s["K"], s["V"] = (_plain_store(x, s.get("keep")) for x in (k, v))
    return s


# ------------------------------------------------------------------------------------- the plain forms


def _plain_pack(x):
    """x [..., D] -> codes, scales and offsets (float32 tensors that hold bf16 values), groups apart."""
    x = x.float().unflatten(-1, (4, -1))
    lo, hi = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
    step = (hi - lo) / 15
    s = ((step.view(torch.int32) + 0xFFFF) & ~0xFFFF).view(torch.float32)
    b = (lo - 16 * s).bfloat16().float()
    # in 64 bits: a value next to the border between two codes
    c = (((x.double() - b.double()) / s.double()).round() - 16).clamp(0, 15)
    return torch.where(s > 0, c, 0.0), s, b


def _plain_values(c, s, b, dtype):
    return (s.double() * (16 + c.double()) + b.double()).flatten(-2).to(dtype)


def _plain_store(x, keep):
    """The 4-bit rows a program keeps: [B][Hkv][n], two codes per byte."""
    x = x.transpose(1, 2)
    if keep is not None:
        x = x.gather(2, keep.long()[..., None].expand_as(x))
    parts = [_plain_pack(one) for one in x]          # a sequence at a time: temporaries are eight bytes an element
    c, s, b = (torch.stack(t) for t in zip(*((c.to(torch.uint8), s.bfloat16(), b.bfloat16()) for c, s, b in parts)))
    return c[..., 0::2] | c[..., 1::2] << 4, s, b


def _plain_load(stored, dtype):
    packed, s, b = stored
    c = torch.stack((packed & 15, packed >> 4), -1).flatten(-2)
    return (s.float() * (16 + c.float()) + b.float()).flatten(-2).to(dtype).float()


def _plain_attention(q, K, V, sees):
    """q [B][T][Hq][D]; K, V [B][Hkv][n][D]; sees: None or [B or 1][Hkv or 1][T][1][n]."""
    B, T, Hq, D = q.shape
    Hkv, n = K.shape[1], K.shape[2]
    x = q.float().view(B, T, Hkv, Hq // Hkv, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, -1, D)
    a = (x @ K.transpose(2, 3) * D ** -0.5).view(B, Hkv, T, Hq // Hkv, n)
    if sees is not None:
        a = a.masked_fill(~sees, float("-inf"))
    p = torch.exp(a - a.amax(-1, keepdim=True))
    p = p / p.sum(-1, keepdim=True)
    o = p.view(B, Hkv, -1, n) @ V
    return o.view(B, Hkv, T, Hq // Hkv, D).permute(0, 2, 1, 3, 4).reshape(B, T, Hq, D)


def _plain_select(s):
    R, W, V, K = s["R"], s["W"], s["V"], s["K"]
    x = s["logits"].double()
    m = x.amax(-1, keepdim=True)
    lse = m + torch.log(torch.exp(x - m).sum(-1, keepdim=True))
    total = (s["scores"].double()[:, None] - lse + x).view(R, W * V)
    total = torch.where(total > float("-inf"), total, float("-inf"))
    order = torch.sort(total, dim=-1, descending=True, stable=True)
    score, at = order.values[:, :K], order.indices[:, :K]
    real = score > float("-inf")
    first = torch.arange(R, device="cuda")[:, None] * W
    return score.float(), torch.where(real, at % V, -1).int(), (first + torch.where(real, at // V, 0)).int()


def run(s):
    kind = s["kind"]
    if kind == "select":
        if own:
            return s["cache"].beam_select(s["logits"], s["scores"], s["W"], s["K"])
        return _plain_select(s)
    if kind == "reorder":
        if own:
            cache = s["cache"]
            cache.reorder(s["parent"], s["first"])
            return [cache.plane(i, kv)[:, :, :s["n"]] for i in range(s["slots"]) for kv in range(2)]
        for x in s["planes"]:
            x[:, :, s["first"]:] = x[s["parent"].long(), :, s["first"]:]
        return s["planes"]
    if kind == "pack":
        if own:
            cache = s["cache"]
            cache.truncate(s["n_ctx"])         # the step starts from the context, whatever ran before
            cache.append(0, s["k"], s["v"])
            return cache.read_rows(0, s["n_ctx"], s["n_new"])
        return tuple(_plain_values(*_plain_pack(x), x.dtype) for x in (s["k"], s["v"]))
    if own:
        return s["cache"].decode_attention(0, s["q"]) if kind == "attend" else s["cache"].prefill_attention(0, s["q"])
    K, V = (_plain_load(s[x], DTYPES[s["dtype"]]) for x in ("K", "V"))
    if kind == "attend":
        sees = None
        if s["ragged"]:
            sees = (torch.arange(s["n"]) < s["lens"][..., None])[:, :, None, None].cuda()
        return _plain_attention(s["q"][:, None], K, V, sees)[:, 0]
    T, n = s["T"], s["n"]
    sees = torch.arange(n, device="cuda") <= torch.arange(n - T, n, device="cuda")[:, None]
    return torch.cat([_plain_attention(s["q"][i:i + 1], K[i:i + 1], V[i:i + 1], sees[None, None, :, None]) for i in range(s["B"])])


# ------------------------------------------------------------------------------- the definitions in 64 bits


def _exact_values(x):
    """[rows][D] -> the values of the codes, not yet rounded to the storage type."""
    rows, D = x.shape
    out = torch.empty(rows, D, dtype=torch.float64, device="cuda")
    for i in range(4):
        part = x[:, i * D // 4:(i + 1) * D // 4].float()
        lo, hi = part.min(1).values, part.max(1).values
        step = (hi - lo) / 15.0                                    # fp32, as the definition says
        down = step.bfloat16()
        up = torch.nextafter(down, torch.full_like(down, float("inf")))
        s = torch.where(down.float() >= step, down, up)
        b = (lo - s.float() * 16.0).bfloat16()
        s, b = s.double()[:, None], b.double()[:, None]
        code = torch.where(s == 0, 0.0, torch.round((part.double() - b) / s.clamp(min=1e-300)) - 16)
        out[:, i * D // 4:(i + 1) * D // 4] = b + s * 16 + s * code.clamp(0, 15)
    return out


def exact(c, seed):
    global own
    kind = c["kind"]
    if kind not in ("attend", "prompt"):
        was, own = own, False
        try:
            s = prepare(c, seed)
        finally:
            own = was
    if kind == "reorder":
        old, parent = s["planes"], s["parent"].tolist()
        return [torch.stack([torch.cat((x[b, :, :c["first"]], x[parent[b], :, c["first"]:]), 1) for b in range(len(parent))]).double()
                for x in old]
    if kind == "select":
        R, W, V, K = c["R"], c["W"], c["V"], c["K"]
        best = torch.empty(R, K, dtype=torch.float64, device="cuda")
        for r in range(R):
            rows = [s["scores"][i].double() + torch.log_softmax(s["logits"][i].double(), 0) for i in range(r * W, (r + 1) * W)]
            every = torch.nan_to_num(torch.cat(rows + [torch.full((K,), -math.inf, dtype=torch.float64, device="cuda")]), nan=-math.inf)
            best[r] = torch.topk(every, K).values
        return best, None, None
    if kind == "pack":
        return tuple(_exact_values(x.flatten(0, 2)).view(x.shape) for x in (s["k"], s["v"]))
    # attention: the same draws as prepare makes, packed and attended to one (sequence, kv-head) at a time
    g = _gen(seed)
    k, v = _kv(g, c, c["n"])
    B, Hq, Hkv, D, n = c["B"], c["Hq"], c["Hkv"], c["D"], c["n"]
    T = c.get("T", 1)
    q = _normal(g, c["dtype"], *((B, Hq, D) if kind == "attend" else (B, T, Hq, D))).view(B, T, Hq, D)
    G = Hq // Hkv
    lens, keep = _lengths(c, seed) if c.get("ragged") else (None, None)
    out = torch.zeros(B, T, Hq, D, dtype=torch.float64, device="cuda")
    hidden = torch.ones(T, n, dtype=torch.bool, device="cuda").triu(n - T + 1) if kind == "prompt" else None
    for b in range(B):
        for h in range(Hkv):
            kr, vr = k[b, :, h], v[b, :, h]
            if keep is not None:
                at = keep[b, h, :int(lens[b, h])].long()
                kr, vr = kr[at], vr[at]
            kr, vr = (_exact_values(x).to(DTYPES[c["dtype"]]).double() for x in (kr, vr))
            for j in range(h * G, (h + 1) * G):
                a = q[b, :, j].double() @ kr.T / math.sqrt(D)
                if hidden is not None:
                    a = torch.where(hidden, -math.inf, a)
                out[b, :, j] = a.softmax(-1) @ vr
    return out[:, 0] if kind == "attend" else out
