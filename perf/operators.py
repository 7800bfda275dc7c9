"""Cases of the cache-side serving operators: what is timed, on which inputs, and what each computes.

Five kinds of pass over a layer's cache slot (layouts as in include/kvs.h):

  rotary   new tokens enter the cache: per-head RMS norm of queries and keys, rotary positions, K/V stored
  tree     attention of a tree of drafted tokens (the newest rows of the cache) over the whole cache
  verify   one verification step of one layer: drafts enter (rotary), tree attention, the accepted path stays
  weights  decode attention that also adds every cached row's softmax weight to a running total
  select   the rows a budget keeps: the newest ones and those with the largest totals

With ``own`` false ``run`` computes a pass in elementary torch operations; with ``own`` true it makes the calls a
program makes of this package.  ``exact`` restates the definitions in float64.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # one decode step's tokens of a grouped-query model: launch latency is what counts
        dict(name="rotary_decode_b8", kind="rotary", dtype="bf16", B=8, n_ctx=4096, n_new=1, Hq=32, Hkv=8, D=128,
             rot=128, interleaved=False, norm=True, fused=True, far=0),
        # a prompt chunk of four long sequences: a streaming pass over 400 MB
        dict(name="rotary_prompt_b4", kind="rotary", dtype="bf16", B=4, n_ctx=0, n_new=4096, Hq=32, Hkv=8, D=128,
             rot=128, interleaved=False, norm=True, fused=True, far=0),
        # fp32 storage, odd token count, partial interleaved rotation at far positions
        dict(name="rotary_f32_partial", kind="rotary", dtype="f32", B=3, n_ctx=129, n_new=1037, Hq=4, Hkv=4, D=64,
             rot=32, interleaved=True, norm=False, fused=False, far=900000),
        # one user, a handful of drafts over a short odd context: latency
        dict(name="tree_b1_n1031_t5", kind="tree", dtype="bf16", B=1, n_ctx=1031, n_t=5, Hq=32, Hkv=8, D=128, pad=False),
        # a batch on a model without grouped heads, sequences with different numbers of drafts (padded)
        dict(name="tree_mha_b8_n4096_t16", kind="tree", dtype="bf16", B=8, n_ctx=4096, n_t=16, Hq=32, Hkv=32, D=128, pad=True),
        # the largest trees over long contexts: 256 query rows for every cached row
        dict(name="tree_gqa_b4_n32768_t64", kind="tree", dtype="bf16", B=4, n_ctx=32768, n_t=64, Hq=32, Hkv=8, D=128, pad=False),
        # the small fp32 configuration, one verification step
        dict(name="verify_f32_b2_n128_t7", kind="verify", dtype="f32", B=2, n_ctx=128, n_t=7, n_acc=3, Hq=4, Hkv=4, D=64),
        # a verification step of a grouped-query batch
        dict(name="verify_gqa_b4_n8192_t32", kind="verify", dtype="bf16", B=4, n_ctx=8192, n_t=32, n_acc=5, Hq=32, Hkv=8, D=128),
        # decode with running totals: one short sequence, and the 13B shape
        dict(name="weights_b1_n1024", kind="weights", dtype="bf16", B=1, n=1024, Hq=32, Hkv=8, D=128),
        dict(name="weights_mha_b16_n8192", kind="weights", dtype="bf16", B=16, n=8192, Hq=40, Hkv=40, D=128),
        # which rows a budget keeps: one long sequence, and a batch with a budget of its own for every head
        dict(name="select_b1_n32768", kind="select", dtype="bf16", B=1, n=32768, Hq=32, Hkv=8, D=128, keep=4096, recent=512, ragged=False),
        dict(name="select_mha_b16_n8192", kind="select", dtype="bf16", B=16, n=8192, Hq=40, Hkv=40, D=128, keep=2048, recent=256, ragged=True),
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
    kind = rng.choice(["rotary", "tree", "tree", "verify", "weights", "select"])
    while True:
        dtype = "f32" if rng.random() < 0.2 else "bf16"
        Hq, Hkv, D = rng.choice(_HEADS_F32 if dtype == "f32" else _HEADS_BF16)
        c = dict(kind=kind, dtype=dtype, B=_log(rng, 1, 32), Hq=Hq, Hkv=Hkv, D=D)
        long = 2048 if dtype == "f32" else 32768
        if kind == "rotary":
            c.update(n_ctx=rng.choice([0, rng.randint(1, 300)]), n_new=1 if rng.random() < 0.25 else _log(rng, 1, 4096),
                     rot=rng.choice([D, D, D // 2]), interleaved=rng.random() < 0.4, norm=rng.random() < 0.7,
                     fused=rng.random() < 0.6, far=rng.choice([0, 0, 1000000]))
        elif kind == "tree":
            c.update(n_ctx=_log(rng, 1, long), n_t=_log(rng, 1, 64), pad=rng.random() < 0.4)
        elif kind == "verify":
            n_t = _log(rng, 2, 64)
            c.update(n_ctx=_log(rng, 1, min(long, 8192)), n_t=n_t, n_acc=rng.randint(1, n_t))
        elif kind == "weights":
            c.update(n=_log(rng, 1, long))
        else:
            n = _log(rng, 16, long)
            keep = rng.randint(max(1, n // 16), n)
            c.update(n=n, keep=keep, recent=rng.randint(0, min(keep, 512)), ragged=rng.random() < 0.5)
        w = work(c)
        # a drawn case costs no more than the largest listed one of its kind
        if w["bytes"] <= most[kind][0] and w["flops"] <= most[kind][1]:
            return c


def work(c):
    e = 4 if c["dtype"] == "f32" else 2
    B, Hq, Hkv, D = c["B"], c["Hq"], c["Hkv"], c["D"]
    if c["kind"] == "rotary":
        toks = B * c["n_new"]
        # norm: square, sum, scale, weight; rotation: 3 per rotated value
        return {"bytes": 2.0 * toks * (Hq + 2 * Hkv) * D * e + 4 * toks, "flops": 7.0 * toks * (Hq + Hkv) * D}
    if c["kind"] == "tree":
        n = c["n_ctx"] + c["n_t"]
        return {"bytes": 2.0 * B * Hkv * n * D * e + 2.0 * B * c["n_t"] * Hq * D * e + 8 * B * c["n_t"],
                "flops": 4.0 * B * Hq * c["n_t"] * D * (c["n_ctx"] + 1)}
    if c["kind"] == "verify":
        n = c["n_ctx"] + c["n_t"]
        # the drafts' q, k, v in; the cache read once; the result and the accepted rows out
        return {"bytes": B * (2.0 * Hkv * n + c["n_t"] * (2 * Hq + 2 * Hkv) + 2 * Hkv * c["n_acc"]) * D * e,
                "flops": 4.0 * B * Hq * c["n_t"] * D * (c["n_ctx"] + 1)}
    if c["kind"] == "weights":
        n = c["n"]
        return {"bytes": 2.0 * B * Hkv * n * D * e + B * Hq * D * (e + 4) + 8.0 * B * Hkv * n, "flops": 4.0 * B * Hq * n * D}
    n, U = c["n"], B * Hkv
    return {"bytes": 4.0 * U * n + 8.0 * U * c["keep"], "flops": 2.0 * U * n}


# ---------------------------------------------------------------------------------------------- inputs


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(g, dtype, *shape):
    return torch.randn(*shape, device="cuda", generator=g, dtype=torch.float32).to(DTYPES[dtype])


def _inv_freq(rot):
    return [10000.0 ** (-2.0 * i / rot) for i in range(rot // 2)]


def _qkv(g, c, n):
    """New tokens' q, k, v [B][n][heads][D]: slices of one projection's output, or three tensors."""
    B, Hq, Hkv, D = c["B"], c["Hq"], c["Hkv"], c["D"]
    if c.get("fused", True):
        x = _normal(g, c["dtype"], B, n, (Hq + 2 * Hkv), D)
        return x[:, :, :Hq], x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:]
    return tuple(_normal(g, c["dtype"], B, n, h, D) for h in (Hq, Hkv, Hkv))


def _tree(seed, B, n_t, pad):
    """Random draft trees: token i's parent is an earlier token or the context.  Returns the visibility masks
    (int64 words, bit j: token i sees token j) and every token's depth.  With `pad` a sequence has only some real
    tokens; the others see none and are seen by none."""
    g = torch.Generator().manual_seed(seed)
    parent = (torch.rand(B, n_t, generator=g) * (torch.arange(n_t) + 1)).long() - 1          # -1 .. i-1
    real = torch.randint(1, n_t + 1, (B,), generator=g) if pad else torch.full((B,), n_t)
    mask, depth = torch.zeros(B, n_t + 1, dtype=torch.int64), torch.full((B, n_t + 1), -1)
    rows = torch.arange(B)
    for i in range(n_t):
        p = torch.where(parent[:, i] < 0, n_t, parent[:, i])                                # column n_t: the context
        bit = (1 << i) if i < 63 else -(1 << 63)
        mask[:, i] = torch.where(i < real, mask[rows, p] | bit, 0)
        depth[:, i] = depth[rows, p] + 1
    return mask[:, :n_t].contiguous().cuda(), depth[:, :n_t].int().contiguous().cuda()


def _cache(c, k, v, max_seq):
    """The cache a program holds: one layer's slot filled with k, v [B][n][Hkv][D]."""
    from paper_2410_18517_b200 import SharedKVCache

    cache = SharedKVCache(1, c["Hq"], c["Hkv"], c["D"], c["B"], max_seq, c["dtype"])
    if k is not None and k.shape[1]:
        cache.append(0, k, v)
    return cache


def prepare(c, seed):
    g = _gen(seed)
    s = dict(c)
    B, Hq, Hkv, D, kind = c["B"], c["Hq"], c["Hkv"], c["D"], c["kind"]
    if kind in ("rotary", "verify"):
        n_new = c["n_new"] if kind == "rotary" else c["n_t"]
        s["q"], s["k"], s["v"] = _qkv(g, c, n_new)
        rot = c.get("rot", D)
        s["inv_freq"] = _inv_freq(rot)
        s["freq64"] = torch.tensor(s["inv_freq"], dtype=torch.float64, device="cuda")
        if kind == "rotary":
            first = c["n_ctx"] + (torch.randint(0, c["far"], (B, 1), device="cuda", generator=g, dtype=torch.int32) if c["far"] else 0)
            s["pos"] = (first + torch.arange(n_new, device="cuda", dtype=torch.int32)[None]).expand(B, n_new).contiguous()
        else:
            s["mask"], depth = _tree(seed, B, n_new, False)
            s["pos"] = depth + c["n_ctx"]
            # the accepted path: draft numbers in ascending order, as many for every sequence
            s["path"] = torch.rand(B, n_new, device="cuda", generator=g).argsort(1)[:, :c["n_acc"]].sort(1).values.int().contiguous()
        norm = c.get("norm", True)
        s["qw"] = 1 + 0.1 * _normal(g, c["dtype"], D) if norm else None
        s["kw"] = 1 + 0.1 * _normal(g, c["dtype"], D) if norm else None
        ctx = c["n_ctx"]
        kc, vc = (_normal(g, c["dtype"], B, ctx, Hkv, D) for _ in range(2))
        if own:
            from paper_2410_18517_b200 import Rotary

            s["cache"] = _cache(c, kc, vc, ctx + n_new)
            s["rotary"] = Rotary(s["inv_freq"], interleaved=c.get("interleaved", False))
        else:
            s["K"], s["V"] = (x.transpose(1, 2).contiguous() for x in (kc, vc))
        return s
    if kind == "tree":
        n = c["n_ctx"] + c["n_t"]
        s["q"] = _normal(g, c["dtype"], B, c["n_t"], Hq, D)
        s["mask"], _ = _tree(seed, B, c["n_t"], c["pad"])
    else:
        n = c["n"]
        s["q"] = _normal(g, c["dtype"], B, Hq, D)
    if kind == "select":
        # running totals as decoding leaves them: most rows small, a few large, many exactly equal
        w = torch.rand(B, Hkv, n, device="cuda", generator=g).pow(6) * 40
        s["weight"] = torch.where(torch.rand(B, Hkv, n, device="cuda", generator=g) < 0.5, (w * 64).floor() / 64, w)
        u = torch.Generator().manual_seed(seed)
        lo = max(c["recent"], 1, c["keep"] // 2)
        s["n_keep"] = (torch.randint(lo, c["keep"] + 1, (B, Hkv), generator=u) if c["ragged"] else torch.full((B, Hkv), c["keep"])).int()
        s["keep_rows"] = torch.full((B, Hkv, c["keep"]), -1, dtype=torch.int32, device="cuda")
        s["kept"] = torch.zeros(B, Hkv, c["keep"], device="cuda")
        if own:
            z = torch.zeros(B, n, Hkv, D, dtype=DTYPES[c["dtype"]], device="cuda")
            s["cache"] = _cache(c, z, z, n)
        return s
    k, v = (_normal(g, c["dtype"], B, n, Hkv, D) for _ in range(2))
    if kind == "weights":
        # totals of a few steps that have already been counted
        s["total"] = torch.rand(B, Hkv, n, device="cuda", generator=g) * (8.0 * Hq / Hkv / n)
        s["total_out"] = torch.empty_like(s["total"])
    if own:
        s["cache"] = _cache(c, k, v, n)
    else:
        s["K"], s["V"] = (x.transpose(1, 2).contiguous() for x in (k, v))
    return s


# ------------------------------------------------------------------------------------- the plain forms


def _plain_norm_rope(x, w, pos, freq, interleaved):
    x = x.float()
    if w is not None:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) * w.float()
    r = 2 * freq.numel()
    a = pos.double()[:, :, None, None] * freq
    cos, sin = a.cos().float(), a.sin().float()
    if interleaved:
        x0, x1 = x[..., 0:r:2], x[..., 1:r:2]
        y = torch.stack((x0 * cos - x1 * sin, x1 * cos + x0 * sin), -1).flatten(-2)
    else:
        x0, x1 = x[..., : r // 2], x[..., r // 2 : r]
        y = torch.cat((x0 * cos - x1 * sin, x1 * cos + x0 * sin), -1)
    return torch.cat((y, x[..., r:]), -1)


def _plain_rotary(s):
    q, k = (_plain_norm_rope(s[x], s[x + "w"], s["pos"], s["freq64"], s.get("interleaved", False)).to(s[x].dtype) for x in ("q", "k"))
    return q, k.transpose(1, 2), s["v"].transpose(1, 2)


def _plain_tree(q, K, V, mask, n_t):
    B, T, Hq, D = q.shape
    Hkv, n = K.shape[1], K.shape[2]
    x = q.float().view(B, T, Hkv, Hq // Hkv, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, -1, D)
    a = (x @ K.float().transpose(2, 3) * D ** -0.5).view(B, Hkv, T, Hq // Hkv, n)
    sees = (mask[:, :, None] >> torch.arange(n_t, device=q.device)) & 1 == 1
    a[..., n - n_t:].masked_fill_(~sees[:, None, :, None], float("-inf"))
    p = torch.exp(a - a.amax(-1, keepdim=True))
    p = p / p.sum(-1, keepdim=True)
    o = p.view(B, Hkv, -1, n) @ V.float()
    return o.view(B, Hkv, T, Hq // Hkv, D).permute(0, 2, 1, 3, 4).reshape(B, T, Hq, D).to(q.dtype)


def _plain_verify(s):
    q, k, v = _plain_rotary(s)
    out = _plain_tree(q, torch.cat((s["K"], k), 2), torch.cat((s["V"], v), 2), s["mask"], s["n_t"])
    at = s["path"].long()[:, None, :, None].expand(-1, s["Hkv"], -1, s["D"])
    return out, k.gather(2, at), v.gather(2, at)


def _plain_weights(s):
    q, K, V = s["q"], s["K"], s["V"]
    B, Hq, D = q.shape
    a = q.float().view(B, K.shape[1], -1, D) @ K.float().transpose(2, 3) * D ** -0.5
    p = torch.exp(a - a.amax(-1, keepdim=True))
    p = p / p.sum(-1, keepdim=True)
    return (p @ V.float()).view(B, Hq, D), s["total"] + p.sum(2)


def _plain_select(s):
    w, n, kmax = s["weight"], s["n"], s["keep"]
    u = w.clone()
    u[..., n - s["recent"]:] = float("inf")
    order = torch.sort(u, dim=-1, descending=True, stable=True).indices
    n_keep = s["n_keep"].cuda()[..., None]
    chosen = torch.zeros_like(w, dtype=torch.bool).scatter_(2, order, torch.arange(n, device="cuda") < n_keep)
    rows = torch.where(chosen, torch.arange(n, device="cuda"), n).sort(-1).values[..., :kmax]
    real = torch.arange(kmax, device="cuda") < n_keep
    rows = torch.where(real, rows, -1)
    return rows.int(), torch.where(real, w.gather(2, rows.clamp(min=0)), 0.0)


def run(s):
    kind = s["kind"]
    if own:
        cache = s["cache"]
        if kind in ("rotary", "verify"):
            ctx = s["n_ctx"]
            cache.truncate(ctx)            # the step starts from the context, whatever ran before
            q = cache.append_rotary(0, s["q"], s["k"], s["v"], s["pos"], s["rotary"], s["qw"], s["kw"], eps=1e-6)
            if kind == "rotary":
                end = ctx + s["n_new"]
                return q, cache.plane(0, 0)[:, :, ctx:end], cache.plane(0, 1)[:, :, ctx:end]
            out = cache.tree_attention(0, q, s["mask"])
            cache.accept_draft(s["path"], [s["n_acc"]] * s["B"], s["n_t"])
            end = ctx + s["n_acc"]
            return out, cache.plane(0, 0)[:, :, ctx:end], cache.plane(0, 1)[:, :, ctx:end]
        if kind == "tree":
            return cache.tree_attention(0, s["q"], s["mask"])
        if kind == "weights":
            out = cache.decode_attention_weights(0, s["q"], s["total"], s["total_out"])
            return out, s["total_out"]
        cache.select_rows(0, s["weight"], s["n_keep"], s["recent"], s["keep_rows"], s["kept"])
        return s["keep_rows"], s["kept"]
    if kind == "rotary":
        return _plain_rotary(s)
    if kind == "tree":
        return _plain_tree(s["q"], s["K"], s["V"], s["mask"], s["n_t"])
    if kind == "verify":
        return _plain_verify(s)
    return _plain_weights(s) if kind == "weights" else _plain_select(s)


# ------------------------------------------------------------------------------- the definitions in 64 bits


def _exact_rope(x, w, s):
    x = x.double()
    if w is not None:
        x = x / (x.pow(2).sum(-1, keepdim=True) / x.shape[-1] + 1e-6).sqrt() * w.double()
    y = x.clone()
    half = len(s["inv_freq"])
    for i, f in enumerate(s["inv_freq"]):
        a, b = (2 * i, 2 * i + 1) if s.get("interleaved") else (i, i + half)
        turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), s["pos"].double() * f)[..., None]
        z = torch.complex(x[..., a], x[..., b]) * turn
        y[..., a], y[..., b] = z.real, z.imag
    return y


def _exact_attention(q, K, V, sees):
    """q [B][T][Hq][D]; sees [B][T][n] or None.  One (sequence, kv-head) at a time."""
    B, T, Hq, D = q.shape
    G = Hq // K.shape[1]
    out = torch.zeros(B, T, Hq, D, dtype=torch.float64, device="cuda")
    p_sum = torch.zeros(B, K.shape[1], K.shape[2], dtype=torch.float64, device="cuda")
    for b in range(B):
        for h in range(K.shape[1]):
            a = torch.einsum("tgd,nd->tgn", q[b, :, h * G:(h + 1) * G].double(), K[b, h].double()) / math.sqrt(D)
            if sees is not None:
                a = torch.where(sees[b][:, None], a, -math.inf)
            p = a.softmax(-1)
            out[b, :, h * G:(h + 1) * G] = torch.einsum("tgn,nd->tgd", p, V[b, h].double())
            p_sum[b, h] = p.sum((0, 1))
    return out, p_sum


def _sees(mask, n_ctx, n_t):
    bits = torch.stack([(mask >> j) % 2 != 0 for j in range(n_t)], -1)
    return torch.cat((torch.ones(*bits.shape[:2], n_ctx, dtype=torch.bool, device="cuda"), bits), -1)


def exact(c, seed):
    global own
    was, own = own, False
    try:
        s = prepare(c, seed)
    finally:
        own = was
    kind = c["kind"]
    if kind == "select":
        weight, n_keep, n = s["weight"].cpu(), s["n_keep"], c["n"]
        kept = torch.zeros(c["B"], c["Hkv"], c["keep"], dtype=torch.float64)
        for b in range(c["B"]):
            for h in range(c["Hkv"]):
                old, want = n - c["recent"], int(n_keep[b, h])
                best = torch.argsort(-weight[b, h, :old].double(), stable=True)[: want - c["recent"]]
                rows = torch.cat((best.sort().values, torch.arange(old, n)))
                kept[b, h, :want] = weight[b, h, rows].double()
        return None, kept
    if kind == "weights":
        out, p_sum = _exact_attention(s["q"][:, None], s["K"], s["V"], None)
        return out[:, 0], s["total"].double() + p_sum
    if kind == "tree":
        return _exact_attention(s["q"], s["K"], s["V"], _sees(s["mask"], c["n_ctx"], c["n_t"]))[0]
    q, k = _exact_rope(s["q"], s["qw"], s), _exact_rope(s["k"], s["kw"], s).transpose(1, 2)
    if kind == "rotary":
        return q, k, s["v"].double().transpose(1, 2)
    # the cache and the queries hold the storage type: rounded once on the way in
    q, k = q.to(s["q"].dtype).double(), k.to(s["q"].dtype).double()
    v = s["v"].double().transpose(1, 2)
    out, _ = _exact_attention(q, torch.cat((s["K"].double(), k), 2), torch.cat((s["V"].double(), v), 2),
                              _sees(s["mask"], c["n_ctx"], c["n_t"]))
    at = s["path"].long()
    pick = lambda x: torch.stack([x[b][:, at[b]] for b in range(c["B"])])  # noqa: E731
    return out, pick(k), pick(v)
