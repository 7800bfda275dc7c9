"""The row of a 4-bit cache, beam selection and reordering, restated with plain loops or float64; shares nothing with the
library.

Rows: s and b are what the definition says in fp32 steps; codes are settled in exact rational arithmetic where float64 could
not tell (it can: elements and parameters have at most 24 bits, and exponents that are close)."""
import math

import torch


def up_to_bf16(x):
    """float32 >= 0 -> the smallest bf16 that is not below it (as float32)."""
    y = x.bfloat16()
    return torch.where(y.float() < x, torch.nextafter(y, torch.full_like(y, math.inf)), y).float()


def pack(x):
    """x [..., D] (CPU) -> codes int64 [..., 4, D/4], s and b float32 [..., 4, 1] (NaN: a group without values)."""
    g = x.float().reshape(*x.shape[:-1], 4, x.shape[-1] // 4)
    broken = ~torch.isfinite(g).all(-1, keepdim=True)
    clean = torch.where(broken, 0.0, g)
    lo, hi = clean.amin(-1, keepdim=True), clean.amax(-1, keepdim=True)
    step = (hi - lo) * torch.tensor(1 / 15)          # both fp32
    s = up_to_bf16(step)
    b = (lo - 16 * s).bfloat16().float()
    broken |= ~(torch.isfinite(step) & torch.isfinite(s) & torch.isfinite(b))
    q = (clean.double() - b.double()) / torch.where(s > 0, s, 1.0).double()
    c = torch.where(s > 0, q.round() - 16, 0.0).clamp(0, 15)
    c = torch.where(broken, 0.0, c).long()
    nan = torch.full_like(s, math.nan)
    return c, torch.where(broken, nan, s), torch.where(broken, nan, b)


def values(x):
    """What a 4-bit cache holds of x [..., D], in x's type (x on the CPU)."""
    c, s, b = pack(x)
    v = s.double() * (16 + c.double()) + b.double()
    return v.reshape(x.shape).to(x.dtype)


def row_bytes(x):
    """The bytes of the rows of x [..., D]: uint8 [..., 16 + D/2]."""
    c, s, b = pack(x)
    pair = torch.cat((s, b), -1)                                                                # [..., 4, 2]
    pair = torch.where(pair.isnan(), 0x7FC0, pair.bfloat16().view(torch.int16)).to(torch.int16)    # a NaN is the quiet one
    head = pair.contiguous().view(torch.uint8).flatten(-2)
    c = c.flatten(-2).to(torch.uint8)
    return torch.cat((head, c[..., 0::2] | c[..., 1::2] << 4), -1)


def error_bound(x):
    """How far a value may be from x: half a step, the rounding of b, the value's own rounding (and that of s, fp32)."""
    c, s, b = pack(x)
    h = torch.finfo(x.dtype).eps / 2
    top = (s * 31).abs() + b.abs()
    e = s.double() / 2 * (1 + 2 ** -20) + b.double().abs() * 2 ** -8 + top.double() * h + 1e-45
    return e.expand(*e.shape[:-1], x.shape[-1] // 4).flatten(-2)


def beams(logits, scores, W, K):
    """Lists of (score float64, token, parent) per request, best first."""
    R, V = logits.shape[0] // W, logits.shape[1]
    out = []
    for r in range(R):
        total = torch.full((W, V), -math.inf, dtype=torch.float64)
        for w in range(W):
            x, s = logits[r * W + w].double().cpu(), float(scores[r * W + w])
            top = x.max()
            base = s - (x - top).exp().sum().log()
            if math.isfinite(float(base)):
                total[w] = base + (x - top)
        flat = total.flatten()
        order = sorted(torch.nonzero(flat > -math.inf).flatten().tolist(), key=lambda i: (-float(flat[i]), i))[:K] if flat.numel() < 5000 else \
            torch.sort(flat, descending=True, stable=True).indices[:K].tolist()
        best = [(float(flat[i]), i % V, r * W + i // V) for i in order if flat[i] > -math.inf]
        out.append(best + [(-math.inf, -1, r * W)] * (K - len(best)))
    return out
