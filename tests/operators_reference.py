"""The serving operators around the cache, restated in float64 with plain loops over (sequence, head), and the error
bounds their tests use.  Written from the definitions; shares nothing with the library.

Bounds.  With u = 2^-24 (half a step of fp32) and h = eps/2 of the output type:
  a score is a dot product of D terms and a scale: off by at most (D + 2) u * sum |q k| * scale =: d (natural log);
  a weight 2^(s - m) then by the factor e^(2 d), the subtraction's and the product's roundings (|s - m| <= 60: 2 * 60 u)
  and the hardware's exp2, 2^-22; a sum of n weights or products adds n u at most (chunked sums stay far below);
  weights held in bf16 on their way into a product are off by 2^-8 each (half a step).
"""
import math

import torch

U = 2.0 ** -24
EXP2 = 2.0 ** -22


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def attend(q, K, V, sees=None):
    """q [T][G][D], K, V [n][D] in float64 (one kv-head); sees [T][n] bool or None.  Returns out [T][G][D], weights
    [T][G][n], sum p|v| [T][G][D] and the largest score error bound d."""
    q, K, V = q.double(), K.double(), V.double()
    D = q.shape[-1]
    s = torch.einsum("tgd,nd->tgn", q, K) / math.sqrt(D)
    mag = torch.einsum("tgd,nd->tgn", q.abs(), K.abs()) / math.sqrt(D)
    if sees is not None:
        hide = ~sees[:, None, :].expand_as(s)
        s = s.masked_fill(hide, -math.inf)
        mag = mag.masked_fill(hide, 0.0)
        V = torch.where(sees.any(0)[:, None], V, 0.0)        # rows nobody sees may hold anything
    m = s.amax(-1, keepdim=True)
    p = torch.where(torch.isinf(m), 0.0, torch.exp(s - torch.where(torch.isinf(m), 0.0, m)))
    total = p.sum(-1, keepdim=True)
    p = torch.where(total > 0, p / total, 0.0)
    out = torch.einsum("tgn,nd->tgd", p, V)
    mass = torch.einsum("tgn,nd->tgd", p, V.abs())
    return out, p, mass, float(mag.max()) * (D + 2) * U


def weight_error(d, n, bf16_weights=False):
    """Relative error bound of a weight's share of the result."""
    return math.expm1(2 * d) + 2 * 120 * U + 2 * EXP2 + 2 * n * U + (2.0 ** -8 if bf16_weights else 0.0)


def norm_rope(x, w, pos, inv_freq, interleaved, eps):
    """x [B][T][H][D] -> the normalised, rotated heads in float64, and the magnitude |x0| + |x1| each element's rounding
    goes by."""
    x = x.double()
    if w is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * w.double()
    y, mag = x.clone(), x.abs().clone()
    half = len(inv_freq)
    for i, f in enumerate(inv_freq):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        ang = pos.double() * f
        c, s = torch.cos(ang)[..., None], torch.sin(ang)[..., None]
        y[..., a] = x[..., a] * c - x[..., b] * s
        y[..., b] = x[..., b] * c + x[..., a] * s
        mag[..., a] = mag[..., b] = x[..., a].abs() + x[..., b].abs()
    return y, mag


def tree_sees(mask, n, n_t):
    """mask: [n_t] Python ints -> bool [n_t][n]."""
    sees = torch.ones(n_t, n, dtype=torch.bool)
    for t in range(n_t):
        for j in range(n_t):
            sees[t, n - n_t + j] = bool(mask[t] >> j & 1)
    return sees


def random_tree(rng, n_t, chain=False):
    """Visibility words of a random tree: each token sees itself and its ancestors."""
    words = []
    for t in range(n_t):
        p = t - 1 if chain else int(rng.integers(-1, t)) if t else -1
        words.append((words[p] if p >= 0 else 0) | 1 << t)
    return words


def to_int64(words):
    return [w - (1 << 64) if w >= 1 << 63 else w for w in words]


def select(total, n, n_keep, n_recent):
    """total: [n] -> ascending row numbers."""
    def rank(j):
        x = float(total[j])
        return (1, 0.0, j) if math.isnan(x) else (0, -x, j)
    old = sorted(range(n - n_recent), key=rank)[: n_keep - n_recent]
    return sorted(old) + list(range(n - n_recent, n))
