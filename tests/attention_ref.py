"""The attention half of a layer in plain 64-bit arithmetic, from the formulas in include/tempo.h; shares no code with the
kernels or with the cases that time them."""
import torch

F64 = torch.float64


def turn(x, w, positions, cos_sin, eps=1e-6, interleaved=False):
    """rot(norm(x) * w), x [T, H, D]; element by element over the pairs."""
    x = x.to(F64).clone()
    D = x.shape[2]
    if w is not None:
        x = x / ((x ** 2).sum(2, keepdim=True) / D + eps).sqrt() * w.to(F64)
    if cos_sin is None:
        return x
    rot = cos_sin.shape[1]
    y = x.clone()
    at = cos_sin.to(F64)[positions.long().clamp(0, cos_sin.shape[0] - 1)]
    for i in range(rot // 2):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
        c, s = at[:, i, None], at[:, i + rot // 2, None]
        y[:, :, a] = x[:, :, a] * c - x[:, :, b] * s
        y[:, :, b] = x[:, :, b] * c + x[:, :, a] * s
    return y


def _scales():
    return torch.tensor(sorted([m * 2.0 ** -17 for m in range(1, 8)] + [m * 2.0 ** e for e in range(-17, 7) for m in range(8, 16)
                                                                        if m * 2.0 ** e <= 768.0]), dtype=F64)


def cached(x):
    """What the cache holds for x [T, H, D]: groups of 32, scale * (code - zero), the least scale whose 15 steps span the group."""
    x = x.to(F64)
    g = x.reshape(*x.shape[:2], -1, 32)
    lo, hi = g.amin(3).clamp(max=0), g.amax(3).clamp(min=0)
    table = _scales().to(x.device)
    s = table[torch.searchsorted(table * 15, (hi - lo).contiguous()).clamp(max=len(table) - 1)][..., None]
    z = (-lo[..., None] / s).round().clamp(max=15)
    c = ((g / s).round() + z).clamp(0, 15)
    return (s * (c - z)).reshape(x.shape)


def attend(q, k, v, scale, first):
    """q [n, H, D], k, v [L, Hkv, D]; query i sees the tokens t <= first + i.  Returns (out, sum p |v|, bound of a score's error)."""
    n, H, D = q.shape
    L, Hkv = k.shape[:2]
    q, k, v = q.to(F64), k.to(F64), v.to(F64)
    k, v = (t.repeat_interleave(H // Hkv, 1) for t in (k, v))
    hidden = torch.arange(L, device=q.device)[None, :] > first + torch.arange(n, device=q.device)[:, None]
    scores = torch.einsum("nhd,lhd->nhl", q, k) * scale
    size = torch.einsum("nhd,lhd->nhl", q.abs(), k.abs()) * abs(scale)
    scores = scores.masked_fill(hidden[:, None], float("-inf"))
    p = torch.exp(scores - scores.amax(2, keepdim=True).clamp(min=-1e300))
    p = p / p.sum(2, keepdim=True).clamp(min=1e-300)
    off = torch.where(hidden[:, None], 0.0, size).amax(2) * (D + 8) * 2.0 ** -24 if L else torch.zeros(n, H, dtype=F64, device=q.device)
    return torch.einsum("nhl,lhd->nhd", p, v), torch.einsum("nhl,lhd->nhd", p, v.abs()), off


def attend_tolerance(out, spread, off, L):
    """|error| of each output: its rounding to bf16 (2^-8 of it), the weights' to fp16 in numerator and sum (2^-11 each, and 2^-32 of
    the largest for those below fp16's normal range), the scores' in 32 bits (off, twice), and a 32-bit sum over L tokens."""
    return out.abs() * 2.0 ** -8 + spread * (2.0 ** -10 + 2 * off[..., None] + (L + 16) * 2.0 ** -23) + L * 2.0 ** -31 * spread.amax() + 1e-12
