"""Plain 64-bit restatements, from their definitions, of what a receiver does that drafts tokens and holds its cache to a
budget: what a token sees, attention and its weights under that, the rows that stay."""
import math

import torch


def unpacked(words, m):
    """Bits bool [m][m] of int32 words [m][ceil(m / 32)], bit by bit in Python."""
    w = words.cpu().tolist()
    return torch.tensor([[(w[r][u // 32] >> (u % 32)) & 1 == 1 for u in range(m)] for r in range(m)], dtype=torch.bool).reshape(m, m)


def seen(m, L, causal=True, window=0, bits=None):
    """bool [m][L]: the rows that each of the m tokens at the end of L rows sees."""
    out = torch.zeros((m, L), dtype=torch.bool)
    t = torch.arange(L)
    for r in range(m):
        at = L - m + r
        if bits is not None:
            u = t - (L - m)
            out[r] = u < 0
            own = u >= 0
            out[r, own] = bits[r][u[own]]
        elif causal:
            out[r] = t <= at
            if window:
                out[r] &= t > at - window
        else:
            out[r] = True
    return out


def attention(q, k, v, scale, sees):
    """q [m][Hq][d], k and v [Hkv][L][d], sees [m][L] in 64 bits: (out, lse, sum of weights times |v|, largest sum of |q k| scale)."""
    m, Hq, d = q.shape
    Hkv, L = k.shape[:2]
    kh, vh = (x.repeat_interleave(Hq // Hkv, 0) for x in (k, v))
    z = torch.einsum("rhd,htd->hrt", q, kh) * scale
    size = float(torch.einsum("rhd,htd->hrt", q.abs(), kh.abs()).amax() * scale) if L and m else 0.0
    z = z.masked_fill(~sees, -math.inf)
    lse = torch.logsumexp(z, -1) if L else torch.full((Hq, m), -math.inf, dtype=torch.float64, device=q.device)
    a = torch.where(sees, torch.exp(z - lse.clamp(min=-1e300)[..., None]), torch.zeros_like(z))
    return torch.einsum("hrt,htd->rhd", a, vh), lse.T, torch.einsum("hrt,htd->rhd", a, vh.abs()), size


def weights(q, k, lse, scale, sees):
    """[Hkv][L]: the tokens' weights exp(scale <q, k> - lse) that each row gathers, and the largest sum of |q k| scale."""
    m, Hq, d = q.shape
    Hkv, L = k.shape[:2]
    kh = k.repeat_interleave(Hq // Hkv, 0)
    z = torch.einsum("rhd,htd->hrt", q, kh) * scale
    size = float(torch.einsum("rhd,htd->hrt", q.abs(), kh.abs()).amax() * scale) if L and m else 0.0
    lse = lse.T[..., None]                                    # [Hq][m][1]
    a = torch.where(sees & torch.isfinite(lse), torch.exp(z - lse), torch.zeros_like(z))
    return a.sum(1).reshape(Hkv, Hq // Hkv, L).sum(1), size


def kept_rows(w, L, keep, first, last):
    """The rows (ascending) of one list that stay, w its weights as a Python list: a plain sort."""
    if L <= keep:
        return list(range(L))
    inner = range(first, L - last)
    value = lambda t: -math.inf if math.isnan(w[t]) else w[t] + 0.0    # noqa: E731
    below = lambda t: 1 if math.isnan(w[t]) else 0                     # noqa: E731
    best = sorted(inner, key=lambda t: (below(t), -value(t), t))[:keep - first - last]
    return list(range(first)) + sorted(best) + list(range(L - last, L))
