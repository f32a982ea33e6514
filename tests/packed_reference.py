"""Plain 64-bit restatements of the receiver's operators, from their definitions: rotary positions, rows
held in 4 bits, attention over them."""
import math

import torch

GROUP = 32
LARGEST = 7.0 * 2 ** 13


def bf16_bits(x):
    return x.contiguous().view(torch.int16)


# --- rows in 4 bits -----------------------------------------------------------------------------

def scale_of(top):
    """The smallest k * 2^e, k in 16..31, that is at least top / 7, within 2^-20 .. 2^13 (one number)."""
    top = min(float(top), LARGEST)
    if top <= 7 * 2.0 ** -20:
        return 2.0 ** -20
    e = math.frexp(top / 7)[1] - 5
    while True:
        for k in range(16, 32):
            if 7 * k * 2.0 ** e >= top:
                return min(k * 2.0 ** e, 2.0 ** 13)
        e += 1


def held_rows(x):
    """(codes, scales) in 64 bits of the rows x (bf16, any shape [..][d]), group by group in plain Python."""
    g = x.double().cpu().reshape(-1, GROUP)
    g = torch.where(torch.isnan(g), torch.zeros_like(g), g).clamp(-LARGEST, LARGEST)
    s = torch.tensor([scale_of(a) for a in g.abs().amax(-1).tolist()], dtype=torch.float64)
    q = g.abs() / s[:, None]
    c = torch.copysign(torch.floor(q + 0.5), g)      # (64 bits: a bf16 number over one of 5 bits, and 1/2, are exact enough)
    return c.reshape(x.shape), s.reshape(x.shape[:-1] + (-1,))


def packed_bytes(c):
    """Codes as a cache holds them: of the eight elements of a word, element i in nibble i / 2 + 4 (i % 2)."""
    u = (c + 8).to(torch.int64).reshape(c.shape[:-1] + (-1, 8))
    word = torch.zeros(u.shape[:-1], dtype=torch.int64)
    for i in range(8):
        word |= u[..., i] << (4 * (i // 2 + 4 * (i % 2)))
    return torch.stack([(word >> (8 * k)) & 255 for k in range(4)], -1).flatten(-2).to(torch.uint8)


def values(codes, scales):
    """The values of packed rows, in 64 bits."""
    b = codes.long().reshape(codes.shape[:-1] + (codes.shape[-1] // 4, 4))
    word = b[..., 0] | (b[..., 1] << 8) | (b[..., 2] << 16) | (b[..., 3] << 24)
    c = torch.stack([((word >> (4 * (i // 2 + 4 * (i % 2)))) & 15) - 8 for i in range(8)], -1).flatten(-2).double()
    return (c.unflatten(-1, (scales.shape[-1], GROUP)) * scales.double().unsqueeze(-1)).flatten(-2)


# --- rotary -------------------------------------------------------------------------------------

def frequencies(dims, base, scaling="none", factor=1.0, original=0, beta_fast=32.0, beta_slow=1.0):
    f = [base ** (-2.0 * k / dims) for k in range(dims // 2)]
    if scaling == "linear":
        return [x / factor for x in f], 1.0
    if scaling == "yarn":
        def pair(turns):
            return dims * math.log(original / (2 * math.pi * turns)) / (2 * math.log(base))
        lo, hi = max(math.floor(pair(beta_fast)), 0), min(math.ceil(pair(beta_slow)), dims - 1)
        hi = hi if hi > lo else lo + 0.001
        w = [min(1.0, max(0.0, (k - lo) / (hi - lo))) for k in range(dims // 2)]
        return [x * (1 - y + y / factor) for x, y in zip(f, w)], 0.1 * math.log(factor) + 1
    return f, 1.0


def rotary(x, pos, f, gain, style, inverse=False):
    """x [..][tokens][heads][d] in 64 bits, pos [tokens]."""
    dims = 2 * len(f)
    a = pos.double()[:, None, None] * torch.tensor(f, dtype=torch.float64, device=x.device)
    if inverse:
        a = -a
    y = x.double().clone()
    first = torch.arange(dims // 2, device=x.device) * (1 if style == "halves" else 2)
    second = first + (dims // 2 if style == "halves" else 1)
    u, v = y[..., first].clone(), y[..., second].clone()
    y[..., first] = gain * (u * a.cos() - v * a.sin())
    y[..., second] = gain * (v * a.cos() + u * a.sin())
    return y


# --- attention ----------------------------------------------------------------------------------

def attention(q, k, v, scale, causal=True, window=0):
    """q [m][Hq][d], k and v [Hkv][L][d] in 64 bits: (out, lse, sum of weights times |v|, largest sum of |q k| scale)."""
    m, Hq, d = q.shape
    Hkv, L = k.shape[:2]
    kh, vh = (x.repeat_interleave(Hq // Hkv, 0) for x in (k, v))
    z = torch.einsum("rhd,htd->hrt", q, kh) * scale
    size = torch.einsum("rhd,htd->hrt", q.abs(), kh.abs()).amax() * scale if L else torch.zeros(())
    t = torch.arange(L, device=q.device)
    at = torch.arange(L - m, L, device=q.device)[:, None]
    seen = torch.ones((m, L), dtype=torch.bool, device=q.device)
    if causal:
        seen = t <= at
        if window:
            seen = seen & (t > at - window)
    z = z.masked_fill(~seen, -math.inf)
    lse = torch.logsumexp(z, -1) if L else torch.full((Hq, m), -math.inf, dtype=torch.float64, device=q.device)
    a = torch.where(seen, torch.exp(z - lse.clamp(min=-1e300)[..., None]), torch.zeros_like(z))
    return torch.einsum("hrt,htd->rhd", a, vh), lse.T, torch.einsum("hrt,htd->rhd", a, vh.abs()), float(size)
