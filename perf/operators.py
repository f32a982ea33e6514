"""The operators of the receiver's side as cases that can be timed and compared: rotary positions,
messages and caches held in 4 bits, and attention over them.

A case is a dict of plain values.  `kind` names what a pass does:

  rotary  pre-rotary query and key vectors of one or more layers turned to their positions
          (halves or interleaved pairs, a part of the head, positions scaled for long contexts;
          `inverse`: the transposed turn, which is the gradient of the forward one)
  pack    selected K/V rows of one or more senders packed into a 4-bit message or into a paged
          4-bit cache, and the message's rows restored as bf16
  attend  one layer's attention of m query tokens a sequence over a 4-bit cache, with the
          log-sum-exp of every row

Held in 4 bits, a row's value is c * s: c a whole number in -7..7, s the scale of its group of 32
neighbouring elements, the smallest number of 5 significant bits that is at least max|x| / 7 (and
within 2^-20 .. 2^13).

Sizes are those of this repository's benchmark and tests (2 to 36 layers, 4 to 32 query heads in
groups of 1, 2 or 4, head dimension 64 or 128, pages of 16 positions, up to 65536 positions).
"""
import functools
import math

import torch

own = False

SPAN, LATENT, GROUP = 16, 40, 32


def _case(name, kind, **kw):
    c = dict(kind=kind, layers=1, q_heads=32, kv_heads=8, d=128, m=1)
    more = {
        "rotary": dict(style="halves", dims=0, base=1e6, scaling="none", factor=1.0, original=0, start=0,
                       scattered=False, inverse=False),
        "pack": dict(senders=1, T=8192, keep=0.25, page=0),
        "attend": dict(sequences=1, T=8192, ragged=False, page=0, causal=True, window=0),
    }[kind]
    c.update(more)
    assert set(kw) <= set(c)
    c.update(kw)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one layer of a decode step: the new token's query and key, far into a long context
        _case("rotary_token", "rotary", start=65000),
        # the receiver's query before it is scored: 64 tokens in all 36 layers
        _case("rotary_query", "rotary", layers=36, m=64, start=8192),
        # keys of a message moved back to no position: the transposed turn at scattered rows
        _case("rotary_scattered_inverse", "rotary", layers=8, m=6001, d=64, q_heads=16, kv_heads=8, scattered=True,
              inverse=True, style="pairs", base=1e4),
        # a long prompt whose context is stretched four times, the rotary part half of the head
        _case("rotary_prompt_scaled", "rotary", layers=4, m=16384, dims=64, scaling="yarn", factor=4.0, original=32768),
        # the smallest state this repository configures, kept as a 4-bit message
        _case("pack_tiny", "pack", layers=2, q_heads=4, kv_heads=2, d=64, T=512),
        # an 8B-shaped sender's selected rows as a 4-bit message
        _case("pack_message", "pack", layers=36),
        # three senders' rows into the pages of a receiver's 4-bit cache
        _case("pack_fanin_paged", "pack", layers=36, senders=3, T=16001, keep=0.1, page=16),
        # one token of one sequence over a message of a quarter of 8192 positions
        _case("attend_token", "attend", T=2048),
        # a served batch: 48 sequences of ragged length in pages, a token each
        _case("attend_batch_paged", "attend", sequences=48, T=8192, ragged=True, page=16),
        # one token over a long context
        _case("attend_token_long", "attend", T=65536),
        # a question of 64 tokens over three senders' kept rows
        _case("attend_query", "attend", m=64, T=12352),
        # a prompt chunk of 1024 tokens at the end of a context, the largest
        _case("attend_prompt", "attend", m=1024, T=16384),
    ]


def _log(rng, a, b):
    return int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))


def draw(rng):
    kind = rng.choice(["rotary"] * 3 + ["pack"] * 3 + ["attend"] * 6)
    kv = rng.choice([2, 4, 8, 8])
    shape = dict(q_heads=kv * rng.choice([4, 4, 4, 2, 1]), kv_heads=kv, d=rng.choice([128, 128, 64]))
    while True:
        if kind == "rotary":
            scaling = rng.choice(["none", "none", "linear", "yarn"])
            c = _case(None, kind, **shape, layers=_log(rng, 1, 36), m=_log(rng, 1, 16384),
                      style=rng.choice(["halves", "halves", "pairs"]),
                      dims=rng.choice([0, 0, shape["d"] // 2, shape["d"] // 4]), base=rng.choice([1e4, 1e6]),
                      scaling=scaling, factor=1.0 if scaling == "none" else rng.choice([2.0, 4.0, 8.0]),
                      original=rng.choice([4096, 32768]) if scaling == "yarn" else 0,
                      start=rng.randrange(0, 65536), scattered=rng.random() < 0.3, inverse=rng.random() < 0.3)
            if c["layers"] * c["m"] * (c["q_heads"] + kv) * c["d"] <= 3.3e8:
                return c
        elif kind == "pack":
            c = _case(None, kind, **shape, layers=_log(rng, 2, 36), senders=rng.choice([1, 1, 2, 3, 5]),
                      T=_log(rng, 64, 65536), keep=round(rng.uniform(0.05, 0.6), 3), page=rng.choice([0, 0, 16]))
            if c["senders"] * c["layers"] * kv * c["T"] * c["d"] <= 1.7e9 and \
                    c["senders"] * c["layers"] * kv * c["T"] * c["d"] * c["keep"] <= 1.8e8:
                return c
        else:
            m = rng.choice([1, 1, 1, _log(rng, 2, 16), _log(rng, 16, 1024), _log(rng, 16, 1024)])
            c = _case(None, kind, **shape, sequences=rng.choice([1, 1, _log(rng, 2, 48)]), T=_log(rng, 64, 65536), m=m,
                      ragged=rng.random() < 0.5, page=rng.choice([0, 0, 16, 64]), causal=rng.random() < 0.8)
            if c["causal"] and rng.random() < 0.2:
                c["window"] = _log(rng, 16, 4096)
            n = c["sequences"]
            if n * kv * c["T"] * c["d"] <= 4.1e8 and n * m * c["q_heads"] * c["T"] * (c["d"] / 128) <= 5.4e8 and \
                    m <= c["T"]:
                return c


# --- inputs -------------------------------------------------------------------------------------

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(shape, gen, dtype=torch.bfloat16):
    return torch.randn(shape, generator=gen, device="cuda", dtype=dtype)


def _keys(shape, gen):
    """Keys as models have them: a few channels of every head are larger than the others."""
    loud = 1 + 2 * (torch.rand(shape[-3:-2] + (1,) + shape[-1:], generator=gen, device="cuda") < 0.03)
    return _randn(shape, gen) * loud.to(torch.bfloat16)


def _quantise(x):
    """(codes in -7..7, scale of every group) of the last dimension of x, both in 32 bits."""
    g = x.float().unflatten(-1, (-1, GROUP))
    a = g.abs().amax(-1, keepdim=True)
    a = a / torch.full_like(a, 7)     # (a quotient, no product with 1/7; x has 8 bits, so no border is nearer than 2^-12)
    s = ((a.view(torch.int32) + 0x7FFFF) >> 19 << 19).view(torch.float32).clamp(2.0 ** -20, 2.0 ** 13)
    c = (torch.floor(g.abs() / s + 0.5) * g.sign()).clamp(-7, 7)
    return c.flatten(-2), s.squeeze(-1)


def _held(x):
    """(codes uint8 [..][d/2], scales bf16 [..][d/32]) as a cache holds them: of the eight elements of a
    32-bit word, element i is in nibble i / 2 + 4 (i mod 2), as c + 8."""
    c, s = _quantise(x)
    w = (c + 8).to(torch.uint8).unflatten(-1, (-1, 4, 2))     # [word][i / 2][i mod 2]
    w = w.transpose(-1, -2).reshape(w.shape[:-2] + (4, 2))    # [word][byte][nibble]
    return (w[..., 0] | (w[..., 1] << 4)).flatten(-2), s.to(torch.bfloat16)


def _values(codes, scales):
    """The values that held rows stand for, in 32 bits."""
    n = torch.stack([codes & 15, codes >> 4], -1).unflatten(-2, (-1, 4)).flatten(-2)     # [word][nibble]
    c = n.unflatten(-1, (2, 4)).transpose(-1, -2).flatten(-3).float() - 8
    return (c.unflatten(-1, (-1, GROUP)) * scales.float().unsqueeze(-1)).flatten(-2)


def _picked(T, B, gen):
    """Selected positions as the span rule leaves them: whole spans, the sink and the tail."""
    score = torch.rand(-(-T // SPAN), generator=gen, device="cuda").repeat_interleave(SPAN)[:T]
    score[:1] = 2
    score[max(0, T - LATENT):] = 2
    return torch.sort(torch.argsort(score, descending=True, stable=True)[:B]).values.to(torch.int32)


def _budget(case):
    T = case["T"]
    return max(min(T, math.ceil(case["keep"] * T)), min(T, LATENT + 1))


def _lengths(case, seed):
    n, T = case["sequences"], case["T"]
    if not case["ragged"]:
        return [T] * n
    r = torch.rand(n, generator=torch.Generator().manual_seed(seed))
    low = max(case["m"], T // 4)
    return [max(1, int(low + x * (T - low) + 0.5)) for x in r.tolist()]


def prepare(case, seed):
    gen = _gen(seed)
    nL, Hq, Hkv, d, m = (case[k] for k in ("layers", "q_heads", "kv_heads", "d", "m"))
    st = dict(case=case)
    if case["kind"] == "rotary":
        st["x"] = [_randn((nL, m, Hq, d), gen), _randn((nL, m, Hkv, d), gen)]
        st["y"] = [torch.empty_like(x) for x in st["x"]]
        pos = torch.arange(m, dtype=torch.int32, device="cuda") + case["start"]
        if case["scattered"]:
            pos += torch.randint(0, 16, (m,), generator=gen, device="cuda", dtype=torch.int32).cumsum(0).to(torch.int32)
            st["pos"] = pos
        else:
            st["pos"] = None
        return st
    if case["kind"] == "pack":
        n, T, P = case["senders"], case["T"], case["page"]
        B = _budget(case)
        st["K"] = [_keys((nL, Hkv, T, d), gen) for _ in range(n)]
        st["V"] = [_randn((nL, Hkv, T, d), gen) for _ in range(n)]
        st["idx"] = [_picked(T, B, gen) for _ in range(n)]
        rows = (nL, Hkv, n * B)
        if P:
            pages = -(-n * B // P)
            total = pages + pages // 4 + 1
            st["table"] = torch.randperm(total, generator=gen, device="cuda")[:pages].to(torch.int32)
            rows = (nL, total, P, Hkv)
        st["held"] = [torch.zeros(rows + (w,), dtype=t, device="cuda")
                      for w, t in ((d // 2, torch.uint8), (d // 2, torch.uint8), (d // GROUP, torch.bfloat16),
                                   (d // GROUP, torch.bfloat16))]
        st["out"] = [torch.empty((nL, Hkv, n * B, d), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        return st
    n, T, P = case["sequences"], case["T"], case["page"]
    Ts = st["Ts"] = _lengths(case, seed)
    st["Q"] = _randn((n, m, Hq, d), gen) * 2
    st["out"] = torch.empty_like(st["Q"])
    st["lse"] = torch.empty((n, m, Hq), dtype=torch.float32, device="cuda")
    st["T"] = torch.tensor(Ts, device="cuda")
    if P:
        pages = -(-T // P)
        total = n * pages + n * pages // 8 + 1
        st["tables"] = torch.randperm(total, generator=gen, device="cuda")[:n * pages].to(torch.int32).view(n, pages)
        shape = (1, total, P, Hkv, d)
    else:
        shape = (n, 1, Hkv, T, d)
    st["K"], st["Ks"] = _held(_keys(shape, gen))
    st["V"], st["Vs"] = _held(_randn(shape, gen))
    return st


# --- one pass -----------------------------------------------------------------------------------

def _freqs(case, device):
    """Turns of every pair a position, in radians and 64 bits, and what cosine and sine are multiplied by."""
    r = case["dims"] or case["d"]
    i = torch.arange(r // 2, dtype=torch.float64, device=device)
    f = case["base"] ** (-2 * i / r)
    if case["scaling"] == "linear":
        return f / case["factor"], 1.0
    if case["scaling"] == "yarn":
        def dim(turns):
            return r * math.log(case["original"] / (2 * math.pi * turns)) / (2 * math.log(case["base"]))
        low, high = max(math.floor(dim(32.0)), 0), min(math.ceil(dim(1.0)), r - 1)
        ramp = ((i - low) / (high - low if high > low else 0.001)).clamp(0, 1)
        return f * (1 - ramp) + f / case["factor"] * ramp, 0.1 * math.log(case["factor"]) + 1
    return f, 1.0


def _turned(case, x, pos, to):
    """x [nL][m][H][d] with every pair of its first `dims` elements turned, in the type `to`."""
    f, a = _freqs(case, x.device)
    if pos is None:
        pos = torch.arange(case["m"], device=x.device) + case["start"]
    t = pos.double()[:, None, None] * f
    cos, sin = (t.cos() * a).to(to), (t.sin() * (-a if case["inverse"] else a)).to(to)
    r = case["dims"] or case["d"]
    z, rest = x[..., :r].to(to), x[..., r:].to(to)
    if case["style"] == "halves":
        u, v = z[..., :r // 2], z[..., r // 2:]
        return torch.cat([u * cos - v * sin, v * cos + u * sin, rest], -1)
    u, v = z[..., 0::2], z[..., 1::2]
    return torch.cat([torch.stack([u * cos - v * sin, v * cos + u * sin], -1).flatten(-2), rest], -1)


def _attention(q, k, v, T, causal, window, scale):
    """(out, log-sum-exp) of q [n][m][Hq][d] over k and v [n][Hkv][t][d]: q's token r is at position T - m + r."""
    n, m, Hq, d = q.shape
    Hkv, t = k.shape[1], k.shape[2]
    q = q.unflatten(2, (Hkv, Hq // Hkv)).permute(0, 2, 3, 1, 4).reshape(n, Hkv, -1, d)      # [n][Hkv][G m][d]
    z = torch.matmul(q, k.transpose(-1, -2)) * scale
    z = z.view(n, Hkv, Hq // Hkv, m, t)
    at = torch.arange(t, device=q.device)
    seen = (at < T[:, None]).view(n, 1, 1, 1, t)
    if causal:
        p = (T[:, None] - m + torch.arange(m, device=q.device)).view(n, 1, 1, m, 1)
        seen = seen & (at <= p)
        if window:
            seen = seen & (at > p - window)
    z = z.masked_fill_(~seen, -math.inf)
    top = z.amax(-1, keepdim=True).clamp(min=torch.finfo(z.dtype).min)
    e = z.sub_(top).exp_()
    total = e.sum(-1, keepdim=True)
    o = torch.matmul(e.view(n, Hkv, -1, t), v).view(n, Hkv, Hq // Hkv, m, d)
    o = torch.where(total > 0, o / total, torch.zeros_like(o))
    lse = (top + total.log()).squeeze(-1)
    return o.permute(0, 3, 1, 2, 4).reshape(n, m, Hq, d), lse.permute(0, 3, 1, 2).reshape(n, m, Hq)


def _cache_values(st, to):
    """K and V [n][Hkv][T][d] of an attend case."""
    kv = []
    for c, s in (("K", "Ks"), ("V", "Vs")):
        c, s = st[c], st[s]
        if st["case"]["page"]:
            at = st["tables"].long()
            c, s = (x[0][at].flatten(1, 2)[:, :st["case"]["T"]].transpose(1, 2) for x in (c, s))    # [n][Hkv][T][..]
        else:
            c, s = c[:, 0], s[:, 0]
        kv.append(_values(c, s).to(to))
    return kv


@functools.lru_cache(maxsize=None)
def _receiver(Hq, Hkv, d, layers, m, T, n):
    import paper_2609_32046_gb300 as cb
    return cb.Receiver(layers, Hq, Hkv, d, m, T, n)


def _own_rotary(st):
    import paper_2609_32046_gb300 as cb
    c = st["case"]
    rx = _receiver(c["q_heads"], c["kv_heads"], c["d"], c["layers"], 1, 1, 2)
    rope = cb.Rotary(c["base"], c["style"], c["dims"], c["scaling"], c["factor"], c["original"])
    rx.rotary(st["x"], rope, st["y"], pos=st["pos"], pos0=c["start"], inverse=c["inverse"])
    return {"q": st["y"][0], "k": st["y"][1]}


def _own_pack(st):
    import paper_2609_32046_gb300 as cb
    c = st["case"]
    n, B = c["senders"], _budget(c)
    rx = _receiver(c["q_heads"], c["kv_heads"], c["d"], c["layers"], 1, max(c["T"], n * B), n)
    held = cb.PackedKV(*st["held"], T=n * B, pages=st.get("table"))
    rx.pack(st["K"], st["V"], [held] * n, [i * B for i in range(n)], idx=st["idx"])
    rx.unpack([held], *st["out"])
    return {"k": st["out"][0], "v": st["out"][1]}


def _own_attend(st):
    import paper_2609_32046_gb300 as cb
    c = st["case"]
    n = c["sequences"]
    rx = _receiver(c["q_heads"], c["kv_heads"], c["d"], 1, c["m"], c["T"], n)
    if "caches" not in st:      # a server's sequences keep their views of the pool and their block tables
        if c["page"]:
            st["caches"] = [cb.PackedKV(st["K"], st["V"], st["Ks"], st["Vs"], T=T, pages=t)
                            for T, t in zip(st["Ts"], st["tables"])]
        else:
            st["caches"] = [cb.PackedKV(*x, T=T) for *x, T in zip(st["K"], st["V"], st["Ks"], st["Vs"], st["Ts"])]
    rx.attend(st["caches"], st["Q"], st["out"], causal=c["causal"], window=c["window"], lses=st["lse"])
    return {"out": st["out"], "lse": st["lse"]}


def run(state):
    c = state["case"]
    if own:
        return {"rotary": _own_rotary, "pack": _own_pack, "attend": _own_attend}[c["kind"]](state)
    if c["kind"] == "rotary":
        q, k = (_turned(c, x, state["pos"], torch.float32).to(x.dtype) for x in state["x"])
        return {"q": q, "k": k}
    if c["kind"] == "pack":
        kept = [torch.cat([x[:, :, i.long()] for x, i in zip(state[n], state["idx"])], 2) for n in ("K", "V")]
        held = [_held(x) for x in kept]
        k, v = (_values(*h).to(torch.bfloat16) for h in held)
        return {"k": k, "v": v}
    k, v = _cache_values(state, torch.float32)
    o, lse = _attention(state["Q"].float(), k, v, state["T"], c["causal"], c["window"], 1 / math.sqrt(c["d"]))
    return {"out": o.to(torch.bfloat16), "lse": lse}


# --- what a pass cannot do without ----------------------------------------------------------------

def work(case):
    nL, Hq, Hkv, d, m = (case[k] for k in ("layers", "q_heads", "kv_heads", "d", "m"))
    held = d // 2 + d // GROUP * 2                               # bytes of one row in 4 bits
    if case["kind"] == "rotary":
        n = nL * m * (Hq + Hkv)
        return {"bytes": n * d * 4 + (4 * m if case["scattered"] else 0), "flops": 3 * n * (case["dims"] or d)}
    if case["kind"] == "pack":
        rows = 2 * nL * Hkv * case["senders"] * _budget(case)
        # the rows in, the message out and in again, the restored rows out
        return {"bytes": rows * (2 * d + 2 * held + 2 * d) + 4 * case["senders"] * _budget(case), "flops": 0}
    pairs = rows = 0
    for T in _lengths(case, 0):
        first = 0
        if not case["causal"]:
            pairs += m * T
        else:
            w = case["window"] or T
            first = max(0, T - m + 1 - w)
            pairs += sum(min(w, T - m + r + 1) for r in range(m) if T - m + r >= 0)
        rows += T - first
    n = case["sequences"]
    return {"bytes": rows * Hkv * 2 * held + n * m * Hq * (d * 4 + 4), "flops": 4 * pairs * Hq * d}


# --- the same in 64 bits ----------------------------------------------------------------------------

def _exact_rotary(case, x, pos):
    """The turn as a product of complex numbers: pair j, at the angle position * f_j."""
    r = case["dims"] or case["d"]
    f, gain = [], 1.0
    for j in range(r // 2):
        w = case["base"] ** (-2.0 * j / r)
        if case["scaling"] == "linear":
            w /= case["factor"]
        if case["scaling"] == "yarn":
            gain = 1 + math.log(case["factor"]) / 10
            edge = [r * math.log(case["original"] / (t * 2 * math.pi)) / math.log(case["base"]) / 2 for t in (32, 1)]
            low, high = max(0, math.floor(edge[0])), min(r - 1, math.ceil(edge[1]))
            share = min(1.0, max(0.0, (j - low) / ((high - low) or 0.001)))
            w = w / case["factor"] * share + w * (1 - share)
        f.append(w)
    f = torch.tensor(f, dtype=torch.float64, device=x.device)
    angle = torch.outer(pos.double(), f) * (-1 if case["inverse"] else 1)
    turn = torch.polar(torch.full_like(angle, gain), angle)[:, None]               # [m][1][r/2]
    y = x.double()
    if case["style"] == "halves":
        z = torch.complex(y[..., :r // 2], y[..., r // 2:r]) * turn
        y[..., :r // 2], y[..., r // 2:r] = z.real, z.imag
    else:
        z = torch.complex(y[..., 0:r:2].contiguous(), y[..., 1:r:2].contiguous()) * turn
        y[..., 0:r:2], y[..., 1:r:2] = z.real, z.imag
    return y


def _exact_held(x):
    """What a row's values become in 4 bits, from the definition: the scale is the smallest k * 2^e with
    k in 16..31 that is at least max|x| / 7, a code the nearest whole number to x / scale (halves away from zero)."""
    g = x.double().unflatten(-1, (-1, GROUP))
    a = g.abs().amax(-1, keepdim=True).clamp(min=1e-30) / 7
    e = torch.floor(torch.log2(a)) - 4
    e = torch.where(a < 16 * torch.exp2(e), e - 1, e)
    e = torch.where(a >= 32 * torch.exp2(e), e + 1, e)
    k = torch.ceil(a * (1 - 1e-13) / torch.exp2(e))      # (a / 2^e is whole or over 2^-12 away from it)
    s = (k * torch.exp2(e)).clamp(2.0 ** -20, 2.0 ** 13)
    q = torch.trunc((2 * g.abs() / s + 1) / 2).clamp(max=7)
    return (torch.copysign(q, g) * s).flatten(-2)


def _exact_attention(case, st):
    """Sequence by sequence and head by head: softmax over the positions that a token sees."""
    kv = []
    for c, s in (("K", "Ks"), ("V", "Vs")):
        c, s = st[c].long(), st[s].double()
        words = (c.unflatten(-1, (-1, 4)) << torch.tensor([0, 8, 16, 24], device=c.device)).sum(-1, keepdim=True)
        at = torch.tensor([4 * (i // 2) + 16 * (i % 2) for i in range(8)], device=c.device)
        kv.append(((((words >> at) & 15) - 8).flatten(-2).unflatten(-1, (-1, GROUP)) * s.unsqueeze(-1)).flatten(-2))
    n, m, Hq, Hkv, d = case["sequences"], case["m"], case["q_heads"], case["kv_heads"], case["d"]
    out = torch.zeros((n, m, Hq, d), dtype=torch.float64, device="cuda")
    lse = torch.full((n, m, Hq), -math.inf, dtype=torch.float64, device="cuda")
    for i, T in enumerate(st["Ts"]):
        if case["page"]:
            at = st["tables"][i].long()
            k, v = (x[0][at].reshape(-1, Hkv, d)[:T].transpose(0, 1) for x in kv)
        else:
            k, v = (x[i, 0, :, :T] for x in kv)
        t = torch.arange(T, device="cuda")
        p = torch.arange(T - m, T, device="cuda")[:, None]
        blind = torch.zeros((m, T), dtype=torch.bool, device="cuda")
        if case["causal"]:
            blind = t > p
            if case["window"]:
                blind |= t <= p - case["window"]
        for h in range(Hq):
            g = h // (Hq // Hkv)
            z = (st["Q"][i, :, h].double() @ k[g].T / math.sqrt(d)).masked_fill(blind, -math.inf)
            lse[i, :, h] = torch.logsumexp(z, -1)
            out[i, :, h] = torch.nan_to_num(torch.softmax(z, -1), nan=0.0) @ v[g]
    return {"out": out, "lse": lse}


def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] == "rotary":
        pos = st["pos"] if st["pos"] is not None else torch.arange(case["m"], device="cuda") + case["start"]
        q, k = (_exact_rotary(case, x, pos) for x in st["x"])
        return {"q": q, "k": k}
    if case["kind"] == "pack":
        k, v = (torch.cat([_exact_held(x[:, :, i.long()]) for x, i in zip(st[n], st["idx"])], 2) for n in ("K", "V"))
        return {"k": k, "v": v}
    return _exact_attention(case, st)
