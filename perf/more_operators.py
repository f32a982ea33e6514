"""Operators of a receiver that drafts tokens and holds its 4-bit cache to a budget, as cases that can be
timed and compared.

A case is a dict of plain values.  `kind` names what a pass does:

  tree    one layer's attention of m drafted tokens a sequence over a 4-bit cache whose last m rows are the
          drafts' own: a draft sees every row before them and, of them, those that its bits name
  weigh   one layer's attention weights of m query tokens, summed over the tokens and the heads of a group, added
          to what the cache's rows had gathered: decay * before + sum exp(scale <q, k> - lse)
  evict   for every layer and KV head the first and the last rows of a cache and the heaviest of the others, in
          their order, moved into a smaller cache
  keep    the rows of accepted drafts moved together behind the rows before the drafts, every layer and head, in
          the cache itself

Held in 4 bits, a row's value is c * s: c a whole number in -7..7, s the scale of its group of 32
neighbouring elements.  evict and keep move rows and change no bit of them, so what they return is the stored
bytes and words, as whole numbers.

Sizes are those of this repository's benchmark and tests (2 to 36 layers, 4 to 32 query heads in groups of
1, 2 or 4, head dimension 64 or 128, pages of 16 positions, up to 65536 positions).
"""
import functools
import math

import torch

own = False

GROUP = 32


def _case(name, kind, **kw):
    c = dict(kind=kind, q_heads=32, kv_heads=8, d=128, sequences=1, T=8192, ragged=False, page=0)
    more = {
        "tree": dict(m=16, bits="tree"),
        "weigh": dict(m=1, bits="causal", window=0, decay=1.0),
        "evict": dict(layers=36, keep=2048, first=4, last=64),
        "keep": dict(layers=36, m=64, path=5),
    }[kind]
    c.update(more)
    assert set(kw) <= set(c)
    c.update(kw)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # four drafts over a message of a quarter of 8192 positions, the smallest call
        _case("tree_four_drafts", "tree", m=4, T=2048),
        # a served batch: 32 sequences of ragged length in pages, 16 drafts each
        _case("tree_batch_paged", "tree", sequences=32, m=16, ragged=True, page=16),
        # one agent's 64 drafts over a long context
        _case("tree_long", "tree", m=64, T=32768),
        # any bits, drafts that see none of their own among them, an odd number of them, the smaller heads
        _case("tree_any_bits_d64", "tree", sequences=4, m=251, T=5003, q_heads=16, d=64, bits="any"),
        # one layer of a decode step whose token's weights are gathered
        _case("weigh_token", "weigh", T=2048),
        # the same for a served batch of 48 ragged sequences in pages
        _case("weigh_batch_paged", "weigh", sequences=48, ragged=True, page=16),
        # drafts' weights in groups of two heads of 64, older weights fading
        _case("weigh_tree_d64", "weigh", sequences=8, m=33, T=6001, q_heads=16, d=64, bits="tree", decay=0.875),
        # a prompt chunk of 1024 tokens at the end of a context: the largest call
        _case("weigh_prompt", "weigh", m=1024, T=16384),
        # the smallest state this repository configures, held to half of its rows
        _case("evict_tiny", "evict", layers=2, q_heads=4, kv_heads=2, d=64, T=512, keep=256, first=1, last=40),
        # an 8B-shaped prompt's cache held to an eighth
        _case("evict_prompt", "evict", T=16384),
        # the accepted path of 64 drafts in every layer
        _case("keep_path", "keep", T=1024),
        # the same for 32 sequences in pages
        _case("keep_batch_paged", "keep", sequences=32, m=16, path=4, T=300, page=16),
    ]


def _log(rng, a, b):
    return int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))


def draw(rng):
    kind = rng.choice(["tree"] * 5 + ["weigh"] * 5 + ["evict"] * 3 + ["keep"] * 2)
    kv = rng.choice([2, 4, 8, 8])
    shape = dict(q_heads=kv * rng.choice([4, 4, 4, 2, 1]), kv_heads=kv, d=rng.choice([128, 128, 64]),
                 sequences=rng.choice([1, 1, _log(rng, 2, 48)]), page=rng.choice([0, 0, 16, 64]))
    while True:
        T = _log(rng, 64, 65536)
        ragged = rng.random() < 0.5
        n, lists = shape["sequences"], shape["sequences"] * kv
        if kind == "tree":
            c = _case(None, kind, **shape, T=T, ragged=ragged, m=rng.choice([_log(rng, 1, 8), _log(rng, 4, 256), _log(rng, 16, 256)]),
                      bits=rng.choice(["tree", "tree", "any"]))
            if c["m"] <= T and lists * T * c["d"] <= 2.7e8 and n * c["m"] * c["q_heads"] * T * (c["d"] / 128) <= 1.3e8:
                return c
        elif kind == "weigh":
            bits = rng.choice(["causal", "causal", "all", "tree"])
            m = rng.choice([1, 1, _log(rng, 2, 16), _log(rng, 16, 256 if bits == "tree" else 1024)])
            c = _case(None, kind, **shape, T=T, ragged=ragged, m=m, bits=bits, decay=rng.choice([1.0, 1.0, 0.9]))
            if bits == "causal" and rng.random() < 0.2:
                c["window"] = _log(rng, 16, 4096)
            if m <= T and lists * T * c["d"] <= 4.1e8 and n * m * c["q_heads"] * T * (c["d"] / 128) <= 5.4e8:
                return c
        elif kind == "evict":
            last = _log(rng, 1, 256)
            first = rng.choice([0, 1, 4, 16])
            keep = max(first + last, int(T * rng.uniform(0.05, 0.9)))
            c = _case(None, kind, **shape, layers=_log(rng, 1, 36), T=T, ragged=ragged, keep=keep, first=first, last=last)
            if c["layers"] * lists * c["d"] * (T + keep) <= 7.5e8:
                return c
        else:
            m = _log(rng, 2, 256)
            T = m + _log(rng, 1, 2000)
            c = _case(None, kind, **shape, layers=_log(rng, 1, 36), T=T, ragged=False, m=m, path=_log(rng, 1, min(m // 2, 32)))
            if c["layers"] * lists * c["d"] * T <= 4e8:
                return c


# --- inputs -------------------------------------------------------------------------------------

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(shape, gen, dtype=torch.bfloat16):
    return torch.randn(shape, generator=gen, device="cuda", dtype=dtype)


def _held(x):
    """(codes uint8 [..][d/2], scales bf16 [..][d/32]) as a cache holds the rows x (bf16): a scale is the smallest
    number of 5 significant bits that is at least max|x| / 7, and of the eight elements of a 32-bit word
    element i is in nibble i / 2 + 4 (i mod 2), as c + 8."""
    g = x.float().unflatten(-1, (-1, GROUP))
    a = g.abs().amax(-1, keepdim=True)
    a = a / torch.full_like(a, 7)
    s = ((a.view(torch.int32) + 0x7FFFF) >> 19 << 19).view(torch.float32).clamp(2.0 ** -20, 2.0 ** 13)
    c = (torch.floor(g.abs() / s + 0.5) * g.sign()).clamp(-7, 7).flatten(-2)
    w = (c + 8).to(torch.uint8).unflatten(-1, (-1, 4, 2))
    w = w.transpose(-1, -2).reshape(w.shape[:-2] + (4, 2))
    return (w[..., 0] | (w[..., 1] << 4)).flatten(-2), s.squeeze(-1).to(torch.bfloat16)


def _values(codes, scales):
    """The values that held rows stand for, in 32 bits."""
    n = torch.stack([codes & 15, codes >> 4], -1).unflatten(-2, (-1, 4)).flatten(-2)
    c = n.unflatten(-1, (2, 4)).transpose(-1, -2).flatten(-3).float() - 8
    return (c.unflatten(-1, (-1, GROUP)) * scales.float().unsqueeze(-1)).flatten(-2)


def _lengths(case, seed):
    n, T = case["sequences"], case["T"]
    if not case["ragged"]:
        return [T] * n
    r = torch.rand(n, generator=torch.Generator().manual_seed(seed))
    low = max(case.get("m", 1), T // 4)
    return [max(1, int(low + x * (T - low) + 0.5)) for x in r.tolist()]


def _bits(case, seed):
    """What drafts see of one another, bool [n][m][m]: themselves and their ancestors in a tree whose nodes are
    numbered parents first, or any (a tenth of the drafts none)."""
    n, m = case["sequences"], case["m"]
    g = torch.Generator().manual_seed(seed)
    if case["bits"] == "any":
        return (torch.rand((n, m, m), generator=g) < 0.4) & (torch.rand((n, m, 1), generator=g) < 0.9)
    u = torch.rand((n, m), generator=g)
    seen = torch.zeros((n, m, m), dtype=torch.bool)
    at = torch.arange(n)
    for r in range(m):
        parent = (u[:, r] * (r + 1)).long() - 1          # -1: follows the cache's last token
        seen[:, r] = seen[at, parent] & (parent >= 0)[:, None]
        seen[:, r, r] = True
    return seen


def _words(seen):
    """Bits [..][m] as int32 words, bit u % 32 of word u / 32."""
    m = seen.shape[-1]
    x = torch.nn.functional.pad(seen.long(), (0, -m % 32)).unflatten(-1, (-1, 32))
    w = (x << torch.arange(32)).sum(-1)
    return torch.where(w >= 1 << 31, w - (1 << 32), w).to(torch.int32)


def _pool(case, gen, rows, layers=1, filled=True):
    """A state's caches of `rows` rows a sequence: codes and scales of K and V, and block tables if in pages."""
    n, P, Hkv, d = case["sequences"], case["page"], case["kv_heads"], case["d"]
    st = {}
    if P:
        pages = -(-rows // P)
        total = n * pages + n * pages // 8 + 1
        st["tables"] = torch.randperm(total, generator=gen, device="cuda")[:n * pages].to(torch.int32).view(n, pages)
        shape = (layers, total, P, Hkv)
    else:
        shape = (n, layers, Hkv, rows)
    if filled == "values":
        loud = 1 + 2 * (torch.rand((1, d), generator=gen, device="cuda") < 0.03)   # a few channels are larger
        st["K"], st["Ks"] = _held(_randn(shape + (d,), gen) * loud.to(torch.bfloat16))
        st["V"], st["Vs"] = _held(_randn(shape + (d,), gen))
        return st
    for c, s in (("K", "Ks"), ("V", "Vs")):
        if filled:
            st[c] = torch.randint(0, 256, shape + (d // 2,), generator=gen, device="cuda", dtype=torch.uint8)
            st[s] = (torch.randint(16, 32, shape + (d // GROUP,), generator=gen, device="cuda") / 256).to(torch.bfloat16)
        else:
            st[c] = torch.zeros(shape + (d // 2,), device="cuda", dtype=torch.uint8)
            st[s] = torch.zeros(shape + (d // GROUP,), device="cuda", dtype=torch.bfloat16)
    return st


def _gathered(shape, gen, spread=2.5, size=1.0):
    """Weights that rows have gathered: a few rows most of them, many rows none."""
    w = (spread * _randn(shape, gen, torch.float32)).exp_().mul_(size)
    return w.masked_fill_(torch.rand(shape, generator=gen, device="cuda") < 0.1, 0)


def prepare(case, seed):
    gen = _gen(seed)
    n, Hq, Hkv, d, T = (case[k] for k in ("sequences", "q_heads", "kv_heads", "d", "T"))
    Ts = _lengths(case, seed)
    st = dict(case=case, Ts=Ts, T=torch.tensor(Ts, device="cuda"))
    if case["kind"] in ("tree", "weigh"):
        m = case["m"]
        st.update(_pool(case, gen, T, filled="values"))
        st["Q"] = _randn((n, m, Hq, d), gen) * 2
        if case["bits"] in ("tree", "any"):
            st["words"] = _words(_bits(case, seed)).cuda()
        if case["kind"] == "tree":
            st["out"] = torch.empty_like(st["Q"])
            st["lse"] = torch.empty((n, m, Hq), dtype=torch.float32, device="cuda")
        else:
            st["weights"] = _gathered((n, Hkv, T), gen, 1.0, m * (Hq // Hkv) / T)     # as a pass or two of this size leaves
            st["to"] = torch.zeros_like(st["weights"])
            st["lse"] = _logits_and_lse(st)[1].permute(0, 3, 1, 2).reshape(n, m, Hq).contiguous()   # as attention left it
        return st
    nL = case["layers"]
    st.update(_pool(case, gen, T, nL))
    st["weights"] = _gathered((n, nL, Hkv, T), gen)
    st["length"] = torch.tensor(Ts, dtype=torch.int32, device="cuda")
    st["left"] = torch.zeros(n, dtype=torch.int32, device="cuda")
    if case["kind"] == "evict":
        st["into"] = _pool(case, gen, case["keep"], nL, filled=False)
        st["weights_into"] = torch.zeros((n, nL, Hkv, case["keep"]), device="cuda")
        st["idx"] = torch.zeros((n, nL, Hkv, case["keep"]), dtype=torch.int32, device="cuda")
    else:
        # an accepted path, node by node: no place among the kept rows is that of another node of the path
        r = torch.rand((n, case["m"]), generator=gen, device="cuda")
        r[:, :case["path"]] = 2
        st["idx"] = torch.sort(torch.argsort(r, dim=1)[:, :case["path"]], dim=1).values.to(torch.int32)
        st["count"] = torch.randint(1, case["path"] + 1, (n,), generator=gen, device="cuda", dtype=torch.int32)
    return st


# --- one pass -----------------------------------------------------------------------------------

def _cache_values(st, c, s):
    """K or V [n][Hkv][T][d] of a case of one layer, in 32 bits."""
    c, s = st[c], st[s]
    if st["case"]["page"]:
        at = st["tables"].long()
        c, s = (x[0][at].flatten(1, 2)[:, :st["case"]["T"]].transpose(1, 2) for x in (c, s))
    else:
        c, s = c[:, 0], s[:, 0]
    return _values(c, s)


def _seen(st):
    """Rows that each token sees, bool [n][m][T]."""
    case, L = st["case"], st["T"].view(-1, 1, 1)
    m, at = case["m"], torch.arange(case["T"], device="cuda")
    seen = (at < L).expand(-1, m, -1)
    p = L - m + torch.arange(m, device="cuda").view(1, m, 1)
    if case["bits"] == "causal":
        seen = seen & (at <= p)
        if case["window"]:
            seen = seen & (at > p - case["window"])
    if "words" in st:
        bit = (st["words"].unsqueeze(-1) >> torch.arange(32, device="cuda", dtype=torch.int32)) & 1
        u = (at - (L - m)).expand(-1, m, -1)
        among = bit.flatten(-2).bool().gather(2, u.clamp(0, m - 1))
        seen = seen & ((u < 0) | among)
    return seen


def _logits_and_lse(st):
    """Logits [n][Hkv][G][m][T], -inf where nothing is seen, and their log-sum-exp, in 32 bits."""
    case = st["case"]
    Hkv = case["kv_heads"]
    n, m, Hq, d = st["Q"].shape
    q = st["Q"].float().unflatten(2, (Hkv, Hq // Hkv)).permute(0, 2, 3, 1, 4).reshape(n, Hkv, -1, d)
    z = torch.matmul(q, _cache_values(st, "K", "Ks").transpose(-1, -2)).div_(math.sqrt(d))
    z = z.view(n, Hkv, Hq // Hkv, m, -1).masked_fill_(~_seen(st)[:, None, None], -math.inf)
    top = z.amax(-1, keepdim=True).clamp(min=torch.finfo(z.dtype).min)
    return z, (top + (z - top).exp_().sum(-1, keepdim=True).log()).squeeze(-1)


def _plain_tree(st):
    z, lse = _logits_and_lse(st)
    n, m, Hq, d = st["Q"].shape
    a = z.sub_(lse.clamp(min=torch.finfo(z.dtype).min).unsqueeze(-1)).exp_()
    o = torch.matmul(a.flatten(2, 3), _cache_values(st, "V", "Vs")).unflatten(2, (-1, m))
    return {"out": o.permute(0, 3, 1, 2, 4).reshape(n, m, Hq, d).to(torch.bfloat16),
            "lse": lse.permute(0, 3, 1, 2).reshape(n, m, Hq)}


def _fresh(st):
    """Rows that have gathered nothing yet: the tokens' own (all that causal tokens and drafts bring with them)."""
    m = st["case"]["m"] if st["case"]["bits"] != "all" else 0
    at = torch.arange(st["case"]["T"], device="cuda")
    return (at >= st["T"].view(-1, 1) - m)[:, None], (at < st["T"].view(-1, 1))[:, None]


def _plain_weigh(st):
    z, _ = _logits_and_lse(st)
    n, m, Hq, _ = st["Q"].shape
    Hkv = z.shape[1]
    lse = st["lse"].unflatten(2, (Hkv, Hq // Hkv)).permute(0, 2, 3, 1)
    lse = torch.where(lse.isfinite(), lse, torch.full_like(lse, math.inf))
    sums = z.sub_(lse.unsqueeze(-1)).exp_().sum((2, 3))
    fresh, there = _fresh(st)
    before = torch.where(fresh, torch.zeros_like(sums), st["weights"] * st["case"]["decay"])
    return {"weights": torch.where(there, before + sums, st["to"])}


def _rows(st, pool, x, at):
    """Rows `at` [n][nL][Hkv][count] of one of a pool's arrays: [n][nL][Hkv][count][width]."""
    P = st["case"]["page"]
    if not P:
        return pool[x].gather(3, at.unsqueeze(-1).expand(at.shape + pool[x].shape[-1:]))
    n, nL, Hkv, _ = at.shape
    page = pool["tables"].long()[torch.arange(n, device="cuda").view(n, 1, 1, 1), at // P]
    layer, head = (torch.arange(k, device="cuda") for k in (nL, Hkv))
    return pool[x][layer.view(1, nL, 1, 1), page, at % P, head.view(1, 1, Hkv, 1)]


def _put(st, pool, x, first, rows):
    """Rows [n][nL][Hkv][count][width] become the sequences' rows from `first` on."""
    P, count = st["case"]["page"], rows.shape[3]
    if not P:
        pool[x][:, :, :, first:first + count] = rows
        return
    at = torch.arange(first, first + count, device="cuda")
    pool[x][:, pool["tables"].long()[:, at // P], at % P] = rows.permute(1, 0, 3, 2, 4)


def _plain_evict(st):
    c, w = st["case"], st["weights"]
    T, keep = c["T"], min(c["T"], c["keep"])
    L, t, j = st["length"].view(-1, 1, 1, 1), torch.arange(T, device="cuda"), torch.arange(keep, device="cuda")
    rank = w.masked_fill((t < c["first"]) | (t >= L - c["last"]), math.inf).masked_fill_(t >= L, -math.inf)
    at = torch.sort(torch.argsort(rank, dim=-1, descending=True, stable=True)[..., :keep], dim=-1).values
    there = j < L
    st["idx"].fill_(-1)[..., :keep] = torch.where(there, at, -torch.ones_like(at))
    st["weights_into"][..., :keep] = torch.where(there, w.gather(-1, at), st["weights_into"][..., :keep])
    torch.clamp(st["length"], max=c["keep"], out=st["left"])
    own_place = j.expand(at.shape)
    for x in ("K", "V", "Ks", "Vs"):
        _put(st, st["into"], x, 0, torch.where(there.unsqueeze(-1), _rows(st, st, x, at), _rows(st, st["into"], x, own_place)))
    return _evicted(st)


def _evicted(st):
    into = st["into"]
    return {"idx": st["idx"], "left": st["left"], "weights": st["weights_into"], "k": into["K"], "v": into["V"],
            "k_scale": into["Ks"].view(torch.int16), "v_scale": into["Vs"].view(torch.int16)}


def _plain_keep(st):
    c = st["case"]
    first = c["T"] - c["m"]
    j, count = torch.arange(c["path"], device="cuda"), st["count"].view(-1, 1)
    at = first + torch.where(j < count, st["idx"].long(), j)
    at = at[:, None, None].expand(-1, c["layers"], c["kv_heads"], -1)
    for x in ("K", "V", "Ks", "Vs"):
        _put(st, st, x, first, _rows(st, st, x, at))
    st["weights"][..., first:first + c["path"]] = st["weights"].gather(-1, at)
    torch.add(st["count"], first, out=st["left"])
    return _kept(st)


def _kept(st):
    return {"left": st["left"], "weights": st["weights"], "k": st["K"], "v": st["V"],
            "k_scale": st["Ks"].view(torch.int16), "v_scale": st["Vs"].view(torch.int16)}


@functools.lru_cache(maxsize=None)
def _receiver(Hq, Hkv, d, layers, m, T, n):
    import paper_2609_32046_gb300 as cb
    return cb.Receiver(layers, Hq, Hkv, d, m, T, n)


def _caches(st, pool, Ts, lengths=None):
    """A server's sequences keep their views of the pool, their block tables and their lengths."""
    import paper_2609_32046_gb300 as cb
    if "caches" not in pool:
        arrays = [pool[x] for x in ("K", "V", "Ks", "Vs")]
        if st["case"]["page"]:
            pool["caches"] = [cb.PackedKV(*arrays, T=T, pages=t) for T, t in zip(Ts, pool["tables"])]
        else:
            pool["caches"] = [cb.PackedKV(*x, T=T) for *x, T in zip(*arrays, Ts)]
        for i, p in enumerate(pool["caches"]):
            p.length = None if lengths is None else lengths[i:i + 1]
    return pool["caches"]


def _own(st):
    c = st["case"]
    n = c["sequences"]
    rx = _receiver(c["q_heads"], c["kv_heads"], c["d"], c.get("layers", 1), c.get("m", 1), c["T"], n)
    if c["kind"] == "tree":
        rx.attend(_caches(st, st, st["Ts"]), st["Q"], st["out"], lses=st["lse"], trees=st["words"])
        return {"out": st["out"], "lse": st["lse"]}
    if c["kind"] == "weigh":
        rx.weigh(_caches(st, st, st["Ts"]), st["Q"], st["lse"], st["weights"], causal=c["bits"] != "all", window=c["window"],
                 trees=st.get("words"), fresh=0 if c["bits"] == "all" else None, decay=c["decay"], outs=st["to"])
        return {"weights": st["to"]}
    caches = _caches(st, st, [c["T"]] * n, st["length"])
    left = [st["left"][i:i + 1] for i in range(n)]
    if c["kind"] == "evict":
        into = _caches(st, st["into"], [c["keep"]] * n)
        rx.evict(caches, st["weights"], c["keep"], first=c["first"], last=c["last"], into=into, weights_into=st["weights_into"],
                 idx=st["idx"], lengths=left)
        return _evicted(st)
    rx.keep(caches, st["idx"], c["m"], counts=st["count"], weights=st["weights"], lengths=left)
    return _kept(st)


def run(state):
    if own:
        return _own(state)
    return {"tree": _plain_tree, "weigh": _plain_weigh, "evict": _plain_evict, "keep": _plain_keep}[state["case"]["kind"]](state)


# --- what a pass cannot do without ----------------------------------------------------------------

def work(case):
    n, Hq, Hkv, d = (case[k] for k in ("sequences", "q_heads", "kv_heads", "d"))
    held = d // 2 + d // GROUP * 2                               # bytes of one row in 4 bits
    Ts = _lengths(case, 0)
    if case["kind"] in ("evict", "keep"):
        lists = case["layers"] * Hkv
        if case["kind"] == "keep":                               # rows read and written, with their weights
            return {"bytes": n * (lists * case["path"] * 2 * (2 * held + 4) + 4 * case["path"]), "flops": 0}
        return {"bytes": sum(lists * (4 * L + min(L, case["keep"]) * (4 * held + 8)) for L in Ts), "flops": 0}
    m = case["m"]
    pairs = rows = 0
    for L in Ts:
        first, window = 0, case.get("window", 0)
        if case["bits"] == "all":
            pairs += m * L
        elif case["bits"] == "causal":
            w = window or L
            first = max(0, L - m + 1 - w)
            pairs += sum(min(w, L - m + r + 1) for r in range(m) if L - m + r >= 0)
        else:
            pairs += m * max(0, L - m) + (m if case["bits"] == "tree" else 0)
        rows += L - first
    words = n * m * -(-m // 32) * 4 if case["bits"] in ("tree", "any") else 0
    if case["kind"] == "tree":
        return {"bytes": rows * Hkv * 2 * held + n * m * Hq * (d * 4 + 4) + words, "flops": 4 * pairs * Hq * d}
    return {"bytes": rows * Hkv * held + sum(Ts) * Hkv * 8 + n * m * Hq * (d * 2 + 4) + words, "flops": 2 * pairs * Hq * d}


# --- the same in 64 bits ----------------------------------------------------------------------------

def _exact_rows(st, i, c, s):
    """Sequence i's rows [Hkv][L][d] of a case of one layer, from the bytes of its cache, in 64 bits."""
    case, L = st["case"], st["Ts"][i]
    if case["page"]:
        at = torch.arange(L, device="cuda")
        page, row = st["tables"][i].long()[at // case["page"]], at % case["page"]
        c, s = st[c][0][page, row].transpose(0, 1), st[s][0][page, row].transpose(0, 1)
    else:
        c, s = st[c][i, 0, :, :L], st[s][i, 0, :, :L]
    b = c.long().unflatten(-1, (-1, 4))
    word = (b << torch.tensor([0, 8, 16, 24], device="cuda")).sum(-1, keepdim=True)
    shift = torch.tensor([4 * (e // 2) + 16 * (e % 2) for e in range(8)], device="cuda")
    return (((word >> shift) & 15) - 8).flatten(-2).double() * s.double().repeat_interleave(GROUP, -1)


def _exact_blind(st, i, seen):
    """Rows that the tokens of sequence i do not see, bool [m][L]."""
    case, L, m = st["case"], st["Ts"][i], st["case"]["m"]
    t = torch.arange(L, device="cuda")
    p = torch.arange(L - m, L, device="cuda")[:, None]
    if case["bits"] == "all":
        return torch.zeros((m, L), dtype=torch.bool, device="cuda")
    if case["bits"] == "causal":
        return (t > p) | (t <= p - (case["window"] or L + m))
    blind = torch.zeros((m, L), dtype=torch.bool, device="cuda")
    have = min(m, L)
    blind[:, L - have:] = ~seen[i][:, m - have:].cuda()
    return blind


def exact(case, seed):
    st = prepare(case, seed)
    n, Hq, Hkv, d = (case[k] for k in ("sequences", "q_heads", "kv_heads", "d"))
    if case["kind"] in ("tree", "weigh"):
        m, G = case["m"], Hq // Hkv
        seen = _bits(case, seed) if case["bits"] in ("tree", "any") else None
        out = torch.zeros((n, m, Hq, d), dtype=torch.float64, device="cuda")
        lse = torch.full((n, m, Hq), -math.inf, dtype=torch.float64, device="cuda")
        weights = torch.zeros((n, Hkv, case["T"]), dtype=torch.float64, device="cuda")
        for i, L in enumerate(st["Ts"]):
            k = _exact_rows(st, i, "K", "Ks")
            v = _exact_rows(st, i, "V", "Vs") if case["kind"] == "tree" else None
            blind = _exact_blind(st, i, seen)
            if case["kind"] == "weigh":
                old = max(0, L - (0 if case["bits"] == "all" else m))
                weights[i, :, :old] = st["weights"][i, :, :old].double() * case["decay"]
            for h in range(Hq):
                z = (st["Q"][i, :, h].double() @ k[h // G].T / math.sqrt(d)).masked_fill(blind, -math.inf)
                if case["kind"] == "tree":
                    lse[i, :, h] = torch.logsumexp(z, -1)
                    out[i, :, h] = torch.nan_to_num(torch.softmax(z, -1), nan=0.0) @ v[h // G]
                else:
                    a = torch.exp(z - st["lse"][i, :, h, None].double())
                    weights[i, h // G, :L] += torch.nan_to_num(a, nan=0.0, posinf=0.0).sum(0)
        return {"out": out, "lse": lse} if case["kind"] == "tree" else {"weights": weights}
    if case["kind"] == "evict":
        # the rows' weights alone: the rest are whole numbers, and equal or not
        weights = torch.zeros(st["weights_into"].shape, dtype=torch.float64, device="cuda")
        for i, L in enumerate(st["Ts"]):
            inner = st["weights"][i][..., case["first"]:max(case["first"], L - case["last"])].double()
            if L <= case["keep"]:
                weights[i][..., :L] = st["weights"][i][..., :L].double()
                continue
            some = case["keep"] - case["first"] - case["last"]
            order = torch.sort(inner, dim=-1, descending=True, stable=True).indices[..., :some].sort(-1).values
            ends = st["weights"][i].double()
            weights[i] = torch.cat([ends[..., :case["first"]], inner.gather(-1, order), ends[..., L - case["last"]:L]], -1)
        return {"idx": None, "left": None, "weights": weights, "k": None, "v": None, "k_scale": None, "v_scale": None}
    for i, count in enumerate(st["count"].tolist()):
        at = st["Ts"][i] - case["m"]
        old = st["weights"][i].clone()
        for j, node in enumerate(st["idx"][i, :count].tolist()):
            st["weights"][i][..., at + j] = old[..., at + node]
    return {"left": None, "weights": st["weights"].double(), "k": None, "v": None, "k_scale": None, "v_scale": None}
