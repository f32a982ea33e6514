"""Gathered attention weights on the GPU against the definition in 64 bits.

Tolerance of a row's weight, S = the sum it gathers, n = m G terms, B = decay * before:
  E S            every term is off by the factor exp(e), |e| <= E = 2 (d + 8) 2^-23 max sum |q k| scale (products summed in
                 fp32 that may be cut off, and the scaling) + 2^-20 (exp2's approximation) + 2^-22 max |lse| (in log2 domain,
                 rounded twice)
  (n + 8) 2^-23 S  their sum
  2^-23 (S + B)  the last rounding
"""
import math

import pytest
import torch

import budget_reference as ref
import paper_2609_32046_gb300 as cb
from test_gpu_attend import Case
from test_gpu_tree import bits_of

pytestmark = pytest.mark.gpu


class Weighed(Case):
    """A Case whose tokens have attended, and what its rows had gathered."""

    def __init__(self, *args, see=None, layer=0, **kw):
        super().__init__(*args, **kw)
        g = torch.Generator(device="cuda").manual_seed(77)
        self.see, self.layer = see or {}, layer
        self.run(layer=layer, **self.see)
        self.before = [torch.randn(self.Hkv, p.capacity, generator=g, device="cuda").abs() for p in self.caches]
        self.weights = [x.clone() for x in self.before]

    def weigh(self, **kw):
        return self.rx.weigh(self.caches, self.q, self.lse, self.weights, layer=self.layer, **{**self.see, **kw})

    def check(self, bits=None, fresh=None, decay=1.0, lengths=None, got=None, before=None):
        self.rx.sync_status()
        for i, q in enumerate(self.q):
            m, T = q.shape[0], self.caches[i].T
            L = T if lengths is None else max(0, min(T, lengths[i]))
            w = (got or self.weights)[i]
            had = (before or self.before)[i]
            if m == 0:
                assert torch.equal(w, self.before[i])
                continue
            k, _ = self.kv(i, self.layer, L)
            b = None if bits is None else bits[i]
            if b is not None and m > L:
                sees = b[:, m - L:].cuda()
            else:
                sees = ref.seen(m, L, self.see.get("causal", True), self.see.get("window", 0), b).cuda()
            lse = self.lse[i].double()
            S, size = ref.weights(q.double(), k, lse, 1 / math.sqrt(self.d), sees)
            old = had[:, :L].double() * decay
            n = m if fresh is None else fresh
            old[:, max(0, L - n):] = 0
            finite = lse[torch.isfinite(lse)]
            E = 2 * (self.d + 8) * 2.0 ** -23 * size + 2.0 ** -20 + 2.0 ** -22 * float(finite.abs().max() if finite.numel() else 0)
            tol = S * (math.expm1(E) + (m * self.Hq // self.Hkv + 8) * 2.0 ** -23) + 2.0 ** -23 * (S + old)
            err = (w[:, :L].double() - old - S).abs()
            assert (err <= tol).all(), "sequence %d: off by %.3g, %.3g over" % (i, float(err.max()), float((err - tol).max()))
            assert torch.equal(w[:, L:], (got or self.before)[i][:, L:] if got is None else w[:, L:])


HEADS = [(128, 32, 8), (128, 4, 2), (128, 2, 2), (64, 8, 2), (64, 4, 4), (64, 2, 1)]


@pytest.mark.parametrize("d,Hq,Hkv", HEADS)
@pytest.mark.parametrize("m,T", [(1, 1), (1, 33), (1, 1000), (1, 4097), (2, 2), (3, 40), (4, 700), (5, 129), (16, 17), (17, 333),
                                 (31, 31), (33, 1000), (64, 2051), (65, 130), (127, 500), (128, 129), (200, 1500), (300, 1111)])
@pytest.mark.parametrize("causal", [True, False])
def test_one_sequence(d, Hq, Hkv, m, T, causal):
    c = Weighed(d, Hq, Hkv, [m], [T], seed=m, see=dict(causal=causal), room=7)
    c.weigh()
    c.check()


@pytest.mark.parametrize("d,Hq,Hkv", [(128, 8, 2), (64, 8, 2), (64, 2, 2)])
@pytest.mark.parametrize("page", [0, 1, 16, 64])
@pytest.mark.parametrize("m", [1, 6, 70])
def test_ragged_batches_in_every_layout(d, Hq, Hkv, page, m):
    Ts = [m, 15 + m, 16 + m, 17 + m, 255 + m, 600, 1, 1025]
    ms = [m, 1, m, max(1, m - 1), m, 0, 1, m]
    c = Weighed(d, Hq, Hkv, ms, Ts, page=page, layers=2, layer=1, layout="positions" if page == 0 else "heads", room=40)
    c.weigh(decay=0.75)
    c.check(decay=0.75)


@pytest.mark.parametrize("d,Hq,Hkv", [(128, 4, 1), (64, 2, 2)])
@pytest.mark.parametrize("m", [1, 5, 150])
@pytest.mark.parametrize("window", [1, 2, 33, 100, 1000, 2 ** 62])
def test_windows(d, Hq, Hkv, m, window):
    """Rows that no token sees only fade."""
    c = Weighed(d, Hq, Hkv, [m, m, m], [m, 400 + m, 2000], seed=5, page=16, see=dict(window=window))
    c.weigh(decay=0.5)
    c.check(decay=0.5)


@pytest.mark.parametrize("d,Hq,Hkv", [(128, 8, 2), (64, 4, 4)])
@pytest.mark.parametrize("m", [1, 4, 15, 40, 200])
@pytest.mark.parametrize("kind", ["tree", "any", "none"])
def test_drafted_tokens(d, Hq, Hkv, m, kind):
    Ts = [m, m + 30, 1000, max(1, m // 2)]
    bits = [bits_of(kind, m, i) for i in range(4)]
    bits[2] = None
    words = [None if x is None else cb.pack_words(x).cuda() for x in bits]
    c = Weighed(d, Hq, Hkv, [m] * 4, Ts, page=16, see=dict(trees=words))
    c.weigh()
    c.check(bits)


@pytest.mark.parametrize("m", [1, 3, 100])
@pytest.mark.parametrize("fresh", [0, 2, 10 ** 6])
def test_rows_that_have_gathered_nothing(m, fresh):
    """`before` of fresh rows is not read (NaN there), nor rows behind the last written."""
    c = Weighed(128, 8, 2, [m, m], [500, 300], room=20)
    for x, b, T in zip(c.weights, c.before, (500, 300)):
        x[:, max(0, T - fresh):] = float("nan")
    kept = [x.clone() for x in c.weights]
    c.weigh(fresh=fresh)
    for x, k, T in zip(c.weights, kept, (500, 300)):
        assert torch.equal(x[:, T:].isnan(), k[:, T:].isnan())
        x[:, T:] = 0
    for b, T in zip(c.before, (500, 300)):
        b[:, T:] = 0
    c.check(fresh=fresh)


@pytest.mark.parametrize("m", [1, 80])
def test_into_other_memory(m):
    """outs beside weights, in one tensor with the sequences first, wider than the cache; weights None."""
    c = Weighed(64, 4, 2, [m] * 3, [m, 200, 333])
    q, lse = torch.stack(c.q), torch.stack(c.lse)
    room = torch.full((3, 2, 600), 9.0, device="cuda")
    had = torch.rand(3, 2, 600, device="cuda")
    got = c.rx.weigh(c.caches, q, lse, had, outs=room, decay=0.25)
    assert got is room
    c.check(got=[x for x in room], before=[x for x in had], decay=0.25)
    assert all((room[i, :, p.T:] == 9).all() for i, p in enumerate(c.caches))
    c.rx.weigh(c.caches, q, lse, None, outs=room, fresh=0)
    c.check(got=[x for x in room], before=[torch.zeros_like(x) for x in had])


@pytest.mark.parametrize("m", [1, 4, 90])
def test_lengths_on_the_device(m):
    Ts, lengths = [900, 900, 900, 900, 300], [1, 899, 5000, 0, 77]
    c = Weighed(128, 8, 2, [m] * 5, Ts, lengths=lengths, page=16)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.run()
        c.weigh()
    for grown in (lengths, [640, 641, 10, 700, -3]):
        for p, x in zip(c.caches, grown):
            p.length.fill_(x)
        for w, b in zip(c.weights, c.before):
            w.copy_(b)
        graph.replay()
        c.check(lengths=grown)


@pytest.mark.parametrize("m", [1, 4, 60])
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_heads_left_out(m, bad):
    """A head whose lse is not finite adds nothing, whatever its query holds."""
    c = Weighed(128, 8, 2, [m, m], [300, 1000])
    c.lse[0][0, 3] = bad
    c.lse[1][:, 1::2] = bad
    c.q[0][0, 3] = float("nan")
    c.q[1][:, 1] = float("inf")
    want = [q.clone() for q in c.q]
    want[0][0, 3] = 0
    want[1][:, 1] = 0
    c.weigh()
    c.q = want
    c.check()


@pytest.mark.parametrize("m", [1, 60])
@pytest.mark.parametrize("scale", [2.0 ** -20, 2.0 ** 13])
def test_scales_at_both_ends(m, scale):
    c = Case(128, 8, 2, [m], [600], seed=9)
    c.caches[0].k_scale.fill_(scale)
    c.q[0].mul_(2.0 ** -13)
    c.run()
    w = torch.zeros(2, 600, device="cuda")
    c.rx.weigh(c.caches, c.q, c.lse, [w])
    c.rx.sync_status()
    k, _ = c.kv(0, 0, 600)
    S, size = ref.weights(c.q[0].double(), k, c.lse[0].double(), 1 / math.sqrt(128), ref.seen(m, 600).cuda())
    E = 2 * 136 * 2.0 ** -23 * size + 2.0 ** -20 + 2.0 ** -22 * float(c.lse[0].abs().max())
    assert ((w.double() - S).abs() <= S * (math.expm1(E) + (4 * m + 9) * 2.0 ** -23)).all()


@pytest.mark.parametrize("m", [1, 40, 130])
def test_bad_scales_and_pages_read_as_zeros(m):
    c = Weighed(128, 8, 2, [m, m], [500, 500], page=16)
    p = c.caches[0]
    page = int(p.pages[2])
    p.k_scale[0, page, 5, 1, 2] = float("nan")
    c.weigh()
    with pytest.raises(cb.CBError) as e:
        c.rx.sync_status()
    assert e.value.status == cb.CB_EDEVICE
    p.k_scale[0, page, 5, 1, 2] = 0
    c.check()
    table = p.pages.clone()
    p.pages[3] = p.n_pages
    for w, b in zip(c.weights, c.before):
        w.copy_(b)
    c.weigh()
    with pytest.raises(cb.CBError):
        c.rx.sync_status()
    p.pages.copy_(table)
    rows = slice(48, 64)
    got = c.weights[0].clone()
    for w, b in zip(c.weights, c.before):
        w.copy_(b)
    c.weigh()
    c.check()
    other = torch.ones(500, dtype=torch.bool, device="cuda")
    other[rows] = False
    assert torch.equal(got[:, :500][:, other], c.weights[0][:, :500][:, other])


@pytest.mark.parametrize("m", [1, 7, 200])
def test_repeated_and_concurrent_runs_are_alike(m):
    c = Weighed(128, 8, 2, [m] * 4, [400 + m, 2000, m, 1300], page=16)
    c.weigh()
    first = [w.clone() for w in c.weights]
    others = [cb.Receiver(1, 8, 2, 128, max(m, 1), 4000, 4) for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in others]
    outs = [[torch.zeros_like(w) for w in c.weights] for _ in others]
    torch.cuda.synchronize()
    for _ in range(5):
        for rx, s, o in zip(others, streams, outs):
            rx.weigh(c.caches, c.q, c.lse, c.before, outs=o, stream=s)
    torch.cuda.synchronize()
    for o in outs:
        for a, b, p in zip(first, o, c.caches):
            assert torch.equal(a[:, :p.T], b[:, :p.T])


@pytest.mark.parametrize("d,Hq,Hkv", [(128, 4, 1), (64, 4, 1), (64, 2, 2)])
@pytest.mark.parametrize("m,T", [(64, 700), (65, 2000), (128, 3333), (129, 129), (500, 1500), (1024, 1024), (1024, 3000)])
@pytest.mark.parametrize("see", [dict(), dict(window=40), dict(window=700), dict(causal=False)])
def test_many_query_rows(d, Hq, Hkv, m, T, see):
    """Rows that stay in shared memory while positions pass, and rows that pass; tiles that no token sees."""
    c = Weighed(d, Hq, Hkv, [m, 20, m], [T, 5000, T // 2 + m], seed=m, page=16, see=see)
    c.weigh(decay=0.5)
    c.check(decay=0.5)


@pytest.mark.parametrize("m", [150, 600, 1024])
def test_many_drafts(m):
    """Trees of more tokens than stay in shared memory."""
    bits = [bits_of("tree", m, 0), None, bits_of("any", m, 2)]
    c = Weighed(128, 4, 1, [m] * 3, [m, 900 + m, 2000], see=dict(trees=[None if x is None else cb.pack_words(x).cuda() for x in bits]))
    c.weigh()
    c.check(bits)


@pytest.mark.parametrize("d", [64, 128])
def test_more_segments_than_blocks(d):
    """Runs of a few tiles that end inside items, many items a block, rows that pass and rows that stay in one call."""
    n = 40
    c = Weighed(d, 16, 8, [9 + 53 * (i % 6) for i in range(n)], [300 + 97 * i for i in range(n)], page=32)
    c.weigh()
    c.check()


def test_a_long_cache():
    """More tiles a block than one segment may have: a row's sum does not depend on the call that it is in."""
    T = 152 * 1024 * 128 + 5000
    g = torch.Generator(device="cuda").manual_seed(3)
    codes = [torch.randint(0, 256, (1, 1, T, 32), generator=g, device="cuda", dtype=torch.uint8) for _ in range(2)]
    scales = [torch.rand((1, 1, T, 2), generator=g, device="cuda").to(torch.bfloat16) for _ in range(2)]
    q = torch.randn((5, 4, 64), generator=g, device="cuda").to(torch.bfloat16)
    lse = torch.full((5, 4), 6.0, device="cuda")
    rx = cb.Receiver(1, 4, 1, 64, 5, T, 2)
    whole, halves = torch.zeros(1, T, device="cuda"), torch.zeros(1, T, device="cuda")
    rx.weigh([cb.PackedKV(*codes, *scales)], [q], [lse], None, outs=[whole], causal=False)
    cut = 7 * 128 * 1000 + 3
    parts = [cb.PackedKV(*[x[:, :, i] for x in codes + scales]) for i in (slice(0, cut), slice(cut, T))]
    for p, out in zip(parts, (halves[:, :cut], halves[:, cut:])):
        rx.weigh([p], [q], [lse], None, outs=[out], causal=False)
    rx.sync_status()
    assert torch.equal(whole, halves) and bool((whole > 0).all())


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("m", [30, 300])
def test_a_wait_that_gives_up(d, m):
    """A bounded wait runs out on a barrier that nothing arrives on: an error status, and the context goes on."""
    c = Weighed(d, 8, 2, [m, m], [1500, 700 + m])
    c.rx.set_wait_limit(20_000_000, stall_next_weigh=True)           # 20 ms
    c.weigh()
    with pytest.raises(cb.CBError) as e:
        c.rx.sync_status()
    assert e.value.status == cb.CB_ETIMEOUT
    for w, b in zip(c.weights, c.before):
        w.copy_(b)
    c.weigh()
    c.check()


@pytest.mark.parametrize("m", [1, 9, 40])
def test_more_heads_than_blocks(m):
    c = Weighed(64, 900, 900, [m, 1], [70, 200])
    c.weigh()
    c.check()


def test_weights_of_a_softmax_sum_to_one():
    c = Weighed(128, 32, 8, [70], [3000])
    w = torch.zeros(8, 3000, device="cuda")
    c.rx.weigh(c.caches, c.q, c.lse, [w])
    assert ((w.double().sum(1) - 70 * 4).abs() < 70 * 4 * 1e-4).all()


def test_more_sequences_than_a_launch_takes():
    n = 70
    c = Weighed(64, 2, 2, [1] * n, [1 + 13 * i for i in range(n)])
    c.weigh()
    c.check()


def test_refusals():
    c = Weighed(128, 8, 2, [8, 8], [100, 100])
    w = c.weights
    rx = c.rx
    for kw in (dict(weights=w[:1]), dict(weights=[w[0].half(), w[1]]), dict(weights=[w[0][:1], w[1]]), dict(weights=[w[0][:, :99], w[1]]),
               dict(weights=None), dict(lses=[c.lse[0][:5], c.lse[1]]), dict(Qs=[c.q[0].float(), c.q[1]]), dict(window=3, causal=False),
               dict(fresh=[1]), dict(weights=[w[0].t().contiguous().t(), w[1]])):
        with pytest.raises(ValueError):
            rx.weigh(**{**dict(caches=c.caches, Qs=c.q, lses=c.lse, weights=w), **kw})
    for kw in (dict(decay=1.5), dict(decay=-0.1), dict(decay=math.nan), dict(fresh=-1), dict(layer=1), dict(window=-1),
               dict(weights=[w[0], w[0]]), dict(weights=[w[0].cpu(), w[1]]),
               dict(outs=[torch.zeros(150, device="cuda").as_strided((2, 100), (50, 1)), None]),
               dict(decay=2.0)):
        with pytest.raises(cb.CBError):
            rx.weigh(**{**dict(caches=c.caches, Qs=c.q, lses=c.lse, weights=w), **kw})
    both = torch.zeros(2, 250, device="cuda")
    with pytest.raises(cb.CBError):
        rx.weigh(c.caches, c.q, c.lse, [both[:, :200], w[1]], outs=[both[:, 20:220], None])        # overlaps `before`
    spare = torch.zeros_like(w[0])
    with pytest.raises(cb.CBError):
        rx.weigh(c.caches, c.q, c.lse, w, outs=[spare, w[0]])                                      # the second writes what the first reads
    rx.sync_status()
    for a, b in zip(c.weights, c.before):
        assert torch.equal(a, b)
