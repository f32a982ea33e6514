"""Attention over 4-bit caches on the GPU against the definition in 64 bits.

Tolerance of an output element, A = sum_t a_t |v_t|:
  2^-8 |out|        its rounding to bf16 (half a step)
  2^-11 A           weights rounded to fp16 (half a step), the values exact
  2^-32 T max|v|    weights below fp16's smallest step: they are held times 2^7 or more over the row's largest,
                    which the sum is no smaller than, and are off by half of 2^-24
  2 E A             every weight is off by the factor exp(e), |e| <= E, in the sum above and in the sum below:
                    E = 2 (d + 8) 2^-23 max sum |q k| scale (products summed in fp32 that may be cut off
                    instead of rounded, and the scaling) + 2^-20 (exp2's approximation) + T 2^-23 (sums of T terms)
The log-sum-exp: E + 2^-22 |lse| + 2^-21."""
import math

import pytest
import torch

import paper_2609_32046_gb300 as cb
import packed_reference as ref

pytestmark = pytest.mark.gpu


class Case:
    """Sequences with packed caches in one layout, their queries, outputs and 64-bit values."""

    def __init__(self, d, Hq, Hkv, ms, Ts, page=0, layers=1, seed=0, layout="heads", spread=1.0, lengths=None, room=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        n = len(Ts)
        randn = lambda *s: torch.randn(s, generator=g, device="cuda").to(torch.bfloat16)   # noqa: E731
        self.d, self.Hq, self.Hkv, self.layers = d, Hq, Hkv, layers
        self.q = [(spread * randn(m, Hq, d)).to(torch.bfloat16) for m in ms]
        self.out = [torch.full_like(q, 7.0) for q in self.q]
        self.lse = [torch.full((m, Hq), 7.0, device="cuda") for m in ms]
        self.caches = []
        self.rx = cb.Receiver(layers, Hq, Hkv, d, max(max(ms), 1), max(max(Ts) + room, 1) + 64, n)
        widths = ((d // 2, torch.uint8),) * 2 + ((d // 32, torch.bfloat16),) * 2
        if page:
            need = [-(-(T + room) // page) for T in Ts]
            total = sum(need) + 5
            order = torch.randperm(total, generator=torch.Generator().manual_seed(seed)).int()
            # what no block table names, and the rows behind each sequence, hold NaN scales
            pool = [torch.full((layers, total, page, Hkv, w), 255 if t == torch.uint8 else float("nan"), dtype=t,
                               device="cuda") for w, t in widths]
        at = 0
        for i, T in enumerate(Ts):
            if page:
                table = order[at:at + need[i]].cuda()
                at += need[i]
                p = cb.PackedKV(*pool, T=T, pages=table)
            elif layout == "heads":
                p = cb.PackedKV(*[torch.full((layers, Hkv, T + room, w), 255 if t == torch.uint8 else float("nan"), dtype=t,
                                             device="cuda") for w, t in widths], T=T)
            else:      # position-major
                p = cb.PackedKV(*[torch.full((layers, T + room, Hkv, w), 255 if t == torch.uint8 else float("nan"), dtype=t,
                                             device="cuda").transpose(1, 2) for w, t in widths], T=T)
            if lengths is not None:
                p.length = torch.tensor([lengths[i]], dtype=torch.int32, device="cuda")
            self.caches.append(p)
            if T:
                self.rx.pack([randn(layers, Hkv, T, d)], [randn(layers, Hkv, T, d)], [p], [0])
        self.rx.sync_status()

    def run(self, **kw):
        self.rx.attend(self.caches, self.q, self.out, lses=self.lse, **kw)

    def kv(self, i, layer, T):
        p = self.caches[i]
        arrays = []
        for c, s in ((p.k, p.k_scale), (p.v, p.v_scale)):
            c, s = c[layer], s[layer]
            if p.pages is not None:
                c, s = (x[p.pages.long()].flatten(0, 1).transpose(0, 1) for x in (c, s))
            arrays.append(ref.values(c[:, :T].contiguous(), s[:, :T].contiguous()))
        return arrays

    def check(self, layer=0, causal=True, window=0, lengths=None, which=None):
        self.rx.sync_status()
        worst = 0.0
        for i in range(len(self.q)) if which is None else which:
            q = self.q[i]
            if q.shape[0] == 0:
                continue
            T = self.caches[i].T
            L = T if lengths is None else max(0, min(T, lengths[i]))
            k, v = self.kv(i, layer, L)
            scale = 1 / math.sqrt(self.d)
            o, lse, A, size = ref.attention(q.double(), k, v, scale, causal, window)
            E = 2 * (self.d + 8) * 2.0 ** -23 * size + 2.0 ** -20 + L * 2.0 ** -23
            big = float(v.abs().max()) if L else 0.0
            tol = o.abs() * 2.0 ** -8 + A * (2.0 ** -11 + 2 * E) + 2.0 ** -32 * L * big
            err = (self.out[i].double() - o).abs()
            assert (err <= tol).all(), "sequence %d: off by %.3g more than %.3g" % (i, float((err - tol).max()), float(tol.mean()))
            empty = torch.isinf(lse)
            assert torch.equal(torch.isinf(self.lse[i]), empty) and (self.out[i][empty] == 0).all()
            off = (self.lse[i].double() - lse)[~empty].abs()
            assert (off <= E + 2.0 ** -22 * lse[~empty].abs() + 2.0 ** -21).all()
            if o.norm() > 0:
                worst = max(worst, float((self.out[i].double() - o).norm() / o.norm()))
        return worst


HEADS = [(128, 32, 8), (128, 4, 2), (128, 2, 2), (64, 8, 2), (64, 4, 4), (64, 2, 1), (128, 4, 1)]


@pytest.mark.parametrize("d,Hq,Hkv", HEADS)
@pytest.mark.parametrize("T", [1, 2, 31, 33, 128, 129, 1000, 4097])
def test_one_token(d, Hq, Hkv, T):
    c = Case(d, Hq, Hkv, [1], [T], seed=T)
    c.run()
    c.check()
    c.run(causal=False)
    c.check(causal=False)


@pytest.mark.parametrize("d,Hq,Hkv", HEADS)
@pytest.mark.parametrize("m,T", [(2, 2), (3, 40), (5, 700), (16, 17), (17, 333), (31, 31), (33, 1000), (64, 64), (64, 2051),
                                 (65, 130), (127, 500), (128, 129), (200, 1500), (257, 257), (300, 1111)])
@pytest.mark.parametrize("causal", [True, False])
def test_several_tokens(d, Hq, Hkv, m, T, causal):
    c = Case(d, Hq, Hkv, [m], [T], seed=m)
    c.run(causal=causal)
    c.check(causal=causal)


@pytest.mark.parametrize("d,Hq,Hkv", [(128, 8, 2), (64, 8, 2), (64, 2, 2)])
@pytest.mark.parametrize("page", [0, 1, 4, 16, 32, 64, 256])
@pytest.mark.parametrize("m", [1, 6, 70])
def test_ragged_batches_in_every_layout(d, Hq, Hkv, page, m):
    """Lengths around pages and tiles, token counts that differ, two layers, unused pages full of NaN."""
    Ts = [m, 15 + m, 16 + m, 17 + m, 255 + m, 600, 1, 1025]
    ms = [m, 1, m, max(1, m - 1), m, 0, 1, m]
    c = Case(d, Hq, Hkv, ms, Ts, page=page, layers=2, layout="positions" if page == 0 else "heads", room=40)
    c.run(layer=1)
    c.check(layer=1)
    assert (c.lse[5] == 7).all() if ms[5] else c.lse[5].numel() == 0
    c.run(layer=0, causal=False)
    c.check(layer=0, causal=False)


@pytest.mark.parametrize("d,Hq,Hkv", [(128, 4, 1), (64, 2, 2)])
@pytest.mark.parametrize("m", [1, 5, 150])
@pytest.mark.parametrize("window", [1, 2, 33, 100, 1000, 100000])
def test_windows(d, Hq, Hkv, m, window):
    c = Case(d, Hq, Hkv, [m, m, m], [m, 400 + m, 2000], seed=window, page=16)
    c.run(window=window)
    c.check(window=window)


@pytest.mark.parametrize("m", [1, 9, 80, 200])
def test_rows_that_see_nothing(m):
    """Fewer rows than tokens, and none at all: the first tokens see nothing."""
    c = Case(128, 8, 2, [m] * 4, [0, 1, m // 2, m], seed=m)
    c.run()
    c.check()
    c.run(causal=False)
    c.check(causal=False)


@pytest.mark.parametrize("m", [1, 4, 90])
def test_lengths_on_the_device(m):
    """Lengths as the kernel finds them: below, at and above T, none, negative; a captured call follows them."""
    Ts = [900, 900, 900, 900, 900, 300]
    lengths = [1, 899, 5000, 0, -3, 77]
    c = Case(128, 8, 2, [m] * 6, Ts, lengths=lengths, page=16)
    c.run()
    c.check(lengths=lengths)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.run()
    for grown in ([2, 900, 899, 1, 0, 78], [640, 641, 10, 700, 3, 300]):
        for p, x in zip(c.caches, grown):
            p.length.fill_(x)
        graph.replay()
        c.check(lengths=grown)


@pytest.mark.parametrize("m", [1, 60])
@pytest.mark.parametrize("spread", [8.0, 60.0])
def test_wide_logits(m, spread):
    """Logits of a standard deviation of 8 and 60: the running maximum rises late and by much."""
    c = Case(128, 8, 2, [m, m], [3000, 5000], spread=spread, seed=5)
    c.caches[0].k_scale[:, :, 2900:] *= 2          # (2 s is a scale as well)
    c.run()
    c.check()


@pytest.mark.parametrize("m", [1, 60, 140])
@pytest.mark.parametrize("scale", [2.0 ** -20, 2.0 ** 13])
def test_scales_at_both_ends(m, scale):
    """Values at the ends of what can be held: products stay exact, outputs in range."""
    c = Case(128, 8, 2, [m], [600], seed=9)
    c.caches[0].v_scale.fill_(scale)
    c.run()
    c.check()


@pytest.mark.parametrize("m", [1, 40, 130])
def test_bad_scales_and_pages_read_as_zeros(m):
    c = Case(128, 8, 2, [m, m], [500, 500], page=16)
    good = [x.clone() for x in c.out]
    c.run()
    c.check()
    good = [x.clone() for x in c.out]
    p = c.caches[0]
    row = (0, int(p.pages[3]), 5, 1)
    p.k_scale[row] = float("nan")
    p.v_scale[row] = float("inf")
    p.v_scale[0, int(p.pages[4]), 2, 0, 1] = -1.0
    c.run()
    with pytest.raises(cb.CBError, match="CB_EDEVICE.*scale"):
        c.rx.sync_status()
    assert torch.equal(c.out[1], good[1])
    for s in (p.k_scale, p.v_scale):
        s[row] = 0
    p.v_scale[0, int(p.pages[4]), 2, 0, 1] = 0
    c.run()
    c.check()
    # block-table entries outside the pool: rows of zeros, of weight exp(0 - lse)
    was = p.pages.clone()
    for bad in (-1, p.n_pages, 1 << 30):
        p.pages[7] = bad
        c.run()
        with pytest.raises(cb.CBError, match="CB_EDEVICE.*block-table"):
            c.rx.sync_status()
        assert torch.equal(c.out[1], good[1])
        p.pages.copy_(was)
        at = int(was[7])
        keep = [x[:, at].clone() for x in (p.k, p.v)]
        p.k[:, at] = 0x88
        p.v[:, at] = 0x88
        c.check(which=[0])
        p.k[:, at], p.v[:, at] = keep


def test_query_strides_and_outputs_beside_others():
    """Queries inside a fused tensor, outputs head-major; sequences that share one cache."""
    c = Case(128, 8, 2, [12, 12], [300, 300])
    c.caches[1] = c.caches[0]
    fused = torch.randn((2, 12, 12, 128), device="cuda").to(torch.bfloat16)
    c.q = [fused[i, :, 2:10] for i in range(2)]
    room = torch.full((2, 9, 12, 128), 5.0, dtype=torch.bfloat16, device="cuda")
    c.out = [room[i, :8].transpose(0, 1) for i in range(2)]
    c.run()
    c.check()
    assert (room[:, 8] == 5).all()


def test_infinite_and_nan_queries_stay_in_their_rows():
    for m in (3, 100):
        c = Case(128, 8, 2, [m], [400])
        c.q[0][1, 2, 7] = float("nan")
        c.q[0][2, 5, 9] = float("inf")
        c.run()
        bad = torch.zeros((m, 8), dtype=torch.bool, device="cuda")
        bad[1, 2] = bad[2, 5] = True
        assert torch.isnan(c.out[0][1, 2]).all()
        c.q[0][bad] = 0
        o = c.out[0].clone()
        c.run()
        c.check()
        assert torch.equal(o[~bad], c.out[0][~bad])


@pytest.mark.parametrize("m", [1, 50])
def test_the_same_bits_every_time_and_on_another_stream(m):
    c = Case(128, 32, 8, [m] * 3, [3000, 100, 1999], page=16)
    c.run()
    torch.cuda.synchronize()
    first = [x.clone() for x in c.out + c.lse]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    c.run(stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, c.out + c.lse))
    c.check()


def test_more_sequences_than_one_launch_takes():
    c = Case(64, 2, 2, [1] * 70, [20 + 3 * i for i in range(70)])
    c.run()
    c.check()


def test_rows_past_32_bits():
    """One layer of a pool whose later layers lie past 2^32 elements, and a long cache in it."""
    Hkv, d, T, layers = 2, 128, 1 << 20, 20
    rx = cb.Receiver(layers, 4, Hkv, d, 2, T, 1)
    arrays = [torch.zeros((layers, Hkv, T, w), dtype=t, device="cuda")
              for w, t in ((d // 2, torch.uint8),) * 2 + ((d // 32, torch.bfloat16),) * 2]
    p = cb.PackedKV(*arrays)
    K, V = (torch.randn((1, Hkv, 1000, d), device="cuda").to(torch.bfloat16) for _ in range(2))
    rx.pack([K], [V], [p], [T - 1000], layer=layers - 1)
    c = Case(d, 4, Hkv, [2], [1])
    c.rx, c.caches = rx, [p]
    c.run(layer=layers - 1, window=900)
    rx.sync_status()
    k, v = (ref.values(a[layers - 1, :, T - 1000:], s[layers - 1, :, T - 1000:]) for a, s in ((p.k, p.k_scale), (p.v, p.v_scale)))
    o, lse, A, size = ref.attention(c.q[0].double(), k, v, 1 / math.sqrt(d), True, 900)
    E = 2 * (d + 8) * 2.0 ** -23 * size + 2.0 ** -20 + 1000 * 2.0 ** -23
    assert ((c.out[0].double() - o).abs() <= o.abs() * 2.0 ** -8 + A * (2.0 ** -11 + 2 * E) + 1e-6).all()


def test_a_score_context_attends_too():
    """A context of cb_create: allocates in its first call, refuses that inside a capture."""
    a = Case(128, 8, 2, [4], [200])
    c = cb.CacheBack(1, 8, 2, 128, 8, 512)
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        graph.capture_begin()
        with pytest.raises(cb.CBError, match="CB_ENOMEM"):
            c.attend(a.caches, a.q, a.out, lses=a.lse)
        torch.zeros(1, device="cuda")
        graph.capture_end()
    torch.cuda.synchronize()
    before = c.scratch_bytes
    c.attend(a.caches, a.q, a.out, lses=a.lse)
    assert c.scratch_bytes > before
    a.check()


def test_a_receivers_step():
    """Score, select and pack a sender's rows; then prompt chunks and single tokens: rotary, pack, attend, all of
    it as one captured graph per token that follows device positions and lengths; against a plain receiver."""
    nL, Hq, Hkv, d, T, m = 2, 8, 2, 128, 700, 24
    g = torch.Generator(device="cuda").manual_seed(0)
    randn = lambda *s: torch.randn(s, generator=g, device="cuda").to(torch.bfloat16)   # noqa: E731
    sender = cb.CacheBack(nL, Hq, Hkv, d, m, T)
    f = cb.Filter(sender, [(randn(nL, Hkv, T, d), randn(nL, Hkv, T, d))], [randn(nL, m, Hq, d)], 0.25)
    f.score(); f.select()
    room, page = 300, 16
    B = f.budgets[0]
    table = torch.randperm(-(-room // page) + 4, generator=g, device="cuda")[:-(-room // page)].int()
    widths = ((d // 2, torch.uint8),) * 2 + ((d // 32, torch.bfloat16),) * 2
    held = cb.PackedKV(*[torch.zeros((nL, len(table) + 4, page, Hkv, w), dtype=t, device="cuda") for w, t in widths],
                       pages=table, length=torch.zeros(1, dtype=torch.int32, device="cuda"))
    assert f.pack(held) is held and held.T == B
    sender.sync_status()
    held.T = held.capacity
    rx = cb.Receiver(nL, Hq, Hkv, d, m, 512)
    rope = cb.Rotary(1e6)
    pos = torch.zeros(m, dtype=torch.int32, device="cuda")
    q, k, v, out = (torch.zeros((nL, m, h, d), dtype=torch.bfloat16, device="cuda") for h in (Hq, Hkv, Hkv, Hq))
    qr, kr = torch.empty_like(q), torch.empty_like(k)

    def step(n):
        for layer in range(nL):
            rx.rotary([q[layer, :n], k[layer, :n]], rope, [qr[layer, :n], kr[layer, :n]], pos=pos[:n])
            rx.pack([kr[layer:layer + 1, :n].transpose(1, 2)], [v[layer:layer + 1, :n].transpose(1, 2)], [held], rows=[pos[:n]],
                    layer=layer)
            rx.attend([held], [qr[layer, :n]], [out[layer, :n]], layer=layer)

    step(1)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(1)
    at = B
    for n in (m, 1, 1, 1, 7, 1):
        pos[:n] = torch.arange(at, at + n, dtype=torch.int32, device="cuda")
        held.length.fill_(at + n)
        for x, h in ((q, Hq), (k, Hkv), (v, Hkv)):
            x[:, :n] = randn(nL, n, h, d)
        if n == 1:
            graph.replay()
        else:
            step(n)
        at += n
        rx.sync_status()
        for layer in range(nL):
            arrays = [ref.values(*(x[layer][table.long()].flatten(0, 1).transpose(0, 1)[:, :at].contiguous() for x in pair))
                      for pair in ((held.k, held.k_scale), (held.v, held.v_scale))]
            want = ref.rotary(k[layer, :n], pos[:n], *ref.frequencies(d, 1e6), "halves")
            assert (arrays[0][:, at - n:at].transpose(0, 1) - want).abs().max() <= want.abs().max() / 14 * 1.07 + 2.0 ** -6
            o, _, A, _ = ref.attention(qr[layer, :n].double(), *arrays, 1 / math.sqrt(d))
            assert ((out[layer, :n].double() - o).abs() <= o.abs() * 2.0 ** -8 + A * 2.0 ** -10).all()


def test_refusals():
    c = Case(128, 8, 2, [4], [64])
    rx, p, q, o = c.rx, c.caches[0], c.q[0], c.out[0]
    before = o.clone()
    big = torch.zeros((5, 8, 128), dtype=torch.bfloat16, device="cuda")
    for status, call in [
            ("CB_ESHAPE", lambda: rx.attend([p], [q], [o], layer=1)),
            ("CB_ESHAPE", lambda: rx.attend([p], [q], [o], layer=-1)),
            ("CB_ESHAPE", lambda: rx.attend([p], [big], [big.clone()])),
            ("CB_ESHAPE", lambda: rx.attend([p] * 2, [q] * 2, [o, o.clone()])),
            ("CB_ESHAPE", lambda: rx.attend([], [], [])),
            ("CB_EINVAL", lambda: rx.attend([p], [q], [o], window=-1)),
            ("CB_EINVAL", lambda: rx.attend([p], [q], [o], window=5, causal=False)),
            ("CB_EINVAL", lambda: rx.attend([p], [q.cpu()], [o])),
            ("CB_EINVAL", lambda: rx.attend([p], [q], [o.cpu()])),
            ("CB_EINVAL", lambda: rx.attend([p], [q], [o], lses=[c.lse[0].cpu()])),
            ("CB_EINVAL", lambda: rx.attend([p], [q], [o[:1].expand(4, 8, 128)])),
            ("CB_EINVAL", lambda: rx.attend([cb.PackedKV.empty(1, 2, 64, 128)], [q], [o])),
            ("CB_ESHAPE", lambda: rx.attend([cb.PackedKV.empty(1, 2, 200, 128, "cuda")], [q], [o]))]:
        with pytest.raises(cb.CBError, match=status):
            call()
    with pytest.raises(ValueError):
        rx.attend([cb.PackedKV.empty(1, 1, 64, 128, "cuda")], [q], [o])
    with pytest.raises(ValueError):
        rx.attend([p], [q[:, :4]], [o[:, :4]])
    rx.sync_status()
    assert torch.equal(o, before)


@pytest.mark.parametrize("d,Hq,Hkv", [(128, 4, 1), (64, 2, 2), (128, 16, 4)])
@pytest.mark.parametrize("m", [1, 4])
def test_items_of_many_parts(d, Hq, Hkv, m):
    """Long caches for few heads beside short ones: parts of one item are joined in groups, then the groups."""
    c = Case(d, Hq, Hkv, [m, m, 1, m], [30001, 300, 0, 12000], page=64)
    for _ in range(2):                           # (the second call finds the tickets as the first did)
        for o in c.out:
            o.fill_(7)
        c.run()
        c.check()
    c.run(window=5000)
    c.check(window=5000)


@pytest.mark.parametrize("m", [2, 40])
def test_two_contexts_at_once(m):
    """Each with its own stream and scratch, over the same caches."""
    a = Case(128, 8, 2, [m, m], [9000, 700])
    b = Case(128, 8, 2, [m, m], [9000, 700])
    a.run()
    a.check()
    want = [x.clone() for x in a.out]
    streams = [torch.cuda.Stream() for _ in range(2)]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    b.q, b.caches = a.q, a.caches
    for _ in range(20):
        a.run(stream=streams[0])
        b.run(stream=streams[1])
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) and torch.equal(x, z) for x, y, z in zip(want, a.out, b.out))
    a.rx.sync_status()
    b.rx.sync_status()


@pytest.mark.parametrize("m", [1, 70])
def test_captured_graphs_share_a_context(m):
    """Two captured calls of one context, of different shapes, replayed in turn on one stream."""
    a = Case(128, 8, 2, [m, 1], [5000, 33])
    b = Case(128, 8, 2, [m], [2222])
    b.rx = a.rx
    graphs = []
    for c in (a, b):
        c.run()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            c.run()
        graphs.append(g)
    for c in (a, b):
        for o in c.out:
            o.fill_(7)
    for _ in range(3):
        for g in graphs:
            g.replay()
    a.check()
    b.check()


def test_more_heads_than_blocks():
    """KV heads that outnumber the blocks an SM count allows: each takes its whole run."""
    for m in (1, 20):
        c = Case(64, 700, 700, [m], [200])
        c.run()
        c.check()


def test_lists_and_types_that_do_not_fit_are_refused():
    c = Case(128, 8, 2, [4], [64])
    for call in (lambda: c.rx.attend(c.caches, c.q * 2, c.out), lambda: c.rx.attend(c.caches, [c.q[0].half()], c.out),
                 lambda: c.rx.attend(c.caches, c.q, [c.out[0].half()]),
                 lambda: c.rx.attend(c.caches, c.q, c.out, lses=[c.lse[0].int()])):
        with pytest.raises(ValueError):
            call()


@pytest.mark.parametrize("m", [1, 3])
def test_sequences_in_one_tensor(m):
    """Queries, outputs and log-sum-exps with the sequences in their first dimension, in slices of wider tensors too."""
    c = Case(128, 8, 2, [m] * 3, [70, 5, 300])
    c.run()
    c.check()
    want = [x.clone() for x in c.out], [x.clone() for x in c.lse]
    for step in (1, 2):
        Q, out = (torch.zeros((3 * step, m, 10, 128), dtype=torch.bfloat16, device="cuda")[::step, :, 1:9] for _ in range(2))
        lse = torch.zeros((3 * step, m, 8), device="cuda")[::step]
        Q.copy_(torch.stack(c.q))
        c.rx.attend(c.caches, Q, out, lses=lse)
        c.rx.sync_status()
        assert torch.equal(out, torch.stack(want[0])) and torch.equal(lse, torch.stack(want[1]))
        out.zero_()
        c.rx.attend(c.caches, Q, out)
        assert torch.equal(out, torch.stack(want[0]))
    for bad in (lambda: c.rx.attend(c.caches, Q[:2], out[:2]), lambda: c.rx.attend(c.caches, Q.half(), out),
                lambda: c.rx.attend(c.caches, Q, out, lses=lse.transpose(0, 1)),
                lambda: c.rx.attend(c.caches, Q, out, lses=lse.double()),
                lambda: c.rx.attend(c.caches, Q[..., :64], out[..., :64])):
        with pytest.raises(ValueError):
            bad()
    one = Case(128, 8, 2, [m], [70])              # one query for all, by a stride of zero
    one.caches = one.caches * 3
    Q, out = one.q[0][None].expand(3, -1, -1, -1), torch.zeros((3, m, 8, 128), dtype=torch.bfloat16, device="cuda")
    one.rx = cb.Receiver(1, 8, 2, 128, m, 200, 3)
    one.rx.attend(one.caches, Q, out)
    one.run = None
    one.out = [out[2]]
    one.lse = [torch.zeros((m, 8), device="cuda")]
    one.rx.attend(one.caches[:1], one.q, [out[0]], lses=one.lse)
    one.check(which=[0])
    assert torch.equal(out[0], out[2]) and torch.equal(out[1], out[2])
