"""Eviction and kept rows on the GPU: which rows stay, and that what moves keeps every bit."""
import math

import pytest
import torch

import budget_reference as ref
import paper_2609_32046_gb300 as cb

pytestmark = pytest.mark.gpu


def bits(x):
    return x if x.dtype == torch.uint8 else x.view(torch.int16)


class Caches:
    """Caches whose bytes are random, their weights, and copies of both."""

    def __init__(self, d, Hkv, Ts, page=0, layers=2, seed=0, layout="heads", room=0, lengths=None, most=None):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.d, self.Hkv, self.layers = d, Hkv, layers
        self.rx = cb.Receiver(layers, Hkv, Hkv, d, 8, 64, len(Ts))
        byte = lambda *s: torch.randint(0, 256, s, generator=g, device="cuda", dtype=torch.uint8)     # noqa: E731
        half = lambda *s: byte(*s, 2).view(torch.bfloat16).squeeze(-1)                               # noqa: E731
        make = ((d // 2, byte), (d // 2, byte), (d // 32, half), (d // 32, half))
        self.caches, self.pool = [], None
        if page:
            need = [-(-(T + room) // page) for T in Ts]
            order = torch.randperm(sum(need) + 3, generator=torch.Generator().manual_seed(seed)).int()
            self.pool = [f(layers, sum(need) + 3, page, Hkv, w) for w, f in make]
        at = 0
        for i, T in enumerate(Ts):
            if page:
                p = cb.PackedKV(*self.pool, T=T, pages=order[at:at + need[i]].cuda())
                at += need[i]
            elif layout == "heads":
                p = cb.PackedKV(*[f(layers, Hkv, T + room, w) for w, f in make], T=T)
            else:
                p = cb.PackedKV(*[f(layers, T + room, Hkv, w).transpose(1, 2) for w, f in make], T=T)
            if lengths is not None:
                p.length = torch.tensor([lengths[i]], dtype=torch.int32, device="cuda")
            self.caches.append(p)
        self.weights = [torch.randn(layers, Hkv, T + room, generator=g, device="cuda").exp_() for T in Ts]
        self.Ts = Ts
        self.was = [self.rows(p) for p in self.caches]
        self.had = [w.clone() for w in self.weights]

    @staticmethod
    def rows(p):
        """All rows that a cache has room for, [layers][Hkv][capacity][..] of its four arrays, copied."""
        out = []
        for x in (p.k, p.v, p.k_scale, p.v_scale):
            x = bits(x)
            if p.pages is not None:
                x = x[:, p.pages.long()].flatten(1, 2).transpose(1, 2)
            out.append(x.clone())
        return out


def check_moved(c, i, at, first, now, weights_now, was=None, behind=True):
    """Rows `first` + j of every list are what rows at[l][g][j] were; the others are as before."""
    was = was or c.was[i]
    for l in range(c.layers):
        for g in range(c.Hkv):
            x = torch.tensor(at[l][g], dtype=torch.long, device="cuda")
            n = len(at[l][g])
            for a, b, o in zip(now, was, c.was[i]):
                assert torch.equal(a[l, g, first:first + n], o[l, g, x])
                if behind:
                    assert torch.equal(a[l, g, first + n:], b[l, g, first + n:]) and torch.equal(a[l, g, :first], b[l, g, :first])
            if weights_now is not None:
                assert torch.equal(weights_now[l, g, first:first + n], c.had[i][l, g, x])


def want(c, i, keep, first, last, L=None):
    w = c.had[i].cpu().tolist()
    return [[ref.kept_rows(w[l][g], c.Ts[i] if L is None else L, keep, first, last) for g in range(c.Hkv)] for l in range(c.layers)]


def check_idx(idx, at, keep):
    for x, y in zip(idx.cpu().tolist(), at):
        for a, b in zip(x, y):
            assert a == b + [-1] * (keep - len(b))


@pytest.mark.parametrize("d,Hkv", [(128, 2), (64, 3)])
@pytest.mark.parametrize("T,keep,first,last", [(1, 1, 0, 0), (2, 1, 0, 1), (5, 5, 1, 2), (33, 32, 0, 0), (100, 40, 3, 10), (300, 299, 1, 1),
                                               (700, 64, 4, 60), (700, 65, 0, 0), (1500, 700, 4, 33), (2100, 2000, 0, 1), (9000, 1000, 4, 64),
                                               (9001, 8999, 1, 2), (300, 41, 1, 40)])
@pytest.mark.parametrize("into", [False, True])
def test_one_cache(d, Hkv, T, keep, first, last, into):
    c = Caches(d, Hkv, [T], seed=T, room=5)
    to = None
    if into:
        o = Caches(d, Hkv, [keep], seed=T + 1, room=3)
        to, wto = o.caches, [torch.full((2, Hkv, keep + 2), -1.0, device="cuda")]
    idx = c.rx.evict(c.caches, c.weights, keep, first, last, into=to, weights_into=wto if into else None)
    c.rx.sync_status()
    at = want(c, 0, keep, first, last)
    check_idx(idx[0], at, keep)
    if into:
        assert all(torch.equal(a, b) for a, b in zip(c.rows(c.caches[0]), c.was[0])) and torch.equal(c.weights[0], c.had[0])
        check_moved(c, 0, at, 0, c.rows(to[0]), wto[0], was=o.was[0])
        assert (wto[0][:, :, keep:] == -1).all() and to[0].T == min(T, keep) and c.caches[0].T == T
    else:
        check_moved(c, 0, at, 0, c.rows(c.caches[0]), c.weights[0])
        assert torch.equal(c.weights[0][:, :, min(T, keep):], c.had[0][:, :, min(T, keep):]) and c.caches[0].T == min(T, keep)


@pytest.mark.parametrize("page", [0, 1, 16, 64])
@pytest.mark.parametrize("into", [False, True])
def test_ragged_batches_in_every_layout(page, into):
    """Lengths below, at and above the budget, a budget a cache, pages that end inside what is kept."""
    Ts, keep = [1, 40, 41, 100, 500, 1030], [7, 41, 41, 41, 17, 600]
    c = Caches(128, 2, Ts, page=page, layers=3, layout="positions")
    o = Caches(128, 2, keep, page=page, layers=3, seed=9) if into else None
    first, last = 2, 5
    idx = c.rx.evict(c.caches, c.weights, keep, first, last, into=o.caches if into else None)
    c.rx.sync_status()
    for i, T in enumerate(Ts):
        at = want(c, i, keep[i], first, last)
        check_idx(idx[i], at, keep[i])
        p = (o if into else c).caches[i]
        check_moved(c, i, at, 0, c.rows(p), None if into else c.weights[i], was=o.was[i] if into else None)
        assert p.T == min(T, keep[i])


@pytest.mark.parametrize("kind", ["equal", "zeros", "few values", "nan", "infinite", "negative", "tiny", "late", "close"])
@pytest.mark.parametrize("T,keep", [(600, 200), (20000, 3001), (9000, 8000)])
def test_weights_of_all_kinds(kind, T, keep):
    """Ties go to the lowest row; -0 is 0, NaN below every number; equal high bits; the heaviest last."""
    c = Caches(64, 1, [T], layers=2)
    g = torch.Generator(device="cuda").manual_seed(1)
    w = c.weights[0]
    r = torch.rand(w.shape, generator=g, device="cuda")
    if kind == "equal":
        w.fill_(0.25)
    elif kind == "zeros":
        w.copy_(torch.where(r < 0.5, torch.zeros_like(w), -torch.zeros_like(w)))
        w[..., 50:60] = 1e-38
    elif kind == "few values":
        w.copy_((r * 4).floor())
    elif kind == "nan":
        w[r < 0.9] = float("nan")
        w[..., 70:90] = -math.inf
    elif kind == "infinite":
        w[r < 0.7] = math.inf
        w[r > 0.9] = -math.inf
    elif kind == "negative":
        w.neg_()
    elif kind == "tiny":
        w.copy_(r * 1e-40)
    elif kind == "late":
        w.copy_(torch.arange(T, device="cuda").float().expand_as(w))
    else:
        w.copy_((torch.full_like(w, 1.0).view(torch.int32) + (r * 100).int()).view(torch.float32))
    c.had = [w.clone()]
    idx = c.rx.evict(c.caches, c.weights, keep, 3, 20)
    c.rx.sync_status()
    at = want(c, 0, keep, 3, 20)
    check_idx(idx[0], at, keep)
    check = [x.view(torch.int32) for x in (c.weights[0], c.had[0])]
    for l in range(2):
        assert torch.equal(check[0][l, 0, :keep], check[1][l, 0, torch.tensor(at[l][0], device="cuda")])


def test_many_lists_of_many_caches():
    """More caches than a launch of either kernel takes, more lists than SMs, in place and not."""
    n = 70
    Ts = [1 + 7 * i for i in range(n)]
    for into in (False, True):
        c = Caches(64, 3, Ts, layers=2)
        o = Caches(64, 3, [100] * n, layers=2, seed=1) if into else None
        idx = c.rx.evict(c.caches, c.weights, 100, 2, 5, into=o.caches if into else None)
        c.rx.sync_status()
        for i in (0, 13, 14, 31, 32, 63, 64, 69):
            at = want(c, i, 100, 2, 5)
            check_idx(idx[i], at, 100)
            check_moved(c, i, at, 0, c.rows((o if into else c).caches[i]), None if into else c.weights[i], was=o.was[i] if into else None)
    c = Caches(64, 3, [300] * n, layers=2)
    path = torch.arange(1, 40, 3, dtype=torch.int32, device="cuda")
    c.rx.keep(c.caches, [path] * n, 40, weights=c.weights)
    c.rx.sync_status()
    for i in (0, 31, 32, 69):
        check_moved(c, i, [[[260 + x for x in path.tolist()]] * 3] * 2, 260, c.rows(c.caches[i]), c.weights[i])


def test_in_place_and_into_others_in_one_call():
    """One tensor of weights to move into, of which a cache that is held in place takes none."""
    c, o = Caches(128, 2, [200, 300, 250]), Caches(128, 2, [90, 90, 90], seed=4)
    weights = torch.zeros(3, 2, 2, 300, device="cuda")
    for i, w in enumerate(c.weights):
        weights[i, :, :, :w.shape[2]] = w
    had = weights.clone()
    to, into = torch.full((3, 2, 2, 90), -1.0, device="cuda"), [o.caches[0], c.caches[1], o.caches[2]]
    idx = torch.zeros(3, 2, 2, 90, dtype=torch.int32, device="cuda")
    c.rx.evict(c.caches, weights, 90, 1, 9, into=into, weights_into=to, idx=idx)
    c.rx.sync_status()
    for i in range(3):
        at = want(c, i, 90, 1, 9)
        check_idx(idx[i], at, 90)
        check_moved(c, i, at, 0, c.rows(into[i]), weights[i] if i == 1 else to[i], was=None if i == 1 else o.was[i])
    assert (to[1] == -1).all() and torch.equal(weights[::2], had[::2])
    assert [p.T for p in c.caches] == [200, 90, 250]


def test_on_another_stream():
    """Work queued behind other work of the stream that is given, not of the current one."""
    c = Caches(128, 2, [3000])
    stream = torch.cuda.Stream()
    w = c.weights[0]
    late = w.flip(-1).contiguous()
    c.had = [late.clone()]
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        torch.cuda._sleep(20_000_000)
        w.copy_(late)
    c.rx.evict(c.caches, c.weights, 500, 1, 9, stream=stream)
    stream.synchronize()
    c.rx.sync_status(stream)
    check_moved(c, 0, want(c, 0, 500, 1, 9), 0, c.rows(c.caches[0]), c.weights[0])


def test_a_long_list():
    """More keys than the blocks of a cluster hold in shared memory, few and many rows kept."""
    T = 8 * 24 * 1024 + 5000
    for keep in (100, T - 7):
        c = Caches(64, 1, [T], layers=1)
        idx = c.rx.evict(c.caches, c.weights, keep, 1, 40)
        c.rx.sync_status()
        w = c.had[0][0, 0]
        inner = torch.sort(w[1:T - 40], descending=True, stable=True).indices[:keep - 41] + 1
        at = torch.cat([torch.zeros(1, dtype=torch.long, device="cuda"), inner.sort().values, torch.arange(T - 40, T, device="cuda")])
        assert torch.equal(idx[0][0, 0].long(), at)
        for a, b in zip(c.rows(c.caches[0]), c.was[0]):
            assert torch.equal(a[0, 0, :keep], b[0, 0, at])


def test_some_layers_and_lengths_of_their_own():
    c = Caches(128, 2, [500], layers=4)
    w = c.weights[0][1:3]
    left = torch.zeros(1, dtype=torch.int32, device="cuda")
    idx = c.rx.evict(c.caches, [w], 100, 1, 9, layer=1, lengths=[left])
    c.rx.sync_status()
    assert int(left) == 100 and c.caches[0].T == 500 and tuple(idx[0].shape) == (2, 2, 100)
    now = c.rows(c.caches[0])
    at = want(c, 0, 100, 1, 9)
    check_idx(idx[0], at[1:3], 100)
    for l in range(4):
        for g in range(2):
            for a, b in zip(now, c.was[0]):
                x = torch.tensor(at[l][g], device="cuda") if l in (1, 2) else torch.arange(100, device="cuda")
                assert torch.equal(a[l, g, :100], b[l, g, x]) and torch.equal(a[l, g, 100:], b[l, g, 100:])


@pytest.mark.parametrize("keep", [50, 300])
def test_lengths_on_the_device(keep):
    """A captured eviction follows lengths, and writes them, its own or one that two caches read."""
    Ts, lengths = [600, 600, 600, 600], [600, 51, 0, 5000]
    c = Caches(128, 2, Ts, page=16, lengths=lengths)
    graph = torch.cuda.CUDAGraph()
    c.rx.evict(c.caches, c.weights, keep, 2, 30)
    idx = [torch.zeros(2, 2, keep, dtype=torch.int32, device="cuda") for _ in Ts]
    with torch.cuda.graph(graph):
        c.rx.evict(c.caches, c.weights, keep, 2, 30, idx=idx)
    for grown in ([600, 301, 300, 49], [-5, 599, 50, 51]):
        c.was, c.had = [c.rows(p) for p in c.caches], [w.clone() for w in c.weights]
        for p, x in zip(c.caches, grown):
            p.length.fill_(x)
        graph.replay()
        c.rx.sync_status()
        for i, x in enumerate(grown):
            L = max(0, min(x, 600))
            at = want(c, i, keep, 2, 30, L)
            check_idx(idx[i], at, keep)
            check_moved(c, i, at, 0, c.rows(c.caches[i]), c.weights[i])
            assert int(c.caches[i].length) == min(L, keep) and c.caches[i].T == 600


def test_a_length_that_all_read():
    c = Caches(128, 2, [400] * 40, layers=1)
    shared = torch.tensor([390], dtype=torch.int32, device="cuda")
    for p in c.caches:
        p.length = shared
    left = [torch.zeros(1, dtype=torch.int32, device="cuda") for _ in c.caches]
    with pytest.raises(cb.CBError):
        c.rx.evict(c.caches, c.weights, 100)                # every one of them would write it
    with pytest.raises(cb.CBError):
        c.rx.evict(c.caches, c.weights, 100, lengths=[shared] + left[1:])
    assert int(shared) == 390 and all(torch.equal(a, b) for p, w in zip(c.caches, c.was) for a, b in zip(c.rows(p), w))
    c.rx.evict(c.caches, c.weights, 100, lengths=left)
    c.rx.sync_status()
    assert [int(x) for x in left] == [100] * 40
    for i in (0, 31, 32, 39):
        check_moved(c, i, want(c, i, 100, 0, 0, 390), 0, c.rows(c.caches[i]), c.weights[i])


def test_bad_pages_leave_their_rows_out():
    c = Caches(128, 2, [200], page=16, room=0)
    p = c.caches[0]
    table = p.pages.clone()
    p.pages[3] = -1
    p.pages[7] = p.n_pages
    c.rx.evict(c.caches, c.weights, 100, 2, 10, idx=None)
    with pytest.raises(cb.CBError) as e:
        c.rx.sync_status()
    assert e.value.status == cb.CB_EDEVICE
    p.pages.copy_(table)
    now = c.rows(p)
    at = want(c, 0, 100, 2, 10)
    for l in range(2):
        for g in range(2):
            for j, t in enumerate(at[l][g]):
                out = t // 16 in (3, 7) or j // 16 in (3, 7)
                for a, b in zip(now, c.was[0]):
                    assert torch.equal(a[l, g, j], b[l, g, j if out else t])


def test_evict_refusals():
    c = Caches(128, 2, [100, 100])
    o = Caches(128, 2, [20, 20])
    w = c.weights
    call = lambda **kw: c.rx.evict(**{**dict(caches=c.caches, weights=w, keep=50), **kw})         # noqa: E731
    for kw in (dict(weights=w[:1]), dict(weights=[w[0].half(), w[1]]), dict(weights=[w[0][:, :1], w[1]]), dict(weights=[w[0][..., :99], w[1]]),
               dict(keep=[50]), dict(idx=[torch.zeros(2, 2, 49, dtype=torch.int32, device="cuda")] * 2),
               dict(weights_into=w), dict(lengths=[None])):
        with pytest.raises(ValueError):
            call(**kw)
    i = torch.zeros(2, 2, 50, dtype=torch.int32, device="cuda")
    for kw in (dict(first=30, last=21), dict(first=-1), dict(last=-1), dict(keep=-1), dict(layer=1), dict(into=o.caches),
               dict(caches=[c.caches[0]] * 2), dict(idx=[i, i]), dict(keep=20, caches=[c.caches[0]] * 2, into=[c.caches[0], o.caches[0]]),
               dict(keep=20, into=[o.caches[0], c.caches[0]]), dict(keep=20, into=[o.caches[0]] * 2),
               dict(keep=20, into=o.caches, weights_into=w), dict(weights=[w[0], w[0]]),
               dict(weights=[w[0].cpu(), w[1]]), dict(weights=[w[0].as_strided((2, 2, 100), (10, 100, 1)), w[1]])):
        if kw.get("keep") == -1:
            kw["idx"] = [i, i.clone()]
            with pytest.raises(ValueError):
                call(**kw)
            continue
        with pytest.raises(cb.CBError):
            call(**kw)
    with pytest.raises(cb.CBError):
        cb.Receiver(2, 2, 2, 128, 8, 64, 1).evict(c.caches, w, 50)
    c.rx.sync_status()
    assert all(torch.equal(a, b) for p, x in zip(c.caches, c.was) for a, b in zip(c.rows(p), x))
    assert all(torch.equal(a, b) for a, b in zip(w, c.had)) and [p.T for p in c.caches] == [100, 100]


@pytest.mark.parametrize("d,Hkv", [(128, 2), (64, 3)])
@pytest.mark.parametrize("m,path", [(1, [0]), (2, [1]), (8, [0, 1, 2]), (8, [3, 5, 7]), (64, [2, 9, 31, 32, 63]), (300, list(range(0, 300, 3))),
                                    (300, list(range(1, 300))), (700, list(range(100, 700))), (5, [])])
@pytest.mark.parametrize("page", [0, 16])
def test_kept_rows(d, Hkv, m, path, page):
    c = Caches(d, Hkv, [m + 40], page=page, room=3)
    idx = torch.tensor(path, dtype=torch.int32, device="cuda")
    c.rx.keep(c.caches, [idx], m, weights=c.weights)
    c.rx.sync_status()
    check_moved(c, 0, [[[40 + x for x in path]] * Hkv] * 2, 40, c.rows(c.caches[0]), c.weights[0])
    assert c.caches[0].T == 40 + len(path)
    n = 40 + len(path)
    assert torch.equal(c.weights[0][..., n:], c.had[0][..., n:]) and torch.equal(c.weights[0][..., :40], c.had[0][..., :40])


@pytest.mark.parametrize("page", [0, 16])
def test_kept_rows_of_a_batch_and_in_a_graph(page):
    """Counts and lengths on the device, below, at and above what is given; without weights, all the rows of a cache."""
    n, m = 6, 20
    Ts = [m + 10 * i for i in range(n)]
    c = Caches(128, 2, Ts, page=page, lengths=Ts)
    path = torch.stack([torch.randperm(m, generator=torch.Generator().manual_seed(i))[:5].sort().values for i in range(n)]).int().cuda()
    counts = torch.tensor([0, 1, 3, 5, 9, -2], dtype=torch.int32, device="cuda")
    graph = torch.cuda.CUDAGraph()
    snapshot = [[x.clone() for x in (p.k, p.v, p.k_scale, p.v_scale)] for p in c.caches]
    c.rx.keep(c.caches, path, m, counts=list(counts.split(1)), weights=None)
    with torch.cuda.graph(graph):
        c.rx.keep(c.caches, path, m, counts=list(counts.split(1)), weights=None)
    for p, s, T in zip(c.caches, snapshot, Ts):
        for a, b in zip((p.k, p.v, p.k_scale, p.v_scale), s):
            bits(a).copy_(bits(b))
        p.length.fill_(T)
    graph.replay()
    c.rx.sync_status()
    for i, x in enumerate([0, 1, 3, 5, 5, 0]):
        at = [Ts[i] - m + y for y in path[i, :x].tolist()]
        check_moved(c, i, [[at] * 2] * 2, Ts[i] - m, c.rows(c.caches[i]), None)
        assert int(c.caches[i].length) == Ts[i] - m + x


def test_rows_that_may_not_be_kept():
    """Entries before their place or behind the drafts skip their rows; a cache of fewer rows than drafts stays as it is."""
    c = Caches(128, 2, [50, 50], lengths=[50, 9])
    idx = torch.tensor([0, 0, 5, -1, 10, 5, 9], dtype=torch.int32, device="cuda")
    c.rx.keep(c.caches, [idx, idx], 10)
    with pytest.raises(cb.CBError) as e:
        c.rx.sync_status()
    assert e.value.status == cb.CB_EDEVICE
    at = [40, 41, 45, 43, 44, 45, 49]
    check_moved(c, 0, [[at] * 2] * 2, 40, c.rows(c.caches[0]), None)
    assert int(c.caches[0].length) == 47 and int(c.caches[1].length) == 9
    assert all(torch.equal(a, b) for a, b in zip(c.rows(c.caches[1]), c.was[1]))


def test_keep_refusals():
    c = Caches(128, 2, [100, 100])
    i = torch.zeros(5, dtype=torch.int32, device="cuda")
    n = torch.zeros(1, dtype=torch.int32, device="cuda")
    call = lambda **kw: c.rx.keep(**{**dict(caches=c.caches, idx=[i, i], drafted=10), **kw})         # noqa: E731
    for kw in (dict(idx=[i]), dict(idx=[i.long(), i]), dict(idx=[i[::2], i]), dict(drafted=[10]), dict(counts=[n, n]),
               dict(weights=[c.weights[0][..., :99], c.weights[1]]), dict(weights=[c.weights[0].half(), c.weights[1]])):
        with pytest.raises(ValueError):
            call(**kw)
    for kw in (dict(drafted=4), dict(drafted=101), dict(drafted=-1), dict(caches=[c.caches[0]] * 2), dict(idx=[i.cpu(), i]),
               dict(lengths=[n, n]), dict(weights=[c.weights[0], c.weights[0]]), dict(counts=[n, n], lengths=[n, n.clone()])):
        with pytest.raises(cb.CBError):
            call(**kw)
    c.rx.sync_status()
    assert all(torch.equal(a, b) for p, x in zip(c.caches, c.was) for a, b in zip(c.rows(p), x)) and [p.T for p in c.caches] == [100, 100]
