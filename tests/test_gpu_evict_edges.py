"""Eviction and kept rows on the GPU: streams, empty caches, what two entries share, lists at the edges of the ranking's forms."""
import pytest
import torch

import paper_2609_32046_gb300 as cb
from test_gpu_evict import Caches, check_idx, check_moved, want

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("by_handle", [False, True])
def test_idx_is_memory_of_the_stream(by_handle):
    """The result dropped, the current stream's next tensors of its size are written while the call's stream still ranks and
    moves: they are other memory, and the rows are right."""
    c = Caches(128, 2, [3000])
    stream = torch.cuda.Stream()
    given = stream.cuda_stream if by_handle else stream
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        torch.cuda._sleep(20_000_000)
    idx = c.rx.evict(c.caches, c.weights, 500, 1, 9, stream=given)
    at = idx[0].data_ptr()
    del idx
    others = [torch.full((2, 2, 500), 2999, dtype=torch.int32, device="cuda") for _ in range(3)]
    assert at not in [x.data_ptr() for x in others]
    stream.synchronize()
    c.rx.sync_status(given)
    torch.cuda.synchronize()
    check_moved(c, 0, want(c, 0, 500, 1, 9), 0, c.rows(c.caches[0]), c.weights[0])


def test_a_stream_by_the_handle_0():
    """The default stream given by its handle while another is current."""
    c = Caches(64, 1, [300])
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        idx = c.rx.evict(c.caches, c.weights, 100, stream=0)
    c.rx.sync_status(0)
    check_idx(idx[0], want(c, 0, 100, 0, 0), 100)


@pytest.mark.parametrize("into", [False, True])
@pytest.mark.parametrize("Ts", [[0], [0, 90, 0], [50, 0, 200, 0]])
def test_empty_caches(Ts, into):
    """A cache without rows is described by T = 0 as by a length of 0: -1 for every row that stays."""
    keep = 60
    c = Caches(128, 2, Ts, room=70)
    o = Caches(128, 2, [keep] * len(Ts), seed=3) if into else None
    idx = [torch.full((2, 2, keep), 7, dtype=torch.int32, device="cuda") for _ in Ts]
    left = [torch.full((1,), 9, dtype=torch.int32, device="cuda") for _ in Ts]
    c.rx.evict(c.caches, c.weights, keep, 2, 5, into=o.caches if into else None, idx=idx, lengths=left)
    c.rx.sync_status()
    for i, T in enumerate(Ts):
        at = want(c, i, keep, 2, 5)
        check_idx(idx[i], at, keep)
        check_moved(c, i, at, 0, c.rows((o if into else c).caches[i]), None if into else c.weights[i], was=o.was[i] if into else None)
        assert int(left[i]) == min(T, keep)
    if Ts[0] == 0:
        assert torch.equal(c.rx.evict(c.caches[:1], c.weights[:1], keep)[0], torch.full((2, 2, keep), -1, dtype=torch.int32, device="cuda"))
        with pytest.raises(cb.CBError):
            c.rx.evict(c.caches[:1], c.weights[:1], keep, idx=[idx[0].cpu()])


def test_weights_that_two_entries_share():
    """Entries whose weights move to where another's are taken from are refused, in place and into other caches; weights that
    two only read are not."""
    c, o = Caches(128, 2, [100, 100, 100]), Caches(128, 2, [20, 20, 20], seed=2)
    w = c.weights
    spare = [torch.zeros(2, 2, 20, device="cuda") for _ in w]
    wide = torch.zeros(2, 2, 100, device="cuda")
    both = torch.rand(500, device="cuda")
    for weights, to, into in (([w[0], w[1]], [w[1], w[0]], None), ([w[0], w[1]], [wide, w[0]], None), ([w[0], w[0]], [w[0], spare[0]], True),
                              ([both[:400].view(2, 2, 100), w[1]], [spare[0], both[390:470].view(2, 2, 20)], None)):
        caches = o.caches[:2] if into is None else [c.caches[0], o.caches[1]]
        with pytest.raises(cb.CBError):
            c.rx.evict(c.caches[:2], weights, 20, into=caches, weights_into=to)
    c.rx.sync_status()
    assert all(torch.equal(a, b) for p, x in zip(c.caches, c.was) for a, b in zip(c.rows(p), x)) and [p.T for p in c.caches] == [100] * 3
    c.had = [w[0].clone() for _ in w]
    idx = c.rx.evict(c.caches, [w[0]] * 3, 20, 1, 2, into=o.caches, weights_into=spare)
    c.rx.sync_status()
    for i in range(3):
        at = want(c, i, 20, 1, 2)
        check_idx(idx[i], at, 20)
        check_moved(c, i, at, 0, c.rows(o.caches[i]), spare[i], was=o.was[i])
    # weights that are ranked by and stay where they are may be what another entry writes: all are ranked first
    c, o = Caches(128, 2, [100, 100], seed=5), Caches(128, 2, [20, 20], seed=2)
    c.had[1] = c.had[0]
    into = [c.caches[0], o.caches[1]]
    idx = c.rx.evict(c.caches, [c.weights[0]] * 2, 20, 1, 2, into=into)
    c.rx.sync_status()
    for i in range(2):
        at = want(c, i, 20, 1, 2)
        check_idx(idx[i], at, 20)
        check_moved(c, i, at, 0, c.rows(into[i]), c.weights[0] if i == 0 else None, was=None if i == 0 else o.was[1])


@pytest.mark.parametrize("T", [24572, 24573, 24576, 24577, 49145, 49152, 49153, 98304])
@pytest.mark.parametrize("lists", [1, 160])
def test_lists_that_just_fit(T, lists):
    """Keys up to the last one that a block's, or a cluster's, shared memory holds, and one more."""
    layers, keep, first, last = (1, 700, 0, 0) if lists == 1 else (20, 90, 3, 10)
    Hkv = lists // layers
    g = torch.Generator(device="cuda").manual_seed(T)
    codes = [torch.randint(0, 256, (layers, Hkv, T, 32), generator=g, device="cuda", dtype=torch.uint8) for _ in range(2)]
    scales = [torch.rand((layers, Hkv, T, 2), generator=g, device="cuda").to(torch.bfloat16) for _ in range(2)]
    into = [torch.zeros(layers, Hkv, keep, x.shape[-1], dtype=x.dtype, device="cuda") for x in codes + scales]
    w = torch.randn((layers, Hkv, T), generator=g, device="cuda").exp_()
    w[..., 100::3] = 1.0                                                    # many ties, past the last rows too
    rx = cb.Receiver(layers, Hkv, Hkv, 64, 8, 64, 1)
    idx = rx.evict([cb.PackedKV(*codes, *scales)], [w], keep, first, last, into=[cb.PackedKV(*into)])
    rx.sync_status()
    inner = torch.sort(w[..., first:T - last], dim=-1, descending=True, stable=True).indices[..., :keep - first - last] + first
    ends = [torch.arange(a, b, device="cuda").expand(layers, Hkv, -1) for a, b in ((0, first), (T - last, T))]
    at = torch.cat([ends[0], inner.sort(-1).values, ends[1]], -1)
    assert torch.equal(idx[0].long(), at)
    for a, b in zip(into, codes + scales):
        assert torch.equal(a.view(torch.uint8), b.gather(2, at[..., None].expand(-1, -1, -1, b.shape[-1])).view(torch.uint8))


@pytest.mark.parametrize("count", [0, 1])
@pytest.mark.parametrize("own", [False, True])
@pytest.mark.parametrize("others", [0, 40])
def test_fewer_rows_than_drafts(count, own, others):
    """A cache of fewer rows than were drafted is reported whether any of them are kept or none, and stays as it is, with its length."""
    n = 1 + others
    c = Caches(64, 2, [60] * n, lengths=[3] + [50] * others, layers=1)
    path = torch.arange(1, 1 + count, dtype=torch.int32, device="cuda")
    left = None if own else [torch.full((1,), 99, dtype=torch.int32, device="cuda") for _ in range(n)]
    c.rx.keep(c.caches, [path] * n, 5, weights=c.weights, lengths=left)
    with pytest.raises(cb.CBError) as e:
        c.rx.sync_status()
    assert e.value.status == cb.CB_EDEVICE
    now = [int(p.length) if own else int(x) for p, x in zip(c.caches, left or c.caches)]
    assert now == [3 if own else 99] + [45 + count] * others
    for i in range(n):
        check_moved(c, i, [[[46] * count if i else []] * 2], 45, c.rows(c.caches[i]), c.weights[i])


def test_all_drafts_of_enough_rows_left_out():
    """No error, and lengths without the drafts: host's, own and others'."""
    c = Caches(64, 2, [60, 60], lengths=[5, 60], layers=1)
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    c.rx.keep(c.caches, [none, none], 5)
    c.rx.sync_status()
    assert [int(p.length) for p in c.caches] == [0, 55]
    c = Caches(64, 2, [60, 60], layers=1)
    c.rx.keep(c.caches, [none, none], [5, 60])
    c.rx.sync_status()
    assert [p.T for p in c.caches] == [55, 0]


@pytest.mark.parametrize("kind", ["equal", "few values", "nan", "late", "first", "close"])
@pytest.mark.parametrize("T,keep", [(30000, 3001), (50000, 45000), (120000, 700)])
def test_long_lists_of_all_kinds(kind, T, keep):
    """Clusters of two, four and eight blocks: ties across the blocks' slices, all that stays in one of them."""
    layers, first, last = 2, 3, 20
    g = torch.Generator(device="cuda").manual_seed(T)
    w = torch.rand((layers, 1, T), generator=g, device="cuda")
    if kind == "equal":
        w.fill_(0.25)
    elif kind == "few values":
        w.mul_(4).floor_()
    elif kind == "nan":
        w[w < 0.95] = float("nan")
    elif kind == "late":
        w.copy_(torch.arange(T, device="cuda").float())
    elif kind == "first":
        w.copy_(-torch.arange(T, device="cuda").float())
    else:
        w.copy_((torch.full_like(w, 1.0).view(torch.int32) + (w * 100).int()).view(torch.float32))
    codes = [torch.randint(0, 256, (layers, 1, T, 32), generator=g, device="cuda", dtype=torch.uint8) for _ in range(2)]
    scales = [torch.rand((layers, 1, T, 2), generator=g, device="cuda").to(torch.bfloat16) for _ in range(2)]
    had, was = w.clone(), [x.clone() for x in codes + scales]
    rx = cb.Receiver(layers, 1, 1, 64, 8, 64, 1)
    idx = rx.evict([cb.PackedKV(*codes, *scales)], [w], keep, first, last)
    rx.sync_status()
    key = torch.nan_to_num(had[..., first:T - last].double(), nan=-1e300)
    inner = torch.sort(key, dim=-1, descending=True, stable=True).indices[..., :keep - first - last] + first
    ends = [torch.arange(a, b, device="cuda").expand(layers, 1, -1) for a, b in ((0, first), (T - last, T))]
    at = torch.cat([ends[0], inner.sort(-1).values, ends[1]], -1)
    assert torch.equal(idx[0].long(), at)
    assert torch.equal(w[..., :keep].view(torch.int32), had.gather(-1, at).view(torch.int32)) and \
        torch.equal(w[..., keep:].view(torch.int32), had[..., keep:].view(torch.int32))
    for a, b in zip(codes + scales, was):
        assert torch.equal(a[:, :, :keep].view(torch.uint8), b.gather(2, at[..., None].expand(-1, -1, -1, b.shape[-1])).view(torch.uint8))


@pytest.mark.parametrize("layers,n", [(2, 1), (20, 12), (36, 2)])
@pytest.mark.parametrize("m", [64, 65, 128, 129, 400])
def test_kept_rows_of_few_and_many_lists(layers, n, m):
    """Rows moved by a warp, a block and the blocks of a cluster, by the number of lists and of rows."""
    c = Caches(64, 8, [m + 20] * n, layers=layers)
    path = torch.arange(m // 7, m, dtype=torch.int32, device="cuda")
    c.rx.keep(c.caches, [path] * n, m, weights=c.weights)
    c.rx.sync_status()
    x = torch.arange(20 + m // 7, 20 + m, device="cuda")
    for i in range(n):
        for a, b in zip(c.rows(c.caches[i]), c.was[i]):
            assert torch.equal(a[:, :, 20:20 + len(x)], b[:, :, x]) and torch.equal(a[:, :, 20 + len(x):], b[:, :, 20 + len(x):])
            assert torch.equal(a[:, :, :20], b[:, :, :20])
        assert torch.equal(c.weights[i][:, :, 20:20 + len(x)], c.had[i][:, :, x])
