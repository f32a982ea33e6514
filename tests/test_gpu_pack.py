"""Rows held in 4 bits on the GPU: packing (bit for bit against the definition) and restoring."""
import pytest
import torch

import paper_2609_32046_gb300 as cb
import packed_reference as ref

pytestmark = pytest.mark.gpu


def _rows(shape, seed, wild=False):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(shape, generator=g)
    if wild:       # groups of every magnitude: beyond both ends of the scales' range too
        x = x * torch.exp2(torch.randint(-30, 17, shape[:-1] + (shape[-1] // 32, 1), generator=g).float()).expand(
            shape[:-1] + (shape[-1] // 32, 32)).reshape(shape)
        x = x.clamp(-50000, 50000)
    return x.to(torch.bfloat16)


def _receiver(nL, Hkv, d, T, n=1):
    return cb.Receiver(nL, Hkv, Hkv, d, 1, T, n)


def _check(held, at, x, s, name):
    """Rows `at` of the packed arrays against the definition of the bf16 rows x [nL][Hkv][rows][d]."""
    c, sc = ref.held_rows(x)
    codes = ref.packed_bytes(c)
    assert torch.equal(held[:, :, at].cpu(), codes), name
    assert torch.equal(s[:, :, at].cpu().double(), sc), name


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("nL,Hkv,T", [(1, 1, 1), (2, 2, 37), (3, 4, 130), (1, 8, 515)])
def test_every_row_is_the_definitions(nL, Hkv, T, d):
    K, V = (_rows((nL, Hkv, T, d), s, wild=True) for s in (1, 2))
    rx = _receiver(nL, Hkv, d, T)
    p = cb.PackedKV.empty(nL, Hkv, T, d, "cuda")
    rx.pack([K.cuda()], [V.cuda()], [p], [0])
    rx.sync_status()
    at = torch.arange(T)
    _check(p.k, at, K, p.k_scale, "K")
    _check(p.v, at, V, p.v_scale, "V")
    ko, vo = torch.empty_like(K, device="cuda"), torch.empty_like(V, device="cuda")
    rx.unpack([p], ko, vo)
    rx.sync_status()
    # every value is a bf16 number: restored exactly
    assert torch.equal(ko.double(), ref.values(p.k, p.k_scale)) and torch.equal(vo.double(), ref.values(p.v, p.v_scale))


def test_every_quotient_rounds_as_defined():
    """Every bf16 mantissa against every scale of one octave: halves away from zero, all signs."""
    tops = torch.arange(128, 256).float()                        # one octave of largest values, 8 bits each
    rows = []
    for t in tops.tolist():
        x = torch.linspace(-t, t, 31).to(torch.bfloat16).tolist()
        rows += x[:31] + [t]
        s = ref.scale_of(t)
        half = [torch.tensor((k + 0.5) * s * sg).to(torch.bfloat16).item() for k in range(7) for sg in (1, -1)]
        rows += (half + [0.0] * 32)[:31] + [t]
    x = torch.tensor(rows).to(torch.bfloat16).reshape(1, 1, -1, 64)
    rx = _receiver(1, 1, 64, x.shape[2])
    p = cb.PackedKV.empty(1, 1, x.shape[2], 64, "cuda")
    rx.pack([x.cuda()], [x.cuda()], [p], [0])
    rx.sync_status()
    _check(p.k, torch.arange(x.shape[2]), x, p.k_scale, "K")


@pytest.mark.parametrize("d", [64, 128])
def test_selected_rows_of_ragged_senders_into_one_message(d):
    nL, Hkv, Ts = 2, 2, [300, 65, 517]
    g = torch.Generator().manual_seed(3)
    senders = [(_rows((nL, Hkv, T, d), i), _rows((nL, Hkv, T, d), 10 + i)) for i, T in enumerate(Ts)]
    idx = [torch.sort(torch.randperm(T, generator=g)[:T // 3]).values.int() for T in Ts]
    off = [5, 5 + len(idx[0]), 5 + len(idx[0]) + len(idx[1])]
    total = off[2] + len(idx[2]) + 4
    rx = _receiver(nL, Hkv, d, max(Ts + [total]), 3)
    p = cb.PackedKV(*[torch.full((nL, Hkv, total, w), 77, dtype=t, device="cuda")
                      for w, t in ((d // 2, torch.uint8),) * 2 + ((d // 32, torch.bfloat16),) * 2])
    dev = [(k.cuda(), v.cuda()) for k, v in senders]
    rx.pack([k for k, _ in dev], [v for _, v in dev], [p] * 3, off, idx=[i.cuda() for i in idx])
    rx.sync_status()
    for (K, V), i, o in zip(senders, idx, off):
        at = torch.arange(o, o + len(i))
        _check(p.k, at, K[:, :, i.long()], p.k_scale, "K")
        _check(p.v, at, V[:, :, i.long()], p.v_scale, "V")
    for edge in (slice(0, 5), slice(total - 4, total)):            # rows around the message are as they were
        assert (p.k[:, :, edge] == 77).all() and (p.v_scale[:, :, edge] == 77).all()
    # some rows back, in another order and twice
    some = torch.tensor([off[1], off[0], off[0], total - 5], dtype=torch.int32, device="cuda")
    ko = torch.zeros((nL, Hkv, 6, d), dtype=torch.bfloat16, device="cuda")
    vo = torch.zeros_like(ko)
    rx.unpack([p], ko, vo, [1], idx=[some])
    rx.sync_status()
    assert torch.equal(ko[:, :, 1:5].double(), ref.values(p.k, p.k_scale)[:, :, some.long()])
    assert (ko[:, :, 0] == 0).all() and (vo[:, :, 5] == 0).all()


@pytest.mark.parametrize("page,d", [(1, 128), (16, 64), (16, 128), (64, 64)])
def test_pages_strides_and_layers(page, d):
    """A paged cache gets one layer's new rows at scattered positions from a position-major tensor."""
    nL, Hkv, T, m = 3, 2, 200, 23
    g = torch.Generator().manual_seed(page)
    n = -(-T // page)
    table = torch.randperm(n + 3, generator=g)[:n].int()
    K, V = (_rows((1, m, Hkv, d), s).cuda().transpose(1, 2) for s in (1, 2))       # [1][Hkv][m][d], position-major
    arrays = [torch.full((nL, n + 3, page, Hkv, w), 3, dtype=t, device="cuda")
              for w, t in ((d // 2, torch.uint8),) * 2 + ((d // 32, torch.bfloat16),) * 2]
    p = cb.PackedKV(*arrays, T=T, pages=table.cuda())
    rows = torch.randperm(T, generator=g)[:m].int()
    rx = _receiver(nL, Hkv, d, T)
    rx.pack([K], [V], [p], rows=[rows.cuda()], layer=1)
    rx.sync_status()
    k, ks = arrays[0], arrays[2]
    at = (table[(rows // page).long()].long(), (rows % page).long())
    c, s = ref.held_rows(K[0].cpu())
    assert torch.equal(k[1].cpu()[at], ref.packed_bytes(c).transpose(0, 1))
    assert torch.equal(ks[1].cpu()[at].double(), s.transpose(0, 1))
    untouched = torch.ones(k.shape[1:3], dtype=torch.bool)
    untouched[at] = False
    assert (k[1].cpu()[untouched] == 3).all() and (k[0] == 3).all() and (k[2] == 3).all()
    # from a paged bf16 cache into a strided one
    pool = torch.zeros((1, n + 3, page, Hkv, d), dtype=torch.bfloat16, device="cuda")
    src = _rows((1, Hkv, n * page, d), 9)
    pool[0, table.long().cuda()] = src[0].transpose(0, 1).reshape(n, page, Hkv, d).cuda()
    paged = cb.PagedKV(pool, pool, table.cuda(), T)
    q = cb.PackedKV.empty(nL, Hkv, T, d, "cuda")
    rx.pack([paged], [paged], [q], [0], layer=2)
    rx.sync_status()
    c, s = ref.held_rows(src[:, :, :T])
    assert torch.equal(q.k[2].cpu(), ref.packed_bytes(c)[0]) and torch.equal(q.v_scale[2].cpu().double(), s[0])


def test_values_that_cannot_be_held():
    """NaN is held as 0, what is above 7 * 2^13 as that; both are reported, and other rows are as ever."""
    x = _rows((1, 1, 40, 128), 4)
    x[0, 0, 3, 5] = float("nan")
    x[0, 0, 7, 40] = float("inf")
    x[0, 0, 8, 41] = -float("inf")
    x[0, 0, 9, 100] = -1e6
    x[0, 0, 11] = float("nan")
    x[0, 0, 12] = 0
    x[0, 0, 13] = -0.0
    x[0, 0, 14, :32] = 7.0 * 2 ** 13
    rx = _receiver(1, 1, 128, 40)
    p = cb.PackedKV.empty(1, 1, 40, 128, "cuda")
    rx.pack([x.cuda()], [_rows((1, 1, 40, 128), 5).cuda()], [p], [0])
    with pytest.raises(cb.CBError, match="CB_EDEVICE.*not finite"):
        rx.sync_status()
    rx.sync_status()
    _check(p.k, torch.arange(40), x, p.k_scale, "K")
    fine = x.clone()
    fine[~torch.isfinite(fine.float()) | (fine.abs() > ref.LARGEST)] = 1.0
    rx.pack([fine.cuda()], [fine.cuda()], [p], [0])          # the largest value that can be held is not reported
    rx.sync_status()


def test_bad_indices_rows_and_pages_are_skipped_and_reported():
    nL, Hkv, T, d = 1, 2, 64, 128
    K, V = (_rows((nL, Hkv, T, d), s).cuda() for s in (1, 2))
    rx = _receiver(nL, Hkv, d, T)

    def fresh():
        return [torch.full((nL, 8, 16, Hkv, w), 9, dtype=t, device="cuda")
                for w, t in ((d // 2, torch.uint8),) * 2 + ((d // 32, torch.bfloat16),) * 2]

    def run(idx=None, rows=None, table=(0, 1, 2, 3), why=""):
        a = fresh()
        p = cb.PackedKV(*a, T=T, pages=torch.tensor(table, dtype=torch.int32, device="cuda"))
        as32 = lambda x: None if x is None else [torch.tensor(x, dtype=torch.int32, device="cuda")]  # noqa: E731
        rx.pack([K], [V], [p], [0], idx=as32(idx), rows=as32(rows))
        with pytest.raises(cb.CBError, match="CB_EDEVICE.*" + why):
            rx.sync_status()
        return a[0][0]

    k = run(idx=[0, -1, 64, 5], why="index")
    c, _ = ref.held_rows(K[0, :, [0, 5]].cpu())
    assert torch.equal(k[0, [0, 3]].cpu(), ref.packed_bytes(c).transpose(0, 1)) and (k[0, 1:3] == 9).all()
    k = run(idx=[0, 1, 2], rows=[-1, 64, 7], why="destination")
    assert (k[0, :7] == 9).all() and (k[0, 7] != 9).any() and (k[4:] == 9).all()
    k = run(table=(5, 8, -1, 6), why="block-table")
    assert (k[[5, 6]] != 9).any() and (k[[0, 1, 2, 3, 4, 7]] == 9).all()
    # restoring through the same table: rows of zeros
    p = cb.PackedKV(*fresh(), T=T, pages=torch.tensor((5, 8, -1, 6), dtype=torch.int32, device="cuda"))
    ko, vo = torch.ones_like(K), torch.ones_like(V)
    rx.unpack([p], ko, vo)
    with pytest.raises(cb.CBError, match="CB_EDEVICE"):
        rx.sync_status()
    assert (ko[:, :, 16:48] == 0).all() and (vo[:, :, 16:48] == 0).all()
    # a scale that is none reads as 0
    p = cb.PackedKV.empty(nL, Hkv, 4, d, "cuda")
    p.k.fill_(0x9F); p.v.fill_(0x9F); p.v_scale.fill_(1.0)
    p.k_scale.copy_(torch.tensor([float("nan"), float("inf"), -1.0, 16384.0])[:, None].expand(4, d // 32))
    ko, vo = (torch.ones((nL, Hkv, 4, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    rx.unpack([p], ko, vo)
    with pytest.raises(cb.CBError, match="CB_EDEVICE.*scale"):
        rx.sync_status()
    assert (ko == 0).all() and (vo != 0).all()


def test_refusals():
    nL, Hkv, T, d = 2, 2, 32, 64
    K = _rows((nL, Hkv, T, d), 1).cuda()
    rx = _receiver(nL, Hkv, d, T, 2)
    p = cb.PackedKV.empty(nL, Hkv, T, d, "cuda")
    idx = torch.zeros(4, dtype=torch.int32, device="cuda")
    for status, call in [
            ("CB_EBUDGET", lambda: rx.pack([K], [K], [p], [1])),
            ("CB_EBUDGET", lambda: rx.pack([K], [K], [p], [-1])),
            ("CB_EBUDGET", lambda: rx.pack([K], [K], [p])),
            ("CB_EBUDGET", lambda: rx.pack([K], [K], [p], [0], counts=[T + 1])),
            ("CB_EBUDGET", lambda: rx.pack([K], [K], [p], [0], counts=[-1])),
            ("CB_ESHAPE", lambda: rx.pack([K], [K], [p], [0], layer=1)),
            ("CB_ESHAPE", lambda: rx.pack([K], [K], [p], [0], layer=-1)),
            ("CB_ESHAPE", lambda: rx.pack([K] * 3, [K] * 3, [p] * 3, [0] * 3, counts=[1] * 3)),
            ("CB_EINVAL", lambda: rx.pack([K.cpu()], [K.cpu()], [p], [0])),
            ("CB_EINVAL", lambda: rx.pack([K], [K], [cb.PackedKV.empty(nL, Hkv, T, d)], [0])),
            ("CB_EINVAL", lambda: rx.pack([K], [K], [p], [0], idx=[idx.cpu()])),
            ("CB_EBUDGET", lambda: rx.unpack([p], K[:, :, :16].contiguous(), K[:, :, :16].contiguous())),
            ("CB_EBUDGET", lambda: rx.unpack([p], K, K, counts=[T + 1], offsets=[0])),
            ("CB_EBUDGET", lambda: rx.unpack([p], K, K, [1])),
            ("CB_EINVAL", lambda: rx.unpack([p], K.cpu(), K.cpu())),
            ("CB_EINVAL", lambda: rx.score([K], [K], [K]))]:
        with pytest.raises(cb.CBError, match=status):
            call()
    for call in (lambda: rx.pack([K], [K], [cb.PackedKV.empty(nL, Hkv, T, 128, "cuda")], [0]),
                 lambda: rx.pack([K], [K], [p], [0], idx=[idx.long()]),
                 lambda: rx.pack([K], [K], [p], [0], idx=[idx], counts=[5]),
                 lambda: rx.unpack([p], K.float(), K.float())):
        with pytest.raises(ValueError):
            call()
    # nothing to do is no error
    rx.pack([K], [K], [p], [T], counts=[0])
    rx.unpack([p], K, K, counts=[0], offsets=[0])
    rx.sync_status()


def test_rows_past_32_bits_of_elements():
    """The last rows of a cache of over 2^32 elements a layer (2.4 GB of codes)."""
    Hkv, T, d = 1, (1 << 25) + 8, 128
    rx = _receiver(1, Hkv, d, T)
    p = cb.PackedKV(*[torch.zeros((1, Hkv, T, w), dtype=t, device="cuda")
                      for w, t in ((d // 2, torch.uint8),) * 2 + ((d // 32, torch.bfloat16),) * 2])
    K, V = (_rows((1, Hkv, 6, d), s).cuda() for s in (1, 2))
    rx.pack([K], [V], [p], [T - 6])
    rx.sync_status()
    c, s = ref.held_rows(V.cpu())
    assert torch.equal(p.v[:, :, T - 6:].cpu(), ref.packed_bytes(c)) and (p.v[:, :, :6] == 0).all()
    ko, vo = torch.zeros_like(K), torch.zeros_like(V)
    idx = torch.arange(T - 6, T, dtype=torch.int32, device="cuda")
    rx.unpack([p], ko, vo, idx=[idx])
    rx.sync_status()
    assert torch.equal(vo.double().cpu(), c * s.repeat_interleave(32, -1))


def test_a_row_written_twice_leaves_the_others_alone():
    Hkv, T, d = 2, 40, 128
    K, V = (_rows((1, Hkv, T, d), s).cuda() for s in (1, 2))
    rx = _receiver(1, Hkv, d, T)
    p = cb.PackedKV(*[torch.full((1, Hkv, T, w), 9, dtype=t, device="cuda")
                      for w, t in ((d // 2, torch.uint8),) * 2 + ((d // 32, torch.bfloat16),) * 2])
    rows = torch.tensor([5, 6, 5, 5, 7], dtype=torch.int32, device="cuda")
    rx.pack([K[:, :, :5]], [V[:, :, :5]], [p], rows=[rows])
    rx.sync_status()                             # codes and scales are well formed
    c, s = ref.held_rows(K[:, :, [1, 4]].cpu())
    assert torch.equal(p.k[:, :, 6:8].cpu(), ref.packed_bytes(c)) and torch.equal(p.k_scale[:, :, 6:8].cpu().double(), s)
    assert (p.k[:, :, :5] == 9).all() and (p.k[:, :, 8:] == 9).all() and (p.v_scale[:, :, 8:] == 9).all()


def test_lists_and_types_that_do_not_fit_are_refused():
    K = _rows((1, 2, 32, 64), 1).cuda()
    rx = _receiver(1, 2, 64, 32, 2)
    p = cb.PackedKV.empty(1, 2, 32, 64, "cuda")
    i32 = torch.zeros(4, dtype=torch.int32, device="cuda")
    for call in (lambda: rx.pack([K, K], [K], [p, p], [0, 0]),
                 lambda: rx.pack([K, K], [K, K], [p], [0, 0]),
                 lambda: rx.pack([K, K], [K, K], [p, p], [0]),
                 lambda: rx.pack([K, K], [K, K], [p, p], [0, 0], counts=[1]),
                 lambda: rx.pack([K, K], [K, K], [p, p], [0, 0], idx=[i32]),
                 lambda: rx.pack([K], [K[:, :, :8]], [p], [0]),
                 lambda: rx.pack([K.half()], [K.half()], [p], [0]),
                 lambda: rx.pack([K], [K], [p], [0], idx=[i32.float()]),
                 lambda: rx.unpack([p, p], K, K, counts=[1, 1], offsets=[0]),
                 lambda: rx.unpack([p], K.half(), K.half())):
        with pytest.raises(ValueError):
            call()
    rx.sync_status()
