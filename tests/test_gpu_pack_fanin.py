"""Messages in 4 bits that are longer than any one sender: max_positions bounds a sender, not the message."""
import pytest
import torch

import paper_2609_32046_gb300 as cb
import packed_reference as ref

pytestmark = pytest.mark.gpu


def _rows(*shape, seed):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16).cuda()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Ts,keep", [([300, 300, 300], 0.5), ([256, 40, 256, 256, 199], 0.35)])
def test_a_filters_message_of_many_senders(d, Ts, keep):
    """Filter.pack holds what Filter.compact sends, of senders whose budgets add up to more than one of them has."""
    nL, Hq, Hkv, m = 2, 4, 2, 8
    c = cb.CacheBack(nL, Hq, Hkv, d, m, max(Ts), len(Ts))
    senders = [(_rows(nL, Hkv, T, d, seed=i), _rows(nL, Hkv, T, d, seed=50 + i)) for i, T in enumerate(Ts)]
    f = cb.Filter(c, senders, [_rows(nL, m, Hq, d, seed=99)] * len(Ts), keep).run()
    assert f.capacity > max(Ts)
    held = f.pack()
    c.sync_status()
    assert held.T == f.capacity
    for x, codes, scales in ((f.k_out, held.k, held.k_scale), (f.v_out, held.v, held.v_scale)):
        want, s = ref.held_rows(x.cpu())
        assert torch.equal(codes.cpu(), ref.packed_bytes(want)) and torch.equal(scales.cpu().double(), s)
    # all of it back, and what attention takes: a receiver's context has room for it
    ko, vo = torch.empty_like(f.k_out), torch.empty_like(f.v_out)
    c.unpack([held], ko, vo)
    c.sync_status()
    assert torch.equal(ko.double(), ref.values(held.k, held.k_scale)) and torch.equal(vo.double(), ref.values(held.v, held.v_scale))
    q = _rows(m, Hq, d, seed=7)
    with pytest.raises(cb.CBError, match="CB_ESHAPE"):
        c.attend([held], [q], [torch.empty_like(q)])
    cb.Receiver(nL, Hq, Hkv, d, m, f.capacity).attend([held], [q], [torch.empty_like(q)])


@pytest.mark.parametrize("page", [0, 16])
def test_rows_behind_max_positions(page):
    """A cache with more room than the context's max_positions: destination rows anywhere in it."""
    Hkv, d, T, room, n = 2, 128, 32, 400, 20
    K, V = (_rows(1, Hkv, T, d, seed=s) for s in (1, 2))
    widths = ((d // 2, torch.uint8),) * 2 + ((d // 32, torch.bfloat16),) * 2
    if page:
        table = torch.randperm(room // page, generator=torch.Generator().manual_seed(3)).int().cuda()
        p = cb.PackedKV(*[torch.full((1, room // page, page, Hkv, w), 9, dtype=t, device="cuda") for w, t in widths], pages=table)
    else:
        p = cb.PackedKV(*[torch.full((1, Hkv, room, w), 9, dtype=t, device="cuda") for w, t in widths])
    rows = torch.randperm(room, generator=torch.Generator().manual_seed(4))[:n].int().cuda()
    assert int(rows.max()) >= 10 * T
    rx = cb.Receiver(1, Hkv, Hkv, d, 1, T)
    rx.pack([K], [V], [p], counts=[n], rows=[rows])
    rx.sync_status()
    ko, vo = (torch.zeros((1, Hkv, n, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    rx.unpack([p], ko, vo, idx=[rows])
    rx.sync_status()
    for x, y in ((K, ko), (V, vo)):
        c, s = ref.held_rows(x[:, :, :n].cpu())
        assert torch.equal(y.double().cpu(), c * s.repeat_interleave(32, -1))
    for bad in (room, -1):
        with pytest.raises(cb.CBError, match="CB_EDEVICE.*destination"):
            rx.pack([K], [V], [p], counts=[1], rows=[torch.tensor([bad], dtype=torch.int32, device="cuda")])
            rx.sync_status()
    with pytest.raises(cb.CBError, match="CB_EBUDGET"):
        rx.pack([K], [V], [p], [room - T + 1])
    rx.pack([K], [V], [p], [room - T])
    rx.sync_status()


def test_pages_of_another_type_are_refused():
    """A paged sender's fp16 rows are no bf16 numbers: refused, as a strided sender's are."""
    Hkv, d, T = 2, 64, 32
    rx = cb.Receiver(1, Hkv, Hkv, d, 1, T)
    p = cb.PackedKV(*[torch.full((1, Hkv, T, w), 9, dtype=t, device="cuda")
                      for w, t in ((d // 2, torch.uint8),) * 2 + ((d // 32, torch.bfloat16),) * 2])
    table = torch.arange(2, dtype=torch.int32, device="cuda")
    pool = torch.ones((1, 2, 16, Hkv, d), dtype=torch.bfloat16, device="cuda")
    for k, v in ((pool.half(), pool.half()), (pool, pool.half()), (pool.half(), pool)):
        paged = cb.PagedKV(k, v, table, T)
        with pytest.raises(ValueError):
            rx.pack([paged], [paged], [p], [0])
    rx.sync_status()
    assert (p.k == 9).all() and (p.v_scale == 9).all()
    paged = cb.PagedKV(pool, pool, table, T)
    rx.pack([paged], [paged], [p], [0])
    rx.sync_status()
    assert (p.k_scale == 19 / 128).all()          # 1 / 7 rounded up to five bits
