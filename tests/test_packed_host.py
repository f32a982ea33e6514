"""PackedKV, Rotary and the packed format on the host (no GPU)."""
import ctypes

import pytest
import torch

import paper_2609_32046_gb300 as cb
import packed_reference as ref
from paper_2609_32046_gb300 import binding
from paper_2609_32046_gb300.build import build


@pytest.fixture(scope="module")
def lib():
    build()
    return binding.load_library()


def _arrays(shape, d):
    return [torch.zeros(shape + (w,), dtype=t) for w, t in ((d // 2, torch.uint8),) * 2 + ((d // 32, torch.bfloat16),) * 2]


@pytest.mark.parametrize("d", [64, 128])
def test_descriptions_of_every_layout(d):
    p = cb.PackedKV(*_arrays((3, 2, 50), d))
    x = p.desc()
    assert (x.T, x.s_layer, x.s_head, x.s_pos) == (50, 100 * d, 50 * d, d) and not x.pages and not x.length
    assert p.bytes == 2 * 3 * 2 * 50 * (d // 2 + d // 16)
    p = cb.PackedKV(*[a.transpose(1, 2) for a in _arrays((3, 50, 2), d)], T=17)
    x = p.desc()
    assert (x.T, x.s_layer, x.s_head, x.s_pos) == (17, 100 * d, d, 2 * d) and p.capacity == 50
    table = torch.arange(4, dtype=torch.int32)
    p = cb.PackedKV(*_arrays((3, 9, 16, 2), d), T=50, pages=table, length=torch.zeros(1, dtype=torch.int32))
    x = p.desc()
    assert (x.page_size, x.n_pages, x.s_page, x.s_layer, x.s_head, x.s_pos) == (16, 9, 32 * d, 288 * d, d, 2 * d)
    assert x.pages == table.data_ptr() and x.length and p.capacity == 64


def test_malformed_caches_are_refused():
    good = _arrays((1, 2, 50), 128)
    table = torch.arange(4, dtype=torch.int32)
    for bad in (lambda: cb.PackedKV(*good[:3], good[3][..., :2]),                       # scales of another width
                lambda: cb.PackedKV(good[0], good[1].transpose(1, 2).contiguous().transpose(1, 2), *good[2:]),   # other strides
                lambda: cb.PackedKV(*good, T=51),
                lambda: cb.PackedKV(*good, T=-1),
                lambda: cb.PackedKV(*good, pages=table),
                lambda: cb.PackedKV(*_arrays((1, 9, 12, 2), 128), pages=table),          # page size no power of two
                lambda: cb.PackedKV(*_arrays((1, 9, 16, 2), 128), pages=table.long()),
                lambda: cb.PackedKV(*good, length=torch.zeros(2, dtype=torch.int32)),
                lambda: cb.PackedKV(good[0].float(), *good[1:])):
        with pytest.raises(ValueError):
            bad()
    for kw in (dict(style="quarters"), dict(scaling="log")):
        with pytest.raises(ValueError):
            cb.Rotary(1e4, **kw)


def test_no_context_no_call(lib):
    assert lib.cb_rotary(None, 1, None, None, None) == binding.CB_EINVAL
    assert lib.cb_pack(None, 1, None, None, None, None, None, None, 0, 1, None) == binding.CB_EINVAL
    assert lib.cb_unpack(None, 1, None, None, None, None, None, 0, None, 0, 0, None) == binding.CB_EINVAL
    assert lib.cb_attend(None, 0, 1, None, None, 0, 0, None) == binding.CB_EINVAL
    assert lib.cb_create_receiver(None, ctypes.byref(ctypes.c_void_p())) == binding.CB_EINVAL


def test_the_formats_restatement_by_hand():
    """A row whose codes and scale are worked out by hand: 7 and -7 at the ends, halves away from zero."""
    x = torch.zeros(64)
    x[0], x[1], x[2], x[3], x[4] = 28.0, -28.0, 2.0, -2.0, 1.9921875          # scale 4: 2 / 4 is a half
    x[32] = 7.3                                                               # 7.3 / 7 lies above 16 / 16: 17 / 16
    c, s = ref.held_rows(x.to(torch.bfloat16)[None])
    assert s[0].tolist() == [4.0, 17 / 16] and c[0, :5].tolist() == [7, -7, 1, -1, 0] and c[0, 32] == 7
    b = ref.packed_bytes(c)[0].tolist()
    assert b[:4] == [0x9F, 0x88, 0x71, 0x88]      # elements 0 and 2, 4 and 6, 1 and 3, 5 and 7, each as c + 8
    assert torch.equal(ref.values(ref.packed_bytes(c), s), c * s.repeat_interleave(32, -1))


def test_packing_in_bf16_is_exact():
    """Codes -7..7 times any scale are bf16 numbers, and fp16 numbers."""
    s = torch.tensor([k * 2.0 ** e for e in range(-24, 9) for k in range(16, 32)] + [2.0 ** 13])
    v = torch.arange(-7.0, 8.0)[None] * s[:, None]
    assert torch.equal(v.to(torch.bfloat16).float(), v) and torch.equal(v.to(torch.float16).float(), v)


def test_a_cache_grows_within_its_room():
    p = cb.PackedKV(*_arrays((1, 2, 50), 128), T=3)
    p.T = 50
    for bad in (51, -1):
        with pytest.raises(ValueError):
            p.T = bad
    assert p.T == 50 and p.desc().T == 50


def test_other_types_are_refused():
    k, v, ks, vs = _arrays((1, 2, 50), 128)
    table = torch.arange(4, dtype=torch.int32)
    for bad in (lambda: cb.PackedKV(k, v, ks.half(), vs.half()), lambda: cb.PackedKV(k, v, ks, vs, length=torch.zeros(1)),
                lambda: cb.PackedKV(*_arrays((1, 9, 16, 2), 128), pages=table.float())):
        with pytest.raises(ValueError):
            bad()


def test_a_cache_is_described_for_each_call_by_itself():
    """Two threads' calls share a cache: one asks for its rows, the other for its room, between any two steps of each."""
    p = cb.PackedKV(*_arrays((1, 2, 50), 128), T=10)
    mine, other = p.desc(), p.desc(p.capacity)
    assert (mine.T, other.T) == (10, 50)
    desc = p.desc
    for meanwhile, after in ((lambda: desc(p.capacity), 10), (lambda: setattr(p, "T", 20), 20),
                             (lambda: setattr(p, "length", None), 20)):
        def late(T=None):
            d = desc(T)
            meanwhile()
            return d
        p.T = p.T                                 # (forgets what is kept)
        p.desc = late
        p._described()
        p.desc = desc
        kept = binding.cb_packed.from_buffer_copy(p._described())
        assert kept.T == p.T == after and kept.k == p.k.data_ptr() and kept.s_head == 50 * 128


def test_a_longer_block_table_is_the_one_that_calls_get():
    p = cb.PackedKV(*_arrays((1, 9, 16, 2), 128), T=40, pages=torch.arange(3, dtype=torch.int32))
    assert binding.cb_packed.from_buffer_copy(p._described()).pages == p.pages.data_ptr()
    longer = torch.arange(5, dtype=torch.int32)
    p.pages = longer
    for d in (p.desc(), binding.cb_packed.from_buffer_copy(p._described())):
        assert d.pages == longer.data_ptr() and d.T == 40
    assert p.pages is longer and p.capacity == 80
    p.T = 80
    for bad in (longer[:4], longer.long(), longer.float(), torch.arange(10, dtype=torch.int32)[::2], longer[None], None):
        with pytest.raises(ValueError):
            p.pages = bad
    assert p.pages is longer and p.desc().pages == longer.data_ptr() and (p.T, p.capacity) == (80, 80)
    flat = cb.PackedKV(*_arrays((1, 2, 50), 128))
    with pytest.raises(ValueError):
        flat.pages = longer
    assert flat.pages is None and not flat.desc().pages


def test_a_caches_arrays_are_its_own_for_good():
    arrays = _arrays((1, 2, 50), 128)
    p = cb.PackedKV(*arrays)
    for name, x in zip(("k", "v", "k_scale", "v_scale"), arrays):
        assert getattr(p, name) is x
        with pytest.raises(AttributeError):
            setattr(p, name, x.clone())
        assert getattr(p, name) is x
    p.k_scale += 1                                # in place: the same array
    assert p.k_scale is arrays[2] and (arrays[2] == 1).all()
