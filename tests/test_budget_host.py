"""Drafted tokens' bits, and what the binding refuses and hands over of cb_weigh, cb_evict and cb_keep, without a GPU: the
library's calls are stood in for by one that writes its arguments down."""
import ctypes

import pytest
import torch

import budget_reference as ref
import paper_2609_32046_gb300 as cb
from paper_2609_32046_gb300 import binding


def ancestors(parents):
    m = len(parents)
    seen = torch.zeros(m, m, dtype=torch.bool)
    for r in range(m):
        u = r
        while u >= 0:
            seen[r, u] = True
            u = parents[u]
    return seen


@pytest.mark.parametrize("m", [1, 2, 31, 32, 33, 64, 65, 200])
def test_words_of_a_tree(m):
    g = torch.Generator().manual_seed(m)
    parents = [[int(torch.randint(-1, r, (1,), generator=g)) if r else -1 for r in range(m)] for _ in range(3)]
    words = cb.tree_words(parents)
    assert words.dtype == torch.int32 and tuple(words.shape) == (3, m, (m + 31) // 32)
    for p, w in zip(parents, words):
        assert torch.equal(ref.unpacked(w, m), ancestors(p))
        assert torch.equal(cb.pack_words(ancestors(p)), w)
    assert torch.equal(cb.tree_words(parents[0]), words[0])


def test_parents_that_are_none():
    for bad in ([0], [-2], [-1, 1], [-1, 0, 2], torch.tensor(3)):
        with pytest.raises(ValueError):
            cb.tree_words(bad)


class Spy:
    """Calls of the library, written down: (name, arguments), arrays copied."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, args))
            return binding.CB_OK
        return call


class tree(ctypes.Structure):
    _fields_ = [("seen", ctypes.c_void_p), ("s_row", ctypes.c_int64)]


class weigh_query(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("q", "lse", "before", "weights")] + [("m", ctypes.c_int32), ("fresh", ctypes.c_int64)] + \
               [(n, ctypes.c_int64) for n in ("s_tok", "s_head", "b_head", "w_head")]


class eviction(ctypes.Structure):
    _fields_ = [("weights", ctypes.c_void_p), ("weights_to", ctypes.c_void_p)] + \
               [(n, ctypes.c_int64) for n in ("w_layer", "w_head", "t_layer", "t_head", "keep", "first", "last")] + \
               [("idx", ctypes.c_void_p), ("length", ctypes.c_void_p)]


class kept(ctypes.Structure):
    _fields_ = [("idx", ctypes.c_void_p), ("count", ctypes.c_int64), ("n_kept", ctypes.c_void_p), ("drafted", ctypes.c_int64),
                ("weights", ctypes.c_void_p), ("w_layer", ctypes.c_int64), ("w_head", ctypes.c_int64), ("length", ctypes.c_void_p)]


class Reading(Spy):
    """A Spy that reads the arrays of a call while it lasts."""

    def __init__(self, at, what, n):
        super().__init__()
        self.at, self.what, self.n, self.seen = at, what, n, None

    def __getattr__(self, name):
        def call(*args):
            at = args[self.at]
            self.seen = [self.what.from_buffer_copy(ctypes.string_at(at + i * ctypes.sizeof(self.what), ctypes.sizeof(self.what)))
                         for i in range(self.n)]
            self.calls.append((name, args))
            return binding.CB_OK
        return call


def receiver(spy, layers=3, Hq=8, Hkv=2, d=64):
    rx = object.__new__(cb.Receiver)
    rx.lib, rx.h, rx._shape = spy, None, (layers, Hkv, d)
    rx.cfg = binding.cb_config(n_layers=layers, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=d)
    return rx


def cache(T, layers=3, Hkv=2, d=64, length=None):
    arrays = [torch.zeros(layers, Hkv, T, w, dtype=t) for w, t in ((d // 2, torch.uint8),) * 2 + ((d // 32, torch.bfloat16),) * 2]
    return cb.PackedKV(*arrays, length=length)


def test_one_tensor_and_lists_hand_over_the_same(monkeypatch):
    monkeypatch.setattr(binding, "_stream_on", lambda stream, x: 0)
    caches = [cache(40), cache(50), cache(7)]
    q, lse = torch.zeros(3, 5, 8, 64, dtype=torch.bfloat16), torch.zeros(3, 5, 8)
    w, o = torch.zeros(3, 2, 60), torch.zeros(2, 3, 64).transpose(0, 1)
    words = torch.zeros(3, 5, 2, dtype=torch.int32)[:, :, :1]
    got = []
    for a in ((q, lse, w, o, words), tuple(list(x) for x in (q, lse, w, o, words))):
        spy = Reading(4, weigh_query, 3)
        assert receiver(spy).weigh(caches, a[0], a[1], a[2], trees=a[4], outs=a[3]) is not None
        got.append([bytes(x) for x in spy.seen])
    assert got[0] == got[1]
    x = weigh_query.from_buffer_copy(got[0][1])
    assert (x.q, x.lse, x.before, x.weights) == (q[1].data_ptr(), lse[1].data_ptr(), w[1].data_ptr(), o[1].data_ptr())
    assert (x.m, x.fresh, x.s_tok, x.s_head, x.b_head, x.w_head) == (5, 5, 8 * 64, 64, 60, 3 * 64)

    w, into = torch.zeros(3, 3, 2, 60), [cache(20) for _ in range(3)]
    wto, idx, left = torch.zeros(3, 3, 2, 24), torch.zeros(3, 3, 2, 20, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    got = []
    for a in ((w, wto, idx, left), tuple(list(x) for x in (w, wto, idx)) + (list(left.split(1)),)):
        spy = Reading(6, eviction, 3)
        receiver(spy).evict(caches, a[0], 20, 1, 2, into=into, weights_into=a[1], idx=a[2], lengths=a[3])
        got.append([bytes(x) for x in spy.seen])
    assert got[0] == got[1]
    x = eviction.from_buffer_copy(got[0][2])
    assert (x.weights, x.weights_to, x.idx, x.length) == (w[2].data_ptr(), wto[2].data_ptr(), idx[2].data_ptr(), left[2:].data_ptr())
    assert (x.w_layer, x.w_head, x.t_layer, x.t_head, x.keep, x.first, x.last) == (120, 60, 48, 24, 20, 1, 2)

    idx, counts, w = torch.zeros(3, 4, dtype=torch.int32), torch.zeros(3, dtype=torch.int32), torch.zeros(3, 3, 2, 60)
    got = []
    for a in ((idx, counts, w), (list(idx), list(counts.split(1)), list(w))):
        spy = Reading(3, kept, 3)
        receiver(spy).keep(caches, a[0], 6, counts=a[1], weights=a[2], lengths=list(left.split(1)))
        got.append([bytes(x) for x in spy.seen])
    assert got[0] == got[1]
    x = kept.from_buffer_copy(got[0][1])
    assert (x.idx, x.count, x.n_kept, x.drafted) == (idx[1].data_ptr(), 4, counts[1:].data_ptr(), 6)
    assert (x.weights, x.w_layer, x.w_head, x.length) == (w[1].data_ptr(), 120, 60, left[1:].data_ptr())


def test_lists_that_do_not_fit(monkeypatch):
    monkeypatch.setattr(binding, "_stream_on", lambda stream, x: 0)
    spy = Spy()
    rx, p = receiver(spy), cache(40)
    q, lse, w = torch.zeros(1, 5, 8, 64, dtype=torch.bfloat16), torch.zeros(1, 5, 8), torch.zeros(1, 2, 40)
    for kw in (dict(Qs=q[..., :32]), dict(Qs=q.float()), dict(lses=lse[..., :4]), dict(lses=lse.double()), dict(weights=w[..., :39]),
               dict(weights=w.half()), dict(weights=w[:, :1]), dict(outs=torch.zeros(1, 2, 39)), dict(weights=None), dict(caches=[p, p]),
               dict(trees=torch.zeros(1, 4, 1, dtype=torch.int32)), dict(trees=torch.zeros(1, 5, 1)), dict(window=2, causal=False),
               dict(caches=[cache(40, layers=2)]), dict(fresh=[1, 2])):
        with pytest.raises(ValueError):
            rx.weigh(**{**dict(caches=[p], Qs=q, lses=lse, weights=w), **kw})
    w, idx = torch.zeros(1, 3, 2, 40), torch.zeros(1, 3, 2, 9, dtype=torch.int32)
    on_device = cache(40, length=torch.zeros(1, dtype=torch.int32))
    for kw in (dict(weights=w[..., :30]), dict(weights=w[0]), dict(weights=w.double()), dict(idx=idx[..., :8]), dict(idx=idx.long()),
               dict(idx=idx.transpose(1, 2)), dict(idx=torch.zeros(1, 3, 2, 18, dtype=torch.int32)[..., ::2]), dict(keep=[9, 9]),
               dict(weights_into=w), dict(into=[cache(9), cache(9)]), dict(caches=[on_device], into=[cache(9)]),
               dict(lengths=[torch.zeros(1)]), dict(lengths=[torch.zeros(2, dtype=torch.int32)])):
        with pytest.raises(ValueError):
            rx.evict(**{**dict(caches=[p], weights=w, keep=9, idx=idx), **kw})
    idx = torch.zeros(1, 3, dtype=torch.int32)
    for kw in (dict(idx=idx.long()), dict(idx=idx[0]), dict(idx=[idx]), dict(counts=idx[0, :1]), dict(caches=[on_device], lengths=[None]),
               dict(weights=w[..., :30]), dict(drafted=[4, 4]), dict(lengths=[torch.zeros(1)])):
        with pytest.raises(ValueError):
            rx.keep(**{**dict(caches=[p], idx=idx, drafted=5), **kw})
    assert not spy.calls and p.T == 40


def test_lengths_on_the_host_follow(monkeypatch):
    monkeypatch.setattr(binding, "_stream_on", lambda stream, x: 0)
    rx, p, small = receiver(Spy()), cache(40), cache(9)
    w = torch.zeros(1, 3, 2, 40)
    rx.evict([p], w, 9, into=[small])
    assert (p.T, small.T) == (40, 9)
    rx.keep([p], torch.zeros(1, 3, dtype=torch.int32), 10)
    assert p.T == 33
    rx.evict([p], w, 50)
    assert p.T == 33
    rx.evict([p], w, 0)
    assert p.T == 0
