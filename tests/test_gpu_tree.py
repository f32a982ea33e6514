"""Attention of drafted tokens over 4-bit caches on the GPU against the definition in 64 bits; the tolerance is that of
test_gpu_attend.py, whose kernels these are."""
import math

import pytest
import torch

import budget_reference as ref
import paper_2609_32046_gb300 as cb
from test_gpu_attend import Case

pytestmark = pytest.mark.gpu


def bits_of(kind, m, seed):
    g = torch.Generator().manual_seed(seed)
    if kind == "chain":
        return torch.ones(m, m, dtype=torch.bool).tril()
    if kind == "none":
        return torch.zeros(m, m, dtype=torch.bool)
    if kind == "all":
        return torch.ones(m, m, dtype=torch.bool)
    if kind == "any":
        return (torch.rand(m, m, generator=g) < 0.4) & (torch.rand(m, 1, generator=g) < 0.8)
    parents = [int(x * (r + 1)) - 1 for r, x in enumerate(torch.rand(m, generator=g).tolist())]
    return ref.unpacked(cb.tree_words(parents), m)


def check(c, bits, lengths=None, layer=0):
    c.rx.sync_status()
    for i, q in enumerate(c.q):
        m = q.shape[0]
        if m == 0:
            continue
        T = c.caches[i].T
        L = T if lengths is None else max(0, min(T, lengths[i]))
        k, v = c.kv(i, layer, L)
        # (drafts without rows: the bits of the last L of them alone say something of a row)
        sees = ref.seen(m, L, bits=bits[i]).cuda() if bits[i] is None or m <= L else bits[i][:, m - L:].cuda()
        o, lse, A, size = ref.attention(q.double(), k, v, 1 / math.sqrt(c.d), sees)
        E = 2 * (c.d + 8) * 2.0 ** -23 * size + 2.0 ** -20 + L * 2.0 ** -23
        big = float(v.abs().max()) if L else 0.0
        tol = o.abs() * 2.0 ** -8 + A * (2.0 ** -11 + 2 * E) + 2.0 ** -32 * L * big
        err = (c.out[i].double() - o).abs()
        assert (err <= tol).all(), "sequence %d: off by %.3g" % (i, float((err - tol).max()))
        empty = torch.isinf(lse)
        assert torch.equal(torch.isinf(c.lse[i]), empty) and (c.out[i][empty] == 0).all()
        off = (c.lse[i].double() - lse)[~empty].abs()
        assert (off <= E + 2.0 ** -22 * lse[~empty].abs() + 2.0 ** -21).all()


@pytest.mark.parametrize("d,Hq,Hkv", [(128, 32, 8), (128, 2, 2), (64, 8, 2), (64, 4, 4), (64, 2, 1)])
@pytest.mark.parametrize("m,T", [(1, 1), (1, 300), (2, 2), (4, 33), (5, 700), (8, 129), (16, 17), (31, 31), (32, 333), (33, 160),
                                 (64, 2051), (65, 130), (129, 500), (250, 1111)])
@pytest.mark.parametrize("kind", ["tree", "any"])
def test_one_sequence(d, Hq, Hkv, m, T, kind):
    c = Case(d, Hq, Hkv, [m], [T], seed=m)
    bits = bits_of(kind, m, m + T)
    c.run(trees=[cb.pack_words(bits).cuda()])
    check(c, [bits])


@pytest.mark.parametrize("m", [3, 20, 70, 256])
@pytest.mark.parametrize("kind", ["none", "all", "chain"])
def test_bits_at_both_ends(m, kind):
    c = Case(128, 8, 2, [m, m], [m, 400 + m], page=16, seed=m)
    bits = bits_of(kind, m, 0)
    c.run(trees=[cb.pack_words(bits).cuda()] * 2)
    check(c, [bits] * 2)
    assert kind != "none" or (c.out[0] == 0).all()


@pytest.mark.parametrize("m", [4, 16, 70])
def test_a_chain_is_causal(m):
    """Each token its ancestors: the bits of cb_attend's own results, and so is a sequence without bits."""
    c = Case(128, 8, 2, [m] * 3, [m, 500, 2000], page=16)
    c.run()
    outs, lses = [x.clone() for x in c.out], [x.clone() for x in c.lse]
    chain = cb.pack_words(bits_of("chain", m, 0)).cuda()
    for trees in ([None] * 3, [chain, None, chain], torch.stack([chain] * 3)):
        for x in c.out + c.lse:
            x.fill_(3)
        c.run(trees=trees)
        c.rx.sync_status()
        for a, b in zip(outs + lses, c.out + c.lse):
            assert torch.equal(a, b)


@pytest.mark.parametrize("d,Hq,Hkv", [(128, 8, 2), (64, 2, 2)])
@pytest.mark.parametrize("page", [0, 1, 16, 64])
@pytest.mark.parametrize("m", [4, 7, 60])
def test_ragged_batches(d, Hq, Hkv, page, m):
    """Lengths around tiles and pages, token counts that differ, some without bits, drafts that have no rows."""
    Ts = [m, 100 + m, 128 + m, 129 + m, 600, m // 2, 1025]
    ms = [m, m, 1, m, 0, m, max(1, m - 1)]
    c = Case(d, Hq, Hkv, ms, Ts, page=page, layers=2, layout="positions", room=9)
    bits = [None if i == 3 else bits_of("any", x, i) for i, x in enumerate(ms)]
    c.run(layer=1, trees=[None if x is None else cb.pack_words(x).cuda() for x in bits])
    check(c, bits, layer=1)


@pytest.mark.parametrize("m", [4, 40])
def test_wide_rows_of_words_and_lengths_on_the_device(m):
    """Words of a wider array, bits behind the last token set; a captured call follows lengths and bits."""
    Ts, lengths = [900, 900, 300], [m, 899, 5000]
    c = Case(128, 8, 2, [m] * 3, Ts, lengths=lengths, page=16)
    bits = [bits_of("any", m, i) for i in range(3)]
    wide = torch.full((3, m, 7), -1, dtype=torch.int32, device="cuda")
    n = (m + 31) // 32

    def put(bits):
        for i, x in enumerate(bits):
            w = cb.pack_words(torch.cat([x, torch.ones(m, -m % 32, dtype=torch.bool)], 1))
            wide[i, :, 2:2 + n].copy_(w)
    put(bits)
    trees = wide[:, :, 2:2 + n]
    c.run(trees=list(trees))
    check(c, bits, lengths)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.run(trees=list(trees))
    for grown in ([m + 1, 640, 2], [899, 0, 300]):
        for p, x in zip(c.caches, grown):
            p.length.fill_(x)
        bits = [bits_of("tree", m, x) for x in grown]
        put(bits)
        graph.replay()
        check(c, bits, grown)


@pytest.mark.parametrize("m", [3, 300])
def test_one_tensor_for_all_and_repeated_runs(m):
    n = 5
    c = Case(128, 4, 1, [m] * n, [m + 50 * i for i in range(n)])
    bits = [bits_of("tree", m, i) for i in range(n)]
    q, out, lse = torch.stack(c.q), torch.stack(c.out), torch.stack(c.lse)
    trees = torch.stack([cb.pack_words(x) for x in bits]).cuda()
    c.rx.attend(c.caches, q, out, lses=lse, trees=trees)
    c.out, c.lse = list(out), list(lse)
    check(c, bits)
    again = torch.empty_like(out)
    c.rx.attend(c.caches, q, again, trees=trees)
    assert torch.equal(again, out)


@pytest.mark.parametrize("m", [2, 30])
def test_more_sequences_than_a_launch_takes(m):
    n = 70
    c = Case(64, 4, 2, [m] * n, [m + 5 * i for i in range(n)])
    bits = [None if i % 7 == 3 else bits_of("tree", m, i) for i in range(n)]
    c.run(trees=[None if x is None else cb.pack_words(x).cuda() for x in bits])
    check(c, bits)


def test_refusals():
    c = Case(128, 8, 2, [8], [100])
    w = cb.pack_words(bits_of("tree", 8, 0)).cuda()
    long = torch.zeros(40, 3, dtype=torch.int32, device="cuda")
    for kw in (dict(trees=[w], causal=False), dict(trees=[w], window=3), dict(trees=[w, w]), dict(trees=[w.float()]),
               dict(trees=[w[:5]]), dict(trees=[long[:8, :0]]), dict(trees=[w.long()])):
        with pytest.raises(ValueError):
            c.run(**kw)
    with pytest.raises(cb.CBError):
        c.run(trees=[w.cpu()])
    d = Case(128, 8, 2, [40], [100])
    with pytest.raises(cb.CBError):
        d.run(trees=[long[:, :2].as_strided((40, 2), (1, 1))])          # rows of words that overlap
    c.rx.sync_status()
    assert (c.out[0] == 7).all() and (c.lse[0] == 7).all()
