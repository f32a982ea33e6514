"""cb_attend at the ends of what it takes, against the definition in 64 bits (tolerances: test_gpu_attend.py)."""
import pytest
import torch

import paper_2609_32046_gb300 as cb
import packed_reference as ref
from test_gpu_attend import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("window", [2 ** 31, 2 ** 32 + 5, 2 ** 62, 2 ** 63 - 65, 2 ** 63 - 1])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("m,Ts", [(1, [5000, 1]), (64, [3000, 40]), (130, [700, 32, 129])])
def test_windows_of_any_size(window, d, m, Ts):
    """A window that reaches past every row is none, to sys.maxsize; tokens before the cache's first row too."""
    c = Case(d, 8, 2, [m] * len(Ts), Ts, seed=m)
    c.run()
    want = [x.clone() for x in c.out + c.lse]
    for x in c.out + c.lse:
        x.fill_(7)
    c.run(window=window)
    c.check()
    assert all(torch.equal(a, b) for a, b in zip(want, c.out + c.lse))


@pytest.mark.parametrize("m", [1, 70])
def test_a_block_table_that_grows(m):
    """A sequence that outgrows its block table is given a longer one: the cache's next calls read that."""
    c = Case(128, 8, 2, [m], [200], page=16, room=400)
    p, whole = c.caches[0], c.caches[0].pages
    short = cb.PackedKV(p.k, p.v, p.k_scale, p.v_scale, T=200, pages=whole[:13].clone())
    c.caches = [short]
    c.run()
    c.check()
    short.pages = whole
    short.T = 600
    K, V = (torch.randn((1, 2, 400, 128), device="cuda").to(torch.bfloat16) for _ in range(2))
    c.rx = cb.Receiver(1, 8, 2, 128, m, 600)
    c.rx.pack([K], [V], [short], [200])
    c.run()
    c.check()


@pytest.mark.parametrize("scale", [2.0 ** -24, 1e-8, 1e-30, 1e-44])
@pytest.mark.parametrize("m,T", [(1, 40), (4, 200), (70, 300)])
def test_softmax_scales_near_zero(scale, m, T):
    """Logits of next to nothing, queries of zeros among them: every row that is seen weighs the same, and rows that
    are not seen weigh nothing."""
    c = Case(128, 8, 2, [m], [T], seed=3)
    c.q[0][0] = 0                                  # a padded token
    c.q[0][m - 1, 3] = 0
    c.q[0][m - 1, 4] = 2.0 ** -130
    c.rx = cb.Receiver(1, 8, 2, 128, m, T, softmax_scale=scale)
    c.run()
    c.rx.sync_status()
    k, v = c.kv(0, 0, T)
    o, lse, A, size = ref.attention(c.q[0].double(), k, v, scale)
    E = 2 * (128 + 8) * 2.0 ** -23 * size + 2.0 ** -20 + T * 2.0 ** -23
    tol = o.abs() * 2.0 ** -8 + A * (2.0 ** -11 + 2 * E) + 2.0 ** -32 * T * float(v.abs().max())
    assert ((c.out[0].double() - o).abs() <= tol).all()
    assert ((c.lse[0].double() - lse).abs() <= E + 2.0 ** -22 * lse.abs() + 2.0 ** -21).all()


@pytest.mark.parametrize("m", [1, 30])
def test_sequences_that_write_the_same_rows_are_refused(m):
    c = Case(128, 8, 2, [m] * 3, [70, 50, 300])
    q, o, e = c.q, c.out, c.lse
    one = torch.full((m, 8, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    stack, lse = torch.stack(q), torch.full((3, m, 8), 7.0, device="cuda")
    flat = torch.full((3 * m * 8 * 128,), 7.0, dtype=torch.bfloat16, device="cuda")
    step = m * 8 * 128 - 128                       # the last row of one sequence is the first of the next
    for call in (lambda: c.rx.attend(c.caches, stack, one[None].expand(3, -1, -1, -1)),
                 lambda: c.rx.attend(c.caches, q, [o[0], o[1], o[0]], lses=e),
                 lambda: c.rx.attend(c.caches, q, o, lses=[e[0], e[0], e[2]]),
                 lambda: c.rx.attend(c.caches, stack, torch.stack(o), lses=lse[:1].expand(3, -1, -1)),
                 lambda: c.rx.attend(c.caches, stack, flat.as_strided((3, m, 8, 128), (step, 1024, 128, 1)))):
        with pytest.raises(cb.CBError, match="CB_EINVAL.*same rows"):
            call()
    torch.cuda.synchronize()
    assert all((x == 7).all() for x in o + e + [one, lse, flat])
    # tokens of the sequences side by side, the other way round in memory, and a sequence without tokens
    room = torch.full((m, 3, 8, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    c.out = [room[:, 2 - i] for i in range(3)]
    c.run()
    c.check()
    c.rx.attend(c.caches, [q[0], q[1][:0], q[2]], [o[0], o[0][:0], o[2]], lses=[e[0], e[0][:0], e[2]])
    c.out = o
    c.check(which=[0, 2])


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("m,Ts", [(20, [300]), (20, [6000, 40, 1]), (40, [300]), (100, [6000, 500])])
def test_a_bounded_wait_gives_up_and_the_context_recovers(d, m, Ts):
    """Failure detection without a GPU fault: the warp that issues the products waits on a barrier that nothing arrives
    on.  After the limit it gives up, every role leaves its loop and meets the others, tensor memory is freed, and
    the host reads CB_ETIMEOUT; the same context's next call is right.  (One row tile's two streams, by tiles
    of up to 128 rows and by halves of more; segments of one block and of many.)"""
    c = Case(d, 8, 2, [m] * len(Ts), Ts, seed=m)
    one = Case(d, 8, 2, [1], [100])
    for _ in range(2):
        c.rx.set_wait_limit(20_000_000, stall_next_attend=True)          # 20 ms
        c.rx.attend(one.caches, one.q, one.out, lses=one.lse)            # the kernel of few rows has no waits
        c.rx.sync_status()
        one.check()
        c.run()
        with pytest.raises(cb.CBError, match="gave up") as e:
            c.rx.sync_status()
        assert e.value.status == cb.CB_ETIMEOUT
        for x in c.out + c.lse:
            x.fill_(7)
        c.run()                                    # the stall was for one call; ordinary waits stay far below the limit
        c.check()
    with pytest.raises(ValueError):
        c.rx.set_wait_limit(0, stall_next_score=True, stall_next_attend=True)
    assert c.rx.lib.cb_set_wait_limit(c.rx.h, 0, 3) == cb.CB_EINVAL


@pytest.mark.parametrize("m", [1, 4, 50, 100])
def test_a_second_run_writes_every_row_again(m):
    """The same bits from a second run, on another stream and out of a captured graph, over outputs that were
    overwritten in between; the outputs of the joins among them."""
    c = Case(128, 32, 8, [m] * 3, [9000, 100, 1999], page=16)
    c.run()
    torch.cuda.synchronize()
    want = [x.clone() for x in c.out + c.lse]
    c.check()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.run()
    for stream, run in ((side, lambda: c.run(stream=side)), (side, graph.replay), (torch.cuda.current_stream(), c.run)):
        with torch.cuda.stream(stream):
            for x in c.out + c.lse:
                x.fill_(7)
            run()
        stream.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, c.out + c.lse))
    c.rx.sync_status()


@pytest.mark.parametrize("m", [2, 40])
def test_two_contexts_on_two_streams_write_their_own(m):
    """Two contexts at once over the same caches: every round's outputs and log-sum-exps are overwritten before it."""
    a = Case(128, 8, 2, [m, m], [9000, 700])
    b = Case(128, 8, 2, [m, m], [9000, 700])
    b.q, b.caches = a.q, a.caches
    a.run()
    a.check()
    want = [x.clone() for x in a.out + a.lse]
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        for s, c in zip(streams, (a, b)):
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                for x in c.out + c.lse:
                    x.fill_(7)
                for _ in range(4):
                    c.run()
        torch.cuda.synchronize()
        for c in (a, b):
            assert all(torch.equal(x, y) for x, y in zip(want, c.out + c.lse))
    a.rx.sync_status()
    b.rx.sync_status()


@pytest.mark.parametrize("m", [1, 70])
def test_graphs_that_share_a_context_write_every_row(m):
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
    for _ in range(3):
        for x in a.out + a.lse + b.out + b.lse:
            x.fill_(7)
        for g in graphs:
            g.replay()
        a.check()
        b.check()


@pytest.mark.parametrize("d,Hq,Hkv", [(128, 4, 1), (64, 8, 2), (128, 2, 2)])
@pytest.mark.parametrize("m,T,window", [(1024, 1024, 0), (1024, 3001, 0), (1023, 5000, 700), (769, 500, 0)])
def test_as_many_tokens_as_a_context_takes(d, Hq, Hkv, m, T, window):
    """Up to sixteen row tiles a sequence; more tokens than rows as well."""
    c = Case(d, Hq, Hkv, [m], [T], seed=m)
    c.run(window=window)
    c.check(window=window)
    c.run(causal=False)
    c.check(causal=False)


@pytest.mark.parametrize("d", [64, 128])
def test_as_many_row_tiles_as_a_launch_takes(d):
    """64 sequences of 1024 tokens in groups of 4: 1024 row tiles."""
    c = Case(d, 4, 1, [1024] * 64, [1 + 37 * i for i in range(64)], page=16)
    c.run()
    c.check()


@pytest.mark.parametrize("d,Hq,Hkv", [(128, 32, 8), (128, 8, 8), (64, 32, 8), (64, 16, 16)])
@pytest.mark.parametrize("causal,window", [(True, 0), (True, 300), (False, 0)])
def test_more_items_than_blocks(d, Hq, Hkv, causal, window):
    """More items (row tile, KV head) than blocks: runs end inside items, and those are joined by the block that they
    begin in."""
    n = 24
    c = Case(d, Hq, Hkv, [33 + 3 * (i % 5) for i in range(n)], [40 + 97 * i for i in range(n)], page=32, seed=d)
    for _ in range(2):
        for x in c.out + c.lse:
            x.fill_(7)
        c.run(causal=causal, window=window)
        c.check(causal=causal, window=window)


@pytest.mark.parametrize("d,Hq,Hkv", [(128, 32, 8), (64, 8, 4)])
@pytest.mark.parametrize("longest", [3, 9, 64, 300])
@pytest.mark.parametrize("window", [0, 129])
def test_token_counts_that_differ(d, Hq, Hkv, longest, window):
    """A batch of decoding sequences with one of more tokens among them."""
    ms = [1] * 12 + [longest, 2, 0, 1]
    Ts = [1 + 233 * i for i in range(12)] + [longest + 900, 1, 50, 2000]
    c = Case(d, Hq, Hkv, ms, Ts, page=16, seed=longest)
    c.run(window=window)
    c.check(window=window)
