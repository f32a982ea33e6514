"""Decoding with drafts under a budget of rows, as a server would run it: pack, attend over the tree, gather weights of what was
accepted, keep it, evict.  Every step against the definitions in 64 bits, on the state that it found; a captured step
does the same."""
import math

import pytest
import torch

import budget_reference as ref
import packed_reference
import paper_2609_32046_gb300 as cb

pytestmark = pytest.mark.gpu

LAYERS, HQ, HKV, D, M, BUDGET, ROOM = 2, 8, 2, 64, 12, 160, 240


class Server:
    def __init__(self, page, n=3):
        g = torch.Generator().manual_seed(7)
        self.n, self.page = n, page
        widths = ((D // 2, torch.uint8),) * 2 + ((D // 32, torch.bfloat16),) * 2
        if page:
            need = -(-ROOM // page)
            pool = [torch.zeros(LAYERS, n * need + 2, page, HKV, w, dtype=t, device="cuda") for w, t in widths]
            order = torch.randperm(n * need + 2, generator=g)[:n * need].int().view(n, need).cuda()
            self.caches = [cb.PackedKV(*pool, T=need * page, pages=t) for t in order]
        else:
            pool = [torch.zeros(n, LAYERS, HKV, ROOM, w, dtype=t, device="cuda") for w, t in widths]
            self.caches = [cb.PackedKV(*[x[i] for x in pool]) for i in range(n)]
        self.pool = pool
        self.length = torch.tensor([150, 158, 20][:n], dtype=torch.int32, device="cuda")
        for i, p in enumerate(self.caches):
            p.length = self.length[i:i + 1]
        self.room = self.caches[0].capacity
        self.weights = (torch.rand(n, LAYERS, HKV, self.room, generator=g) * 4).cuda()
        self.rx = cb.Receiver(LAYERS, HQ, HKV, D, M, self.room, n)
        first = [torch.randn(LAYERS, HKV, 160, D, generator=g).bfloat16().cuda() for _ in range(2)]
        self.rx.pack([first[0]] * n, [first[1]] * n, self.caches, [0] * n)
        # one step's inputs, written before each
        self.rows = [torch.zeros(M, dtype=torch.int32, device="cuda") for _ in range(n)]
        self.kv = [torch.zeros(2, LAYERS, HKV, M, D, dtype=torch.bfloat16, device="cuda") for _ in range(n)]
        self.q = torch.zeros(LAYERS, n, M, HQ, D, dtype=torch.bfloat16, device="cuda")
        self.trees = torch.zeros(n, M, 1, dtype=torch.int32, device="cuda")
        self.path = torch.zeros(n, 4, dtype=torch.int32, device="cuda")
        self.count = torch.zeros(n, dtype=torch.int32, device="cuda")
        self.left_out = torch.zeros(n, M, 1, device="cuda")           # infinity for drafts that are not accepted
        self.out, self.lse = torch.zeros_like(self.q), torch.zeros(LAYERS, n, M, HQ, device="cuda")
        self.idx = torch.zeros(n, LAYERS, HKV, BUDGET, dtype=torch.int32, device="cuda")

    def new_step(self, seed):
        g = torch.Generator().manual_seed(seed)
        for i in range(self.n):
            L = int(self.length[i])
            self.rows[i].copy_(torch.arange(L, L + M).int())
            self.kv[i].copy_(torch.randn(2, LAYERS, HKV, M, D, generator=g).bfloat16())
            parents = [int(torch.randint(-1, r, (1,), generator=g)) if r else -1 for r in range(M)]
            self.trees[i].copy_(cb.tree_words(parents))
            path, at = [], int(torch.randint(0, M, (1,), generator=g))
            while at >= 0:
                path.insert(0, at)
                at = parents[at]
            path = path[:4]
            self.path[i].copy_(torch.tensor(path + [M - 1] * (4 - len(path))).int())
            self.count[i] = len(path)
            self.left_out[i].fill_(math.inf)
            self.left_out[i][path] = 0
        self.q.copy_(torch.randn(self.q.shape, generator=g).bfloat16())

    def draft(self):
        for i in range(self.n):
            self.rx.pack([self.kv[i][0]], [self.kv[i][1]], [self.caches[i]], rows=[self.rows[i]])
        self.length += M
        for layer in range(LAYERS):
            self.rx.attend(self.caches, self.q[layer], self.out[layer], layer=layer, lses=self.lse[layer], trees=self.trees)

    def gather(self):
        for layer in range(LAYERS):
            self.rx.weigh(self.caches, self.q[layer], self.lse[layer] + self.left_out, self.weights[:, layer], layer=layer, trees=self.trees)

    def accept(self):
        self.rx.keep(self.caches, self.path, M, counts=self.count, weights=self.weights)

    def hold(self):
        self.rx.evict(self.caches, self.weights, BUDGET, first=2, last=20, idx=self.idx)

    def step(self):
        self.draft()
        self.gather()
        self.accept()
        self.hold()

    def bytes(self, i):
        p, out = self.caches[i], []
        for x in (p.k, p.v, p.k_scale, p.v_scale):
            x = x if x.dtype == torch.uint8 else x.view(torch.int16)
            out.append((x[:, p.pages.long()].flatten(1, 2).transpose(1, 2) if self.page else x).clone())
        return out

    def state(self):
        return [x.clone() for i in range(self.n) for x in self.bytes(i)] + [self.weights.clone(), self.length.clone()]


def check_step(s):
    """One step, each part against its definition on what it found."""
    before = [int(x) for x in s.length]
    w0 = s.weights.clone()
    s.draft()
    s.gather()
    s.rx.sync_status()
    scale = 1 / math.sqrt(D)
    for i, L0 in enumerate(before):
        L = L0 + M
        sees = ref.seen(M, L, bits=ref.unpacked(s.trees[i], M)).cuda()
        p = s.bytes(i)
        for layer in range(LAYERS):
            k, v = (packed_reference.values(c[layer][:, :L].contiguous(), x[layer][:, :L].contiguous().view(torch.bfloat16))
                    for c, x in ((p[0], p[2]), (p[1], p[3])))
            q = s.q[layer, i].double()
            o, lse, A, size = ref.attention(q, k, v, scale, sees)
            E = 2 * (D + 8) * 2.0 ** -23 * size + 2.0 ** -20 + L * 2.0 ** -23
            tol = o.abs() * 2.0 ** -8 + A * (2.0 ** -11 + 2 * E) + 2.0 ** -32 * L * float(v.abs().max())
            assert ((s.out[layer, i].double() - o).abs() <= tol).all()
            got = s.lse[layer, i].double()
            assert ((got - lse).abs() <= E + 2.0 ** -22 * lse.abs() + 2.0 ** -21).all()
            S, _ = ref.weights(q, k, got + s.left_out[i].double(), scale, sees)
            old = w0[i, layer, :, :L].double()
            old[:, L0:] = 0
            E = 2 * (D + 8) * 2.0 ** -23 * size + 2.0 ** -20 + 2.0 ** -22 * float(got.abs().max())
            tol = S * (math.expm1(E) + (M * HQ // HKV + 8) * 2.0 ** -23) + 2.0 ** -23 * (S + old)
            assert ((s.weights[i, layer, :, :L].double() - old - S).abs() <= tol).all()
            assert torch.equal(s.weights[i, layer, :, L:], w0[i, layer, :, L:])
    was, w1 = [s.bytes(i) for i in range(s.n)], s.weights.clone()
    s.accept()
    s.rx.sync_status()
    for i, L0 in enumerate(before):
        c = int(s.count[i])
        at = torch.cat([torch.arange(L0, device="cuda"), L0 + s.path[i, :c].long(), torch.arange(L0 + c, s.room, device="cuda")])
        for a, b in zip(s.bytes(i), was[i]):
            assert torch.equal(a, b[:, :, at])
        assert torch.equal(s.weights[i], w1[i][..., at]) and int(s.length[i]) == L0 + c
    was, w1, lengths = [s.bytes(i) for i in range(s.n)], s.weights.clone(), [int(x) for x in s.length]
    s.hold()
    s.rx.sync_status()
    for i, L in enumerate(lengths):
        n = min(L, BUDGET)
        assert int(s.length[i]) == n
        for layer in range(LAYERS):
            for g in range(HKV):
                at = ref.kept_rows(w1[i, layer, g].tolist(), L, BUDGET, 2, 20)
                assert s.idx[i, layer, g].tolist() == at + [-1] * (BUDGET - n)
                at = torch.tensor(at + list(range(n, s.room)), device="cuda")
                for a, b in zip(s.bytes(i), was[i]):
                    assert torch.equal(a[layer, g], b[layer, g, at])
                assert torch.equal(s.weights[i, layer, g], w1[i, layer, g, at])


@pytest.mark.parametrize("page", [0, 16])
def test_steps_against_the_definitions(page):
    s = Server(page)
    for seed in range(8):
        s.new_step(seed)
        check_step(s)
    assert [int(x) for x in s.length][:2] == [BUDGET] * 2


@pytest.mark.parametrize("page", [0, 16])
def test_a_captured_step(page):
    """The same steps by one graph, on another stream, end in the same bytes."""
    a, b = Server(page), Server(page)
    stream = torch.cuda.Stream()
    b.new_step(99)
    stream.wait_stream(torch.cuda.current_stream())
    start = b.state()
    pool = [x.clone() for x in b.pool]
    with torch.cuda.stream(stream):
        b.step()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            b.step()
        for x, y in zip(b.pool, pool):
            x.copy_(y)
        b.weights.copy_(start[-2])
        b.length.copy_(start[-1])
    torch.cuda.current_stream().wait_stream(stream)
    for seed in range(4):
        a.new_step(seed)
        b.new_step(seed)
        a.step()
        graph.replay()
        a.rx.sync_status()
        b.rx.sync_status()
        for x, y in zip(a.state(), b.state()):
            assert torch.equal(x, y)
