"""cb_attend at the ends of what it takes, against the definition in 64 bits (tolerances: test_gpu_attend.py)."""
import pytest
import torch

import paper_2609_32046_gb300 as cb
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
