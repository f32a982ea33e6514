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
