"""Gathered attention weights on the GPU: what lies behind a cache's rows in the arrays that are written."""
import pytest
import torch

from test_gpu_weigh import Weighed

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("m", [1, 4, 5, 90, 400])
@pytest.mark.parametrize("given", [True, False])
@pytest.mark.parametrize("lengths", [None, [0, 1, 129, 333, 2000, 5000]])
def test_rows_behind_the_last_stay(m, given, lengths):
    """outs in other memory: rows from L on and other heads' gaps keep their bits, whether there was something before or not."""
    Ts = [m, m + 1, m + 127, 600, 2 * m + 1000, m + 3000]
    c = Weighed(64, 8, 2, [m] * 6, Ts, lengths=lengths, page=16)
    most = max(p.capacity for p in c.caches)
    room = torch.rand(6, 2, most + 400, device="cuda")
    was, outs = room.clone(), room[:, :, :most + 130]
    before = torch.rand(6, 2, most + 7, device="cuda") if given else None
    had = [torch.zeros(2, most + 7, device="cuda") for _ in Ts] if before is None else [x.clone() for x in before]
    c.rx.weigh(c.caches, torch.stack(c.q), torch.stack(c.lse), before, outs=outs, decay=0.5)
    c.check(got=[x for x in outs], before=had, decay=0.5, lengths=lengths)
    for i, T in enumerate(Ts):
        L = T if lengths is None else min(T, lengths[i])
        assert torch.equal(room[i, :, L:], was[i, :, L:])
    if given:
        assert all(torch.equal(a, b) for a, b in zip(before, had))
