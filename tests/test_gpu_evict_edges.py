"""Eviction and kept rows on the GPU: streams, empty caches, what two entries share, lists at the edges of the ranking's forms."""
import pytest
import torch

import paper_2609_32046_gb300 as cb
from test_gpu_evict import Caches, check_idx, check_moved, want

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("by_handle", [False, True])
def test_idx_is_memory_of_the_stream(by_handle):
    """The result dropped, the current stream's next tensors of its size are written while the call's stream still ranks and
    moves: they are other memory, and the rows are right."""
    c = Caches(128, 2, [3000])
    stream = torch.cuda.Stream()
    given = stream.cuda_stream if by_handle else stream
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        torch.cuda._sleep(20_000_000)
    idx = c.rx.evict(c.caches, c.weights, 500, 1, 9, stream=given)
    at = idx[0].data_ptr()
    del idx
    others = [torch.full((2, 2, 500), 2999, dtype=torch.int32, device="cuda") for _ in range(3)]
    assert at not in [x.data_ptr() for x in others]
    stream.synchronize()
    c.rx.sync_status(given)
    torch.cuda.synchronize()
    check_moved(c, 0, want(c, 0, 500, 1, 9), 0, c.rows(c.caches[0]), c.weights[0])


def test_a_stream_by_the_handle_0():
    """The default stream given by its handle while another is current."""
    c = Caches(64, 1, [300])
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        idx = c.rx.evict(c.caches, c.weights, 100, stream=0)
    c.rx.sync_status(0)
    check_idx(idx[0], want(c, 0, 100, 0, 0), 100)


@pytest.mark.parametrize("into", [False, True])
@pytest.mark.parametrize("Ts", [[0], [0, 90, 0], [50, 0, 200, 0]])
def test_empty_caches(Ts, into):
    """A cache without rows is described by T = 0 as by a length of 0: -1 for every row that stays."""
    keep = 60
    c = Caches(128, 2, Ts, room=70)
    o = Caches(128, 2, [keep] * len(Ts), seed=3) if into else None
    idx = [torch.full((2, 2, keep), 7, dtype=torch.int32, device="cuda") for _ in Ts]
    left = [torch.full((1,), 9, dtype=torch.int32, device="cuda") for _ in Ts]
    c.rx.evict(c.caches, c.weights, keep, 2, 5, into=o.caches if into else None, idx=idx, lengths=left)
    c.rx.sync_status()
    for i, T in enumerate(Ts):
        at = want(c, i, keep, 2, 5)
        check_idx(idx[i], at, keep)
        check_moved(c, i, at, 0, c.rows((o if into else c).caches[i]), None if into else c.weights[i], was=o.was[i] if into else None)
        assert int(left[i]) == min(T, keep)
    if Ts[0] == 0:
        assert torch.equal(c.rx.evict(c.caches[:1], c.weights[:1], keep)[0], torch.full((2, 2, keep), -1, dtype=torch.int32, device="cuda"))
        with pytest.raises(cb.CBError):
            c.rx.evict(c.caches[:1], c.weights[:1], keep, idx=[idx[0].cpu()])
