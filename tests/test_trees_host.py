"""Drafted tokens' bits at the ends of what they may be, without a GPU."""
import pytest
import torch

import paper_2609_32046_gb300 as cb
from paper_2609_32046_gb300 import binding
from test_budget_host import Spy, cache, receiver


@pytest.mark.parametrize("shape", [(0,), (3, 0), (0, 5), (2, 3, 0)])
def test_no_tokens(shape):
    """A sequence that drafted nothing has no words (a call skips it), nor has a batch of no sequences."""
    words = cb.tree_words(torch.zeros(shape, dtype=torch.int64))
    assert words.dtype == torch.int32 and tuple(words.shape) == shape + ((shape[-1] + 31) // 32,)


def test_a_batch_whose_sequences_drafted_nothing(monkeypatch):
    monkeypatch.setattr(binding, "_stream_on", lambda stream, x: 0)
    spy = Spy()
    q = [torch.zeros(m, 8, 64, dtype=torch.bfloat16) for m in (0, 2)]
    receiver(spy).attend([cache(40), cache(30)], q, [x.clone() for x in q], trees=[cb.tree_words([]), cb.tree_words([-1, 0])])
    assert [name for name, _ in spy.calls] == ["cb_attend_tree"]


def test_batches_of_trees():
    """Any leading dimensions, as many trees one by one."""
    parents = torch.tensor([[[-1, 0, 1], [-1, -1, -1]], [[-1, 0, 0], [-1, -1, 1]]])
    words = cb.tree_words(parents)
    assert tuple(words.shape) == (2, 2, 3, 1)
    for i in range(2):
        for j in range(2):
            assert torch.equal(words[i, j], cb.tree_words(parents[i, j]))
