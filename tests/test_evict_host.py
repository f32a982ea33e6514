"""Eviction's host side without a GPU."""
import contextlib
from types import SimpleNamespace

import pytest
import torch

import host_program
from paper_2609_32046_gb300 import binding
from test_budget_host import Spy, cache, receiver


def test_memory_comes_from_the_streams_own(monkeypatch):
    """What a call on a stream allocates is that stream's: another stream's next allocation would get the memory while
    the call still uses it."""
    names = {"pool": SimpleNamespace(cuda_stream=64), "default": SimpleNamespace(cuda_stream=0)}
    monkeypatch.setattr(torch.cuda, "Stream", SimpleNamespace)
    monkeypatch.setattr(torch.cuda, "stream", lambda s: ("on", s))
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle, device: ("external", handle, device))
    monkeypatch.setattr(torch.cuda, "default_stream", lambda device: names["default"])
    x = SimpleNamespace(device=torch.device("cuda", 3), is_cuda=True)
    for current in (0, 32, 64):
        monkeypatch.setattr(binding, "_raw_stream", lambda index, current=current: current)
        for stream, handle, want in ((names["pool"], 64, names["pool"]), (64, 64, ("external", 64, x.device)), (0, 0, names["default"])):
            got = binding._memory_for(stream, x)
            if handle == current:
                assert isinstance(got, contextlib.nullcontext)
            else:
                assert got == ("on", want)
        assert isinstance(binding._memory_for(None, x), contextlib.nullcontext)
        assert isinstance(binding._memory_for(64, torch.zeros(1)), contextlib.nullcontext)


@pytest.mark.parametrize("stream", [None, 64])
def test_evict_allocates_there(monkeypatch, stream):
    inside, made, empty = [], [], torch.empty

    @contextlib.contextmanager
    def memory_for(s, tensor):
        inside.append(s)
        yield
        inside.append("left")

    def allocate(*args, **kw):
        made.append(list(inside))
        return empty(*args, **kw)

    monkeypatch.setattr(binding, "_memory_for", memory_for)
    monkeypatch.setattr(binding, "_stream_on", lambda s, x: s or 0)
    monkeypatch.setattr(torch, "empty", allocate)
    caches, w = [cache(40), cache(30)], [torch.zeros(3, 2, 40)] * 2
    rx = receiver(Spy())
    idx = rx.evict(caches, w, 9, stream=stream)
    assert [tuple(x.shape) for x in idx] == [(3, 2, 9)] * 2 and made == [[stream]] * 2
    rx.evict(caches, w, 9, idx=idx, stream=stream)
    assert len(made) == 2


def test_what_one_part_reads_and_another_writes(tmp_path):
    """Parts (from, to, dense, of whom): found where both begin at one place, or both are dense and overlap, in any order."""
    cases = [([], [], 0), ([(0, 8, 1, 0)], [], 0), ([(0, 8, 1, 0), (8, 16, 1, 1)], [(0, 8, 1, 0), (8, 16, 1, 1)], 0),         # in place
             ([(0, 8, 1, 0), (8, 16, 1, 1)], [(8, 16, 1, 0), (0, 8, 1, 1)], 1),                                               # exchanged
             ([(0, 8, 1, 0), (8, 16, 1, 1)], [(40, 48, 1, 0), (20, 28, 1, 1)], 0),
             ([(0, 8, 1, 0), (8, 16, 1, 1)], [(20, 28, 1, 0), (0, 8, 0, 1)], 1),                                              # begins there
             ([(0, 8, 1, 0), (8, 16, 1, 1)], [(20, 28, 1, 0), (7, 9, 1, 1)], 1),
             ([(0, 8, 1, 0), (8, 16, 1, 1)], [(20, 28, 1, 0), (7, 9, 0, 1)], 0),                                              # between rows
             ([(0, 100, 0, 0), (10, 110, 0, 1)], [(20, 120, 0, 0), (30, 130, 0, 1)], 0),
             ([(0, 100, 1, 0)], [(0, 10, 1, 0), (10, 20, 1, 0), (50, 60, 1, 1), (200, 300, 1, 2)], 1),
             ([(0, 100, 1, 0)], [(90, 110, 1, 0), (100, 102, 0, 1), (110, 120, 1, 2)], 0),
             ([(100, 110, 1, 5)], [(0, 101, 1, 4)], 1), ([(100, 110, 1, 5)], [(0, 100, 1, 4), (110, 111, 1, 3)], 0)]
    part = lambda p: "cbk::PartOf{{%du, %du, %s}, %d}" % (p[0], p[1], "true" if p[2] else "false", p[3])       # noqa: E731
    body = "".join("std::printf(\"%%d\\n\", (int)cbk::read_and_written({%s}, {%s}));\n" % tuple(", ".join(map(part, x)) for x in (r, w))
                   for r, w, _ in cases)
    lines = host_program.run(tmp_path, "#include <cstdio>\n#include \"cb_ctx.cuh\"\nint main() {\n%sreturn 0; }\n" % body)
    assert [int(x) for x in lines] == [want for _, _, want in cases]


def test_weights_that_two_entries_share(tmp_path):
    """cb_evict's look over a call's entries: weights that one writes and another moves."""
    program = r"""
#include <cstdio>
#include "cb_receiver.cu"
int main() {
    // two entries: where the weights of each are read (-1: they do not move) and written, 100 bytes each
    const long long calls[][4] = {{0, 500, 100, 600}, {0, 0, 100, 100}, {0, 100, 100, 0}, {0, 500, 100, 0}, {0, 500, 100, 50}, {0, 500, -1, -1}};
    for (auto& c : calls) {
        Places p;
        for (int i = 0; i < 2; ++i) {
            if (c[2 * i] < 0) continue;
            const uintptr_t from = 1000 + c[2 * i], to = 1000 + c[2 * i + 1];
            p.weights.push_back(Written{to, to + 100, true});
            p.weights_to.push_back(PartOf{p.weights.back(), i});
            p.weights_from.push_back(PartOf{{from, from + 100, true}, i});
        }
        std::printf("%d\n", (int)p.clash());
    }
    return 0;
}
"""
    objects = ["cb_api", "cb_rotary", "cb_pack", "cb_attend", "cb_attend_tc", "cb_weigh", "cb_weigh_tc", "cb_evict", "cb_score", "cb_score_tc_0",
               "cb_score_tc_64", "cb_score_tc_128", "cb_select", "cb_compact", "cb_gather", "cb_rope", "cb_depage"]
    lines = host_program.run(tmp_path, program, objects)
    assert [int(x) for x in lines] == [0, 0, 1, 1, 1, 0]


def test_blocks_of_a_list(tmp_path):
    """k_rank's plan: as few blocks a list as hold its keys, however many lists there are; the form that does not hold them where
    eight blocks do not."""
    keys = 24 * 1024
    rows = sorted({0, 1, 2, 100, 16384, 200000, 8 * keys + 40} |
                  {c * keys + x for c in (1, 2, 4, 8) for x in (-5, -4, -3, -1, 0, 1, 2, 7)})
    program = r"""
#include <cstdio>
#include <cstring>
#include "cb_receiver.cuh"
int main() {
    static cbk::RankBatch b;
    for (int lists : {288, 76, 1})
        for (long long T : {%s}) {
            std::memset(&b, 0, sizeof b);
            b.n = 2;
            b.n_layers = 1;
            b.n_kv_heads = lists;
            b.s[1].T = T;
            const cbk::RankPlan p = cbk::rank_plan(b);
            std::printf("%%d %%lld %%d\n", p.blocks, (long long)p.slice, (int)p.held);
        }
    return 0;
}
""" % ", ".join("%dll" % T for T in rows)
    lines = iter(host_program.run(tmp_path, program, ["cb_evict"]))
    for lists in (288, 76, 1):
        for T in rows:
            blocks, part, held = map(int, next(lines).split())
            for n in {T, max(0, T - 1), max(0, T - 65)}:                    # inner rows: the kernel's slices hold them all
                assert (-(-n // blocks) + 3) // 4 * 4 <= part
            assert held == (part <= keys) and (held or blocks == 8)
            assert held == (T <= 8 * keys)
            assert blocks == next((c for c in (1, 2, 4) if T <= c * keys), 8)
