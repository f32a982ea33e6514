"""cb_attend's host side without a GPU: how much work a launch is planned for."""
import host_program

SHAPES = [(1, 1, 4, 8, 16384), (1, 1024, 4, 8, 16384), (8, 64, 4, 8, 12352), (16, 32, 4, 2, 3), (64, 1024, 1, 1, 0),
          (1, 17, 4, 1, 2 ** 31 - 4096)]                       # sequences, tokens, group, KV heads, rows
WINDOWS = [0, 1, 1000, 2 ** 31, 2 ** 32, 2 ** 62, 2 ** 63 - 1 - 1024, 2 ** 63 - 1]
TILES = [16, 256]

PROGRAM = r"""
#include <cstdio>
#include <cstring>
#include "cb_attend.cuh"
int main() {
    const long long shapes[][5] = {%s};
    const long long windows[] = {%s};
    const int tiles[] = {%s};
    static cbk::AttendBatch b;
    for (auto& s : shapes)
        for (long long w : windows)
            for (int t : tiles) {
                std::memset(&b, 0, sizeof b);
                b.n = (int)s[0];
                b.G = (int)s[2];
                b.n_kv_heads = (int)s[3];
                b.causal = 1;
                b.window = w;
                for (int i = 0; i < b.n; ++i) {
                    b.span[i].m = (int)s[1];
                    b.span[i].T = s[4];
                }
                const long long units = cbk::attend_pairs(b, t);
                std::printf("%%lld %%lld %%d\n", units, (long long)b.window, b.pairs);
            }
    return 0;
}
"""


def test_a_window_of_any_size_is_planned_for(tmp_path):
    """Units of 128 positions that a launch may have: never fewer than the tiles have, whatever the window is (a
    grid that is larger than the scratch would follow from a count below zero), and windows that reach past
    everything are all alike."""
    program = PROGRAM % (", ".join("{%s}" % ", ".join("%dll" % x for x in s) for s in SHAPES),
                         ", ".join("%dll" % w for w in WINDOWS), ", ".join(map(str, TILES)))
    lines = iter(host_program.run(tmp_path, program, ["cb_attend", "cb_attend_tc"]))
    for n, m, G, Hkv, T in SHAPES:
        for w in WINDOWS:
            for tile in TILES:
                units, window, pairs = map(int, next(lines).split())
                tiles = -(-m * G // tile)
                reach = min(T, w + m) if w else T
                assert pairs == n * tiles
                assert units == n * tiles * Hkv * (reach // 128 + 2)
                # what the kernels compute with: no sum or difference of it, rows and tokens leaves 64 bits
                assert window == w or T + m <= window <= min(w, 2 ** 40)


def test_what_two_parts_of_a_call_write(tmp_path):
    """Parts that begin at the same place or overlap densely are found, in any order; slices beside one another are not."""
    cases = [([], 0), ([(0, 8, 1)], 0), ([(0, 8, 1), (8, 16, 1), (16, 24, 1)], 0), ([(16, 24, 1), (8, 16, 1), (0, 8, 1)], 0),
             ([(0, 8, 1), (0, 8, 1)], 1), ([(8, 16, 1), (0, 9, 1)], 1), ([(0, 100, 1), (200, 300, 1), (99, 120, 1)], 1),
             ([(0, 100, 0), (10, 110, 0), (20, 120, 0)], 0),               # heads of one array, interleaved
             ([(0, 100, 0), (10, 110, 0), (0, 100, 0)], 1), ([(0, 100, 0), (50, 60, 1)], 0),
             ([(0, 100, 1), (40, 60, 0), (90, 95, 1)], 1)]
    body = "".join("{ std::vector<cbk::Written> w = {%s}; std::printf(\"%%d\\n\", (int)cbk::written_twice(w)); }\n" %
                   ", ".join("{%du, %du, %s}" % (a, b, "true" if c else "false") for a, b, c in w) for w, _ in cases)
    lines = host_program.run(tmp_path, "#include <cstdio>\n#include \"cb_ctx.cuh\"\nint main() {\n%sreturn 0; }\n" % body)
    assert [int(x) for x in lines] == [want for _, want in cases]
