"""The mapping from a running number to a product's tile (csrc/worker_tiles.cuh), compiled for the host: every tile
once, none that does not exist, up to the most columns that the entry points accept."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include <cstdio>
#include <cstdlib>
#include <vector>
#include "worker_tiles.cuh"
using namespace gar::worker;

template <bool OUTER> bool whole(int mt, int nt, int splits, int steps) {
    const Tiling a{mt, nt, splits, OUTER ? 1 : group_rows(steps, mt), steps};
    if (a.group_m < 1 || a.group_m > mt) return false;
    const unsigned tiles = unsigned(mt) * unsigned(nt) * unsigned(splits);
    std::vector<bool> seen(tiles);
    std::vector<int> covered(splits);
    for (unsigned i = 0; i < tiles; ++i) {
        const Place t = place_in<OUTER>(a, i);
        if (t.m < 0 || t.m >= mt || t.n < 0 || t.n >= nt || t.split < 0 || t.split >= splits) return false;
        const size_t at = (size_t(t.split) * mt + t.m) * nt + t.n;
        if (seen[at]) return false;
        seen[at] = true;
        // a part's steps: all of them for a worker, otherwise one after the other up to the last
        if (OUTER || splits == 1) {
            if (t.first != 0 || t.steps != steps) return false;
        } else {
            if (t.steps < 1 || t.first + t.steps > steps) return false;
            covered[t.split] = t.steps;
        }
    }
    int sum = 0;
    for (int c : covered) sum += c;
    return OUTER || splits == 1 || sum == steps;
}

int main() {
    int bad = 0;
    auto say = [&](bool ok, const char* what, int mt, int nt, int splits, int steps) {
        if (!ok) { std::printf("%s %d %d %d %d\n", what, mt, nt, splits, steps); ++bad; }
    };
    const int counts[] = {1, 2, 3, 7, 8, 9, 33, 74};
    for (int mt : counts) for (int nt : counts) for (int steps : {1, 2, 8, 127, 128, 129, 1000, 1 << 25}) {
        say(whole<false>(mt, nt, 1, steps), "plain", mt, nt, 1, steps);
        say(whole<true>(mt, nt, 5, steps), "outer", mt, nt, 5, steps);
        for (int best : {2, 3, 16}) {
            const int part = (steps + best - 1) / best, splits = (steps + part - 1) / part;      // no part is empty
            say(whole<false>(mt, nt, splits, steps), "split", mt, nt, splits, steps);
        }
    }
    // one step of the contraction, 2^22 column tiles and more: 2^30 columns of 256, the most there are of 128 and 64
    for (int nt : {(1 << 22) - 1, 1 << 22, (1 << 22) + 1, 1 << 23, 1 << 24, 1 << 25}) say(whole<false>(1, nt, 1, 1), "wide", 1, nt, 1, 1);
    say(whole<false>(3, 1 << 22, 1, 1), "wide", 3, 1 << 22, 1, 1);
    say(whole<false>(1025, 4099, 1, 1), "tall", 1025, 4099, 1, 1);
    return bad != 0;
}
"""


def test_every_tile_once(tmp_path):
    src = tmp_path / "tiles.cpp"
    src.write_text(PROGRAM)
    exe = tmp_path / "tiles"
    subprocess.check_call(["g++", "-std=c++17", "-O2", "-I" + os.path.join(ROOT, "paper_1905_04374_b200", "csrc"), str(src), "-o", str(exe)])
    done = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300)
    assert done.returncode == 0, done.stdout[-2000:]
