"""The ring's places in csrc/kv_ring.cuh, run on the CPU through every run length: what is filled and taken, and
that a wait given up at any fill leaves no fill that is not waited for."""
import os
import subprocess
import tempfile

from conftest import ROOT

CSRC = os.path.join(ROOT, "paper_2608_02244_gb300", "csrc")
PROGRAM = r"""
#include "kv_ring.cuh"
#include <cstdio>
#include <vector>
#define CHECK(x) do { if (!(x)) { std::printf("line %d: total %d, given up at %d, at %d\n", __LINE__, total, quit, at); return false; } } while (0)

// fill number i goes to stage i % N in its turn i / N; the kernel's order of fills, waits and takes
template <int N>
bool run(int total, int quit) {
    isjl::RingPlace<N> place;
    std::vector<int> holds(N, -1);
    int filled = 0, at = 0;
    auto feed = [&](int stage) {
        if (filled == total) return true;
        CHECK(stage == filled % N && holds[stage] < at);      // in turn, over a fill that was taken
        holds[stage] = filled++;
        return true;
    };
    for (int i = 0; i < N - 1; ++i) if (!feed(i)) return false;
    for (; at < total; ++at) {
        if (!feed(place.before())) return false;
        CHECK(at < filled && place.stage == at % N && place.phase == (uint32_t)(at / N & 1));
        if (at == quit) {
            for (int k = place.under_way(total - at); k > 0; --k, ++at, place.take())
                CHECK(at < filled && holds[place.stage] == at && place.phase == (uint32_t)(at / N & 1));
            CHECK(at == filled);                              // nothing is left under way
            return true;
        }
        place.take();
    }
    CHECK(filled == total);
    return true;
}
template <int N>
bool all() {
    for (int total = 2; total <= 6 * N; total += 2)
        for (int quit = -1; quit < total; ++quit)
            if (!run<N>(total, quit)) return false;
    return true;
}
int main() { return all<2>() && all<3>() && all<4>() && all<6>() ? 0 : 1; }
"""


def test_fills_takes_and_giving_up():
    with tempfile.TemporaryDirectory() as d:
        src, exe = os.path.join(d, "ring.cpp"), os.path.join(d, "ring")
        open(src, "w").write(PROGRAM)
        subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-I", CSRC, src, "-o", exe], check=True)
        r = subprocess.run([exe], capture_output=True, text=True)
        assert r.returncode == 0, r.stdout
