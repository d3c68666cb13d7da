"""The line of work of prompts' attention (csrc/kv_prompt_line.cuh), on the host: sums of tiles against counting them,
and that every visible tile of an item is on the line once."""
import os
import subprocess

from conftest import ROOT

PROG = r"""
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <vector>
#include "kv_prompt_line.cuh"
using namespace isjl;
static uint32_t state = 12345;
static uint32_t rnd(uint32_t n) { state = state * 1664525u + 1013904223u; return (uint32_t)(((uint64_t)(state >> 4) * n) >> 28); }
static uint32_t size(int bits) { return rnd(1u << (1 + rnd(bits))); }
int main() {
    for (int t = 0; t < 200000; ++t) {
        const uint32_t n = size(6), m = 1 + size(8), a = size(9), b = size(12);
        int64_t want = 0;
        for (uint32_t i = 0; i < n; ++i) want += (a * i + b) / m;
        if (line_sum(n, m, a, b) != want) { printf("line_sum %u %u %u %u\n", n, m, a, b); return 1; }
    }
    long checked = 0;
    for (int t = 0; t < 3000; ++t) {
        PromptShape s;
        s.keys = rnd(2) ? 128 : 64;
        const int group = 1 + rnd(rnd(2) ? 8 : 130), rows = group < 128 ? group : 128;
        s.step = (s.keys == 128 ? 2 : 1) * (128 / rows);
        s.window = rnd(2) ? 0 : 1 + size(12);
        s.sinks = s.window && rnd(2) ? size(9) : 0;
        s.extra = rnd(2) ? 0 : rnd(6);
        PromptRow r;
        r.count = 1 + size(11);
        r.first = rnd(2) ? 0 : size(13);
        int64_t sum = 0;
        for (int p = 0; p < r.items(s); ++p) {
            if (r.before(s, p) != sum) { printf("before %d: %ld, not %ld\n", p, (long)r.before(s, p), (long)sum); return 1; }
            // tiles that some query of the item sees
            const int q0 = r.first + p * s.step, q1 = r.end(s, p);
            std::vector<int> want, got;
            for (int y = 0; y * s.keys < q1; ++y) {
                bool seen = false;
                for (int x = y * s.keys; x < (y + 1) * s.keys && !seen; ++x)
                    for (int q = q0; q < q1 && !seen; ++q) seen = x <= q && (!s.window || x > q - s.window || x < s.sinks);
                if (seen) want.push_back(y);
            }
            for (int j = 0; j < r.tiles(s, p); ++j) got.push_back(PromptRow::tile(s, r.skip(s, p), j));
            // the line may hold tiles between the two parts that nobody sees, never lack one or have one twice
            size_t at = 0;
            for (size_t i = 0; i < got.size(); ++i) {
                if (i && got[i] <= got[i - 1]) { printf("order\n"); return 1; }
                if (at < want.size() && got[i] == want[at]) ++at;
            }
            if (at != want.size() || got.back() != want.back()) { printf("lacks a tile\n"); return 1; }
            if (got.size() > want.size() + 1) { printf("%zu tiles for %zu\n", got.size(), want.size()); return 1; }
            sum += s.extra + r.tiles(s, p);
            ++checked;
        }
        if (r.before(s, r.items(s)) != sum) { printf("all\n"); return 1; }
    }
    // the largest numbers: no sum wraps
    PromptShape s = {128, 256, 0, 0, 3};
    PromptRow r = {2147483647 - 255 - 5, 5};
    int64_t want = 0;
    for (int p = 0; p < r.items(s); ++p) want += s.extra + r.tiles(s, p);
    if (r.before(s, r.items(s)) != want) { printf("largest %ld %ld\n", (long)r.before(s, r.items(s)), (long)want); return 1; }
    s.window = 70000; s.sinks = 1000; want = 0;
    for (int p = 0; p < r.items(s); ++p) want += s.extra + r.tiles(s, p);
    if (r.before(s, r.items(s)) != want) { printf("largest with a window\n"); return 1; }
    r.first = 2147483647 - 255 - 1000; r.count = 1000; s.window = 2147483647 - 300; s.step = 2; want = 0;
    for (int p = 0; p < r.items(s); ++p) want += s.extra + r.tiles(s, p);
    if (r.before(s, r.items(s)) != want) { printf("largest place\n"); return 1; }
    printf("checked\n");
    return checked > 10000 ? 0 : 1;
}
"""


def test_line(tmp_path):
    src, exe = tmp_path / "line.cpp", tmp_path / "line"
    src.write_text(PROG)
    subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", "-Werror", "-fsanitize=undefined", "-fno-sanitize-recover",
                    "-I", os.path.join(ROOT, "paper_2608_02244_gb300", "csrc"), str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True)
    assert out.returncode == 0 and out.stdout == "checked\n", out.stdout + out.stderr
