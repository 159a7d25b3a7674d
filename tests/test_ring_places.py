"""The norm join's walk through the places of its ring, on the CPU: the index
arithmetic of csrc/places.h, compiled for the host with checks for signed
overflow, at token counts up to the limit of the interface."""
import os
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_22922_gb300", "csrc")

# The ring as the kernels drive it: `stages` places filled at the start, a place
# filled again when its last token is done.  Every fill has to lie inside
# [t0, t1), and each token to be in exactly one.
WALK = r"""
#include <stdint.h>
#include <stdio.h>
#include <vector>
#include "places.h"

static int walk(int t0, int t1, int per, int stages) {
    std::vector<char> seen(t1 - t0, 0);
    auto fill = [&](int64_t t, int n) {
        if (n <= 0 || t < t0 || t + n > t1) return false;
        for (int i = 0; i < n; ++i)
            if (seen[t - t0 + i]++) return false;
        return true;
    };
    for (int i = 0; i < stages; ++i)
        if (const int n = ifvs::place_count(t0, t1, per, i))
            if (!fill((int64_t)t0 + i * per, n)) return 1;
    int first = t0;
    for (int t = t0; t < t1; ++t) {
        if (!seen[t - t0]) return 2;
        if (!ifvs::ends_place(t, first, t1, per)) continue;
        if (const int n = ifvs::place_count(first, t1, per, stages))
            if (!fill((int64_t)first + stages * per, n)) return 3;
        first = t + 1;
    }
    for (char c : seen)
        if (c != 1) return 4;
    return 0;
}

int main() {
    const int ends[] = {1, 40, 1000, 2147483647 - 20, 2147483647 - 1, 2147483647};
    for (int t1 : ends)
        for (int n = 0; n <= 60 && n <= t1; ++n)
            for (int per = 1; per <= 8; ++per)
                for (int stages = 1; stages <= 3; ++stages)
                    if (const int e = walk(t1 - n, t1, per, stages)) {
                        printf("tokens [%d, %d), %d a place, %d places: %d\n", t1 - n, t1, per, stages, e);
                        return 1;
                    }
    puts("ok");
    return 0;
}
"""


def test_every_fill_lies_inside_the_teams_tokens(tmp_path):
    src, exe = tmp_path / "walk.cpp", tmp_path / "walk"
    src.write_text(WALK)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-fsanitize=signed-integer-overflow", "-fno-sanitize-recover=all", "-I", CSRC,
                           "-o", str(exe), str(src)])
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout == "ok\n", r.stdout + r.stderr
