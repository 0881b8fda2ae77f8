"""How the embedding's gradient finds the pieces that a run of equal tokens spans
(csrc/runs.h, the kernel's own code, compiled for the host): the right ones, for
every piece that a CTA goes over, without a key looked up outside the tokens.
The key lookup of the host program ends it at the first index out of range."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>
#include "runs.h"

struct Warp {
    template <typename F> unsigned operator()(const F &f) const {
        unsigned v = 0;
        for (int lane = 0; lane < 32; ++lane) v |= (unsigned)f(lane) << lane;
        return v;
    }
    template <typename F, typename G> void operator()(const F &f, const G &g, unsigned &b, unsigned &c) const {
        b = (*this)(f);
        c = (*this)(g);
    }
};

static void check(const std::vector<int> &keys, int piece, int per_cta) {
    const int64_t n = (int64_t)keys.size(), pieces = (n + piece - 1) / piece;
    const auto key = [&](int64_t i) {
        if (i < 0 || i >= n) {
            std::printf("key %lld of %lld looked up: pieces of %d, %d to a CTA\n", (long long)i, (long long)n, piece, per_cta);
            std::exit(1);
        }
        return keys[i];
    };
    for (int64_t p = 0; p < (pieces + per_cta - 1) / per_cta * per_cta; ++p) {
        const mbscan::RunEnds r = mbscan::run_ends(Warp{}, key, n, piece, pieces, p);
        if (p >= pieces) continue;   // nothing there
        const int64_t q0 = p * piece, q1 = q0 + piece < n ? q0 + piece : n;
        int64_t begin = p, end = p;
        for (int64_t i = q0; i > 0 && keys[i - 1] == keys[q0]; --i) begin = (i - 1) / piece;
        for (int64_t i = q1; i < n && keys[i] == keys[q1 - 1]; ++i) end = i / piece;
        if (r.begin != begin || r.end != end) {
            std::printf("piece %lld of %lld: [%lld, %lld], not [%lld, %lld]\n", (long long)p, (long long)pieces,
                        (long long)r.begin, (long long)r.end, (long long)begin, (long long)end);
            std::exit(1);
        }
    }
}

int main(int argc, char **argv) {
    const int per_cta = std::atoi(argv[1]);
    std::mt19937 g(7);
    for (int n : {1, 2, 15, 16, 17, 63, 64, 65, 1000, 1024, 1025, 4099, 20000})
        for (int piece : {16, 17, 100, 320})
            for (int kind = 0; kind < 6; ++kind) {
                std::vector<int> keys;
                for (int i = 0, k = 0; i < n; ++i) {
                    keys.push_back(kind == 0 ? 0 : kind == 1 ? 300 : kind == 2 ? i : kind == 3 ? (i >= n / 2) * 9 : k);
                    k += kind == 4 ? g() % 3 == 0 : g() % 700 == 0;
                }
                check(keys, piece, per_cta);
            }
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    if not shutil.which("g++"):
        pytest.skip("no g++")
    d = tmp_path_factory.mktemp("runs")
    (d / "runs.cpp").write_text(PROGRAM)
    subprocess.run(["g++", "-O1", "-std=c++17", "-I", os.path.join(ROOT, "paper_2401_13660_gb300", "csrc"),
                    str(d / "runs.cpp"), "-o", str(d / "runs")], check=True)
    return str(d / "runs")


@pytest.mark.parametrize("per_cta", [1, 2, 4, 8, 16, 32, 64])
def test_runs_are_found_within_the_tokens(program, per_cta):
    r = subprocess.run([program, str(per_cta)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout
