"""How a product of 8-bit matrices is cut into tiles (csrc/matmul_plan.h, the library's own code, compiled for the host): what
the kernel needs of every plan, over sizes from the smallest to the largest and devices of several kinds, and that clusters
which the device does not run are never asked for. And the query of the form on the C ABI."""
import ctypes
import os
import shutil
import subprocess

import pytest

from paper_2401_13660_gb300 import mbscan as mb

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include <cstdio>
#include <cstdlib>
#include "matmul_plan.h"
using namespace mbscan;

static void fail(const char *what, long rows, long n, long width, int bf16) {
    std::printf("%s: %ld x %ld x %ld, bf16 %d\n", what, rows, width, n, bf16);
    std::exit(1);
}

int main(int argc, char **argv) {
    // SMs; clusters of 2, 4 and 8 that fit
    const int sms = std::atoi(argv[1]), fit[9] = {0, sms, std::atoi(argv[2]), 0, std::atoi(argv[3]), 0, 0, 0, std::atoi(argv[4])};
    const MatmulLimits lim{sms, 228 * 1024, 1024, 227 * 1024};
    const size_t least = lim.smem_sm / 3 + lim.smem_reserved;   // what a CTA takes of an SM at the least
    long seen[3] = {0, 0, 0};
    for (long rows = 1; rows < 300000; rows += rows < 300 ? 1 : rows / 7)
        for (long n = 8; n < 150000; n += n < 264 ? 8 : n / 40 * 8)
            for (long width = 16; width < 40000; width += width < 640 ? 112 : width / 64 * 16)
                for (int bf16 = 0; bf16 < 2; ++bf16) {
                    if (rows * n > 1l << 31 || n * width > 1l << 31 || rows * width > 1l << 31) continue;
                    const MatmulPlan p = plan_matmul(rows, n, width, bf16, lim, [&](int size) { return fit[size]; });
                    const Tiles &t = p.t;
                    const long wide = kFeatures * p.ctas, tiles = (long)t.features * t.rows;
                    if ((long)t.features * wide < n || (long)t.rows * t.height < rows) fail("not covered", rows, n, width, bf16);
                    if (t.height % (rows <= 16 ? 16 : kChunk) || t.height > kMaxRows || t.height % t.split) fail("height", rows, n, width, bf16);
                    if (p.ctas == 2 && (t.split != 1 || t.deep != 1)) fail("pair", rows, n, width, bf16);
                    if (t.split > 2 && fit[t.split] <= 0) fail("clusters that the device does not run", rows, n, width, bf16);
                    if (p.team != (p.ctas == 2 ? 2 : t.split) || p.teams * p.team > lim.sms) fail("more CTAs than SMs", rows, n, width, bf16);
                    if (t.sums == 1 ? p.teams != tiles : t.split != 1 || p.teams >= tiles) fail("tiles of a CTA", rows, n, width, bf16);
                    // every part of a sum has blocks: whole stages
                    if ((t.blocks + t.deep - 1) / t.deep < t.split) fail("an empty part", rows, n, width, bf16);
                    if (t.stages < 1 || t.stages > kMaxStages) fail("stages", rows, n, width, bf16);
                    const size_t stage = (size_t)t.deep * (kFeatures + t.height / p.ctas) * kK;
                    const size_t chunks = (size_t)kGroups * t.held * kChunk * kFeatures * (bf16 ? 2 : 4);
                    if (t.ring < t.stages * stage || t.ring % 1024) fail("ring", rows, n, width, bf16);
                    if (t.sums == 1 && (t.ring < chunks || (t.split > 1 && t.ring < (size_t)t.height * kFeatures * 4)))
                        fail("room where the ring was", rows, n, width, bf16);
                    if (1024 + t.ring + kSlots * kSlotBytes + (t.sums == 1 ? 0 : chunks) > p.smem) fail("shared memory", rows, n, width, bf16);
                    if (p.smem + kBarrierBytes > lim.smem_optin) fail("more shared memory than there is", rows, n, width, bf16);
                    if ((int)t.columns < t.sums * t.height + 2 * kScaleColumns || (t.columns & (t.columns - 1)) || t.columns > 512)
                        fail("columns of tensor memory", rows, n, width, bf16);
                    // two CTAs to an SM, of any two products, have their columns at once; three never fit
                    if (p.smem + lim.smem_reserved + least <= lim.smem_sm && t.columns > 256) fail("waits for columns", rows, n, width, bf16);
                    if (3 * (p.smem + lim.smem_reserved) <= lim.smem_sm) fail("three to an SM", rows, n, width, bf16);
                    ++seen[p.ctas == 2 ? 2 : t.split > 1];
                }
    if (sms > 16 && (!seen[0] || !seen[1] || !seen[2])) fail("a form that is never taken", seen[0], seen[1], seen[2], 0);
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    if not shutil.which("g++"):
        pytest.skip("no g++")
    d = tmp_path_factory.mktemp("plan")
    (d / "plan.cpp").write_text(PROGRAM)
    subprocess.run(["g++", "-O2", "-std=c++17", "-I", os.path.join(ROOT, "paper_2401_13660_gb300", "csrc"),
                    str(d / "plan.cpp"), "-o", str(d / "plan")], check=True)
    return str(d / "plan")


@pytest.mark.parametrize("device", [(152, 76, 36, 16), (152, 76, 38, 19), (148, 74, 34, 15), (152, 76, 36, 0), (152, 76, 0, 0), (16, 8, 4, 2)],
                         ids=str)
def test_plans(program, device):
    r = subprocess.run([program, *map(str, device)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout


def test_form_refuses_what_the_product_refuses():
    lib, form = mb.load_library(), (ctypes.c_int64 * 5)(*[7] * 5)
    for (rows, n, width, dtype), want in (((-1, 8, 16, 1), mb.MB_ERR_INVALID_ARG), ((1, 8, 24, 1), mb.MB_ERR_UNSUPPORTED),
                                          ((1, 12, 16, 1), mb.MB_ERR_UNSUPPORTED), ((1, 8, 16, 2), mb.MB_ERR_INVALID_ARG),
                                          ((1 << 28, 16, 16, 0), mb.MB_ERR_INVALID_ARG), ((1, 1 << 28, 16, 0), mb.MB_ERR_INVALID_ARG)):
        assert lib.mb_matmul_q8_form(rows, n, width, dtype, form) == want and list(form) == [7] * 5
    assert lib.mb_matmul_q8_form(1, 8, 16, 1, None) == mb.MB_ERR_INVALID_ARG
    for sizes in ((0, 8, 16), (3, 0, 16), (3, 8, 0)):
        assert set(mb.mb_matmul_q8_form(*sizes).values()) == {0}
