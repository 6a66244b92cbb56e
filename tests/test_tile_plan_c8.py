"""The tiles of the 8-bit product at any number of rows and channels, on the CPU: every 64-channel unit of every row tile (the last of both
may reach beyond the matrix) is dealt to exactly one worker, inside the boxes and stages it was planned with, for every size that
can_plan() lets through."""
import os
import subprocess

import paper_2509_21302_b200 as q

CSRC = os.path.join(os.path.dirname(q.__file__), "csrc")
PROGRAM = r"""
#include <cstdio>
#include <vector>
#include "gemm_c8_plan.cuh"
using namespace gemm_c8;
#define CHECK(c) do { if (!(c)) { std::printf("%s: M %d N %d K %d workers %d\n", #c, M, N, K, W); return 1; } } while (0)
static int check(int M, int N, int K, int W)
{
    int workers = 0;
    CHECK(can_plan(M, N));
    const Plan p = make_plan(M, N, K, W, &workers);
    const long long rows = (M + 255LL) / 256, units = (N + 63LL) / 64;
    const bool resident = K > 896 && K <= 1024;
    std::vector<unsigned char> dealt((size_t)(rows * units));
    CHECK(workers >= 1 && workers <= W);
    CHECK(p.stages >= 2 && p.stages <= (resident ? RES_KB : MAX_STAGES));
    CHECK((resident ? RES_KB * A_BYTES : 0) + p.stages * p.stage_bytes <= OPS_BYTES);
    CHECK(p.wide * (UNIT / 2) <= 256 && p.cut * (UNIT / 2) <= 256);
    for (int w = 0; w < workers; ++w) {
        Tiles t(p, w);
        CHECK(t.count >= 1);
        for (int i = 0; i < t.count; ++i, t.next()) {
            const int box = i < p.runs * p.run + p.rounds ? p.wide : p.cut;
            CHECK(t.units >= 1 && t.units <= box && box <= MAX_UNITS && (resident ? 0 : A_BYTES) + box * UNIT_BYTES <= p.stage_bytes);
            CHECK(t.row >= 0 && t.row < rows && t.unit >= 0 && t.unit + t.units <= units);
            for (int u = 0; u < t.units; ++u) ++dealt[(size_t)(t.row * units + t.unit + u)];
        }
    }
    for (int d : dealt) CHECK(d == 1);
    return 0;
}
int main()
{
    unsigned long long r = 4711;
    auto below = [&](int n) { r = r * 6364136223846793005ull + 1442695040888963407ull; return (int)((r >> 33) % n); };
    for (int i = 0; i < 30000; ++i)
        if (check(1 + below(i % 2 ? 20000 : 2000), 1 + below(i % 3 ? 6000 : 300), 1 + below(i % 4 ? 1400 : 131056), below(3) ? 74 : 1 + below(100))) return 1;
    if (check(2147483392, 64, 16, 74) || check(2147483392, 5, 1024, 74) || check(1, 40000000, 16, 74) || check(300, 8000000, 1000, 74) || check(70000001, 300, 64, 74)) return 1;
    int M = 1, N = 2147483647, K = 1, W = 1;
    CHECK(!can_plan(M, N) && !can_plan(2147483392, 2000000) && can_plan(2147483392, 10000) && can_plan(1, 60000000));
    return 0;
}
"""


def test_every_unit_is_dealt_once(tmp_path):
    (tmp_path / "plan.cpp").write_text(PROGRAM)
    subprocess.check_call([os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-I", CSRC, "-o", str(tmp_path / "plan"), str(tmp_path / "plan.cpp")])
    r = subprocess.run([str(tmp_path / "plan")], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout
