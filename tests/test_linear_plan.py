"""How a product of 8-bit codes is cut up, on the CPU: for many sizes the split kernel's tiles cover the tokens and channels once, within
what its launch and instructions take, and the sizes that the comment's figures were measured at go where they say."""
import os
import subprocess

import paper_2509_21302_b200 as q

CSRC = os.path.join(os.path.dirname(q.__file__), "csrc")
PROGRAM = r"""
#include <cstdio>
#include "linear_plan.cuh"
using namespace linear_plan;
#define CHECK(c) do { if (!(c)) { std::printf("%s: M %d N %d K %d sms %d\n", #c, M, N, K, sms); return 1; } } while (0)
static int check(int M, int N, int K, int sms)
{
    Split s = {};
    if (choose(M, N, K, sms, &s) != SPLIT) return 0;
    const int KB = (K + 127) / 128;
    CHECK(s.split == 1 || s.split == 2 || s.split == 4 || s.split == 8);
    CHECK(s.split <= KB);
    CHECK(s.tok >= 16 && s.tok <= MAX_TOK && s.tok % 16 == 0);
    CHECK((long long)s.tok * s.row_tiles >= M && (long long)s.tok * (s.row_tiles - 1) < M);      // no tile is empty
    CHECK(s.tiles * CH >= N && (s.tiles - 1) * CH < N);
    CHECK(s.row_tiles >= 1 && s.row_tiles <= 65535 && s.tiles * s.split <= 2147483647LL);
    CHECK(s.us > 0.0f);
    return 0;
}
int main()
{
    unsigned long long r = 99;
    auto below = [&](int n) { r = r * 6364136223846793005ull + 1442695040888963407ull; return (int)((r >> 33) % n); };
    for (int i = 0; i < 300000; ++i)
        if (check(1 + below(i % 2 ? 40 : 600), 1 + below(i % 3 ? 9000 : 200000), 1 + below(i % 5 ? 9000 : 131056), below(3) ? 148 : 1 + below(200))) return 1;
    int M = 1, N = 2147483647, K = 131056, sms = 148;
    if (check(M, N, K, sms) || check(512, N, 1, sms) || check(1, 1, 1, sms)) return 1;
    Split s = {};
    CHECK(choose(1, 1024, 1024, sms, &s) == TOKEN);
    CHECK(choose(1, 4096, 16384, sms, &s) == TOKEN && choose(2, 4096, 16384, sms, &s) == SPLIT);
    CHECK(choose(4, 4096, 4096, sms, &s) == TOKEN && choose(5, 4096, 4096, sms, &s) == SPLIT);
    CHECK(choose(1, 200000, 64, sms, &s) == SPLIT);
    CHECK(choose(8, 1024, 1024, sms, &s) == FEW);
    CHECK(choose(8, 1, 131056, sms, &s) == SPLIT);
    CHECK(choose(16, 1024, 1024, sms, &s) == SPLIT);
    CHECK(choose(128, 1024, 1024, sms, &s) == TILES);
    CHECK(choose(8, 4096, 4096, sms, &s) == SPLIT && s.split == 4);
    CHECK(choose(64, 4096, 4096, sms, &s) == SPLIT);
    CHECK(choose(128, 16384, 4096, sms, &s) == TILES);
    CHECK(choose(256, 1024, 4096, sms, &s) == SPLIT && s.tok < 256);
    CHECK(choose(2147483392, 4096, 4096, sms, &s) == TILES);
    return 0;
}
"""


def test_the_tiles_cover_the_product(tmp_path):
    (tmp_path / "plan.cpp").write_text(PROGRAM)
    subprocess.check_call([os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-Wall", "-I", CSRC, "-o", str(tmp_path / "plan"), str(tmp_path / "plan.cpp")])
    r = subprocess.run([str(tmp_path / "plan")], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout
