"""The product's last channels, on the CPU: which groups of four results are stored at once, for every number of channels that an int holds."""
import os
import subprocess

import paper_2509_21302_b200 as q

CSRC = os.path.join(os.path.dirname(q.__file__), "csrc")
PROGRAM = r"""
#include <cstdio>
#include "gemm_c8_plan.cuh"
#include "linear_plan.cuh"
using namespace linear_plan;
int main()
{
    Split beyond = {};      // the sizes of test_gpu_linear_wide.py: meant for the tiles kernel, beyond what it counts with
    if (choose(40, 67200003, 17, 148, &beyond) != TILES || gemm_c8::can_plan(40, 67200003)) { std::printf("not beyond the tiles kernel\n"); return 1; }
    for (long long N = 1; N <= 2147483647LL; N += N == 600 ? 2147483647LL - 1200 : 1) {
        Split s = {};
        if (N > 600 && choose(8, (int)N, 1, 148, &s) != SPLIT) { std::printf("N %lld: another kernel\n", N); return 1; }
        const long long last = (N - 1) / CH * CH;                    // the first channel of the last tile
        for (long long n = last > CH ? last - CH : 0; n < N; n += 4) // as a lane has them, from its first channel that exists
            if (four_channels((int)n, (int)N) != (n + 3 < N)) { std::printf("N %lld n %lld\n", N, n); return 1; }
    }
    return 0;
}
"""


def test_four_results_are_stored_where_four_exist(tmp_path):
    """A lane of the split kernel has four channels and stores their results at once where all of them exist.  Near 2^31 the number behind the last of
    them is no int: N = 2147483645 once let the lane store four results where one exists."""
    (tmp_path / "edges.cpp").write_text(PROGRAM)
    # -fwrapv: an overflow gives a wrong answer here, not anything
    subprocess.check_call([os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-Wall", "-fwrapv", "-I", CSRC, "-o", str(tmp_path / "edges"), str(tmp_path / "edges.cpp")])
    r = subprocess.run([str(tmp_path / "edges")], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout
