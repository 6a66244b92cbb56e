"""What the rotation-free 8-bit calls do once in a process: their first call inside a stream capture, and a wait that runs out (which stays in
the device's status word).  Each runs in a process of its own."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

FIRST_CALL_CAPTURED = """
import torch
import paper_2509_21302_b200 as q
M, K, N = {M}, 1024, 1536
x, r = torch.zeros(M, K, dtype=torch.bfloat16, device="cuda"), torch.zeros(M, K, dtype=torch.bfloat16, device="cuda")
gamma, w = torch.ones(K, device="cuda"), torch.randint(-127, 128, (N, K), dtype=torch.int8, device="cuda")
ws = torch.rand(N, device="cuda")
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    xq, a, h = q.rmsnorm_quantize_c8(x, gamma, 1e-6, r)
    y = q.linear_c8(xq, a, w, ws)
    yq, b = q.quantize_c8(y)
    v = q.dequantize_c8(yq, b)
    z = q.rmsnorm(v, torch.ones(N, device="cuda"))
for seed in range(2):
    torch.manual_seed(seed)
    x.normal_()
    r.normal_()
    graph.replay()
    want = q.rmsnorm_quantize_c8(x, gamma, 1e-6, r)
    y2 = q.linear_c8(want[0], want[1], w, ws)
    yq2, b2 = q.quantize_c8(y2)
    z2 = q.rmsnorm(q.dequantize_c8(yq2, b2), torch.ones(N, device="cuda"))
    assert all(torch.equal(s, t) for s, t in zip((xq, a, h, y, yq, b, z), want + (y2, yq2, b2, z2)))
    assert y.abs().max() > 0
assert q.linear_status() == 0
print("done")
"""

STARVED = """
import time
import torch
import paper_2509_21302_b200 as q
M, N, K = {M}, {N}, 1000
xq = torch.ones(M, 1008, dtype=torch.int8, device="cuda")[:, :K]
w = torch.ones(N, 1008, dtype=torch.int8, device="cuda")[:, :K]
a, ws, y = torch.ones(M, device="cuda"), torch.ones(N, device="cuda"), torch.zeros(M, N, dtype=torch.bfloat16, device="cuda")
assert torch.all(q.linear_c8(xq, a, w, ws) == K) and q.linear_status() == 0
began = time.time()
assert q.debug_starved_linear(xq, a, w, ws, y, 200000) == 0
code = q.linear_status()
assert 1 <= code <= 6, code
assert time.time() - began < 20
assert torch.all(q.linear_c8(xq, a, w, ws) == K)            # the context and its tensor memory are as they were
assert q.linear_status() == code                            # sticky
print("done")
"""


def _run(program):
    r = subprocess.run([sys.executable, "-c", program], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "done" in r.stdout, r.stdout + r.stderr


@pytest.mark.parametrize("M", [1, 24, 600])
def test_the_first_call_may_be_captured(M):
    _run(FIRST_CALL_CAPTURED.format(M=M))


@pytest.mark.parametrize("M,N", [(5, 300), (100, 128)])
def test_a_wait_that_runs_out_ends_the_launch(M, N):
    _run(STARVED.format(M=M, N=N))
