"""The product of 8-bit codes with more channels than the kernel for large products counts with: another one takes it, in tiles of 32 rows."""
import pytest
import torch

import paper_2509_21302_b200 as q

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_tens_of_millions_of_channels(dtype):
    """Two tiles of rows, the second ragged; K and N end inside their pieces; 2.7e9 results, over 2^31.  One fp32 rounding is U."""
    M, N, K = 40, 67200003, 17
    g = torch.Generator(device="cuda").manual_seed(5)
    xq = torch.randint(-128, 128, (M, 32), generator=g, device="cuda", dtype=torch.int8)[:, :K]
    wq = torch.empty(N, 32, device="cuda", dtype=torch.int8)
    for n in range(0, N, 1 << 24):
        wq[n:n + (1 << 24)] = torch.randint(-128, 128, wq[n:n + (1 << 24)].shape, generator=g, device="cuda", dtype=torch.int8)
    wq = wq[:, :K]
    a, w = torch.rand(M, generator=g, device="cuda") * 0.01 + 0.001, torch.rand(N, generator=g, device="cuda") * 0.01 + 0.001
    b = torch.randn(N, generator=g, device="cuda").to(dtype)
    y = q.linear_c8(xq, a, wq, w, b, dtype)
    assert y.shape == (M, N) and y.dtype == dtype
    half, tiny = torch.finfo(dtype).eps / 2, torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps
    for n in range(0, N, 1 << 21):
        s = slice(n, n + (1 << 21))
        p = (xq.double() @ wq[s].double().t()) * (a.double()[:, None] * w[s].double())
        z = p + b[s].double()
        # the conversion of the sum (below 2^24: exact) and the product of the scales: at most 2 U of p; the multiply-add: U of z; the type: half of z
        bound = (2 * U + 2 * U * U) * p.abs() * (1 + half) + (U + half + U * half) * z.abs() + tiny
        assert torch.all((y[:, s].double() - z).abs() <= bound), n
    assert q.linear_status() == 0
