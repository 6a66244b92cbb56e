"""The row operators of the rotation-free 8-bit path over batches of any size: which launch takes them, how many rows a CTA of it works
through and how many are on their way ahead go by the number of rows, and must not show."""
import pytest
import torch

import paper_2509_21302_b200 as q

pytestmark = pytest.mark.gpu

TYPES = [torch.bfloat16, torch.float16, torch.float32]


def _matrix(M, K, dtype, seed, pad=0, shift=0):
    """Rows with a few large channels; `pad` elements between them, the first one `shift` elements into its memory."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = torch.full((shift + M * (K + pad),), 7.0, dtype=dtype, device="cuda")[shift:].view(M, K + pad)[:, :K]
    v = torch.randn(M, K, generator=g, device="cuda")
    v[:, torch.randint(K, (3,), generator=g, device="cuda")] *= 30.0
    t.copy_(v)
    return t


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pad,shift", [(0, 0), (3, 1)])
@pytest.mark.parametrize("K", [64, 100, 512, 1024, 1025, 1032, 1536, 1544, 2048, 2050, 4096, 5001, 8704, 16384, 16385, 20000, 32768, 32776])
def test_a_row_does_not_depend_on_the_batch(K, pad, shift, dtype):
    """Codes, scales, norms and sums are bit for bit those of the same rows in smaller batches."""
    M = 4200
    x, r = _matrix(M, K, dtype, K, pad, shift), _matrix(M, K, dtype, K + 1, pad, shift)
    gamma = torch.rand(K, generator=torch.Generator(device="cuda").manual_seed(K), device="cuda") + 0.5
    calls = (lambda s: q.quantize_c8(x[s]), lambda s: q.rmsnorm_quantize_c8(x[s], gamma, 1e-6), lambda s: q.rmsnorm_quantize_c8(x[s], gamma, 1e-6, r[s]),
             lambda s: (q.rmsnorm(x[s], gamma, 1e-6),), lambda s: q.rmsnorm(x[s], gamma, 1e-6, r[s]))
    for i, call in enumerate(calls):
        whole = call(slice(0, M))
        for part in (slice(0, 4096), slice(0, 4095), slice(100, 1100), slice(M - 3, M), slice(7, 8)):
            for w, p in zip(whole, call(part)):
                assert torch.equal(w[part], p), (i, part)
