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


U = 2.0 ** -24          # one fp32 rounding, relative to the value
# fp32 roundings in a norm: the sum h (1), two products (2), and 1 / sqrt: itself (at most 2 units in the last place: 4) and half of what its
# argument is off by: squares of rounded sums 2, at most 40 additions on the way of a term to the total, 1 / K, the multiply-add with it.
# 1 + 2 + 4 + 44 / 2 = 29.
NORM_REL = 29 * U


def _rows_for(K, turns):
    """Rows enough that CTAs work through `turns` of them (16-bit types; fp32: two at most), and some more, so that the last CTA, and the last
    warp where a warp takes several rows, has fewer."""
    chunks = (K + 7) // 8
    if chunks <= 64:
        lanes = 8 if chunks <= 8 else 16 if chunks <= 16 else 32
        ctas_per_sm, rows_per_cta = 4, 256 // lanes
    else:
        threads = (chunks + 63) // 64 * 32 if chunks <= 128 else (chunks + 127) // 128 * 32
        ctas_per_sm, rows_per_cta = 1024 // threads, 1
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    return turns * turns * sms * ctas_per_sm * rows_per_cta + 13


def _out(M, K, dtype, off):
    """A matrix for results: rows as the library makes them, or off every wide boundary with known values between and around them."""
    if not off:
        return None, None
    t = torch.full((1 + M * (K + 3),), 3, dtype=dtype, device="cuda")
    return t, t[1:].view(M, K + 3)[:, :K]


def _untouched(t, K):
    if t is not None:
        assert t[0] == 3 and (t[1:].view(-1, K + 3)[:, K:] == 3).all()


@pytest.mark.parametrize("dtype,turns", [(torch.bfloat16, 2), (torch.bfloat16, 4), (torch.bfloat16, 8), (torch.float16, 4), (torch.float32, 2)])
@pytest.mark.parametrize("off", [False, True])
@pytest.mark.parametrize("K", [64, 61, 125, 200, 500, 1024, 1029, 1032, 4096, 4104, 16384, 20001])
def test_every_row_of_long_batches(K, off, dtype, turns):
    """Every launch of the row operators where its CTAs take several rows, with copies of the next ones on their way; inputs and outputs on 16-byte
    boundaries, or off them.  Every row against the definition in 64 bits."""
    M = _rows_for(K, turns)
    pad, shift = (3, 1) if off else (-K % 8, 0)
    x, r = _matrix(M, K, dtype, K, pad, shift), _matrix(M, K, dtype, K + turns, pad, shift)
    gamma = torch.rand(K, generator=torch.Generator(device="cuda").manual_seed(K), device="cuda") + 0.5
    half, tiny = torch.finfo(dtype).eps / 2, torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps

    def slices():
        step = max(1, (1 << 25) // K)
        return [slice(m, min(M, m + step)) for m in range(0, M, step)]

    def check_codes(codes, scale, y, slack, rel):
        amax = y.abs().amax(1).clamp_min(1e-8)
        assert torch.all((scale.double() - amax / 127).abs() <= (rel + U) * amax / 127)
        off_by = (codes.double() - y * (127 / amax)[:, None]).abs()
        assert torch.all(off_by <= 0.5 + slack), float(off_by.max())
        assert codes.min() >= -127

    t, o = _out(M, K, torch.int8, off)
    codes, scale = q.quantize_c8(x, o)
    _untouched(t, K)
    for s in slices():
        f = x[s].float()
        amax = f.abs().amax(1, keepdim=True).clamp_min(1e-8)
        assert torch.equal(codes[s], (f * (amax.reciprocal() * 127.0)).round().to(torch.int8))        # the formula in fp32, bit for bit
        # the reciprocal of amax, 127 times it and the product with that are rounded: positions up to 127 are off by 3 * 127 U (and their products)
        check_codes(codes[s], scale[s], x[s].double(), 127 * 3.1 * U, 0.0)
    del codes, t, o
    for residual in (None, r):
        (ty, oy), (th, oh) = _out(M, K, dtype, off), _out(M, K, dtype, off)
        if not off and residual is None:
            oh = torch.empty_like(x)
        y, h = q.rmsnorm(x, gamma, 1e-6, residual, oy, oh)
        _untouched(ty, K)
        _untouched(th, K)
        tc, oc = _out(M, K, torch.int8, off)
        th2, oh2 = _out(M, K, dtype, off)
        codes, scale, h2 = q.rmsnorm_quantize_c8(x, gamma, 1e-6, residual, oc, None, torch.empty_like(x) if oh2 is None else oh2)
        _untouched(tc, K)
        _untouched(th2, K)
        assert torch.equal(h, h2)
        for s in slices():
            h64 = x[s].double() if residual is None else x[s].double() + residual[s].double()
            y64 = h64 / torch.sqrt(h64.square().mean(1, keepdim=True) + 1e-6) * gamma.double()
            assert torch.all((y[s].double() - y64).abs() <= (half + 2 * NORM_REL) * y64.abs() + tiny)
            assert torch.all((h[s].double() - h64).abs() <= (half + 2 * U) * h64.abs() + tiny)
            # value and largest value are each off by NORM_REL, the reciprocal, factor and product by U
            check_codes(codes[s], scale[s], y64, 127 * (2 * NORM_REL + 3.1 * U), NORM_REL)
        if residual is None:                                          # and without the sum, which is another path through the launch
            again = q.rmsnorm_quantize_c8(x, gamma, 1e-6)
            assert torch.equal(again[0], codes) and torch.equal(again[1], scale) and torch.equal(q.rmsnorm(x, gamma, 1e-6), y)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("off", [False, True])
@pytest.mark.parametrize("K", [64, 125, 500, 1024, 1029, 4096, 4100, 20001])
def test_in_place_with_rows_ahead(K, off, dtype):
    """Results in the place of X or of the residual while the CTA's next rows are already on their way."""
    M = _rows_for(K, 4)
    pad, shift = (3, 1) if off else (-K % 8, 0)
    gamma = torch.rand(K, device="cuda") + 0.5
    x, r = _matrix(M, K, dtype, 1, pad, shift), _matrix(M, K, dtype, 2, pad, shift)
    y, h = q.rmsnorm(x, gamma, 1e-6, r)
    codes, scale, _ = q.rmsnorm_quantize_c8(x, gamma, 1e-6, r)
    y0, (c0, s0) = q.rmsnorm(x, gamma, 1e-6), q.rmsnorm_quantize_c8(x, gamma, 1e-6)

    def copies():
        return _matrix(M, K, dtype, 1, pad, shift), _matrix(M, K, dtype, 2, pad, shift)

    a, b = copies()
    q.rmsnorm(a, gamma, 1e-6, b, Y=a, H=b)
    assert torch.equal(a, y) and torch.equal(b, h)
    a, b = copies()
    q.rmsnorm(a, gamma, 1e-6, b, Y=b, H=a)
    assert torch.equal(b, y) and torch.equal(a, h)
    for place in (0, 1):                                              # the sum in the place of the residual, or of X
        a, b = copies()
        c, s, _ = q.rmsnorm_quantize_c8(a, gamma, 1e-6, b, H=(b, a)[place])
        assert torch.equal(c, codes) and torch.equal(s, scale) and torch.equal((b, a)[place], h) and torch.equal((a, b)[place], (x, r)[place])
    a, _ = copies()
    q.rmsnorm(a, gamma, 1e-6, Y=a)
    assert torch.equal(a, y0)
    a, _ = copies()
    c, s, _ = q.rmsnorm_quantize_c8(a, gamma, 1e-6, H=a)              # h is x itself
    assert torch.equal(c, c0) and torch.equal(s, s0) and torch.equal(a, x)
