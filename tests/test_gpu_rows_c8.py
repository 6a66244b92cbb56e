"""The row operators of the rotation-free 8-bit path (quantizer, its inverse, RMS norm, norm with 8-bit output) against the definitions in
64 bits.  One fp32 rounding is 2^-24 of the value (U below); a rounding to an output's type is half its eps."""
import pytest
import torch

import paper_2509_21302_b200 as q
from paper_2509_21302_b200 import binding

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = [torch.bfloat16, torch.float16, torch.float32]
SIZES = [(1, 1), (3, 7), (1, 8), (9, 9), (2, 64), (33, 64), (35, 61), (18, 128), (7, 100), (6001, 64), (5003, 127), (17, 255), (8, 257), (33, 512), (5, 1003), (300, 1024), (7, 1025), (4, 2048), (65, 4096), (3, 5001),
         (2, 16384), (2, 32768), (2, 32776), (1, 131056)]


def _matrix(M, K, dtype, seed, pad=0, shift=0, scale=1.0):
    """Rows with a few large channels; `pad` elements between them, the first one `shift` elements into its memory."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = torch.full((shift + M * (K + pad),), 7.0, dtype=dtype, device="cuda")[shift:].view(M, K + pad)[:, :K]
    v = torch.randn(M, K, generator=g, device="cuda") * scale
    v[:, torch.randint(K, (3,), generator=g, device="cuda")] *= 30.0
    t.copy_(v)
    return t


def _check_codes(codes, scale, y, slack, rel):
    """codes and scales of the rows y (64 bits) whose computed values are off by at most `rel` of themselves."""
    amax = y.abs().amax(1).clamp_min(1e-8)
    assert torch.all((scale.double() - amax / 127).abs() <= (rel + U) * amax / 127)
    off = (codes.double() - y * (127 / amax)[:, None]).abs()
    assert torch.all(off <= 0.5 + slack), float(off.max())
    assert codes.abs().max() <= 127


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,K", SIZES)
def test_quantize(M, K, dtype):
    x = _matrix(M, K, dtype, M + K)
    codes, scale = q.quantize_c8(x)
    assert codes.shape == (M, K) and codes.dtype == torch.int8 and (M == 1 or codes.stride(0) % 16 == 0)
    # the reciprocal of amax, 127 times it and the product with that are rounded, U each: positions up to 127 are off by 3 * 127 U (and
    # the products of these)
    _check_codes(codes, scale, x.double(), 127 * 3.1 * U, 0.0)
    amax = x.float().abs().amax(1, keepdim=True).clamp_min(1e-8)            # bit for bit the formula's operations in fp32
    assert torch.equal(codes, (x.float() * (amax.reciprocal() * 127.0)).round().to(torch.int8))


def _norm64(x, r, gamma, eps):
    h = x.double() if r is None else x.double() + r.double()
    return h, h / torch.sqrt(h.square().mean(1, keepdim=True) + eps) * gamma.double()


# fp32 roundings in y: the sum h (1), two products (2), and 1 / sqrt: itself (at most 2 units in the last place: 4) and half of what its
# argument is off by: squares of rounded sums 2, at most 40 additions on the way of a term to the total, 1 / K, the multiply-add with it.
# 1 + 2 + 4 + 44 / 2 = 29.
NORM_REL = 29 * U


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("M,K", SIZES)
def test_rmsnorm(M, K, residual, dtype):
    x, r = _matrix(M, K, dtype, 3 * M + K), _matrix(M, K, dtype, 5 * M + K, scale=2.0) if residual else None
    gamma = torch.randn(K, device="cuda") * 0.2 + 1.0
    h64, y64 = _norm64(x, r, gamma, 1e-6)
    out = q.rmsnorm(x, gamma, 1e-6, r)
    y, h = out if residual else (out, None)
    half, tiny = torch.finfo(dtype).eps / 2, torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps
    assert y.dtype == dtype and y.shape == (M, K)
    assert torch.all((y.double() - y64).abs() <= (half + 2 * NORM_REL) * y64.abs() + tiny)
    if residual:
        assert torch.all((h.double() - h64).abs() <= (half + 2 * U) * h64.abs() + tiny)
    codes, scale, *more = q.rmsnorm_quantize_c8(x, gamma, 1e-6, r)
    # value and largest value are each off by NORM_REL, the reciprocal, factor and product by U
    _check_codes(codes, scale, y64, 127 * (2 * NORM_REL + 3.1 * U), NORM_REL)
    if residual:
        assert torch.equal(more[0], h)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,K", SIZES)
def test_dequantize(M, K, dtype):
    g = torch.Generator(device="cuda").manual_seed(K)
    codes = torch.randint(-128, 128, (M, K), generator=g, device="cuda", dtype=torch.int8)
    scale = torch.rand(M, generator=g, device="cuda") * 0.01 + 0.001
    y = q.dequantize_c8(codes, scale, dtype)
    want = codes.double() * scale.double()[:, None]
    assert torch.all((y.double() - want).abs() <= (torch.finfo(dtype).eps / 2 + U) * want.abs() * (1 + U))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("K", [1, 15, 64, 127, 1003, 1024, 3001, 33000])
@pytest.mark.parametrize("pad,shift", [(5, 0), (0, 1), (8, 8), (3, 3)])
def test_strides_and_offsets_change_nothing(K, pad, shift, dtype):
    """Any row stride and first element give the results of the aligned layout, and what lies between the rows is left as it was."""
    M = 11
    x, r = _matrix(M, K, dtype, K), _matrix(M, K, dtype, K + 1)
    xs, rs = _matrix(M, K, dtype, K, pad, shift), _matrix(M, K, dtype, K + 1, pad + 1, shift)
    store = torch.full((1 + M * (K + 7),), 3.0, device="cuda")
    gamma = store[1:1 + K].clone().uniform_(0.5, 1.5)
    gs = torch.empty(K + 1, device="cuda")[1:]
    gs.copy_(gamma)

    def out(kind):
        t = torch.full((shift + M * (K + pad),), 3, dtype=kind, device="cuda")
        return t, t[shift:].view(M, K + pad)[:, :K]

    def untouched(t):
        edge = t[:shift].tolist() + t[shift:].view(M, K + pad)[:, K:].reshape(-1).tolist()
        assert all(v == 3 for v in edge)

    (codes, scale), (y, h) = q.quantize_c8(x), q.rmsnorm(x, gamma, 1e-5, r)
    nq, ns, nh = q.rmsnorm_quantize_c8(x, gamma, 1e-5, r)
    t, o = out(torch.int8)
    a = torch.empty(M, device="cuda")
    got = q.quantize_c8(xs, o, a)
    assert got[0] is o and got[1] is a and torch.equal(o, codes) and torch.equal(a, scale)
    untouched(t)
    t, o = out(dtype)
    t2, o2 = out(dtype)
    q.rmsnorm(xs, gs, 1e-5, rs, o, o2)
    assert torch.equal(o, y) and torch.equal(o2, h)
    untouched(t)
    untouched(t2)
    t, o = out(torch.int8)
    t2, o2 = out(dtype)
    q.rmsnorm_quantize_c8(xs, gs, 1e-5, rs, o, a, o2)
    assert torch.equal(o, nq) and torch.equal(a, ns) and torch.equal(o2, nh)
    untouched(t)
    t2, o2 = out(dtype)
    q.dequantize_c8(o, a, Y=o2)
    assert torch.equal(o2, q.dequantize_c8(nq, ns, dtype))
    untouched(t2)


@pytest.mark.parametrize("K", [40, 100, 1024, 4096, 40000])
def test_in_place(K):
    M, dtype = 6, torch.bfloat16
    gamma = torch.rand(K, device="cuda") + 0.5
    x, r = _matrix(M, K, dtype, 1), _matrix(M, K, dtype, 2)
    y, h = q.rmsnorm(x, gamma, 1e-6, r)
    codes, scale, _ = q.rmsnorm_quantize_c8(x, gamma, 1e-6, r)
    x1, r1 = x.clone(), r.clone()
    q.rmsnorm(x1, gamma, 1e-6, r1, Y=x1, H=r1)
    assert torch.equal(x1, y) and torch.equal(r1, h)
    x1, r1 = x.clone(), r.clone()
    q.rmsnorm(x1, gamma, 1e-6, r1, Y=r1, H=x1)
    assert torch.equal(r1, y) and torch.equal(x1, h)
    r1 = r.clone()
    c1, s1, h1 = q.rmsnorm_quantize_c8(x, gamma, 1e-6, r1, H=r1)
    assert h1 is r1 and torch.equal(c1, codes) and torch.equal(s1, scale) and torch.equal(r1, h)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("K", [31, 1024, 5000, 40000])
def test_rows_of_zeros_ties_and_non_finite_values(K, dtype):
    x = _matrix(8, K, dtype, K)
    x[1] = 0
    x[2, K // 2] = float("nan")
    x[3, 0] = float("inf")
    x[4, K - 1] = float("-inf")
    x[5] = 0
    x[5, :2] = torch.tensor([127.0, 2.5])           # exact ties go to the even code
    x[5, 2:5] = torch.tensor([3.5, -0.5, -1.5])
    x[6] = 1e-12 if dtype != torch.float16 else 0   # far below the floor of the step size
    codes, scale = q.quantize_c8(x)
    for m in (2, 3, 4):
        assert torch.isnan(scale[m]) and not codes[m].any()
    assert not codes[1].any() and not codes[6].any()
    assert scale[1] == scale[6] == torch.tensor(1e-8) / torch.tensor(127.0)
    assert codes[5, :5].tolist() == [127, 2, 4, 0, -2] and scale[5] == 1.0
    for m in (0, 7):                                # the other rows are what they are without these
        c, s = q.quantize_c8(x[m:m + 1])
        assert torch.equal(c[0], codes[m]) and s[0] == scale[m]
    v = q.dequantize_c8(codes, scale)
    assert torch.isnan(v[2:5]).all() and torch.isfinite(v[[0, 1, 5, 6, 7]]).all()
    gamma = torch.ones(K, device="cuda")
    y = q.rmsnorm(x, gamma, 1e-6)
    assert not y[1].any() and torch.isnan(y[2]).all()
    assert torch.isnan(y[3, 0]) and torch.isnan(y[4, K - 1]) and not y[3, 1:].any()     # inf / inf, finite / inf
    codes, scale = q.rmsnorm_quantize_c8(x, gamma, 1e-6)
    assert torch.isnan(scale[2:5]).all() and not codes[1:5].any() and torch.isfinite(scale[[0, 1, 5, 6, 7]]).all()
    y = q.rmsnorm(x, gamma, 0.0)                    # 0 / 0
    assert torch.isnan(y[1]).all() and torch.isfinite(y[0]).all()


@pytest.mark.parametrize("K", [64, 100, 1024, 5000, 40000])
def test_rows_at_the_ends_of_the_range(K):
    """Sums of squares beyond fp32 give 0; rows that no epsilon holds up are not finite; the largest and smallest fp32 values quantize."""
    x = torch.ones(5, K, device="cuda")
    x[0], x[1], x[2], x[3] = 1e25, 0.0, 1e-30, 3e38
    gamma = torch.ones(K, device="cuda")
    assert not q.rmsnorm(x, gamma)[0].any()
    codes, scale = q.rmsnorm_quantize_c8(x, gamma, 1e-6)
    assert not codes[0].any() and scale[0] == scale[1] == torch.tensor(1e-8) / torch.tensor(127.0) and not codes[1].any()
    assert torch.all(codes[4] == 127)
    codes, scale = q.rmsnorm_quantize_c8(x, gamma, 0.0)             # 0 / 0, and 1e-30 / sqrt(1e-60), which is 0 in fp32
    assert torch.isnan(scale[1]) and torch.isnan(scale[2]) and not codes[1:3].any() and torch.all(codes[4] == 127)
    codes, scale = q.quantize_c8(x)
    assert torch.all(codes[3] == 127) and torch.all(codes[0] == 127) and torch.isfinite(scale).all() and not codes[1:3].any()


def test_empty_batches():
    for dtype in TYPES:
        x = torch.empty(0, 100, dtype=dtype, device="cuda")
        codes, scale = q.quantize_c8(x)
        assert codes.shape == (0, 100) and scale.shape == (0,)
        assert q.dequantize_c8(codes, scale).shape == (0, 100)
        y, h = q.rmsnorm(x, torch.ones(100, device="cuda"), residual=x)
        assert y.shape == h.shape == (0, 100)


def test_elements_beyond_2_to_the_31():
    M, K = 530000, 4100                             # 2.2e9 elements: the last rows lie beyond 2^31 elements and 2^32 bytes
    x = torch.zeros(M, K, dtype=torch.bfloat16, device="cuda")
    tail = _matrix(40, K, torch.bfloat16, 9)
    x[-40:] = tail
    x[100:140] = tail
    gamma = torch.rand(K, device="cuda") + 0.5
    want = q.rmsnorm_quantize_c8(tail.contiguous(), gamma, 1e-6, tail.contiguous())
    codes, scale, h = q.rmsnorm_quantize_c8(x, gamma, 1e-6, x)
    for rows in (slice(M - 40, M), slice(100, 140)):
        assert torch.equal(codes[rows], want[0]) and torch.equal(scale[rows], want[1]) and torch.equal(h[rows], want[2])
    assert not codes[140:200].any() and not codes[M - 100:M - 40].any()
    del h
    y = q.dequantize_c8(codes, scale)
    assert torch.equal(y[-40:], q.dequantize_c8(want[0], want[1]))


def test_streams_and_graphs():
    M, K, dtype = 300, 1024, torch.bfloat16
    x, r, gamma = _matrix(M, K, dtype, 1), _matrix(M, K, dtype, 2), torch.rand(K, device="cuda") + 0.5
    want = q.rmsnorm_quantize_c8(x, gamma, 1e-6, r)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = q.rmsnorm_quantize_c8(x, gamma, 1e-6, r)
        v = q.dequantize_c8(got[0], got[1])
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    xs, rs = torch.zeros_like(x), torch.zeros_like(r)
    with torch.cuda.graph(graph):
        captured = q.rmsnorm_quantize_c8(xs, gamma, 1e-6, rs)
        cv = q.dequantize_c8(captured[0], captured[1])
    for k in range(3):
        xs.copy_(x.roll(k, 0))
        rs.copy_(r.roll(k, 0))
        graph.replay()
        assert all(torch.equal(a, b.roll(k, 0)) for a, b in zip(captured, want)) and torch.equal(cv, v.roll(k, 0))


def test_both_routes_of_the_binding(monkeypatch):
    for M, K, dtype in ((5, 1003, torch.float16), (1, 64, torch.bfloat16), (0, 33, torch.float32)):
        x, r, gamma = _matrix(M, K, dtype, 1), _matrix(M, K, dtype, 2), torch.rand(K, device="cuda")

        def calls():
            c, s = q.quantize_c8(x)
            return [c, s, q.dequantize_c8(c, s, torch.float32), q.rmsnorm(x, gamma), *q.rmsnorm(x, gamma, 1e-5, r), *q.rmsnorm_quantize_c8(x, gamma),
                    *q.rmsnorm_quantize_c8(x, gamma, 1e-5, r), *q.rmsnorm(x, gamma, H=torch.empty_like(x))]

        fast = calls()
        monkeypatch.setattr(binding, "_fast", None)
        slow = calls()
        monkeypatch.undo()
        assert len(fast) == len(slow)
        for a, b in zip(fast, slow):
            assert a.shape == b.shape and a.dtype == b.dtype and (M < 2 or a.stride() == b.stride()) and torch.equal(a, b)


def test_refusals():
    x, g = torch.zeros(4, 64, dtype=torch.bfloat16, device="cuda"), torch.ones(64, device="cuda")
    xq, a = q.quantize_c8(x)
    for bad in (lambda: q.quantize_c8(x.double()), lambda: q.quantize_c8(x.t()), lambda: q.quantize_c8(x[0]), lambda: q.quantize_c8(x, xq.view(torch.uint8)),
                lambda: q.quantize_c8(x, xq[:2]), lambda: q.quantize_c8(x, xq, a.double()), lambda: q.quantize_c8(x, xq, a[:3]), lambda: q.quantize_c8(x.cpu()),
                lambda: q.dequantize_c8(xq, a, torch.float64), lambda: q.dequantize_c8(xq, a[:2]), lambda: q.dequantize_c8(xq.view(torch.uint8), a),
                lambda: q.rmsnorm(x, g.bfloat16()), lambda: q.rmsnorm(x, g[:63]), lambda: q.rmsnorm(x, g, 1e-6, x.half()), lambda: q.rmsnorm(x, g, 1e-6, x[:2]),
                lambda: q.rmsnorm(x, g, H=x.float()), lambda: q.rmsnorm_quantize_c8(x, g, Xq8=xq[:, :32])):
        with pytest.raises(AssertionError):
            bad()
    for bad in (lambda: q.quantize_c8(x[:1].expand(4, 64)), lambda: q.rmsnorm(x, g, 1e-6, x[:1].expand(4, 64))):     # rows on top of one another
        with pytest.raises(q.QvggtError) as e:
            bad()
        assert e.value.status == -2
    with pytest.raises(q.QvggtError) as e:
        q.rmsnorm(x, g, -1.0)
    assert e.value.status == -4


@pytest.mark.parametrize("seed", range(6))
def test_random_sizes(seed):
    import random
    rng = random.Random(seed)
    for _ in range(25):
        M, K = int(2 ** rng.uniform(0, 12)), int(2 ** rng.uniform(0, 13.5))
        dtype, pad, shift = rng.choice(TYPES), rng.choice((0, 1, 3, 8, 24)), rng.choice((0, 0, 1, 8))
        x, r = _matrix(M, K, dtype, rng.randrange(1000), pad, shift), _matrix(M, K, dtype, rng.randrange(1000), rng.choice((0, pad)))
        gamma = torch.rand(K, device="cuda") + 0.5
        codes, scale = q.quantize_c8(x)
        _check_codes(codes, scale, x.double(), 127 * 3.1 * U, 0.0)
        h64, y64 = _norm64(x, r, gamma, 1e-6)
        half, tiny = torch.finfo(dtype).eps / 2, torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps
        y, h = q.rmsnorm(x, gamma, 1e-6, r)
        assert torch.all((y.double() - y64).abs() <= (half + 2 * NORM_REL) * y64.abs() + tiny)
        assert torch.all((h.double() - h64).abs() <= (half + 2 * U) * h64.abs() + tiny)
        codes, scale, h2 = q.rmsnorm_quantize_c8(x, gamma, 1e-6, r)
        _check_codes(codes, scale, y64, 127 * (2 * NORM_REL + 3.1 * U), NORM_REL)
        assert torch.equal(h, h2)
