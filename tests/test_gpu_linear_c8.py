"""The product of 8-bit codes with scales for each token and channel against the definition in 64 bits, and the rotation-free path as a
layer runs it.  One fp32 rounding is 2^-24 of the value (U below); a rounding to an output's type is half its eps."""
import pytest
import torch

import paper_2509_21302_b200 as q
from paper_2509_21302_b200 import binding

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _no_wait_expired():
    yield
    assert q.linear_status() == 0


U = 2.0 ** -24
TYPES = [torch.bfloat16, torch.float16, torch.float32]


def _codes(rows, K, seed, lo=-127, pad=0):
    """Codes whose rows are 16 bytes apart or a multiple; the bytes behind K are anything but zero."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = torch.randint(lo, 128, (rows, (K + 15) // 16 * 16 + pad), generator=g, device="cuda", dtype=torch.int8)
    t[:, K:] = 77
    return t[:, :K]


def _problem(M, N, K, dtype, bias, seed=0, lo=-127, pad=0):
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    a, w = torch.rand(M, generator=g, device="cuda") * 0.01 + 0.001, torch.rand(N, generator=g, device="cuda") * 0.01 + 0.001
    b = torch.randn(N, generator=g, device="cuda").to(dtype) if bias else None
    return _codes(M, K, seed + 2, lo, pad), a, _codes(N, K, seed + 3, lo, pad), w, b


def _check(y, xq, a, wq, w, b):
    acc = xq.double() @ wq.double().t()                     # exact: below 2^53
    p = acc * (a.double()[:, None] * w.double())
    z = p if b is None else p + b.double()
    half, tiny = torch.finfo(y.dtype).eps / 2, torch.finfo(y.dtype).smallest_normal * torch.finfo(y.dtype).eps
    # the conversion of acc and the product of the scales: 2 U of p (and their product); the multiply-add: U of z; the type: half of z
    bound = (2 * U + 2 * U * U) * p.abs() * (1 + half) + (U + half + U * half) * z.abs() + tiny
    off = (y.double() - z).abs()
    assert torch.all(off <= bound), float((off / bound).max())


EDGES = [(1, 1, 1), (1, 16, 15), (1, 17, 16), (2, 100, 17), (5, 33, 127), (7, 64, 128), (8, 65, 129), (9, 128, 1000), (16, 200, 1024), (17, 129, 1025),
         (32, 64, 2011), (33, 256, 4096), (40, 5003, 640), (64, 1000, 8193), (77, 77, 77), (127, 130, 1024), (128, 128, 4096), (129, 192, 333), (200, 1024, 16384),
         (255, 257, 511), (256, 256, 896), (257, 64, 1024), (300, 2000, 1100), (1374, 1024, 1024), (1001, 1003, 1005), (2000, 520, 4096), (3000, 4096, 192)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,N,K", EDGES)
def test_against_64_bits(M, N, K, dtype):
    for bias in (False, True):
        p = _problem(M, N, K, dtype, bias, M + N + K)
        y = q.linear_c8(*p, dtype=dtype)
        assert y.shape == (M, N) and y.dtype == dtype
        _check(y, *p)


@pytest.mark.parametrize("M", [1, 20, 100, 300, 700])
def test_the_largest_sums(M):
    """Every code -128 at the longest row: sums of 2147221504, just below 2^31."""
    K, N = 131056, 65
    xq, wq = torch.full((M, K), -128, dtype=torch.int8, device="cuda"), torch.full((N, K), -128, dtype=torch.int8, device="cuda")
    y = q.linear_c8(xq, torch.ones(M, device="cuda"), wq, torch.ones(N, device="cuda"), dtype=torch.float32)
    assert torch.all(y == float(torch.tensor(128 * 128 * K, dtype=torch.float32)))


@pytest.mark.parametrize("N,K", [(64, 96), (1003, 1003), (4096, 1024), (640, 4096)])
def test_a_row_does_not_depend_on_the_batch(N, K):
    M = 1500
    xq, a, wq, w, b = _problem(M, N, K, torch.float32, True, 5)
    whole = q.linear_c8(xq, a, wq, w, b, torch.float32)
    for m in (1, 8, 9, 31, 33, 64, 65, 128, 130, 256, 400, 777):
        part = q.linear_c8(xq[M - m:], a[M - m:].clone(), wq, w, b, torch.float32)
        assert torch.equal(part, whole[M - m:]), m


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,N,K", [(3, 50, 64), (40, 129, 200), (150, 1003, 333), (600, 1001, 1024), (513, 64, 1024)])
@pytest.mark.parametrize("pad,shift", [(0, 0), (5, 0), (0, 1), (8, 8), (3, 3)])
def test_results_of_any_stride(M, N, K, pad, shift, dtype):
    """Results go to rows of any stride and first element, and what lies around them is left as it was."""
    p = _problem(M, N, K, dtype, True, 7, pad=32)
    want = q.linear_c8(*p, dtype=dtype)
    t = torch.full((shift + (M + 2) * (N + pad),), 3.0, dtype=dtype, device="cuda")
    y = t[shift:].view(M + 2, N + pad)[:M, :N]
    assert q.linear_c8(*p, Y=y) is y
    assert torch.equal(y, want)
    rest = t[shift:].view(M + 2, N + pad)
    assert (t[:shift] == 3).all() and (rest[:M, N:] == 3).all() and (rest[M:] == 3).all()
    odd = torch.empty(N + 1, dtype=dtype, device="cuda")[1:]            # parameters off every wide boundary
    odd.copy_(p[4])
    w = torch.empty(N + 1, device="cuda")[1:]
    w.copy_(p[3])
    a = torch.empty(M + 1, device="cuda")[1:]
    a.copy_(p[1])
    assert torch.equal(q.linear_c8(p[0], a, p[2], w, odd, dtype), want)


def test_non_finite_scales_stay_in_their_rows():
    for M in (5, 300):
        xq, a, wq, w, b = _problem(M, 200, 256, torch.bfloat16, True, 3)
        clean = q.linear_c8(xq, a, wq, w, b)
        a2 = a.clone()
        a2[2] = float("nan")
        y = q.linear_c8(xq, a2, wq, w, b)
        assert torch.isnan(y[2]).all()
        assert torch.equal(y[[0, 1, 3, 4]], clean[[0, 1, 3, 4]]) and torch.equal(y[5:], clean[5:])


def test_results_beyond_2_to_the_31():
    M, N, K = 270000, 8200, 16                              # 2.2e9 results
    xq, a, wq, w, b = _problem(64, N, K, torch.bfloat16, True, 11)
    big, scales = torch.zeros(M, K, dtype=torch.int8, device="cuda"), torch.ones(M, device="cuda")
    want = q.linear_c8(xq, a, wq, w, b)
    for rows in (slice(0, 64), slice(M - 64, M)):
        big[rows], scales[rows] = xq, a
    y = q.linear_c8(big, scales, wq, w, b)
    assert torch.equal(y[:64], want) and torch.equal(y[-64:], want) and torch.equal(y[M - 65], b) and torch.equal(y[64], b)


def test_codes_beyond_2_to_the_31():
    M, N, K = 70, 17000, 131056                             # 2.2e9 weight codes
    wq = torch.ones(N, K, dtype=torch.int8, device="cuda")
    wq[-5:] = _codes(5, K, 1)
    xq, a, w = _codes(M, K, 2), torch.ones(M, device="cuda"), torch.ones(N, device="cuda")
    y = q.linear_c8(xq, a, wq, w, dtype=torch.float32)
    _check(y[:, -20:].contiguous(), xq, a, wq[-20:], w[-20:], None)
    _check(y[:, :20].contiguous(), xq, a, wq[:20], w[:20], None)


def test_empty_batch():
    y = q.linear_c8(torch.empty(0, 64, dtype=torch.int8, device="cuda"), torch.empty(0, device="cuda"), _codes(40, 64, 1), torch.ones(40, device="cuda"))
    assert y.shape == (0, 40)


@pytest.mark.parametrize("M", [1, 50, 200, 1374])
def test_streams_graphs_and_repetition(M):
    p = _problem(M, 1030, 2000, torch.bfloat16, True, 13)
    want = q.linear_c8(*p)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = [q.linear_c8(*p) for _ in range(12)]          # back to back: a launch may begin while the one before it drains
    side.synchronize()
    assert all(torch.equal(y, want) for y in got)
    other = _problem(M, 1030, 2000, torch.bfloat16, True, 14)
    want2 = q.linear_c8(*other)
    with torch.cuda.stream(side):                           # two at once
        y2 = [q.linear_c8(*other) for _ in range(8)]
    y1 = [q.linear_c8(*p) for _ in range(8)]
    torch.cuda.synchronize()
    assert all(torch.equal(y, want) for y in y1) and all(torch.equal(y, want2) for y in y2)
    graph = torch.cuda.CUDAGraph()
    xs, as_ = torch.zeros_like(p[0]), torch.zeros_like(p[1])
    xs = torch.zeros(M, 2000, dtype=torch.int8, device="cuda")
    with torch.cuda.graph(graph):
        y = q.linear_c8(xs, as_, *p[2:])
    for s in (p, other):
        xs.copy_(s[0])
        as_.copy_(s[1])
        graph.replay()
        assert torch.equal(y, q.linear_c8(s[0], s[1], *p[2:]))


def test_both_routes_of_the_binding(monkeypatch):
    for M, N, K, dtype in ((5, 100, 64, torch.float16), (1, 7, 33, torch.float32), (130, 1003, 1003, torch.bfloat16)):
        p = _problem(M, N, K, dtype, True, 1)
        y = lambda: torch.empty(M, N + 1, dtype=dtype, device="cuda")[:, :N]
        fast = [q.linear_c8(*p, dtype=dtype), q.linear_c8(*p, Y=y())]
        monkeypatch.setattr(binding, "_fast", None)
        slow = [q.linear_c8(*p, dtype=dtype), q.linear_c8(*p, Y=y())]
        monkeypatch.undo()
        for a, b in zip(fast, slow):
            assert a.dtype == b.dtype and (M == 1 or a.stride() == b.stride()) and torch.equal(a, b)


def test_refusals():
    xq, a, wq, w, b = _problem(4, 32, 64, torch.bfloat16, True)
    for bad in (lambda: q.linear_c8(xq.view(torch.uint8), a, wq, w), lambda: q.linear_c8(xq, a[:3], wq, w), lambda: q.linear_c8(xq, a, wq[:, :32], w),
                lambda: q.linear_c8(xq, a, wq, w[:31]), lambda: q.linear_c8(xq, a, wq, w, b.half()), lambda: q.linear_c8(xq, a, wq, w, b[:31]),
                lambda: q.linear_c8(xq, a, wq, w, b, torch.float64), lambda: q.linear_c8(xq, a.double(), wq, w), lambda: q.linear_c8(xq, a, wq.float(), w),
                lambda: q.linear_c8(xq, a, wq, w, b, Y=torch.empty(4, 33, device="cuda").bfloat16()), lambda: q.linear_c8(xq[:, ::2], a, wq[:, ::2], w),
                lambda: q.linear_c8(xq, a, wq, w, b, Y=torch.empty(32, 4, dtype=torch.bfloat16, device="cuda").t()), lambda: q.linear_c8(xq.cpu(), a, wq, w)):
        with pytest.raises(AssertionError):
            bad()
    for bad in (lambda: q.linear_c8(torch.zeros(4, 65, dtype=torch.int8, device="cuda")[:, 1:], a, wq, w),                  # rows off a 16-byte boundary
                lambda: q.linear_c8(xq, a, torch.zeros(32, 65, dtype=torch.int8, device="cuda")[:, :64], w)):
        with pytest.raises(q.QvggtError) as e:
            bad()
        assert e.value.status == -3


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("M,K,N", [(1, 256, 512), (45, 1003, 700), (600, 1024, 4096)])
def test_a_layer(M, K, N, dtype):
    """From attention's output to fc1's: quantize, product, residual + norm + quantize, product -- each step against its definition in 64
    bits on the step's own inputs, the whole within the errors of 8-bit codes against the layer in full precision."""
    g = torch.Generator(device="cuda").manual_seed(M)
    attn, res = torch.randn(M, K, generator=g, device="cuda").to(dtype), torch.randn(M, K, generator=g, device="cuda").to(dtype)
    w1, w2 = (torch.randn(n, K, generator=g, device="cuda") / K ** 0.5 for n in (K, N))
    gamma = torch.rand(K, generator=g, device="cuda") + 0.5
    b1 = torch.randn(K, generator=g, device="cuda").to(dtype)
    (q1, s1), (q2, s2) = q.quantize_c8(w1), q.quantize_c8(w2)
    xq, a = q.quantize_c8(attn)
    o = q.linear_c8(xq, a, q1, s1, b1, dtype)
    _check(o, xq, a, q1, s1, b1)
    hq, ha, h = q.rmsnorm_quantize_c8(o, gamma, 1e-6, res)
    y = q.linear_c8(hq, ha, q2, s2, None, dtype)
    _check(y, hq, ha, q2, s2, None)
    assert torch.equal(h, (o.float() + res.float()).to(dtype))
    full = attn.double() @ w1.double().t() + b1.double() + res.double()
    want = full / torch.sqrt(full.square().mean(1, keepdim=True) + 1e-6) * gamma.double() @ w2.double().t()
    # A code is off by at most half a step of amax / 127, evenly spread: step / sqrt(12).  Normal rows of up to 4096 values have amax < 6
    # rms (gamma adds 1.5), so each of the four quantized operands is off by less than 9 / 127 / sqrt(12) = 2.1 % of its rms: 4.1 % in all,
    # with the 16-bit roundings below 0.5 % each.
    assert (y.double() - want).norm() <= 0.05 * want.norm()


@pytest.mark.parametrize("M", [1, 20, 90, 300, 1500])
def test_what_the_call_before_wrote(M):
    """Weights, activations and scales written by the calls directly in front of the product, new ones every time: a launch may set itself
    up, and bring weights to L2, while the one before it still runs."""
    N, K = 1100, 2048
    g = torch.Generator(device="cuda").manual_seed(M)
    Ws = [torch.randn(N, K, generator=g, device="cuda") for _ in range(6)]
    Xs = [torch.randn(M, K, generator=g, device="cuda").bfloat16() for _ in range(6)]
    want = []
    for W, X in zip(Ws, Xs):
        c, s = q.quantize_c8(W)
        xq, a = q.quantize_c8(X)
        torch.cuda.synchronize()
        want.append(q.linear_c8(xq, a, c, s, dtype=torch.float32))
        torch.cuda.synchronize()
    c, s = q.quantize_c8(torch.zeros_like(Ws[0]))
    xq, a = q.quantize_c8(torch.zeros_like(Xs[0]))
    for _ in range(3):
        got = []
        for W, X in zip(Ws, Xs):
            q.quantize_c8(X, xq, a)
            q.quantize_c8(W, c, s)
            got.append(q.linear_c8(xq, a, c, s, dtype=torch.float32))
        assert all(torch.equal(x, y) for x, y in zip(got, want))
        got = []
        for W, X in zip(Ws, Xs):
            q.quantize_c8(W, c, s)
            q.quantize_c8(X, xq, a)
            got.append(q.linear_c8(xq, a, c, s, dtype=torch.float32))
        assert all(torch.equal(x, y) for x, y in zip(got, want))


@pytest.mark.parametrize("seed", range(6))
def test_random_sizes(seed):
    import random
    r = random.Random(seed)
    for _ in range(25):
        M = int(2 ** r.uniform(0, 11))
        N, K = int(2 ** r.uniform(0, 13)), int(2 ** r.uniform(0, 13))
        dtype = r.choice(TYPES)
        p = _problem(M, N, K, dtype, r.random() < 0.5, r.randrange(1000), pad=16 * r.randrange(3))
        pad = r.choice((0, 0, 1, 8))
        y = torch.full((M + 1, N + pad), 5.0, dtype=dtype, device="cuda")
        q.linear_c8(*p, Y=y[:M, :N])
        _check(y[:M, :N].contiguous(), *p)
        assert (y[M] == 5).all() and (y[:, N:] == 5).all(), (M, N, K, dtype, pad)


@pytest.mark.parametrize("M", [1, 2, 3, 4, 5])
@pytest.mark.parametrize("N,K", [(1, 1), (3, 15), (2, 511), (5, 513), (7, 1025), (65, 2047), (1, 16385), (33, 131056), (4097, 1024), (8193, 1023), (8193, 1024), (1001, 2500)])
def test_single_tokens(M, N, K):
    """One to five rows where their warps share a row or do not, with extreme codes; the rows are those of a longer call bit for bit."""
    for dtype in TYPES:
        p = _problem(M, N, K, dtype, dtype != torch.float16, K + M, lo=-128)
        y = q.linear_c8(*p, dtype=dtype)
        _check(y, *p)
        xq, a = torch.zeros(40, (K + 15) // 16 * 16, dtype=torch.int8, device="cuda"), torch.ones(40, device="cuda")
        xq[7:7 + M, :K], a[7:7 + M] = p[0], p[1]
        assert torch.equal(q.linear_c8(xq[:, :K], a, *p[2:], dtype=dtype)[7:7 + M], y)
