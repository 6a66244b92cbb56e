"""CPU checks of the rotation-free 8-bit entry points: the host answers what they refuse before anything touches a GPU."""
import paper_2509_21302_b200 as q

FAKE = 0x1000          # an aligned non-NULL address that is never dereferenced on these paths
BF16, FP16, FP32 = 0, 1, 2
NULL, SHAPE, ALIGN, UNSUPPORTED = -1, -2, -3, -4
MAX_ROWS, MAX_K = 2147483392, 131056


def _quantize(X=FAKE, type=BF16, ldx=64, M=4, K=64, Xq=FAKE, ldq=64, a=FAKE):
    return q.lib().qvggt_quantize_c8(X, type, ldx, M, K, Xq, ldq, a, None)


def _dequantize(Xq=FAKE, ldq=64, a=FAKE, M=4, K=64, Y=FAKE, type=BF16, ldy=64):
    return q.lib().qvggt_dequantize_c8(Xq, ldq, a, M, K, Y, type, ldy, None)


def _norm(quant, X=FAKE, R=FAKE, type=BF16, ldx=64, ldr=64, M=4, K=64, g=FAKE, eps=1e-6, H=FAKE, ldh=64, Y=FAKE, ldy=64, a=FAKE):
    if quant:
        return q.lib().qvggt_rmsnorm_quantize_c8(X, R, type, ldx, ldr, M, K, g, eps, H, ldh, Y, ldy, a, None)
    return q.lib().qvggt_rmsnorm(X, R, type, ldx, ldr, M, K, g, eps, H, ldh, Y, ldy, None)


def _linear(Xq=FAKE, ldx=64, a=FAKE, Wq=FAKE, ldw=64, w=FAKE, b=FAKE, M=4, N=32, K=64, Y=FAKE, type=BF16, ldy=32):
    return q.lib().qvggt_linear_c8(Xq, ldx, a, Wq, ldw, w, b, M, N, K, Y, type, ldy, None)


def test_missing_pointers():
    for name in ("X", "Xq", "a"):
        assert _quantize(**{name: None}) == NULL, name
    for name in ("Xq", "a", "Y"):
        assert _dequantize(**{name: None}) == NULL, name
    for quant in (False, True):
        for name in ("X", "g", "Y") + (("a",) if quant else ()):
            assert _norm(quant, **{name: None}) == NULL, name
    for name in ("Xq", "a", "Wq", "w", "Y"):
        assert _linear(**{name: None}) == NULL, name
    assert q.lib().qvggt_linear_status(None, None) == NULL


def test_sizes_and_strides():
    for f in (_quantize, _dequantize, lambda **k: _norm(False, **k), lambda **k: _norm(True, **k), _linear):
        assert f(M=-1) == SHAPE and f(M=MAX_ROWS + 1) == SHAPE
        assert f(K=0) == SHAPE and f(K=-5) == SHAPE
        assert f(M=0) == 0                                  # nothing to do, nothing looked at
        assert f(M=0, K=0) == SHAPE
    assert _quantize(ldx=63) == SHAPE and _quantize(ldq=63) == SHAPE
    assert _quantize(K=MAX_K + 1, ldx=1 << 20, ldq=1 << 20) == SHAPE
    assert _dequantize(ldq=63) == SHAPE and _dequantize(ldy=63) == SHAPE
    for quant in (False, True):
        for name in ("ldx", "ldr", "ldh", "ldy"):
            assert _norm(quant, **{name: 63}) == SHAPE, name
    assert _linear(N=0) == SHAPE and _linear(ldx=48) == SHAPE and _linear(ldw=48) == SHAPE and _linear(ldy=31) == SHAPE
    assert _linear(K=MAX_K + 1, ldx=1 << 20, ldw=1 << 20) == SHAPE


def test_alignment():
    assert _quantize(X=FAKE + 1) == ALIGN and _quantize(X=FAKE + 2, type=FP32) == ALIGN and _quantize(a=FAKE + 2) == ALIGN
    assert _dequantize(Y=FAKE + 1) == ALIGN and _dequantize(Y=FAKE + 2, type=FP32) == ALIGN and _dequantize(a=FAKE + 2) == ALIGN
    for quant in (False, True):
        for name in ("X", "R", "H"):
            assert _norm(quant, **{name: FAKE + 1}) == ALIGN and _norm(quant, type=FP32, **{name: FAKE + 2}) == ALIGN, name
        assert _norm(quant, g=FAKE + 2) == ALIGN
    assert _norm(False, Y=FAKE + 1) == ALIGN and _norm(True, a=FAKE + 2) == ALIGN
    for bad in (dict(Xq=FAKE + 8), dict(Wq=FAKE + 8), dict(ldx=72), dict(ldw=72), dict(a=FAKE + 2), dict(w=FAKE + 2), dict(b=FAKE + 1), dict(Y=FAKE + 1)):
        assert _linear(**bad) == ALIGN, bad
    assert _linear(b=FAKE + 2, type=FP32) == ALIGN and _linear(Y=FAKE + 2, type=FP32) == ALIGN


def test_types_and_epsilon():
    for t in (-1, 3, 7):
        assert _quantize(type=t) == _dequantize(type=t) == _norm(False, type=t) == _norm(True, type=t) == _linear(type=t) == UNSUPPORTED
    for eps in (-1e-6, float("nan"), float("inf")):
        assert _norm(False, eps=eps) == UNSUPPORTED and _norm(True, eps=eps) == UNSUPPORTED


def test_the_binding_refuses_host_tensors():
    import pytest
    import torch
    x, g = torch.zeros(4, 64, dtype=torch.bfloat16), torch.ones(64)
    xq, a, w = torch.zeros(4, 64, dtype=torch.int8), torch.ones(4), torch.zeros(32, 64, dtype=torch.int8)
    for call in (lambda: q.quantize_c8(x), lambda: q.dequantize_c8(xq, a), lambda: q.rmsnorm(x, g), lambda: q.rmsnorm_quantize_c8(x, g),
                 lambda: q.linear_c8(xq, a, w, torch.ones(32))):
        with pytest.raises(AssertionError):
            call()


def test_the_starved_launch_is_bounded():
    def starved(M=4, limit=100000, Xq=FAKE):
        return q.lib().qvggt_debug_starved_linear(Xq, 64, FAKE, FAKE, 64, FAKE, M, 32, 64, FAKE, 32, limit, None)

    assert starved(M=0) == SHAPE and starved(M=513) == SHAPE and starved(limit=999) == SHAPE and starved(limit=2000000000) == SHAPE
    assert starved(Xq=None) == NULL and starved(Xq=FAKE + 8) == ALIGN
