"""The rotation-free 8-bit path of a transformer layer: RMS norm with the residual's addition and 8-bit output, the row quantizer and
its inverse, and the integer product with one scale per token and per channel, as a program that serves a model runs them.

A case names an operator, its sizes and its types:

    op        rmsnorm           y = h / sqrt(mean h^2 + eps) * gamma, h = x (+ residual)
              rmsnorm_quantize  the same, written as 8-bit codes with one scale per row
              quantize          rows to 8-bit codes and scales (activations without a norm in front, weights)
              linear            codes x codes -> results, scales and bias applied outside the integer sum
              layer             from the attention's output to fc1's: quantize, product, residual + norm + quantize, product
    rows, k   the activation matrix; n: output channels (linear, layer: of the second product; the first is k x k)
    type      bf16, fp16 or fp32: of activations, residual, results and bias
    residual, bias   whether there is one
    pad       extra elements between the rows of the activations (a column slice of a wider tensor)

Codes are returned as the values that they stand for, in 16 bits, next to their scales.
"""
import math

import torch

own = False

FRAME = 1374            # tokens of one image
SPECIAL = 5             # the first tokens of a frame, a hundred times as large as the others
EPS = 1e-6
TYPES = dict(bf16=torch.bfloat16, fp16=torch.float16, fp32=torch.float32)
BYTES = dict(bf16=2, fp16=2, fp32=4)
MAX_ELEMENTS = 32 * FRAME * 4096        # of the largest listed activation matrix
MAX_OPS = 2.0 * 8 * FRAME * 4096 * 4096     # of the largest listed product


def listed():
    return [
        # one new token behind the attention of a decoder: the smallest call, latency only
        dict(name="norm_one_token", op="rmsnorm", rows=1, k=4096, type="bf16", residual=True, pad=0),
        # a ragged batch of tokens of an odd width, sliced out of a wider tensor
        dict(name="norm_odd", op="rmsnorm", rows=FRAME + 77, k=1003, type="fp16", residual=False, pad=21),
        # the special tokens of eight frames: a small batch through the norm in front of qkv
        dict(name="norm8_special", op="rmsnorm_quantize", rows=8 * SPECIAL, k=1024, type="bf16", residual=True, pad=0),
        # eight frames at the width of the model
        dict(name="norm8_8f", op="rmsnorm_quantize", rows=8 * FRAME, k=1024, type="bf16", residual=True, pad=64),
        # 32 frames of a wide model: the largest activation
        dict(name="norm8_32f_wide", op="rmsnorm_quantize", rows=32 * FRAME, k=4096, type="bf16", residual=True, pad=0),
        # a weight matrix kept in 32 bits, quantized when a model is loaded
        dict(name="quantize_weights", op="quantize", rows=4096, k=1024, type="fp32", residual=False, pad=0),
        # the input of fc2 over eight frames
        dict(name="quantize_8f", op="quantize", rows=8 * FRAME, k=4096, type="fp16", residual=False, pad=0),
        # one token through a wide projection: the weights' bytes are all there is
        dict(name="linear_one_token", op="linear", rows=1, k=4096, n=4096, type="bf16", bias=False),
        # a decoding batch of odd sizes, results in 32 bits
        dict(name="linear_batch_odd", op="linear", rows=77, k=2011, n=5003, type="fp32", bias=True),
        # one frame through fc2
        dict(name="linear_frame", op="linear", rows=FRAME, k=4096, n=1024, type="fp16", bias=True),
        # eight frames through a square projection of a wide model: the largest product
        dict(name="linear_8f_wide", op="linear", rows=8 * FRAME, k=4096, n=4096, type="bf16", bias=True),
        # from the attention's output to fc1's over two frames less a few tokens
        dict(name="layer_2f", op="layer", rows=2 * FRAME - 17, k=1024, n=4096, type="bf16", residual=True, bias=True, pad=0),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def _width(rng, lo, hi):
    """A matrix width: a multiple of 64 or of 16 as often as any other number."""
    w = _spread(rng, lo, hi)
    step = rng.choice((1, 1, 16, 64))
    return max(lo, w - w % step)


def draw(rng):
    op = rng.choice(("rmsnorm", "rmsnorm_quantize", "quantize", "linear", "linear", "layer"))
    t = rng.choice(("bf16", "bf16", "fp16", "fp32" if op != "layer" else "bf16"))
    k = _width(rng, 64, 8192)
    case = dict(op=op, k=k, type=t)
    if op in ("linear", "layer"):
        n = _width(rng, 64, 8192)
        per_row = 2.0 * k * (n + (k if op == "layer" else 0))
        case.update(n=n, bias=rng.random() < 0.5, rows=_spread(rng, 1, min(32 * FRAME, MAX_OPS / per_row)))
    else:
        case["rows"] = _spread(rng, 1, min(32 * FRAME, MAX_ELEMENTS // k // (BYTES[t] // 2)))
    if op != "linear":
        case["pad"] = rng.choice((0, 0, 8, 21, 64))
        case["residual"] = op == "layer" or (op != "quantize" and rng.random() < 0.7)
    return case


def _activations(g, rows, k, pad, dtype, outliers=True):
    """Token rows with eight outlier channels (x50) and the special tokens of every frame (x100; x10 in fp16, whose range ends at 65504)."""
    x = torch.empty((rows, k + pad), dtype=dtype, device="cuda")
    step = max(1, (1 << 26) // (k + pad))
    hot = torch.randperm(k, generator=g, device="cuda")[:8]
    for m0 in range(0, rows, step):
        m1 = min(rows, m0 + step)
        v = torch.empty((m1 - m0, k + pad), dtype=torch.float32, device="cuda").normal_(generator=g)
        if outliers:
            v[:, hot] *= 50.0
            special = torch.arange(m0, m1, device="cuda") % FRAME < SPECIAL
            v *= torch.where(special, 10.0 if dtype == torch.float16 else 100.0, 1.0)[:, None]
        x[m0:m1] = v
    return x[:, :k]


def _codes(g, rows, k):
    """8-bit codes as a quantizer leaves them, rows 16 bytes apart or a multiple of that; every row reaches +-127."""
    q = torch.empty((rows, (k + 15) // 16 * 16), dtype=torch.int8, device="cuda")
    step = max(1, (1 << 26) // q.shape[1])
    for m0 in range(0, rows, step):
        v = torch.empty((min(rows, m0 + step) - m0, q.shape[1]), dtype=torch.float32, device="cuda").normal_(generator=g)
        q[m0:m0 + step] = (v * 32.0).round().clamp(-127, 127)
    q[:, 0] = 127
    return q[:, :k]


def _scales(g, n, size):
    return (torch.rand((n,), generator=g, device="cuda") * 0.5 + 0.75) * size


def _vector(g, n, mean, dev, dtype):
    return torch.empty((n,), dtype=torch.float32, device="cuda").normal_(mean, dev, generator=g).to(dtype)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    op, rows, k, dtype = case["op"], case["rows"], case["k"], TYPES[case["type"]]
    s = dict(op=op, type=dtype)

    def codes(m, w):
        return torch.empty((m, (w + 15) // 16 * 16), dtype=torch.int8, device="cuda")[:, :w]

    def results(m, w, kind):
        return torch.empty((m, (w + 7) // 8 * 8), dtype=kind, device="cuda")[:, :w]

    if op == "linear":
        n = case["n"]
        s.update(xq=_codes(g, rows, k), a=_scales(g, rows, 0.03), wq=_codes(g, n, k), w=_scales(g, n, 0.0006),
                 b=_vector(g, n, 0.0, 0.01, dtype) if case["bias"] else None, y=results(rows, n, dtype))
        return s
    s["x"] = _activations(g, rows, k, case["pad"], dtype)
    if op != "quantize":
        s["gamma"] = _vector(g, k, 1.0, 0.1, torch.float32)
        s["res"] = _activations(g, rows, k, case["pad"], dtype, False) if case["residual"] else None
        s["h"] = results(rows, k, dtype) if case["residual"] else None
    if op == "rmsnorm":
        s["y"] = results(rows, k, dtype)
    else:
        s.update(q=codes(rows, k), a=torch.empty((rows,), dtype=torch.float32, device="cuda"))
        s["v"] = results(rows, k, torch.bfloat16 if dtype == torch.float32 else dtype)
    if op == "layer":
        n = case["n"]
        s.update(wq1=_codes(g, k, k), w1=_scales(g, k, 0.0006), wq2=_codes(g, n, k), w2=_scales(g, n, 0.0006), o=results(rows, k, dtype),
                 y=results(rows, n, dtype), b1=_vector(g, k, 0.0, 0.01, dtype) if case["bias"] else None,
                 b2=_vector(g, n, 0.0, 0.01, dtype) if case["bias"] else None,
                 q2=codes(rows, k), a2=torch.empty((rows,), dtype=torch.float32, device="cuda"))
    return s


# ---------------------------------------------------------------- the plain forms: 32 bits, each output rounded once
def _plain_norm(x, res, gamma):
    h = x.float() if res is None else x.float() + res.float()
    return h * torch.rsqrt((h * h).mean(1, keepdim=True) + EPS) * gamma, h


def _plain_quantize(y):
    """Codes (as 32-bit floats) and scales."""
    amax = y.abs().amax(1).clamp_min(1e-8)
    return (y * (127.0 / amax)[:, None]).round().clamp_(-127, 127), amax / 127.0


def _plain_linear(q, a, wq, w, b, dtype):
    y = (q.float() @ wq.float().t()) * (a[:, None] * w[None, :])
    return (y if b is None else y + b.float()).to(dtype)


def _plain(s):
    op, dtype = s["op"], s["type"]
    if op == "linear":
        return _plain_linear(s["xq"], s["a"], s["wq"], s["w"], s["b"], dtype)
    if op == "quantize":
        q, a = _plain_quantize(s["x"].float())
        return (q * a[:, None]).to(s["v"].dtype), a
    if op == "layer":
        q, a = _plain_quantize(s["x"].float())
        o = _plain_linear(q, a, s["wq1"], s["w1"], s["b1"], dtype)
        y, h = _plain_norm(o, s["res"], s["gamma"])
        q, a = _plain_quantize(y)
        return _plain_linear(q, a, s["wq2"], s["w2"], s["b2"], dtype), h.to(dtype)
    y, h = _plain_norm(s["x"], s["res"], s["gamma"])
    more = () if s["res"] is None else (h.to(dtype),)
    if op == "rmsnorm":
        return (y.to(dtype),) + more
    q, a = _plain_quantize(y)
    return ((q * a[:, None]).to(s["v"].dtype), a) + more


def _own(s):
    import paper_2509_21302_b200 as q

    op = s["op"]
    if op == "linear":
        return q.linear_c8(s["xq"], s["a"], s["wq"], s["w"], s["b"], Y=s["y"])
    if op == "quantize":
        q.quantize_c8(s["x"], Xq8=s["q"], a_scale=s["a"])
        return q.dequantize_c8(s["q"], s["a"], Y=s["v"]), s["a"]
    if op == "layer":
        q.quantize_c8(s["x"], Xq8=s["q"], a_scale=s["a"])
        q.linear_c8(s["q"], s["a"], s["wq1"], s["w1"], s["b1"], Y=s["o"])
        q.rmsnorm_quantize_c8(s["o"], s["gamma"], EPS, s["res"], Xq8=s["q2"], a_scale=s["a2"], H=s["h"])
        return q.linear_c8(s["q2"], s["a2"], s["wq2"], s["w2"], s["b2"], Y=s["y"]), s["h"]
    more = () if s["res"] is None else (s["h"],)
    if op == "rmsnorm":
        q.rmsnorm(s["x"], s["gamma"], EPS, s["res"], Y=s["y"], H=s["h"])
        return (s["y"],) + more
    q.rmsnorm_quantize_c8(s["x"], s["gamma"], EPS, s["res"], Xq8=s["q"], a_scale=s["a"], H=s["h"])
    return (q.dequantize_c8(s["q"], s["a"], Y=s["v"]), s["a"]) + more


def run(state):
    return _own(state) if own else _plain(state)


def work(case):
    """Each input read once and each output written once, codes included where they are an output; integer operations of the products
    (elsewhere about six per element)."""
    op, m, k, e = case["op"], case["rows"], case["k"], BYTES[case["type"]]
    if op in ("linear", "layer"):
        n, b = case["n"], e * case["bias"]
        second = n * k + n * (4.0 + b) + m * n * e
        if op == "linear":
            return dict(bytes=m * (k + 4.0) + second, flops=2.0 * m * n * k)
        first = k * k + k * (4.0 + b) + 4.0 * k
        return dict(bytes=first + second + 3.0 * m * k * e, flops=2.0 * m * k * (k + n))
    h = 2.0 * e * m * k * case["residual"]                       # residual in, sum out
    if op == "rmsnorm":
        return dict(bytes=2.0 * e * m * k + h + 4.0 * k, flops=6.0 * m * k)
    # codes, the values that they stand for, scales
    return dict(bytes=m * k * (e + 3.0) + h + 4.0 * m + (4.0 * k if op == "rmsnorm_quantize" else 0.0), flops=6.0 * m * k)


# ---------------------------------------------------------------- the definitions in 64 bits
def _by_rows(rows, width, f):
    """f(m0, m1) -> arrays of rows m0 .. m1, put together; a slice holds at most 2^26 numbers."""
    outs, step = None, max(1, (1 << 26) // width)
    for m0 in range(0, rows, step):
        got = f(m0, min(rows, m0 + step))
        if outs is None:
            outs = [torch.empty((rows,) + tuple(v.shape[1:]), dtype=torch.float64, device="cuda") for v in got]
        for o, v in zip(outs, got):
            o[m0:m0 + step] = v
    return outs


def exact(case, seed):
    s = prepare(case, seed)
    op, rows, k, dtype = case["op"], case["rows"], case["k"], s["type"]
    f64 = torch.float64

    def steps_of(y):                                    # step size of each row, whole steps of each element
        step = torch.maximum(y.abs().max(dim=1, keepdim=True).values, torch.full((1, 1), 1e-8, dtype=f64, device="cuda")) / 127
        return step, torch.round(y / step)

    def normed(x, m0, m1):
        h = x if s["res"] is None else x + s["res"][m0:m1].to(f64)
        return h, h / torch.sqrt(h.square().sum(dim=1, keepdim=True) / k + EPS) * s["gamma"].to(f64)

    def product(q, step, wq, w, b):
        y = torch.einsum("mk,nk->mn", q, wq.to(f64)) * step * w.to(f64)
        return y if b is None else y + b.to(f64)

    def part(m0, m1):
        if op == "linear":
            return (product(s["xq"][m0:m1].to(f64), s["a"][m0:m1, None].to(f64), s["wq"], s["w"], s["b"]),)
        x = s["x"][m0:m1].to(f64)
        if op == "quantize":
            step, q = steps_of(x)
            return q * step, step[:, 0]
        if op == "layer":
            step, q = steps_of(x)
            o = product(q, step, s["wq1"], s["w1"], s["b1"]).to(dtype).to(f64)      # the first product's results are kept in the type
            h, y = normed(o, m0, m1)
            step, q = steps_of(y)
            return product(q, step, s["wq2"], s["w2"], s["b2"]), h
        h, y = normed(x, m0, m1)
        more = () if s["res"] is None else (h,)
        if op == "rmsnorm":
            return (y,) + more
        step, q = steps_of(y)
        return (q * step, step[:, 0]) + more

    got = _by_rows(rows, max(k, case.get("n", 0)), part)
    return got[0] if op == "linear" else tuple(got)
