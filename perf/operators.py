"""Microscaled 4-bit floating point next to the look-up tables: the calls of its users as cases that can be timed and compared.

A matrix in this format holds E2M1 codes (0, 0.5, 1, 1.5, 2, 3, 4, 6 and a sign), two to a byte, the even element in the low half, and one
scale byte per 32 neighbouring elements of a row, which stands for 2^(byte - 127).  A row is padded with zeros to a multiple of 128
elements.  One pass of a case is what a program does between two of its own steps: it quantises a matrix and reads the values back,
expands a packed matrix, multiplies a packed layer with one to sixteen fp16 columns, quantises the activations of many tokens and
multiplies them with a packed layer, or takes the three products of a linear layer's training step.  Weights are Student-t(4) of scale
0.02; activations are normal with a few wide channels; gradients are normal and small.  Everything is drawn on the GPU from the seed.
"""
import math

import torch

own = False

BLOCK = 32
ROW = 128                        # elements a packed row is padded to
MAX_WEIGHTS = 22016 * 8192
MAX_PRODUCT = 4096 * 22016 * 8192    # tokens x rows x columns of one pass
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


# ---------------------------------------------------------------------------------------------- the cases
def listed():
    return [
        # one token through a narrow projection: launch latency and the host's share of a call
        dict(name="gemv_256x4096", kind="gemv", M=256, N=4096, batch=1),
        # one token through the largest layer of a 65B-shaped model
        dict(name="gemv_22016x8192", kind="gemv", M=22016, N=8192, batch=1),
        # an odd batch of sequences on a 13B-shaped MLP projection, and a full one on a 65B-shaped attention projection
        dict(name="gemv_13824x5120_batch5", kind="gemv", M=13824, N=5120, batch=5),
        dict(name="gemv_8192x8192_batch16", kind="gemv", M=8192, N=8192, batch=16),
        # weights of a projection to the format and back, to judge what the format costs them
        dict(name="quantize_11008x4096_f16", kind="quantize", M=11008, N=4096, direction="rows", dtype="f16"),
        # a ragged matrix of activations along both of its axes, as a backward pass needs it
        dict(name="quantize_1999x5120_both_bf16", kind="quantize", M=1999, N=5120, direction="both", dtype="bf16"),
        # expansion of a packed layer for a product in fp16, and of a small one to fp32 for inspection
        dict(name="dequantize_13824x5120_f16", kind="dequantize", M=13824, N=5120, dtype="f16"),
        dict(name="dequantize_1000x2048_f32", kind="dequantize", M=1000, N=2048, dtype="f32"),
        # more sequences than the gemv takes: a decode step of 33 through an MLP projection
        dict(name="linear_33x11008x4096_f16", kind="linear", T=33, M=11008, N=4096, dtype="f16"),
        # a prefill of 4096 tokens through the largest layer
        dict(name="linear_4096x22016x8192_bf16", kind="linear", T=4096, M=22016, N=8192, dtype="bf16"),
        # forward and backward of an attention projection over one short sequence, and of an MLP projection over a ragged batch of tokens
        dict(name="train_301x5120x5120_f16", kind="train", T=301, M=5120, N=5120, dtype="f16"),
        dict(name="train_2047x4096x11008_bf16", kind="train", T=2047, M=4096, N=11008, dtype="bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    kind = rng.choice(["gemv", "gemv", "gemv", "quantize", "quantize", "dequantize", "linear", "linear", "linear", "train"])
    dtype = rng.choice(["f16", "bf16", "bf16", "f32"])
    if kind == "gemv":                # rows of any number, columns a multiple of 128 as for the other matvecs
        N = max(2, _log_int(rng, 256, 22016) // ROW) * ROW
        M = _log_int(rng, 200, min(22016, MAX_WEIGHTS // N))
        return dict(kind="gemv", M=M, N=N, batch=rng.choice([1, 1, rng.randint(2, 16)]))
    if kind in ("quantize", "dequantize"):
        N = _log_int(rng, 256, 11008)
        M = _log_int(rng, 200, min(13824, 13824 * 5120 // N))
        case = dict(kind=kind, M=M, N=N, dtype=dtype)
        if kind == "quantize":
            case["direction"] = rng.choice(["rows", "rows", "columns", "both"])
        return case
    N = _log_int(rng, 512, 11008)
    M = _log_int(rng, 512, min(22016, MAX_WEIGHTS // N))
    passes = 3 if kind == "train" else 1
    T = _log_int(rng, 17 if kind == "linear" else 256, min(8192, MAX_PRODUCT // (2 * passes * M * N)))
    return dict(kind=kind, T=T, M=M, N=N, dtype=dtype)


# ---------------------------------------------------------------------------------------------- inputs
def _weights(M, N, dtype, g):
    """Student-t with four degrees of freedom, scale 0.02: Z / sqrt(chi2_4 / 4), chi2_4 = -2 ln(u1 u2)"""
    z = torch.randn((M, N), generator=g, device="cuda")
    u = torch.rand((M, N), generator=g, device="cuda").clamp_(min=1e-7)
    u *= torch.rand((M, N), generator=g, device="cuda").clamp_(min=1e-7)
    return z.div_(u.log_().mul_(-0.5).sqrt_()).mul_(0.02).to(dtype)


def _activations(T, N, dtype, g):
    """N(0, 1), one channel in 128 twenty times as wide"""
    x = torch.randn((T, N), generator=g, device="cuda")
    wide = torch.rand((N,), generator=g, device="cuda") < 1.0 / 128.0
    return torch.where(wide, x * 20.0, x).to(dtype)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    kind = case["kind"]
    dtype = TYPES[case.get("dtype", "f16")]
    state = dict(case, dtype=dtype)
    if kind == "quantize":
        state["w"] = _weights(case["M"], case["N"], dtype, g)
        return state
    if kind == "train":
        state["w"] = _weights(case["M"], case["N"], dtype, g)
        state["x"] = _activations(case["T"], case["N"], dtype, g)
        state["dy"] = (torch.randn((case["T"], case["M"]), generator=g, device="cuda") * 1e-3).to(dtype)
        return state
    codes, scales = _pack(*_quantize(_weights(case["M"], case["N"], torch.float16, g)))
    state["codes"], state["scales"] = codes, scales
    if kind == "gemv":
        state["x"] = torch.randn((case["N"], case["batch"]), generator=g, device="cuda").to(torch.float16)
    elif kind == "linear":
        state["x"] = _activations(case["T"], case["N"], dtype, g)
    if own:
        import paper_2306_07629_amd as sq
        state["packed"] = sq.MxMatrix(case["M"], case["N"], codes, scales)
    return state


# ---------------------------------------------------------------------------------------------- the plain form
def _power_of_two(e):
    """2^e in 64 bits, exact"""
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _quantize(w):
    """(code values, their exponents) of the blocks of the rows: float32 [M, blocks, 32] on the E2M1 grid, int64 [M, blocks]"""
    M, N = w.shape
    v = torch.nn.functional.pad(w.float(), (0, -N % ROW)).view(M, -1, BLOCK)
    top = v.abs().amax(dim=2)
    e = (top.double().view(torch.int64) >> 52) - 1023 - 2               # exponent field: floor(log2), below everything for zero
    e = e.clamp(-127, 125)
    t = (v.double() / _power_of_two(e).unsqueeze(2)).float()
    a = t.abs()
    step = torch.where(a < 2.0, 0.5, torch.where(a < 4.0, 1.0, 2.0))
    q = (torch.round(a / step) * step).clamp(max=6.0)                   # half to even: an even multiple is an even code
    return torch.where(t < 0, -q, q), e


def _pack(q, e):
    M = q.shape[0]
    a = q.abs()
    code = torch.where(a < 2.0, a * 2.0, torch.where(a < 4.0, a + 2.0, a * 0.5 + 4.0)).to(torch.uint8)
    code = (code | ((q < 0).to(torch.uint8) << 3)).view(M, -1, 2)
    return code[:, :, 0] | (code[:, :, 1] << 4), (e + 127).to(torch.uint8)


def _values(q, e, N):
    """the numbers that codes and exponents stand for, in 32 bits"""
    return (q.double() * _power_of_two(e).unsqueeze(2)).float().view(q.shape[0], -1)[:, :N]


def _expand(codes, scales, N):
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=codes.device)
    grid = torch.cat([grid, -grid])
    M = codes.shape[0]
    pairs = torch.stack([grid[(codes & 15).long()], grid[(codes >> 4).long()]], dim=2).view(M, -1, BLOCK)
    return (pairs * _power_of_two(scales.to(torch.int64) - 127).float().unsqueeze(2)).view(M, -1)[:, :N]


def _round_trip(w):
    q, e = _quantize(w)
    return _values(q, e, w.shape[1])


def _run_plain(s):
    kind, dtype = s["kind"], s["dtype"]
    if kind == "quantize":
        rows = _round_trip(s["w"]).to(dtype) if s["direction"] != "columns" else None
        columns = _round_trip(s["w"].t()).to(dtype) if s["direction"] != "rows" else None
        return [v for v in (rows, columns) if v is not None]
    if kind == "train":
        x, w, dy = s["x"], s["w"], s["dy"]
        y = _round_trip(x) @ _round_trip(w).t()
        dx = _round_trip(dy) @ _round_trip(w.t()).t()
        dw = _round_trip(dy.t()) @ _round_trip(x.t()).t()
        return [y.to(dtype), dx.to(dtype), dw]
    w = _expand(s["codes"], s["scales"], s["N"])
    if kind == "dequantize":
        return w.to(dtype)
    if kind == "gemv":
        return (w @ s["x"].float()).to(torch.float16)
    return (_round_trip(s["x"]) @ w.t()).to(dtype)


# ---------------------------------------------------------------------------------------------- the framework's calls
def _run_own(s):
    import paper_2306_07629_amd as sq
    kind, dtype = s["kind"], s["dtype"]
    if kind == "quantize":
        packed = sq.mx_quantize(s["w"], s["direction"])
        return [p.dequantize(dtype) for p in (packed if s["direction"] == "both" else (packed,))]
    if kind == "train":
        x, x_t = sq.mx_quantize(s["x"], "both")
        w, w_t = sq.mx_quantize(s["w"], "both")
        y = sq.mx_gemm(x, w, dtype)
        dx, dw = sq.mx_linear_backward(s["dy"], x_t, w_t, dtype)
        return [y, dx, dw]
    if kind == "dequantize":
        return s["packed"].dequantize(dtype)
    if kind == "gemv":
        return sq.mx_gemv(s["packed"], s["x"])
    return sq.mx_linear(s["x"], s["packed"], dtype)


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---------------------------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    kind, M, N = case["kind"], case["M"], case["N"]
    size = {"f16": 2, "bf16": 2, "f32": 4}[case.get("dtype", "f16")]
    packed = M * N // 2 + M * ((N + BLOCK - 1) // BLOCK)
    if kind == "gemv":
        return {"bytes": packed + 2 * case["batch"] * (M + N), "flops": 2 * M * N * case["batch"]}
    if kind == "quantize":
        outputs = 2 if case["direction"] == "both" else 1
        return {"bytes": (1 + outputs) * M * N * size, "flops": 2 * outputs * M * N}
    if kind == "dequantize":
        return {"bytes": packed + M * N * size, "flops": M * N}
    T = case["T"]
    if kind == "linear":
        return {"bytes": packed + T * (M + N) * size, "flops": 2 * T * M * N}
    return {"bytes": (2 * T * (M + N) + M * N) * size + 4 * M * N, "flops": 6 * T * M * N}


# ---------------------------------------------------------------------------------------------- the definition in 64 bits
def _scale_value(byte):
    """2^(byte - 127), from a table"""
    return torch.tensor([2.0 ** (b - 127) for b in range(256)], dtype=torch.float64, device=byte.device)[byte]


def _nearest(w):
    """every entry replaced by what its block of 32 along the rows makes of it, in 64 bits"""
    M, N = w.shape
    blocks = -(-N // BLOCK)
    v = torch.zeros((M, blocks * BLOCK), dtype=torch.float64, device=w.device)
    v[:, :N] = w
    v = v.view(M, blocks, BLOCK)
    top = torch.maximum(v.amax(dim=2), -v.amin(dim=2))
    exponent = torch.frexp(top).exponent - 3                            # top = m 2^k with m in [1/2, 1): floor(log2) is k - 1
    exponent = torch.where(top == 0, -127, exponent).clamp(-127, 125)
    unit = _scale_value(exponent.long() + 127).unsqueeze(2)
    a = v.abs() / unit
    out = torch.zeros_like(a)
    # the borders lie half way between neighbours; on a border the neighbour with the even code is taken
    for border, even_above, gain in ((0.25, False, 0.5), (0.75, True, 0.5), (1.25, False, 0.5), (1.75, True, 0.5),
                                     (2.5, False, 1.0), (3.5, True, 1.0), (5.0, False, 2.0)):
        out += gain * ((a >= border) if even_above else (a > border)).double()
    return (torch.copysign(out, v) * unit).view(M, -1)[:, :N]


def _unpacked(s):
    """the numbers of a packed matrix, in 64 bits, from the fields of its codes"""
    c = torch.stack([s["codes"] & 15, s["codes"] >> 4], dim=2).view(s["M"], -1).to(torch.int64)
    field, low = (c >> 1) & 3, (c & 1).double()
    magnitude = torch.where(field == 0, 0.5 * low, (1.0 + 0.5 * low) * _scale_value(field + 126))
    v = torch.where(c >= 8, -magnitude, magnitude).view(s["M"], -1, BLOCK)
    return (v * _scale_value(s["scales"].long()).unsqueeze(2)).view(s["M"], -1)[:, :s["N"]]


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "quantize":
        out = [] if case["direction"] == "columns" else [_nearest(s["w"])]
        return out if case["direction"] == "rows" else out + [_nearest(s["w"].t())]
    if kind == "train":
        x, w, dy = s["x"], s["w"], s["dy"]
        return [torch.mm(_nearest(x), _nearest(w).t()), torch.mm(_nearest(dy), _nearest(w.t()).t()),
                torch.mm(_nearest(dy.t()), _nearest(x.t()).t())]
    if kind == "dequantize":
        return _unpacked(s)
    if kind == "gemv":
        return torch.mm(_unpacked(s), s["x"].double())
    return torch.mm(_nearest(s["x"]), _unpacked(s).t())
