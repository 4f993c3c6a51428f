"""Quantisation to and expansion from microscaled 4-bit floating point on the GPU: codes and scale bytes bit for bit, both directions, all
types, every length around a block and a row unit, strides, unaligned rows, special values, and what lies between and behind the rows."""
import numpy as np
import pytest

from oracle import mx_oracle as mx

pytestmark = pytest.mark.gpu
KINDS = {"f16": 0, "bf16": 1, "f32": 2}
UINT = {"f16": np.uint16, "bf16": np.uint16, "f32": np.uint32}


def bits_of(kind, shape, rng):
    """numbers with the magnitudes of weights, blocks of very different sizes, exact zeros and ties"""
    M, N = shape
    v = rng.standard_t(4, shape) * 0.02 * np.exp(rng.normal(size=(M, -(-N // 32))).repeat(32, axis=1)[:, :N] * 3)
    v[rng.random(shape) < 0.02] = 0.0
    ties = rng.random(shape) < 0.05
    v[ties] = np.ldexp(rng.choice([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.0], ties.sum()), -6) * rng.choice([-1, 1], ties.sum())
    return mx.from_double(v, kind)


def dtype_of(kind):
    import torch
    return {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}[kind]


def upload(bits, kind, ld=None, offset=0):
    """[M, N] on the GPU with row stride ld and the first element `offset` elements behind an aligned address; what is between holds NaN bits"""
    import torch
    M, N = bits.shape
    ld = ld or N
    flat = np.full(offset + max(M, 1) * ld + 8, np.iinfo(UINT[kind]).max, UINT[kind])
    for i in range(M):
        flat[offset + i * ld:offset + i * ld + N] = bits[i]
    t = torch.from_numpy(flat.view({2: np.int16, 4: np.int32}[flat.itemsize])).cuda().view(dtype_of(kind))
    return t[offset:offset + M * ld].view(M, ld)[:, :N] if M else t[:0].view(0, N)


def check(packed, v):
    code, scale = mx.quantize(v)
    assert np.array_equal(packed.scales.cpu().numpy(), scale)
    assert np.array_equal(packed.codes.cpu().numpy(), mx.pack(code))


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("M,N", [(1, 1), (1, 128), (3, 31), (5, 32), (5, 33), (2, 127), (129, 1), (128, 130), (130, 257), (31, 2049), (300, 1000), (1, 28673)])
def test_quantisation_in_both_directions(M, N, kind):
    import torch
    import paper_2306_07629_amd as sq
    print(f"mx quantize {M}x{N} {kind}", flush=True)
    bits = bits_of(kind, (M, N), np.random.default_rng(M * 1000 + N))
    v = mx.to_double(bits, kind)
    w = upload(bits, kind)
    check(sq.mx_quantize(w), v)
    check(sq.mx_quantize(w, "columns"), v.T)
    rows, columns = sq.mx_quantize(w, "both")
    check(rows, v)
    check(columns, v.T)
    torch.cuda.synchronize()


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("ld,offset", [(300, 1), (304, 0), (301, 0), (304, 8), (304, 4), (299, 0)])
def test_strided_and_unaligned_matrices(ld, offset, kind):
    import paper_2306_07629_amd as sq
    bits = bits_of(kind, (70, 299), np.random.default_rng(ld + offset))
    v = mx.to_double(bits, kind)
    w = upload(bits, kind, ld, offset)
    rows, columns = sq.mx_quantize(w, "both")
    check(rows, v)
    check(columns, v.T)
    check(sq.mx_quantize(w), v)
    # a transposed view has no contiguous rows: the binding copies it
    check(sq.mx_quantize(w.t()), v.T)


@pytest.mark.parametrize("kind", list(KINDS))
def test_every_end_of_a_row(kind):
    """rows that end at every place of a lane's eight elements, of one lane and of several, with NaN bits behind them"""
    import torch
    import paper_2306_07629_amd as sq
    for N in (*range(1, 26), *range(120, 138)):
        for M, ld, offset in ((9, N, 0), (140, N + 3, 1)):
            bits = bits_of(kind, (M, N), np.random.default_rng(N))
            v = mx.to_double(bits, kind)
            rows, columns = sq.mx_quantize(upload(bits, kind, ld, offset), "both")
            check(rows, v)
            check(columns, v.T)
            check(sq.mx_quantize(upload(bits, kind, ld, offset)), v)
            want = mx.from_double(mx.expand(rows.codes.cpu().numpy(), rows.scales.cpu().numpy(), N), kind)
            got = rows.dequantize(dtype_of(kind)).view(torch.int32 if kind == "f32" else torch.int16).cpu().numpy().view(UINT[kind])
            assert np.array_equal(mx.to_double(got, kind), mx.to_double(want, kind), equal_nan=True), (M, N)


@pytest.mark.parametrize("kind", list(KINDS))
def test_special_values(kind):
    """one kind of block per pair of rows and columns: zeros of both signs, subnormals, the largest numbers, infinities, NaNs, borders of the scale"""
    import paper_2306_07629_amd as sq
    rng = np.random.default_rng(3)
    big = {"f16": 65504.0, "bf16": 2.0 ** 127 * 1.9921875, "f32": float(np.finfo(np.float32).max)}[kind]
    tiny = {"f16": 2.0 ** -24, "bf16": 2.0 ** -133, "f32": 2.0 ** -149}[kind]
    blocks = [np.zeros(32), -np.zeros(32), rng.integers(-20, 20, 32) * tiny, rng.integers(-1, 2, 32) * tiny, rng.integers(-120, 120, 32) * tiny, rng.uniform(-1, 1, 32) * big, np.full(32, -big),
              np.where(np.arange(32) == 7, np.inf, 1.0), np.where(np.arange(32) == 31, -np.inf, big), np.where(np.arange(32) == 0, np.nan, 0.0), np.where(np.arange(32) == 0, big, tiny),
              np.ldexp(1.0, -np.arange(32) % 14), np.ldexp(1.999, -(np.arange(32) % 14)), rng.choice([2.0 ** -14, 2.0 ** -15, 2.0 ** -126, 2.0 ** -127], 32)]
    v = np.concatenate(blocks)[None, :].repeat(35, axis=0)
    v[1::2] *= np.where(np.isfinite(v[1::2]), rng.choice([-1, 1], v[1::2].shape), 1)
    bits = mx.from_double(v, kind)
    v = mx.to_double(bits, kind)
    w = upload(bits, kind)
    rows, columns = sq.mx_quantize(w, "both")
    check(rows, v)
    check(columns, v.T)
    check(sq.mx_quantize(w), v)


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("M,N", [(1, 1), (3, 7), (5, 32), (4, 129), (70, 299), (33, 4096)])
def test_expansion_of_every_code_and_scale(M, N, kind):
    import torch
    import paper_2306_07629_amd as sq
    print(f"mx dequantize {M}x{N} {kind}", flush=True)
    rng = np.random.default_rng(M + N)
    P = mx.padded(N)
    codes = rng.integers(0, 256, (M, P // 2), dtype=np.uint8)
    scales = rng.integers(0, 256, (M, P // 32), dtype=np.uint8)
    want = mx.expand(codes, scales, N)
    m = sq.MxMatrix(M, N, torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda())
    got = m.dequantize(dtype_of(kind)).cpu()
    gbits = got.view(torch.int32 if kind == "f32" else torch.int16).numpy().view(UINT[kind])
    nan = np.isnan(want)
    assert np.array_equal(np.isnan(mx.to_double(gbits, kind)), nan)
    assert np.array_equal(gbits[~nan], mx.from_double(want, kind)[~nan])


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("ld,offset", [(299, 0), (301, 1), (304, 0), (304, 3)])
def test_expansion_into_a_larger_matrix_leaves_the_rest_alone(ld, offset, kind):
    import torch
    import paper_2306_07629_amd as sq
    M, N = 37, 299
    rng = np.random.default_rng(ld)
    bits = bits_of(kind, (M, N), rng)
    m = sq.mx_quantize(upload(bits, kind))
    it = torch.int32 if kind == "f32" else torch.int16
    buf = torch.full((offset + M * ld + 64,), 0x5A5A, dtype=it, device="cuda")
    sq.sqllm_mx_dequantize(M, N, KINDS[kind], m.codes, m.scales, buf[offset:], ld)
    torch.cuda.synchronize()
    got = buf.cpu().numpy()
    inside = np.zeros(got.shape, bool)
    for i in range(M):
        inside[offset + i * ld:offset + i * ld + N] = True
    assert (got[~inside] == 0x5A5A).all()
    code, scale = mx.quantize(mx.to_double(bits, kind))
    want = mx.from_double(mx.expand(mx.pack(code), scale, N), kind)
    assert np.array_equal(got[inside].view(UINT[kind]).reshape(M, N), want)


def test_packed_arrays_are_written_to_their_end_and_no_further():
    import torch
    import paper_2306_07629_amd as sq
    M, N = 130, 200
    bits = bits_of("f16", (M, N), np.random.default_rng(1))
    w = upload(bits, "f16")
    bufs = []
    for rows, cols in ((M, N), (N, M)):
        for nbytes in sq.sqllm_mx_bytes(rows, cols):
            b = torch.full((nbytes + 512,), 0xA5, dtype=torch.uint8, device="cuda")
            bufs.append((b, nbytes))
    for given in ((0, 1), (0, 1, 2, 3), (2, 3)):
        for b, _ in bufs:
            b.fill_(0xA5)
        args = [bufs[k][0][256:] if k in given else None for k in range(4)]
        sq.sqllm_mx_quantize(M, N, 0, w, N, *args)
        torch.cuda.synchronize()
        v = mx.to_double(bits, "f16")
        for k, (b, nbytes) in enumerate(bufs):
            got = b.cpu().numpy()
            assert (got[:256] == 0xA5).all() and (got[256 + nbytes:] == 0xA5).all()
            if k in given:
                code, scale = mx.quantize(v if k < 2 else v.T)
                assert np.array_equal(got[256:256 + nbytes], (scale if k & 1 else mx.pack(code)).reshape(-1))
            else:
                assert (got == 0xA5).all()


def test_a_packed_matrix_behind_four_gigabytes():
    """offsets of rows beyond 2^32 bytes of input and 2^31 of codes: the last rows are right"""
    import torch
    import paper_2306_07629_amd as sq
    M, N = (1 << 19) + 300, 8192
    w = torch.zeros((M, N), dtype=torch.float16, device="cuda")
    bits = bits_of("f16", (300, N), np.random.default_rng(8))
    w[-300:] = upload(bits, "f16")
    q = sq.mx_quantize(w)
    del w
    code, scale = mx.quantize(mx.to_double(bits, "f16"))
    assert np.array_equal(q.scales[-300:].cpu().numpy(), scale) and np.array_equal(q.codes[-300:].cpu().numpy(), mx.pack(code))
    assert int(q.codes[:-300].max()) == 0 and int(q.scales[:-300].max()) == 0
    want = mx.expand(mx.pack(code), scale, N)                            # a few numbers left fp16: their blocks are NaN
    back = q.dequantize(torch.float16)[-300:].cpu().numpy().astype(np.float64)
    assert np.array_equal(back, want, equal_nan=True)
    x = torch.randn((N, 1), device="cuda").half()
    got = sq.mx_gemv(q, x).cpu().numpy().astype(np.float64)
    x64 = x.cpu().numpy().astype(np.float64)
    ref, S = want @ x64, np.abs(want) @ np.abs(x64)
    nan = np.isnan(ref)
    assert np.array_equal(np.isnan(got[-300:]), nan) and not nan.all() and (got[:-300] == 0).all()
    tol = 2.0 ** -11 * np.abs(ref) + 2.0 ** -25 + (64 + N / 64) * 2.0 ** -23 * S
    assert (np.abs(got[-300:] - ref) <= tol)[~nan & (np.abs(ref) < 65000)].all()
