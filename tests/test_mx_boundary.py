"""Arguments of the microscaled 4-bit entry points that are refused on the host (no kernel is launched by any test in this file)."""
import pytest
import torch

import paper_2306_07629_amd as sq
from paper_2306_07629_amd import binding

A = 1 << 20   # an aligned, never dereferenced device address


def status(fn, *args, **kw):
    with pytest.raises(sq.SqllmError) as e:
        fn(*args, **kw)
    assert len(str(e.value)) > 20
    return binding.STATUS_NAMES[e.value.status]


@pytest.mark.parametrize("M,N,codes,scales", [(0, 1, 0, 0), (1, 1, 64, 4), (3, 128, 192, 12), (3, 129, 384, 24), (22016, 8192, 22016 * 4096, 22016 * 256), (2, 0x7FFFFF80, 0x7FFFFF80, 0x7FFFFF8),
                                              (0x7FFFFFFF, 128, 0x7FFFFFFF * 64, 0x7FFFFFFF * 4)])
def test_sizes(M, N, codes, scales):
    assert sq.sqllm_mx_bytes(M, N) == (codes, scales)


def test_sizes_refused():
    for M, N in ((-1, 128), (4, 0), (4, -3), (4, 0x7FFFFF81)):
        assert status(sq.sqllm_mx_bytes, M, N) == "SQLLM_ERR_SHAPE"
    assert sq.lib().sqllm_mx_bytes(4, 128, None, None) == binding.STATUS_NAMES.index("SQLLM_ERR_NULL")


QUANT = dict(M=4, N=100, type=0, w=A, ldw=100, codes=A, scales=A, codes_t=A, scales_t=A, stream=0)
DEQUANT = dict(M=4, N=100, type=0, codes=A, scales=A, w_out=A, ldw=100, stream=0)
GEMV = dict(M=4, N=128, B=2, codes=A, scales=A, x=A, y=A, accumulate=0, stream=0)
GEMM = dict(T=3, M=4, N=100, type=2, x_codes=A, x_scales=A, w_codes=A, w_scales=A, y=A, ldy=4, accumulate=0, stream=0)


@pytest.mark.parametrize("fn,base,name,change", [
    (f, b, n, c) for f, b, cases in (
        ("sqllm_mx_quantize", QUANT, [("SHAPE", dict(M=-1)), ("SHAPE", dict(N=0)), ("SHAPE", dict(ldw=99)), ("SHAPE", dict(ldw=-1)), ("SHAPE", dict(ldw=1 << 41)), ("TYPE", dict(type=3)), ("TYPE", dict(type=-1)),
                                      ("NULL", dict(w=None)), ("NULL", dict(codes=None)), ("NULL", dict(scales=None)), ("NULL", dict(codes_t=None)), ("NULL", dict(scales_t=None)),
                                      ("NULL", dict(codes=None, scales=None, codes_t=None, scales_t=None)), ("ALIGN", dict(w=A + 1)), ("ALIGN", dict(w=A + 2, type=2)), ("ALIGN", dict(codes=A + 8)),
                                      ("ALIGN", dict(scales=A + 2)), ("ALIGN", dict(codes_t=A + 4)), ("ALIGN", dict(scales_t=A + 1)), ("SHAPE", dict(M=0x7FFFFF81)), ("SHAPE", dict(N=0x7FFFFF81, ldw=1 << 32))]),
        ("sqllm_mx_dequantize", DEQUANT, [("SHAPE", dict(M=-1)), ("SHAPE", dict(N=-5)), ("SHAPE", dict(ldw=99)), ("TYPE", dict(type=7)), ("NULL", dict(codes=None)), ("NULL", dict(scales=None)), ("NULL", dict(w_out=None)),
                                          ("ALIGN", dict(w_out=A + 1)), ("ALIGN", dict(w_out=A + 2, type=2)), ("ALIGN", dict(codes=A + 1)), ("ALIGN", dict(scales=A + 2))]),
        ("sqllm_mx_gemv", GEMV, [("SHAPE", dict(M=-1)), ("SHAPE", dict(N=0)), ("SHAPE", dict(N=100)), ("SHAPE", dict(N=28672 + 128)), ("BATCH", dict(B=0)), ("BATCH", dict(B=17)), ("NULL", dict(codes=None)),
                                 ("NULL", dict(scales=None)), ("NULL", dict(x=None)), ("NULL", dict(y=None)), ("ALIGN", dict(codes=A + 8)), ("ALIGN", dict(scales=A + 2)), ("ALIGN", dict(x=A + 8)), ("ALIGN", dict(y=A + 1))]),
        ("sqllm_mx_gemm", GEMM, [("SHAPE", dict(T=-1)), ("SHAPE", dict(M=-1)), ("SHAPE", dict(N=0)), ("SHAPE", dict(ldy=3)), ("TYPE", dict(type=9)), ("NULL", dict(x_codes=None)), ("NULL", dict(x_scales=None)),
                                 ("NULL", dict(w_codes=None)), ("NULL", dict(w_scales=None)), ("NULL", dict(y=None)), ("ALIGN", dict(x_codes=A + 8)), ("ALIGN", dict(w_scales=A + 2)), ("ALIGN", dict(y=A + 2)),
                                 ("ALIGN", dict(y=A + 1, type=1))])) for n, c in cases])
def test_refusals(fn, base, name, change):
    assert status(getattr(sq, fn), **dict(base, **change)) == "SQLLM_ERR_" + name


def test_empty_problems_are_ok_without_a_device():
    sq.sqllm_mx_quantize(**dict(QUANT, M=0))
    sq.sqllm_mx_dequantize(**dict(DEQUANT, M=0))
    sq.sqllm_mx_gemv(**dict(GEMV, M=0))
    sq.sqllm_mx_gemm(**dict(GEMM, T=0))
    sq.sqllm_mx_gemm(**dict(GEMM, M=0, ldy=0))


def test_empty_problems_need_no_addresses():
    """arrays of no elements have none to give"""
    none = dict.fromkeys(("w", "codes", "scales", "codes_t", "scales_t", "w_out", "x", "y", "x_codes", "x_scales", "w_codes", "w_scales"))
    for fn, base, empty in ((sq.sqllm_mx_quantize, QUANT, "M"), (sq.sqllm_mx_dequantize, DEQUANT, "M"), (sq.sqllm_mx_gemv, GEMV, "M"), (sq.sqllm_mx_gemm, GEMM, "M"), (sq.sqllm_mx_gemm, GEMM, "T")):
        fn(**dict({k: none.get(k, v) for k, v in base.items()}, **{empty: 0}))


def test_status_name():
    assert sq.lib().sqllm_status_string(9) == b"SQLLM_ERR_TYPE" and binding.STATUS_NAMES[9] == "SQLLM_ERR_TYPE"


class OnGpu(torch.Tensor):
    """a CPU tensor that passes for one on a GPU, for the checks that come before any call"""
    is_cuda = True


def fake(*shape, dtype=torch.uint8):
    return torch.zeros(shape, dtype=dtype).as_subclass(OnGpu)


def packed(M, N):
    P = -(-N // 128) * 128
    return sq.MxMatrix(M, N, fake(M, P // 2), fake(M, P // 32))


def test_packed_matrices_are_checked():
    packed(3, 130)
    assert status(sq.MxMatrix, 3, 130, fake(3, 64), fake(3, 8)) == "SQLLM_ERR_SHAPE"
    assert status(sq.MxMatrix, 3, 130, fake(3, 128), fake(3, 4)) == "SQLLM_ERR_SHAPE"
    assert status(sq.MxMatrix, 3, 130, fake(128, 3).t(), fake(3, 8)) == "SQLLM_ERR_SHAPE"
    assert status(sq.MxMatrix, 3, 0, fake(3, 0), fake(3, 0)) == "SQLLM_ERR_SHAPE"
    assert status(sq.MxMatrix, 3, 130, fake(3, 128, dtype=torch.int8), fake(3, 8)) == "SQLLM_ERR_TYPE"
    assert status(sq.MxMatrix, 3, 130, torch.zeros((3, 128), dtype=torch.uint8), fake(3, 8)) == "SQLLM_ERR_DEVICE"


@pytest.mark.parametrize("M,N", [(1 << 31, 128), (1 << 32, 1), (3, (1 << 31) - 127), (1, (1 << 32) + 128), (-1, 128), (0, 0)])
def test_sizes_beyond_the_librarys_are_refused(M, N):
    for make in (lambda: sq.MxMatrix.empty(M, N, "cpu"), lambda: sq.MxMatrix(M, N, fake(1, 64), fake(1, 4))):
        assert status(make) == "SQLLM_ERR_SHAPE"


def test_operands_are_checked():
    f16 = dict(dtype=torch.float16)
    assert status(sq.mx_quantize, torch.zeros(3, 4)) == "SQLLM_ERR_DEVICE"
    assert status(sq.mx_quantize, fake(3, 4, dtype=torch.float64)) == "SQLLM_ERR_TYPE"
    assert status(sq.mx_quantize, fake(3, **f16)) == "SQLLM_ERR_SHAPE"
    with pytest.raises(ValueError):
        sq.mx_quantize(fake(3, 4, **f16), "diagonal")
    assert status(packed(3, 130).dequantize, torch.float64) == "SQLLM_ERR_TYPE"
    w = packed(5, 256)
    assert status(sq.mx_gemv, w, fake(128, 1, **f16)) == "SQLLM_ERR_SHAPE"
    assert status(sq.mx_gemv, w, fake(256, **f16)) == "SQLLM_ERR_SHAPE"
    assert status(sq.mx_gemv, w, fake(256, 1, dtype=torch.bfloat16)) == "SQLLM_ERR_TYPE"
    assert status(sq.mx_gemv, w, fake(256, 1, **f16), fake(4, 1, **f16)) == "SQLLM_ERR_SHAPE"
    assert status(sq.mx_gemv, w, fake(256, 2, **f16), fake(2, 5, **f16).t()) == "SQLLM_ERR_SHAPE"
    assert status(sq.mx_gemv, w, fake(256, 1, **f16), None, True) == "SQLLM_ERR_NULL"
    assert status(sq.mx_gemm, packed(3, 128), w) == "SQLLM_ERR_SHAPE"
    assert status(sq.mx_gemm, packed(3, 256), w, torch.int8) == "SQLLM_ERR_TYPE"
    assert status(sq.mx_gemm, packed(3, 256), w, accumulate=True) == "SQLLM_ERR_NULL"
    assert status(sq.mx_gemm, packed(3, 256), w, y=fake(3, 4, **f16)) == "SQLLM_ERR_SHAPE"
    assert status(sq.mx_gemm, packed(3, 256), w, y=fake(5, 3, **f16).t()) == "SQLLM_ERR_SHAPE"
    assert status(sq.mx_gemm, packed(3, 256), w, y=fake(1, 5, **f16).expand(3, 5)) == "SQLLM_ERR_SHAPE"
    assert status(sq.mx_gemm, packed(3, 256), w, y=fake(3, 5, dtype=torch.int32)) == "SQLLM_ERR_TYPE"
    assert status(sq.mx_linear_backward, fake(3, 6, **f16), packed(256, 3), packed(256, 5)) == "SQLLM_ERR_SHAPE"
