"""Packed products and autograd on the GPU: the calls take operands that require gradients and record nothing; a program's own autograd function gets the
gradients from mx_linear_backward."""
import numpy as np
import pytest

from oracle import mx_oracle as mx
from test_gpu_mx_products import close, host

pytestmark = pytest.mark.gpu


def leaf(shape, seed, scale=1.0):
    import torch
    return (torch.randn(shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)) * scale).half().requires_grad_()


def test_nothing_is_recorded():
    import torch
    import paper_2306_07629_amd as sq
    x, w, col, y = leaf((6, 256), 1), leaf((40, 256), 2), leaf((256, 3), 3), leaf((6, 40), 4)
    packed, packed_t = sq.mx_quantize(w, "both")
    _, x_t = sq.mx_quantize(x, "both")
    before = y.detach().clone()
    results = [packed.dequantize(), sq.mx_gemv(packed, col), sq.mx_linear(x, packed), *sq.mx_linear_backward(y, x_t, packed_t)]
    assert not any(t.requires_grad or t.grad_fn is not None for t in results)
    assert sq.mx_gemm(sq.mx_quantize(x), packed, y=y, accumulate=True) is y and y.is_leaf and not torch.equal(y, before)
    empty = sq.mx_quantize(x[:, :0])
    assert sq.mx_gemm(empty, sq.mx_quantize(w[:, :0]), y=y) is y and y.is_leaf and not bool(y.any())
    assert all(t.grad is None for t in (x, w, col, y))


def test_a_layer_with_gradients():
    import torch
    import paper_2306_07629_amd as sq

    class Linear(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, w):
            x, ctx.x_t = sq.mx_quantize(x, "both")
            w, ctx.w_t = sq.mx_quantize(w, "both")
            return sq.mx_gemm(x, w)

        @staticmethod
        def backward(ctx, dy):
            dx, dw = sq.mx_linear_backward(dy, ctx.x_t, ctx.w_t)
            return dx, dw.half()
    x, w, dy = leaf((70, 300), 1), leaf((130, 300), 2, 0.02), leaf((70, 130), 3, 1e-2).detach()
    y = Linear.apply(x, w)
    y.backward(dy)

    def q(a):
        code, scale = mx.quantize(a)
        return mx.expand(mx.pack(code), scale, a.shape[1])
    X, W, G = host(x), host(w), host(dy)
    for got, a, b in ((y, q(X), q(W)), (x.grad, q(G), q(np.ascontiguousarray(W.T))), (w.grad, q(np.ascontiguousarray(G.T)), q(np.ascontiguousarray(X.T)))):
        # dw is rounded to fp32 before fp16: half a step of fp32 more
        S = np.abs(a) @ np.abs(b).T
        close(host(got), a @ b.T, S, a.shape[1], extra=2.0 ** -24 * S)


@pytest.mark.parametrize("T,M", [(1, 1), (1, 130), (70, 1), (70, 130)])
def test_a_broadcast_gradient(T, M):
    """what y.sum().backward() hands on: one number with strides of zero"""
    import torch
    import paper_2306_07629_amd as sq
    x, w = leaf((T, 300), 1).detach(), leaf((M, 300), 2).detach()
    x_t, w_t = sq.mx_quantize(x, "columns"), sq.mx_quantize(w, "columns")
    one = torch.ones((), dtype=torch.float16, device="cuda").expand(T, M)
    got = sq.mx_linear_backward(one, x_t, w_t)
    want = sq.mx_linear_backward(one.clone(memory_format=torch.contiguous_format), x_t, w_t)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    near = host(x_t.dequantize(torch.float32)).sum(axis=1)
    close(host(got[1]), np.broadcast_to(near, (M, 300)), np.broadcast_to(np.abs(host(x_t.dequantize(torch.float32))).sum(axis=1), (M, 300)), T, "f32")
