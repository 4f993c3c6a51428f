"""Arguments of the backward products that are refused before anything is launched (no GPU)."""
import pytest
import torch

import paper_2306_07629_amd as sq
from paper_2306_07629_amd import binding
from test_mx_boundary import fake, packed, status

T, M, N = 6, 5, 300


@pytest.mark.parametrize("name,change", [("TYPE", dict(dw=fake(M, N, dtype=torch.float16))), ("TYPE", dict(dw=fake(M, N, dtype=torch.bfloat16))), ("TYPE", dict(dw=fake(M, N, dtype=torch.float64))),
                                         ("SHAPE", dict(dw=fake(N, M, dtype=torch.float32))), ("SHAPE", dict(dw=fake(M, N + 1, dtype=torch.float32))), ("DEVICE", dict(dw=torch.zeros(M, N))),
                                         ("SHAPE", dict(x_t=packed(N + 1, T))), ("SHAPE", dict(x_t=packed(N, T + 1))), ("SHAPE", dict(w_t=packed(N, M + 1)))])
def test_refused_before_dy_is_packed(name, change, monkeypatch):
    def launched(*args):
        raise AssertionError("reached the library")
    monkeypatch.setattr(sq.mx, "_call", launched)
    good = dict(dy=fake(T, M, dtype=torch.float16), x_t=packed(N, T), w_t=packed(N, M), dw=fake(M, N, dtype=torch.float32))
    with pytest.raises(AssertionError, match="reached"):
        sq.mx_linear_backward(**good)
    assert status(sq.mx_linear_backward, **{**good, **change}) == "SQLLM_ERR_" + name


def refused(name, fn, *args, **kw):
    """as status(), without keeping the error, whose traceback would keep GPU tensors alive in a cycle that is freed at some later time"""
    try:
        fn(*args, **kw)
    except sq.SqllmError as e:
        return binding.STATUS_NAMES[e.status] == "SQLLM_ERR_" + name
    return False


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_a_refused_sum_of_gradients_is_left_as_it_was(dtype):
    x, w, dy = (torch.ones(s, dtype=dtype, device="cuda") for s in ((T, N), (M, N), (T, M)))
    x_t, w_t = sq.mx_quantize(x, "columns"), sq.mx_quantize(w, "columns")
    dw = torch.full((M, N), 3.0, dtype=dtype, device="cuda")
    assert refused("TYPE", sq.mx_linear_backward, dy, x_t, w_t, dw=dw)
    assert bool((dw == 3.0).all())
    held = dw.float()
    assert sq.mx_linear_backward(dy, x_t, w_t, dw=held)[1] is held and bool((held == 3.0 + T).all())
