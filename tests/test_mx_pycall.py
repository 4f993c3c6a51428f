"""The native call path of the sqllm_mx_* entry points takes and refuses the arguments that the ctypes path takes and refuses.  No GPU: every
call here fails validation on the host, or is not for the native path."""
import ctypes

import numpy as np
import pytest

import paper_2306_07629_amd as sq
from paper_2306_07629_amd import binding, build

A = 4096
GOOD = [dict(M=4, N=100, type=0, w=A, ldw=100, codes=A, scales=A, codes_t=None, scales_t=None, stream=0),
        dict(M=4, N=100, type=0, codes=A, scales=A, w_out=A, ldw=100, stream=0),
        dict(M=4, N=128, B=2, codes=A, scales=A, x=A, y=A, accumulate=0, stream=0),
        dict(T=3, M=4, N=100, type=2, x_codes=A, x_scales=A, w_codes=A, w_scales=A, y=A, ldy=4, accumulate=0, stream=0)]


class Tensor:
    def __init__(self, p):
        self.p = p

    def data_ptr(self):
        return self.p


class Stream:
    cuda_stream = 0


@pytest.fixture(scope="module")
def native():
    if build.pycall_is_stale():
        build.build_pycall()
    from paper_2306_07629_amd import _pycall
    asked = []
    L = sq.lib()
    _pycall.bind_mx(*[ctypes.cast(getattr(L, n), ctypes.c_void_p).value for n in binding._MX_ENTRIES], lambda: 3, lambda dev: asked.append(dev) or 0)
    yield _pycall.mx, asked
    binding._mx_call = binding._mx_first                                 # binds again, to the real streams


@pytest.mark.parametrize("entry,change", [(0, dict(type=3)), (0, dict(N=0)), (0, dict(ldw=99)), (0, dict(ldw=1 << 41)), (0, dict(M=-1)), (0, dict(w=None)), (0, dict(w=A + 1)), (0, dict(codes=None)),
                                          (0, dict(codes=Tensor(A + 8))), (0, dict(scales=A + 1)), (0, dict(codes_t=A)), (0, dict(type=True, w=Tensor(A + 1))), (0, dict(type=9, stream=Stream())), (0, dict(N=(1 << 32) - 5)),
                                          (1, dict(w_out=None)), (1, dict(ldw=-1)), (1, dict(codes=Tensor(0))), (1, dict(type=-1)), (1, dict(scales=A + 2)),
                                          (2, dict(B=17)), (2, dict(N=100)), (2, dict(x=A + 8)), (2, dict(y=None)), (2, dict(codes=A + 4)),
                                          (3, dict(ldy=3)), (3, dict(T=-1)), (3, dict(y=A + 2)), (3, dict(w_scales=None)), (3, dict(x_codes=A + 1)), (3, dict(type=77))])
def test_same_status_and_message_as_ctypes(native, entry, change):
    args = list({**GOOD[entry], **change}.values())
    want = binding._mx_ctypes(entry, *args)
    text = sq.lib().sqllm_last_error_string()
    assert want != 0
    assert native[0](entry, *args) == want and sq.lib().sqllm_last_error_string() == text


@pytest.mark.parametrize("entry", range(4))
@pytest.mark.parametrize("change", [dict(M=4.0), dict(N="128"), dict(M=np.int64(3)), dict(stream=Tensor(0))])
def test_other_arguments_are_left_to_ctypes(native, entry, change):
    bad = {"type": 9} if entry != 2 else {"B": 99}                       # no launch, whichever path
    args = list({**GOOD[entry], **bad, **change}.values())
    try:
        got = native[0](entry, *args)
    except AttributeError:
        with pytest.raises(AttributeError):
            binding._mx_ctypes(entry, *args)
        return
    assert got is None
    if isinstance(change.get("M"), np.integer):                          # ctypes takes what has an index
        assert binding._mx_ctypes(entry, *args) == (6 if entry == 2 else 9)
    else:
        with pytest.raises((ctypes.ArgumentError, AttributeError)):
            binding._mx_ctypes(entry, *args)


def test_unknown_entries_and_counts_are_left_alone(native):
    mx = native[0]
    assert mx() is None and mx("2") is None and mx(4, 0) is None and mx(-1) is None and mx(2) is None
    assert mx(2, *list(GOOD[2].values())[:-1]) is None and mx(0, *GOOD[0].values(), 0) is None


def test_current_stream_is_asked_for_the_current_device(native):
    del native[1][:]
    assert native[0](2, *{**GOOD[2], "B": 99, "stream": None}.values()) == 6
    assert native[1] == [3]


def test_errors_of_data_ptr_arrive(native):
    class Gone:
        def data_ptr(self):
            raise RuntimeError("freed")
    with pytest.raises(RuntimeError, match="freed"):
        native[0](2, *{**GOOD[2], "x": Gone()}.values())
