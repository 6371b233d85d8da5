"""What the binding takes for a pointer and for a number (on the CPU: calls that are refused before anything is launched)."""
import ctypes

import numpy as np
import pytest

import paper_2111_05972_amd as pkg


class Tensor:
    def __init__(self, at):
        self.at = at

    def data_ptr(self):
        return self.at


class Stream:
    cuda_stream = 0


def _call(inp, out=4096, stream=None, M=8, p=0.5):
    return pkg.tp_layer_dropout_fwd(pkg.TPL_BF16, M, 64, p, 4096, 0, 0, 0, 64, inp, None, None, out, stream=stream, check=False)


# An address that is not a multiple of 16 is refused for that: it has arrived.
@pytest.mark.parametrize("make", [int, np.int64, np.uint64, Tensor, ctypes.c_void_p])
def test_addresses(make):
    assert _call(make(4096 + 1)) == pkg.TPL_EALIGN
    assert _call(4096, out=make(4096 + 1)) == pkg.TPL_EALIGN
    assert _call(make(0)) == pkg.TPL_EINVAL


@pytest.mark.parametrize("stream", [None, 0, Stream(), ctypes.c_void_p(0), ctypes.c_void_p(None), np.int64(0)])
def test_streams(stream):
    for _ in range(2):
        assert _call(4097, stream=stream) == pkg.TPL_EALIGN


def test_none_is_null():
    assert _call(None) == pkg.TPL_EINVAL


@pytest.mark.parametrize("bad", [object(), "a", [4096], b"12a"])
def test_others_are_refused(bad):
    with pytest.raises(TypeError):
        _call(bad)


def test_numbers():
    assert _call(4097, M=np.int64(8)) == pkg.TPL_EALIGN
    assert _call(4097, p=np.float64(0.5)) == pkg.TPL_EALIGN and _call(4097, p=0) == pkg.TPL_EALIGN
    for M in (1 << 63, -(1 << 63) - 1, 1 << 70):
        with pytest.raises(OverflowError):
            _call(4097, M=M)
    for M in (8.0, "8", None):
        with pytest.raises(TypeError):
            _call(4097, M=M)


# An error inside data_ptr() is the caller's to see.
def test_errors_of_data_ptr():
    class Broken:
        def data_ptr(self):
            raise ValueError("gone")

    with pytest.raises(ValueError):
        _call(Broken())
