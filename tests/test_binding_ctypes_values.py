"""Numbers and addresses that ctypes made are taken by their values (on the CPU: calls that are refused before anything is launched)."""
import ctypes as c

import pytest

import paper_2111_05972_amd as pkg


def _call(inp=4097, M=8, p=0.5, dtype=pkg.TPL_BF16):
    return pkg.tp_layer_dropout_fwd(dtype, M, 64, p, 4096, 0, 0, 0, 64, inp, None, None, 4096, check=False)


@pytest.mark.parametrize("make", [c.c_int64, c.c_int32, c.c_size_t, c.c_uint8, c.c_short])
def test_numbers(make):
    assert _call(M=make(8)) == pkg.TPL_EALIGN and _call(M=make(0)) == pkg.TPL_EINVAL
    assert _call(dtype=make(1)) == pkg.TPL_EALIGN and _call(dtype=make(5)) == pkg.TPL_EINVAL
    assert pkg.tp_layer_dropout_workspace_bytes(make(8), make(64)) == pkg.tp_layer_dropout_workspace_bytes(8, 64)


@pytest.mark.parametrize("make", [c.c_float, c.c_double])
def test_real_numbers(make):
    assert _call(p=make(0.5)) == pkg.TPL_EALIGN and _call(p=make(1.0)) == pkg.TPL_EINVAL


@pytest.mark.parametrize("make", [c.c_void_p, c.c_size_t, c.c_uint64])
def test_addresses(make):
    assert _call(make(4097)) == pkg.TPL_EALIGN and _call(make(0)) == pkg.TPL_EINVAL


def test_what_does_not_fit():
    with pytest.raises(OverflowError):
        _call(M=c.c_uint64(2 ** 63))
    with pytest.raises(OverflowError):
        _call(dtype=c.c_int64(2 ** 31))
    for bad in (c.c_double(8.0), c.c_char_p(b"8"), c.c_void_p(None)):
        with pytest.raises(TypeError):
            _call(M=bad)


# An attribute of that name alone makes no number of an object.
def test_others_are_refused():
    class Value:
        value = 8

    for kw in (dict(M=Value()), dict(p=Value()), dict(inp=Value())):
        with pytest.raises(TypeError):
            _call(**kw)
