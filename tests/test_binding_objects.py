"""Objects of one type that are now a stream, now a tensor, whichever comes first (on the CPU: calls that are refused before anything is launched)."""
from types import SimpleNamespace

import pytest

import paper_2111_05972_amd as pkg


def _call(inp, stream=None):
    return pkg.tp_layer_dropout_fwd(pkg.TPL_BF16, 8, 64, 0.5, 4096, 0, 0, 0, 64, inp, None, None, 4096, stream=stream, check=False)


def test_streams_and_tensors_of_one_type():
    stream, tensor = SimpleNamespace(cuda_stream=0), SimpleNamespace(data_ptr=lambda: 4097)
    for _ in range(2):
        assert _call(tensor) == pkg.TPL_EALIGN
        assert _call(4097, stream) == pkg.TPL_EALIGN
        assert _call(tensor, stream) == pkg.TPL_EALIGN
        with pytest.raises(TypeError):
            _call(SimpleNamespace())


def test_errors_of_a_stream():
    class Broken:
        @property
        def cuda_stream(self):
            raise ValueError("gone")

    with pytest.raises(ValueError):
        _call(4097, Broken())
