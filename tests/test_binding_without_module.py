"""The binding where the module that calls the library is not built for this Python: the same calls through ctypes, with the same arguments."""
import sys

import pytest

import paper_2111_05972_amd as pkg
import test_abi_block_host as block
import test_abi_packed_host as packed
import test_abi_window_host as window
import test_binding_ctypes_values as numbers
import test_binding_pointers as pointers
from paper_2111_05972_amd import binding


@pytest.fixture(autouse=True)
def without_module(monkeypatch):
    monkeypatch.setitem(sys.modules, "paper_2111_05972_amd._calls", None)        # an import of it fails
    monkeypatch.delattr(pkg, "_calls", raising=False)
    monkeypatch.setattr(binding, "_lib", None)
    assert not type(pkg.load_library().tp_layer_dropout_fwd).__name__.startswith("builtin")


def _cases():
    for m in (pointers, numbers, block, window, packed):
        for name in sorted(vars(m)):
            if not name.startswith("test_"):
                continue
            marks = [k for k in getattr(getattr(m, name), "pytestmark", []) if k.name == "parametrize"]
            sets = [{}]
            for k in marks:
                names, values = [n.strip() for n in k.args[0].split(",")], k.args[1]
                sets = [{**s, **dict(zip(names, v if len(names) > 1 else (v,)))} for s in sets for v in values]
            for i, kw in enumerate(sets):
                yield pytest.param(getattr(m, name), kw, id=f"{m.__name__}-{name}-{i}")


@pytest.mark.parametrize("test,kw", _cases())
def test_the_same(test, kw):
    test(**kw)


@pytest.mark.gpu
def test_on_the_gpu():
    torch = pytest.importorskip("torch")
    import test_gpu_dropout as dropout
    d = dropout.Drop(37, 520, 0.1, torch.bfloat16)
    d.run()
    d.check()
