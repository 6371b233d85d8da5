"""What a build writes (the commands alone, nothing is compiled)."""
import os

from paper_2111_05972_amd import build


def _outputs(monkeypatch, **kw):
    written = []
    monkeypatch.setattr(build, "_run", lambda cmd, verbose: written.append(cmd[cmd.index("-o") + 1]))
    build.build(**kw)
    return {x for x in written if not x.endswith(".o")}


def test_the_package(monkeypatch):
    assert _outputs(monkeypatch) == {build.LIB, build.CALLS}


# Another library beside the package's leaves the package as it is.
def test_another_library(monkeypatch, tmp_path):
    out = str(tmp_path / "variant.so")
    assert _outputs(monkeypatch, out=out, extra=["-DX"]) == {out}


def test_without_headers(monkeypatch, tmp_path):
    monkeypatch.setattr(build.sysconfig, "get_paths", lambda: {"include": str(tmp_path)})
    assert _outputs(monkeypatch) == {build.LIB}
    assert not os.listdir(tmp_path)
