"""`python -m paper_2012_15469_amd.build` builds the library for programs of the C ABI also where the operators' Python module cannot be built; build_all() needs both."""
import sys

import pytest

from paper_2012_15469_amd import build


def without(monkeypatch, what, tmp_path):
    if what == "torch":
        monkeypatch.setitem(sys.modules, "torch.utils.cpp_extension", None)
    elif what == "torch's C++ headers":
        monkeypatch.setattr("torch.utils.cpp_extension.include_paths", lambda *a, **k: [str(tmp_path)])
    elif what == "Python's headers":
        monkeypatch.setattr("sysconfig.get_paths", lambda *a, **k: {"include": str(tmp_path)})
    else:
        monkeypatch.setenv("CXX", str(tmp_path / "no-compiler"))


@pytest.mark.parametrize("what", ["torch", "torch's C++ headers", "Python's headers", "a host compiler"])
def test_the_library_alone(what, monkeypatch, tmp_path, capsys):
    built = []
    monkeypatch.setattr(build, "build_libcada", lambda: built.append("libcada"))
    monkeypatch.setattr(build, "OPS_BINDING", str(tmp_path / "_ops.so"))
    without(monkeypatch, what, tmp_path)
    assert build.main() == 0 and built == ["libcada"]
    out, err = capsys.readouterr()
    assert "built" in out and "_ops.so, which needs %s" % what in err
    with pytest.raises((RuntimeError, ImportError, OSError)):
        build.build_all()


def test_both(monkeypatch, capsys):
    built = []
    monkeypatch.setattr(build, "build_libcada", lambda: built.append("libcada"))
    monkeypatch.setattr(build, "build_ops_binding", lambda: built.append("ops"))
    assert build.ops_binding_lacks() == "" and build.main() == 0 and built == ["libcada", "ops"]
