"""CPU-only: the library is built whether or not the marshalling module can be."""
import os
import shutil
import stat
import sysconfig

import pytest

from paper_2609_32882_b200 import binding as vb
from paper_2609_32882_b200 import build as vbuild

NVCC = """#!/bin/sh
# stands in for the compiler: writes its output file and notes the call
echo "$@" >> "{log}"
while [ $# -gt 0 ]; do
  if [ "$1" = "-o" ]; then : > "$2"; fi
  shift
done
"""


@pytest.fixture
def tree(tmp_path, monkeypatch):
    """A tree with one CUDA source and the real module, built by a stand-in for nvcc."""
    csrc = tmp_path / "pkg" / "csrc"
    csrc.mkdir(parents=True)
    (csrc / "one.cu").write_text("")
    shutil.copy(os.path.join(vbuild.CSRC, "marshal.c"), csrc)
    shutil.copytree(os.path.join(vbuild.ROOT, "include"), tmp_path / "include")
    bin_dir = tmp_path / "bin"
    bin_dir.mkdir()
    (bin_dir / "nvcc").write_text(NVCC.format(log=tmp_path / "calls"))
    os.chmod(bin_dir / "nvcc", stat.S_IRWXU)
    monkeypatch.setenv("PATH", f"{bin_dir}:{os.environ['PATH']}")
    for name, value in (("HERE", csrc.parent), ("ROOT", tmp_path), ("CSRC", csrc), ("LIB_PATH", csrc.parent / "libvsa2.so"), ("MARSHAL_PATH", csrc.parent / "_marshal.so")):
        monkeypatch.setattr(vbuild, name, str(value))
    return tmp_path


def calls(tree):
    return (tree / "calls").read_text().count("\n") if (tree / "calls").exists() else 0


def without_headers(tree, monkeypatch):
    paths = dict(sysconfig.get_paths(), include=str(tree / "nothing"))
    monkeypatch.setattr(sysconfig, "get_paths", lambda *a, **k: paths)


def test_library_and_module(tree):
    assert vbuild.build_library() == vbuild.LIB_PATH
    assert os.path.exists(vbuild.LIB_PATH) and os.path.getsize(vbuild.MARSHAL_PATH) > 0
    before = calls(tree)
    vbuild.build_library()
    assert calls(tree) == before
    os.remove(vbuild.MARSHAL_PATH)                      # the module alone is missing
    vbuild.build_library()
    assert os.path.exists(vbuild.MARSHAL_PATH) and calls(tree) == before


def test_no_python_headers(tree, monkeypatch, capfd):
    without_headers(tree, monkeypatch)
    assert vbuild.build_library() == vbuild.LIB_PATH
    assert os.path.exists(vbuild.LIB_PATH) and not os.path.exists(vbuild.MARSHAL_PATH)
    assert "Python.h" in capfd.readouterr().err
    before = calls(tree)
    vbuild.build_library()
    assert calls(tree) == before                        # the CUDA sources are not compiled again
    monkeypatch.setattr(vb, "_MARSHAL", None)
    monkeypatch.setattr(vb, "MARSHAL_PATH", vbuild.MARSHAL_PATH)
    with pytest.raises(FileNotFoundError):
        vb._marshal()


def test_a_module_of_another_header_does_not_stay(tree, monkeypatch):
    vbuild.build_library()
    without_headers(tree, monkeypatch)
    later = os.path.getmtime(vbuild.MARSHAL_PATH) + 10
    os.utime(os.path.join(vbuild.ROOT, "include", "vsa2.h"), (later, later))
    vbuild.build_library()
    assert not os.path.exists(vbuild.MARSHAL_PATH)


def test_no_c_compiler(tree, monkeypatch):
    which = shutil.which
    monkeypatch.setattr(shutil, "which", lambda name, *a, **k: str(tree / "none") if name in ("gcc", "cc") else which(name, *a, **k))
    vbuild.build_library()
    assert os.path.exists(vbuild.LIB_PATH) and not os.path.exists(vbuild.MARSHAL_PATH)
