"""The compiled marshalling is built for one Python version: its file says so,
and where it cannot be built the binding does without."""
import os
import shutil
import sysconfig

from paper_2606_22541_gb300 import build as build_mod


def test_the_file_carries_the_python_version():
    assert os.path.basename(build_mod.MARSHAL) == "_marshal" + sysconfig.get_config_var("EXT_SUFFIX")
    assert os.path.basename(build_mod.MARSHAL) != "_marshal.so"


def test_a_file_without_a_version_goes_away(monkeypatch, tmp_path):
    """Every Python version would load it."""
    old = tmp_path / "_marshal.so"
    old.write_bytes(b"")
    monkeypatch.setattr(build_mod, "PKG", str(tmp_path))
    monkeypatch.setattr(build_mod, "MARSHAL", str(tmp_path / "_marshal.tag.so"))
    build_mod.build_marshal()
    assert not old.exists()
    assert (tmp_path / "_marshal.tag.so").exists() == (shutil.which("gcc") is not None and os.path.exists(
        os.path.join(sysconfig.get_paths()["include"], "Python.h")))


def test_without_a_compiler_there_is_no_file(monkeypatch, tmp_path):
    monkeypatch.setattr(build_mod, "PKG", str(tmp_path))
    monkeypatch.setattr(build_mod, "MARSHAL", str(tmp_path / "_marshal.tag.so"))
    monkeypatch.setenv("PATH", str(tmp_path))
    build_mod.build_marshal(force=True)
    assert not list(tmp_path.iterdir())
