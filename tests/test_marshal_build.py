"""How the argument marshalling is built: beside a library that does not need it, and for the interpreter that it is built under alone."""
import os
import subprocess
import sys
import sysconfig

import pytest

from paper_2311_02103_amd import build as b


@pytest.fixture
def place(tmp_path, monkeypatch):
    """The build's outputs in a folder of the test."""
    monkeypatch.setattr(b, "HERE", str(tmp_path))
    for name in ("MARSHAL", "LIB", "OBJ"):
        monkeypatch.setattr(b, name, str(tmp_path / os.path.basename(getattr(b, name))))
    return tmp_path


def files(place):
    return sorted(f for f in os.listdir(place) if f.startswith("_marshal"))


def test_the_extension_is_named_for_its_interpreter(place):
    (place / "_marshal.so").write_bytes(b"of another build")                # the name that every interpreter would take
    made = b.build_marshal()
    suffix = sysconfig.get_config_var("EXT_SUFFIX")
    assert files(place) == ["_marshal" + suffix] and made == str(place / ("_marshal" + suffix)) and sys.implementation.cache_tag.replace("-", "") in suffix.replace("-", "")
    code = "import importlib.util as u, sys\nspec = u.spec_from_file_location('_marshal', sys.argv[1])\nm = u.module_from_spec(spec)\nspec.loader.exec_module(m)\nm.Seqs([1], [2])"
    subprocess.run([sys.executable, "-c", code, made], check=True, timeout=120)


@pytest.mark.parametrize("compiler", ["false", "/nowhere/cc", "a compiler that is not there"])
def test_without_a_compiler_the_library_is_built_all_the_same(place, monkeypatch, capfd, compiler):
    """And no extension of an earlier build stays, which may be of other sources: binding.py then does the same in Python."""
    for stale in ("_marshal.so", "_marshal" + sysconfig.get_config_var("EXT_SUFFIX")):
        (place / stale).write_bytes(b"stale")
    monkeypatch.setenv("CC", compiler)
    monkeypatch.setattr(b, "sources", lambda: ["one.hip"])
    monkeypatch.setattr(b, "_compile", lambda src: str(place / "one.o"))
    monkeypatch.setattr(b, "HIPCC", "true")
    assert b.build(verbose=False) == b.LIB
    assert files(place) == [] and "marshal" in capfd.readouterr().err
