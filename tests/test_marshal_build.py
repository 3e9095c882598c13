"""The binding's compiled part belongs to the Python that it was built for, and says so in its name: another one finds no such module."""
import importlib.machinery
import os
import sysconfig

from paper_2104_09455_amd import binding as B
from paper_2104_09455_amd import build


def test_the_module_s_name_carries_its_interpreter():
    module = B._compiled().__file__
    assert os.path.basename(module) == "_marshal" + sysconfig.get_config_var("EXT_SUFFIX")
    assert os.path.samefile(module, build.MARSHAL)


def test_building_leaves_no_module_that_any_interpreter_loads(tmp_path, monkeypatch):
    old = tmp_path / "_marshal.so"
    old.write_bytes(b"")
    monkeypatch.setattr(build, "HERE", str(tmp_path))
    monkeypatch.setattr(build, "MARSHAL", str(tmp_path / os.path.basename(build.MARSHAL)))
    build.build_marshal()
    assert os.listdir(tmp_path) == ["_marshal" + importlib.machinery.EXTENSION_SUFFIXES[0]]
