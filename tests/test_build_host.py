"""The binding's native argument check is optional: the library is built without it, and a module of another torch or Python is not used."""
import importlib
import sysconfig

import pytest
import torch

from paper_2604_21335_b200 import binding as Bd
from paper_2604_21335_b200 import build as B


@pytest.fixture()
def elsewhere(tmp_path, monkeypatch):
    """The library is up to date; the module's place is an empty folder."""
    B.build()
    name = Bd.args_library().name
    monkeypatch.setattr(Bd, "args_library", lambda: tmp_path / name)
    return tmp_path / name


@pytest.mark.parametrize("compiler", ["/no/such/compiler", "false"])
def test_the_library_is_built_without_a_compiler_for_the_module(elsewhere, monkeypatch, capfd, compiler):
    monkeypatch.setenv("CXX", compiler)
    elsewhere.write_bytes(b"an older build")
    assert B.build() == B.LIB and B.LIB.exists()           # (up to date by its time: not compiled, not touched)
    B._build_args(force=True)
    assert not elsewhere.exists() and "argument check" in capfd.readouterr().err
    assert B.build() == B.LIB
    assert Bd._native_module() is None


def test_the_module_belongs_to_one_torch_and_one_python(monkeypatch):
    B.build()
    here = Bd.args_library()
    assert here.exists() and torch.__version__ in here.name and here.name.endswith(sysconfig.get_config_var("EXT_SUFFIX"))
    assert Bd._native_module() is not None
    monkeypatch.setattr(torch, "__version__", "0.0.1")
    assert Bd.args_library() != here and Bd._native_module() is None


def test_the_module_is_loaded_once_it_is_built(monkeypatch):
    """A program that builds after the import has it from the first call of the library on."""
    B.build()
    for name in ("_native_addresses", "_sizes_are", "_native_token_rows", "_lib"):
        monkeypatch.setattr(Bd, name, None)
    Bd.load_library()
    assert Bd._native_addresses is not None and Bd._sizes_are is not None and Bd._native_token_rows is not None
    assert importlib.import_module("paper_2604_21335_b200").load_library() is Bd._lib
