"""The module that marshals the token-by-token calls is theirs alone: what the block decoder calls is built, loaded and
bound without it, and it is held against the very torch that it was built for, whatever that one's version looks like."""
import sys
import types

import pytest
import torch

import paper_2607_17652_b200 as package
from paper_2607_17652_b200 import binding as B
from paper_2607_17652_b200 import build as build_module
from tests.test_token_refusals import GOOD, cache_tensors, tensors

NAME = "paper_2607_17652_b200._marshal_token"


@pytest.fixture(scope="module", autouse=True)
def built():
    build_module.build()


@pytest.fixture
def unloaded(monkeypatch):
    """The binding as it is before its first call."""
    for name in ("_lib", "_m", "_mt"):
        monkeypatch.setattr(B, name, None)


def append(ctx):
    t = tensors()
    B.fb_append_kv(ctx, cache_tensors(), t["k"], t["v"], t["pool"], t["pool"], t["status"], stream=0)


def test_block_calls_load_without_it(unloaded, monkeypatch):
    monkeypatch.setitem(sys.modules, NAME, None)      # (an import of it fails)
    monkeypatch.delattr(package, "_marshal_token", raising=False)
    monkeypatch.setattr(B, "_device", lambda: -1)
    B.lib()
    assert B._m is not None
    ctx = B.Context(**GOOD)
    assert ctx.workspace_bytes() > 0
    with pytest.raises(RuntimeError, match="paper_2607_17652_b200.build"):
        append(ctx)


def test_a_module_for_another_torch_is_refused_by_its_own_calls_alone(unloaded, monkeypatch):
    monkeypatch.setattr(B, "_device", lambda: -1)
    monkeypatch.setattr(torch, "__version__", "2.12.0.dev20260101+cu130")
    B.lib()
    ctx = B.Context(**GOOD)
    assert ctx.workspace_bytes() > 0
    with pytest.raises(RuntimeError, match="another torch"):
        append(ctx)


def test_it_says_the_whole_version_that_it_was_built_for():
    from paper_2607_17652_b200 import _marshal_token
    assert _marshal_token.torch_version == torch.__version__


@pytest.mark.parametrize("version", ["2.12.0.dev20260101+cu130", "2.11.0a0+git70d99e9", "2.11.0"])
def test_versions_as_torch_gives_them(version, tmp_path):
    (tmp_path / "version.py").write_text(f"__version__ = {version!r}\ncuda = None\n")
    assert build_module.torch_version(str(tmp_path)) == version


@pytest.mark.parametrize("missing", ["torch", "headers", "compiler"])
def test_building_goes_on_without_what_it_needs(missing, monkeypatch, tmp_path, capsys):
    def run(cmd):
        raise AssertionError("nothing can be compiled here")
    (tmp_path / "version.py").write_text("__version__ = '2.11.0'\n")
    header = tmp_path / "include" / "torch" / "csrc" / "autograd"
    header.mkdir(parents=True)
    if missing != "headers":
        (header / "python_variable.h").write_text("")
    spec = None if missing == "torch" else types.SimpleNamespace(submodule_search_locations=[str(tmp_path)])
    monkeypatch.setattr(build_module.importlib.util, "find_spec", lambda name: spec)
    if missing == "compiler":
        monkeypatch.setenv("CXX", str(tmp_path / "no such compiler"))
    build_module._build_marshal_token(run, True, 0.0)
    said = capsys.readouterr().err
    assert "fb_token_attn" in said and missing in said
