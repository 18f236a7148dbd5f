"""Which torch the native marshalling takes for the one that it was built with: that of the same full name, development builds and local parts
included, and of the same C++ ABI."""
import importlib
import os
import subprocess
import types

import pytest

torch = pytest.importorskip("torch")


@pytest.fixture
def looked_up(monkeypatch):
    """Looks for the native marshalling anew, under a name of torch's and the module's own."""
    from paper_2304_01089_amd import binding
    import paper_2304_01089_amd as rp
    if not os.path.exists(rp.library_path()):
        pytest.skip("librptq.so is not built")
    lib = rp.load_library()
    try:
        calls = importlib.import_module("paper_2304_01089_amd._calls")
    except ImportError as e:
        pytest.skip("no native marshalling here: %s" % e)

    def look(here, built):
        monkeypatch.setattr(binding, "_CALLS", None)
        monkeypatch.setattr(binding, "_CALLS_SOUGHT", False)
        monkeypatch.setattr(torch, "__version__", here)
        monkeypatch.setattr(calls, "torch_version", built.partition("+")[0])
        monkeypatch.setattr(calls, "torch_local", built.partition("+")[2], raising=False)
        binding._set_up_calls(lib)
        assert binding._CALLS_SOUGHT
        return binding._CALLS is calls
    return look


@pytest.mark.parametrize("name", ["2.10.0", "2.10.0+rocm7.0", "2.11.0.dev20260101+rocm7.1", "2.11.0a0+git449b176", "3.0.0rc1"])
def test_the_same_name_is_the_same_torch(looked_up, name):
    assert looked_up(name, name)


@pytest.mark.parametrize("here,built", [("2.10.0+rocm7.0", "2.10.0+cpu"), ("2.10.0+rocm7.0", "2.10.0"), ("2.10.0", "2.10.0+rocm7.0"), ("2.11.0a0+git449b176", "2.11.0a0+git0000000"),
                                        ("2.11.0.dev20260102", "2.11.0.dev20260101"), ("2.11.0a0", "2.11.0")])
def test_another_name_is_another_torch(looked_up, here, built):
    assert not looked_up(here, built)


def test_the_module_here_was_built_with_the_torch_here():
    try:
        from paper_2304_01089_amd import _calls
    except ImportError as e:
        pytest.skip("no native marshalling here: %s" % e)
    if _calls.torch_version != torch.__version__.partition("+")[0]:
        pytest.skip("built with another torch")
    assert _calls.torch_local == torch.__version__.partition("+")[2]


@pytest.mark.parametrize("abi", [True, False])
@pytest.mark.parametrize("name", ["2.10.0+rocm7.0", "2.11.0a0"])
def test_what_the_module_is_compiled_with(tmp_path, monkeypatch, abi, name):
    from paper_2304_01089_amd import build
    module, ran = tmp_path / os.path.basename(build.CALLS), []

    def compiler(cmd, **how):
        ran.append(cmd)
        (tmp_path / (module.name + ".tmp")).write_bytes(b"new")
        return types.SimpleNamespace(returncode=0, stdout="", stderr="")

    monkeypatch.setattr(build, "CALLS", str(module))
    monkeypatch.setattr(build.shutil, "which", lambda what: "/usr/bin/" + what)
    monkeypatch.setattr(subprocess, "run", compiler)
    monkeypatch.setattr(torch, "__version__", name)
    monkeypatch.setattr(torch._C, "_GLIBCXX_USE_CXX11_ABI", abi)
    if build.build_calls() is None:
        pytest.skip("no headers of Python's or torch's")
    assert module.read_bytes() == b"new" and len(ran) == 1
    version, _, local = name.partition("+")
    for flag in ("-D_GLIBCXX_USE_CXX11_ABI=%d" % abi, '-DRPTQ_TORCH_VERSION="%s"' % version, '-DRPTQ_TORCH_LOCAL="%s"' % local):
        assert flag in ran[0]


def test_a_torch_that_cannot_be_loaded(tmp_path, monkeypatch, capsys):
    """Its headers alone make no module; one of an older source goes."""
    from paper_2304_01089_amd import build
    module = tmp_path / os.path.basename(build.CALLS)
    module.write_bytes(b"older")
    folder = tmp_path / "torch"
    (folder / "include" / "torch" / "csrc" / "api" / "include" / "torch").mkdir(parents=True)
    (folder / "include" / "torch" / "csrc" / "api" / "include" / "torch" / "version.h").write_text("")
    (tmp_path / "Python.h").write_text("")
    monkeypatch.setattr(build, "CALLS", str(module))
    monkeypatch.setattr(build.shutil, "which", lambda what: "/usr/bin/" + what)
    monkeypatch.setattr(build.sysconfig, "get_paths", lambda: {"include": str(tmp_path)})
    monkeypatch.setattr(build.importlib.util, "find_spec", lambda name: types.SimpleNamespace(submodule_search_locations=[str(folder)]))
    monkeypatch.setitem(__import__("sys").modules, "torch", None)
    assert build.build_calls() is None
    assert not module.exists() and "torch" in capsys.readouterr().err
