"""What is loaded for which call: the library for all, the compiled marshalling for a decode step's alone."""
import types

import pytest

import paper_2603_05210_b200.binding as binding
import paper_2603_05210_b200.build as build


@pytest.fixture
def fresh(monkeypatch, tmp_path):
    """The binding as it is before its first call, without a compiled marshalling; the names of what is built."""
    binding.lib()                                # built, where it was not
    built = []
    monkeypatch.setattr(binding, "_lib", None)
    monkeypatch.setattr(binding, "_fast", None)
    monkeypatch.setattr(binding, "MARSHAL_PATH", str(tmp_path / "_vt_torch.so"))
    for name in ("build", "build_library", "build_marshal"):
        monkeypatch.setattr(build, name, lambda *a, _n=name, **k: built.append((_n, k.get("force", False))), raising=False)
    return built


def test_the_library_needs_no_marshalling(fresh):
    assert binding.lib().vt_strerror(0) and fresh == []
    assert binding.vt_tree_attention_workspace_bytes(8, 2, 64, 4) > 0 and fresh == []


def test_the_marshalling_is_built_by_its_first_use(fresh, monkeypatch):
    told = []
    monkeypatch.setattr(binding.importlib, "import_module", lambda name, package: types.SimpleNamespace(init=lambda *a: told.append(a)))
    assert binding._marshal() is binding._marshal()
    assert fresh == [("build_marshal", False)] and len(told) == 1 and all(told[0])


def test_one_of_another_pytorch_is_built_again(fresh, monkeypatch):
    def load(name, package):
        if ("build_marshal", True) not in fresh:
            raise ImportError("undefined symbol")
        return types.SimpleNamespace(init=lambda *a: None)

    open(binding.MARSHAL_PATH, "w").close()
    monkeypatch.setattr(binding.importlib, "import_module", load)
    binding._marshal()
    assert fresh == [("build_marshal", True)]

    def never(name, package):
        raise ImportError("undefined symbol")

    monkeypatch.setattr(binding, "_fast", None)
    monkeypatch.setattr(binding.importlib, "import_module", never)
    with pytest.raises(ImportError):
        binding._marshal()
