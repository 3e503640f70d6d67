"""What the package does where its CPython module is not there, or was built from other sources: it can be imported (to build it), every call says which, and
nothing that went wrong is lost. No GPU, no launch."""
import importlib.util
import types

import pytest

import paper_2509_15235_amd as vs
from paper_2509_15235_amd import binding

CALLS = binding._NATIVE + binding._NATIVE_MORE


def _binding_with(monkeypatch, native):
    monkeypatch.setattr(vs, "_native", native)
    spec = importlib.util.spec_from_file_location("paper_2509_15235_amd._other_binding", binding.__file__)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def _raises(error):
    def setup(*args):
        raise error
    return setup


@pytest.mark.parametrize("error", [TypeError("argument 7 must be type, not int"), AttributeError("no such thing")])
def test_a_module_that_does_not_fit_says_what_was_wrong(monkeypatch, error):
    other = _binding_with(monkeypatch, types.SimpleNamespace(setup=_raises(error)))
    for name in CALLS:
        with pytest.raises(ImportError, match="does not fit") as e:
            getattr(other, name)(1, 2, x=3)
        assert str(error) in str(e.value) and e.value.__cause__ is error


def test_a_module_without_a_call(monkeypatch):
    other = _binding_with(monkeypatch, types.SimpleNamespace(setup=lambda *a: None, **{name: print for name in binding._NATIVE}))
    with pytest.raises(ImportError, match="does not fit") as e:
        other.vs_rope_apply()
    assert isinstance(e.value.__cause__, AttributeError) and "vs_rope_apply" in str(e.value.__cause__)


def test_other_errors_are_the_callers(monkeypatch):
    with pytest.raises(ValueError, match="of its own"):
        _binding_with(monkeypatch, types.SimpleNamespace(setup=_raises(ValueError("of its own"))))


def test_a_module_that_is_not_there(monkeypatch):
    with pytest.raises(FileNotFoundError, match="is missing"):
        binding._missing("vs_rope_apply")()
    assert binding._missing("vs_rope_apply").__name__ == "vs_rope_apply"
