"""The build where the module of ops.py cannot be compiled (runs without a GPU)."""
import os

import pytest

from paper_1611_09482_amd import build as B


@pytest.fixture
def elsewhere(tmp_path, monkeypatch):
    """A build into another folder, of one source."""
    for name, at in (("LIB", "libfwg.so"), ("MARSHAL", "_marshal.so"), ("OBJDIR", "_build")):
        monkeypatch.setattr(B, name, str(tmp_path / at))
    monkeypatch.setattr(B, "SOURCES", [os.path.join(B.CSRC, "fwg_ops.cpp")])
    return tmp_path


@pytest.mark.parametrize("compiler", ["/bin/false", "/no/such/compiler"])
def test_the_library_is_built_without_a_host_compiler(compiler, elsewhere, monkeypatch):
    """ops.py works without the module, so it does not cost the library; one of other sources does not stay."""
    pytest.importorskip("torch")
    monkeypatch.setenv("CXX", compiler)
    with open(B.MARSHAL, "w") as f:
        f.write("an earlier module")
    with pytest.warns(UserWarning, match="_marshal was not built"):
        assert B.build() == B.LIB
    assert os.path.exists(B.LIB) and not os.path.exists(B.MARSHAL)


def test_a_failed_library_is_an_error_that_names_its_compiler(elsewhere, monkeypatch):
    monkeypatch.setattr(B, "HIPCC", "/bin/false")
    monkeypatch.setenv("CXX", "/bin/true")
    with pytest.raises(RuntimeError, match="/bin/false failed"):
        B.build()
    assert not os.path.exists(B.LIB)
