"""The module of ops.py beside the library: built where it can be, found where it fits (runs without a GPU)."""
import os

import pytest

from paper_1611_09482_amd import build as B


@pytest.fixture
def elsewhere(tmp_path, monkeypatch):
    """A build into another folder, of one source."""
    for name, at in (("LIB", "libfwg.so"), ("MARSHAL", "_marshal"), ("OBJDIR", "_build")):
        monkeypatch.setattr(B, name, str(tmp_path / at))
    monkeypatch.setattr(B, "SOURCES", [os.path.join(B.CSRC, "fwg_ops.cpp")])
    return tmp_path


@pytest.mark.parametrize("compiler", ["/bin/false", "/no/such/compiler"])
def test_the_library_is_built_without_a_host_compiler(compiler, elsewhere, monkeypatch):
    """ops.py works without the module, so it does not cost the library; one of other sources does not stay."""
    pytest.importorskip("torch")
    monkeypatch.setenv("CXX", compiler)
    for name in (B.marshal_path(), B.MARSHAL + ".so"):
        with open(name, "w") as f:
            f.write("an earlier module")
    with pytest.warns(UserWarning, match="_marshal was not built"):
        assert B.build() == B.LIB
    assert sorted(os.listdir(elsewhere)) == ["_build", "libfwg.so"]


def test_a_failed_library_is_an_error_that_names_its_compiler(elsewhere, monkeypatch):
    monkeypatch.setattr(B, "HIPCC", "/bin/false")
    monkeypatch.setattr(B, "build_marshal", lambda verbose: None)
    with pytest.raises(RuntimeError, match="/bin/false failed"):
        B.build()
    assert not os.path.exists(B.LIB)


@pytest.fixture
def built():
    torch = pytest.importorskip("torch")
    if B.is_stale():
        B.build()
    return torch


def test_the_module_is_this_pythons_and_this_torchs(built, monkeypatch):
    """Another version's module reads tensors by other layouts: it is neither found nor taken for built."""
    import sysconfig
    path = B.marshal_path()
    assert os.path.exists(path) and str(built.__version__) in path and path.endswith(sysconfig.get_config_var("EXT_SUFFIX"))
    assert not B.is_stale()
    monkeypatch.setattr(built, "__version__", "0.1.2")
    assert B.marshal_path() != path and B.is_stale()


def test_a_module_that_is_gone_is_built_again(built, tmp_path, monkeypatch):
    monkeypatch.setattr(B, "MARSHAL", str(tmp_path / "_marshal"))
    assert B.is_stale()
    old = tmp_path / "_marshal-torch0.1.2.cpython-39-x86_64-linux-gnu.so"
    old.write_text("another version's")
    B.build_marshal()
    assert not B.is_stale() and os.listdir(tmp_path) == [os.path.basename(B.marshal_path())]


def test_the_module_is_found_when_it_is_built_after_the_import(built, tmp_path, monkeypatch):
    """The library is loaded by the first call, and so is the module: until then both may be built."""
    from paper_1611_09482_amd import ops
    for name in ("_lib", "_marshal", "_plain"):
        monkeypatch.setattr(ops, name, None)
    assert ops._library() is not None and ops._plain is not None and ops._plain is ops._marshal
    x = built.zeros(3)
    assert ops._plain.quant_mx(0, 0, x, x, x, None) is None  # it runs, and declines what is not on a device
    for name in ("_lib", "_marshal", "_plain"):
        monkeypatch.setattr(ops, name, None)
    monkeypatch.setattr(B, "MARSHAL", str(tmp_path / "_marshal"))
    assert ops._library() is not None and ops._plain is None  # without it the calls go through ops.py
    with open(B.marshal_path(), "w") as f:
        f.write("no module at all")
    monkeypatch.setattr(ops, "_lib", None)
    assert ops._library() is not None and ops._plain is None
