"""Sizes past 32 bits are refused by the functions on tensors; they do not reach the library cut short (no GPU needed)."""
import pytest

from paper_1611_09482_amd import binding as B

torch = pytest.importorskip("torch")
from paper_1611_09482_amd import ops  # noqa: E402

PAST = [2 ** 31, 2 ** 32 + 3, 2 ** 32 + 256, 2 ** 40 + 5]  # the low 32 bits of most are sizes that would pass


@pytest.fixture(scope="module", autouse=True)
def lib():
    from paper_1611_09482_amd import build
    if build.is_stale():
        build.build()
    return B.load_library()


def refused(call, code=B.FWG_EUNSUPPORTED):
    with pytest.raises(ops.FwgError) as e:
        call()
    assert e.value.code == code


@pytest.mark.parametrize("n", PAST)
def test_workspace_sizes(n):
    refused(lambda: ops._bytes("fwg_embed_grad_workspace", 5000, n, 64))
    refused(lambda: ops._bytes("fwg_embed_grad_workspace", 5000, 256, n))
    refused(lambda: ops._bytes("fwg_matmul_quant_workspace", 5000, n, 64))
    refused(lambda: ops._bytes("fwg_matmul_quant_workspace", 5000, 64, n))
    refused(lambda: ops._bytes("fwg_log_probs_workspace", 0, 5, n, 3))
    refused(lambda: ops._bytes("fwg_log_probs_workspace", 0, 5, 256, n))
    refused(lambda: ops._bytes("fwg_log_probs_workspace", 0, 5, 256, -2 ** 32 + 3), B.FWG_EINVAL)
    assert ops._bytes("fwg_embed_grad_workspace", 5000, 256, 64) > 0  # what fits still does


@pytest.mark.parametrize("n", PAST)
def test_rows_and_tables(n):
    """Tensors without memory: only shapes and strides are looked at."""
    row = torch.empty((1, n), dtype=torch.bfloat16, device="meta")
    for out in (False, True):
        refused(lambda: ops._matrix("x", row, row.get_device(), out))
        refused(lambda: ops._matrix("x", row.view(1, 1, n), row.get_device(), out))
    refused(lambda: ops._rows("x", torch.empty((3, n), dtype=torch.int8, device="meta")))
    table = torch.empty((n, 2), dtype=torch.float32, device="meta")
    assert ops._matrix("logits", table, table.get_device()) == (B.FWG_F32, n, 2, 2)  # rows are counted in 64 bits
    refused(lambda: ops._table("table", table, table.get_device()))
    small = torch.empty((7, 2), dtype=torch.float32, device="meta")
    assert ops._table("table", small, small.get_device()) == (B.FWG_F32, 7, 2, 2)
    with pytest.raises(ValueError):
        ops._table("table", small.view(1, 7, 2), small.get_device())


LIMIT = 1 << 29  # of vocabularies and outputs, as include/fwg.h says


@pytest.mark.parametrize("size,code", [(LIMIT, B.FWG_OK), (LIMIT + 1, B.FWG_EUNSUPPORTED)])
def test_limits_of_vocabularies_and_outputs(lib, size, code):
    """No rows: what passes the checks does nothing."""
    import ctypes
    at, n = 1 << 30, ctypes.c_size_t(0)
    f32 = B.FWG_F32
    assert lib.fwg_embed(f32, f32, 0, size, 4, at, 4, at, 1.0, at, 4, None) == code
    assert lib.fwg_embed_grad_workspace(5, size, 4, ctypes.byref(n)) == code
    assert lib.fwg_matmul_quant(f32, 0, size, 4, at, 4, at, at, 4, at, None, at, size, None, 0, None) == code
    assert lib.fwg_matmul_quant_workspace(5, size, 4, ctypes.byref(n)) == code
    assert lib.fwg_log_probs(f32, 0, size, at, size, at, 0, at, at, at, None, None, None, 0, None) == code
    assert lib.fwg_log_probs_workspace(f32, 5, size, 4, ctypes.byref(n)) == code
    assert lib.fwg_log_probs_grad(f32, 0, size, at, size, at, at, at, at, at, at, size, None) == code
