"""The module _marshal takes plain arguments only and declines the rest (runs without a GPU: nothing here is on one)."""
import pytest

torch = pytest.importorskip("torch")
from paper_1611_09482_amd import build, ops  # noqa: E402


@pytest.fixture(scope="module")
def marshal():
    if build.is_stale():
        build.build()
    ops._library()
    assert ops._plain is not None and ops._plain is ops._marshal  # built beside the library
    return ops._plain


def test_other_tensors_and_objects_are_declined(marshal):
    x = torch.zeros((2, 64))
    q, e = torch.zeros((2, 32), dtype=torch.uint8), torch.zeros((2, 2), dtype=torch.uint8)
    f = torch.zeros(2)
    for bad in (x, x.to_sparse(), x[:, ::2], torch.zeros(()), torch.empty((2, 64), device="meta"), [1, 2], None, "x"):
        for at in range(4):
            args = [x, q, e, None]
            args[at] = bad
            assert marshal.quant_mx(0, 0, *args) is None
            assert marshal.norm_mx(0, 0, bad, None, x, 1e-6, q, e, f, None, None) is None
            assert marshal.matmul_mx(0, 0, q, e, q, e, f, None, bad) is None
            assert marshal.adjust_logits(0, 0, bad, None, None, None, None, None, None, None, None, x) is None


def test_other_calls_are_declined(marshal):
    x = torch.zeros((2, 64))
    assert marshal.quant_mx() is None and marshal.quant_mx(0, 0, x) is None
    assert marshal.quant_mx("0", 0, x, x, x, x) is None and marshal.quant_mx(0, -1.5, x, x, x, x) is None
    assert marshal.norm_mx(0, 0, x, None, None, 0, x, x, x, None, None) is None  # eps is no float
    with pytest.raises(TypeError):
        marshal.bind(1, 2)
