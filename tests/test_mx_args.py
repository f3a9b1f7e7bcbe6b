"""The 4-bit operators and adjust_logits refuse bad arguments on the host, before any device work (runs without a GPU)."""
import ctypes
import math

import pytest

from paper_1611_09482_amd import binding as B

FAKE = 1 << 30  # an aligned address that is never dereferenced: the checks fail first
EINVAL, ENOSPACE, EUNSUPPORTED = B.FWG_EINVAL, B.FWG_ENOSPACE, B.FWG_EUNSUPPORTED


@pytest.fixture(scope="module")
def lib():
    from paper_1611_09482_amd import build
    if build.is_stale():
        build.build()
    return B.load_library()


GOOD = {
    "fwg_quant_mx": dict(dtype=0, rows=5, channels=70, x=FAKE, x_stride=70, q=FAKE, q_stride=48, scale=FAKE, scale_stride=3,
                         values=FAKE, values_stride=70, stream=None),
    "fwg_norm_mx": dict(dtype=1, rows=5, channels=70, x=FAKE, x_stride=70, residual=FAKE, residual_stride=70, gain=FAKE,
                        eps=1e-6, summed=FAKE, summed_stride=70, q=FAKE, q_stride=48, scale=FAKE, scale_stride=3,
                        row_scale=FAKE, values=FAKE, values_stride=70, stream=None),
    "fwg_matmul_mx": dict(out_dtype=0, rows=5, outputs=7, blocks=3, x=FAKE, x_stride=48, x_scale=FAKE, x_scale_stride=3,
                          w=FAKE, w_stride=48, w_scale=FAKE, w_scale_stride=3, row_scale=FAKE, bias=FAKE, out=FAKE,
                          out_stride=7, ws=FAKE, ws_bytes=1 << 30, stream=None),
    "fwg_adjust_logits": dict(dtype=0, rows=5, vocab=70, logits=FAKE, logits_stride=70, history=9, tokens=FAKE,
                              tokens_stride=9, lengths=FAKE, prompts=FAKE, repetition=FAKE, presence=FAKE, frequency=FAKE,
                              bias=FAKE, bias_stride=70, allowed=FAKE, allowed_stride=3, out=FAKE, out_stride=70,
                              stream=None),
}

CASES = [
    ("fwg_quant_mx", dict(dtype=2), EINVAL), ("fwg_quant_mx", dict(rows=-1), EINVAL),
    ("fwg_quant_mx", dict(rows=(1 << 40) + 1), EUNSUPPORTED), ("fwg_quant_mx", dict(channels=0), EINVAL),
    ("fwg_quant_mx", dict(channels=(1 << 20) + 1, q_stride=1 << 21, scale_stride=1 << 20), EUNSUPPORTED),
    ("fwg_quant_mx", dict(x=None), EINVAL), ("fwg_quant_mx", dict(x=FAKE + 2), EINVAL),
    ("fwg_quant_mx", dict(x_stride=-1), EINVAL), ("fwg_quant_mx", dict(q=None), EINVAL),
    ("fwg_quant_mx", dict(q_stride=47), EINVAL), ("fwg_quant_mx", dict(scale=None), EINVAL),
    ("fwg_quant_mx", dict(scale_stride=2), EINVAL), ("fwg_quant_mx", dict(values=FAKE + 1), EINVAL),
    ("fwg_quant_mx", dict(values_stride=69), EINVAL),
    ("fwg_norm_mx", dict(dtype=-1), EINVAL), ("fwg_norm_mx", dict(channels=32769, q_stride=1 << 20, scale_stride=1 << 20,
                                                                    summed_stride=1 << 20, values_stride=1 << 20), EUNSUPPORTED),
    ("fwg_norm_mx", dict(eps=-1e-6), EINVAL), ("fwg_norm_mx", dict(eps=math.nan), EINVAL),
    ("fwg_norm_mx", dict(eps=math.inf), EINVAL), ("fwg_norm_mx", dict(residual=FAKE + 1), EINVAL),
    ("fwg_norm_mx", dict(residual_stride=-1), EINVAL), ("fwg_norm_mx", dict(gain=FAKE + 2), EINVAL),
    ("fwg_norm_mx", dict(summed=FAKE + 1), EINVAL), ("fwg_norm_mx", dict(summed_stride=69), EINVAL),
    ("fwg_norm_mx", dict(row_scale=None), EINVAL), ("fwg_norm_mx", dict(row_scale=FAKE + 2), EINVAL),
    ("fwg_norm_mx", dict(q=None), EINVAL), ("fwg_norm_mx", dict(scale=None), EINVAL),
    ("fwg_norm_mx", dict(q_stride=47), EINVAL), ("fwg_norm_mx", dict(scale_stride=2), EINVAL),
    ("fwg_matmul_mx", dict(out_dtype=9), EINVAL), ("fwg_matmul_mx", dict(rows=-1), EINVAL),
    ("fwg_matmul_mx", dict(rows=(1 << 30) + 1), EUNSUPPORTED), ("fwg_matmul_mx", dict(outputs=0), EINVAL),
    ("fwg_matmul_mx", dict(outputs=(1 << 29) + 1), EUNSUPPORTED), ("fwg_matmul_mx", dict(blocks=0), EINVAL),
    ("fwg_matmul_mx", dict(blocks=32769), EUNSUPPORTED), ("fwg_matmul_mx", dict(x=None), EINVAL),
    ("fwg_matmul_mx", dict(x_scale=None), EINVAL), ("fwg_matmul_mx", dict(w=None), EINVAL),
    ("fwg_matmul_mx", dict(w_scale=None), EINVAL), ("fwg_matmul_mx", dict(x_stride=-1), EINVAL),
    ("fwg_matmul_mx", dict(x_scale_stride=-1), EINVAL), ("fwg_matmul_mx", dict(w_stride=-1), EINVAL),
    ("fwg_matmul_mx", dict(w_scale_stride=-1), EINVAL), ("fwg_matmul_mx", dict(out_stride=6), EINVAL),
    ("fwg_matmul_mx", dict(row_scale=FAKE + 1), EINVAL), ("fwg_matmul_mx", dict(bias=FAKE + 2), EINVAL),
    ("fwg_matmul_mx", dict(out=None), EINVAL), ("fwg_matmul_mx", dict(out=FAKE + 2), EINVAL),
    ("fwg_adjust_logits", dict(dtype=2), EINVAL), ("fwg_adjust_logits", dict(rows=-1), EINVAL),
    ("fwg_adjust_logits", dict(vocab=0), EINVAL), ("fwg_adjust_logits", dict(vocab=(1 << 29) + 1), EUNSUPPORTED),
    ("fwg_adjust_logits", dict(history=-1), EINVAL), ("fwg_adjust_logits", dict(logits=None), EINVAL),
    ("fwg_adjust_logits", dict(logits=FAKE + 2), EINVAL), ("fwg_adjust_logits", dict(logits_stride=-1), EINVAL),
    ("fwg_adjust_logits", dict(tokens=None), EINVAL), ("fwg_adjust_logits", dict(tokens=FAKE + 2), EINVAL),
    ("fwg_adjust_logits", dict(tokens_stride=-1), EINVAL), ("fwg_adjust_logits", dict(lengths=FAKE + 1), EINVAL),
    ("fwg_adjust_logits", dict(prompts=FAKE + 1), EINVAL), ("fwg_adjust_logits", dict(repetition=FAKE + 1), EINVAL),
    ("fwg_adjust_logits", dict(presence=FAKE + 1), EINVAL), ("fwg_adjust_logits", dict(frequency=FAKE + 1), EINVAL),
    ("fwg_adjust_logits", dict(bias=FAKE + 1), EINVAL), ("fwg_adjust_logits", dict(bias_stride=-1), EINVAL),
    ("fwg_adjust_logits", dict(allowed=FAKE + 1), EINVAL), ("fwg_adjust_logits", dict(allowed_stride=-1), EINVAL),
    ("fwg_adjust_logits", dict(out=None), EINVAL), ("fwg_adjust_logits", dict(out_stride=69), EINVAL),
    # written where an input of another stride is read: the input's later rows would be the output's
    ("fwg_adjust_logits", dict(logits_stride=0), EINVAL), ("fwg_adjust_logits", dict(out_stride=71), EINVAL),
    ("fwg_norm_mx", dict(x_stride=0), EINVAL), ("fwg_norm_mx", dict(x_stride=71, residual=2 * FAKE), EINVAL),
    ("fwg_norm_mx", dict(residual_stride=0, x=2 * FAKE), EINVAL),
]


@pytest.mark.parametrize("name,change,code", CASES)
def test_refusals(lib, name, change, code):
    args = dict(GOOD[name])
    assert set(change) <= set(args)
    args.update(change)
    assert getattr(lib, name)(*args.values()) == code
    assert lib.fwg_last_error().decode()


@pytest.mark.parametrize("name", sorted(GOOD))
def test_no_rows_is_no_work(lib, name):
    assert getattr(lib, name)(*dict(GOOD[name], rows=0).values()) == B.FWG_OK


def workspace(lib, *args):
    n = ctypes.c_size_t(0)
    return lib.fwg_matmul_mx_workspace(*args, ctypes.byref(n)), n.value


def test_workspace_sizes(lib):
    assert workspace(lib, 0, 10, 10) == (B.FWG_OK, 0)
    assert workspace(lib, 1, 10, 0)[0] == EINVAL
    assert workspace(lib, 1, 0, 10)[0] == EINVAL
    assert workspace(lib, -1, 10, 10)[0] == EINVAL
    assert workspace(lib, 1, 10, 32769)[0] == EUNSUPPORTED
    assert workspace(lib, 1 << 30, 1 << 29, 32768)[0] == B.FWG_OK
    assert lib.fwg_matmul_mx_workspace(1, 1, 1, None) == EINVAL


def test_tensor_checks_without_a_device():
    torch = pytest.importorskip("torch")
    from paper_1611_09482_amd import ops
    if torch.cuda.is_available():
        pytest.skip("the messages below are those of a machine without a GPU")
    assert ops._mx_shapes(torch.Size((2, 3, 70))) == ((2, 3, 48), (2, 3, 3))
    assert ops._mx_shapes(torch.Size((1,))) == ((16,), (1,))
    row = torch.zeros(7)
    assert ops._one_or_each("bias", row, torch.float32, (5,), 7, row.get_device()) == (row.data_ptr(), 0)
    each = torch.zeros((5, 9))[:, :7]
    assert ops._one_or_each("bias", each, torch.float32, (5,), 7, each.get_device()) == (each.data_ptr(), 9)
    assert ops._one_or_each("bias", None, torch.float32, (5,), 7, 0) == (None, 0)
    for bad in (torch.zeros(8), torch.zeros((4, 7)), torch.zeros((5, 14))[:, ::2]):
        with pytest.raises(ValueError):
            ops._one_or_each("bias", bad, torch.float32, (5,), 7, bad.get_device())
    with pytest.raises(TypeError):
        ops._one_or_each("bias", row.double(), torch.float32, (5,), 7, row.get_device())
