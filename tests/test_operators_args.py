"""The token operators refuse bad arguments on the host, before any device work (runs without a GPU)."""
import ctypes
import math

import pytest

from paper_1611_09482_amd import binding as B

FAKE = 1 << 30  # an aligned address that is never dereferenced: the checks fail first


@pytest.fixture(scope="module")
def lib():
    from paper_1611_09482_amd import build
    if build.is_stale():
        build.build()
    return B.load_library()


GOOD = {
    "fwg_embed": dict(dtype=1, out_dtype=0, n=5, vocab=9, channels=4, table=FAKE, table_stride=4, tokens=FAKE, scale=1.0,
                      out=FAKE, out_stride=4, stream=None),
    "fwg_embed_grad": dict(dtype=1, out_dtype=0, n=5000, vocab=9, channels=4, grad=FAKE, grad_stride=4, tokens=FAKE,
                           scale=1.0, out=FAKE, out_stride=4, ws=FAKE, ws_bytes=1 << 20, stream=None),
    "fwg_quant_rows": dict(dtype=0, rows=5, channels=4, x=FAKE, x_stride=4, q=FAKE, q_stride=4, scale=FAKE, stream=None),
    "fwg_norm_quant": dict(dtype=0, rows=5, channels=4, x=FAKE, x_stride=4, residual=FAKE, residual_stride=4, gain=FAKE,
                           eps=1e-6, summed=FAKE, summed_stride=4, q=FAKE, q_stride=4, scale=FAKE, values=FAKE,
                           values_stride=4, stream=None),
    "fwg_matmul_quant": dict(out_dtype=0, rows=5, outputs=7, inner=4, x=FAKE, x_stride=4, x_scale=FAKE, w=FAKE, w_stride=4,
                             w_scale=FAKE, bias=FAKE, out=FAKE, out_stride=7, ws=FAKE, ws_bytes=1 << 30, stream=None),
    "fwg_log_probs": dict(dtype=0, rows=5, vocab=9, logits=FAKE, logits_stride=9, tokens=FAKE, top=3, logp=FAKE,
                          entropy=FAKE, lse=FAKE, top_ids=FAKE, top_logp=FAKE, ws=FAKE, ws_bytes=1 << 30, stream=None),
    "fwg_log_probs_grad": dict(dtype=0, rows=5, vocab=9, logits=FAKE, logits_stride=9, tokens=FAKE, lse=FAKE, entropy=FAKE,
                               grad_logp=FAKE, grad_entropy=FAKE, out=FAKE, out_stride=9, stream=None),
}

EINVAL, ENOSPACE, EUNSUPPORTED = B.FWG_EINVAL, B.FWG_ENOSPACE, B.FWG_EUNSUPPORTED

CASES = [
    ("fwg_embed", dict(dtype=2), EINVAL), ("fwg_embed", dict(out_dtype=-1), EINVAL), ("fwg_embed", dict(n=-1), EINVAL),
    ("fwg_embed", dict(vocab=0), EINVAL), ("fwg_embed", dict(vocab=(1 << 30) + 1), EUNSUPPORTED),
    ("fwg_embed", dict(channels=0), EINVAL), ("fwg_embed", dict(channels=(1 << 20) + 1), EUNSUPPORTED),
    ("fwg_embed", dict(table=None), EINVAL), ("fwg_embed", dict(tokens=None), EINVAL), ("fwg_embed", dict(out=None), EINVAL),
    ("fwg_embed", dict(table=FAKE + 1), EINVAL), ("fwg_embed", dict(tokens=FAKE + 2), EINVAL),
    ("fwg_embed", dict(out=FAKE + 2), EINVAL), ("fwg_embed", dict(table_stride=-4), EINVAL),
    ("fwg_embed", dict(out_stride=3), EINVAL), ("fwg_embed", dict(n=(1 << 40) + 1), EUNSUPPORTED),
    ("fwg_embed_grad", dict(dtype=7), EINVAL), ("fwg_embed_grad", dict(out_dtype=7), EINVAL),
    ("fwg_embed_grad", dict(n=-1), EINVAL), ("fwg_embed_grad", dict(n=(1 << 30) + 1), EUNSUPPORTED),
    ("fwg_embed_grad", dict(vocab=-3), EINVAL), ("fwg_embed_grad", dict(channels=0), EINVAL),
    ("fwg_embed_grad", dict(grad=None), EINVAL), ("fwg_embed_grad", dict(grad=FAKE + 1), EINVAL),
    ("fwg_embed_grad", dict(tokens=None), EINVAL), ("fwg_embed_grad", dict(out=None), EINVAL),
    ("fwg_embed_grad", dict(n=0, out=None), EINVAL), ("fwg_embed_grad", dict(out_stride=3), EINVAL),
    ("fwg_embed_grad", dict(ws=None), EINVAL), ("fwg_embed_grad", dict(ws_bytes=64), ENOSPACE),
    ("fwg_embed_grad", dict(ws=FAKE + 16), ENOSPACE),
    ("fwg_quant_rows", dict(dtype=3), EINVAL), ("fwg_quant_rows", dict(rows=-1), EINVAL),
    ("fwg_quant_rows", dict(channels=0), EINVAL), ("fwg_quant_rows", dict(channels=32769, q_stride=32769), EUNSUPPORTED),
    ("fwg_quant_rows", dict(x=None), EINVAL), ("fwg_quant_rows", dict(x=FAKE + 2), EINVAL),
    ("fwg_quant_rows", dict(q=None), EINVAL), ("fwg_quant_rows", dict(scale=None), EINVAL),
    ("fwg_quant_rows", dict(q_stride=3), EINVAL), ("fwg_quant_rows", dict(x_stride=-1), EINVAL),
    ("fwg_norm_quant", dict(eps=-1e-6), EINVAL), ("fwg_norm_quant", dict(eps=math.nan), EINVAL),
    ("fwg_norm_quant", dict(eps=math.inf), EINVAL), ("fwg_norm_quant", dict(residual=FAKE + 1), EINVAL),
    ("fwg_norm_quant", dict(residual_stride=-1), EINVAL), ("fwg_norm_quant", dict(gain=FAKE + 2), EINVAL),
    ("fwg_norm_quant", dict(summed_stride=3), EINVAL), ("fwg_norm_quant", dict(summed=FAKE + 2), EINVAL),
    ("fwg_norm_quant", dict(values_stride=3), EINVAL), ("fwg_norm_quant", dict(values=FAKE + 1), EINVAL),
    ("fwg_norm_quant", dict(scale=FAKE + 1), EINVAL),
    ("fwg_matmul_quant", dict(out_dtype=9), EINVAL), ("fwg_matmul_quant", dict(rows=-1), EINVAL),
    ("fwg_matmul_quant", dict(rows=(1 << 30) + 1), EUNSUPPORTED), ("fwg_matmul_quant", dict(outputs=0), EINVAL),
    ("fwg_matmul_quant", dict(inner=0), EINVAL), ("fwg_matmul_quant", dict(inner=131072), EUNSUPPORTED),
    ("fwg_matmul_quant", dict(x=None), EINVAL), ("fwg_matmul_quant", dict(w=None), EINVAL),
    ("fwg_matmul_quant", dict(x_scale=None), EINVAL), ("fwg_matmul_quant", dict(w_scale=FAKE + 1), EINVAL),
    ("fwg_matmul_quant", dict(bias=FAKE + 1), EINVAL), ("fwg_matmul_quant", dict(out=FAKE + 2), EINVAL),
    ("fwg_matmul_quant", dict(out_stride=6), EINVAL), ("fwg_matmul_quant", dict(w_stride=-1), EINVAL),
    ("fwg_log_probs", dict(dtype=2), EINVAL), ("fwg_log_probs", dict(rows=-1), EINVAL),
    ("fwg_log_probs", dict(vocab=0), EINVAL), ("fwg_log_probs", dict(top=-1), EINVAL),
    ("fwg_log_probs", dict(top=10), EINVAL), ("fwg_log_probs", dict(top=65, vocab=100, logits_stride=100), EUNSUPPORTED),
    ("fwg_log_probs", dict(logits=None), EINVAL), ("fwg_log_probs", dict(logits=FAKE + 2), EINVAL),
    ("fwg_log_probs", dict(tokens=None), EINVAL), ("fwg_log_probs", dict(logp=None), EINVAL),
    ("fwg_log_probs", dict(entropy=None), EINVAL), ("fwg_log_probs", dict(lse=FAKE + 1), EINVAL),
    ("fwg_log_probs", dict(top_ids=None), EINVAL), ("fwg_log_probs", dict(top_logp=None), EINVAL),
    ("fwg_log_probs", dict(logits_stride=-1), EINVAL),
    ("fwg_log_probs", dict(vocab=200000, logits_stride=200000, ws=None), EINVAL),
    ("fwg_log_probs", dict(vocab=200000, logits_stride=200000, ws_bytes=8), ENOSPACE),
    ("fwg_log_probs", dict(vocab=200000, logits_stride=200000, ws=FAKE + 4), ENOSPACE),
    ("fwg_log_probs_grad", dict(dtype=2), EINVAL), ("fwg_log_probs_grad", dict(vocab=0), EINVAL),
    ("fwg_log_probs_grad", dict(out=None), EINVAL), ("fwg_log_probs_grad", dict(out_stride=8), EINVAL),
    ("fwg_log_probs_grad", dict(lse=None), EINVAL), ("fwg_log_probs_grad", dict(grad_logp=None), EINVAL),
    ("fwg_log_probs_grad", dict(entropy=None), EINVAL), ("fwg_log_probs_grad", dict(tokens=FAKE + 1), EINVAL),
]


@pytest.mark.parametrize("name,change,code", CASES)
def test_refusals(lib, name, change, code):
    args = dict(GOOD[name])
    assert set(change) <= set(args)
    args.update(change)
    assert getattr(lib, name)(*args.values()) == code
    assert lib.fwg_last_error().decode()


@pytest.mark.parametrize("name", ["fwg_embed", "fwg_quant_rows", "fwg_norm_quant", "fwg_matmul_quant", "fwg_log_probs",
                                  "fwg_log_probs_grad"])
def test_no_rows_is_no_work(lib, name):
    args = dict(GOOD[name])
    args["n" if "n" in args else "rows"] = 0
    assert getattr(lib, name)(*args.values()) == B.FWG_OK


def size(fn, *args):
    n = ctypes.c_size_t(0)
    return fn(*args, ctypes.byref(n)), n.value


def test_workspace_sizes(lib):
    assert size(lib.fwg_embed_grad_workspace, 0, 10, 10) == (B.FWG_OK, 0)
    rc, small = size(lib.fwg_embed_grad_workspace, 1000, 256, 64)
    assert rc == B.FWG_OK and small >= 2 * 8 * 1000
    rc, large = size(lib.fwg_embed_grad_workspace, 100000, 256, 64)
    assert rc == B.FWG_OK and large > small
    assert size(lib.fwg_embed_grad_workspace, -1, 10, 10)[0] == EINVAL
    assert lib.fwg_embed_grad_workspace(1, 1, 1, None) == EINVAL
    assert size(lib.fwg_matmul_quant_workspace, 0, 10, 10) == (B.FWG_OK, 0)
    assert size(lib.fwg_matmul_quant_workspace, 1, 10, 0)[0] == EINVAL
    assert lib.fwg_matmul_quant_workspace(1, 1, 1, None) == EINVAL
    assert size(lib.fwg_log_probs_workspace, 0, 100000, 256, 4) == (B.FWG_OK, 0)
    rc, one = size(lib.fwg_log_probs_workspace, 0, 1, 200000, 4)
    assert rc == B.FWG_OK and one > 0
    assert size(lib.fwg_log_probs_workspace, 5, 1, 256, 4)[0] == EINVAL
    assert lib.fwg_log_probs_workspace(0, 1, 256, 4, None) == EINVAL


def test_tensor_checks_without_a_device():
    torch = pytest.importorskip("torch")
    from paper_1611_09482_amd import ops
    if torch.cuda.is_available():
        pytest.skip("the messages below are those of a machine without a GPU")
    x = torch.zeros((2, 4))
    with pytest.raises(TypeError):
        ops._matrix("x", [1, 2], 0)
    for bad in (torch.zeros((2, 4, 3)).transpose(1, 2), torch.zeros(())):
        with pytest.raises(ValueError):
            ops._rows("x", bad)
    with pytest.raises(ValueError):
        ops._rows("x", torch.zeros((4, 3, 8))[:, ::2])  # rows of a plane lie 16 apart, planes 24
    with pytest.raises(ValueError):
        ops._rows("out", x[:1].expand(3, 4), True)
    assert ops._rows("x", torch.zeros((4, 3, 8))[:, :, 1:6]) == (12, 5, 8)
    assert ops._rows("x", x[:1].expand(3, 4)) == (3, 4, 0)
    assert ops._rows("x", torch.zeros((6, 4, 8))[::2, :1]) == (3, 8, 64)
    assert ops._rows("x", torch.zeros(5)) == (1, 5, 5)
