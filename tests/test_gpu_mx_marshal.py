"""Which calls the module _marshal takes (0, the entry's own answer) and which it leaves to ops.py (None), and that both agree."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("needs a GPU", allow_module_level=True)

from paper_1611_09482_amd import ops  # noqa: E402
from test_gpu_mx import BF16, F32, TYPES, ints, odd_view, randn, request, same  # noqa: E402

OPERATORS = {"quant_mx", "norm_mx", "matmul_mx", "adjust_logits"}


class Recorder:
    """The module, with what it answered."""

    def __init__(self, module):
        self.module, self.seen = module, []

    def __getattr__(self, name):
        entry = getattr(self.module, name)

        def call(*args):
            rc = entry(*args)
            self.seen.append((name, rc))
            return rc
        return call


def answers(monkeypatch, call):
    """[(entry, answer)] of one call, whose results equal those of ops.py alone."""
    ops.quant_mx(randn(1, 2, 32))  # the library is loaded
    assert ops._plain is not None
    recorder = Recorder(ops._plain)
    copies = lambda r: [None if t is None else t.clone() for t in ((r,) if torch.is_tensor(r) else r)]  # noqa: E731
    with monkeypatch.context() as m:
        m.setattr(ops, "_plain", recorder)
        fast = copies(call())
    with monkeypatch.context() as m:
        m.setattr(ops, "_plain", None)
        slow = copies(call())
    assert len(fast) == len(slow)
    for a, b in zip(fast, slow):
        assert (a is None and b is None) or (a.dtype == b.dtype and a.shape == b.shape and same(a, b))
    return recorder.seen


def calls(lead, dtype, see):
    """(entry, call) of every operator with all of its arguments; see(t) is what a call gets of a tensor."""
    n, D, V, H = math.prod(lead), 200, 600, 9
    x, res, gain = see(randn(1, *lead, D).to(dtype)), see(randn(2, *lead, D).to(dtype)), 1 + 0.1 * randn(3, D)
    w = ops.quant_mx(randn(4, V, D))
    new = lambda kind, *shape: see(torch.zeros(lead + shape, dtype=kind, device="cuda"))  # noqa: E731
    plain = ops.quant_mx(randn(5, *lead, D))
    kw = request(8, n, V, H)
    per_row = {k: v.view(lead) for k, v in kw.items() if v.dim() == 1}
    rows = {k: see(v.view(lead + v.shape[1:])) for k, v in kw.items() if v.dim() == 2}
    z = see(randn(7, *lead, V).to(dtype))
    u8, f = torch.uint8, randn(6, *lead)
    bias, words = randn(9, V), ints(10, -2 ** 31, 2 ** 31 - 1, 19)
    return [
        ("quant_mx", lambda: ops.quant_mx(x, out=(new(u8, 112), new(u8, 7), new(BF16, D)))),
        ("quant_mx", lambda: ops.quant_mx(x, values=True)),
        ("quant_mx", lambda: ops.quant_mx(x)),
        ("norm_mx", lambda: ops.norm_mx(x, gain, residual=res, eps=1e-5, values=True)),
        ("norm_mx", lambda: ops.norm_mx(x, out=(new(u8, 112), new(u8, 7), torch.zeros(lead, device="cuda"), None, None))),
        ("matmul_mx", lambda: ops.matmul_mx(see(plain.q), see(plain.scale), w.q, w.scale, row_scale=f, bias=bias, dtype=dtype)),
        ("matmul_mx", lambda: ops.matmul_mx(see(plain.q), plain.scale, w.q, w.scale, out=new(F32, V))),
        ("adjust_logits", lambda: ops.adjust_logits(z, out=new(dtype, V), **per_row, **rows)),
        ("adjust_logits", lambda: ops.adjust_logits(z, rows["tokens"], presence=per_row["presence"], allowed=words)),
        ("adjust_logits", lambda: ops.adjust_logits(z, bias=bias)),
    ]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lead", [(1,), (7,), (2, 3), (300,)])
def test_plain_arguments_are_taken(lead, dtype, monkeypatch):
    taken = set()
    for name, call in calls(lead, dtype, lambda t: t):
        assert answers(monkeypatch, call) == [(name, 0)]
        taken.add(name)
    assert taken == OPERATORS


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lead", [(7,), (2, 3)])
def test_views_are_left_to_the_thorough_checks(lead, dtype, monkeypatch):
    for name, call in calls(lead, dtype, odd_view):
        assert answers(monkeypatch, call) == [(name, None)]


def test_parameters_are_plain_tensors(monkeypatch):
    x, gain = torch.nn.Parameter(randn(1, 6, 96)), torch.nn.Parameter(randn(2, 96))
    assert answers(monkeypatch, lambda: ops.norm_mx(x, gain, values=True)) == [("norm_mx", 0)]


def test_other_objects_and_numbers_are_left(monkeypatch):
    class Named(torch.Tensor):
        pass
    x = randn(1, 6, 96)
    assert answers(monkeypatch, lambda: ops.quant_mx(x.as_subclass(Named))) == [("quant_mx", None)]
    assert answers(monkeypatch, lambda: ops.norm_mx(x, eps=1)) == [("norm_mx", None)]
    assert answers(monkeypatch, lambda: ops.quant_mx(x.t().contiguous().t()[:0])) == [("quant_mx", 0)]  # no rows
