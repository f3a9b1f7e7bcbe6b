"""Calls of the 4-bit operators and adjust_logits at the limits of launches and of their types, against plain evaluations.

Bars: as derived in test_gpu_mx.py.
"""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("needs a GPU", allow_module_level=True)

from paper_1611_09482_amd import ops  # noqa: E402
from test_gpu_mx import BF16, F32, INF, TYPES, U, ints, plain_adjust, rand, randn  # noqa: E402


# ---- more rows than a launch takes ----

@pytest.mark.parametrize("V,n", [(3, (1 << 23) + 5), (2050, (1 << 23) // 9 + 11)])
def test_adjust_more_rows_than_one_launch_takes(V, n):
    """A launch takes 2^23 rows of up to 256 logits, fewer of wider ones; the second one begins where the first ends."""
    z, tokens = randn(1, n, V).to(BF16), ints(2, -1, V + 1, n, 2)
    lengths, presence = ints(3, 0, 3, n), rand(4, n)
    allowed = ints(5, -2 ** 31, 2 ** 31 - 1, n, (V + 31) // 32)
    out = ops.adjust_logits(z, tokens, lengths, presence=presence, allowed=allowed)
    per = (1 << 23) // ((V + 255) // 256)
    for r in (slice(0, 30), slice(per // 2 - 10, per // 2 + 10), slice(per - 20, n)):
        want, bar = plain_adjust(z[r], tokens=tokens[r], lengths=lengths[r], presence=presence[r], allowed=allowed[r])
        bar = bar + 2.0 ** -8 * (want.abs() + bar)
        d = out[r].double()
        assert bool(((d == want) | ((d - want).abs() <= bar)).all())
    mine = z.clone()
    assert torch.equal(ops.adjust_logits(mine, tokens, lengths, presence=presence, allowed=allowed, out=mine), out)
