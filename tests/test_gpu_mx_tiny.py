"""norm_mx of rows whose squares float32 does not hold, against 64 bits.

Bar of row_scale: as in test_gpu_mx.py at most 54 roundings of positive terms, halved by the root, and four more: below
2e-6, 4e-6 is allowed.  Elements come down to float32's smallest number, 2^-149, and scaling them by a power of two rounds
nothing, so that the bar is the same for every size of row.
"""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("needs a GPU", allow_module_level=True)

from paper_1611_09482_amd import ops  # noqa: E402
from test_gpu_mx import BF16, F32, TYPES, pack, plain_rows, randn, same  # noqa: E402

BIG = torch.finfo(F32).max


def check(x, gain, eps, residual=None):
    """Returns the row scales.  h and h * gain are one float32 operation each, which torch's float32 does alike."""
    h = x.float() if residual is None else x.float() + residual.float()
    code, byte, value = plain_rows(h if gain is None else h * gain)
    factor = 1 / torch.sqrt(h.double().square().mean(1) + float(torch.tensor(eps, dtype=F32)))
    factor = torch.where((byte == 0).all(1), 0.0, torch.where(factor > BIG, math.nan, factor))
    r = ops.norm_mx(x, gain, residual=residual, eps=eps, values=True)
    assert torch.equal(r.scale.long(), byte.long()) and torch.equal(r.q, pack(code))
    near = ((r.row_scale.double() - factor).abs() <= 4e-6 * factor) | (torch.isnan(r.row_scale) & torch.isnan(factor))
    assert bool(near.all()), (r.row_scale[~near], factor[~near])
    want, got = value * factor[:, None], r.values.double()
    ok = ((got - want).abs() <= (2.0 ** -8 + 5e-6) * want.abs() + 2.0 ** -134) | (torch.isnan(got) & torch.isnan(want))
    assert bool(ok.all()), (got[~ok][:4], want[~ok][:4])
    return r.row_scale


# every kernel: one wave a row with one and two pieces, four waves with one and two, sixteen with one, two and four
CHANNELS = [40, 600, 2000, 4096, 5000, 16384, 32768]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("channels", CHANNELS)
@pytest.mark.parametrize("eps", [0.0, 2.0 ** -149, 2.0 ** -141, 2.0 ** -120, 2.0 ** -101, 2.0 ** -100, 1e-6])
def test_rows_of_every_size(channels, dtype, eps):
    sizes = [0, -40, -48, -49, -50, -51, -52, -55, -58, -60, -63, -66, -70, -72, -74, -76, -80, -90, -96]
    x = randn(channels, len(sizes), channels).to(dtype)
    for i, e in enumerate(sizes):
        x[i] = (x[i].double() * 2.0 ** e).to(dtype)
    scale = check(x, 1 + 0.2 * randn(1, channels), eps)
    assert not bool(torch.isnan(scale).any())
    if eps == 0:
        assert bool((scale[1:] > 2.0 ** 38).all())
    check(x, None, eps, residual=(x.flip(0).double() * 2.0 ** -3).to(dtype))


@pytest.mark.parametrize("channels", CHANNELS)
def test_rows_that_a_gain_lifts(channels):
    """Elements below 2^-100, down to the smallest, with a gain of 2^60: 1 / rms is a number up to rms = 2^-128."""
    sizes = [-101, -110, -120, -126, -127, -130, -140, -149]
    x = torch.empty((len(sizes), channels), device="cuda")
    for i, e in enumerate(sizes):
        x[i] = (randn(i, channels).sign().double() * 2.0 ** e).float()
    scale = check(x, torch.full((channels,), 2.0 ** 60, device="cuda"), 0.0)
    assert torch.isnan(scale).tolist() == [False] * 5 + [True] * 3
    assert not bool(check(x, torch.full((channels,), 2.0 ** 60, device="cuda"), 2.0 ** -140).isnan().any())
    assert not bool(check(x, None, 0.0).any())  # nothing in 4 bits without it


@pytest.mark.parametrize("channels", CHANNELS)
def test_one_element_beside_nothing(channels):
    """A single element, and one beside others whose squares vanish next to its own."""
    x = torch.zeros((4, channels), device="cuda")
    x[0, channels // 2] = 2.0 ** -80
    x[1, -1] = -(2.0 ** -99)
    x[2], x[2, 0] = 2.0 ** -70, 2.0 ** -49
    x[3], x[3, 0] = 2.0 ** -120, 2.0 ** -60
    assert not bool(torch.isnan(check(x, None, 0.0)).any())


def test_rows_out_of_the_ordinary_without_eps():
    x = randn(1, 6, 700)
    x[0] = 0.0
    x[1] *= 2.0 ** -70
    x[1, 3] = math.nan
    x[2] *= 2.0 ** -70
    x[2, 5] = math.inf
    x[3] = 2.0 ** 64  # the sum of squares passes float32
    x[4] *= 2.0 ** 50
    gain = torch.ones(700, device="cuda")
    scale = ops.norm_mx(x, gain, eps=0.0).row_scale
    assert torch.isnan(scale).tolist() == [False, True, True, True, False, False] and scale[0] == 0
    gain[9] = math.inf  # of a row of nothing this makes a block of NaN, and no factor makes sense of it
    r = ops.norm_mx(x[:1], gain, eps=0.0, values=True)
    assert bool(torch.isnan(r.row_scale).all()) and bool(torch.isnan(r.values[:, :32]).all())


@pytest.mark.parametrize("channels", CHANNELS)
@pytest.mark.parametrize("eps", [0.0, 1e-6])
def test_rows_without_a_block_are_zero_whatever_their_size(channels, eps):
    """A gain of zero leaves nothing, also of a row whose sum of squares passes float32; NaN and infinity stay something."""
    x = randn(channels, 6, channels)
    x[1] = 0.0
    x[2] = torch.finfo(F32).max
    x[3] = x[3].sign() * 2.0 ** 100
    x[4, 0] = math.nan
    x[5, channels - 1] = math.inf
    r = ops.norm_mx(x, torch.zeros(channels, device="cuda"), eps=eps, values=True)
    assert torch.isnan(r.row_scale).tolist() == [False] * 4 + [True] * 2
    assert not r.row_scale[:4].any() and not r.scale[:4].any() and not r.values[:4].any()
    assert bool((r.scale[4:] == 255).any(1).all())


def test_the_same_bits_in_place_and_again():
    x = (randn(1, 9, 3000) * 2.0 ** -70).to(BF16)
    want = ops.norm_mx(x, residual=x, eps=0.0, values=True)
    again = ops.norm_mx(x, residual=x, eps=0.0, values=True)
    mine = x.clone()
    got = ops.norm_mx(mine, residual=x, eps=0.0, out=tuple(t.clone() for t in want[:3]) + (mine, None))
    for a, b in zip(want, again):
        assert torch.equal(a, b)
    assert torch.equal(got.row_scale, want.row_scale) and torch.equal(got.q, want.q) and same(mine, want.summed)
