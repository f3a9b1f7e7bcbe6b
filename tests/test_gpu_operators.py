"""The token operators on the GPU against plain evaluations in 64 bits.

Bars, with u = 2^-24 (float32) and a final rounding to bf16 of 2^-8 of the value where the output is bf16:
  * lookup: one float32 product per element, so bit-exact;
  * table gradient: (m + 4) u times the sum of the magnitudes added, m = tokens of the row (any order of m float32
    additions, the scaling and the rounding);
  * 8-bit rows: whole numbers equal to the 64-bit ones except where y / scale lies within 2e-4 of the middle between
    two (127 (a few u) < 5e-5 is the error of the quotient); scales within 4e-6 (at most 32 additions in a row per
    thread, then 6 + 16 over lanes and waves, of squares, halved by the root, and the epilogue's roundings);
  * 8-bit product: the sum is exact; 4 u (|product| + |bias|) for the epilogue's float32 operations;
  * log probabilities, log sums and entropies: 1e-5 + 4 u |value|.  The terms' own errors are below 2 u (1 + |d|) of
    e^d, and up to ~2,200 terms are added in a row per lane, whose roundings grow like a random walk: sqrt(2200) u =
    2.8e-6.  The alternatives' tokens are exact, ties included;
  * gradients of log probabilities: (1e-5 + 8 u) of |g| p + |gH| p (|log p| + H) plus, at the token, 2 u |g|.
"""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("needs a GPU", allow_module_level=True)

from paper_1611_09482_amd import ops  # noqa: E402

U = 2.0 ** -24
F32, BF16 = torch.float32, torch.bfloat16
TYPES = [F32, BF16]
INF = math.inf


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def randn(seed, *shape):
    return torch.randn(shape, generator=gen(seed), device="cuda")


def ints(seed, lo, hi, *shape):
    return torch.randint(lo, hi, shape, generator=gen(seed), device="cuda", dtype=torch.int32)


def odd_view(t, off=1):
    """The same values as rows of a wider array that start at an odd element."""
    wide = torch.zeros((t.shape[0], t.shape[1] + 3), dtype=t.dtype, device=t.device)
    v = wide[:, off:off + t.shape[1]]
    v.copy_(t)
    return v


def out_rounding(dtype):
    return 2.0 ** -8 if dtype == BF16 else 0.0


# ---- lookup ----

@pytest.mark.parametrize("channels", [1, 3, 8, 100, 512, 1030, 2049, 5000])
@pytest.mark.parametrize("dtype", TYPES)
def test_embed(channels, dtype):
    V = 77
    table = randn(channels, V, channels).to(dtype)
    for n, out_dtype in [(1, F32), (7, BF16), (1000, dtype)]:
        tok = ints(n, -2, V + 2, n)
        inside = (tok >= 0) & (tok < V)
        want = table[torch.where(inside, tok, 0).long()].float() * 3.25
        want = torch.where(inside[:, None], want, 0.0).to(out_dtype)
        for t in (table, odd_view(table)):
            got = ops.embed(t, tok, scale=3.25, out=torch.full((n, channels), 7.0, dtype=out_dtype, device="cuda"))
            assert torch.equal(got, want), (n, out_dtype, t.stride())
        wide = torch.full((n, channels + 5), 7.0, dtype=out_dtype, device="cuda")
        ops.embed(table, tok, scale=3.25, out=wide[:, 1:1 + channels])
        assert torch.equal(wide[:, 1:1 + channels], want) and torch.all(wide[:, 0] == 7) and torch.all(wide[:, 1 + channels:] == 7)


def test_embed_many_rows_and_shapes():
    """Several rows per thread (large calls), leading dimensions, no tokens at all."""
    table = randn(1, 300, 64).to(BF16)
    tok = ints(2, 0, 300, 4, 50, 999)
    assert torch.equal(ops.embed(table, tok), table[tok.long()])
    assert ops.embed(table, tok[:0]).shape == (0, 50, 999, 64)
    big = ints(3, 0, 300, 400003)
    assert torch.equal(ops.embed(table, big, scale=0.5), (table[big.long()].float() * 0.5).to(BF16))


def test_embed_rows_past_four_gigabytes():
    V, D = 1100, 1 << 21  # 4.6 GB of bf16
    table = torch.empty((V, D), dtype=BF16, device="cuda")
    tok = torch.tensor([0, V - 1, 1023, 1024, V - 1], dtype=torch.int32, device="cuda")
    for v in (0, 1023, 1024, V - 1):
        table[v] = v + 1
    got = ops.embed(table[:, :512], tok)
    assert torch.equal(got.float(), (tok + 1).to(BF16).float()[:, None].expand(-1, 512))


# ---- the table's gradient ----

def plain_embed_grad(grad, tok, V, scale):
    """(sums, sums of magnitudes, tokens per row) in 64 bits."""
    inside = (tok >= 0) & (tok < V)
    t, g = tok[inside].long(), grad[inside].double()
    zero = torch.zeros((V, grad.shape[1]), dtype=torch.float64, device=grad.device)
    return (zero.index_add(0, t, g) * scale, zero.index_add(0, t, g.abs()) * abs(scale),
            torch.bincount(t, minlength=V).double())


def token_pattern(kind, n, V, seed):
    if kind == "uniform":
        return ints(seed, 0, V, n)
    if kind == "same":
        return torch.full((n,), V // 2, dtype=torch.int32, device="cuda")
    if kind == "frequent":
        w = 1 / (torch.arange(V, device="cuda", dtype=torch.float64) + 2)
        at = torch.cumsum(w / w.sum(), 0)
        u = torch.rand((n,), generator=gen(seed), device="cuda", dtype=torch.float64)
        return torch.searchsorted(at, u).clamp(max=V - 1).int()
    if kind == "descending":
        return (V - 1 - torch.arange(n, device="cuda") % V).sort(descending=True).values.int()
    assert kind == "padded"
    t = ints(seed, 0, V, n)
    t[::2] = -1
    t[1::5] = V
    return t


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,V,D,kind", [
    (1, 1, 1, "uniform"), (1, 50001, 8, "uniform"), (2, 2, 3, "same"), (63, 5, 64, "uniform"), (64, 256, 100, "padded"),
    (65, 257, 257, "frequent"), (2047, 600, 33, "descending"), (2049, 256, 512, "frequent"), (4096, 256, 40, "same"),
    (10656, 256, 512, "uniform"), (9999, 50001, 130, "frequent"), (70000, 511, 72, "same"), (70001, 512, 24, "padded"),
    (70000, 300000, 16, "frequent"), (140001, 1000, 520, "frequent"), (3000, 256, 2056, "padded"),
    (5000, 1 << 20, 9, "uniform"), (5000, (1 << 27) + 5, 1, "uniform"), (300000, 70, 1100, "frequent"),
    (40000, 2500, 2048, "uniform"), (1000, 60, 64, "uniform"), (30000, 3, 4, "same"),
    (511, 300, 520, "frequent"), (512, 70000, 100, "padded"), (513, 40, 1024, "frequent"), (512, 9, 300, "same"),
    (500, 17, 1031, "descending"), (1024, 256, 512, "frequent"), (1024, 4096, 250, "same"), (1024, 1, 1030, "same"),
    (1025, 31, 20, "padded"), (1024, 4097, 64, "frequent"), (700, 900, 3, "padded"), (512, 2049, 256, "same"),
    (511, 2048, 256, "descending"), (66, 5000, 2, "frequent"), (1, 1, 2056, "uniform"), (20000, 300000, 67, "frequent"),
    (16385, 5, 64, "padded"), (17000, 511, 65, "same"), (30000, 66000, 64, "descending"),
])
def test_embed_grad(n, V, D, kind, dtype):
    tok = token_pattern(kind, n, V, n + V)
    grad = randn(n, n, D).to(dtype)
    padding = (tok < 0) | (tok >= V)
    grad[padding] = math.nan  # padding tokens take no part
    want, mag, count = plain_embed_grad(grad, tok, V, 1.5)
    for out_dtype in TYPES:
        got = ops.embed_grad(grad, tok, V, scale=1.5, out=torch.full((V, D), 9.0, dtype=out_dtype, device="cuda"))
        bar = (count[:, None] + 4) * U * mag + out_rounding(out_dtype) * want.abs()
        assert bool(((got.double() - want).abs() <= bar).all()), float((got.double() - want).abs().max())
        assert bool((got[count == 0] == 0).all())
    again = ops.embed_grad(odd_view(grad), tok, V, scale=1.5)
    assert torch.equal(again, ops.embed_grad(grad, tok, V, scale=1.5))


def test_embed_grad_nothing_and_broadcast():
    out = torch.full((40, 10), 3.0, device="cuda")
    assert not ops.embed_grad(torch.empty((0, 10), device="cuda"), ints(1, 0, 40, 0), 40, out=out).any()
    tok = ints(2, -1, 40, 5, 30)
    assert not ops.embed_grad(randn(1, 5, 30, 10), torch.full_like(tok, -1), 40).any()
    row = randn(3, 10)
    got = ops.embed_grad(row.expand(5, 30, 10), tok, 40, scale=2.0)
    count = torch.bincount(tok[tok >= 0].long(), minlength=40)
    want = count[:, None] * row.double() * 2
    assert bool(((got - want).abs() <= (count[:, None] + 4) * U * want.abs()).all())
    wide = torch.full((40, 14), 5.0, device="cuda")
    ops.embed_grad(row.expand(5, 30, 10), tok, 40, scale=2.0, out=wide[:, 3:13])
    assert torch.equal(wide[:, 3:13], got) and bool((wide[:, :3] == 5).all()) and bool((wide[:, 13:] == 5).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,V,D", [(17000, 700, 67), (20000, 150001, 90), (40000, 400, 1030)])
def test_embed_grad_clears_between(n, V, D, dtype):
    """Rows named by one call and not by the next are cleared, and nothing is written beside the rows."""
    grad, even = randn(1, n, D), ints(2, 0, V // 2, n) * 2
    wide = torch.full((V, D + 5), 7.0, dtype=dtype, device="cuda")
    for tok in (even, even + 1, even, torch.full_like(even, V), even + 1):
        wide[:, 1:D + 1] = 9.0
        ops.embed_grad(grad, tok, V, out=wide[:, 1:D + 1])
        want, mag, count = plain_embed_grad(grad, tok, V, 1.0)
        got = wide[:, 1:D + 1].double()
        assert bool(((got - want).abs() <= (count[:, None] + 4) * U * mag + out_rounding(dtype) * want.abs()).all())
        assert bool((got[count == 0] == 0).all()) and bool((wide[:, 0] == 7).all()) and bool((wide[:, D + 1:] == 7).all())


def test_embed_grad_against_differences():
    """The lookup is linear in the table, so a difference of any width is its derivative."""
    V, D, n = 30, 48, 500
    table, d, w = randn(1, V, D), randn(2, V, D), randn(3, n, D)
    tok = ints(4, -1, V, n)
    up, down = ops.embed(table + d, tok, scale=0.75), ops.embed(table - d, tok, scale=0.75)
    slope = float((w.double() * (up.double() - down.double())).sum() / 2)
    terms = ops.embed_grad(w, tok, V, scale=0.75).double() * d.double()
    bar = 40 * U * float((w.abs().double() * (up.abs() + down.abs())).sum() + terms.abs().sum())
    assert abs(slope - float(terms.sum())) <= bar


def test_embed_grad_rows_past_four_gigabytes():
    n, D = 1100, 1 << 21
    grad = torch.empty((n, D), dtype=BF16, device="cuda")[:, :64]
    grad.copy_(randn(5, n, 64))
    tok = ints(6, 0, 50, n)
    want, mag, count = plain_embed_grad(grad, tok, 50, 1.0)
    got = ops.embed_grad(grad, tok, 50)
    assert bool(((got.double() - want).abs() <= (count[:, None] + 4) * U * mag).all())


# ---- 8-bit rows ----

def check_rows(y, q, scale):
    """q, scale against the float64 rows y."""
    top = y.abs().amax(-1)
    s = top / 127
    assert bool(((scale.double() - s).abs() <= 4e-6 * s).all())
    x = y / s[..., None]
    want = torch.round(x)
    near_middle = ((x - torch.floor(x)) - 0.5).abs() < 2e-4
    assert bool(((q.double() == want) | (near_middle & ((q.double() - want).abs() <= 1))).all())
    assert int(q.abs().max()) <= 127 and bool((q.abs().amax(-1) == 127).all())


WIDTHS = [1, 7, 8, 9, 500, 512, 513, 1024, 1030, 2048, 2049, 4096, 5001, 8192, 8200, 16384, 20000, 32768]


@pytest.mark.parametrize("channels", WIDTHS)
@pytest.mark.parametrize("dtype", TYPES)
def test_norm_quant(channels, dtype):
    for rows in (1, 5):
        x, r = randn(rows, rows, channels).to(dtype), (3 * randn(9, rows, channels)).to(dtype)
        gain = 1 + 0.3 * randn(4, channels)
        gain[gain.abs() < 0.05] = 0.05  # a row of one channel stays away from zero
        h = x.double() + r.double()
        y = h / torch.sqrt((h * h).mean(-1, keepdim=True) + 1e-5) * gain.double()
        got = ops.norm_quant(x, gain, residual=r, eps=1e-5, values=True)
        check_rows(y, got.q, got.scale)
        assert torch.equal(got.summed, (x.float() + r.float()).to(dtype))
        assert torch.equal(got.values, (got.q.float() * got.scale[:, None]).to(BF16))
        # no residual, no gain, rows that start at odd elements
        h = x.double()
        y = h / torch.sqrt((h * h).mean(-1, keepdim=True) + 1e-6)
        got = ops.norm_quant(odd_view(x))
        check_rows(y, got.q, got.scale)
        assert got.summed is None and got.values is None
        got = ops.quant_rows(x)
        check_rows(x.double(), got.q, got.scale)


def test_norm_quant_in_place_and_views():
    x, r, gain = randn(1, 6, 5, 300).to(BF16), randn(2, 6, 5, 300).to(BF16), 1 + 0.1 * randn(3, 300)
    want = ops.norm_quant(x, gain, residual=r, values=True)
    stream = r.clone()
    got = ops.norm_quant(x, gain, residual=stream, out=(torch.empty_like(want.q), torch.empty_like(want.scale), stream, None))
    assert got.summed is stream and torch.equal(stream, want.summed)
    assert torch.equal(got.q, want.q) and torch.equal(got.scale, want.scale)
    q = torch.full((30, 311), 99, dtype=torch.int8, device="cuda")
    v = torch.full((30, 303), 9.0, dtype=BF16, device="cuda")
    ops.norm_quant(x.view(30, 300)[::1], gain, residual=r.view(30, 300),
                   out=(q[:, 11:], torch.empty(30, device="cuda"), None, v[:, 1:301]))
    assert torch.equal(q[:, 11:], want.q.view(30, 300)) and bool((q[:, :11] == 99).all())
    assert torch.equal(v[:, 1:301], want.values.view(30, 300)) and bool((v[:, 0] == 9).all()) and bool((v[:, 301:] == 9).all())
    one = ops.norm_quant(x[0, :1].expand(4, 300), gain, residual=r[0, :1].expand(4, 300))
    assert torch.equal(one.q, want.q[0, :1].expand(4, 300))
    assert ops.norm_quant(x[:0]).q.shape == (0, 5, 300)


@pytest.mark.parametrize("channels", [5, 300, 3000, 9000])
@pytest.mark.parametrize("dtype", TYPES)
def test_norm_quant_special_rows(channels, dtype):
    x = randn(1, 8, channels).to(dtype)
    x[1] = 0
    x[2, channels // 2] = math.nan
    x[3, channels - 1] = INF
    x[4, 0] = -INF
    x[5] = 2.0 ** -126 if dtype == F32 else 2.0 ** -120
    x[5] *= 2.0 ** -4  # below what is told apart from zero
    for got in (ops.norm_quant(x, values=True), ops.quant_rows(x)):
        assert torch.isnan(got.scale).tolist() == [False, False, True, True, True, False, False, False]
        assert got.scale[1] == 0 and got.scale[5] == 0
        for r in range(1, 6):
            assert not got.q[r].any()
    clean = ops.norm_quant(x[[0, 6, 7]], values=True)
    got = ops.norm_quant(x, values=True)
    assert torch.equal(got.q[[0, 6, 7]], clean.q) and torch.equal(got.values[[0, 6, 7]], clean.values)
    assert torch.isnan(got.values[2:5].float()).all() and not got.values[1].any() and not got.values[5].any()
    zero_gain = ops.norm_quant(x[:1], torch.zeros(channels, device="cuda"))
    assert zero_gain.scale[0] == 0 and not zero_gain.q.any()


# ---- 8-bit product ----

def plain_matmul(x, sx, w, sw, bias):
    """(result, magnitude for the bar) in 64 bits; the integer sums are exact in them."""
    y = torch.matmul(x.double(), w.double().t().contiguous()) * sx.double()[:, None] * sw.double()
    b = torch.zeros_like(sw).double() if bias is None else bias.double()
    return y + b, y.abs() + b.abs()


def check_matmul(x, w, bias, seed, out_dtype, got=None):
    M, N = x.shape[0], w.shape[0]
    sx, sw = 0.5 + torch.rand(M, device="cuda", generator=gen(seed)), 0.01 + torch.rand(N, device="cuda", generator=gen(seed + 1))
    want, mag = plain_matmul(x, sx, w, sw, bias)
    got = ops.matmul_quant(x, sx, w, sw, bias=bias, dtype=out_dtype)
    bar = 4 * U * mag + out_rounding(out_dtype) * want.abs()
    worst = float(((got.double() - want).abs() - bar).max())
    assert worst <= 0, worst


def bytes_(seed, *shape):
    return torch.randint(-128, 128, shape, generator=gen(seed), device="cuda", dtype=torch.int8)


@pytest.mark.parametrize("M", [1, 2, 15, 16, 17, 33, 64, 65, 128, 129, 300])
@pytest.mark.parametrize("K", [1, 15, 16, 17, 63, 64, 65, 127, 128, 129, 300, 1000, 4096, 5000])
def test_matmul_quant(M, K):
    for N, out_dtype, with_bias in [(1, F32, True), (3, BF16, False), (63, F32, False), (130, BF16, True), (515, F32, True)]:
        x, w = bytes_(M + K, M, K), bytes_(N + K, N, K)
        check_matmul(x, w, randn(1, N) if with_bias else None, M, out_dtype)


@pytest.mark.parametrize("M", [5, 40, 200, 700])
def test_matmul_quant_views(M):
    """Rows that start at any byte, repeated rows, outputs between other columns, leading dimensions."""
    K, N = 333, 150
    x, w, b = bytes_(1, M, K), bytes_(2, N, K), randn(3, N)
    check_matmul(odd_view(x), odd_view(w, 2), b, 3, F32)
    check_matmul(odd_view(x, 3), w, b, 3, BF16)
    check_matmul(x[:1].expand(M, K), w, None, 3, F32)
    sx, sw = torch.rand(M, device="cuda"), torch.rand(N, device="cuda")
    want = ops.matmul_quant(x, sx, w, sw, bias=b, dtype=F32)
    for dtype in TYPES:
        wide = torch.full((M, N + 9), 7.0, dtype=dtype, device="cuda")
        ops.matmul_quant(x, sx, w, sw, bias=b, out=wide[:, 5:5 + N])
        assert torch.equal(wide[:, 5:5 + N], want.to(dtype))
        assert bool((wide[:, :5] == 7).all()) and bool((wide[:, 5 + N:] == 7).all())
    y = ops.matmul_quant(x.view(M // 5, 5, K), sx.view(M // 5, 5), w, sw, bias=b, dtype=F32)
    assert torch.equal(y.view(M, N), want)
    assert ops.matmul_quant(x[:0], sx[:0], w, sw).shape == (0, N)


@pytest.mark.parametrize("M,N", [(3, 40), (140, 140)])
def test_matmul_quant_largest_sums(M, N):
    """Sums that reach the ends of 32 bits, with signs of both kinds."""
    K = 131071
    x = torch.full((M, K), -128, dtype=torch.int8, device="cuda")
    w = torch.full((N, K), -128, dtype=torch.int8, device="cuda")
    w[1::2] = 127
    one, many = torch.ones(M, device="cuda"), torch.ones(N, device="cuda")
    got = ops.matmul_quant(x, one, w, many, dtype=F32)
    assert bool((got[:, 0::2] == float(np.float32(16384 * K))).all())
    assert bool((got[:, 1::2] == float(np.float32(-128 * 127 * K))).all())


@pytest.mark.parametrize("M,N,K", [(1000, 1500, 640), (260, 4100, 2112), (2049, 770, 1040)])
def test_matmul_quant_large(M, N, K):
    check_matmul(bytes_(1, M, K), bytes_(2, N, K), randn(3, N), 4, F32)
    check_matmul(bytes_(1, M, K), bytes_(2, N, K), None, 4, BF16)


@pytest.mark.parametrize("M,N,K", [(4100, 8200, 200), (4099, 8193, 128), (130, 48001, 130), (257, 40000, 129)])
def test_matmul_quant_several_tiles_per_block(M, N, K):
    """More tiles than the device holds blocks, with ragged last ones, K of one and two stages and a byte more."""
    x, w, b = bytes_(1, M, K), bytes_(2, N, K), randn(3, N)
    check_matmul(x, w, b, 4, BF16)
    check_matmul(odd_view(x), odd_view(w), None, 4, F32)


@pytest.mark.parametrize("M,N,K", [(70, 90, 8192), (100, 300, 5001), (300, 515, 4097), (129, 129, 1100)])
def test_matmul_quant_k_in_parts(M, N, K):
    """Few tiles and a long sum: parts of k are summed apart and added."""
    x, w, b = bytes_(1, M, K), bytes_(2, N, K), randn(3, N)
    check_matmul(x, w, b, 4, F32)
    check_matmul(x, w, None, 4, BF16)
    check_matmul(odd_view(x, 2), odd_view(w), b, 4, F32)


def test_matmul_quant_rows_far_apart():
    """Rows megabytes apart: offsets inside a tile pass 2^31."""
    K, far = 300, (1 << 23) + 16
    x = torch.zeros((200, far), dtype=torch.int8, device="cuda")[:, :K]
    x.copy_(bytes_(1, 200, K))
    w = torch.zeros((260, far), dtype=torch.int8, device="cuda")[:, :K]
    w.copy_(bytes_(2, 260, K))
    check_matmul(x, w, randn(3, 260), 4, F32)
    check_matmul(x[:9], w, None, 4, F32)
    check_matmul(x[:50], w, None, 4, BF16)


def test_matmul_quant_scales_not_finite():
    """A row or channel whose scale is NaN (a poisoned 8-bit row) poisons its own outputs only."""
    x, w = bytes_(1, 20, 64), bytes_(2, 30, 64)
    sx, sw = torch.ones(20, device="cuda"), torch.ones(30, device="cuda")
    want = ops.matmul_quant(x, sx, w, sw, dtype=F32)
    sx[3], sw[7] = math.nan, 0.0
    got = ops.matmul_quant(x, sx, w, sw, dtype=F32)
    assert torch.isnan(got[3]).all() and bool((got[:3, 7] == 0).all())
    got[3], got[:, 7] = want[3], want[:, 7]
    assert torch.equal(got, want)


# ---- log probabilities ----

def plain_log_probs(z, tok, top):
    """Float64 (logp, entropy, lse, ids, top log probabilities) with the rules for rows without tokens."""
    z = z.double()
    V = z.shape[1]
    bad = (torch.isnan(z) | (z == INF)).any(1)
    empty = (z == -INF).all(1) & ~bad
    m = z.amax(1, keepdim=True)
    d = z - torch.where(empty[:, None], 0.0, m)  # beside logits of 1e38 the log of the sum would be lost even in 64 bits
    ls = torch.log(d.exp().sum(1))
    lse = torch.where(empty, -INF, m[:, 0] + ls)
    lp = torch.where(empty[:, None], -INF, d - ls[:, None])
    p = lp.exp()
    ent = -torch.where(p > 0, p * lp, 0.0).sum(1)
    inside = (tok >= 0) & (tok < V)
    logp = torch.where(inside, lp.gather(1, torch.where(inside, tok, 0).long()[:, None])[:, 0], 0.0)
    ids = torch.sort(torch.where(torch.isnan(z), -INF, z) + 0.0, dim=1, descending=True, stable=True).indices[:, :top]
    tlp = lp.gather(1, ids)
    nan = torch.full((), math.nan, dtype=torch.float64, device=z.device)
    logp = torch.where(bad & inside, nan, logp)
    return logp, torch.where(bad, nan, ent), torch.where(bad, nan, lse), ids, torch.where(bad[:, None], nan, tlp)


def near(got, want):
    got = got.double()
    bar = 1e-5 + 4 * U * want.abs()
    ok = (got == want.float().double()) | (torch.isnan(got) & torch.isnan(want)) | ((got - want).abs() <= bar)
    assert bool(ok.all()), (got[~ok][:4], want[~ok][:4])


def check_log_probs(z, tok, top):
    got, want = ops.log_probs(z, tok, top=top), plain_log_probs(z, tok, top)
    near(got.lse, want[2])
    near(got.entropy, want[1])
    near(got.logp, want[0])
    assert torch.equal(got.top_ids.long(), want[3])
    near(got.top_logp, want[4])


VOCABS = [1, 2, 5, 63, 64, 65, 255, 256, 257, 512, 513, 1023, 1024, 1025, 2047, 2049, 4097, 50001, 140001]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", VOCABS)
def test_log_probs(V, dtype):
    for rows, top in [(1, min(V, 64)), (5, min(V, 7)), (3, 0), (2, 1)]:
        z = (3 * randn(V + rows, rows, V)).to(dtype)
        z[0] *= 0.1
        tok = ints(rows, 0, V, rows)
        tok[-1] = V if rows > 1 else tok[-1]
        check_log_probs(z, tok, top)
        check_log_probs(odd_view(z), tok, top)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", [3, 200, 256, 1500, 6001, 70000])
def test_log_probs_masks(V, dtype):
    low = torch.finfo(dtype).min
    rows = 16
    z = (2 * randn(V, rows, V)).to(dtype)
    tok = ints(1, 0, V, rows)
    z[0] = -INF                                   # nothing left
    z[1] = -INF
    z[1, V - 1] = -5.0                            # one token left
    z[2] = low                                    # all at the type's lowest value: even
    z[3, : V // 2] = low                          # half masked that way
    z[4, 1:] = -INF                               # the first only
    z[5, ::2] = -INF
    z[6, V // 2] = math.nan
    z[7, V - 1] = INF
    z[8] = z[8] + 10000                           # far from zero
    z[9] = torch.finfo(dtype).max                 # even at the other end
    z[10] = 0.0
    z[10, ::2] = -0.0                             # zeros of both signs are equal
    z[11] = torch.round(z[11].float()).to(dtype)  # many ties
    z[12, 1:] = low
    z[12, 0] = torch.finfo(dtype).max             # the type's whole range between two logits
    z[13] = -INF
    z[13, 0] = math.nan                           # NaN and nothing else
    z[14, 0] = -INF
    tok[14] = 0                                   # a masked token is given
    tok[15] = -1
    for top in (0, 1, min(V, 20), min(V, 64)):
        check_log_probs(z, tok, top)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", [256, 3000, 90000])
def test_log_probs_orders(V, dtype):
    """Rising, falling and constant rows: every batch, or none after the first, has new alternatives."""
    ramp = torch.arange(V, device="cuda").float() / V * 30
    z = torch.stack([ramp, ramp.flip(0), torch.full((V,), 1.5, device="cuda"), (ramp * 7) % 3]).to(dtype)
    for top in (1, 5, 64):
        check_log_probs(z, ints(1, 0, V, 4), top)


def test_log_probs_many_rows_and_views():
    z = 4 * randn(1, 3001, 256)
    check_log_probs(z, ints(2, -3, 259, 3001), 4)
    check_log_probs(z.to(BF16)[::7], ints(3, 0, 256, 429), 64)
    check_log_probs(z[:1].expand(50, 256), ints(4, 0, 256, 50), 2)
    got = ops.log_probs(z.view(3001, 1, 256)[:30].view(5, 6, 256), ints(2, -3, 259, 3001)[:30].view(5, 6), top=4)
    flat = ops.log_probs(z[:30], ints(2, -3, 259, 3001)[:30], top=4)
    assert got.logp.shape == (5, 6) and got.top_ids.shape == (5, 6, 4)
    for a, b in zip(got, flat):
        assert torch.equal(a.reshape(b.shape), b)
    wide = 2 * randn(5, 1500, 5000)
    check_log_probs(wide, ints(6, 0, 5000, 1500), 3)
    empty = ops.log_probs(z[:0], ints(1, 0, 9, 0), top=4)
    assert empty.logp.shape == (0,) and empty.top_ids.shape == (0, 4)


def test_log_probs_rows_past_four_gigabytes():
    z = torch.empty((1100, 1 << 21), dtype=BF16, device="cuda")[:, :5000]
    z.copy_(2 * randn(7, 1100, 5000))
    tok = ints(8, 0, 5000, 1100)
    check_log_probs(z, tok, 5)
    check_grad(z, tok, True)


# ---- their gradient ----

def plain_grad(z, tok, lse, ent, g, gh):
    """(gradient, magnitude of the bar) in 64 bits."""
    z, lse, ent, g = z.double(), lse.double(), ent.double(), g.double()
    gh = torch.zeros_like(g) if gh is None else gh.double()
    V = z.shape[1]
    empty = lse == -INF
    inside = (tok >= 0) & (tok < V) & ~empty
    lp = z - torch.where(empty, 0.0, lse)[:, None]
    p = lp.exp()
    plp = torch.where(p > 0, p * lp, 0.0)
    g0 = torch.where(inside, g, 0.0)
    hot = torch.zeros_like(z).scatter_(1, torch.where(inside, tok, 0).long()[:, None], g0[:, None])
    d = hot - g0[:, None] * p - gh[:, None] * (plp + p * ent[:, None])
    mag = (1e-5 + 8 * U) * (g0.abs()[:, None] * p + gh.abs()[:, None] * (plp.abs() + p * ent.abs()[:, None])) + 2 * U * hot.abs()
    return d, mag


def check_grad(z, tok, entropy, in_place=False):
    rows = z.shape[0]
    st = ops.log_probs(z, tok)
    g, gh = randn(11, rows), randn(12, rows) if entropy else None
    want, bar = plain_grad(z, tok, st.lse, st.entropy, g, gh)
    bar = bar + out_rounding(z.dtype) * want.abs() + 1e-40
    got = ops.log_probs_grad(z, tok, st.lse, st.entropy if entropy else None, g, gh, out=z if in_place else None)
    assert got.dtype == z.dtype
    worst = float(((got.double() - want).abs() - bar).max())
    assert worst <= 0, worst


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", [1, 2, 7, 64, 255, 256, 257, 512, 1025, 2049, 4096, 50001])
def test_log_probs_grad(V, dtype):
    for rows, entropy in [(1, False), (6, True)]:
        z = (2 * randn(V, rows, V)).to(dtype)
        tok = ints(rows, -1, V + 1, rows)
        check_grad(z, tok, entropy)
        check_grad(odd_view(z), tok, entropy)
        check_grad(z.clone(), tok, entropy, in_place=True)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", [9, 300, 5000])
def test_log_probs_grad_masks(V, dtype):
    z = (2 * randn(V, 7, V)).to(dtype)
    z[0] = -INF
    z[1, 1:] = -INF
    z[2] = torch.finfo(dtype).min
    z[3, ::2] = torch.finfo(dtype).min
    z[4, ::3] = -INF
    z[5] = z[5] + 1000
    tok = torch.tensor([0, 0, 1, 2, 3, -1, V], dtype=torch.int32, device="cuda")  # row 4: a masked token
    check_grad(z, tok, True)
    check_grad(z, tok, False)
    z[6, V // 2] = math.nan
    st = ops.log_probs(z, tok)
    d = ops.log_probs_grad(z, tok, st.lse, st.entropy, randn(1, 7), randn(2, 7))
    assert torch.isnan(d[6].float()).all() and not torch.isnan(d[:6].float()).any() and not d[0].any()


def test_log_probs_grad_against_differences():
    """Central differences of sum(w logp + v H) along a random direction.  Width 2^-6: the third derivatives of
    these sums are a few cumulants of the direction under p, below 100 for four rows, so the truncation is below
    2^-12 / 6 * 100 = 4e-3; rounding adds 8 values' 1e-5 / 2^-6 = 5e-3."""
    z, d = 1.5 * randn(1, 4, 37), randn(2, 4, 37)
    w, v, tok, e = randn(3, 4), randn(4, 4), ints(5, 0, 37, 4), 2.0 ** -6

    def value(x):
        r = ops.log_probs(x, tok)
        return float((w.double() * r.logp.double() + v.double() * r.entropy.double()).sum())

    slope = (value(z + e * d) - value(z - e * d)) / (2 * e)
    st = ops.log_probs(z, tok)
    grad = ops.log_probs_grad(z, tok, st.lse, st.entropy, w, v)
    assert abs(slope - float((grad.double() * d.double()).sum())) <= 9e-3


# ---- streams, graphs, order of results ----

def everything(table, tok, x, r, gain, wq, logits):
    e = ops.embed(table, tok, scale=2.0)
    n = ops.norm_quant(e + x, gain, residual=r, values=True)
    y = ops.matmul_quant(n.q, n.scale, wq.q, wq.scale, dtype=F32)
    s = ops.log_probs(y, tok, top=5)
    t = ops.log_probs(logits, tok, top=5)
    dy = ops.log_probs_grad(y, tok, s.lse, s.entropy, s.logp, s.entropy)
    dt = ops.embed_grad(dy[:, :e.shape[1]], tok, table.shape[0])
    return list(n) + list(s) + list(t) + [y, dy, dt]


def chain_inputs(seed):
    V, D, n = 700, 256, 90
    table = randn(seed, V, D)
    return (table, ints(seed + 1, -1, V, n), randn(seed + 2, n, D), randn(seed + 3, n, D), 1 + 0.1 * randn(seed + 4, D),
            ops.quant_rows(table), randn(seed + 5, n, 60000))


def test_another_stream_and_the_same_bits():
    args = chain_inputs(20)
    want = everything(*args)
    for a, b in zip(want, everything(*args)):
        assert torch.equal(a, b)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        late = tuple(a.clone() if torch.is_tensor(a) else a for a in args)  # written on the side stream just before
        got = everything(*late)
    side.synchronize()
    for a, b in zip(want, got):
        assert torch.equal(a, b)


def test_graph_replays():
    args = chain_inputs(30)
    for _ in range(2):
        everything(*args)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        everything(*args)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = everything(*args)
    for seed in (40, 50, 60):
        for a, b in zip(args, chain_inputs(seed)):
            if torch.is_tensor(a):
                a.copy_(b)
            else:
                for p, q in zip(a, b):
                    p.copy_(q)
        want = everything(*args)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(want, got):
            assert torch.equal(a, b)


# ---- refusals that need a device's tensors ----

def test_refusals():
    x, tok = randn(1, 4, 6), ints(2, 0, 6, 4)
    f32 = torch.zeros(4, device="cuda")
    i8 = torch.zeros((4, 6), dtype=torch.int8, device="cuda")
    for error, call in [
        (TypeError, lambda: ops.embed(x.half(), tok)),
        (TypeError, lambda: ops.embed(x, tok.long())),
        (ValueError, lambda: ops.embed(x.cpu(), tok)),
        (ValueError, lambda: ops.embed(x.t(), tok)),
        (ValueError, lambda: ops.embed(x, ints(2, 0, 6, 8)[::2])),
        (ValueError, lambda: ops.embed(x, tok, out=x[:, :5])),
        (ValueError, lambda: ops.embed_grad(x[:3], tok, 9)),
        (TypeError, lambda: ops.embed_grad(i8, tok, 9)),
        (ValueError, lambda: ops.embed_grad(x, tok, 9, out=randn(1, 8, 6))),
        (TypeError, lambda: ops.quant_rows(i8)),
        (ValueError, lambda: ops.norm_quant(x, f32)),
        (TypeError, lambda: ops.norm_quant(x, residual=x.to(BF16))),
        (ValueError, lambda: ops.norm_quant(x, residual=x[:2])),
        (ValueError, lambda: ops.norm_quant(x, out=(i8, f32, x[:1].expand(4, 6), None))),
        (TypeError, lambda: ops.matmul_quant(x, f32, i8, f32)),
        (ValueError, lambda: ops.matmul_quant(i8, f32, i8[:, :5], f32)),
        (ValueError, lambda: ops.matmul_quant(i8, f32[:3], i8, f32)),
        (ValueError, lambda: ops.matmul_quant(i8, f32, i8, f32, bias=f32[:2])),
        (TypeError, lambda: ops.matmul_quant(i8, f32, i8, f32, dtype=torch.float16)),
        (ValueError, lambda: ops.log_probs(x, tok[:3])),
        (TypeError, lambda: ops.log_probs(x.double(), tok)),
        (ops.FwgError, lambda: ops.log_probs(x, tok, top=7)),
        (ops.FwgError, lambda: ops.log_probs(randn(1, 4, 100), tok, top=65)),
        (ValueError, lambda: ops.log_probs_grad(x, tok, f32, None, f32, f32)),
        (TypeError, lambda: ops.log_probs_grad(x, tok, f32, f32, f32, out=x.to(BF16))),
        (ops.FwgError, lambda: ops.quant_rows(torch.zeros((1, 32769), device="cuda"))),
        (ops.FwgError, lambda: ops.matmul_quant(torch.zeros((1, 131072), dtype=torch.int8, device="cuda"), f32[:1],
                                                torch.zeros((1, 131072), dtype=torch.int8, device="cuda"), f32[:1])),
    ]:
        with pytest.raises(error):
            call()


# ---- the example: all of them together ----

def test_example_trains_and_serves():
    import examples.score_tokens as example
    first, full, eight = example.main(streams=8, length=600, steps=60)
    assert full < first - 0.5, (first, full)
    # 8 bits: rows and weights are within half a 127th of their largest element, which moves a logit by a few
    # hundredths and a mean log probability by less
    assert abs(eight - full) < 0.03, (full, eight)
