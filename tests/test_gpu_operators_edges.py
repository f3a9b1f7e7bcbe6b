"""The token operators at arguments and sizes where only one of their kernels' paths, or none of the ordinary ones, runs.

Plain evaluations, helpers and bars are those of test_gpu_operators.py."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("needs a GPU", allow_module_level=True)

from paper_1611_09482_amd import ops  # noqa: E402
from test_gpu_operators import (BF16, F32, TYPES, U, bytes_, check_matmul, check_rows, ints, odd_view,  # noqa: E402
                                plain_embed_grad, randn)


# ---- 8-bit rows ----

@pytest.mark.parametrize("channels", [5, 300, 3000, 9000])
@pytest.mark.parametrize("dtype", TYPES)
def test_norm_quant_without_eps(channels, dtype):
    """eps = 0: rows whose every |h gain| is below 2^-120 are zero, whatever 1 / sqrt(mean h^2) is."""
    x = randn(channels, 7, channels).to(dtype)
    x[1] = 0
    x[2] = 2.0 ** -121
    x[3] = (x[3].float() * 2.0 ** -50).to(dtype)  # small, and the squares are normal numbers
    x[4, channels // 2] = math.nan
    x[5] = 0
    x[5, channels - 1] = -3.0
    gain = 1 + 0.1 * randn(1, channels).clamp(-3, 3)
    got = ops.norm_quant(x, gain, eps=0.0, values=True)
    assert torch.isnan(got.scale).tolist() == [False, False, False, False, True, False, False]
    for r in (1, 2):
        assert got.scale[r] == 0 and not got.q[r].any() and not got.values[r].any()
    h = x[[0, 3, 5, 6]].double()
    check_rows(h / torch.sqrt((h * h).mean(-1, keepdim=True)) * gain.double(), got.q[[0, 3, 5, 6]], got.scale[[0, 3, 5, 6]])
    gone = ops.norm_quant(x[:2], gain, residual=-x[:2], eps=0.0)  # the residual takes all of the row away
    assert not gone.scale.any() and not gone.q.any() and not gone.summed.any()
    for rows in (x[:1], x[1:2]):  # a gain of zero
        got = ops.norm_quant(rows, torch.zeros_like(gain), eps=0.0)
        assert got.scale[0] == 0 and not got.q.any()


def test_padding_tokens_rows_through_the_product():
    """The zero row of a padding token stays one: its outputs are the bias."""
    table, tok = randn(1, 50, 256), torch.tensor([3, -1, 7], dtype=torch.int32, device="cuda")
    w, bias = ops.quant_rows(randn(2, 40, 256)), randn(3, 40)
    x = ops.norm_quant(ops.embed(table, tok), eps=0.0)
    y = ops.matmul_quant(x.q, x.scale, w.q, w.scale, bias=bias, dtype=F32)
    assert torch.equal(y[1], bias) and not torch.isnan(y).any()


# ---- sizes past 32 bits ----

def test_sizes_past_32_bits():
    """Refused before anything is allocated or enqueued."""
    x, tok, n = randn(1, 4, 6), torch.zeros(4, dtype=torch.int32, device="cuda"), 2 ** 32 + 6
    wide = torch.empty((1, n), dtype=torch.int8, device="cuda")
    one = torch.ones(1, device="cuda")
    before = torch.cuda.max_memory_allocated()
    for call in (lambda: ops.embed_grad(x, tok, n), lambda: ops.log_probs(x, tok, top=2 ** 32 + 3),
                 lambda: ops.matmul_quant(wide, one, wide, one), lambda: ops.matmul_quant(wide[:, :1], one, wide.t(), one)):
        with pytest.raises(ops.FwgError):
            call()
    assert torch.cuda.max_memory_allocated() == before


# ---- 8-bit product ----

@pytest.mark.parametrize("dtype", TYPES)
def test_matmul_quant_outputs_past_one_launch(dtype):
    """Few rows and 2^27 outputs and more: more blocks of 16 or 32 outputs than one launch has threads for.  Scales are
    powers of two and sums below 256, so every result is exact in both types."""
    rows, N, K = 2, (1 << 27) + 45, 4
    w = torch.randint(-3, 4, (N, K), dtype=torch.int8, device="cuda")
    x = torch.tensor([[1, -2, 3, 1], [2, 0, -1, 3]], dtype=torch.int8, device="cuda")
    sx, sw = torch.tensor([2.0, 0.5], device="cuda"), torch.ones(N, device="cuda")
    sw[::3] = 4.0
    got = ops.matmul_quant(x, sx, w, sw, dtype=dtype)
    for r in range(rows):
        total = torch.zeros(N, device="cuda")
        for k in range(K):
            total += w[:, k] * float(x[r, k])
        assert torch.equal(got[r], (total * sx[r] * sw).to(dtype))
    # the last slice's bias and outputs, rows at odd bytes
    tail = 1 << 26
    bias = (torch.arange(N, device="cuda") % 64).float()
    odd = torch.empty(N * K + 1, dtype=torch.int8, device="cuda")[1:].view(N, K)
    odd.copy_(w)
    again = ops.matmul_quant(x, sx, odd, torch.ones_like(sw), bias=bias, dtype=F32)
    plain = (got.float() / sw + bias)[:, -tail:]
    assert torch.equal(again[:, -tail:], plain)


# ---- the table's gradient ----

def test_embed_grad_tasks_past_one_launch():
    """As many tokens as are supported, one repeated row of gradients: more blocks than one launch has threads for.
    Sums are whole numbers below 2^24, so they are exact."""
    n, V, D = 1 << 30, 256, 769
    if torch.cuda.mem_get_info()[0] < 150 << 30:
        pytest.skip("needs 150 GB of free memory: the workspace holds two partial sums of 64 tokens each")
    tok = torch.arange(n, dtype=torch.int32, device="cuda")
    tok.bitwise_and_(V - 1)
    tok[:V] = 7
    row = torch.arange(D, device="cuda").remainder_(4).float()
    got = ops.embed_grad(row.expand(n, D), tok, V)
    count = torch.full((V,), float(n // V - 1), device="cuda")
    count[7] += V
    del tok
    torch.cuda.empty_cache()
    assert torch.equal(got, count[:, None] * row)


@pytest.mark.parametrize("n,V", [(5, 9), (300, 9), (300, 5000), (512, 70000), (513, 9), (1024, 5000), (3000, 700), (20000, 700)])
def test_padding_at_the_ends_of_32_bits(n, V):
    """The largest and smallest tokens are padding like any other, in every form of the gradient."""
    tok = ints(n, 0, V, n)
    far = torch.tensor([-2 ** 31, -2 ** 31 + 1, 2 ** 31 - 1, 2 ** 31 - 16, V, -1], dtype=torch.int32, device="cuda")
    tok[::2] = far.repeat(n)[:n][::2]
    grad = randn(V, n, 72)
    want, mag, count = plain_embed_grad(grad, tok, V, 1.0)
    got = ops.embed_grad(grad, tok, V, out=torch.full((V, 72), 9.0, device="cuda"))
    assert bool(((got.double() - want).abs() <= (count[:, None] + 4) * U * mag).all()) and bool((got[count == 0] == 0).all())
    rows = ops.embed(got, tok)
    inside = (tok >= 0) & (tok < V)
    assert torch.equal(rows, torch.where(inside[:, None], got[torch.where(inside, tok, 0).long()], 0.0))


# ---- kernels that only large sizes reach ----

@pytest.mark.parametrize("M,N,K", [(3001, 4203, 400), (3001, 4203, 1024), (3001, 4096, 656), (4099, 8193, 272)])
def test_matmul_quant_large_tiles_over_k(M, N, K):
    """Rows on 16 bytes in 256 x 256 tiles: several stages of k, the last one whole or ragged, one tile or several for a
    block.  K ends inside a piece of 16 bytes where rows are longer than it."""
    x, w, b = bytes_(1, M, K), bytes_(2, N, K), randn(3, N)
    check_matmul(x, w, b, 4, BF16)
    check_matmul(x[:, :K - 7], w[:, :K - 7], None, 4, F32)


@pytest.mark.parametrize("M", [1, 5, 16])
@pytest.mark.parametrize("K", [64, 2048, 2176, 4096, 4500, 6148])
def test_matmul_quant_few_rows_many_outputs(M, K):
    """Two tiles of outputs for a block; k ends before, at and after what the sixteen waves take in one and two turns."""
    N = 8205
    x, w, b = bytes_(M, M, K + 1), bytes_(K, N, K + 1), randn(3, N)
    check_matmul(x[:, :K].contiguous(), w[:, :K].contiguous(), b, 4, F32)      # words
    check_matmul(x, w, None, 4, BF16)                                          # any byte, k one longer
    check_matmul(odd_view(x[:, :K - 1], 3), odd_view(w[:, :K - 1]), b, 4, F32)


@pytest.mark.parametrize("M", [17, 31, 32, 33, 64])
@pytest.mark.parametrize("K", [2176, 4097, 6149])
def test_matmul_quant_rows_at_any_byte(M, K):
    """Random bytes through the shifted loads, where several turns of k are in flight."""
    x, w = bytes_(M, M, K), bytes_(K, 515, K)
    check_matmul(odd_view(x), odd_view(w, 2), randn(3, 515), 4, F32)
    check_matmul(odd_view(x, 3), w, None, 4, BF16)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("channels", [31, 1031, 2048])
def test_embed_past_the_caches(channels, dtype):
    """Outputs of 192 MB and more have a store of their own: the same values, nothing beside the rows."""
    n, V = (200 << 20) // (channels * dtype.itemsize), 301
    table, tok = randn(channels, V, channels).to(dtype), ints(2, -2, V + 2, n)
    inside = (tok >= 0) & (tok < V)
    wide = torch.full((n, channels + 3), 7.0, dtype=dtype, device="cuda")
    got = ops.embed(table, tok, scale=3.25, out=wide[:, 1:1 + channels])
    want = ((table.float() * 3.25).to(dtype))[torch.where(inside, tok, 0).long()]
    want[~inside] = 0
    assert torch.equal(got, want) and bool((wide[:, 0] == 7).all()) and bool((wide[:, 1 + channels:] == 7).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("channels", [300, 900, 2048, 3001, 5001, 9001, 20001])
def test_norm_quant_past_the_caches(channels, dtype):
    """Outputs of 192 MB and more: the bits of smaller calls, whose rows are compared in 64 bits."""
    n = (200 << 20) // (channels * (3 + dtype.itemsize)) + 1
    x, r, gain = randn(1, n, channels).to(dtype), (2 * randn(2, n, channels)).to(dtype), 1 + 0.1 * randn(3, channels)
    got = ops.norm_quant(x, gain, residual=r, values=True)
    for i in range(0, n, n // 5):
        part = slice(i, min(n, i + n // 5))
        for a, b in zip(got, ops.norm_quant(x[part], gain, residual=r[part], values=True)):
            assert torch.equal(a[part], b)
    h = x[-9:].double() + r[-9:].double()
    check_rows(h / torch.sqrt((h * h).mean(-1, keepdim=True) + 1e-6) * gain.double(), got.q[-9:], got.scale[-9:])


# ---- more rows than one launch takes ----

MANY = (1 << 23) + 5  # of up to 256 elements: two launches, the second of five rows


def test_embed_of_many_rows():
    table, tok = randn(1, 9, 3), ints(2, -1, 10, MANY)
    inside = (tok >= 0) & (tok < 9)
    got = ops.embed(table, tok, scale=0.5)
    assert torch.equal(got, torch.where(inside[:, None], (table * 0.5)[torch.where(inside, tok, 0).long()], 0.0))


def halves(call, *tensors):
    """The results of a call on the first rows and on the others, put together."""
    cut = 1 << 22
    first, rest = call(*(t[:cut] for t in tensors)), call(*(t[cut:] for t in tensors))
    return [None if a is None else torch.cat([a, b]) for a, b in zip(first, rest)]


def test_rows_of_many_rows():
    x, r, gain = randn(1, MANY, 5), randn(2, MANY, 5), 1 + 0.1 * randn(3, 5)

    def norm(x, r):
        return ops.norm_quant(x, gain, residual=r, values=True)

    for call, tensors in ((norm, (x, r)), (ops.quant_rows, (x,))):
        for a, b in zip(call(*tensors), halves(call, *tensors)):
            assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", TYPES)
def test_log_probs_of_many_rows(dtype):
    z, tok, g, gh = randn(1, MANY, 5).to(dtype), ints(2, -1, 6, MANY), randn(3, MANY), randn(4, MANY)

    def both(z, tok, g, gh):
        s = ops.log_probs(z, tok, top=3)
        return list(s) + [ops.log_probs_grad(z, tok, s.lse, s.entropy, g, gh)]

    for a, b in zip(both(z, tok, g, gh), halves(both, z, tok, g, gh)):
        assert torch.equal(a, b)
