"""The token operators at arguments and sizes where only one of their kernels' paths, or none of the ordinary ones, runs.

Plain evaluations, helpers and bars are those of test_gpu_operators.py."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("needs a GPU", allow_module_level=True)

from paper_1611_09482_amd import ops  # noqa: E402
from test_gpu_operators import F32, TYPES, U, check_rows, ints, plain_embed_grad, randn  # noqa: E402


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
