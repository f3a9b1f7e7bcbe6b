"""The operators at the two ends of a token model, as cases whose time and outputs are measured.

A case names an operator (`op`) and its sizes:

  embed            rows of a table by token, scaled; padding tokens give zero rows
  embed_grad       the table's gradient: for every row the sum of the gradients at its tokens
  norm_quant       residual addition, RMS norm, 8-bit rows with a scale each; the new residual and the values that
                   the 8 bits stand for come back
  matmul_quant     product of 8-bit rows with 8-bit weights, a scale per token and per output channel
  log_probs        log probability of a given token per row of logits, entropy, log-sum, top alternatives
  log_probs_grad   the logits' gradient, from the gradients of the log probability and of the entropy

With `own` false, `run` computes them by elementary torch operations in 32 bits; with `own` true it calls
`paper_1611_09482_amd.ops`.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
TINY = 2.0 ** -100  # rows whose largest magnitude lies below this are zero in 8 bits


def _case(name, op, **sizes):
    return dict({"op": op}, **(dict(sizes, name=name) if name else sizes))


def listed():
    return [
        # one step of 32 streams of a class model (8-bit mu-law classes, 512 channels): the smallest call
        _case("embed_step", "embed", tokens=32, vocab=256, channels=512, dtype="f32", padded=False),
        # a batch of ragged sequences in one call, padding tokens between them
        _case("embed_batch", "embed", tokens=65521, vocab=50001, channels=2048, dtype="bf16", padded=True),
        # training a class model: few rows, each named by many tokens
        _case("embed_grad_classes", "embed_grad", tokens=32 * 333, vocab=256, channels=512, dtype="f32", padded=False),
        # training with a large vocabulary: most rows rare, some named thousands of times
        _case("embed_grad_vocab", "embed_grad", tokens=65521, vocab=50001, channels=2048, dtype="bf16", padded=True),
        # the last norm before the output product, one token of each of 64 streams
        _case("norm_quant_step", "norm_quant", rows=64, channels=4096, dtype="bf16"),
        # the same over whole sequences
        _case("norm_quant_batch", "norm_quant", rows=16381, channels=4096, dtype="bf16"),
        # logits of one token of 16 streams: the weights are read for few rows
        _case("matmul_quant_step", "matmul_quant", rows=16, outputs=32000, inner=4096, dtype="f32", bias=False),
        # logits of whole sequences
        _case("matmul_quant_batch", "matmul_quant", rows=4093, outputs=32000, inner=4096, dtype="bf16", bias=True),
        # scoring recordings with a class model: 64 streams of 3001 samples
        _case("log_probs_classes", "log_probs", rows=64 * 3001, vocab=256, dtype="f32", top=4, masked=False),
        # one token of 16 streams with 20 alternatives: few long rows
        _case("log_probs_step", "log_probs", rows=16, vocab=131072, dtype="bf16", top=20, masked=True),
        # scoring sequences, odd row length
        _case("log_probs_vocab", "log_probs", rows=4093, vocab=50001, dtype="f32", top=8, masked=True),
        # training: the gradient of the same rows, in bf16
        _case("log_probs_grad_vocab", "log_probs_grad", rows=8190, vocab=50001, dtype="bf16", masked=True),
    ]


def _log(rng, lo, hi):
    """A whole number from lo to hi, spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)) - 1e-9)))))


def draw(rng):
    op = rng.choice(("embed", "embed_grad", "norm_quant", "matmul_quant", "matmul_quant", "log_probs", "log_probs",
                     "log_probs_grad"))
    dtype = rng.choice(("f32", "bf16"))
    if op in ("embed", "embed_grad"):
        channels = _log(rng, 32, 2048)
        return _case("", op, tokens=_log(rng, 1, 65521), vocab=rng.choice((256, _log(rng, 200, 100000))),
                     channels=channels if rng.random() < 0.3 else (channels + 7) // 8 * 8, dtype=dtype,
                     padded=rng.random() < 0.5)
    if op == "norm_quant":
        channels = _log(rng, 32, 8192)
        channels = channels if rng.random() < 0.3 else (channels + 7) // 8 * 8
        return _case("", op, rows=_log(rng, 1, min(16381, 67000000 // channels)), channels=channels, dtype=dtype)
    if op == "matmul_quant":
        inner = _log(rng, 32, 8192)
        inner = inner if rng.random() < 0.3 else (inner + 15) // 16 * 16
        outputs = _log(rng, 64, 32000)
        rows = _log(rng, 1, min(8192, 530000000000 // (inner * outputs)))
        return _case("", op, rows=rows, outputs=outputs, inner=inner, dtype=dtype, bias=rng.random() < 0.5)
    vocab = rng.choice((256, _log(rng, 200, 131072)))
    rows = _log(rng, 1, min(200000, 200000000 // vocab))
    if op == "log_probs":
        return _case("", op, rows=rows, vocab=vocab, dtype=dtype, top=rng.choice((0, 1, 4, 8, 20, 64)),
                     masked=rng.random() < 0.5)
    return _case("", op, rows=rows, vocab=vocab, dtype=dtype, masked=rng.random() < 0.5)


def _probabilities(vocab, device):
    """How often each token comes: mu-law classes of quiet sound for small vocabularies, word frequencies else."""
    v = torch.arange(vocab, device=device, dtype=torch.float64)
    w = torch.exp(-(v - vocab // 2).abs() / 24) + 1e-4 if vocab <= 1024 else 1 / (v + 2.7)
    return w / w.sum()


def _tokens(gen, n, vocab, padded):
    at = torch.cumsum(_probabilities(vocab, "cuda"), 0)
    u = torch.rand((n,), generator=gen, device="cuda", dtype=torch.float64)
    t = torch.searchsorted(at, u).clamp(max=vocab - 1).to(torch.int32)
    if padded:
        t[torch.rand((n,), generator=gen, device="cuda") < 0.02] = -1
    return t


def _logits(gen, tokens, vocab, dtype, masked):
    """Logits of a model that is often right: the given token stands out of noise; masked: the vocabulary's padded
    end and some words are excluded (-inf), and a few rows have nothing left."""
    rows = tokens.shape[0]
    z = torch.randn((rows, vocab), generator=gen, device="cuda").mul_(2.5)
    z[torch.arange(rows, device="cuda"), tokens.long()] += 6.0
    if masked:
        z[:, vocab - vocab // 64:] = -math.inf
        z.masked_fill_(torch.rand((1, vocab), generator=gen, device="cuda") < 0.05, -math.inf)
        z[torch.rand((rows,), generator=gen, device="cuda") < 0.01] = -math.inf
        tokens[torch.rand((rows,), generator=gen, device="cuda") < 0.02] = -1
    return z.to(dtype)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(6151 * seed + 29)
    op, dtype = case["op"], TYPES[case["dtype"]]

    def randn(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    def empty(shape, dtype):
        return torch.empty(shape, dtype=dtype, device="cuda")

    s = {"case": case}
    if op in ("embed", "embed_grad"):
        n, V, D = case["tokens"], case["vocab"], case["channels"]
        s["tokens"] = _tokens(gen, n, V, case["padded"])
        s["scale"] = math.sqrt(D)
        if op == "embed":
            s["table"] = (randn(V, D) / math.sqrt(D)).to(dtype)
            s["out"] = empty((n, D), dtype)
        else:
            s["grad"] = (randn(n, D) * 1e-2).to(dtype)
            s["out"] = empty((V, D), torch.float32)
    elif op == "norm_quant":
        n, D = case["rows"], case["channels"]
        s["x"] = (randn(n, D) * 0.5).to(dtype)
        s["residual"] = (randn(n, D) * (1 + 3 * torch.rand((n, 1), generator=gen, device="cuda"))).to(dtype)
        s["gain"] = 1 + 0.1 * randn(D)
        s["out"] = (empty((n, D), torch.int8), empty((n,), torch.float32), empty((n, D), dtype),
                    empty((n, D), torch.bfloat16))
    elif op == "matmul_quant":
        M, N, K = case["rows"], case["outputs"], case["inner"]
        s["x"] = (randn(M, K) * 32).round_().clamp_(-127, 127).to(torch.int8)
        s["w"] = (randn(N, K) * 32).round_().clamp_(-127, 127).to(torch.int8)
        s["x_scale"] = 0.02 + 0.02 * torch.rand((M,), generator=gen, device="cuda")
        s["w_scale"] = (0.5 + torch.rand((N,), generator=gen, device="cuda")) / (32 * math.sqrt(K))
        s["bias"] = 0.1 * randn(N) if case["bias"] else None
        s["out"] = empty((M, N), dtype)
    else:
        n, V = case["rows"], case["vocab"]
        s["tokens"] = _tokens(gen, n, V, False)
        s["logits"] = _logits(gen, s["tokens"], V, dtype, case["masked"])
        if op == "log_probs":
            k = case["top"]
            s["out"] = (empty((n,), torch.float32), empty((n,), torch.float32), empty((n,), torch.float32),
                        empty((n, k), torch.int32), empty((n, k), torch.float32))
        else:
            # what the forward call left for the gradient, and a weighted loss with an entropy bonus
            s["lse"], s["entropy"] = _statistics(s["logits"])[1:]
            s["grad_logp"] = -(0.5 + torch.rand((n,), generator=gen, device="cuda")) / n
            s["grad_entropy"] = torch.full((n,), -0.01 / n, device="cuda")
            s["out"] = torch.empty_like(s["logits"])
    return s


def _statistics(logits):
    """(logits, lse, entropy) in float32; a row with nothing left has lse -inf and entropy 0."""
    z = logits.float()
    m = z.amax(1, keepdim=True)
    d = z - torch.where(m == -math.inf, 0.0, m)
    e = torch.exp(d)
    total = e.sum(1)
    weighted = torch.where(e > 0, e * d, 0.0).sum(1)
    empty = total == 0
    log_total = torch.log(total)
    return z, m[:, 0] + log_total, torch.where(empty, 0.0, log_total - weighted / torch.where(empty, 1.0, total))


def _embed(s):
    table, t = s["table"], s["tokens"].long()
    inside = (t >= 0) & (t < table.shape[0])
    rows = table[torch.where(inside, t, 0)].float() * s["scale"]
    return torch.where(inside[:, None], rows, 0.0).to(table.dtype)


def _embed_grad(s):
    t, V = s["tokens"].long(), s["case"]["vocab"]
    inside = (t >= 0) & (t < V)
    total = torch.zeros((V + 1, s["grad"].shape[1]), device="cuda")
    total.index_add_(0, torch.where(inside, t, V), s["grad"].float())
    return total[:V] * s["scale"]


def _norm_quant(s):
    h = s["x"].float() + s["residual"].float()
    y = h * torch.rsqrt((h * h).mean(1, keepdim=True) + 1e-6) * s["gain"]
    top = y.abs().amax(1, keepdim=True)
    scale = torch.where(top < TINY, 0.0, top / 127)
    q = torch.round(y / torch.where(scale == 0, 1.0, scale))
    return {"summed": h.to(s["x"].dtype), "scale": scale[:, 0], "values": (q * scale).to(torch.bfloat16)}


def _matmul_quant(s):
    y = (s["x"].float() @ s["w"].float().t()) * s["x_scale"][:, None] * s["w_scale"]
    return (y if s["bias"] is None else y + s["bias"]).to(s["out"].dtype)


def _log_probs(s):
    z, lse, entropy = _statistics(s["logits"])
    t, k, V = s["tokens"].long(), s["case"]["top"], s["case"]["vocab"]
    inside = (t >= 0) & (t < V)
    at = z.gather(1, torch.where(inside, t, 0)[:, None])[:, 0]
    logp = torch.where(inside, torch.where(lse == -math.inf, -math.inf, at - lse), 0.0)
    # whole numbers that order by (logit descending, index ascending)
    bits = (z + 0.0).view(torch.int32).long()
    order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits)
    key = order * (1 << 32) - torch.arange(V, device="cuda")
    ids = (-key.topk(k, dim=1).values) & 0xFFFFFFFF
    top = z.gather(1, ids)
    return {"logp": logp, "entropy": entropy, "lse": lse, "top_ids": ids.to(torch.int32),
            "top_logp": torch.where(top == -math.inf, top, top - lse[:, None])}


def _log_probs_grad(s):
    z, t, V = s["logits"].float(), s["tokens"].long(), s["case"]["vocab"]
    empty = s["lse"] == -math.inf
    inside = (t >= 0) & (t < V) & ~empty
    log_p = z - torch.where(empty, 0.0, s["lse"])[:, None]
    p = torch.exp(log_p)
    g = torch.where(inside, s["grad_logp"], 0.0)[:, None]
    d = -p * g - torch.where(p > 0, p * (log_p + s["entropy"][:, None]), 0.0) * s["grad_entropy"][:, None]
    d.scatter_add_(1, torch.where(inside, t, 0)[:, None], g)
    return d.to(s["logits"].dtype)


def _plain(s):
    return {"embed": _embed, "embed_grad": _embed_grad, "norm_quant": _norm_quant, "matmul_quant": _matmul_quant,
            "log_probs": _log_probs, "log_probs_grad": _log_probs_grad}[s["case"]["op"]](s)


def run(s):
    if not own:
        return _plain(s)
    from paper_1611_09482_amd import ops
    case, op, out = s["case"], s["case"]["op"], s["out"]
    if op == "embed":
        return ops.embed(s["table"], s["tokens"], scale=s["scale"], out=out)
    if op == "embed_grad":
        return ops.embed_grad(s["grad"], s["tokens"], case["vocab"], scale=s["scale"], out=out)
    if op == "norm_quant":
        r = ops.norm_quant(s["x"], s["gain"], residual=s["residual"], eps=1e-6, out=out)
        return {"summed": r.summed, "scale": r.scale, "values": r.values}
    if op == "matmul_quant":
        return ops.matmul_quant(s["x"], s["x_scale"], s["w"], s["w_scale"], bias=s["bias"], out=out)
    if op == "log_probs":
        r = ops.log_probs(s["logits"], s["tokens"], top=case["top"], out=out)
        return {"logp": r.logp, "entropy": r.entropy, "lse": r.lse, "top_ids": r.top_ids, "top_logp": r.top_logp}
    return ops.log_probs_grad(s["logits"], s["tokens"], s["lse"], s["entropy"], s["grad_logp"], s["grad_entropy"],
                              out=out)


def work(case):
    op, es = case["op"], 4 if case["dtype"] == "f32" else 2
    if op in ("embed", "embed_grad"):
        n, V, D = case["tokens"], case["vocab"], case["channels"]
        if op == "embed_grad":
            return {"bytes": 4 * n + n * D * es + V * D * 4, "flops": n * D}
        p = _probabilities(V, "cpu")
        distinct = float((1 - torch.exp(n * torch.log1p(-p))).sum())  # rows that n tokens are expected to name
        return {"bytes": 4 * n + (distinct + n) * D * es, "flops": n * D}
    if op == "norm_quant":
        n, D = case["rows"], case["channels"]
        return {"bytes": n * D * (3 * es + 2) + 4 * (n + D), "flops": 8 * n * D}
    if op == "matmul_quant":
        M, N, K = case["rows"], case["outputs"], case["inner"]
        return {"bytes": M * K + N * K + M * N * es + 4 * (M + N * (2 if case["bias"] else 1)), "flops": 2 * M * N * K}
    n, V = case["rows"], case["vocab"]
    if op == "log_probs":
        return {"bytes": n * V * es + n * (16 + 8 * case["top"]), "flops": 6 * n * V}
    return {"bytes": 2 * n * V * es + 20 * n, "flops": 6 * n * V}


def _blocks(n, per):
    return [slice(i, min(n, i + per)) for i in range(0, n, per)]


def exact(case, seed):
    """The operators' definitions in 64 bits, some rows at a time."""
    s, op = prepare(case, seed), case["op"]
    if op == "embed":
        table = torch.cat([s["table"].double() * s["scale"], s["table"].new_zeros((1, case["channels"])).double()])
        return table[s["tokens"].long()]  # -1 names the zero row at the end
    if op == "embed_grad":
        # tokens in order of their rows; the sum of a row is a difference of running sums over its tokens
        t, at = torch.sort(s["tokens"].long(), stable=True)
        edge = torch.searchsorted(t, torch.arange(case["vocab"] + 1, device="cuda"))
        out = []
        for c in _blocks(case["channels"], 256):
            run_ = torch.cumsum(s["grad"][:, c].double()[at], 0)
            run_ = torch.cat([torch.zeros_like(run_[:1]), run_])
            out.append((run_[edge[1:]] - run_[edge[:-1]]) * s["scale"])
        return torch.cat(out, 1)
    if op == "norm_quant":
        h = s["x"].double() + s["residual"].double()
        y = h / torch.sqrt(h.pow(2).sum(1, keepdim=True) / case["channels"] + 1e-6) * s["gain"].double()
        step = y.abs().max(1, keepdim=True).values / 127
        return {"summed": h, "scale": step[:, 0], "values": torch.round(y / step) * step}
    if op == "matmul_quant":
        w, b = s["w"].double(), s["bias"]
        out = []
        for r in _blocks(case["rows"], 1024):
            y = torch.matmul(s["x"][r].double(), w.t()) * torch.outer(s["x_scale"][r].double(), s["w_scale"].double())
            out.append(y if b is None else y + b.double())
        return torch.cat(out)
    parts = []
    for r in _blocks(case["rows"], max(1, (1 << 27) // case["vocab"])):
        log_p = torch.log_softmax(s["logits"][r].double(), 1)
        empty = torch.isnan(log_p[:, 0])
        log_p = torch.where(empty[:, None], -math.inf, log_p)
        t = s["tokens"][r].long()
        some = t >= 0
        t = t.clamp(min=0)
        p = log_p.exp()
        plogp = torch.where(p > 0, p * log_p, 0.0)
        entropy = -plogp.sum(1)
        if op == "log_probs":
            lse = torch.logsumexp(s["logits"][r].double(), 1)
            logp = torch.where(some, log_p[torch.arange(len(t), device="cuda"), t], 0.0)
            parts.append((logp, entropy, lse, log_p.sort(1, descending=True).values[:, :case["top"]]))
        else:
            g = torch.where(some & ~empty, s["grad_logp"][r].double(), 0.0)
            d = torch.zeros_like(p)
            d[torch.arange(len(t), device="cuda"), t] = g
            d -= g[:, None] * p
            d -= s["grad_entropy"][r].double()[:, None] * (plogp + p * entropy[:, None])
            parts.append(d.to(s["logits"].dtype) if case["rows"] * case["vocab"] > 1 << 30 else d)
    if op == "log_probs_grad":
        return torch.cat(parts)
    logp, entropy, lse, top = (torch.cat(x) for x in zip(*parts))
    return {"logp": logp, "entropy": entropy, "lse": lse, "top_ids": None, "top_logp": top}
