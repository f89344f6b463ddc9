"""What the operators on quantized weights and on a teacher's logits are measured on: one pass of each call that a
program makes when it runs layers from their compressed form, compares the answers with those of the original
checkpoint and works out the gradients.  `run` computes them in plain torch operations, or with `own` set by this
library's calls.

A case is a dict of plain values.  op "linear" and "linear_grad": rows of activations through one layer whose weight
is held as symbols, bin centres and protected values.
  rows, n_in, n_out; in_out: the weight is stored [n_in][n_out] (else [n_out][n_in]); bins: centres of the codebook;
  type of the activations; activation, bias, residual, pre (the sums before the activation are returned too);
  protect_ppm, protect_bf16: protected values; gap: elements between the rows of the activations
op "top_logits" and "distill": rows of logits
  rows, vocab, k, type, temperature; gap; tail: the list comes with the mass of the other logits;
  masked: part of the vocabulary that no row may use (its logits are -inf)
"""
import math

import torch

own = False

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
ACTIVATIONS = ("none", "relu", "gelu", "gelu_tanh", "silu")


def _layer(name, op, rows, n_in, n_out, bins, type, activation="none", bias=True, residual=False, pre=False, in_out=False,
           protect_ppm=1000, protect_bf16=False, gap=0):
    return dict(name=name, op=op, rows=rows, n_in=n_in, n_out=n_out, bins=bins, type=type, activation=activation, bias=bias,
                residual=residual, pre=pre, in_out=in_out, protect_ppm=protect_ppm, protect_bf16=protect_bf16, gap=gap)


def _logits(name, op, rows, vocab, k, type, temperature=1.0, tail=True, masked=0.0, gap=0):
    return dict(name=name, op=op, rows=rows, vocab=vocab, k=k, type=type, temperature=temperature, tail=tail, masked=masked,
                gap=gap)


def listed():
    return [
        # one token through the first half of GPT-2 medium's feed-forward block, weight stored [in][out]: latency
        _layer("token_gpt2_fc", "linear", 1, 1024, 4096, 16, "bf16", "gelu_tanh", in_out=True),
        # one token through a wide layer of a 7B model
        _layer("token_llama_gate", "linear", 1, 4096, 11008, 32, "bf16", "silu", bias=False),
        # a small batch of tokens through the layer back to the residual stream, many protected values
        _layer("batch_llama_down", "linear", 24, 11008, 4096, 64, "f16", residual=True, bias=False, protect_ppm=10000),
        # evaluation in full precision on few rows, odd everything
        _layer("odd_f32", "linear", 197, 1023, 2049, 12, "f32", "gelu", residual=True, pre=True, gap=5, protect_bf16=True),
        # evaluation batches: a prompt's worth of rows through BERT's and a 7B model's layers
        _layer("rows_bert_out", "linear", 512, 768, 768, 8, "f32", residual=True),
        _layer("prompt_llama_gate", "linear", 2048, 4096, 11008, 32, "bf16", "silu", bias=False, pre=True),
        # gradients of a layer for the sensitivities of its weights
        _layer("grad_gpt2_fc", "linear_grad", 1024, 1024, 4096, 16, "bf16", "gelu_tanh", in_out=True),
        _layer("grad_odd_f32", "linear_grad", 515, 1000, 1537, 256, "f32", "gelu", gap=3),
        # the teacher's side: one row while decoding, and the rows of an evaluation batch
        _logits("top_one_row", "top_logits", 1, 50257, 20, "f32"),
        _logits("top_batch", "top_logits", 4096, 32000, 64, "bf16", temperature=2.0),
        # the loss and its gradient: a few rows without the rest's mass, and a batch over GPT-2's vocabulary in padded rows
        _logits("distill_few", "distill", 9, 30522, 16, "f32", tail=False, masked=0.125),
        _logits("distill_batch", "distill", 4096, 50257, 64, "bf16", temperature=2.0, gap=47),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("linear", "linear", "linear_grad", "top_logits", "distill"))
    type = rng.choice(("f32", "bf16", "bf16", "f16"))
    gap = rng.choice((0, 0, rng.randint(1, 64)))
    if op in ("linear", "linear_grad"):
        grad = op == "linear_grad"
        # (fp32 rows and gradients cost several times a bf16 pass; none costs more than the largest listed one)
        budget = 2048 * 4096 * 11008 // (4 if type == "f32" else 3 if grad else 1)
        while True:
            rows, n_in, n_out = _log_int(rng, 1, 2048), _log_int(rng, 64, 11008), _log_int(rng, 64, 11008)
            if rng.random() < 0.5:
                n_in, n_out = -(-n_in // 64) * 64, -(-n_out // 64) * 64
            if rows * n_in * n_out <= budget:
                break
        residual = not grad and rng.random() < 0.5
        return dict(op=op, rows=rows, n_in=n_in, n_out=n_out, bins=rng.choice((4, 6, 8, 12, 16, 32, 64, 128, 256)),
                    type=type, activation=rng.choice(ACTIVATIONS), bias=rng.random() < 0.7, residual=residual,
                    pre=not grad and rng.random() < 0.5, in_out=rng.random() < 0.5,
                    protect_ppm=rng.choice((0, 100, 1000, 5000, 10000)), protect_bf16=rng.random() < 0.3, gap=gap)
    while True:
        rows, vocab = _log_int(rng, 1, 4096), _log_int(rng, 500, 131072)
        if rows * vocab <= (4096 * 32000 if op == "top_logits" else 4096 * 50257) // (2 if type == "f32" else 1):
            break
    return dict(op=op, rows=rows, vocab=vocab, k=_log_int(rng, 1, 128), type=type, temperature=rng.choice((0.5, 1.0, 2.0, 4.0)),
                tail=rng.random() < 0.7, masked=rng.choice((0.0, 0.0, 0.125)), gap=gap)


def _width(bins):
    return (bins + 1).bit_length()


def _rows(gen, rows, cols, gap, type, scale):
    """Rows of normal values, `gap` elements of nobody's between them."""
    x = torch.randn((rows, cols + gap), generator=gen, device=DEV, dtype=torch.float32).mul_(scale).to(TYPES[type])
    return x[:, :cols]


def _codes(gen, case):
    """Symbols, centres and protected values of a weight as the quantizer leaves them: a tenth pruned, equally full bins of
    normal values, the largest magnitudes protected."""
    n, K, w = case["n_in"] * case["n_out"], case["bins"], _width(case["bins"])
    sym = torch.randint(0, 10 * K, (n,), generator=gen, device=DEV, dtype=torch.int32)
    sym = torch.where(torch.rand((n,), generator=gen, device=DEV) < 0.1, 0, sym % K + 2).to(torch.int16)
    count = n * case["protect_ppm"] // 1000000
    at = torch.randint(0, n, (count,), generator=gen, device=DEV).unique()
    sym[at] = 1
    sd = case["n_in"] ** -0.5
    value = (torch.randn((at.numel(),), generator=gen, device=DEV).sign() * sd * (3.0 + torch.rand((at.numel(),), generator=gen, device=DEV)))
    mid = (torch.arange(K, device=DEV, dtype=torch.float64) + 0.5) / K
    centres = torch.zeros(256, device=DEV, dtype=torch.float32)
    centres[:K] = (sd * math.sqrt(2.0) * torch.erfinv(2.0 * mid - 1.0)).float()
    # little-endian bit stream in words of 64 bits
    words = (n * w + 63) // 64
    fields = torch.zeros((-(-n // 64) * 64, w), dtype=torch.uint8, device=DEV)
    fields[:n] = ((sym.unsqueeze(1) >> torch.arange(w, device=DEV, dtype=torch.int16)) & 1).to(torch.uint8)
    octets = (fields.view(-1, 8) << torch.arange(8, device=DEV, dtype=torch.uint8)).sum(1, dtype=torch.uint8)
    packed = octets.view(torch.int64)[:words].clone()
    value = value.to(torch.bfloat16) if case["protect_bf16"] else value
    return dict(packed=packed, centres=centres, index=at.to(torch.int32), value=value)


def _generator(seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed))
    return gen


def _untaught(rows):
    """Rows that a teacher says nothing of (padding): every sixteenth, the tenth first."""
    return torch.arange(rows, device=DEV) % 16 == 9


def prepare(case, seed):
    gen = _generator(seed)
    s = dict(case)
    if case["op"] in ("linear", "linear_grad"):
        rows, n_in, n_out, type, gap = case["rows"], case["n_in"], case["n_out"], case["type"], case["gap"]
        s["codes"] = _codes(gen, case)
        s["x"] = _rows(gen, rows, n_in, gap, type, 1.0)
        s["b"] = torch.randn((n_out,), generator=gen, device=DEV) * 0.1 if case["bias"] else None
        if case["op"] == "linear":
            s["r"] = _rows(gen, rows, n_out, gap, type, 1.0) if case["residual"] else None
        else:
            s["dy"] = _rows(gen, rows, n_out, gap, type, 0.01)
            s["a"] = _rows(gen, rows, n_out, gap, type, 1.0) if case["activation"] != "none" else None
        if own:  # the handle that a program keeps for a layer
            from paper_2306_11800_amd import api
            c, n = s["codes"], n_in * n_out
            room = torch.zeros(1, dtype=torch.int32, device=DEV)
            index, value = (c["index"], c["value"]) if c["index"].numel() else (room, room.float())
            q = api.Quantized(n, 0, (c["packed"], c["centres"], c["centres"], index, value), bins=case["bins"])
            q.n_outlier, q.bf16 = c["index"].numel(), case["protect_bf16"]
            s["layer"] = api.QuantizedLayer(q, n_out, n_in, in_out=case["in_out"], bias=s["b"], activation=case["activation"])
        return s
    rows, vocab, k = case["rows"], case["vocab"], case["k"]
    teacher = torch.randn((rows, vocab), generator=gen, device=DEV) * 2.5
    banned = int(vocab * case["masked"])
    teacher[:, vocab - banned:] = float("-inf")
    if case["op"] == "top_logits":
        s["logits"] = torch.empty((rows, vocab + case["gap"]), dtype=TYPES[case["type"]], device=DEV)[:, :vocab]
        s["logits"].copy_(teacher)
        return s
    T = case["temperature"]
    value, index = torch.topk(teacher, k, 1)
    rest = teacher.scatter(1, index, float("-inf")).div_(T)
    s["tail"] = torch.logsumexp(rest, 1) if case["tail"] else None
    s["index"] = index.to(torch.int32).masked_fill_(_untaught(rows)[:, None], -1)
    s["value"] = value.contiguous()
    # the quantized model answers nearly the same
    noise = torch.randn((rows, vocab), generator=gen, device=DEV) * 0.4
    s["logits"] = torch.empty((rows, vocab + case["gap"]), dtype=TYPES[case["type"]], device=DEV)[:, :vocab]
    s["logits"].copy_(teacher + noise)
    s["g"] = (0.5 + torch.rand((rows,), generator=gen, device=DEV)) / rows
    return s


# ---- the framework's calls ------------------------------------------------------------------------

_kept = []


def _context():
    """The context of the program, made once."""
    if not _kept:
        from paper_2306_11800_amd import api
        _kept.append(api.Context(torch.device(DEV)))
    return _kept[0]


def _own(s):
    ctx = _context()
    if s["op"] == "linear":
        return ctx.linear(s["layer"], s["x"], residual=s["r"], want_pre=s["pre"])
    if s["op"] == "linear_grad":
        return ctx.linear_grad(s["layer"], s["x"], s["dy"], s["a"])
    if s["op"] == "top_logits":
        top = ctx.top_logits(s["logits"], s["k"], s["temperature"])
        return top.index, top.value, top.tail
    from paper_2306_11800_amd import api
    top = api.TopLogits(s["index"], s["value"], s["tail"], s["temperature"])
    loss, saved = ctx.distill(s["logits"], top)
    return loss, ctx.distill_grad(s["logits"], top, saved, s["g"])


# ---- the plain forms -------------------------------------------------------------------------------

def _weight(s):
    """The weight as [n_out][n_in] values in 32 bits."""
    c, K, n, w = s["codes"], s["bins"], s["n_in"] * s["n_out"], _width(s["bins"])
    octets = torch.cat([c["packed"].view(torch.uint8), torch.zeros(2, dtype=torch.uint8, device=DEV)])
    bit = torch.arange(n, device=DEV) * w
    at = bit >> 3
    two = octets[at].to(torch.int32) | (octets[at + 1].to(torch.int32) << 8)
    sym = (two >> (bit & 7).to(torch.int32)) & ((1 << w) - 1)
    table = torch.cat([torch.zeros(2, device=DEV), c["centres"][:K]])
    W = table[sym]
    W[c["index"].to(torch.int64)] = c["value"].float()
    return W.view(s["n_in"], s["n_out"]).t() if s["in_out"] else W.view(s["n_out"], s["n_in"])


def _act(a, kind):
    if kind == "relu":
        return torch.clamp_min(a, 0.0)
    if kind == "gelu":
        return 0.5 * a * (1.0 + torch.erf(a * math.sqrt(0.5)))
    if kind == "gelu_tanh":
        return 0.5 * a * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (a + 0.044715 * a * a * a)))
    if kind == "silu":
        return a / (1.0 + torch.exp(-a))
    return a


def _act_grad(a, kind):
    if kind == "relu":
        return (a > 0.0).to(a.dtype)
    if kind == "gelu":
        return 0.5 * (1.0 + torch.erf(a * math.sqrt(0.5))) + a * torch.exp(-0.5 * a * a) / math.sqrt(2.0 * math.pi)
    if kind == "gelu_tanh":
        c = math.sqrt(2.0 / math.pi)
        t = torch.tanh(c * (a + 0.044715 * a * a * a))
        return 0.5 * (1.0 + t) + 0.5 * a * (1.0 - t * t) * c * (1.0 + 3.0 * 0.044715 * a * a)
    if kind == "silu":
        g = 1.0 / (1.0 + torch.exp(-a))
        return g * (1.0 + a * (1.0 - g))
    return torch.ones_like(a)


def run(s):
    if own:
        return _own(s)
    if s["op"] == "linear":
        a = torch.matmul(s["x"].float(), _weight(s).t())
        if s["b"] is not None:
            a = a + s["b"]
        y = _act(a, s["activation"])
        if s["r"] is not None:
            y = y + s["r"].float()
        y = y.to(TYPES[s["type"]])
        return (y, a.to(TYPES[s["type"]])) if s["pre"] else y
    if s["op"] == "linear_grad":
        d = s["dy"].float()
        if s["a"] is not None:
            d = d * _act_grad(s["a"].float(), s["activation"])
        dx = torch.matmul(d, _weight(s)).to(TYPES[s["type"]])
        x = s["x"].float()
        return dx, torch.matmul(x.t(), d) if s["in_out"] else torch.matmul(d.t(), x), d.sum(0)
    if s["op"] == "top_logits":
        z = s["logits"].float()
        order = torch.sort(z, dim=1, descending=True, stable=True)
        k, scaled = s["k"], order.values / s["temperature"]
        high = scaled[:, k:k + 1]
        high = torch.where(torch.isfinite(high), high, torch.zeros_like(high))
        tail = torch.log(torch.exp(scaled[:, k:] - high).sum(1)) + high[:, 0]
        return order.indices[:, :k].to(torch.int32), order.values[:, :k].contiguous(), tail
    # (the few listed entries, and the normalisers, in 64 bits: the loss is a small difference of logarithms)
    T, u, index = s["temperature"], s["logits"].float() / s["temperature"], s["index"].to(torch.int64)
    there = index >= 0
    none = torch.full_like(s["value"], float("-inf"), dtype=torch.float64)
    t = torch.where(there, s["value"].double() / T, none)
    tail = s["tail"].double() if s["tail"] is not None else none[:, 0]
    taught = there.any(1)
    log_t = torch.where(taught, torch.log(torch.exp(t).sum(1) + torch.exp(tail)), 0.0)
    high = u.amax(1, keepdim=True)
    e = torch.exp(u - high)
    listed_e = torch.where(there, torch.gather(e, 1, index.clamp_min(0)), 0.0)
    rest = e.scatter(1, index.clamp_min(0), torch.where(there, 0.0, torch.gather(e, 1, index.clamp_min(0))))
    sum_in, sum_out = listed_e.double().sum(1), rest.sum(1, dtype=torch.float64)
    total = (sum_in + sum_out)[:, None]
    log_s = torch.log(total) + high.double()
    P, PT = torch.exp(t - log_t[:, None]), torch.exp(tail - log_t)
    v = torch.gather(s["logits"], 1, index.clamp_min(0)).double() / T
    dist = torch.where(there, (v - log_s) - (t - log_t[:, None]), 0.0)
    dist_rest = torch.log(sum_out / total[:, 0]) - (tail - log_t)
    one = P * (torch.expm1(dist) - dist)
    other = torch.where(PT > 0, PT * (torch.expm1(dist_rest) - dist_rest), sum_out / total[:, 0])
    loss = torch.where(taught, one.sum(1) + other, 0.0).float()
    keep = (1.0 - PT * total[:, 0] / sum_out).float()[:, None]
    g = torch.where(taught, s["g"] / T, 0.0)[:, None]
    grad = e * (keep * g / total.float())
    q = torch.exp(v - log_s)
    at_listed = torch.where(there, (g * (q - P)).float(), torch.gather(grad, 1, index.clamp_min(0)))
    return loss, grad.scatter(1, index.clamp_min(0), at_listed).to(s["logits"].dtype)


# ---- in 64 bits, from the definitions ------------------------------------------------------------------

def _weight_exact(s):
    """The weight as it is stored, in 64 bits: every symbol from its own bits."""
    c, n, w = s["codes"], s["n_in"] * s["n_out"], _width(s["bins"])
    out = torch.empty(n, dtype=torch.float64, device=DEV)
    power = 2 ** torch.arange(w, device=DEV, dtype=torch.int16)
    per = 64 * 65536
    for i0 in range(0, n, per):
        i1 = min(n, i0 + per)
        words = c["packed"][i0 * w // 64:(i1 * w + 63) // 64]
        bits = ((words[:, None] >> torch.arange(64, device=DEV)) & 1).to(torch.int16).view(-1)[:(i1 - i0) * w]
        sym = (bits.view(-1, w) * power).sum(1)
        level = c["centres"].double()[(sym - 2).clamp_min(0)]
        out[i0:i1] = torch.where(sym >= 2, level, 0.0)
    out.index_copy_(0, c["index"].long(), c["value"].double())
    return out


def exact(case, seed):
    s = prepare(case, seed)
    f = torch.float64
    if case["op"] in ("linear", "linear_grad"):
        n_in, n_out, kind = case["n_in"], case["n_out"], case["activation"]
        W = _weight_exact(s)
        W = W.view(n_in, n_out) if case["in_out"] else W.view(n_out, n_in).t().contiguous()  # [n_in][n_out]
        x = s["x"].to(f)
        phi = torch.distributions.Normal(torch.zeros((), dtype=f, device=DEV), torch.ones((), dtype=f, device=DEV))
        bend = lambda a: (2.0 / math.pi) ** 0.5 * (a + 0.044715 * a ** 3)  # noqa: E731
        if case["op"] == "linear":
            a = x @ W + (s["b"].to(f) if s["b"] is not None else 0.0)
            y = {"none": lambda: a, "relu": lambda: a.where(a > 0, torch.zeros_like(a)), "gelu": lambda: a * phi.cdf(a),
                 "gelu_tanh": lambda: a * torch.sigmoid(2.0 * bend(a)), "silu": lambda: a * torch.sigmoid(a)}[kind]()
            y = y + s["r"].to(f) if s["r"] is not None else y
            return (y, a) if case["pre"] else y
        d = s["dy"].to(f)
        if s["a"] is not None:
            a = s["a"].to(f)
            p, h = torch.sigmoid(a), torch.sigmoid(2.0 * bend(a))
            slope = (2.0 / math.pi) ** 0.5 * (1.0 + 0.134145 * a ** 2)
            d = d * {"relu": lambda: (a > 0).to(f), "gelu": lambda: phi.cdf(a) + a * phi.log_prob(a).exp(),
                     "gelu_tanh": lambda: h + 2.0 * a * h * (1.0 - h) * slope, "silu": lambda: p + a * p * (1.0 - p)}[kind]()
        dW = x.t() @ d
        return d @ W.t().contiguous(), dW if case["in_out"] else dW.t().contiguous(), d.sum(0)
    T, k = case["temperature"], case["k"]
    z = s["logits"].to(f)
    if case["op"] == "top_logits":
        z = z.sort(1, descending=True).values
        return None, z[:, :k].contiguous(), torch.logsumexp(z[:, k:] / T, 1)
    loss = torch.zeros(case["rows"], dtype=f, device=DEV)
    q = torch.log_softmax(z / T, 1)
    grad = torch.zeros_like(z)
    taught = torch.nonzero((s["index"] >= 0).any(1))[:, 0]
    at = s["index"][taught].long()
    lists = s["value"][taught].to(f) / T
    if case["tail"]:
        lists = torch.cat([lists, s["tail"][taught].to(f)[:, None]], 1)
    p = torch.log_softmax(lists, 1)
    q_in = q[taught].gather(1, at)
    q_out = torch.logsumexp(q[taught].scatter(1, at, float("-inf")), 1, keepdim=True)
    loss[taught] = (p.exp() * (p - torch.cat([q_in, q_out], 1)[:, :p.shape[1]])).sum(1)
    over = p[:, k:].exp() / q_out.exp() if case["tail"] else torch.zeros_like(q_out)
    rest = q[taught].exp() * (1.0 - over)
    grad[taught] = rest.scatter(1, at, q_in.exp() - p[:, :k].exp())
    return loss, grad * (s["g"].to(f) / T)[:, None]


def work(case):
    t = 4 if case["type"] == "f32" else 2
    if case["op"] in ("linear", "linear_grad"):
        M, K, N = case["rows"], case["n_in"], case["n_out"]
        codes = K * N * _width(case["bins"]) / 8 + 8 * (K * N * case["protect_ppm"] // 1000000) + 4 * case["bins"]
        if case["op"] == "linear":
            moved = M * K + M * N * (1 + case["residual"] + case["pre"])
            return {"bytes": codes + t * moved + 4 * N * case["bias"], "flops": 2 * M * K * N}
        moved = 2 * M * K + M * N * (1 + (case["activation"] != "none"))
        return {"bytes": codes + t * moved + 4 * K * N + 4 * N, "flops": 4 * M * K * N}
    M, V, k = case["rows"], case["vocab"], case["k"]
    if case["op"] == "top_logits":
        return {"bytes": t * M * V + M * (8 * k + 4), "flops": 4 * M * V}
    # (the loss reads the logits, and its gradient, which waits for what comes down from above, reads them again)
    return {"bytes": 3 * t * M * V + M * (16 * k + 16), "flops": 10 * M * V}
