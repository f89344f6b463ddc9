"""GPU: the quality of a compressed checkpoint's answers and its gradients, and the report that prints it."""
import json

import numpy as np
import pytest
import torch

from paper_2306_11800_amd import api, quality, ratio_report
from tests import answers as A

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def ctx():
    c = api.Context(torch.device(DEV))
    yield c
    c.close()


def chain(ctx, rng, bits, hidden=48, ff=96, vocab=300):
    sizes = [("wte", vocab * hidden), ("h2.mlp.c_fc.weight", hidden * ff), ("h2.mlp.c_fc.bias", ff),
             ("h2.mlp.c_proj.weight", ff * hidden), ("h2.mlp.c_proj.bias", hidden), ("h10.mlp.c_fc.weight", hidden * ff),
             ("h10.mlp.c_fc.bias", ff), ("h10.mlp.c_proj.weight", ff * hidden), ("h10.mlp.c_proj.bias", hidden)]
    ts = [torch.from_numpy((0.1 * rng.standard_t(4, n)).astype(np.float32)).to(DEV) for _, n in sizes]
    qs = ctx.quantize(ts, [(bits, 0, 10_000)] * len(ts))
    return quality.gpt2_ending([n for n, _ in sizes], ts, qs, ctx, hidden), ts, qs


def by_torch(ctx, steps, x, k, T, W):
    """The mean divergence in 64 bits for the weights W (one per step, on the CPU)."""
    def run(ws, bs):
        h = [x.cpu().double()]
        for s, w, b in zip(steps, ws, bs):
            w = w.view(s.layer.n_in, s.layer.n_out) if s.layer.in_out else w.view(s.layer.n_out, s.layer.n_in).t()
            y = A.act(h[-1] @ w + (0 if b is None else b), s.layer.activation)
            h.append(y if s.residual is None else y + h[s.residual])
        return h[-1]

    f = lambda t: None if t is None else t.cpu().double()  # noqa: E731
    teacher = run([f(s.weight) for s in steps], [f(s.bias) for s in steps])
    student = run(W, [f(s.layer.bias) for s in steps])
    t, i = teacher.topk(k, 1)
    rest = torch.logsumexp(teacher.scatter(1, i, float("-inf")) / T, 1, keepdim=True)
    p = torch.log_softmax(torch.cat([t / T, rest], 1), 1)
    q = torch.log_softmax(student / T, 1)
    q = torch.cat([q.gather(1, i), torch.logsumexp(q.scatter(1, i, float("-inf")), 1, keepdim=True)], 1)
    return (p.exp() * (p - q)).sum(1).mean(), (teacher.argmax(1) == student.argmax(1)).double().mean()


def test_degradation_and_gradients(ctx):
    rng = np.random.default_rng(1)
    x = torch.from_numpy(rng.standard_normal((37, 48)).astype(np.float32)).to(DEV)
    for bits in (2, 4, 8):
        steps, ts, _ = chain(ctx, rng, bits)
        assert len(steps) == 3 and steps[0].weight.data_ptr() == ts[5].data_ptr()  # the last block, by number
        W = [w.cpu().double().requires_grad_(True) for w in ctx.dequantize([s.layer.q for s in steps])]
        want, top1 = by_torch(ctx, steps, x, 20, 2.0, W)
        want.backward()
        got = quality.degradation(ctx, steps, x, 20, 2.0)
        # fp32 chains of three products (a few hundred roundings of 2^-24) on either side, in a loss that is a square of
        # their differences: 1e-4 of it and 1e-9 are a hundred times that
        assert abs(got["loss"] - float(want.detach())) <= 1e-4 * float(want.detach()) + 1e-9
        assert round(got["top1"] * 37) == round(float(top1) * 37)  # (a share of 37 rows in fp32)
        for g, w in zip(quality.weight_gradients(ctx, steps, x, 20, 2.0), W):
            assert g.shape == w.shape
            assert float((g.cpu().double() - w.grad).abs().max()) <= 1e-4 * float(w.grad.abs().max()) + 1e-9


def test_gradients_go_to_the_partition_by_sensitivity(ctx):
    rng = np.random.default_rng(2)
    x = torch.from_numpy(rng.standard_normal((20, 48)).astype(np.float32)).to(DEV)
    steps, _, _ = chain(ctx, rng, 4)
    grads = quality.weight_gradients(ctx, steps, x)
    weights = [s.weight for s in steps]
    qs, info = ctx.quantize_sens(weights, grads, [(4, 100_000, 5_000)] * 3, [True] * 3)
    for q, w, g, (tau, _, _) in zip(qs, weights, grads, info):
        n = w.numel()
        assert tau == float((w * g).abs().sort().values[n - 1 - n * 5_000 // 1_000_000])
        assert q.n_outlier >= n * 5_000 // 1_000_000


def test_bf16_states(ctx):
    rng = np.random.default_rng(3)
    x = torch.from_numpy(rng.standard_normal((64, 48)).astype(np.float32)).to(DEV)
    steps, _, _ = chain(ctx, rng, 3)
    full, half = (quality.degradation(ctx, steps, y, 20) for y in (x, x.bfloat16()))
    # bf16 states are off by 2^-9, the 3-bit weights by a tenth: the loss, a square, moves by a few hundredths at most
    assert half["loss"] > 0 and abs(half["loss"] - full["loss"]) <= 0.1 * full["loss"]


def test_report(monkeypatch, capsys):
    monkeypatch.setattr("sys.argv", ["ratio_report", "--scale", "0.01", "--steps", "2", "--threads", "4", "--quality", "16"])
    ratio_report.main()
    lines = [json.loads(line) for line in capsys.readouterr().out.splitlines() if line.startswith("{")]
    for line in lines[:2]:
        assert line["quality_loss"] >= 0 and 0 <= line["quality_top1"] <= 1
    monkeypatch.setattr("sys.argv", ["ratio_report", "--scale", "0.01", "--steps", "2", "--threads", "4"])
    ratio_report.main()
    plain = [json.loads(line) for line in capsys.readouterr().out.splitlines() if line.startswith("{")]
    drop = ("quality_loss", "quality_top1", "host_encode_s")
    assert [{k: v for k, v in a.items() if k not in drop} for a in lines] == [{k: v for k, v in a.items() if k not in drop} for a in plain]
