"""GPU: gradients of the quality from hidden states of 16 bits."""
import numpy as np
import pytest
import torch

from paper_2306_11800_amd import api, quality
from tests import answers as A
from tests.test_gpu_logits import plain_distill
from tests.test_gpu_quality import chain

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def ctx():
    c = api.Context(torch.device(DEV))
    yield c
    c.close()


def test_gradients_from_fp16_states(ctx):
    """Entries of a gradient of a mean over many rows lie below the smallest fp16 number; none is lost for it.  Against
    the backward pass in 64 bits from the same states."""
    rng = np.random.default_rng(1)
    rows, k, T = 2000, 20, 2.0
    steps, _, _ = chain(ctx, rng, 4, vocab=1200)
    x = torch.from_numpy(rng.standard_normal((rows, 48)).astype(np.float32)).to(DEV).half()
    got = quality.weight_gradients(ctx, steps, x, k, T)
    top = ctx.top_logits(quality.teacher_logits(steps, x), k, T)
    h, pre = (
        [None if t is None else t.cpu().double() for t in s] for s in quality.student_states(ctx, steps, x, for_gradients=True))
    d = plain_distill(h[-1], top.index.cpu(), top.value.cpu().double(), top.tail.cpu().double(), T,
                      torch.full((rows,), 1.0 / rows, dtype=torch.float64))[1]
    assert float((d.abs() < 2.0 ** -25).double().mean()) > 0.5  # (what fp16 rounds to nothing)
    into = [None] * len(h)
    into[-1] = d
    for i in range(len(steps) - 1, -1, -1):
        s = steps[i]
        W = ctx.dequantize([s.layer.q])[0].cpu().double()
        W = W.view(s.layer.n_in, s.layer.n_out).t() if s.layer.in_out else W.view(s.layer.n_out, s.layer.n_in)
        below = into[i + 1] if pre[i] is None else into[i + 1] * A.slope(pre[i], s.layer.activation)
        dw = below.t() @ h[i]
        dw = (dw.t() if s.layer.in_out else dw).reshape(-1)
        # (fp32 steps of a few hundred terms: a hundred times their roundings)
        assert float((got[i].cpu().double() - dw).abs().max()) <= 1e-4 * float(dw.abs().max())
        for j, g in ((i, below @ W), (s.residual, into[i + 1])):
            if j is not None:
                into[j] = g if into[j] is None else into[j] + g


def test_no_rows(ctx):
    rng = np.random.default_rng(2)
    steps, _, _ = chain(ctx, rng, 4)
    for g, s in zip(quality.weight_gradients(ctx, steps, torch.empty((0, 48), device=DEV)), steps):
        assert g.numel() == s.layer.n_in * s.layer.n_out and not bool(g.any())
