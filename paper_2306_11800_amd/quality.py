"""How much of a model's answers a compressed checkpoint keeps, on the layers it ends with (Sec. 5: a configuration is judged
by the quality of the quantized model), and the gradients of that quality, which quantize_sens takes as sensitivities.

The teacher is the original checkpoint: its layers run from their full-precision weights by the library's products.  The
student's layers run from the compressed form (Context.linear).  Compared are the student's logits with the teacher's k
largest and the mass of the others (Context.top_logits, Context.distill)."""
from __future__ import annotations

from dataclasses import dataclass
from typing import List, Optional, Sequence

import torch

from . import api


@dataclass
class Step:
    """One layer of a chain: hidden state i + 1 = layer(hidden state i), plus hidden state `residual` where given.
    weight (float32, the tensor that was quantized) and bias are the teacher's."""
    layer: api.QuantizedLayer
    weight: torch.Tensor
    bias: Optional[torch.Tensor] = None
    residual: Optional[int] = None


_TORCH = {"none": lambda a: a, "relu": torch.relu, "gelu": torch.nn.functional.gelu, "silu": torch.nn.functional.silu,
          "gelu_tanh": lambda a: torch.nn.functional.gelu(a, approximate="tanh")}


def teacher_logits(steps: Sequence[Step], x: torch.Tensor) -> torch.Tensor:
    """The last hidden state of the original layers, float32."""
    h = [x.float()]
    for s in steps:
        w = s.weight.view(s.layer.n_in, s.layer.n_out) if s.layer.in_out else s.weight.view(s.layer.n_out, s.layer.n_in).t()
        a = h[-1] @ w
        y = _TORCH[s.layer.activation](a if s.bias is None else a + s.bias)
        h.append(y if s.residual is None else y + h[s.residual])
    return h[-1]


def student_states(ctx: api.Context, steps: Sequence[Step], x: torch.Tensor, for_gradients: bool = False):
    """(hidden states, values below the activations) of the compressed layers; x in any type of linear."""
    h, pre = [x], []
    for s in steps:
        r = None if s.residual is None else h[s.residual]
        if for_gradients and s.layer.activation != "none":
            y, a = ctx.linear(s.layer, h[-1], r, want_pre=True)
        else:
            y, a = ctx.linear(s.layer, h[-1], r), None
        h.append(y)
        pre.append(a)
    return h, pre


def degradation(ctx: api.Context, steps: Sequence[Step], x: torch.Tensor, k: int = 64, temperature: float = 1.0):
    """dict(loss = mean divergence of the student's answers from the teacher's, top1 = share of rows whose largest logit is
    the teacher's)."""
    top = ctx.top_logits(teacher_logits(steps, x), k, temperature)
    logits = student_states(ctx, steps, x)[0][-1]
    loss, _ = ctx.distill(logits, top, want_saved=False)
    same = ctx.top_logits(logits, 1, want_tail=False).index[:, 0] == top.index[:, 0]
    return dict(loss=float(loss.mean()), top1=float(same.float().mean()))


def weight_gradients(ctx: api.Context, steps: Sequence[Step], x: torch.Tensor, k: int = 64, temperature: float = 1.0
                     ) -> List[torch.Tensor]:
    """The gradient of the mean divergence for each layer's weight: float32, in the layout and of the size of the tensor
    that was quantized."""
    top = ctx.top_logits(teacher_logits(steps, x), k, temperature)
    h, pre = student_states(ctx, steps, x, for_gradients=True)
    if x.dtype == torch.float16:  # (a share of the mean over many rows is less than the smallest number of this type, 6e-8)
        h, pre = [t.float() for t in h], [t if t is None else t.float() for t in pre]
    _, saved = ctx.distill(h[-1], top)
    each = torch.full((x.shape[0],), 1.0 / max(1, x.shape[0]), dtype=torch.float32, device=x.device)
    d: List[Optional[torch.Tensor]] = [None] * len(h)
    d[-1] = ctx.distill_grad(h[-1], top, saved, each)
    out: List[torch.Tensor] = [None] * len(steps)  # type: ignore[list-item]
    for i in range(len(steps) - 1, -1, -1):
        s = steps[i]
        dx, dw, _ = ctx.linear_grad(s.layer, h[i], d[i + 1], pre[i], want_dx=i > 0, want_dbias=False)
        out[i] = dw.view(-1)
        for j, g in ((i, dx), (s.residual, d[i + 1])):
            if j:  # (nobody asks for the gradient of x)
                d[j] = g if d[j] is None else d[j] + g
    return out


def gpt2_ending(names: Sequence[str], weights: Sequence[torch.Tensor], quantized: Sequence[api.Quantized],
                ctx: api.Context, hidden: int) -> List[Step]:
    """The chain a GPT-2 checkpoint ends with: the last block's feed-forward layers, where they fit together (a scaled-down
    report cuts them), and the head, which is the embedding."""
    at = {n: i for i, n in enumerate(names)}
    fc = max((n for n in names if n.endswith("mlp.c_fc.weight")), key=lambda n: int(n.split(".")[0][1:]), default=None)
    steps: List[Step] = []
    if fc is not None:
        pj = fc.replace("c_fc", "c_proj")
        f, p, fb, pb = (at[n] for n in (fc, pj, fc.replace("weight", "bias"), pj.replace("weight", "bias")))
        ff = weights[fb].numel()
        if weights[f].numel() == hidden * ff and weights[p].numel() == ff * hidden and weights[pb].numel() == hidden:
            b = ctx.dequantize([quantized[fb], quantized[pb]])
            steps += [Step(api.QuantizedLayer(quantized[f], ff, hidden, True, b[0], "gelu_tanh"), weights[f], weights[fb]),
                      Step(api.QuantizedLayer(quantized[p], hidden, ff, True, b[1]), weights[p], weights[pb], residual=0)]
    e = at["wte"]
    steps.append(Step(api.QuantizedLayer(quantized[e], weights[e].numel() // hidden, hidden), weights[e]))
    return steps
