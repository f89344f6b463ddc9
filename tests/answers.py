"""Plain forms of the operators on compressed layers and on a teacher's logits, in 64 bits on the CPU, and how far a
result may be from them.

A result in type t is rounded once: off by at most HALF[t] of its magnitude.  Before that, with S the sum of the
magnitudes of the products of one result:
  - its factors are fp16 numbers scaled by powers of two; what that leaves out of a product is PRODUCT[t] of it, or
    2^-40 of (largest of the row) * (largest of the weight) where that is more (it is less for every input used here
    but those made for it, and is allowed for in full)
  - K products are added in fp32 in some order: K * 2^-24 * S
  - bias, scales, activation and residual are a few fp32 operations: 2^-20 of what they work on (the library functions
    are good to a few units of 2^-24)
"""
import math

import numpy as np
import torch

HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
# bf16: a factor of 11 bits on the weight's side (2^-11), and on the other one where it is no bf16 number (the gradient
# below an activation); fp16: 22 bits on either side; fp32: 22 bits on either side and the product of the low parts
PRODUCT = {torch.float32: 4 * 2.0 ** -22, torch.bfloat16: 2.5 * 2.0 ** -11, torch.float16: 3 * 2.0 ** -22}
TINY = {torch.float32: 2.0 ** -126, torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -24}


def width(bins):
    return (bins + 1).bit_length()


def pack(sym, w):
    """u64 words of the little-endian bit stream."""
    bits = ((sym[:, None].astype(np.uint32) >> np.arange(w, dtype=np.uint32)) & 1).astype(np.uint8).reshape(-1)
    bits = np.concatenate([bits, np.zeros(-len(bits) % 64, np.uint8)])
    return np.packbits(bits, bitorder="little").view(np.int64)


class Codes:
    """A weight of n values in compressed form: symbols, centres, protected list; `values` are what it decodes to."""

    def __init__(self, rng, n, bins, protected=0, bf16=False, scale=0.05, pruned=0.1):
        self.n, self.bins, self.bf16 = n, bins, bf16
        self.sym = rng.integers(2, bins + 2, n).astype(np.uint16)
        self.sym[rng.random(n) < pruned] = 0
        self.index = np.sort(rng.choice(n, min(protected, n), replace=False)).astype(np.uint32)
        self.sym[self.index] = 1
        self.centres = np.sort(rng.normal(0, scale, bins)).astype(np.float32)
        v = (rng.choice([-1.0, 1.0], self.index.size) * scale * rng.uniform(3, 6, self.index.size)).astype(np.float32)
        self.protected = torch.from_numpy(v).to(torch.bfloat16 if bf16 else torch.float32)
        self.decode()

    def decode(self):
        table = np.concatenate([[0.0, 0.0], self.centres.astype(np.float64)])
        self.values = table[self.sym]
        self.values[self.index] = self.protected.double().numpy()

    def quantized(self, api, device):
        t = lambda a, d=None: torch.from_numpy(a).to(device)  # noqa: E731
        room = torch.zeros(1, dtype=torch.int32, device=device)
        centres = np.zeros(256, np.float32)
        centres[:self.bins] = self.centres
        q = api.Quantized(self.n, 0, (t(pack(self.sym, width(self.bins))), t(centres), t(centres),
                                      t(self.index.view(np.int32)) if self.index.size else room,
                                      self.protected.to(device) if self.index.size else room.float()), bins=self.bins)
        q.n_outlier, q.bf16 = self.index.size, self.bf16
        return q


def act(a, kind):
    if kind == "relu":
        return a.clamp_min(0)
    if kind == "gelu":
        return a * 0.5 * torch.erfc(-a * math.sqrt(0.5))
    if kind == "gelu_tanh":
        return 0.5 * a * (1 + torch.tanh(math.sqrt(2 / math.pi) * (a + 0.044715 * a ** 3)))
    if kind == "silu":
        return a * torch.sigmoid(a)
    return a


def slope(a, kind):
    """act'(a), by torch's differentiation of act in 64 bits."""
    a = a.clone().requires_grad_(True)
    act(a, kind).sum().backward()
    return a.grad


def linear(x, W, b, r, kind):
    """(y, pre, S) of x [rows][n_in], W [n_out][n_in] in 64 bits; S: sums of the magnitudes behind pre."""
    a = x @ W.t()
    S = x.abs() @ W.abs().t()
    if b is not None:
        a, S = a + b, S + b.abs()
    y = act(a, kind)
    return (y if r is None else y + r), a, S


def tol_sum(S, K, dtype, top):
    """Of a sum before it is rounded to its type; top: largest of the row times largest of the weight."""
    return S * (PRODUCT[dtype] + (K + 8) * 2.0 ** -24) + K * 2.0 ** -39 * top


def tol_linear(y, r, S, K, dtype, top):
    t = 1.13 * tol_sum(S, K, dtype, top) + 2.0 ** -20 * S  # (no activation is steeper than 1.13)
    t = t + (0 if r is None else 2.0 ** -23 * (y.abs() + r.abs()))
    return t * (1 + HALF[dtype]) + HALF[dtype] * y.abs() + TINY[dtype]
