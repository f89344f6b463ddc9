"""CPU: what the operators on compressed layers and on logits refuse before anything reaches a device."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2306_11800_amd import api
from tests import answers as A


@pytest.fixture()
def ctx():
    """A context without a device: the library answers its calls with INSHR_E_ARG."""
    c = api.Context.__new__(api.Context)
    c.lib, c._device, c.h = api.load_library(), torch.device("cpu"), None
    return c


def layer(n_out=8, n_in=16, bins=12, **kw):
    codes = A.Codes(np.random.default_rng(0), n_out * n_in, bins, 5)
    return api.QuantizedLayer(codes.quantized(api, "cpu"), n_out, n_in, **kw)


def test_layers():
    q = layer().q
    for args, kw in (((8, 15), {}), ((0, 16), {}), ((8, 16), dict(activation="tanh")),
                     ((8, 16), dict(bias=torch.zeros(7))), ((8, 16), dict(bias=torch.zeros(8, dtype=torch.float64))),
                     ((8, 16), dict(bias=torch.zeros(16)[::2]))):
        with pytest.raises(ValueError):
            api.QuantizedLayer(q, *args, **kw)
    assert api.QuantizedLayer(q, 16, 8, in_out=True, bias=torch.zeros(16), activation="silu").n_in == 8


def test_bounds():
    lib, need = api.load_library(), C.c_uint64()
    bound = lambda c, rows=100: lib.inshr_linear_bound(C.byref(c), rows, C.byref(need))  # noqa: E731
    c = layer()._c[0]
    assert bound(c) == 0 and bound(c, 0) == 0 and need.value == 0
    assert bound(c, (1 << 22) + 1) == -1
    assert lib.inshr_linear_bound(C.byref(c), 4, None) == -1 and lib.inshr_linear_bound(None, 4, C.byref(need)) == -1
    assert lib.inshr_linear_grad_bound(C.byref(c), 4, 1, 1, C.byref(need)) == 0

    def changed(**kw):
        d = layer()._c[0]
        for k, v in kw.items():
            setattr(d if hasattr(d, k) else d.weight, k, v)
        return d

    for kw, rc in ((dict(type=3), -1), (dict(activation=5), -1), (dict(reserved=1), -1), (dict(n_out=0), -1),
                   (dict(n_in=17), -1), (dict(n_out=(1 << 30) + 1), -1), (dict(packed=None), -1), (dict(codebook=None), -1),
                   (dict(outlier_idx=None), -1), (dict(outlier_val=2), -1), (dict(bias=2), -1), (dict(bins=257), -2),
                   (dict(bins=0, bits=9), -2), (dict(n_outlier=8 * 16 + 1), -5)):
        assert bound(changed(**kw)) == rc, kw
        assert lib.inshr_linear_grad_bound(C.byref(changed(**kw)), 4, 1, 1, C.byref(need)) == rc, kw
    big = changed(n_out=1 << 20, n_in=1 << 12)  # 2^32 values: more than a tensor has
    big.weight.n = 1 << 32
    assert bound(big) == -1


def test_no_context():
    lib, none = api.load_library(), api.CMatrix(None, 0)
    c, d = layer()._c[0], api.CDistillIn()
    assert lib.inshr_linear(None, C.byref(c), none, none, none, none, 1, None, 0) == -1
    assert lib.inshr_linear_grad(None, C.byref(c), none, none, none, none, None, None, 1, None, 0) == -1
    assert lib.inshr_top_logits(None, none, 0, 1, 10, 1, 1.0, None, None, None) == -1
    assert lib.inshr_distill(None, C.byref(d), None, None) == -1
    assert lib.inshr_distill_grad(None, C.byref(d), None, None, none) == -1


def test_tensors(ctx):
    l, x = layer(), torch.zeros((3, 16))
    for bad in (x[:, :8], x[0], x.double(), torch.zeros((3, 32))[:, ::2], torch.zeros((16, 3)).t()):
        with pytest.raises(ValueError, match="x must"):
            ctx.linear(l, bad)
    for kw in (dict(residual=torch.zeros((3, 7))), dict(residual=torch.zeros((3, 8), dtype=torch.bfloat16)),
               dict(out=torch.zeros((2, 8)))):
        with pytest.raises(ValueError, match="(residual|out) must"):
            ctx.linear(l, x, **kw)
    far = layer()
    far.device = torch.device("meta")
    with pytest.raises(ValueError, match="the layer is on meta"):
        ctx.linear(far, x)
    with pytest.raises(ValueError, match="the layer is on meta"):
        ctx.linear_grad(far, x, torch.zeros((3, 8)))
    dy = torch.zeros((3, 8))
    with pytest.raises(ValueError, match="dw needs x"):
        ctx.linear_grad(l, None, dy)
    with pytest.raises(ValueError, match="needs pre"):
        ctx.linear_grad(layer(activation="gelu"), x, dy)
    with pytest.raises(ValueError, match="x must"):
        ctx.linear_grad(l, x.bfloat16(), dy)
    with pytest.raises(ValueError, match="pre must"):
        ctx.linear_grad(layer(activation="gelu"), x, dy, x)
    z = torch.zeros((3, 50))
    for k in (0, 51):
        with pytest.raises(ValueError, match="k must"):
            ctx.top_logits(z, k)
    with pytest.raises(ValueError, match="logits must"):
        ctx.top_logits(z[0], 3)
    i, v = torch.zeros((3, 4), dtype=torch.int32), torch.zeros((3, 4))
    for top in (api.TopLogits(i.long(), v, None), api.TopLogits(i, v[:, :3], None), api.TopLogits(i[:2], v[:2], None),
                api.TopLogits(i, v, torch.zeros(4)), api.TopLogits(i, v.half(), None)):
        with pytest.raises(ValueError, match="(index|value|tail) must"):
            ctx.distill(z, top)
    top = api.TopLogits(i, v, None)
    with pytest.raises(ValueError, match="saved must"):
        ctx.distill_grad(z, top, torch.zeros((3, 2), dtype=torch.float64))
    with pytest.raises(ValueError, match="grad_loss must"):
        ctx.distill_grad(z, top, torch.zeros((3, 4), dtype=torch.float64), torch.zeros(4))
