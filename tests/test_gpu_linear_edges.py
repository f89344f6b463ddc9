"""GPU: layers at the ends of what the header allows, against plain forms in 64 bits."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2306_11800_amd import api
from tests import answers as A
from tests.test_gpu_linear import case, check_grad, check_linear, f64, near, rows_of

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def ctx():
    c = api.Context(torch.device(DEV))
    yield c
    c.close()


def test_bits_of_a_product(ctx):
    """Of one product a result, what the header says: 2^-21 of it for fp32 (and the rounding of the result), with few and
    with many rows and in the gradients; dw of exact factors is rounded once."""
    rng = np.random.default_rng(9)
    for rows in (3, 40, 300):
        for in_out in (False, True):
            layer, W, x, _ = case(rng, rows, 1, 500, 256, F32, in_out=in_out, bias=False)
            y = f64(ctx.linear(layer, x))
            want = f64(x) @ W.t()
            near(y, want, (2.0 ** -21 + 2.0 ** -24) * want.abs() + 2.0 ** -38 * f64(x).abs() * W.abs().max() + A.TINY[F32])
    for dtype, bits in ((F32, 2.0 ** -21 + 2.0 ** -24), (BF16, 2.0 ** -24), (F16, 2.0 ** -24)):
        layer, W, x, _ = case(rng, 1, 300, 200, 16, dtype, bias=False)
        dy = rows_of(rng, 1, 200, dtype)
        want = f64(dy).t() @ f64(x)
        near(ctx.linear_grad(layer, x, dy)[1], want, bits * want.abs() + A.TINY[F32])


def test_centres_at_the_end_of_the_range(ctx):
    """Centres above the largest bfloat16 number, times rows that bring the products back."""
    rng = np.random.default_rng(6)
    for in_out in (False, True):
        codes = A.Codes(rng, 96 * 40, 4, 0)
        codes.centres = np.array([-3.4e38, -1.0, 3.39e38, 3.4028234e38], np.float32)
        codes.decode()
        layer = api.QuantizedLayer(codes.quantized(api, DEV), 40, 96, in_out)
        W = torch.from_numpy(codes.values)
        W = W.view(96, 40).t() if in_out else W.view(40, 96)
        for rows in (2, 20, 120):
            for dtype in (F32, BF16):
                check_linear(ctx, layer, W, rows_of(rng, rows, 96, dtype) * 2.0 ** -100, None)


@pytest.mark.parametrize("in_out", [False, True], ids=["oi", "io"])
def test_a_protected_symbol_without_a_list_counts_as_zero(ctx, in_out):
    """... in few rows, many rows and the gradients alike."""
    rng = np.random.default_rng(7)
    codes = A.Codes(rng, 130 * 70, 12, 900)
    codes.protected = codes.protected * 0.0
    codes.decode()
    q = codes.quantized(api, DEV)
    q.n_outlier = 0
    layer = api.QuantizedLayer(q, 70, 130, in_out)
    W = torch.from_numpy(codes.values)
    W = W.view(130, 70).t() if in_out else W.view(70, 130)
    for dtype in (F32, BF16, F16):
        for rows in (1, 3, 30, 200):
            stale = torch.full((1 << 22,), float("nan"), device=DEV)  # what a workspace may hold
            torch.cuda.synchronize()
            del stale
            x = rows_of(rng, rows, 130, dtype)
            check_linear(ctx, layer, W, x, None)
            check_grad(ctx, layer, W, x, rows_of(rng, rows, 70, dtype), None)


def test_results_in_one_place_are_refused(ctx):
    rng = np.random.default_rng(8)
    layer, _, x, _ = case(rng, 4, 64, 64, 16, F32)
    dy, room = rows_of(rng, 4, 64, F32), torch.empty((64, 64), device=DEV)
    c, need = layer._c[0], C.c_uint64()
    assert ctx.lib.inshr_linear_grad_bound(C.byref(c), 4, 1, 1, C.byref(need)) == 0
    ws = torch.empty(need.value, dtype=torch.uint8, device=DEV)
    m = lambda t: api.CMatrix(t.data_ptr(), 64)  # noqa: E731
    grad = lambda dx, dw, db: ctx.lib.inshr_linear_grad(  # noqa: E731
        ctx.h, C.byref(c), m(x), m(dy), api.CMatrix(None, 0), dx, dw, db, 4, ws.data_ptr(), need.value)
    p, none = room.data_ptr(), api.CMatrix(None, 0)
    assert grad(m(room), p, None) == -1 and grad(m(room), None, p) == -1 and grad(none, p, p) == -1
    assert grad(m(room), torch.empty(64 * 64, device=DEV).data_ptr(), None) == 0
    ctx.sync()


def test_a_context_of_the_default_stream_is_not_captured(ctx):
    """... but refuses, and leaves the capture as it was."""
    rng = np.random.default_rng(10)
    layer, _, x, _ = case(rng, 20, 64, 40, 16, F32)
    dy = rows_of(rng, 20, 40, F32)
    assert ctx.stream.cuda_stream == 0
    want, top = ctx.linear(layer, x), ctx.top_logits(x, 4)
    _, saved = ctx.distill(x, top)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        twice = x * 2.0
        for call in (lambda: ctx.linear(layer, x), lambda: ctx.linear_grad(layer, x, dy), lambda: ctx.top_logits(x, 4),
                     lambda: ctx.distill(x, top), lambda: ctx.distill_grad(x, top, saved)):
            with pytest.raises(RuntimeError, match="default stream"):
                call()
        again = twice + x
    for _ in range(3):
        x.copy_(torch.randn_like(x))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(twice, x * 2.0) and torch.equal(again, x * 2.0 + x)
    assert ctx.linear(layer, x).shape == want.shape


def test_captured_while_profiled(ctx):
    """A launch that is captured is not timed, and the calls after it go on."""
    rng = np.random.default_rng(11)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        c2 = api.Context(torch.device(DEV))
    layer, _, x, _ = case(rng, 120, 64, 40, 16, F32)
    want = ctx.linear(layer, x)
    torch.cuda.synchronize()
    c2.profile(True)
    try:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            y = c2.linear(layer, x)
        assert c2.profile_read() == {}
        for _ in range(3):
            y.zero_()
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(y, want) and torch.equal(c2.linear(layer, x), want)
        times = c2.profile_read()
        assert times["k_product"][1] == 3 and all(n == 3 and ms > 0 for ms, n in times.values())
    finally:
        c2.profile(False)
    c2.close()


class Bytes:
    """A weight of n values made on the device: 128 centres, so that a symbol is a byte."""

    def __init__(self, n, protected, seed):
        gen = torch.Generator(device=DEV).manual_seed(seed)
        self.sym = torch.randint(0, 129, (-(-n // 8) * 8,), generator=gen, device=DEV, dtype=torch.uint8)
        self.sym += self.sym >= 1
        self.sym[n:] = 0
        index = torch.cat([torch.randint(0, n, (protected,), generator=gen, device=DEV), torch.tensor([0, n - 1], device=DEV)]).unique()
        self.sym[index] = 1
        centres = torch.zeros(256, device=DEV)
        centres[:128] = torch.randn(128, generator=gen, device=DEV).mul_(0.05).sort().values
        value = torch.randn(index.numel(), generator=gen, device=DEV).sign() * 0.2
        self.n, self.index, self.value = n, index, value.double()
        self.table = torch.cat([torch.zeros(2, device=DEV), centres[:128]]).double()
        self.q = api.Quantized(n, 0, (self.sym.view(torch.int64), centres, centres, index.to(torch.int32), value), bins=128)
        self.q.n_outlier = index.numel()

    def at(self, places):
        """The values of these places (a tensor of any shape), in 64 bits."""
        v = self.table[self.sym[places].long()]
        j = torch.searchsorted(self.index, places).clamp_max(self.index.numel() - 1)
        return torch.where(self.index[j] == places, self.value[j], v)


def check_columns(ctx, w, layer, x, cols, dy=None):
    """The outputs `cols` of linear, and (for dy) the inputs `cols` of its gradient."""
    n_in, n_out = layer.n_in, layer.n_out
    if dy is None:
        got, rows_, K = ctx.linear(layer, x)[:, cols], x.double(), n_in
        r, c = cols[:, None], torch.arange(n_in, device=DEV)[None, :]
    else:
        got, rows_, K = ctx.linear_grad(layer, x, dy, want_dw=False, want_dbias=False)[0][:, cols], dy.double(), n_out
        r, c = torch.arange(n_out, device=DEV)[None, :], cols[:, None]
    W = w.at(c * n_out + r if layer.in_out else r * n_in + c)
    want, S = (rows_ @ W.t()).cpu(), (rows_.abs() @ W.abs().t()).cpu()
    top = rows_.abs().amax(1, keepdim=True).cpu() * 0.25
    near(got, want, A.tol_sum(S, K, x.dtype, top) * (1 + A.HALF[x.dtype]) + A.HALF[x.dtype] * want.abs() + A.TINY[x.dtype])


@pytest.mark.parametrize("in_out", [False, True], ids=["oi", "io"])
def test_streams_of_more_than_2_32_bits(ctx, in_out):
    n_out, n_in = (8200, 65539) if in_out else (65539, 8200)
    w = Bytes(n_in * n_out, 4000, 3)
    assert w.n * 8 > 1 << 32
    layer = api.QuantizedLayer(w.q, n_out, n_in, in_out)
    rng = np.random.default_rng(1)
    cols = lambda n: torch.cat([torch.arange(40), torch.from_numpy(rng.integers(0, n, 40)), torch.arange(n - 40, n)]).to(DEV)  # noqa: E731
    for rows, dtype in ((1, BF16), (3, F32), (30, F16), (130, BF16)):
        check_columns(ctx, w, layer, rows_of(rng, rows, n_in, dtype), cols(n_out))
    check_columns(ctx, w, layer, rows_of(rng, 70, n_in, BF16), cols(n_in), rows_of(rng, 70, n_out, BF16))


@pytest.mark.parametrize("rows", [1, 24, 256])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_head_over_a_vocabulary(ctx, rows, dtype):
    n_in, n_out = 1024, 50257
    w = Bytes(n_in * n_out, 50_000, 5)
    layer = api.QuantizedLayer(w.q, n_out, n_in)
    rng = np.random.default_rng(rows)
    x = rows_of(rng, rows, n_in, dtype)
    check_columns(ctx, w, layer, x, torch.arange(n_out, device=DEV))
    dy = rows_of(rng, rows, n_out, dtype, scale=0.01)
    check_columns(ctx, w, layer, x, torch.arange(n_in, device=DEV), dy)
    _, dw, db = ctx.linear_grad(layer, x, dy, want_dx=False)
    d = dy.double()
    want, S = (d.t() @ x.double()).cpu(), (d.abs().t() @ x.double().abs()).cpu()
    top = (d.abs().amax(0)[:, None] * x.double().abs().amax(0)[None, :]).cpu()
    near(dw, want, A.tol_sum(S, rows, F32, top) + 2.0 ** -24 * want.abs() + A.TINY[F32])
    near(db, d.sum(0).cpu(), d.abs().sum(0).cpu() * rows * 2.0 ** -24 + A.TINY[F32])


@pytest.mark.parametrize("n_out", [2048, 2049, 4096, 4097, 8192, 8193, 16384, 16385])
@pytest.mark.parametrize("dtype,bins", [(F32, 16), (BF16, 64), (BF16, 128), (F16, 16)], ids=["f32", "bf16-7", "bf16-8", "f16"])
def test_numbers_of_rows_and_outputs(ctx, n_out, dtype, bins):
    """Either side of the numbers at which rows go straight from the stream or by planes."""
    rng = np.random.default_rng(n_out)
    n_in = 70
    codes = A.Codes(rng, n_in * n_out, bins, n_out // 4)
    layer = api.QuantizedLayer(codes.quantized(api, DEV), n_out, n_in, activation="relu")
    W = torch.from_numpy(codes.values).view(n_out, n_in)
    for rows in (32, 33, 64, 65, 96, 97):
        check_linear(ctx, layer, W, rows_of(rng, rows, n_in, dtype), rows_of(rng, rows, n_out, dtype))


@pytest.mark.parametrize("n_in,n_out", [(640, 65536), (640, 65544), (768, 65536), (768, 65400), (4001, 12001)])
def test_runs_of_a_token(ctx, n_in, n_out):
    """Weights stored [in][out] either side of the sizes at which a thread takes longer runs."""
    w = Bytes(n_in * n_out, 20_000, n_in)
    layer = api.QuantizedLayer(w.q, n_out, n_in, in_out=True)
    rng = np.random.default_rng(n_out)
    for rows, dtype in ((1, BF16), (1, F32), (2, F32)):
        check_columns(ctx, w, layer, rows_of(rng, rows, n_in, dtype), torch.arange(n_out, device=DEV))


@pytest.mark.parametrize("in_out", [False, True], ids=["oi", "io"])
@pytest.mark.parametrize("rows,n_in,n_out", [(130, 1, 1), (130, 300, 1), (97, 1, 300), (5, 1, 40), (3, 500, 1), (40, 2, 1),
                                             (2, 300_007, 17), (100, 17, 100_003), (70, 100_003, 9)])
def test_thin_layers(ctx, rows, n_in, n_out, in_out):
    rng = np.random.default_rng(n_in + n_out)
    for dtype in (F32, BF16):
        layer, W, x, r = case(rng, rows, n_in, n_out, 16, dtype, "silu", in_out, residual=True)
        check_linear(ctx, layer, W, x, r)
        check_grad(ctx, layer, W, x, rows_of(rng, rows, n_out, dtype), rows_of(rng, rows, n_out, dtype))


def test_rows_far_apart(ctx):
    """Rows 2^31 elements apart, of inputs and of results: offsets of more than 32 bits."""
    rng = np.random.default_rng(12)
    far, rows = 1 << 31, 4
    room = torch.empty(far * (rows - 1) + 4096, dtype=BF16, device=DEV)
    at = lambda k, cols: room[k:].as_strided((rows, cols), (far, 1))  # noqa: E731
    for in_out in (False, True):
        layer, W, x, r = case(rng, rows, 200, 120, 16, BF16, "gelu", in_out, residual=True)
        dy, pre = rows_of(rng, rows, 120, BF16), rows_of(rng, rows, 120, BF16)
        places = [at(0, 200), at(256, 120), at(512, 120), at(768, 120)]
        for place, t in zip(places, (x, r, dy, pre)):
            place.copy_(t)
        out = at(1024, 120)
        assert torch.equal(ctx.linear(layer, places[0], places[1], out=out), ctx.linear(layer, x, r))
        for got, want in zip(ctx.linear_grad(layer, places[0], *places[2:]), ctx.linear_grad(layer, x, dy, pre)):
            assert torch.equal(got, want)
    wide = A.Codes(rng, 64 * 48, 16)
    layer = api.QuantizedLayer(wide.quantized(api, DEV), 48, 64)
    x = rows_of(rng, 130, 64, BF16)
    far = 1 << 25  # 130 rows by planes, the last of them past 2^32
    place = room[:far * 129 + 64].as_strided((130, 64), (far, 1))
    place.copy_(x)
    assert torch.equal(ctx.linear(layer, place), ctx.linear(layer, x))


def test_many_rows(ctx):
    """As many rows as a call takes, through a small layer, and one more."""
    rng = np.random.default_rng(13)
    rows = 1 << 22
    for dtype in (BF16, F32):
        codes = A.Codes(rng, 12 * 9, 8, 5)
        layer = api.QuantizedLayer(codes.quantized(api, DEV), 9, 12, activation="relu")
        W = torch.from_numpy(codes.values).view(9, 12).to(DEV)
        x = torch.randn((rows, 12), device=DEV).to(dtype)
        y, pre = ctx.linear(layer, x, want_pre=True)
        want, S = x.double() @ W.t(), x.double().abs() @ W.abs().t()
        tol = A.tol_sum(S, 12, dtype, x.double().abs().amax(1, keepdim=True) * W.abs().max())
        near(pre, want.cpu(), (tol * (1 + A.HALF[dtype]) + A.HALF[dtype] * want.abs() + A.TINY[dtype]).cpu())
        assert torch.equal(y, pre.clamp_min(0.0))
        dy = torch.randn((rows, 9), device=DEV).to(dtype)
        dx, dw, db = ctx.linear_grad(layer, x, dy, pre)
        d = dy.double() * (pre > 0)
        want, S = d @ W, d.abs() @ W.abs()
        tol = A.tol_sum(S, 9, dtype, d.abs().amax(1, keepdim=True) * W.abs().max())
        near(dx, want.cpu(), (tol * (1 + A.HALF[dtype]) + A.HALF[dtype] * want.abs() + A.TINY[dtype]).cpu())
        want, S = d.t() @ x.double(), d.abs().t() @ x.double().abs()
        near(dw, want.cpu(), A.tol_sum(S, rows, F32, d.abs().amax(0)[:, None] * x.double().abs().amax(0)[None]).cpu())
        near(db, d.sum(0).cpu(), (d.abs().sum(0) * rows * 2.0 ** -24).cpu())
        with pytest.raises(RuntimeError):
            ctx.linear(layer, x[:1].expand(rows + 1, 12))


def test_non_finite_gradients(ctx):
    """NaN and infinities in a row of dy, pre or x reach the results that they enter and no others."""
    rng = np.random.default_rng(14)
    for rows in (40, 200):
        for dtype in (F32, BF16, F16):
            for in_out in (False, True):
                layer, _, x, _ = case(rng, rows, 96, 70, 16, dtype, "silu", in_out)
                dy, pre = rows_of(rng, rows, 70, dtype), rows_of(rng, rows, 70, dtype)
                dx, dw, db = ctx.linear_grad(layer, x, dy, pre)
                dy[3, 5], pre[7, 9], x[11, 13] = float("inf"), float("nan"), float("-inf")
                dx2, dw2, db2 = ctx.linear_grad(layer, x, dy, pre)
                dw, dw2 = (t.t() if in_out else t for t in (dw, dw2))
                r = [i for i in range(rows) if i not in (3, 7)]
                o, i = [n for n in range(70) if n not in (5, 9)], [k for k in range(96) if k != 13]
                assert torch.equal(dx[r], dx2[r]) and not bool(torch.isfinite(dx2[[3, 7]]).any())
                assert torch.equal(db[o], db2[o]) and not bool(torch.isfinite(db2[[5, 9]]).any())
                assert torch.equal(dw[o][:, i], dw2[o][:, i])
                assert not bool(torch.isfinite(dw2[[5, 9]]).any()) and not bool(torch.isfinite(dw2[:, 13]).any())


@pytest.mark.parametrize("in_out", [False, True], ids=["oi", "io"])
def test_nothing_left(ctx, in_out):
    """A weight whose values are all pruned, centres of zero, rows of zeros: zeros come out, and the bias."""
    rng = np.random.default_rng(15)
    for kind in ("pruned", "centres", "rows"):
        codes = A.Codes(rng, 96 * 40, 8, 0, pruned=2.0 if kind == "pruned" else 0.1)
        if kind == "centres":
            codes.centres[:] = 0.0
            codes.decode()
        b = torch.randn(40, device=DEV)
        layer = api.QuantizedLayer(codes.quantized(api, DEV), 40, 96, in_out, b)
        for rows in (1, 3, 30, 120):
            for dtype in (F32, BF16, F16):
                x = rows_of(rng, rows, 96, dtype)
                x = x * 0.0 if kind == "rows" else x
                assert torch.equal(ctx.linear(layer, x), b.to(dtype).expand(rows, 40))
                dx, dw, _ = ctx.linear_grad(layer, x, rows_of(rng, rows, 40, dtype))
                assert kind == "rows" or not bool(dx.any())
                assert kind != "rows" or not bool(dw.any())
