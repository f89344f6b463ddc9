"""GPU: a teacher's largest logits, the distillation loss on them and its gradient, against plain forms in 64 bits."""
import numpy as np
import pytest
import torch

from paper_2306_11800_amd import api
from tests import answers as A

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
INF = float("inf")


@pytest.fixture(scope="module")
def ctx():
    c = api.Context(torch.device(DEV))
    yield c
    c.close()


def logits_of(rng, rows, vocab, dtype, gap=0, at=0, scale=3.0):
    room = torch.from_numpy((scale * rng.standard_normal(rows * (vocab + gap) + at)).astype(np.float32)).to(dtype).to(DEV)
    return room[at:].view(rows, vocab + gap)[:, :vocab] if rows else room.new_empty((0, vocab))


def plain_top(z, k, T):
    """(index, value, tail) of z in 64 bits."""
    o = z.sort(dim=1, descending=True, stable=True)  # (-0.0 and +0.0 are equal, equal ones by rising index)
    return o.indices[:, :k], o.values[:, :k], torch.logsumexp(o.values[:, k:] / T, 1)


def check_top(ctx, logits, k, T=1.0):
    T = float(np.float32(T))  # (the library's temperature is an fp32 number: 0.7 is another one)
    top = ctx.top_logits(logits, k, T)
    ctx.sync()
    z = logits.cpu().double()
    index, value, tail = plain_top(z, k, T)
    assert torch.equal(top.index.cpu().long(), index)
    assert torch.equal(top.value.cpu().double(), value)
    got = top.tail.cpu().double()
    tail = tail.float().double()  # (below the range of fp32, 2 * -3.4e38 among them, the nearest fp32 number is -inf)
    low = torch.isinf(tail)
    assert torch.equal(got[low], tail[low])
    # every exponential and its argument in fp32 (2^-21 of the sum), the logarithm rounded to fp32
    assert not bool(((got - tail).abs()[~low] > 2.0 ** -20 + 2.0 ** -23 * tail.abs()[~low]).any())
    assert ctx.top_logits(logits, k, T, want_tail=False).tail is None
    return top


@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,vocab,k", [(1, 1, 1), (2, 5, 5), (3, 31, 7), (1, 1000, 1), (4, 1000, 256), (2, 2040, 255),
                                          (3, 256, 256), (5, 8193, 64), (2, 50257, 20), (1, 262144, 256), (40, 3001, 33)])
def test_top(ctx, rows, vocab, k, dtype):
    rng = np.random.default_rng(vocab + k)
    check_top(ctx, logits_of(rng, rows, vocab, dtype), k)
    check_top(ctx, logits_of(rng, rows, vocab, dtype, gap=3, at=1), k, 2.5)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_top_with_equal_and_masked_logits(ctx, dtype):
    rng = np.random.default_rng(3)
    for vocab, k in ((50, 9), (5000, 40), (70001, 128)):
        z = logits_of(rng, 8, vocab, dtype)
        z[0] = 0.0                                   # all equal
        z[0, ::2] = -0.0
        z[1] = -INF                                  # nothing allowed
        z[2, k // 2:] = -INF                         # fewer than k allowed, the first ones
        z[3, :-(k // 2)] = -INF                      # ... the last ones
        z[4] = torch.finfo(dtype).min                # the type's lowest value as a mask
        z[4, 7] = 1.0
        z[5] = torch.from_numpy(rng.integers(0, 3, vocab).astype(np.float32)).to(DEV)  # many equal ones
        z[6] = -1000.0                               # far below the one that is listed first
        z[6, vocab // 2] = 1000.0
        z[7] = torch.arange(vocab, device=DEV).to(dtype)
        check_top(ctx, z, k, 0.5)
        check_top(ctx, z, 1)


def test_top_with_nan_and_infinity(ctx):
    z = logits_of(np.random.default_rng(4), 4, 3000, F32)
    z[0, 100], z[0, 200] = float("nan"), INF
    z[1, 5], z[1, 4] = INF, -float("nan")
    z[2] = float("nan")
    top = ctx.top_logits(z, 4)
    ctx.sync()
    assert top.index[0, :2].tolist() == [100, 200] and top.index[1, :2].tolist() == [4, 5]
    assert top.index[2].tolist() == [0, 1, 2, 3] and bool(torch.isnan(top.tail[:3]).all())
    assert bool(torch.isfinite(top.tail[3])) and torch.equal(top.index[3].long(), plain_top(z[3:].cpu().double(), 4, 1.0)[0][0].to(DEV))


def test_the_same_every_time(ctx):
    rng = np.random.default_rng(20)
    for rows, vocab, k in ((600, 5000, 60), (20, 40000, 200)):
        z = logits_of(rng, rows, vocab, F32)
        z[::3, 100:900] = 2.0  # more equal ones than there are places
        a, b = (ctx.top_logits(z, k, 1.5) for _ in range(2))
        (la, sa), (lb, sb) = (ctx.distill(z * 0.5, a) for _ in range(2))
        assert torch.equal(a.index, b.index) and torch.equal(a.value, b.value) and torch.equal(a.tail, b.tail)
        assert torch.equal(la, lb) and torch.equal(sa, sb)


def plain_distill(z, index, value, tail, T, g):
    """(loss, gradient, sum of the magnitudes behind the loss) in 64 bits, row by row, from the definitions."""
    rows, vocab = z.shape
    loss, grad, size = torch.zeros(rows, dtype=torch.float64), torch.zeros_like(z), torch.zeros(rows, dtype=torch.float64)
    for r in range(rows):
        seen, t = [], []
        for i, v in zip(index[r].tolist(), value[r].tolist()):
            if 0 <= i < vocab and i not in seen:
                seen.append(i)
                t.append(v / T)
        t = torch.tensor(t + ([float(tail[r])] if tail is not None else []), dtype=torch.float64)
        if not seen or bool((t == -INF).all()) or bool((z[r] == -INF).all()):
            continue
        p = torch.log_softmax(t, 0)
        lq = torch.log_softmax(z[r] / T, 0)
        rest = lq.clone()
        rest[seen] = -INF
        out = torch.logsumexp(rest, 0)
        q = torch.cat([lq[seen], out[None]])[:p.numel()]
        on = p > -INF
        terms = p[on].exp() * (p[on] - q[on])
        loss[r], size[r] = terms.sum(), (p[on].exp() * (p[on] - q[on]).abs()).sum()
        # q_v (1 - P_tail / q_rest) = (q_v / q_rest) (q_rest - P_tail), also where q_rest is less than fp64 holds
        if out > -INF:
            grad[r] = (rest - out).exp() * (out.exp() - (p[-1].exp() if tail is not None else 0.0))
        grad[r][seen] = lq[seen].exp() - p[:len(seen)].exp()
        grad[r] *= g[r] / T
    return loss, grad, size


def check_distill(ctx, logits, index, value, tail, T, g=None):
    T = float(np.float32(T))  # (the library's temperature is an fp32 number: 0.7 is another one)
    top = api.TopLogits(index, value, tail, T)
    loss, saved = ctx.distill(logits, top)
    grad = ctx.distill_grad(logits, top, saved, g)
    ctx.sync()
    z = logits.cpu().double()
    gg = g.cpu().double() if g is not None else torch.ones(z.shape[0], dtype=torch.float64)
    want, wgrad, size = plain_distill(z, index.cpu(), value.cpu().double(), None if tail is None else tail.cpu().double(), T, gg)
    got = loss.cpu().double()
    inf = torch.isinf(want)
    assert torch.equal(got[inf], want[inf])
    # The sums of exponentials have 2^-21 of relative error each; the loss moves by that times sum |q - P|, which is at
    # most sqrt(2 loss) and at most 2; roundings of its own are 2^-23 of the terms' sum.
    off = (got - want).abs()[~inf] - (2.0 ** -21 * torch.sqrt(2 * want[~inf].clamp(0, 2)) + 2.0 ** -23 * want[~inf] + 1e-12 * (1 + size[~inf]))
    assert off.numel() == 0 or float(off.max()) <= 0.0, float(off.max())
    # gradient: q with 2^-18 (the exponential of an argument of up to 60 in fp32), P in fp64, the share that the rest
    # keeps with 2^-20 of 1 + its size
    dt = logits.dtype
    q = torch.softmax(z / T, 1).nan_to_num(0.0)
    spread = q * gg.abs()[:, None] / T + wgrad.abs()
    assert bool(torch.isfinite(grad).all())
    tol = A.HALF[dt] * wgrad.abs() + 2.0 ** -18 * spread + A.TINY[dt]
    bad = ((grad.cpu().double() - wgrad).abs() > tol)
    assert not bool(bad.any()), (int(bad.sum()), float(((grad.cpu().double() - wgrad).abs() / tol).max()))
    assert torch.equal(loss, ctx.distill(logits, top, want_saved=False)[0])
    same = logits.clone()
    assert torch.equal(ctx.distill_grad(same, top, saved, g, out=same), grad)  # in the logits' place
    return got, grad


def teacher_list(z, k, T):
    o = z.float().topk(k, 1)
    rest = z.float().scatter(1, o.indices, -INF)
    return o.indices.to(torch.int32), o.values.contiguous(), torch.logsumexp(rest.double() / T, 1).float()


@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,vocab,k", [(1, 1, 1), (2, 3, 2), (4, 40, 40), (3, 1000, 1), (5, 2051, 64), (2, 30522, 256),
                                          (1, 262144, 100), (37, 515, 17)])
def test_distill(ctx, rows, vocab, k, dtype):
    rng = np.random.default_rng(vocab)
    for T, near, gap, at in ((1.0, 0.3, 0, 0), (2.0, 1e-3, 8, 0), (0.7, 3.0, 5, 1)):
        t = logits_of(rng, rows, vocab, F32)
        index, value, tail = teacher_list(t, k, T)
        z = logits_of(rng, rows, vocab, dtype, gap, at)
        z.copy_(t + near * torch.randn_like(t))
        g = torch.from_numpy(rng.uniform(-1, 2, rows).astype(np.float32)).to(DEV)
        check_distill(ctx, z, index, value, tail if k < vocab else None, T, g)
        check_distill(ctx, z, index, value, None, T)


def test_distill_places_and_masks(ctx):
    rng = np.random.default_rng(5)
    rows, vocab, k, T = 14, 901, 12, 1.5
    t = logits_of(rng, rows, vocab, F32)
    index, value, tail = teacher_list(t, k, T)
    for dtype in (F32, BF16):
        for with_tail in (False, True):
            i, v, l = index.clone(), value.clone(), tail.clone()
            z = (t + 0.2 * torch.randn_like(t)).to(dtype)
            i[0] = -1                             # nothing listed
            i[1, 3:] = -1                         # places left empty
            i[2, 0], i[2, 5] = vocab, 1 << 30     # outside the vocabulary
            i[3, 4:8] = i[3, 0]                   # an index that stands several times
            i[4] = i[4, 3]
            v[5] = -INF                           # the teacher allows none of the listed ones
            v[6, 2] = -INF                        # ... not one of them
            z[7] = -INF                           # the student allows nothing
            z[8, 300:] = -INF                     # a masked part, some of it listed
            z[9] = z[9].masked_fill(~torch.zeros(vocab, dtype=torch.bool, device=DEV).scatter(0, i[9].long(), True), -INF)
            z[10] = torch.finfo(dtype).min        # the type's lowest value as a mask
            z[10, i[10].long()] = 1.0
            l[11] = -INF
            z[12, i[12].long()] = -INF            # nothing listed is allowed
            l[5] = -INF if not with_tail else l[5]
            check_distill(ctx, z, i, v, l if with_tail else None, T, torch.ones(rows, device=DEV))


def test_distill_nan_stays_in_its_row(ctx):
    rng = np.random.default_rng(6)
    t = logits_of(rng, 5, 3000, F32)
    index, value, tail = teacher_list(t, 8, 1.0)
    top = api.TopLogits(index, value, tail)
    z = t + 0.1
    clean = ctx.distill(z, top)
    grad = ctx.distill_grad(z, top, clean[1])
    z[1, 2999], z[3, 17] = float("nan"), INF
    loss, saved = ctx.distill(z, top)
    g2 = ctx.distill_grad(z, top, saved)
    keep = [0, 2, 4]
    assert torch.equal(loss[keep], clean[0][keep]) and torch.equal(g2[keep], grad[keep])
    assert bool(torch.isnan(loss[[1, 3]]).all()) and bool(torch.isnan(g2[[1, 3]]).all())


def test_distill_of_the_teacher_itself_is_zero(ctx):
    rng = np.random.default_rng(7)
    z = logits_of(rng, 6, 5003, F32)
    top = ctx.top_logits(z, 50, 2.0)
    loss, saved = ctx.distill(z, top)
    # the tail is rounded to fp32: log P is off by up to 2^-24 of a tail of at most 16, and the loss by its square
    assert float(loss.abs().max()) < (16 * 2.0 ** -23) ** 2 + 1e-12
    assert float(ctx.distill_grad(z, top, saved).abs().max()) < 2.0 ** -17


def test_distill_differences(ctx):
    rng = np.random.default_rng(8)
    t = logits_of(rng, 3, 200, F32)
    index, value, tail = teacher_list(t, 6, 2.0)
    z = t + 0.5 * torch.randn_like(t)
    top = api.TopLogits(index, value, tail, 2.0)
    _, saved = ctx.distill(z, top)
    grad = ctx.distill_grad(z, top, saved).cpu().double()
    zz, h, one = z.cpu().double(), 1e-5, torch.ones(3)
    f = lambda zz: plain_distill(zz, index.cpu(), value.cpu().double(), tail.cpu().double(), 2.0, one)[0]  # noqa: E731
    for col in (0, 77, 199, int(index[0, 0]), int(index[2, 5])):
        e = torch.zeros_like(zz)
        e[:, col] = h
        assert float(((f(zz + e) - f(zz - e)) / (2 * h) - grad[:, col]).abs().max()) < 1e-6


def test_streams_and_graphs(ctx):
    rng = np.random.default_rng(9)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        c2 = api.Context(torch.device(DEV))
    teacher, z = logits_of(rng, 20, 5000, BF16), logits_of(rng, 20, 5000, BF16)
    g0 = torch.rand(20, device=DEV)

    def run(c):
        top = c.top_logits(teacher, 30, 2.0)
        loss, saved = c.distill(z, top)
        return [top.index, top.value, top.tail, loss, saved, c.distill_grad(z, top, saved, g0)]

    assert all(torch.equal(a, b) for a, b in zip(run(ctx), run(c2)))
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        out = run(c2)
    for _ in range(3):
        for t in (teacher, z, g0):
            t.copy_(torch.randn_like(t))
        want = run(ctx)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, out))
    c2.close()


def test_no_rows(ctx):
    z = torch.empty((0, 100), device=DEV)
    top = ctx.top_logits(z, 5)
    loss, saved = ctx.distill(z, top)
    assert top.index.shape == (0, 5) and loss.shape == (0,) and ctx.distill_grad(z, top, saved).shape == (0, 100)


def test_refusals(ctx):
    import ctypes as C
    z = torch.zeros((4, 100), device=DEV)
    i, v = torch.zeros((4, 5), dtype=torch.int32, device=DEV), torch.zeros((4, 5), device=DEV)
    lib, h, m = ctx.lib, ctx.h, api.CMatrix
    top = lambda z=m(z.data_ptr(), 100), type=0, rows=4, vocab=100, k=5, T=1.0, i=i.data_ptr(), v=v.data_ptr(): (  # noqa: E731
        lib.inshr_top_logits(h, z, type, rows, vocab, k, T, i, v, None))
    assert top() == 0
    assert top(z=m(None, 100)) == -1 and top(z=m(z.data_ptr() + 2, 100)) == -1 and top(type=3) == -1
    assert top(k=0) == -1 and top(k=101) == -1 and top(vocab=1000, k=257) == -1 and top(vocab=(1 << 18) + 1) == -1
    for T in (0.0, -1.0, float("nan"), INF):
        assert top(T=T) == -1
    assert top(i=None) == -1 and top(v=None) == -1 and top(rows=(1 << 22) + 1) == -1
    d = lambda **k: api.CDistillIn(**{**dict(logits=m(z.data_ptr(), 100), index=i.data_ptr(), value=v.data_ptr(), tail=None,  # noqa: E731
                                             rows=4, n_vocab=100, k=5, type=0, temperature=1.0), **k})
    loss, saved = torch.empty(4, device=DEV), torch.empty((4, 4), dtype=torch.float64, device=DEV)
    run = lambda c: lib.inshr_distill(h, C.byref(c), loss.data_ptr(), saved.data_ptr())  # noqa: E731
    assert run(d()) == 0
    for bad in (dict(index=None), dict(value=None), dict(k=0), dict(k=257), dict(temperature=0.0), dict(type=9),
                dict(n_vocab=0), dict(logits=m(None, 100)), dict(tail=loss.data_ptr() + 2)):
        assert run(d(**bad)) == -1, bad
    g = lambda out, s=saved.data_ptr(): lib.inshr_distill_grad(h, C.byref(d()), s, None, out)  # noqa: E731
    out = torch.empty_like(z)
    assert g(m(out.data_ptr(), 100)) == 0 and g(m(z.data_ptr(), 100)) == 0
    assert g(m(out.data_ptr(), 99)) == -1 and g(m(None, 100)) == -1 and g(m(z.data_ptr(), 101)) == -1
    assert g(m(out.data_ptr(), 100), None) == -1
    ctx.sync()
