"""GPU: rows of logits at the ends of what the header allows, against plain forms in 64 bits."""
import numpy as np
import pytest
import torch

from paper_2306_11800_amd import api
from tests.test_gpu_logits import check_distill, check_top, logits_of, teacher_list

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def ctx():
    c = api.Context(torch.device(DEV))
    yield c
    c.close()


@pytest.mark.parametrize("rows,vocab,k", [(14, 700, 12), (600, 300, 3), (14, 9000, 200)])
def test_nan_is_never_a_loss_of_zero(ctx, rows, vocab, k):
    """Rows with NaN or +inf have loss and gradient NaN, whatever else stands in them; a row of which the teacher says
    nothing has 0, whatever stands in it; the rows beside them do not change."""
    rng = np.random.default_rng(vocab)
    for dtype in (F32, BF16):
        t = logits_of(rng, rows, vocab, F32)
        index, value, tail = teacher_list(t, k, 1.0)
        for with_tail in (False, True):
            i, v, l = index.clone(), value.clone(), tail.clone()
            z = (t + 0.1).to(dtype)
            top = api.TopLogits(i, v, l if with_tail else None)
            clean, saved = ctx.distill(z, top)
            cgrad = ctx.distill_grad(z, top, saved)
            unlisted = int(t[3].argmin())
            z[0] = NAN                                   # what a layer makes of a row with NaN
            z[1] = -INF
            z[1, i[1, 0].long()] = NAN                   # nothing but NaN is there, and it is listed
            z[2] = -INF
            z[2, int(t[2].argmin())] = NAN               # ... not listed
            z[3, unlisted] = NAN
            z[3, :unlisted] = -INF                       # the masked ones too
            z[4] = -INF
            z[4, i[4, -1].long()] = INF
            z[5] = INF
            v[6] = NAN                                   # the teacher
            v[7] = -INF
            v[7, -1] = NAN
            l[7] = -INF
            v[8, 0] = INF
            i[9], z[9] = -1, NAN                         # padding
            v[10], l[10], z[10] = -INF, -INF, NAN        # a teacher that allows nothing
            if with_tail:
                v[11], l[11] = -INF, NAN
            else:
                v[11] = NAN
            i[12, 1:] = -1
            v[12, 1:] = NAN                              # values of empty places do not count
            loss, saved = ctx.distill(z, top)
            grad = ctx.distill_grad(z, top, saved)
            bad, none = [0, 1, 2, 3, 4, 5, 6, 7, 8, 11], [9, 10]
            keep = [r for r in range(rows) if r not in bad + none + [12]]
            assert torch.isnan(loss).nonzero()[:, 0].tolist() == bad
            assert torch.isnan(grad).all(1).nonzero()[:, 0].tolist() == bad and not bool(torch.isnan(grad[none + keep + [12]]).any())
            assert not bool(loss[none].any()) and not bool(grad[none].any())
            assert torch.equal(loss[keep], clean[keep]) and torch.equal(grad[keep], cgrad[keep])
            same = z.clone()
            again = ctx.distill_grad(same, top, saved, out=same)
            assert torch.equal(again.isnan(), grad.isnan()) and torch.equal(again.nan_to_num(), grad.nan_to_num())


def test_teachers_far_apart(ctx):
    """P that fp64 does not hold, where q is anything: listed values and tails far below the largest, masks of the type's
    lowest value on either side.  (A P that is 0 in 64 bits counts as 0.)"""
    rng = np.random.default_rng(2)
    rows, vocab, k = 12, 400, 10
    low = torch.finfo(F32).min
    for T in (0.5, 1.0, 4.0):
        for dtype in (F32, BF16, F16):
            t = logits_of(rng, rows, vocab, F32)
            index, value, tail = teacher_list(t, k, T)
            z = (t + 0.3 * torch.randn_like(t)).to(dtype)
            value[0, 4:] -= 800 * T
            value[1, 2:] -= 720 * T                       # e^d is past fp64, P e^d is not
            value[2, 1:] = low                            # masked by the lowest value: one allowed, and what is left
            tail[2] = low / T if T >= 1.0 else -INF
            tail[3] = -900.0
            tail[4] = value[4, 0] / T - 730.0
            value[5, 3:] = torch.finfo(BF16).min
            value[6, 1:], tail[6] = low, -INF
            z[7, index[7, 1:].long()] = -INF              # the student masks by -inf what the teacher masks by the lowest
            value[7, 1:], tail[7] = low, -INF
            value[8, 1:] -= 745 * T                       # P at the end of fp64
            value[9, ::2] += 1000 * T
            # (where q is 0 too the plain form has no value: a P of 0 is what -inf in the list gives)
            runs, none = [], value.clone()
            none[7, 1:] = -INF
            for v in (value, none):
                top = api.TopLogits(index, v, tail, T)
                loss, saved = ctx.distill(z, top)
                runs.append((loss, ctx.distill_grad(z, top, saved)))
            assert all(torch.equal(a, b) for a, b in zip(*runs))
            check_distill(ctx, z, index, none, tail, T)
            check_distill(ctx, z, index, none, None, T)


def test_small_temperatures(ctx):
    """A masked or large logit times log2 e / T leaves the range of fp32, and of two logarithms that far out nothing but the
    difference is left.  (A tail of 13 / T has to lie within fp32.)"""
    rng = np.random.default_rng(3)
    rows, vocab, k = 8, 3000, 7
    for T in (1e-3, 1e-8, 1e-12, 1e-30, 2.0 ** -120):
        for dtype in (F32, BF16):
            t = logits_of(rng, rows, vocab, F32)
            t[3] = torch.finfo(F32).min
            t[3, 5:9] = torch.tensor([1.0, 1.0, 2.0, 0.5], device=DEV)
            t[4] *= min(T, 1.0) * 2.0                     # logits that lie T apart
            index, value, _ = teacher_list(t, k, 1.0)
            z = t.clamp(torch.finfo(dtype).min, -torch.finfo(dtype).min).to(dtype)
            z[0, ::3] = torch.finfo(dtype).min
            top = check_top(ctx, z, k, T)
            # (loss and gradient of other rows are of the size of 1 / T, which fp32 holds down to 1e-30 or so)
            scale = torch.full((rows,), 2.0 ** -20 * T, device=DEV)
            check_distill(ctx, z, top.index, top.value, top.tail, T, scale)


def test_logits_near_the_end_of_the_range(ctx):
    rng = np.random.default_rng(4)
    for dtype in (F32, BF16):
        z = logits_of(rng, 7, 1000, dtype)
        z[0, 100:110] = 3.2e38
        z[1, 50] = -3.2e38
        z[2] = -3.0e38
        z[2, ::5] = -2.9e38
        z[3, 17] = 3.2e38
        z[4] = torch.finfo(dtype).min                 # all masked by the lowest value
        z[5] = torch.finfo(dtype).min                 # all but one
        z[5, 500] = 1.0
        z[6] = 1e-30
        index, value, tail = teacher_list(z, 30, 1.0)
        check_distill(ctx, z, index, value, tail, 1.0)
        check_distill(ctx, z, index, value, None, 0.7)


def test_temperatures_below_the_normal_numbers_are_refused(ctx):
    z = torch.zeros((4, 100), device=DEV)
    top = ctx.top_logits(z, 5, 2.0 ** -126)
    for T in (1e-39, 1e-45):
        with pytest.raises(RuntimeError):
            ctx.top_logits(z, 5, T)
        top.temperature = T
        with pytest.raises(RuntimeError):
            ctx.distill(z, top)
    ctx.sync()


@pytest.mark.parametrize("vocab", [300, 512, 1000, 1500, 1536, 2048, 2049, 8192, 8500, 50257])
def test_top_of_masked_rows(ctx, vocab):
    """Most of a row masked, by -inf or by finite values, in one piece or scattered: fewer than k allowed, exactly k, and
    more than there is room for; equal logits around the last place."""
    rng = np.random.default_rng(vocab)
    for rows, dtype in ((16, F32), (16, BF16), (600, BF16)):
        z = logits_of(rng, rows, vocab, dtype)
        some = torch.from_numpy(rng.permutation(vocab)).to(DEV)
        for r, mask in enumerate((-INF, -1000.0, torch.finfo(dtype).min)):
            for j, allowed in enumerate((some[:30], torch.arange(vocab - 40, vocab, device=DEV), some[:64])):
                keep = z[4 * r + j, allowed]
                z[4 * r + j] = mask
                z[4 * r + j, allowed] = keep
            z[4 * r + 3, vocab - vocab // 8:] = mask
        z[12] = -1000.0                                   # everything equal, and ...
        z[12, some[0]] = -2000.0
        z[13] = (z[13] * 2).round() / 2                   # many equal ones everywhere
        z[14] = -5.0
        z[14, some[:vocab // 2]] = -3.0                   # half of the row is what the last places are taken from
        z[14, some[:3]] = 1.0
        z[15, 1:] = -INF
        for k in (1, 30, 64, 65, 256):
            top = check_top(ctx, z, k, 2.0)
            again = ctx.top_logits(z, k, 2.0)
            assert torch.equal(top.index, again.index) and torch.equal(top.tail, again.tail)


def test_numbers_of_rows(ctx):
    """Either side of the numbers of rows, and sizes of a vocabulary, at which a row has more threads."""
    rng = np.random.default_rng(11)
    for vocab in (8191, 8192):
        z = logits_of(rng, 512, vocab, BF16)
        for rows in (256, 257):
            check_top(ctx, z[:rows], 20)
    t = logits_of(rng, 512, 900, F32)
    index, value, tail = teacher_list(t, 10, 1.0)
    z = (t + 0.3 * torch.randn_like(t)).to(BF16)
    for rows in (511, 512):
        check_distill(ctx, z[:rows], index[:rows], value[:rows], tail[:rows], 1.0)


def test_many_rows(ctx):
    """As many rows as a call takes, of a small vocabulary, and one more."""
    rows = 1 << 22
    z = torch.randn((rows, 5), device=DEV).to(BF16)
    top = ctx.top_logits(z, 2)
    order = z.float().sort(dim=1, descending=True, stable=True)
    assert torch.equal(top.index.long(), order.indices[:, :2]) and torch.equal(top.value, order.values[:, :2])
    assert float((top.tail - torch.logsumexp(order.values[:, 2:], 1)).abs().max()) < 2.0 ** -19
    s = torch.randn((rows, 5), device=DEV).to(BF16)
    loss, saved = ctx.distill(s, top)
    grad = ctx.distill_grad(s, top, saved)
    some = torch.tensor([0, 1, 65535, 65536, (1 << 21) + 3, rows - 1], device=DEV)
    few = api.TopLogits(top.index[some], top.value[some], top.tail[some])
    l2, s2 = ctx.distill(s[some], few)
    assert torch.equal(loss[some], l2) or float((loss[some] - l2).abs().max()) < 2.0 ** -19
    assert float((grad[some].float() - ctx.distill_grad(s[some], few, s2).float()).abs().max()) <= 2.0 ** -8
    assert bool((loss >= 0).all()) and float(grad.float().sum(1).abs().max()) < 2.0 ** -6  # (five roundings of 2^-9 and less)
    with pytest.raises(RuntimeError):
        ctx.top_logits(z[:1].expand(rows + 1, 5), 2)


def test_rows_far_apart(ctx):
    """Rows 2^31 elements apart: offsets of more than 32 bits."""
    rng = np.random.default_rng(12)
    far, rows, vocab = 1 << 31, 4, 5000
    room = torch.empty(far * (rows - 1) + 16384, dtype=BF16, device=DEV)
    z, out = (room[k:].as_strided((rows, vocab), (far, 1)) for k in (1, 6000))
    near = logits_of(rng, rows, vocab, BF16)
    z.copy_(near)
    a, b = ctx.top_logits(z, 30), ctx.top_logits(near, 30)
    assert torch.equal(a.index, b.index) and torch.equal(a.value, b.value) and torch.equal(a.tail, b.tail)
    student = (near.float() + 0.2).to(BF16)
    z.copy_(student)
    (la, sa), (lb, sb) = ctx.distill(z, a), ctx.distill(student, b)
    assert torch.equal(la, lb)
    assert torch.equal(ctx.distill_grad(z, a, sa, out=out), ctx.distill_grad(student, b, sb))


def test_large_temperatures(ctx):
    """Up to the largest number: every allowed logit counts the same, and what is masked by -inf counts nothing."""
    rng = np.random.default_rng(13)
    for T in (1e30, 3e37, 3e38):
        for dtype in (F32, BF16):
            t = logits_of(rng, 6, 2000, F32)
            t[1, 1000:] = -INF
            t[2, 4:] = -INF
            index, value, tail = teacher_list(t, 9, T)
            z = t.to(dtype)
            z[3, ::2] = -INF
            check_top(ctx, z, 9, T)
            check_distill(ctx, z, index, value, tail, T, torch.full((6,), T / 4, device=DEV))
