"""MI355X-native hot path of the checkpoint compressor: search, quantize, delta, and layers run from their compressed form.

The work is done by HIP kernels behind the C ABI of include/inshr.h (libinshr.so); this package only
marshals arguments.  `synth` holds the seeded input generators used by tests and bench."""
from . import synth  # noqa: F401


def Context(*args, **kwargs):
    """inshr_create: see api.Context."""
    from .api import Context as _C
    return _C(*args, **kwargs)


def inshr_search(ctx, tensors, grid, eps, want_scores=True):
    return ctx.search(tensors, grid, eps, want_scores)


def inshr_quantize(ctx, tensors, cfgs, reuse_search=False, out=None):
    return ctx.quantize(tensors, cfgs, reuse_search, out)


def inshr_delta(ctx, prev, cur, want_perm=False, prev_perm=None, out=None):
    return ctx.delta(prev, cur, want_perm, prev_perm, out)


def inshr_linear(ctx, layer, x, residual=None, out=None, want_pre=False):
    return ctx.linear(layer, x, residual, out, want_pre)


def inshr_linear_grad(ctx, layer, x, dy, pre=None, want_dx=True, want_dw=True, want_dbias=True):
    return ctx.linear_grad(layer, x, dy, pre, want_dx, want_dw, want_dbias)


def inshr_top_logits(ctx, logits, k, temperature=1.0, want_tail=True):
    return ctx.top_logits(logits, k, temperature, want_tail)


def inshr_distill(ctx, logits, top, want_saved=True):
    return ctx.distill(logits, top, want_saved)


def inshr_distill_grad(ctx, logits, top, saved, grad_loss=None, out=None):
    return ctx.distill_grad(logits, top, saved, grad_loss, out)
