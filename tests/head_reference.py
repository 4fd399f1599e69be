"""The operators at a model's output end from their formulas, in 64 bits on the CPU, and how far 32-bit kernels may be off.

Bounds, in units of U = 2^-24 (a rounding to 32 bits is at most U of the value):

* Sum of squares: all terms are positive, each is rounded with its addition; a lane has at most 32 of them one after another and 22
  additions join lanes and waves, so at most 54 U of the sum.  Half of that is left in the root, and mean, eps, root and reciprocal
  round once each: a norm's factor is off by at most ROOT = 32 U.
* A norm's element has two more roundings, a scale of 8-bit rows two (the quotient is 64-bit).  8-bit values are exact: the rounding
  of the 64-bit quotient.
* Gradient of x, with h = s rstd: sum of g w h with two roundings a term and at most 54 additions: 58 U of the sum of magnitudes, its
  mean two more; the element g w - h m has four roundings of its parts.
* Gradient of the weights: two roundings a term and at most 256 additions in 32 bits, the rest in 64.
* An 8-bit product's sum is exact: its conversion and the two scales round once each.
* Adjusted logits: a product with the penalty or its rounded reciprocal, presence + frequency c, their difference and a bias: at most one
  rounding each of values no larger than the sum of the parts' magnitudes.  Their gradient: that product.
"""
import math

import torch

U = 2.0 ** -24
ROOT = 32 * U


def summed(x, residual):
    return x.cpu() if residual is None else (x.cpu().float() + residual.cpu().float()).to(x.dtype)


def norm(s, weight, eps):
    """(norm, factor) in 64 bits of rows s."""
    s, weight = s.cpu().double(), weight.cpu().double()
    root = 1 / (s.square().mean(1) + eps).sqrt()
    return s * root[:, None] * weight, root


def rows_8bit(p, factor):
    """(8-bit rows, scales in 64 bits) of rows p of products in 64 bits; `factor` is what the rows are multiplied by besides."""
    top = p.abs().amax(1, keepdim=True)
    fine = torch.isfinite(p).all(1, keepdim=True) & torch.isfinite(factor.reshape(-1, 1))
    q = torch.where(fine & (top > 0), (p * 127 / torch.where(top > 0, top, 1.0)).round(), 0.0)
    scales = torch.where(fine, torch.where(top > 0, top * factor.reshape(-1, 1) / 127, 0.0), math.nan)
    return q.to(torch.int8), scales.reshape(-1)


def in_range(want, dtype):
    """What rounding to float16 makes of values beyond its range: from 65,520 on, half a step above its largest number, infinity.
    (The wider types' ranges are not reached here.)"""
    return torch.where(want.abs() >= 65520, want.sign() * math.inf, want) if dtype == torch.float16 else want


def norm_grad(g, s, weight, rstd, more=None):
    """((gradient of x, bound), (gradient of the weights, bound)) from a factor that is given."""
    g, s, weight, rstd = (t.cpu().double() for t in (g, s, weight, rstd))
    h, u = s * rstd[:, None], g * weight
    mean, size = (u * h).mean(1, keepdim=True), (u * h).abs().mean(1, keepdim=True)
    to_x = rstd[:, None] * (u - h * mean)
    off = U * rstd[:, None] * (4 * u.abs() + h.abs() * (4 * mean.abs() + 62 * size))
    if more is not None:
        to_x = to_x + more.cpu().double()
        off = off + U * to_x.abs()
    to_weight = g * h
    return (to_x, off), (to_weight.sum(0), 260 * U * to_weight.abs().sum(0))


def project(q, scales, weight, weight_scales):
    total = q.cpu().double() @ weight.cpu().double().t()
    return total * scales.cpu().double()[:, None] * weight_scales.cpu().double()


def _rows(x, n, width):
    """Three numbers for all rows, or a row's own."""
    return torch.tensor(x, dtype=torch.float64).expand(n, width) if isinstance(x, tuple) else x.cpu().double()


def counts(vocab, ids, begin, end):
    n = len(begin)
    c = torch.zeros(n, vocab, dtype=torch.float64)
    for t in range(n):
        mine = ids.cpu()[max(0, int(begin[t])):max(0, min(len(ids), int(end[t])))].long()
        mine = mine[(mine >= 0) & (mine < vocab)]
        c[t].index_add_(0, mine, torch.ones(len(mine), dtype=torch.float64))
    return c


def allowed(n, vocab, mask, state):
    if mask is None:
        return torch.ones(n, vocab, dtype=torch.bool)
    bits = (mask.cpu()[:, torch.arange(vocab) // 32] >> (torch.arange(vocab) % 32).to(torch.int32)) & 1 != 0
    if state is None:
        return bits.expand(n, vocab) if len(bits) == 1 else bits
    state = state.cpu().long()
    free = (state < 0) | (state >= len(bits))
    return bits[torch.where(free, 0, state)] | free[:, None]


def adjust(logits, ids=None, begin=None, end=None, penalties=None, bias=None, mask=None, state=None):
    """(adjusted logits in 64 bits, bounds)"""
    x = logits.cpu().double().clone()
    n, vocab = x.shape
    size = torch.zeros_like(x)
    if ids is not None:
        p = _rows(penalties or (1.0, 0.0, 0.0) if not isinstance(penalties, torch.Tensor) else penalties, n, 3)
        c = counts(vocab, ids, begin, end)
        once = p[:, 1:2] + p[:, 2:3] * c
        scaled = torch.where(x > 0, x / p[:, :1], x * p[:, :1])
        size = torch.where(c > 0, scaled.abs() + p[:, 1:2].abs() + (p[:, 2:3] * c).abs(), size)
        x = torch.where(c > 0, scaled - once, x)
    if bias is not None:
        bias_ids, values, bias_begin, bias_end = (t.cpu() for t in bias)
        for t in range(n):
            last = {}
            for i in range(max(0, int(bias_begin[t])), min(len(bias_ids), int(bias_end[t]))):
                if 0 <= int(bias_ids[i]) < vocab:
                    last[int(bias_ids[i])] = float(values[i])
            for v, b in last.items():
                x[t, v] += b
                size[t, v] += abs(b)
    keep = allowed(n, vocab, mask, state)
    size = torch.where(torch.isfinite(size), size, 0.0)
    return torch.where(keep, x, -math.inf), 4 * U * size


def adjust_grad(grad, logits, ids=None, begin=None, end=None, penalties=None, mask=None, state=None):
    g = grad.cpu().double().clone()
    n, vocab = g.shape
    if ids is not None:
        p = _rows(penalties or (1.0, 0.0, 0.0) if not isinstance(penalties, torch.Tensor) else penalties, n, 3)[:, :1]
        g = torch.where(counts(vocab, ids, begin, end) > 0, torch.where(logits.cpu().double() > 0, g / p, g * p), g)
    g = torch.where(allowed(n, vocab, mask, state), g, 0.0)
    return g, U * g.abs()                            # (the reciprocal's; the product's is the result's own)
