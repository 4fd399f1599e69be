"""The operators on token batches from their formulas, in 64 bits on the CPU, and how far 32-bit kernels may be off.

Bounds.  One rounding to 32 bits is at most U = 2^-24 of the value, one to the output's type at most half of its `eps`.

* exp(x - m) in 32 bits: the difference is rounded (U |x - m| of the exponential), scaled by log2 e (the same again) and
  raised by the hardware (2 U).  Terms with |x - m| > 24 are below 2^-34 of the largest and do not matter, so a sum's terms are
  each off by at most 50 U.  Up to 1,024 additions a lane and 24 more to join them add up like a random walk, 34 U.  So the
  logarithm of the sum is off by at most LOG_SUM = 96 U, and a log-probability by that and its own rounding.
* A gradient's term u p: U (96 + 2 |x - lse| + 6) of its value.  At the target u (1 - p): the error of p, and 4 U of u.
* Products and sums of an embedding's gradient: every term has one rounding of the product, and joining k of them in any
  order costs at most k roundings of the sum of their magnitudes.
"""
import numpy as np
import torch

U = 2.0 ** -24
LOG_SUM = 96 * U
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF_ULP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
# half of the smallest positive number of the type (f32: what the hardware's exponential may flush to zero)
SMALLEST = {torch.float32: 2.0 ** -126, torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -25}


def logprobs(logits, targets):
    """(logprobs, lse) in 64 bits; 0 for rows that are not scored."""
    x, vocab = logits.double().cpu(), logits.shape[1]
    t = targets.long().cpu()
    scored = (t >= 0) & (t < vocab)
    lp, lse = torch.zeros(len(t), dtype=torch.float64), torch.zeros(len(t), dtype=torch.float64)
    rows = scored.nonzero().squeeze(1)
    if len(rows):
        m = x[rows].amax(1, keepdim=True)
        log_sum = (x[rows] - m).exp().sum(1).log()
        lse[rows] = m.squeeze(1) + log_sum
        lp[rows] = x[rows, t[rows]] - m.squeeze(1) - log_sum      # (of huge logits lse keeps nothing of the sum)
    return lp, lse


def logits_grad(logits, targets, upstream, lse=None):
    """(gradient in 64 bits, how far each of its elements may be off before it is rounded to the output's type).  With `lse`,
    from that: what a caller that keeps it between two calls has."""
    x, u = logits.double().cpu(), upstream.double().cpu()
    t = targets.long().cpu()
    scored = ((t >= 0) & (t < x.shape[1]) & (u != 0)).nonzero().squeeze(1)
    grad, off = torch.zeros_like(x), torch.zeros_like(x)
    if len(scored):
        if lse is None:
            d = x[scored] - x[scored].amax(1, keepdim=True)
            d = d - d.exp().sum(1, keepdim=True).log()
        else:
            d = x[scored] - lse.double().cpu()[scored, None]
        p, c = d.exp(), u[scored, None]
        far = torch.where(torch.isfinite(d), d.abs(), 0.0)
        grad[scored] = -c * p
        off[scored] = c.abs() * p * U * (102 + 2 * far)
        at = t[scored]
        grad[scored, at] += u[scored]
        off[scored, at] += 4 * U * u[scored].abs()
    return grad, off


def assert_near(got, want, off, what=""):
    """|got - want| <= off and a rounding to got's type, everywhere; NaN and infinities where `want` has them."""
    dtype, got, want = got.dtype, got.double().cpu(), want.double()
    odd = ~torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), f"{what}: NaN in other places"
    assert torch.equal(got[odd & ~torch.isnan(want)], want[odd & ~torch.isnan(want)]), f"{what}: infinities differ"
    bound = torch.as_tensor(off) + (want.abs() + torch.as_tensor(off)) * HALF_ULP[dtype] + SMALLEST[dtype]
    bad = ((got - want).abs() > bound) & ~odd
    if bad.any():
        at = tuple(int(i) for i in bad.nonzero()[0])
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} too far off, the first at {at}: got {got[at]}, want {want[at]}, "
                             f"bound {bound.expand_as(want)[at]}")


def next_tokens(ids, offsets, first=None):
    out = np.full(len(ids), -1, dtype=np.int32)
    for i in range(len(offsets) - 1):
        b, e = int(offsets[i]), int(offsets[i + 1])
        lead = 1 if first is None else max(1, int(first[i]))
        for t in range(b, e - 1):
            if t + 1 - b >= lead:
                out[t] = ids[t + 1]
    return out


def strings_of(rows, offsets):
    """The string of each row, -1 outside."""
    out = torch.full((rows,), -1, dtype=torch.long)
    for i, (b, e) in enumerate(zip(offsets, offsets[1:])):
        out[int(b):int(e)] = i
    return out


def preference(lp, targets, offsets, vocab, reference, beta, smoothing):
    """(loss, margins) from log-probabilities in 64 bits, differentiable in them."""
    string = strings_of(len(lp), offsets)
    scored = (targets >= 0) & (targets < vocab) & (string >= 0)
    apart = torch.where(scored, lp - (torch.where(scored, reference.double(), 0.0) if reference is not None else 0.0), 0.0)
    sums = torch.stack([apart[string == i].sum() for i in range(len(offsets) - 1)]) if len(offsets) > 1 else torch.zeros(0)
    z = beta * (sums[0::2] - sums[1::2])
    zero = torch.zeros_like(z)                            # (exp(z) alone would overflow from 710 on)
    each = (1 - smoothing) * torch.logaddexp(zero, -z) + smoothing * torch.logaddexp(zero, z)
    return (each.mean() if len(z) else each.sum()), z


def policy(lp, targets, offsets, vocab, old, advantages, reference, low, high, kl_weight, by_string):
    """The loss from log-probabilities in 64 bits, differentiable in them."""
    string = strings_of(len(lp), offsets)
    scored = ((targets >= 0) & (targets < vocab) & (string >= 0)).nonzero().squeeze(1)
    total = lp.new_zeros(())
    batch = len(offsets) - 1
    for t in scored.tolist():
        i = int(string[t])
        w = 1 / (batch * int((string[scored] == i).sum())) if by_string else 1 / len(scored)
        a = float(advantages[i if by_string and len(advantages) == batch else t])
        r = torch.exp(lp[t] - float(old[t]))
        cut = min(max(float(r.detach()), 1 - low), 1 + high)
        value = -r * a if float(r.detach()) * a <= cut * a else -lp.new_tensor(cut * a)
        if reference is not None:
            d = float(reference[t]) - lp[t]
            value = value + kl_weight * (torch.exp(d) - d - 1)
        total = total + w * value
    return total
