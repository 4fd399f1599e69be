"""The preference loss where a target is masked, so that its string is impossible: a pair's margin is infinite, and the pair adds what
-log sigmoid has there, 0 or infinity, but for terms whose weight is 0, which are left out."""
import numpy as np
import pytest
import torch

import ops_reference as ref
from ops_reference import LOG_SUM, TYPES, U, assert_near
from test_gpu_logits import dev, some_logits

pytestmark = pytest.mark.gpu

INF = float("inf")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [9, 33000])
@pytest.mark.parametrize("side", [0, 1])
@pytest.mark.parametrize("smoothing", [0.0, 0.25, 1.0])
def test_masked_target(dtype, vocab, side, smoothing):
    import paper_2507_11941_amd as bpe

    lens, beta, scale = [3, 4, 2, 5], 0.5, 4.0
    ends = np.concatenate([[0], np.cumsum(lens)])
    n = int(ends[-1])
    x, t = some_logits(n, vocab, TYPES[dtype], 1), torch.arange(n, dtype=torch.int32) % vocab
    row = int(ends[2 + side])                            # the second pair's: the preferred string's first row, or the other's
    x[row, int(t[row])] = -INF
    lp, _ = ref.logprobs(x, t)
    z = [beta * (lp[ends[k]:ends[k + 1]].sum() - lp[ends[k + 1]:ends[k + 2]].sum()).item() for k in (0, 2)]
    assert z[1] == (INF if side else -INF)

    def term(v):                                         # -log sigmoid(v)
        return 0.0 if v == INF else INF if v == -INF else float(np.logaddexp(0.0, -v))

    want = [sum(w * term(s * v) for w, s in ((1 - smoothing, 1), (smoothing, -1)) if w > 0) for v in z]
    slope = [smoothing - 1 / (1 + np.exp(v)) for v in z]
    loss, margins, got_lp, grad = bpe.preference_loss(x, t.to(dev()), torch.from_numpy(ends).to(dev()), None, beta, smoothing, scale)
    far = beta * n * LOG_SUM
    assert_near(got_lp, lp, LOG_SUM, "logprobs")
    assert_near(margins, torch.tensor(z, dtype=torch.float64), far, "margins")
    assert_near(loss, torch.tensor(sum(want) / 2, dtype=torch.float64), far + 4 * U, "loss")
    upstream = torch.cat([torch.full((int(ends[i + 1] - ends[i]),), (1 - i % 2 * 2) * scale * beta / 2 * slope[i // 2], dtype=torch.float64)
                          for i in range(4)])
    want_grad, off = ref.logits_grad(x, t, upstream)
    assert_near(grad, want_grad, off + scale * beta / 2 * far / 4 + 4 * U * upstream.abs()[:, None], "gradient")
