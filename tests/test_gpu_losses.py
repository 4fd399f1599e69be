"""next_tokens, the preference loss and the policy loss against 64 bits (their gradients by differentiating the formulas, and
against differences): strings without a scored token, empty ones, rows outside every string, values that nobody may read,
clipping on both sides, weights by token and by string."""
import numpy as np
import pytest
import torch

import ops_reference as ref
from ops_reference import LOG_SUM, TYPES, U, assert_near
from test_gpu_logits import dev, some_logits

pytestmark = pytest.mark.gpu


def batch_of(lens, vocab, seed, before=0, after=0, prompts=True):
    """(ids, offsets, first) on the host; `before` and `after`: rows that are in no string."""
    rng = np.random.default_rng(seed)
    offsets = np.concatenate([[0], np.cumsum(lens)]).astype(np.int64) + before
    ids = rng.integers(0, vocab, offsets[-1] + after).astype(np.int32)
    first = np.array([rng.integers(-1, n + 2) if prompts else 0 for n in lens], dtype=np.int32)
    return ids, offsets, first


def up(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(dev())


@pytest.mark.parametrize("lens,before,after", [([], 0, 0), ([], 0, 5), ([0, 0], 0, 0), ([1], 0, 0), ([2], 0, 0), ([1, 0, 2, 0, 0, 3], 2, 4),
                                               ([500, 0, 1, 700, 3], 0, 300), ([7] * 600, 1, 0), ([70000], 0, 1)])
def test_next_tokens(lens, before, after):
    import paper_2507_11941_amd as bpe

    for prompts in (False, True):
        ids, offsets, first = batch_of(lens, 1000, 1, before, after, prompts)
        got = bpe.next_tokens(up(ids), up(offsets), up(first) if prompts else None)
        assert np.array_equal(got.cpu().numpy(), ref.next_tokens(ids, offsets, first if prompts else None))




PAIRS = [[3, 4], [0, 5], [1, 1], [0, 0], [40, 7, 300, 512, 1, 0, 2, 2], [900, 1100], [5000, 3, 0, 2600], [2049, 700]]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [11, 1256, 33000])
@pytest.mark.parametrize("lens", PAIRS, ids=str)
def test_preference(dtype, vocab, lens):
    import paper_2507_11941_amd as bpe

    if sum(lens) * vocab > 1 << 24:
        lens = [n // 16 for n in lens]
    ids, offsets, first = batch_of(lens, vocab, 3, 2, 3)
    n = len(ids)
    x = some_logits(n, vocab, TYPES[dtype], 1, vocab + 1, 1)
    targets = bpe.next_tokens(up(ids), up(offsets), up(first))
    targets[0] = 1                                        # scored, but in no string
    t = targets.cpu()
    lp, _ = ref.logprobs(x, t)
    reference = (lp + torch.randn(n, generator=torch.Generator().manual_seed(5)).double()).float()
    for refs, beta, smoothing, scale in ((reference, 0.1, 0.0, 1.0), (None, 0.05, 0.1, 1.0), (reference, 2.0, 0.3, 256.0)):
        beta, smoothing = float(np.float32(beta)), float(np.float32(smoothing))
        leaf = lp.clone().requires_grad_()
        want_loss, want_z = ref.preference(leaf, t, offsets, vocab, refs, beta, smoothing)
        want_loss.backward()
        upstream = leaf.grad * scale
        given = None if refs is None else refs.clone()
        if given is not None:
            given[(t < 0)] = float("nan")                 # not read
        y = x.clone()
        y[(t < 0).to(dev())] = float("nan")
        y = torch.as_strided(y, x.shape, y.stride())
        loss, margins, got_lp, grad = bpe.preference_loss(y, targets, up(offsets), None if given is None else given.to(dev()), beta, smoothing, scale)
        want_grad, off = ref.logits_grad(x, t, upstream)
        # a margin adds up one error for each of its tokens
        far = beta * max(1, sum(lens)) * LOG_SUM
        assert_near(got_lp, lp, LOG_SUM, "logprobs")
        assert_near(margins, want_z.detach(), far, "margins")
        assert_near(loss, want_loss.detach(), far + 4 * U, "loss")
        # the slope changes by a quarter of the margin's error at most
        slope = scale * beta / (len(lens) // 2) * far / 4
        assert_near(grad, want_grad, off + slope + 4 * U * upstream.abs()[:, None], "gradient")
        assert (grad[targets < 0] == 0).all() and (grad[0] == 0).all()


def test_preference_without_pairs():
    import paper_2507_11941_amd as bpe

    for n in (0, 5):
        x, targets = torch.full((n, 7), 2.0, device=dev()), torch.zeros(n, dtype=torch.int32, device=dev())
        loss, margins, lp, grad = bpe.preference_loss(x, targets, torch.zeros(1, dtype=torch.int64, device=dev()))
        assert loss.item() == 0 and margins.shape == (0,) and not grad.any()
        assert_near(lp, ref.logprobs(x, targets)[0], LOG_SUM)


def test_preference_of_far_apart_strings():
    """Margins of thousands: the loss grows with them and neither overflows nor becomes NaN."""
    import paper_2507_11941_amd as bpe

    n, vocab = 4000, 64
    x = torch.zeros(n, vocab, device=dev())
    targets = torch.zeros(n, dtype=torch.int32, device=dev())
    x[:2000, 1], x[2000:, 0] = 60.0, 60.0
    offsets = up(np.array([0, 2000, 4000]))
    for turn in (1.0, -1.0):
        loss, margins, _, grad = bpe.preference_loss(x, targets, offsets, None, turn)
        assert_near(margins, torch.tensor([turn * -120000.0]), 4000 * LOG_SUM + 120000 * U)
        assert_near(loss, torch.tensor(120000.0 if turn > 0 else 0.0), 4000 * LOG_SUM + 120000 * U)
        assert torch.isfinite(grad).all() and bool(grad.any()) == (turn > 0)


POLICIES = [[5], [3, 4, 0, 1], [0, 0], [64, 300, 1, 2, 700], [900], [1500, 3, 0, 1100, 1024], [1500, 3, 0, 0, 1, 2, 1100, 1],
            [9000, 2, 0, 4097, 63], [2049, 64, 65]]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [13, 1256, 33000])
@pytest.mark.parametrize("lens", POLICIES, ids=str)
def test_policy(dtype, vocab, lens):
    import paper_2507_11941_amd as bpe

    if sum(lens) * vocab > 1 << 24:
        lens = [n // 16 for n in lens]
    ids, offsets, first = batch_of(lens, vocab, 4, 1, 2)
    n, batch = len(ids), len(lens)
    x = some_logits(n, vocab, TYPES[dtype], 1, vocab + 3, 2)
    targets = bpe.next_tokens(up(ids), up(offsets), up(first))
    targets[0] = 1
    t = targets.cpu()
    lp, _ = ref.logprobs(x, t)
    g = torch.Generator().manual_seed(6)
    away = 0.4 * torch.randn(n, generator=g).double()
    low, high, kl = (float(np.float32(v)) for v in (0.2, 0.28, 0.05))
    for bound in (1 - low, 1 + high):                     # no ratio within 1e-3 of a bound, where there is no derivative
        away = torch.where((away.exp() - bound).abs() < 1e-3, 0.0, away)
    old = (lp - away).float()
    reference = (lp + 0.5 * torch.randn(n, generator=g).double()).float()
    for per, whole, refs, scale in (("token", False, None, 1.0), ("string", True, reference, 1.0), ("token", True, reference, 512.0),
                                    ("string", False, None, 3.0)):
        if whole and batch == n:
            continue
        advantages = torch.randn(batch if whole else n, generator=g)
        at = ref.strings_of(n, offsets).clamp(min=0)
        leaf = lp.clone().requires_grad_()
        want_loss = ref.policy(leaf, t, offsets, vocab, old, advantages[at] if whole else advantages, refs, low, high, kl, per == "string")
        upstream = torch.zeros_like(lp)
        if want_loss.requires_grad:
            want_loss.backward()
            upstream = leaf.grad * scale
        dead = (t < 0)
        hide = [v.clone() if v is not None else None for v in (old, refs, None if whole else advantages)]
        for v in hide:
            if v is not None:
                v[dead] = float("nan")                    # not read
        y = x.clone()
        y[dead.to(dev())] = float("inf")
        loss, got_lp, grad = bpe.policy_loss(y, targets, up(offsets), hide[0].to(dev()), (advantages if whole else hide[2]).to(dev()),
                                             None if refs is None else hide[1].to(dev()), low, high, kl, per, scale)
        inside = ((t >= 0) & (ref.strings_of(n, offsets) >= 0))
        assert_near(got_lp, torch.where(inside, lp, 0.0), LOG_SUM, "logprobs")
        # A token's loss and its slope are ratio x A and the KL term's: relative errors of LOG_SUM for the log-probability and 8 U for
        # exponentials, products and the weight.  Weights add up to 1 (no advantage here is above 5, no ratio above 8).
        size = 5 * 8 + kl * 8
        assert_near(loss, want_loss.detach(), size * (LOG_SUM + 8 * U), "loss")
        share = torch.zeros(n, dtype=torch.float64)
        for i in range(batch):
            rows = inside & (ref.strings_of(n, offsets) == i)
            share[rows] = 1 / (batch * max(1, int(rows.sum()))) if per == "string" else 1 / max(1, int(inside.sum()))
        want_grad, off = ref.logits_grad(x, t, upstream)
        assert_near(grad, want_grad, off + (scale * share * size * (LOG_SUM + 8 * U))[:, None], "gradient")
        assert (grad[targets < 0] == 0).all() and (grad[0] == 0).all()


def test_policy_by_hand():
    """Two logits, one token: p = 1/2, and every branch of the clipped term."""
    import paper_2507_11941_amd as bpe

    x, targets = torch.zeros(1, 2, device=dev()), torch.zeros(1, dtype=torch.int32, device=dev())
    offsets = torch.tensor([0, 1], device=dev())
    for ratio, advantage, value, slope in ((1.0, 2.0, -2.0, -2.0), (2.0, 1.0, -1.25, 0.0), (2.0, -1.0, 2.0, 2.0), (0.5, 1.0, -0.5, -0.5),
                                           (0.5, -1.0, 0.75, 0.0), (1.125, -4.0, 4.5, 4.5), (0.875, 0.0, 0.0, 0.0)):
        old = torch.tensor([np.log(0.5) - np.log(ratio)], dtype=torch.float32, device=dev())
        loss, lp, grad = bpe.policy_loss(x, targets, offsets, old, torch.tensor([advantage], device=dev()), clip_low=0.25, clip_high=0.25)
        assert abs(loss.item() - value) <= 16 * U * max(1, abs(value)) and abs(lp.item() - np.log(0.5)) <= 4 * U
        assert abs(grad[0, 0].item() - slope / 2) <= 16 * U * max(1, abs(slope)) and grad[0, 1].item() == -grad[0, 0].item()
    loss, _, grad = bpe.policy_loss(x, targets, offsets, torch.tensor([np.log(0.5)], dtype=torch.float32, device=dev()), torch.zeros(1, device=dev()),
                                    torch.tensor([np.log(0.5) + np.log(2.0)], dtype=torch.float32, device=dev()), kl_weight=0.5)
    assert abs(loss.item() - 0.5 * (2 - np.log(2) - 1)) <= 16 * U and abs(grad[0, 0].item() - 0.5 * (1 - 2) / 2) <= 16 * U


def test_policy_with_nothing_scored():
    import paper_2507_11941_amd as bpe

    for n, ends in ((0, [0]), (0, [0, 0, 0]), (6, [0]), (6, [0, 3, 6])):
        x = torch.full((n, 9), float("nan"), dtype=torch.bfloat16, device=dev())
        rest = torch.full((n,), float("nan"), device=dev())
        for per in ("token", "string"):
            loss, lp, grad = bpe.policy_loss(x, torch.full((n,), -1, dtype=torch.int32, device=dev()), torch.tensor(ends, device=dev()), rest, rest,
                                             rest, kl_weight=0.1, per=per)
            assert loss.item() == 0 and not lp.any() and not grad.any()


def test_losses_against_differences():
    """The gradients against central differences of the losses themselves, over a step of 2^-5 in each logit.  Third derivatives
    of either loss along a logit are below 4; each loss is off by 40 U at most."""
    import paper_2507_11941_amd as bpe

    vocab, lens = 5, [4, 3]
    ids, offsets, _ = batch_of(lens, vocab, 9, prompts=False)
    x, targets = some_logits(len(ids), vocab, torch.float32, 2, spread=1.0), bpe.next_tokens(up(ids), up(offsets))
    lp = bpe.token_logprobs(x, targets)[0]
    old, reference, advantages = lp - 0.03, lp + 0.2, torch.tensor([1.0, -0.5], device=dev())
    losses = (lambda y: bpe.preference_loss(y, targets, up(offsets), reference, 0.5, 0.1),
              lambda y: bpe.policy_loss(y, targets, up(offsets), old, advantages, reference, 0.5, 0.5, 0.1, "string"))
    h = 2.0 ** -5
    for f in losses:
        grad = f(x)[-1].cpu()
        for r in range(len(ids)):
            for j in range(vocab):
                values = []
                for step in (h, -h):
                    y = x.clone()
                    y[r, j] += step
                    values.append(f(y)[0].double().item())
                far = 4 * h * h / 6 + (80 * U + LOG_SUM * sum(lens)) / (2 * h)
                assert abs((values[0] - values[1]) / (2 * h) - grad[r, j].item()) <= far


@pytest.mark.parametrize("loss", ["preference", "policy"])
def test_in_place_again_on_another_stream_and_in_a_graph(loss):
    import paper_2507_11941_amd as bpe

    vocab, lens = 1256, [50, 31, 0, 40]
    ids, offsets, first = batch_of(lens, vocab, 9, 0, 3)
    n = len(ids)
    x, targets, ends = some_logits(n, vocab, torch.bfloat16, 2), bpe.next_tokens(up(ids), up(offsets), up(first)), up(offsets)
    lp = bpe.token_logprobs(x, targets)[0]
    old, advantages = lp + 0.1, torch.randn(4, device=dev())

    def f(y, **more):
        if loss == "preference":
            return bpe.preference_loss(y, targets, ends, old, **more)
        return bpe.policy_loss(y, targets, ends, old, advantages, old, kl_weight=0.1, per="string", **more)

    want = f(x)
    assert all(torch.equal(a, b) for a, b in zip(want, f(x))), "not the same bits again"
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = f(x, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got)), "on another stream"
    y = x.clone()
    assert all(torch.equal(a, b) for a, b in zip(want, f(y, out=y))), "in place"
    graph, y = torch.cuda.CUDAGraph(), x.clone()
    with torch.cuda.graph(graph):
        captured = f(y)
    for seed in (5, 6, 7):
        y.copy_(some_logits(n, vocab, torch.bfloat16, seed))
        for t in captured:
            t.fill_(7.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(f(y), captured)), "replayed"


def test_refusals():
    import paper_2507_11941_amd as bpe

    x, targets, u = some_logits(4, 10, torch.float32, 1), torch.zeros(4, dtype=torch.int32, device=dev()), torch.zeros(4, device=dev())
    two, three = torch.tensor([0, 2, 4], device=dev()), torch.tensor([0, 1, 2, 4], device=dev())
    for bad in (lambda: bpe.preference_loss(x, targets, three), lambda: bpe.preference_loss(x, targets, two.int()), lambda: bpe.preference_loss(x, targets, two, u[:2]),
                lambda: bpe.preference_loss(x, targets, two[:0]), lambda: bpe.preference_loss(x, targets, two, u.double()),
                lambda: bpe.preference_loss(x, targets, two, smoothing=1.5), lambda: bpe.preference_loss(x, targets, two, beta=float("nan")),
                lambda: bpe.policy_loss(x, targets, two, u, u[:3]), lambda: bpe.policy_loss(x, targets, two, u[:3], u), lambda: bpe.policy_loss(x, targets, two, u, u, per="batch"),
                lambda: bpe.policy_loss(x, targets, two, u, u, clip_low=-0.1), lambda: bpe.policy_loss(x, targets, two, u, u, kl_weight=-1.0),
                lambda: bpe.next_tokens(targets.long(), two), lambda: bpe.next_tokens(targets, two, targets[:1]), lambda: bpe.next_tokens(targets, two, out=targets[:2]),
                lambda: bpe.policy_loss(x, targets, two, u, u, out=torch.empty(4, 9, device=dev()))):
        with pytest.raises((ValueError, bpe.BpeError)):
            bad()
    torch.cuda.synchronize()
