"""Penalties, biases and masks on logits, and their gradient, against 64 bits."""
import math

import pytest
import torch

import head_reference as ref
from ops_reference import TYPES, assert_near

pytestmark = pytest.mark.gpu


def dev():
    return torch.device("cuda:0")


def logits_of(n, vocab, dtype, seed, spread=0, at=0):
    g = torch.Generator().manual_seed(seed)
    room = torch.full((n * (vocab + spread) + at,), 9.0, dtype=dtype, device=dev())
    view = room[at:].as_strided((n, vocab), (vocab + spread, 1))
    view.copy_(torch.randn(n, vocab, generator=g) * 3)
    return view


def histories(n, vocab, longest, seed, padded=True):
    """Packed histories of 0 to `longest` tokens, few tokens often; ids outside the vocabulary among them."""
    g = torch.Generator().manual_seed(seed)
    lens = torch.randint(0, longest + 1, (n,), generator=g)
    if n > 1:
        lens[0] = 0
    ends = lens.cumsum(0)
    ids = (torch.rand(int(ends[-1]), generator=g) ** 3 * vocab).to(torch.int32)
    if padded and len(ids):
        ids[torch.rand(len(ids), generator=g) < 0.1] = -1
        ids[torch.rand(len(ids), generator=g) < 0.05] = vocab
        ids[torch.rand(len(ids), generator=g) < 0.05] = 2 ** 31 - 1
        ids[torch.rand(len(ids), generator=g) < 0.05] = -2 ** 31
    return ids.to(dev()), (ends - lens).to(dev()), ends.to(dev())


def biases(n, vocab, longest, seed):
    """Lists of 0 to `longest` biases, tokens named twice among them."""
    ids, begin, end = histories(n, vocab, longest, seed)
    return ids, torch.randn(len(ids), generator=torch.Generator().manual_seed(seed)).to(dev()) * 4, begin, end


def masks(states, n, vocab, seed):
    g = torch.Generator().manual_seed(seed)
    words = (vocab + 31) // 32
    mask = torch.randint(-2 ** 31, 2 ** 31, (states, words), generator=g, dtype=torch.int64).to(torch.int32)
    mask[0] = 0                                          # nothing left
    if states > 1:
        mask[1] = -1                                     # everything
    if states > 2:
        mask[2] = 0
        mask[2, words // 2] = 1 << 7
    state = torch.randint(-2, states + 2, (n,), generator=g, dtype=torch.int32)
    return mask.to(dev()), state.to(dev())


def penalties_of(n, seed):
    g = torch.Generator().manual_seed(seed)
    return (torch.rand(n, 3, generator=g) * torch.tensor([1.0, 2.0, 0.5]) + torch.tensor([0.6, -0.5, -0.1])).to(dev())


FORMS = ["penalties", "rows", "bias", "mask", "all", "nothing", "lists"]


def arguments(form, n, vocab, seed, longest=40):
    history = histories(n, vocab, longest, seed)
    own, listed = penalties_of(n, seed + 1), biases(n, vocab, 12, seed + 2)
    mask, state = masks(5, n, vocab, seed + 3)
    return {"penalties": dict(ids=history[0], begin=history[1], end=history[2], penalties=(1.25, 0.5, 0.25)),
            "rows": dict(ids=history[0], begin=history[1], end=history[2], penalties=own),
            "bias": dict(bias=listed), "mask": dict(mask=mask, state=state), "nothing": {},
            "lists": dict(ids=history[0], begin=history[1], end=history[2], penalties=own, bias=listed),
            "all": dict(ids=history[0], begin=history[1], end=history[2], penalties=own, bias=listed, mask=mask, state=state)}[form]


def without_bias(more):
    return {k: v for k, v in more.items() if k != "bias"}


def check(logits, more, seed):
    import paper_2507_11941_amd as bpe

    n, vocab = logits.shape
    want, off = ref.adjust(logits, **more)
    got = bpe.adjust_logits(logits, **more)
    assert got is not logits
    assert_near(got, want, off, "adjusted")
    same = torch.empty_strided(logits.shape, logits.stride(), dtype=logits.dtype, device=dev()).copy_(logits)
    before = same._version
    assert bpe.adjust_logits(same, **more, out=same) is same and same._version > before
    assert torch.equal(same.isnan(), got.isnan()) and torch.equal(same.nan_to_num(0.0, math.inf, -math.inf), got.nan_to_num(0.0, math.inf, -math.inf))
    grad = logits_of(n, vocab, logits.dtype, seed)
    want, off = ref.adjust_grad(grad, logits, **without_bias(more))
    got = bpe.adjust_logits_grad(grad, logits, **without_bias(more))
    assert_near(got, want, off, "gradient")
    assert bpe.adjust_logits_grad(grad, logits, **without_bias(more), out=grad) is grad and torch.equal(grad, got)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("form", FORMS)
def test_adjusted(form, dtype):
    for n, vocab in ((1, 1), (3, 2), (4, 7), (5, 31), (4, 32), (6, 33), (9, 100), (5, 1256), (3, 4095), (3, 4096), (3, 4097), (4, 10001)):
        print(n, vocab, flush=True)
        check(logits_of(n, vocab, TYPES[dtype], n), arguments(form, n, vocab, vocab), 8)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_views(dtype):
    for n, vocab, spread, at in ((5, 1256, 3, 1), (4, 999, 1, 0), (3, 5000, 60, 3)):
        check(logits_of(n, vocab, TYPES[dtype], n, spread, at), arguments("all", n, vocab, vocab), 8)


@pytest.mark.parametrize("longest", [300, 5000, 70000])
def test_long_histories(longest):
    n, vocab = 3, 9000
    more = arguments("all", n, vocab, 5, longest)
    more["begin"][2], more["end"][2] = 0, len(more["ids"])           # all of it
    check(logits_of(n, vocab, torch.float32, 1), more, 2)
    # one token throughout
    ids = torch.full((longest,), 4321, dtype=torch.int32, device=dev())
    bounds = torch.tensor([0, 1, longest - 1], device=dev()), torch.tensor([longest, longest - 1, longest], device=dev())
    check(logits_of(n, vocab, torch.float32, 1), dict(ids=ids, begin=bounds[0], end=bounds[1], penalties=(1.5, 0.0, 2.0 ** -10)), 2)


def test_bounds_that_overlap_or_lie_outside():
    n, vocab = 8, 500
    ids = histories(4, vocab, 60, 3)[0]
    k = len(ids)
    begin = torch.tensor([0, 0, 5, -9, 7, k, k + 5, 2 ** 40], device=dev())
    end = torch.tensor([k, 10, 4, 3, k + 100, k, k + 9, 2 ** 41], device=dev())
    logits = logits_of(n, vocab, torch.float32, 1)
    check(logits, dict(ids=ids, begin=begin, end=end, penalties=(2.0, 1.0, 0.5)), 2)
    values = torch.randn(k, device=dev())
    check(logits, dict(bias=(ids, values, begin, end)), 2)
    none = torch.empty(0, dtype=torch.int32, device=dev())
    zero = torch.zeros(n, dtype=torch.int64, device=dev())
    check(logits, dict(ids=none, begin=zero, end=zero + 3, penalties=(2.0, 1.0, 0.5)), 2)


def test_prefixes_of_packed_strings():
    """Each position of a batch with what is before it in its string."""
    offsets = torch.tensor([0, 0, 40, 41, 90])
    n, vocab = 90, 64
    ids = torch.randint(0, vocab, (n,), generator=torch.Generator().manual_seed(1), dtype=torch.int32).to(dev())
    begin = offsets[torch.searchsorted(offsets, torch.arange(n), right=True) - 1].to(dev())
    check(logits_of(n, vocab, torch.bfloat16, 1), dict(ids=ids, begin=begin, end=torch.arange(n, device=dev()), penalties=(1.5, 0.5, 0.25)), 2)


def test_masks_without_a_state():
    n, vocab = 6, 300
    mask, _ = masks(6, n, vocab, 1)
    logits = logits_of(n, vocab, torch.bfloat16, 1)
    check(logits, dict(mask=mask), 2)
    check(logits, dict(mask=mask[3:4]), 2)
    wide = torch.full((6, mask.shape[1] + 3), -1, dtype=torch.int32, device=dev())
    wide[:, :mask.shape[1]] = mask
    check(logits, dict(mask=wide[:, :mask.shape[1]]), 2)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_what_logits_may_hold(dtype):
    """Infinities, NaN and the type's lowest value: kept where they are allowed, -inf where they are not; their gradient is a number."""
    import paper_2507_11941_amd as bpe

    T = TYPES[dtype]
    low = torch.finfo(T).min
    odd = [math.inf, -math.inf, math.nan, 0.0, -0.0, low, torch.finfo(T).max, torch.finfo(T).tiny]
    logits = torch.tensor([odd * 5] * 4, dtype=T, device=dev())
    ids = torch.arange(0, 24, dtype=torch.int32, device=dev())
    bounds = torch.zeros(4, dtype=torch.int64, device=dev()), torch.tensor([0, 24, 24, 24], device=dev())
    mask = torch.tensor([[-1, -1], [0x00ff00ff, 0xff], [0, 0]], dtype=torch.int32, device=dev())
    state = torch.tensor([0, 0, 1, 2], dtype=torch.int32, device=dev())
    check(logits, dict(ids=ids, begin=bounds[0], end=bounds[1], penalties=(1.0, 0.0, 0.0), mask=mask, state=state), 3)
    got = bpe.adjust_logits(logits, mask=mask, state=state)
    assert torch.equal(got[3], torch.full_like(got[3], -math.inf))
    grad = torch.full_like(logits, math.nan)
    assert not bpe.adjust_logits_grad(grad, logits, mask=mask, state=state)[3].any()


def test_gradients_against_differences():
    n, vocab = 3, 40
    logits = logits_of(n, vocab, torch.float32, 1).cpu().double()
    more = {k: v.cpu() for k, v in arguments("rows", n, vocab, 3).items()}
    mask, state = masks(4, n, vocab, 3)
    more.update(mask=mask.cpu(), state=torch.tensor([1, 3, -1], dtype=torch.int32))
    grad = logits_of(n, vocab, torch.float32, 2).cpu().double()
    want, _ = ref.adjust_grad(grad, logits, **more)
    keep = ref.allowed(n, vocab, more["mask"], more["state"])
    for i, j in ((0, 0), (1, 3), (2, 1), (2, 39), (1, 20)):
        ends = []
        for d in (1e-6, -1e-6):
            x = logits.clone()
            x[i, j] += d
            ends.append((torch.where(keep, ref.adjust(x, **more)[0], 0.0) * grad).sum())
        assert abs((ends[0] - ends[1]) / 2e-6 - want[i, j]) < 1e-5 * (1 + abs(want[i, j]))


def test_automatic_differentiation():
    import paper_2507_11941_amd as bpe

    n, vocab = 5, 700
    more = arguments("all", n, vocab, 4)
    logits, grad = logits_of(n, vocab, torch.float32, 1), logits_of(n, vocab, torch.float32, 2)
    leaf = logits.clone().requires_grad_()
    got = bpe.adjust_logits(leaf, **more)
    assert got.requires_grad and torch.equal(got, bpe.adjust_logits(logits, **more))
    got.backward(grad)
    assert torch.equal(leaf.grad, bpe.adjust_logits_grad(grad, logits, **without_bias(more)))
    with pytest.raises(ValueError):
        bpe.adjust_logits(leaf, **more, out=torch.empty_like(logits))
    with pytest.raises(ValueError):
        bpe.adjust_logits(logits, **{**more, "penalties": more["penalties"].clone().requires_grad_()})
    with pytest.raises(ValueError):
        bias = more["bias"]
        bpe.adjust_logits(logits, **{**more, "bias": (bias[0], bias[1].clone().requires_grad_(), bias[2], bias[3])})
    # the policy's loss on what its answers were drawn from, and on to the logits themselves
    targets = torch.tensor([3, -1, 5, 699, 0], dtype=torch.int32, device=dev())
    leaf.grad = None
    adjusted = bpe.adjust_logits(leaf, more["ids"], more["begin"], more["end"], (1.25, 0.5, 0.0))
    zeros = torch.zeros(n, device=dev())
    _, _, to_adjusted = bpe.policy_loss(adjusted, targets, torch.tensor([0, n], device=dev()), zeros, zeros + 1)
    adjusted.backward(to_adjusted)
    assert torch.equal(leaf.grad, bpe.adjust_logits_grad(to_adjusted, logits, more["ids"], more["begin"], more["end"], (1.25, 0.5, 0.0)))
    got = bpe.adjust_logits(leaf, **more)
    more["ids"][:1] = 3
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        got.backward(grad)


def test_nothing_else_is_written():
    import paper_2507_11941_amd as bpe

    for vocab in (40, 5001):
        n = 6
        more = arguments("all", n, vocab, 4)
        logits = logits_of(n, vocab, torch.bfloat16, 1)
        room = torch.full((n + 2, vocab + 3), 5.0, dtype=torch.bfloat16, device=dev())
        out = room[1:-1, 1:vocab + 1]
        assert bpe.adjust_logits(logits, **more, out=out) is out
        assert torch.equal(out, bpe.adjust_logits(logits, **more))
        out.fill_(5.0)
        assert bool((room == 5.0).all())
        out.copy_(logits)
        bpe.adjust_logits(out, **more, out=out)
        assert torch.equal(out, bpe.adjust_logits(logits, **more))
        out.fill_(5.0)
        assert bool((room == 5.0).all())
    assert bpe.adjust_logits(logits[:0]).shape == (0, vocab)
