"""Norms of sums with the residual, into their type and into 8 bits, rows into 8 bits and the norm's gradient, against 64 bits."""
import math

import pytest
import torch

import head_reference as ref
from ops_reference import TYPES, assert_near

pytestmark = pytest.mark.gpu

EPS = 2.0 ** -20


def dev():
    return torch.device("cuda:0")


def matrix(rows, columns, dtype, seed, spread=0, at=0):
    """Numbers of different sizes, as a view with `spread` columns between rows, `at` elements behind an aligned address."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, columns, generator=g) * torch.exp(torch.randn(columns, generator=g)) * torch.exp(torch.randn(rows, 1, generator=g))
    room = torch.full((rows * (columns + spread) + at,), 7.0, dtype=dtype, device=dev())
    view = room[at:].as_strided((rows, columns), (columns + spread, 1))
    view.copy_(x)
    return view


# rows that a wave, a workgroup and no workgroup holds; one element; behind whole vectors
DIMS = [1, 2, 3, 7, 8, 9, 64, 255, 256, 257, 387, 511, 513, 1000, 1024, 2047, 2048, 2051, 4096, 4099, 8192, 8200]
LONG = [8193, 16384, 16397, 40001]


def check_norm(n, dim, dtype, weight_dtype, residual, spread=0, at=0):
    import paper_2507_11941_amd as bpe

    x = matrix(n, dim, dtype, 1, spread, at)
    more = matrix(n, dim, dtype, 2, spread // 2, at) if residual else None
    weight = matrix(1, dim, weight_dtype, 3).reshape(-1)
    s = ref.summed(x, more)
    want, root = ref.norm(s, weight, EPS)
    y, total, rstd = bpe.add_norm(x, weight, more, EPS)
    assert torch.equal(total.cpu(), s) and (residual or total is x)
    assert_near(rstd, root, ref.ROOT * root, "factor")
    assert_near(y, want, (ref.ROOT + 2 * ref.U) * want.abs(), "norm")
    q, scales, total = bpe.add_norm_8bit(x, weight, more, EPS)
    want, factor = ref.rows_8bit(s.double() * weight.cpu().double(), root)
    assert torch.equal(total.cpu(), s)
    assert torch.equal(q.cpu(), want)
    assert_near(scales, factor, (ref.ROOT + 2 * ref.U) * factor, "scales")


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("residual", [False, True])
def test_norms(dtype, residual):
    for dim in DIMS + LONG:
        print(dim, flush=True)
        for weight_dtype in {torch.float32, TYPES[dtype]}:
            check_norm(5 if dim < 5000 else 2, dim, TYPES[dtype], weight_dtype, residual)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_norms_of_views(dtype):
    for n, dim, spread, at in ((1, 387, 0, 1), (33, 387, 4, 3), (3, 1024, 1, 0), (300, 64, 64, 1), (2, 9001, 3, 1), (2, 16500, 3, 1)):
        print(n, dim, flush=True)
        check_norm(n, dim, TYPES[dtype], TYPES[dtype], True, spread, at)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_rows_in_8_bits(dtype):
    import paper_2507_11941_amd as bpe

    for dim in DIMS + LONG:
        x = matrix(4, dim, TYPES[dtype], dim, 3, 1)
        q, scales = bpe.quantize_rows(x)
        want, factor = ref.rows_8bit(x.cpu().double(), torch.ones(4, dtype=torch.float64))
        assert torch.equal(q.cpu(), want), dim
        assert_near(scales, factor, 2 * ref.U * factor, "scales")
        assert q.stride(0) % 16 == 0 and q.stride(1) == 1


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_ties_and_borders_in_8_bits(dtype):
    """Values half-way between two integers go to the even one, also where 32 bits cannot tell them from their neighbours."""
    import paper_2507_11941_amd as bpe

    halves = torch.arange(-254, 255, dtype=torch.float32) / 2                  # the largest is 127: quotients are the values themselves
    x = torch.stack([halves, halves / 64, halves * 3]).to(TYPES[dtype]).to(dev())
    q, scales = bpe.quantize_rows(x)
    want, factor = ref.rows_8bit(x.cpu().double(), torch.ones(3, dtype=torch.float64))
    assert torch.equal(q.cpu(), want)
    if dtype == "f32":
        assert int((halves[want[0].double() != halves.double()] % 1 == 0.5).sum()) == 254
        near = torch.nextafter(halves, torch.full_like(halves, math.inf)).clamp(max=127)
        x = torch.stack([near, -near, near / 7]).to(dev())
        want, _ = ref.rows_8bit(x.cpu().double(), torch.ones(3, dtype=torch.float64))
        assert torch.equal(bpe.quantize_rows(x)[0].cpu(), want)
    weight = torch.full((x.shape[1],), 3.0, device=dev())
    q, _, _ = bpe.add_norm_8bit(x, weight)
    want, _ = ref.rows_8bit(x.cpu().double() * 3.0, torch.ones(3, dtype=torch.float64))
    assert torch.equal(q.cpu(), want)


@pytest.mark.parametrize("dim", [37, 1500, 20000])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_without_a_norm_and_of_extreme_sizes(dtype, dim):
    import paper_2507_11941_amd as bpe

    base = matrix(10, dim, torch.float32, 5).cpu()
    base = base / base.abs().amax(1, keepdim=True)
    base[0] = 0.0
    base[1] *= 1e-25
    base[2] *= 2e37
    base[3, 5] = math.inf
    base[4, 7] = math.nan
    base[5, 8] = -math.inf
    base[6] *= 1e-38
    base[7] *= 1e19
    x = base.to(TYPES[dtype]).to(dev())
    for eps in (EPS, 0.0):
        weight = torch.linspace(0.5, 2, dim, device=dev())
        weight64 = weight.cpu().double()
        y, _, rstd = bpe.add_norm(x, weight, None, eps)
        want, root = ref.norm(x, weight, eps)
        # (with eps = 0 a row of zeros has no norm, and the factor of one of the smallest numbers is beyond the 32-bit range)
        ordinary = torch.tensor([i for i in range(10) if i not in (3, 4, 5) and (eps > 0 or i not in (0, 6))])
        assert_near(rstd[ordinary.to(dev())], root[ordinary], ref.ROOT * root[ordinary], "factor")
        if eps > 0:
            assert_near(y[ordinary.to(dev())], want[ordinary], (ref.ROOT + 2 * ref.U) * want[ordinary].abs(), "norm")
        assert bool(torch.isnan(y.float()).any(1)[3:6].all())
        q, scales, _ = bpe.add_norm_8bit(x, weight, None, eps)
        want_q, factor = ref.rows_8bit(x.cpu().double() * weight64, root)
        assert torch.equal(q.cpu()[ordinary], want_q[ordinary])
        assert_near(scales[ordinary.to(dev())], factor[ordinary], (ref.ROOT + 2 * ref.U) * factor[ordinary] + 2.0 ** -149, "scales")
        assert not q[3:6].any() and bool(torch.isnan(scales[3:6]).all())
    q, scales = bpe.quantize_rows(x)
    want_q, factor = ref.rows_8bit(x.cpu().double(), torch.ones(10, dtype=torch.float64))
    assert torch.equal(q.cpu(), want_q)
    assert_near(scales, factor, 2 * ref.U * factor + 2.0 ** -149, "scales")
    weight = torch.ones(dim, device=dev())
    weight[3] = math.nan
    q, scales, _ = bpe.add_norm_8bit(x, weight)
    assert not q.any() and bool(torch.isnan(scales).all())


@pytest.mark.parametrize("dtype,weight_dtype", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f16", "f32"), ("f16", "f16")])
def test_gradients(dtype, weight_dtype):
    import paper_2507_11941_amd as bpe

    T, W = TYPES[dtype], TYPES[weight_dtype]
    for n, dim, spread, at in ((1, 1, 0, 0), (2, 7, 1, 1), (5, 64, 0, 0), (700, 387, 3, 1), (1100, 512, 0, 0), (3, 2048, 0, 0), (9, 4099, 1, 0),
                               (5, 8192, 0, 0), (2, 8200, 0, 0), (3, 16400, 1, 1), (600, 16400, 0, 0)):
        print(n, dim, flush=True)
        s, g, more = (matrix(n, dim, T, seed, spread, at) for seed in (1, 2, 3))
        weight = matrix(1, dim, W, 4).reshape(-1)
        _, _, rstd = bpe.add_norm(s, weight, None, EPS)
        for extra in (None, more):
            (to_x, off), (to_weight, off_weight) = ref.norm_grad(g, s, weight, rstd, extra)
            to_x = ref.in_range(to_x, T)                 # (a float16 element of 86,404 +- 42 is infinite)
            for kind in {torch.float32, W}:
                got, got_weight = bpe.add_norm_grad(g, s, weight, rstd, extra, dtype=kind)
                assert_near(got, to_x, off, "gradient of x")
                assert got_weight.dtype == kind
                assert_near(got_weight, to_weight, off_weight, "gradient of the weights")
        # added to what there is, and in place of either gradient
        total = matrix(1, dim, W, 5).reshape(-1)
        before = total.clone()
        in_place = g.clone()
        got, got_weight = bpe.add_norm_grad(in_place, s, weight, rstd, more, out=in_place, out_weight=total, accumulate=True)
        assert got is in_place and got_weight is total
        assert_near(in_place, to_x, off, "in place of the norm's gradient")
        assert_near(total, to_weight + before.cpu().double(), off_weight + ref.U * before.cpu().double().abs(), "accumulated")
        in_place = more.clone()
        bpe.add_norm_grad(g, s, weight, rstd, in_place, out=in_place)
        assert_near(in_place, to_x, off, "in place of the sum's gradient")


def test_gradient_of_very_many_weights():
    """More columns than one launch has workgroups for: the weights' gradient about the borders of the launches that join it."""
    import paper_2507_11941_amd as bpe

    dim = 2 ** 28 + 65
    g = torch.arange(dim, dtype=torch.int32, device=dev()).remainder_(251).sub_(125).to(torch.bfloat16).view(1, dim)
    s = torch.arange(dim, dtype=torch.int32, device=dev()).remainder_(241).sub_(120).to(torch.bfloat16).view(1, dim)
    weight = torch.ones(dim, dtype=torch.bfloat16, device=dev())
    rstd = torch.full((1,), 0.0078125, device=dev())
    for accumulate in (False, True):
        total = torch.full((dim,), 3.0, device=dev())
        bpe.add_norm_grad(g, s, weight, rstd, out_weight=total, accumulate=accumulate)
        for begin in (0, 2 ** 27 - 70, 2 ** 28 - 70, dim - 70):
            some = slice(begin, begin + 70)
            # (products of two integers of at most 7 bits and a power of two, and 3 more: exact in 32 bits)
            want = g[0, some].double() * s[0, some].double() * 0.0078125 + (3.0 if accumulate else 0.0)
            assert torch.equal(total[some].double(), want), (accumulate, begin)


def test_gradients_against_differences():
    """The formula's gradient in 64 bits, which the kernels' is compared with, against differences of the norm's formula."""
    g, x, w = (matrix(3, 17, torch.float32, seed).cpu().double() for seed in (1, 2, 3))
    w = w[0]
    _, root = ref.norm(x, w, EPS)
    (to_x, _), (to_weight, _) = ref.norm_grad(g, x, w, root)
    step = 1e-6
    for i, j in ((0, 0), (1, 5), (2, 16)):
        for which, want in ((0, to_x[i, j]), (1, to_weight[j])):
            ends = []
            for d in (step, -step):
                y, v = x.clone(), w.clone()
                if which == 0:
                    y[i, j] += d
                else:
                    v[j] += d
                ends.append((ref.norm(y, v, EPS)[0] * g).sum())
            assert abs((ends[0] - ends[1]) / (2 * step) - want) < 1e-5 * (1 + abs(want))


@pytest.mark.parametrize("dim", [40, 3000, 20001])
def test_nothing_else_is_written_and_places_may_be_shared(dim):
    import paper_2507_11941_amd as bpe

    n, T = 6, torch.bfloat16
    x, more = matrix(n, dim, T, 1), matrix(n, dim, T, 2)
    weight = matrix(1, dim, T, 3).reshape(-1)
    y, total, rstd = bpe.add_norm(x, weight, more, EPS)
    room, room2 = (torch.full((n + 2, dim + 3), 5.0, dtype=T, device=dev()) for _ in range(2))
    out, kept = room[1:-1, 1:dim + 1], room2[1:-1, 2:dim + 2]
    bpe.add_norm(x, weight, more, EPS, out=out, summed=kept)
    assert torch.equal(out, y) and torch.equal(kept, total)
    out.fill_(5.0), kept.fill_(5.0)
    assert bool((room == 5.0).all()) and bool((room2 == 5.0).all())
    for take in (0, 1):                                  # the sum in place of the residual or of x, the norm in place of the other
        a, b = x.clone(), more.clone()
        places = (b, a) if take == 0 else (a, b)
        got, kept, _ = bpe.add_norm(a, weight, b, EPS, out=places[1], summed=places[0])
        assert torch.equal(got, y) and torch.equal(kept, total)
    a = x.clone()
    alone, _, _ = bpe.add_norm(x, weight, None, EPS)
    assert torch.equal(bpe.add_norm(a, weight, None, EPS, out=a)[0], alone)
    b = more.clone()
    q, scales, kept = bpe.add_norm_8bit(x, weight, b, EPS, summed=b)
    assert kept is b and torch.equal(b, total)
    again = bpe.add_norm_8bit(x, weight, more, EPS)
    assert torch.equal(q, again[0]) and torch.equal(scales, again[1])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("residual", [False, True])
def test_automatic_differentiation(dtype, residual):
    import paper_2507_11941_amd as bpe

    n, dim = 7, 130
    x, more, g, gs = (matrix(n, dim, dtype, seed) for seed in (1, 2, 3, 4))
    weight = matrix(1, dim, torch.float32, 5).reshape(-1)
    _, s, rstd = bpe.add_norm(x, weight, more if residual else None, EPS)
    want, want_weight = bpe.add_norm_grad(g, s, weight, rstd, gs if residual else None)
    leaves = [t.clone().requires_grad_() for t in ((x, weight, more) if residual else (x, weight))]
    y, total, factor = bpe.add_norm(leaves[0], leaves[1], leaves[2] if residual else None, EPS)
    assert y.requires_grad and not factor.requires_grad and (residual or total is leaves[0])
    if residual:
        torch.autograd.backward([y, total], [g, gs])
        assert torch.equal(leaves[2].grad, want)
    else:
        y.backward(g.t().contiguous().t())               # (a gradient that lies by columns)
    assert torch.equal(leaves[0].grad, want) and torch.equal(leaves[1].grad, want_weight)
    if residual:                                         # only the sum is used
        leaves = [t.clone().requires_grad_() for t in (x, weight, more)]
        bpe.add_norm(leaves[0], leaves[1], leaves[2], EPS)[1].backward(gs)
        assert torch.equal(leaves[0].grad, gs) and torch.equal(leaves[2].grad, gs) and leaves[1].grad is None
    with pytest.raises(ValueError):
        bpe.add_norm(leaves[0], leaves[1], out=torch.empty_like(x))
    with pytest.raises(ValueError):
        bpe.add_norm_8bit(leaves[0], weight)
    with pytest.raises(ValueError):
        bpe.quantize_rows(leaves[0])
    with torch.no_grad():
        assert not bpe.add_norm(leaves[0], leaves[1])[0].requires_grad
        bpe.add_norm_8bit(leaves[0], weight)
    y, total, _ = bpe.add_norm(leaves[0], leaves[1], leaves[2] if residual else None, EPS)
    with torch.no_grad():
        leaves[1].mul_(2.0)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward(g)
