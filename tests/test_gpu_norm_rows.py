"""The norms' plans that depend on the number of rows, against 64 bits: one wave with four vectors a lane for a thousand rows and more, launches of
2^21 rows, and the gradient with several rows a workgroup of every size."""
import pytest
import torch

import head_reference as ref
from ops_reference import TYPES, assert_near
from test_gpu_norm import EPS, check_norm, dev, matrix

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [999, 1000, 1003])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_a_thousand_rows(dtype, n):
    """On both sides of the number from which a row has one wave, and of the widths that one wave holds."""
    import paper_2507_11941_amd as bpe

    T = TYPES[dtype]
    for dim in (259, 260, 387, 520, 1027, 1028) if dtype == "f32" else (519, 520, 700, 1029, 2048, 2055, 2056):
        print(dim, flush=True)
        for weight_dtype in {torch.float32, T}:
            check_norm(n, dim, T, weight_dtype, dim % 2 == 0, spread=dim % 3, at=dim % 2)
        x = matrix(n, dim, T, dim, 3, 1)
        q, scales = bpe.quantize_rows(x)
        want, factor = ref.rows_8bit(x.cpu().double(), torch.ones(n, dtype=torch.float64))
        assert torch.equal(q.cpu(), want)
        assert_near(scales, factor, 2 * ref.U * factor, "scales")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_thousand_rows_write_nothing_else(dtype):
    import paper_2507_11941_amd as bpe

    n, dim, T = 1003, 701, TYPES[dtype]
    x, more = matrix(n, dim, T, 1), matrix(n, dim, T, 2)
    weight = matrix(1, dim, T, 3).reshape(-1)
    y, total, _ = bpe.add_norm(x, weight, more, EPS)
    room, room2 = (torch.full((n + 2, dim + 3), 5.0, dtype=T, device=dev()) for _ in range(2))
    out, kept = room[1:-1, 1:dim + 1], room2[1:-1, 2:dim + 2]
    bpe.add_norm(x, weight, more, EPS, out=out, summed=kept)
    assert torch.equal(out, y) and torch.equal(kept, total)
    out.fill_(5.0), kept.fill_(5.0)
    assert bool((room == 5.0).all()) and bool((room2 == 5.0).all())
    a, b = x.clone(), more.clone()                       # in place
    got, kept, _ = bpe.add_norm(a, weight, b, EPS, out=a, summed=b)
    assert torch.equal(got, y) and torch.equal(kept, total)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_rows_of_extreme_sizes_among_a_thousand(dtype):
    """Rows that are summed again in 64 bits, zeros and odd rows, where a row has one wave."""
    import paper_2507_11941_amd as bpe

    T = TYPES[dtype]
    n, dim = 1001, 700
    base = matrix(n, dim, torch.float32, 5).cpu()
    base = base / base.abs().amax(1, keepdim=True)
    base[0] = 0.0
    if dtype != "f16":
        base[1] *= 1e-25
        base[2] *= 2e37
    base[3, 5], base[4, 7] = float("inf"), float("nan")
    x = base.to(T).to(dev())
    weight = torch.linspace(0.5, 2, dim, device=dev())
    fine = torch.tensor([i for i in range(n) if i not in (3, 4)])
    y, _, rstd = bpe.add_norm(x, weight, None, EPS)
    want, root = ref.norm(x, weight, EPS)
    assert_near(rstd.cpu()[fine], root[fine], ref.ROOT * root[fine], "factor")
    assert_near(y.cpu()[fine], want[fine], (ref.ROOT + 2 * ref.U) * want[fine].abs(), "norm")
    assert bool(torch.isnan(y.float()).any(1)[3:5].all())
    q, scales, _ = bpe.add_norm_8bit(x, weight, None, EPS)
    want_q, factor = ref.rows_8bit(x.cpu().double() * weight.cpu().double(), root)
    assert torch.equal(q.cpu(), want_q)
    assert_near(scales, factor, (ref.ROOT + 2 * ref.U) * factor + 2.0 ** -149, "scales")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_more_rows_than_one_launch_has(dtype):
    """About the row with which the second launch begins, and all rows against those of calls that are one launch each."""
    import paper_2507_11941_amd as bpe

    n, dim, T = 2 ** 21 + 9, 3, TYPES[dtype]
    g = torch.Generator(device=dev()).manual_seed(1)
    x, more = (torch.randn(n, dim, generator=g, device=dev()).to(T) for _ in range(2))
    weight = torch.tensor([0.5, 1.0, 3.0], device=dev())
    y, total, rstd = bpe.add_norm(x, weight, more, EPS)
    q, scales, _ = bpe.add_norm_8bit(x, weight, more, EPS)
    rows, row_scales = bpe.quantize_rows(x)
    for some in (slice(0, 7), slice(2 ** 21 - 7, n)):
        s = ref.summed(x[some], more[some])
        want, root = ref.norm(s, weight, EPS)
        assert torch.equal(total[some].cpu(), s)
        assert_near(y[some], want, (ref.ROOT + 2 * ref.U) * want.abs(), "norm")
        assert_near(rstd[some], root, ref.ROOT * root, "factor")
        want, factor = ref.rows_8bit(s.double() * weight.cpu().double(), root)
        assert torch.equal(q[some].cpu(), want)
        assert_near(scales[some], factor, (ref.ROOT + 2 * ref.U) * factor, "scales")
        want, factor = ref.rows_8bit(x[some].cpu().double(), torch.ones(len(want), dtype=torch.float64))
        assert torch.equal(rows[some].cpu(), want)
        assert_near(row_scales[some], factor, 2 * ref.U * factor, "scales")
    for some in (slice(0, 2 ** 20), slice(2 ** 20, n)):
        again = bpe.add_norm(x[some], weight, more[some], EPS)
        assert torch.equal(again[0], y[some]) and torch.equal(again[1], total[some]) and torch.equal(again[2], rstd[some])
        again = bpe.quantize_rows(x[some])
        assert torch.equal(again[0], rows[some]) and torch.equal(again[1], row_scales[some])


# threads of the gradient's workgroups: 64, 128, 256, 512, 1,024 in 32 bits; one vector a lane and elements behind whole vectors
@pytest.mark.parametrize("dtype,dim", [("f32", 255), ("f32", 515), ("f32", 1024), ("f32", 1027), ("f32", 2049), ("f32", 4096), ("f32", 4099),
                                       ("bf16", 1031), ("bf16", 2050), ("f16", 2048), ("bf16", 4097), ("bf16", 8199)])
def test_gradients_of_several_rows_a_workgroup(dtype, dim):
    import paper_2507_11941_amd as bpe

    T = TYPES[dtype]
    for n in (513, 1100, 4100):                          # two, three and five rows of a workgroup, the last ones fewer
        if n * dim > 10_000_000 and dim % 2 == 0:
            continue
        print(n, flush=True)
        s, g, more = (matrix(n, dim, T, seed, seed, 1) for seed in (1, 2, 3))
        weight = matrix(1, dim, torch.float32, 4).reshape(-1)
        _, _, rstd = bpe.add_norm(s, weight, None, EPS)
        (to_x, off), (to_weight, off_weight) = ref.norm_grad(g, s, weight, rstd, more)
        to_x = ref.in_range(to_x, T)
        got, got_weight = bpe.add_norm_grad(g, s, weight, rstd, more)
        assert_near(got, to_x, off, "gradient of x")
        assert_near(got_weight, to_weight, off_weight, "gradient of the weights")
        for _ in range(3):
            again = bpe.add_norm_grad(g, s, weight, rstd, more)
            assert torch.equal(again[0], got) and torch.equal(again[1], got_weight)
        in_place = g.clone()
        bpe.add_norm_grad(in_place, s, weight, rstd, more, out=in_place)
        assert torch.equal(in_place, got)


@pytest.mark.parametrize("dim", [9, 261])
def test_gradients_of_the_most_rows_a_workgroup(dim):
    """More rows than 1,024 workgroups have with 256 each, of one wave and of two."""
    import paper_2507_11941_amd as bpe

    n = 2 ** 18 + 777
    g, s = (torch.randn(n, dim, generator=torch.Generator(device=dev()).manual_seed(seed), device=dev()) for seed in (1, 2))
    weight = torch.linspace(0.5, 2, dim, device=dev())
    _, _, rstd = bpe.add_norm(s, weight, None, EPS)
    got, got_weight = bpe.add_norm_grad(g, s, weight, rstd)
    h = s.double() * rstd.double()[:, None]
    to_weight, size = (g * h).sum(0).cpu(), (g * h).abs().sum(0).cpu()
    assert_near(got_weight, to_weight, 260 * ref.U * size, "gradient of the weights")
    for some in (slice(0, 600), slice(2 ** 18 - 300, n)):
        (to_x, off), _ = ref.norm_grad(g[some], s[some], weight, rstd[some])
        assert_near(got[some], to_x, off, "gradient of x")
