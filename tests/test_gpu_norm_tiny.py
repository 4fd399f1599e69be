"""Norms of rows whose reciprocal root is beyond the 32-bit numbers, or among those that hold fewer bits, against 64 bits: with eps = 0 the norm of
the smallest numbers is as ordinary as that of any others."""
import pytest
import torch

import head_reference as ref
from ops_reference import TYPES, assert_near
from test_gpu_norm import dev, matrix

pytestmark = pytest.mark.gpu

# of a row's largest element; a row of 2^-149 has a few whole multiples of the smallest 32-bit number
SIZES = [2.0 ** e for e in (-149, -147, -140, -133, -130, -128, -127, -126, -120, -110, -102, -101, -100, -99, -98, -64, 0, 62, 64, 98, 100, 102, 120, 126, 127)]


@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("dim", [1, 37, 700, 1500, 6000, 20000])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_of_all_sizes_without_eps(dtype, dim, residual):
    import paper_2507_11941_amd as bpe

    base = matrix(len(SIZES), dim, torch.float32, 5).cpu().double()
    base = (base / base.abs().amax(1, keepdim=True) * torch.tensor(SIZES, dtype=torch.float64)[:, None]).to(TYPES[dtype])
    base = torch.where(base.float().abs().amax(1, keepdim=True) > 0, base, torch.ones_like(base))      # (bfloat16 has no 2^-149)
    for repeats in (1, 50):                              # few rows, and more than a thousand
        x = base.repeat(repeats, 1).to(dev())
        if repeats > 1 and dim > 1500:
            continue
        more = torch.zeros_like(x) if residual else None
        for weight in (torch.linspace(0.5, 2, dim, device=dev()), torch.full((dim,), 2.0 ** 60, device=dev())):
            y, total, rstd = bpe.add_norm(x, weight, more, 0.0)
            assert torch.equal(total, x)
            want, root = ref.norm(x, weight, 0.0)
            assert_near(y, want, (ref.ROOT + 2 * ref.U) * want.abs(), f"norm of {dim}")
            # (a factor beyond the 32-bit numbers is infinite: from 2^128 - 2^103 on, half a step above the largest, 2^128 - 2^104)
            beyond = root >= 2.0 ** 128 - 2.0 ** 103
            assert bool(beyond.any()) and bool(torch.isinf(rstd.cpu()[beyond]).all())
            assert_near(rstd.cpu()[~beyond], root[~beyond], ref.ROOT * root[~beyond], "factor")


@pytest.mark.parametrize("dim", [40, 20000])
def test_rows_of_zeros_and_odd_rows_are_as_they_were(dim):
    """A row of zeros has no norm without an eps; infinities and NaN are not hidden."""
    import paper_2507_11941_amd as bpe

    x = torch.zeros(4, dim, device=dev())
    x[1], x[2], x[3] = 1e-44, 3e38, 1e-44
    x[1, 3], x[2, 4], x[3, 5] = float("inf"), -float("inf"), float("nan")
    y, _, rstd = bpe.add_norm(x, torch.ones(dim, device=dev()), None, 0.0)
    assert bool(torch.isnan(y[0]).all()) and bool(torch.isnan(y[3]).all()) and bool(torch.isinf(rstd[0]))
    for row, at in ((1, 3), (2, 4)):                     # the formula's: 0, and infinity times 0
        assert bool(torch.isnan(y[row, at])) and not y[row].nan_to_num().any() and float(rstd[row]) == 0.0
    y, _, _ = bpe.add_norm(x, torch.ones(dim, device=dev()))
    assert not y[0].any()


@pytest.mark.parametrize("dim", [37, 1500, 20000])
def test_in_place(dim):
    """The norm in the place of x, and of the residual with the sum in that of x."""
    import paper_2507_11941_amd as bpe

    x = matrix(len(SIZES), dim, torch.float32, 5).cpu().double()
    x = (x / x.abs().amax(1, keepdim=True) * torch.tensor(SIZES, dtype=torch.float64)[:, None]).float().to(dev())
    weight, zeros = torch.linspace(0.5, 2, dim, device=dev()), torch.zeros_like(x)
    want = bpe.add_norm(x, weight, None, 0.0)[0]
    a = x.clone()
    assert torch.equal(bpe.add_norm(a, weight, None, 0.0, out=a)[0], want)
    a, b = x.clone(), zeros.clone()
    got, total, _ = bpe.add_norm(a, weight, b, 0.0, out=b, summed=a)
    assert torch.equal(got, want) and torch.equal(total, x)
