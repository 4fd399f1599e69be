"""The norm's gradient where the weights want none: the same gradient of x, and nothing computed for the weights."""
import pytest
import torch

from ops_reference import TYPES
from test_gpu_norm import EPS, dev, matrix

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,dim", [(0, 5), (1, 1), (7, 130), (1100, 387), (20, 2048), (3, 4099), (5, 9001), (600, 16400)])
def test_without_the_weights_gradient(n, dim, dtype):
    """Rows that a workgroup's registers hold, and rows that none does."""
    import paper_2507_11941_amd as bpe

    T = TYPES[dtype]
    s, g, more = (matrix(n, dim, T, seed, 3, 1) for seed in (1, 2, 3))
    weight = matrix(1, dim, T, 4).reshape(-1)
    _, _, rstd = bpe.add_norm(s, weight, None, EPS)
    for extra in (None, more):
        want, _ = bpe.add_norm_grad(g, s, weight, rstd, extra)
        got, none = bpe.add_norm_grad(g, s, weight, rstd, extra, weights=False)
        assert none is None and torch.equal(got, want)
        in_place = g.clone()
        assert bpe.add_norm_grad(in_place, s, weight, rstd, extra, out=in_place, weights=False) == (in_place, None)
        assert torch.equal(in_place, want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got, none = bpe.add_norm_grad(g, s, weight, rstd, more, weights=False, stream=side)
    torch.cuda.synchronize()
    assert none is None and torch.equal(got, want)


@pytest.mark.parametrize("dim", [40, 9001])
def test_backward_pass_of_a_frozen_weight(dim, monkeypatch):
    import paper_2507_11941_amd as bpe
    from paper_2507_11941_amd import _head

    n = 6
    x, more, g, gs = (matrix(n, dim, torch.float32, seed) for seed in (1, 2, 3, 4))
    weight = matrix(1, dim, torch.float32, 5).reshape(-1)
    wanted, original = [], _head.add_norm_grad
    monkeypatch.setattr(_head, "add_norm_grad", lambda *a, **k: wanted.append(k["weights"]) or original(*a, **k))
    results = []
    for frozen in (False, True):
        leaves = [x.clone().requires_grad_(), weight.clone().requires_grad_(not frozen), more.clone().requires_grad_()]
        y, total, _ = bpe.add_norm(*leaves, EPS)
        torch.autograd.backward([y, total], [g, gs])
        assert (leaves[1].grad is None) == frozen
        results.append((leaves[0].grad, leaves[2].grad))
    assert wanted == [True, False]
    assert all(torch.equal(a, b) for a, b in zip(*results))


def test_refusals():
    import paper_2507_11941_amd as bpe

    x, w, v = torch.zeros(4, 6, device=dev()), torch.ones(6, device=dev()), torch.ones(4, device=dev())
    for more in (dict(out_weight=w.clone()), dict(dtype=torch.float32), dict(accumulate=True), dict(workspace=torch.zeros(1 << 20, dtype=torch.uint8, device=dev()))):
        with pytest.raises(ValueError, match="weights' gradient"):
            bpe.add_norm_grad(x, x, w, v, weights=False, **more)
