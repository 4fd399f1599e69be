"""The embedding's gradient of a token that occurs millions of times: what is added late is not lost."""
import pytest
import torch

from ops_reference import HALF_ULP, TYPES, U

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,n,dim", [("f32", 1 << 22, 9), ("bf16", (1 << 22) + 77, 24), ("f16", 3000001, 7), ("bf16", 1 << 24, 3)])
def test_equal_rows(dtype, n, dim):
    """All rows alike, so that roundings do not cancel: up to 31 additions of a chunk round by U / 2 of half the chunk's sum on average,
    8 U, those of 32 pieces by 8 U, and 64 bits round nothing to speak of; the scale and the result round by U each."""
    import paper_2507_11941_amd as bpe

    dev = torch.device("cuda:0")
    x = torch.tensor(0.7, dtype=TYPES[dtype])
    grad = torch.full((n, dim), x.item(), dtype=TYPES[dtype], device=dev)
    ids = torch.full((n,), 5, dtype=torch.int32, device=dev)
    ids[::7] = 3
    got = bpe.embed_tokens_grad(grad, ids, 8, 2.0 ** -8, dtype=torch.float32).double()
    threes = (n + 6) // 7
    for token, many in ((3, threes), (5, n - threes)):
        want = many * x.double().item() * 2.0 ** -8
        assert ((got[token] - want).abs() <= want * (16 + 4) * U).all(), token
    got[[3, 5]] = 0
    assert not got.any()
    start = torch.full((8, dim), 1.0, device=dev)
    bpe.embed_tokens_grad(grad, ids, 8, 2.0 ** -8, out=start, accumulate=True)
    want = 1 + (n - threes) * x.double().item() * 2.0 ** -8
    assert ((start[5].double() - want).abs() <= want * ((16 + 4) * U + HALF_ULP[torch.float32])).all()
