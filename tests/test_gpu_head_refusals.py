"""What the binding of the operators at a model's output end refuses: ValueError, before anything is enqueued."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_refusals():
    import paper_2507_11941_amd as bpe

    dev = torch.device("cuda:0")
    x, w, v = torch.zeros(4, 6, device=dev), torch.ones(6, device=dev), torch.zeros(4, device=dev)
    half = x.to(torch.bfloat16)
    q, head, head_scales = torch.zeros(4, 6, dtype=torch.int8, device=dev), torch.zeros(9, 6, dtype=torch.int8, device=dev), torch.zeros(9, device=dev)
    ids, at = torch.zeros(5, dtype=torch.int32, device=dev), torch.zeros(4, dtype=torch.int64, device=dev)
    logits, mask = torch.zeros(4, 70, device=dev), torch.zeros(4, 3, dtype=torch.int32, device=dev)
    one = torch.zeros(4, dtype=torch.int32, device=dev)
    for bad in (
            lambda: bpe.add_norm(x.double(), w), lambda: bpe.add_norm(x[0], w), lambda: bpe.add_norm(x.t(), w), lambda: bpe.add_norm(x[:, :5], w),
            lambda: bpe.add_norm(x, w.cpu()), lambda: bpe.add_norm(x, w.half()), lambda: bpe.add_norm(x, w[::2]), lambda: bpe.add_norm(x, w, half),
            lambda: bpe.add_norm(x, w, x[:3]), lambda: bpe.add_norm(x, w, summed=x), lambda: bpe.add_norm(x, w, out=half), lambda: bpe.add_norm(x, w, out=x[:3]),
            lambda: bpe.add_norm(x, w, x.cpu()), lambda: bpe.add_norm(x.new_zeros(4, 0), w),
            lambda: bpe.add_norm_8bit(x, w, summed=x), lambda: bpe.add_norm_8bit(x.expand(4, 6)[:1].expand(4, 6), w), lambda: bpe.quantize_rows(q),
            lambda: bpe.add_norm_grad(x, half, w, v), lambda: bpe.add_norm_grad(x, x, w, v[:3]), lambda: bpe.add_norm_grad(x, x, w, v.double()),
            lambda: bpe.add_norm_grad(x, x, w, v, dtype=torch.float16), lambda: bpe.add_norm_grad(x, x, w, v, accumulate=True),
            lambda: bpe.add_norm_grad(x, x, w, v, out_weight=w, dtype=torch.bfloat16), lambda: bpe.add_norm_grad(x, x, w, v, out_weight=w[:5]),
            lambda: bpe.add_norm_grad(x, x, w, v, workspace=torch.zeros(8, dtype=torch.uint8, device=dev)), lambda: bpe.add_norm_grad(x, x, w, v, half),
            lambda: bpe.project_8bit(x, v, head, head_scales), lambda: bpe.project_8bit(q, v, head[:, :5], head_scales),
            lambda: bpe.project_8bit(q, v[:3], head, head_scales), lambda: bpe.project_8bit(q, v, head, head_scales[:8]),
            lambda: bpe.project_8bit(q, v, head, head_scales, torch.float64), lambda: bpe.project_8bit(q, v, head.cpu(), head_scales),
            lambda: bpe.project_8bit(q, v, head, head_scales, torch.float32, logits[:, :9].half()), lambda: bpe.project_8bit(q, v, head, head_scales, out=logits),
            lambda: bpe.project_8bit(q, v, head[:0], head_scales[:0]),
            lambda: bpe.project_8bit(torch.zeros(1, 131072, dtype=torch.int8, device=dev), v[:1], torch.zeros(1, 131072, dtype=torch.int8, device=dev), v[:1]),
            lambda: bpe.adjust_logits(logits, ids), lambda: bpe.adjust_logits(logits, ids, at), lambda: bpe.adjust_logits(logits, ids, at, at[:3]),
            lambda: bpe.adjust_logits(logits, ids.long(), at, at), lambda: bpe.adjust_logits(logits, ids, at.int(), at),
            lambda: bpe.adjust_logits(logits, ids, at, at, torch.ones(4, 2, device=dev)), lambda: bpe.adjust_logits(logits, ids, at, at, torch.ones(3, 3, device=dev)),
            lambda: bpe.adjust_logits(logits, ids, at, at, (1.0, 0.0)), lambda: bpe.adjust_logits(logits, bias=(ids, v, at, at)),
            lambda: bpe.adjust_logits(logits, bias=(ids, torch.zeros(5, device=dev), at, at[:3])), lambda: bpe.adjust_logits(logits, mask=mask[:, :2]),
            lambda: bpe.adjust_logits(logits, mask=mask.long()), lambda: bpe.adjust_logits(logits, mask=mask[:3]), lambda: bpe.adjust_logits(logits, state=one),
            lambda: bpe.adjust_logits(logits, mask=mask, state=one[:3]), lambda: bpe.adjust_logits(logits, mask=mask[:0], state=one),
            lambda: bpe.adjust_logits(logits, mask=mask.t().contiguous().t()), lambda: bpe.adjust_logits(logits, out=logits[:3]),
            lambda: bpe.adjust_logits_grad(logits, logits[:3]), lambda: bpe.adjust_logits_grad(logits, logits.half()),
            lambda: bpe.adjust_logits_grad(logits, logits, mask=mask, out=logits.half())):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: bpe.add_norm(x, w, None, -1.0), lambda: bpe.add_norm(x, w, None, float("nan")), lambda: bpe.adjust_logits(logits, ids, at, at, (0.0, 0.0, 0.0)),
                lambda: bpe.adjust_logits(logits, ids, at, at, (1.0, float("inf"), 0.0))):
        with pytest.raises(bpe.BpeError):
            bad()
    for empty in (bpe.add_norm(x[:0], w)[0], bpe.add_norm_8bit(x[:0], w)[0], bpe.quantize_rows(x[:0])[0], bpe.add_norm_grad(x[:0], x[:0], w, v[:0])[0]):
        assert empty.shape == (0, 6)
    assert not bpe.add_norm_grad(x[:0], x[:0], w, v[:0])[1].any()
