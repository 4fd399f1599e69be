"""include/bpe_head.h: the library exports what it declares, and refuses bad arguments before it touches a device."""
import os
import re

import pytest
import torch

import paper_2507_11941_amd as bpe
from paper_2507_11941_amd import _head

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
EINVAL = -1
A = 1 << 20                                              # an address that is aligned to everything and never followed
BIG = 1 << 40


def test_library_exports_every_declared_symbol():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "bpe_head.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(bpe_[a-z_0-9]+)\s*\(", text)))
    assert len(names) == 8
    for name in names:
        assert hasattr(bpe.load_library(), name), name


def call(name, good, bad):
    """Whether each of the changes `bad` ({argument: value}) of the arguments `good` is refused."""
    function = getattr(_head._load(), "bpe_" + name)
    for at, value in bad:
        args = {**good, at: value} if isinstance(at, str) else {**good, **dict(zip(at, value))}
        assert list(args) == list(good)
        assert function(*args.values()) == EINVAL, (name, at, value)


nan, inf = float("nan"), float("inf")
NORM = dict(x=A, dtype=1, n=4, dim=7, stride=7, residual=A, residual_stride=7, weight=A, weight_dtype=0, eps=1e-6, summed=A + 4096, summed_stride=7)
BAD_NORM = [("x", None), ("x", A + 1), ("dtype", 3), ("dtype", -1), ("n", -1), ("n", BIG), ("dim", 0), ("dim", BIG), ("stride", 6), ("stride", BIG),
            ("residual", None), ("residual", A + 1), ("residual_stride", 6), ("weight", None), ("weight", A + 2), ("weight_dtype", 2),
            ("weight_dtype", 5), ("eps", -1.0), ("eps", nan), ("eps", inf), ("summed", None), ("summed", A + 1), ("summed_stride", 6)]


def test_norm_arguments():
    call("add_norm", dict(NORM, rstd=A, out=A, out_stride=7, stream=None), [*BAD_NORM, ("rstd", A + 2), ("out", None), ("out", A + 1), ("out", A + 4096), ("out_stride", 6)])
    call("add_norm_8bit", dict(NORM, q=A, q_stride=7, scales=A, stream=None),
         [*BAD_NORM, ("q", None), ("q_stride", 6), ("q_stride", BIG), ("scales", None), ("scales", A + 2)])
    call("quantize_rows", dict(x=A, dtype=1, n=4, dim=7, stride=7, q=A, q_stride=7, scales=A, stream=None),
         [*BAD_NORM[:10], ("q", None), ("q_stride", 6), ("scales", None), ("scales", A + 1)])
    good = dict(grad=A, dtype=1, n=4, dim=7, grad_stride=7, summed=A, summed_stride=7, weight=A, weight_dtype=0, rstd=A, more=None, more_stride=0,
                grad_x=A, grad_x_stride=7, grad_weight=A, grad_weight_dtype=0, accumulate=0, workspace=A, workspace_bytes=1 << 20, stream=None)
    call("add_norm_grad", good,
         [("grad", None), ("grad", A + 1), ("dtype", 3), ("n", -1), ("n", BIG), ("dim", 0), ("dim", BIG), ("grad_stride", 6), ("summed", None),
          ("summed_stride", 6), ("weight", None), ("weight", A + 2), ("weight_dtype", 2), ("rstd", None), ("rstd", A + 2), (("more", "more_stride"), (A, 6)),
          (("more", "more_stride"), (A + 1, 7)), ("grad_x", None), ("grad_x_stride", 6), ("grad_weight", A + 2), ("grad_weight_dtype", 1),
          ("workspace", None), ("workspace", A + 128), ("workspace_bytes", 0)])
    lib = _head._load()
    for n, dim in ((-1, 5), (5, 0), (1 << 30, 5), (5, BIG)):
        assert lib.bpe_add_norm_grad_workspace_bytes(n, dim) == 0
    for n in (0, 1, 1000, 10 ** 6):
        assert lib.bpe_add_norm_grad_workspace_bytes(n, 513) >= 513 * 4


def test_product_arguments():
    good = dict(q=A, n=4, dim=7, q_stride=7, scales=A, weight=A, vocab=9, weight_stride=7, weight_scales=A, out=A, dtype=1, out_stride=9, stream=None)
    call("project_8bit", good,
         [("q", None), ("n", -1), ("n", BIG), ("dim", 0), ("dim", 131072), ("q_stride", 6), ("q_stride", BIG), ("scales", None), ("scales", A + 2),
          ("weight", None), ("vocab", 0), ("vocab", BIG), ("weight_stride", 6), ("weight_scales", None), ("weight_scales", A + 1), ("out", None),
          ("out", A + 1), ("dtype", 4), ("out_stride", 8), (("n", "vocab", "out_stride"), ((1 << 30) - 1, 1 << 28, 1 << 28))])
    assert _head._load().bpe_project_8bit(*{**good, "n": 0, "q": None, "scales": None, "out": None}.values()) == 0


LOGITS = dict(logits=A, dtype=1, n=4, vocab=40, stride=40)
BAD_LOGITS = [("logits", None), ("logits", A + 1), ("dtype", 3), ("n", -1), ("n", BIG), ("vocab", 0), ("vocab", BIG), ("stride", 39)]
HISTORY = dict(ids=A, n_ids=9, begin=A, end=A, penalties=None, repetition=1.5)
BAD_HISTORY = [("ids", None), ("ids", A + 2), ("n_ids", -1), ("n_ids", BIG), ("begin", None), ("end", None), ("begin", A + 4), ("end", A + 4),
               ("penalties", A + 1), ("repetition", 0.0), ("repetition", -1.0), ("repetition", nan), ("repetition", inf)]
MASK = dict(mask=A, states=3, mask_stride=2, state=A)
BAD_MASK = [("mask", A + 2), ("states", 0), ("states", -1), ("states", BIG), ("mask_stride", 1), ("mask_stride", BIG), ("state", A + 1), ("state", None)]
OUT = dict(out=A + 4096, out_stride=40, stream=None)
BAD_OUT = [("out", None), ("out", A + 1), ("out_stride", 39), (("out", "out_stride"), (A, 41))]


def test_adjustment_arguments():
    good = dict(LOGITS, **HISTORY, presence=0.0, frequency=0.0, bias_ids=A, bias_values=A, n_biases=5, bias_begin=A, bias_end=A, **MASK, **OUT)
    call("adjust_logits", good,
         [*BAD_LOGITS, *BAD_HISTORY, ("presence", nan), ("presence", inf), ("frequency", nan), ("bias_ids", None), ("bias_ids", A + 1),
          ("bias_values", None), ("bias_values", A + 2), ("n_biases", -1), ("bias_begin", None), ("bias_end", None), ("bias_begin", A + 4), *BAD_MASK,
          *BAD_OUT])
    good = dict(LOGITS, from_=A, from_stride=40, **HISTORY, **MASK, **OUT)
    call("adjust_logits_grad", good, [*BAD_LOGITS, ("from_", None), ("from_", A + 1), ("from_stride", 39), *BAD_HISTORY, *BAD_MASK, *BAD_OUT])
    assert _head._load().bpe_adjust_logits_grad(*{**good, "n": 0, "logits": None, "from_": None, "out": None}.values()) == 0


def test_tensors_that_are_not_on_the_gpu_are_refused():
    x, v = torch.zeros(3, 5), torch.zeros(3)
    q = torch.zeros(3, 5, dtype=torch.int8)
    for bad in (lambda: bpe.add_norm(x, x[0]), lambda: bpe.add_norm_8bit(x, x[0]), lambda: bpe.quantize_rows(x), lambda: bpe.add_norm_grad(x, x, x[0], v),
                lambda: bpe.project_8bit(q, v, q, v), lambda: bpe.adjust_logits(x), lambda: bpe.adjust_logits_grad(x, x)):
        with pytest.raises(ValueError):
            bad()
