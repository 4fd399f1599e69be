"""include/bpe_head.h: an output in the place of an input has to lie as that does; the norms refuse it with other strides, as the adjustment does."""
from test_head_abi import A, NORM, call

FAR = A + (1 << 16)


def test_norms_in_the_place_of_an_input():
    good = dict(NORM, residual=A + (1 << 15), summed=FAR, rstd=None, out=FAR + (1 << 15), out_stride=7, stream=None)
    x, residual = good["x"], good["residual"]
    both = [(("summed", "summed_stride"), (x, 8)), (("summed", "summed_stride"), (residual, 9)), (("stride", "summed"), (8, x)),
            (("residual_stride", "summed"), (8, residual))]
    call("add_norm", good, [*both, (("out", "out_stride"), (x, 8)), (("out", "out_stride"), (residual, 8)), (("stride", "out"), (9, x))])
    call("add_norm_8bit", {**{k: v for k, v in good.items() if k not in ("rstd", "out", "out_stride", "stream")}, "q": FAR, "q_stride": 7, "scales": A,
                           "stream": None}, both)
    call("add_norm", {**good, "residual": None, "residual_stride": 0, "summed": None, "summed_stride": 0}, [(("out", "out_stride"), (x, 8))])


def test_gradients_in_the_place_of_an_input():
    good = dict(grad=A, dtype=1, n=4, dim=7, grad_stride=7, summed=FAR, summed_stride=7, weight=A, weight_dtype=0, rstd=A, more=A + (1 << 15), more_stride=7,
                grad_x=FAR + (1 << 15), grad_x_stride=7, grad_weight=A, grad_weight_dtype=0, accumulate=0, workspace=A, workspace_bytes=1 << 20,
                stream=None)
    call("add_norm_grad", good, [(("grad_x", "grad_x_stride"), (good["grad"], 8)), (("grad_x", "grad_x_stride"), (good["more"], 8)),
                                 (("grad_stride", "grad_x"), (8, good["grad"]))])
