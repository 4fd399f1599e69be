"""Timed cases of the operators at a language model's output end: the norm with the residual's addition, into 8 bits with
scales or with its gradient; the product with 8-bit weights that gives logits; and the adjustment of logits by what a string
already holds, by biases and by a grammar's masks, with its gradient.

The vocabularies are those of the benchmark's tables (256 byte tokens and 1,000, 32,000 or 100,000 merges, the last with four
special tokens).  Histories are packed as the encoder writes a batch: int32 ids back to back and int64 offsets.

A case is a dict:
  op        "norm_8bit", "norm_step" (forward and backward), "logits", "adjust" or "adjust_step" (forward and backward)
  rows      number of tokens
  dim       (norms, logits) columns of the hidden states
  vocab     (logits, adjust) columns of the logits
  dtype     of hidden states and logits: "f32", "bf16" or "f16"
  residual  (norm_step) whether the norm is of a sum
  weight    (norm_step) type of the norm's weights
  source    (logits) where the 8-bit rows come from: "given"; "rows" (hidden states, quantised first) or "norm" (a norm into 8
            bits of the sum with the residual)
  history   (adjust) tokens of a row's history on average; (adjust_step) tokens of a string: each row has those before it
  each      (adjust) whether rows have penalties of their own
  biases    (adjust) number of tokens of each row that have a bias
  states    (adjust) number of masks that rows choose theirs from; 0: no masks
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZES = {"f32": 4, "bf16": 2, "f16": 2}
VOCABS = (1256, 32256, 100260)
EPS = 1e-6
PENALTIES = (1.25, 0.5, 0.125)       # for all rows: of repeated tokens, once and for each time


def _norm_8bit(name, rows, dim, dtype):
    return _named(name, {"op": "norm_8bit", "rows": rows, "dim": dim, "dtype": dtype})


def _norm_step(name, rows, dim, dtype, weight, residual):
    return _named(name, {"op": "norm_step", "rows": rows, "dim": dim, "dtype": dtype, "weight": weight, "residual": residual})


def _logits(name, rows, dim, vocab, dtype, source):
    return _named(name, {"op": "logits", "rows": rows, "dim": dim, "vocab": vocab, "dtype": dtype, "source": source})


def _adjust(name, rows, vocab, dtype, history, each, biases, states):
    return _named(name, {"op": "adjust", "rows": rows, "vocab": vocab, "dtype": dtype, "history": history, "each": each,
                         "biases": biases, "states": states})


def _adjust_step(name, rows, vocab, dtype, history, states):
    return _named(name, {"op": "adjust_step", "rows": rows, "vocab": vocab, "dtype": dtype, "history": history, "each": False,
                         "biases": 0, "states": states})


def _named(name, case):
    return dict(case, name=name) if name else case


def listed():
    return [
        # a step of a serving loop, one token for each of 32 conversations, ahead of an 8-bit product
        _norm_8bit("norm to 8 bits, 32 rows", 32, 4096, "bf16"),
        # the prompts of a batch
        _norm_8bit("norm to 8 bits, 8191 rows", 8191, 4096, "bf16"),
        # a small model's training step, everything in 32 bits, an odd width, no residual
        _norm_step("norm step, 2003 rows", 2003, 387, "f32", "f32", False),
        # a training step in 16 bits under weights in 32
        _norm_step("norm step, 8209 rows", 8209, 2048, "bf16", "f32", True),
        # the next token's logits of 8 conversations: the weights' reading
        _logits("logits, 8 rows", 8, 4096, 100260, "bf16", "given"),
        # the end of a serving step from the last layer's output on: norm, then product
        _logits("logits, 61 rows", 61, 2048, 32256, "bf16", "norm"),
        # some conversations scored, from hidden states
        _logits("logits, 500 rows", 500, 2048, 100260, "f16", "rows"),
        # a batch scored under 8-bit weights: the largest
        _logits("logits, 8191 rows", 8191, 2048, 100260, "bf16", "given"),
        # a few short answers under a small vocabulary: latency
        _adjust("adjust, 3 rows", 3, 1256, "f32", 40, False, 0, 2),
        # a step of a serving loop: each conversation with its own penalties and biases, some held by a grammar
        _adjust("adjust, 32 rows", 32, 100260, "bf16", 1000, True, 24, 16),
        # a large batch with long histories
        _adjust("adjust, 509 rows", 509, 100260, "bf16", 4000, False, 0, 64),
        # a policy trained under the penalties and masks that its answers were drawn with: each position has those before it
        _adjust_step("adjust step, 2011 rows", 2011, 32256, "bf16", 250, 8),
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, even over its logarithm."""
    return min(hi, max(lo, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    op = rng.choice(["norm_8bit", "norm_step", "logits", "logits", "adjust", "adjust_step"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    vocab = rng.choice(VOCABS)
    dim = _spread(rng, 64, 4096)
    dim -= rng.choice([0, dim % 8, dim % 64])
    if op == "norm_8bit":
        return _norm_8bit(None, _spread(rng, 1, min(16384, (32 << 20) // dim)), dim, dtype)
    if op == "norm_step":
        return _norm_step(None, _spread(rng, 1, min(16384, (32 << 20) // dim)), dim, dtype, rng.choice(["f32", dtype]), rng.random() < 0.5)
    if op == "logits":
        most = int(8191 * 2048 * 100260 / (dim * vocab))
        most = min(16384, most, (1600 << 20) // (vocab * SIZES[dtype]))
        return _logits(None, _spread(rng, 1, max(1, most)), dim, vocab, dtype, rng.choice(["given", "rows", "norm"]))
    most = (200 << 20) // (vocab * SIZES[dtype])
    if op == "adjust":
        return _adjust(None, _spread(rng, 1, min(2048, most)), vocab, dtype, _spread(rng, 1, 4000), rng.random() < 0.5, rng.choice([0, 1, 40]),
                       rng.choice([0, 1, 16]))
    return _adjust_step(None, _spread(rng, 16, min(8192, most)), vocab, dtype, _spread(rng, 8, 500), rng.choice([0, 8]))


def _words(vocab):
    return (vocab + 31) // 32


def _history(case):
    """(begin, end) of the rows' histories, and the number of ids: the same for all seeds."""
    n, mean = case["rows"], case["history"]
    if case["op"] == "adjust_step":                               # strings one after another, each row with what is before it
        at = np.arange(n, dtype=np.int64)
        return at // mean * mean, at, n
    share = np.exp(0.5 * np.random.default_rng((n, mean)).standard_normal(n))
    lens = np.rint(share / share.mean() * mean).astype(np.int64)
    ends = np.cumsum(lens)
    return ends - lens, ends, int(ends[-1])


def _ids(g, dev, count, vocab):
    """Token ids as texts have them: frequencies fall with the rank, ranks lie anywhere in the vocabulary."""
    share = 1.0 / (torch.arange(vocab, device=dev, dtype=torch.float64) + 2.7)
    at = torch.searchsorted(torch.cumsum(share, 0) / share.sum(),
                            torch.rand(count, generator=g, device=dev, dtype=torch.float64)).clamp_(max=vocab - 1)
    return torch.randperm(vocab, generator=g, device=dev)[at].to(torch.int32)


def prepare(case, seed):
    dev = torch.device("cuda:0")
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed) * 7919 + 23)
    n, dtype = case["rows"], TYPES[case["dtype"]]
    state = {"case": case}

    def hidden():
        """Rows as layers leave them: of different sizes, some columns far larger than the others."""
        x = torch.randn(n, case["dim"], generator=g, device=dev)
        columns = torch.exp(0.5 * torch.randn(case["dim"], generator=g, device=dev))
        columns = torch.where(torch.rand(case["dim"], generator=g, device=dev) < 0.005, 20 * columns, columns)
        return (x * columns * torch.exp(0.3 * torch.randn(n, 1, generator=g, device=dev))).to(dtype)

    if case["op"] in ("norm_8bit", "norm_step") or case.get("source") == "norm":
        state["x"] = hidden()
        state["residual"] = hidden() if case.get("residual", True) else None
        state["gain"] = (1 + 0.1 * torch.randn(case["dim"], generator=g, device=dev)).to(TYPES[case.get("weight", case["dtype"])])
    if case["op"] == "norm_step":
        state["grad"] = torch.randn(n, case["dim"], generator=g, device=dev).to(dtype)
        state["grad_summed"] = torch.randn(n, case["dim"], generator=g, device=dev).to(dtype) if case["residual"] else None
    if case["op"] == "logits":
        if case["source"] == "rows":
            state["x"] = hidden()
        elif case["source"] == "given":
            state["q"] = _bytes(g, dev, n, case["dim"])
            state["scales"] = 0.02 * torch.exp(0.3 * torch.randn(n, generator=g, device=dev))
        state["head"] = _bytes(g, dev, case["vocab"], case["dim"])
        state["head_scales"] = 0.001 * torch.exp(0.3 * torch.randn(case["vocab"], generator=g, device=dev))
    if case["op"] in ("adjust", "adjust_step"):
        vocab = case["vocab"]
        begin, end, count = _history(case)
        state["begin"], state["end"] = torch.from_numpy(begin).to(dev), torch.from_numpy(end).to(dev)
        state["named"] = int((end - begin).sum())
        state["ids"] = _ids(g, dev, count, vocab)
        state["logits"] = torch.randn(n, vocab, generator=g, device=dev).mul_(2.5).to(dtype)
        state["penalties"] = PENALTIES
        if case["each"]:
            state["penalties"] = torch.rand(n, 3, generator=g, device=dev) * 0.5 + torch.tensor([1.0, 0.0, 0.0], device=dev)
        if case["biases"]:
            # (no token twice in a row's list)
            apart = vocab // case["biases"]
            at = torch.arange(case["biases"], device=dev) * apart + torch.randint(apart, (n, case["biases"]), generator=g, device=dev)
            state["bias"] = (at.reshape(-1).to(torch.int32), 5 * torch.randn(n * case["biases"], generator=g, device=dev),
                             torch.arange(n, device=dev) * case["biases"], torch.arange(1, n + 1, device=dev) * case["biases"])
        if case["states"]:
            # grammars allow few tokens in some states and nearly all in others; a fifth of the rows is free
            words = _words(vocab)
            allowed = torch.rand(case["states"], 1, generator=g, device=dev) ** 3
            bits = torch.rand(case["states"], words * 32, generator=g, device=dev) < allowed
            place = torch.ones(32, dtype=torch.int64, device=dev) << torch.arange(32, device=dev)
            state["mask"] = (bits.reshape(case["states"], words, 32) * place).sum(2).to(torch.int32)
            state["state"] = torch.randint(-1 - case["states"] // 4, case["states"], (n,), generator=g, device=dev).clamp_(min=-1).to(torch.int32)
        if case["op"] == "adjust_step":
            state["grad"] = torch.randn(n, vocab, generator=g, device=dev).mul_(0.01).to(dtype)
    return state


def _bytes(g, dev, rows, columns):
    """8-bit rows as quantised ones are: the largest of each is 127."""
    x = torch.randn(rows, columns, generator=g, device=dev)
    return x.mul_(127 / x.abs().amax(1, keepdim=True)).round_().to(torch.int8)


# ---- the plain form ------------------------------------------------------------------------------------------

def _summed(state):
    x = state["x"]
    return x if state["residual"] is None else (x.float() + state["residual"].float()).to(x.dtype)


def _to_8bit(p):
    """(whole numbers, largest magnitudes) of rows of products, in 64 bits: what is next to a border falls on its side."""
    top = p.abs().amax(1, keepdim=True)
    return (p * 127 / top).round(), top


def _norm_8bit_plain(state):
    s = _summed(state)
    q, top = _to_8bit(s.double() * state["gain"].double())
    r = (s.float().square().mean(1, keepdim=True) + EPS).rsqrt()
    return q.float(), top.float() * r / 127, s


def _counts(state):
    """How often each token is in each row's history."""
    n, vocab = state["logits"].shape
    lens = state["end"] - state["begin"]
    row = torch.repeat_interleave(torch.arange(n, device=lens.device), lens, output_size=state["named"])
    at = torch.arange(state["named"], device=lens.device) - (lens.cumsum(0) - lens)[row] + state["begin"][row]
    counts = torch.zeros(n * vocab, device=lens.device)
    return counts.index_add_(0, row * vocab + state["ids"][at].long(), torch.ones_like(at, dtype=torch.float32)).reshape(n, vocab)


def _penalties(state):
    p = state["penalties"]
    return p if isinstance(p, tuple) else (p[:, 0:1], p[:, 1:2], p[:, 2:3])


def _allowed(state, vocab):
    v = torch.arange(vocab, device=state["mask"].device)
    words = state["mask"][state["state"].clamp(min=0).long()][:, v // 32]
    return ((words >> (v % 32).to(torch.int32)) & 1 != 0) | (state["state"] < 0)[:, None]


def _adjust_plain(state, counts):
    x, (repeated, presence, frequency) = state["logits"].float(), _penalties(state)
    named = counts > 0
    x = torch.where(named, torch.where(x > 0, x / repeated, x * repeated) - (presence + frequency * counts), x)
    if "bias" in state:
        ids, values, begin, _ = state["bias"]
        row = torch.searchsorted(begin, torch.arange(len(ids), device=ids.device), right=True) - 1
        x = x.index_put((row, ids.long()), values, accumulate=True)
    if "mask" in state:
        x = torch.where(_allowed(state, x.shape[1]), x, -math.inf)
    return x.to(state["logits"].dtype)


def _run_plain(state):
    case = state["case"]
    op = case["op"]
    if op == "norm_8bit":
        q, scales, s = _norm_8bit_plain(state)
        return q * scales, s
    if op == "norm_step":
        s = _summed(state)
        f, gain, g = s.float(), state["gain"].float(), state["grad"].float()
        r = (f.square().mean(1, keepdim=True) + EPS).rsqrt()
        u = g * gain
        to_x = r * u - f * (r ** 3 * (u * f).mean(1, keepdim=True))
        if state["grad_summed"] is not None:
            to_x = to_x + state["grad_summed"].float()
        return (f * r * gain).to(s.dtype), s, to_x.to(s.dtype), (g * f * r).sum(0)
    if op == "logits":
        s = None
        if case["source"] == "norm":
            q, scales, s = _norm_8bit_plain(state)
        elif case["source"] == "rows":
            q, top = _to_8bit(state["x"].double())
            q, scales = q.float(), top.float() / 127
        else:
            q, scales = state["q"].float(), state["scales"][:, None]
        out = (q @ state["head"].float().t()).mul_(scales).mul_(state["head_scales"]).to(TYPES[case["dtype"]])
        return out if s is None else (out, s)
    counts = _counts(state)
    out = _adjust_plain(state, counts)
    if op == "adjust":
        return out
    repeated = _penalties(state)[0]
    x, g = state["logits"].float(), state["grad"].float()
    g = torch.where(counts > 0, torch.where(x > 0, g / repeated, g * repeated), g)
    if "mask" in state:
        g = torch.where(_allowed(state, x.shape[1]), g, 0.0)
    return out, g.to(state["grad"].dtype)


# ---- the framework's operators -------------------------------------------------------------------------------

def _run_own(state):
    import paper_2507_11941_amd as bpe

    case = state["case"]
    op = case["op"]
    if op == "norm_8bit":
        q, scales, s = bpe.add_norm_8bit(state["x"], state["gain"], state["residual"], EPS)
        return q * scales[:, None], s
    if op == "norm_step":
        y, s, r = bpe.add_norm(state["x"], state["gain"], state["residual"], EPS)
        to_x, to_gain = bpe.add_norm_grad(state["grad"], s, state["gain"], r, state["grad_summed"], dtype=torch.float32)
        return y, s, to_x, to_gain
    if op == "logits":
        s = None
        if case["source"] == "norm":
            q, scales, s = bpe.add_norm_8bit(state["x"], state["gain"], state["residual"], EPS)
        elif case["source"] == "rows":
            q, scales = bpe.quantize_rows(state["x"])
        else:
            q, scales = state["q"], state["scales"]
        out = bpe.project_8bit(q, scales, state["head"], state["head_scales"], TYPES[case["dtype"]])
        return out if s is None else (out, s)
    masks = (state.get("mask"), state.get("state"))
    out = bpe.adjust_logits(state["logits"], state["ids"], state["begin"], state["end"], state["penalties"], state.get("bias"), *masks)
    if op == "adjust":
        return out
    return out, bpe.adjust_logits_grad(state["grad"], state["logits"], state["ids"], state["begin"], state["end"], state["penalties"], *masks)


def run(state):
    return _run_own(state) if own else _run_plain(state)


def work(case):
    n, size = case["rows"], SIZES[case["dtype"]]
    if case["op"] in ("norm_8bit", "norm_step"):
        each = case["rows"] * case["dim"]
        if case["op"] == "norm_8bit":                              # x and residual in, the sum and the values out
            return {"bytes": each * (3.0 * size + 1) + 4.0 * n, "flops": 6.0 * each}
        # in: x, grad, with a residual that and the sum's gradient; out: y, grad_x, with a residual the sum
        return {"bytes": each * size * (7.0 if case["residual"] else 4.0) + 8.0 * n + 8.0 * case["dim"], "flops": 16.0 * each}
    vocab = case["vocab"]
    if case["op"] == "logits":
        dim = case["dim"]
        rows = n * dim * {"given": 1.0, "rows": 1.0 * size, "norm": 3.0 * size}[case["source"]]
        return {"bytes": rows + float(vocab) * dim + float(n) * vocab * size + 4.0 * (n + vocab), "flops": 2.0 * n * vocab * dim}
    _, _, count = _history(case)
    extra = 4.0 * count + 16.0 * n + 8.0 * n * case["biases"] + 4.0 * case["states"] * _words(vocab)
    passes = 4.0 if case["op"] == "adjust_step" else 2.0
    return {"bytes": passes * n * vocab * size + extra, "flops": passes * n * vocab}


# ---- the definitions in 64 bits ------------------------------------------------------------------------------

def _exact_8bit(rows, factor):
    """(values, scales) of rows in 64 bits; `factor` is what a row's values are multiplied by besides."""
    top = torch.linalg.vector_norm(rows, math.inf, dim=1)
    whole = torch.div(rows * 127.0, top[:, None]).round()
    return whole, top * factor / 127.0


def exact(case, seed):
    state = prepare(case, seed)
    op = case["op"]
    if op in ("norm_8bit", "norm_step") or case.get("source") == "norm":
        s = state["x"].double()
        if state["residual"] is not None:
            s = (s + state["residual"].double()).to(TYPES[case["dtype"]]).double()
        gain = state["gain"].double()
        r = 1.0 / torch.sqrt(torch.einsum("ij,ij->i", s, s) / case["dim"] + EPS)
    if op == "norm_8bit":
        whole, scales = _exact_8bit(s * gain, r)
        return whole * scales[:, None], s
    if op == "norm_step":
        unit = s * r[:, None]                                      # the norm's output before its weights
        g = state["grad"].double()
        along = torch.einsum("ij,ij,j->i", g, unit, gain) / case["dim"]
        to_x = (g * gain - unit * along[:, None]) * r[:, None]
        if state["grad_summed"] is not None:
            to_x = to_x + state["grad_summed"].double()
        return unit * gain, s, to_x, torch.einsum("ij,ij->j", g, unit)
    if op == "logits":
        if case["source"] == "norm":
            whole, scales = _exact_8bit(s * gain, r)
        elif case["source"] == "rows":
            whole, scales = _exact_8bit(state["x"].double(), 1.0)
        else:
            whole, scales = state["q"].double(), state["scales"].double()
        out = torch.empty(case["rows"], case["vocab"], dtype=torch.float64, device=whole.device)
        for at in range(0, case["vocab"], 16384):                  # whole numbers: exact
            part = slice(at, min(case["vocab"], at + 16384))
            out[:, part] = torch.mm(whole, state["head"][part].double().t())
            out[:, part] *= scales[:, None] * state["head_scales"][part].double()
        return (out, s) if case["source"] == "norm" else out
    x = state["logits"].double()
    g = state["grad"].double() if op == "adjust_step" else None
    begin, end = state["begin"].tolist(), state["end"].tolist()
    chosen = state["state"].tolist() if "mask" in state else None
    place = torch.arange(32, device=x.device)
    for t in range(case["rows"]):
        tokens, times = torch.unique(state["ids"][begin[t]:end[t]].long(), return_counts=True)
        p = state["penalties"]
        repeated, presence, frequency = p if isinstance(p, tuple) else p[t].double()
        at = x[t, tokens]
        factor = torch.where(at > 0, torch.ones_like(at) / repeated, torch.ones_like(at) * repeated)
        x[t, tokens] = at * factor - presence - frequency * times.double()
        if g is not None:
            g[t, tokens] *= factor
        if "bias" in state:
            ids, values, _, _ = state["bias"]
            mine = slice(t * case["biases"], (t + 1) * case["biases"])
            x[t, ids[mine].long()] += values[mine].double()
        if chosen is not None and chosen[t] >= 0:
            banned = ((state["mask"][chosen[t]][:, None] >> place) & 1).reshape(-1)[:case["vocab"]] == 0
            x[t, banned] = -math.inf
            if g is not None:
                g[t, banned] = 0.0
    return x if g is None else (x, g)
