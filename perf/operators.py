"""Timed cases of the operators on token batches: embedding lookup and its gradient, token log-probabilities with
their gradient, a preference loss and a clipped policy loss, both from logits to the gradient of the logits.

The vocabularies are those of the benchmark's tables (256 byte tokens and 1,000, 32,000 or 100,000 merges, the
last with four special tokens, so that rows of logits are no multiple of 16 bytes).  A batch of strings is packed as
the encoder writes it: int32 ids back to back and int64 offsets, lengths ragged.

A case is a dict:
  op       "embed", "embed_grad", "score" (log-probabilities alone), "step" (log-probabilities and the logits'
           gradient, the weights known before), "backward" (the same in two calls: the weights come from the
           log-probabilities), "preference" or "policy"
  tokens   number of tokens, which is the number of rows of logits
  vocab    rows of the embedding, columns of the logits
  dim      (embedding) columns
  dtype    of weights, logits and their gradients: "f32", "bf16" or "f16"
  into     (embed_grad) type of the weights' gradient
  padded   (embedding) share of the ids that are padding, -1
  strings  (losses) number of strings, of which each has a prompt whose tokens are not scored
  reference, per   (policy) whether a reference's log-probabilities keep the policy near; "string": an advantage
           for each string, strings weigh the same; "token": one for each token, tokens weigh the same
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZES = {"f32": 4, "bf16": 2, "f16": 2}
VOCABS = (1256, 32256, 100260)
SCALE = 0.125                        # of the embedding's rows: a power of two, as models with scaled embeddings have
BETA, SMOOTHING = 0.1, 0.05          # of the preference loss
LOW, HIGH, KL = 0.2, 0.28, 0.04      # of the policy loss: ratios in [1 - LOW, 1 + HIGH], weight of the KL term
GRAD_SCALE = {"f32": 1.0, "bf16": 1.0, "f16": 1024.0}    # of the losses' gradients: 16-bit floats lose small ones otherwise


def _embed(name, tokens, vocab, dim, dtype, padded=0.0):
    return _named(name, {"op": "embed", "tokens": tokens, "vocab": vocab, "dim": dim, "dtype": dtype, "padded": padded})


def _embed_grad(name, tokens, vocab, dim, dtype, into, padded=0.0):
    return _named(name, {"op": "embed_grad", "tokens": tokens, "vocab": vocab, "dim": dim, "dtype": dtype, "into": into,
                         "padded": padded})


def _logits(name, op, tokens, vocab, dtype, strings):
    return _named(name, {"op": op, "tokens": tokens, "vocab": vocab, "dtype": dtype, "strings": strings})


def _policy(name, tokens, vocab, dtype, strings, reference, per):
    return _named(name, {"op": "policy", "tokens": tokens, "vocab": vocab, "dtype": dtype, "strings": strings,
                         "reference": reference, "per": per})


def _named(name, case):
    return dict(case, name=name) if name else case


def listed():
    return [
        # a step of a serving loop: one new token for each of 32 conversations
        _embed("embed, 32 new tokens", 32, 100260, 4096, "bf16"),
        # the prompts of a batch, padded to whole tiles
        _embed("embed, 40961 tokens of prompts", 40961, 32256, 2048, "bf16", 0.1),
        # a small model's step: one table of 1,000 merges, everything in 32 bits, an odd width
        _embed_grad("embedding gradient, 2003 tokens", 2003, 1256, 387, "f32", "f32"),
        # a training step's gradient of the embedding, kept in 32 bits
        _embed_grad("embedding gradient, 65536 tokens", 65536, 100260, 2048, "bf16", "f32", 0.02),
        # how likely the next token of a few conversations was: latency
        _logits("score, 8 rows", "score", 8, 100260, "bf16", 1),
        # the reference model's log-probabilities of a batch, before a preference or policy step
        _logits("score, 8191 rows", "score", 8191, 100260, "bf16", 16),
        # fine-tuning: the loss of each token and the gradient of the logits, weights known before
        _logits("step, 8209 rows", "step", 8209, 32256, "bf16", 24),
        # the same where the weights follow from the log-probabilities, in 32 bits
        _logits("backward, 1021 rows", "backward", 1021, 32256, "f32", 8),
        # pairs of short answers under a small vocabulary
        _logits("preference, 4 small pairs", "preference", 301, 1256, "f32", 8),
        # pairs of answers of some hundreds of tokens
        _logits("preference, 16 pairs", "preference", 8003, 100260, "bf16", 32),
        # a few answers, an advantage for each token, no reference
        _policy("policy, 500 rows", 500, 32256, "f16", 4, False, "token"),
        # groups of answers to the same prompts, an advantage for each answer, kept near a reference
        _policy("policy, 8190 rows", 8190, 100260, "bf16", 32, True, "string"),
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, even over its logarithm."""
    n = min(hi, max(lo, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))
    return n + 1 if n == 3072 else n


def draw(rng):
    op = rng.choice(["embed", "embed_grad", "score", "step", "backward", "preference", "policy"])
    vocab, dtype = rng.choice(VOCABS), rng.choice(["bf16", "bf16", "f16", "f32"])
    if op in ("embed", "embed_grad"):
        dim = _spread(rng, 64, 4096)
        dim -= rng.choice([0, dim % 8, dim % 64])
        dim += 64 if dim == 3072 else 0
        padded = rng.choice([0.0, 0.02, 0.1])
        tokens = _spread(rng, 1, min(65536, (128 << 20) // dim))
        if op == "embed":
            return _embed(None, tokens, vocab, dim, dtype, padded)
        if vocab * dim > 100260 * 2048:
            vocab = 32256
        return _embed_grad(None, tokens, vocab, dim, dtype, rng.choice(["f32", dtype]), padded)
    most = (640 << 20) // (vocab * SIZES[dtype] // 2)
    if op == "score":
        tokens = _spread(rng, 1, min(16384, most))
        return _logits(None, op, tokens, vocab, dtype, min(tokens, rng.randint(1, 64)))
    strings = 2 * rng.randint(1, 32)
    tokens = _spread(rng, 8 * strings, max(8 * strings + 1, min(16384, most)))
    if op == "policy":
        return _policy(None, tokens, vocab, dtype, strings, rng.random() < 0.5, rng.choice(["string", "token"]))
    return _logits(None, op, tokens, vocab, dtype, strings)


def _lengths(case):
    """(lengths, prompts' lengths) of a case's strings: the same for all seeds but for their order."""
    n, total = case["strings"], case["tokens"]
    rng = np.random.default_rng((n, total))
    share = np.exp(0.6 * rng.standard_normal(n))
    ends = np.rint(np.cumsum(share) / share.sum() * total).astype(np.int64)
    lens = np.diff(ends, prepend=0)
    if case["op"] in ("preference", "policy"):                   # a prompt: a sixteenth to a half of its string
        first = np.rint(lens * rng.uniform(1 / 16, 1 / 2, n)).astype(np.int64)
    else:
        first = np.zeros(n, dtype=np.int64)
    return lens, first


def _ids(g, dev, count, vocab, padded=0.0):
    """Token ids as texts have them: frequencies fall with the rank, ranks lie anywhere in the vocabulary."""
    share = 1.0 / (torch.arange(vocab, device=dev, dtype=torch.float64) + 2.7)
    at = torch.searchsorted(torch.cumsum(share, 0) / share.sum(),
                            torch.rand(count, generator=g, device=dev, dtype=torch.float64)).clamp_(max=vocab - 1)
    ids = torch.randperm(vocab, generator=g, device=dev)[at].to(torch.int32)
    if padded:
        ids[torch.rand(count, generator=g, device=dev) < padded] = -1
    return ids


def prepare(case, seed):
    dev = torch.device("cuda:0")
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed) * 7919 + 17)
    n, vocab, dtype = case["tokens"], case["vocab"], TYPES[case["dtype"]]
    state = {"case": case}
    if case["op"] == "embed":
        state["ids"] = _ids(g, dev, n, vocab, case["padded"])
        state["weight"] = torch.randn(vocab, case["dim"], generator=g, device=dev, dtype=dtype)
        return state
    if case["op"] == "embed_grad":
        state["ids"] = _ids(g, dev, n, vocab, case["padded"])
        state["grad"] = torch.randn(n, case["dim"], generator=g, device=dev, dtype=dtype)
        return state

    lens, first = _lengths(case)
    turn = np.random.default_rng(int(seed)).permutation(len(lens))
    lens, first = lens[turn], first[turn]
    offsets = np.zeros(len(lens) + 1, dtype=np.int64)
    np.cumsum(lens, out=offsets[1:])
    state["ids"] = _ids(g, dev, n, vocab)
    state["offsets"] = torch.from_numpy(offsets).to(dev)
    state["first"] = torch.from_numpy(first.astype(np.int32)).to(dev)
    targets = _next_tokens(state["ids"], state["offsets"], state["first"])
    if case["op"] == "score" and case["strings"] == 1:           # each row a conversation of its own
        targets = state["ids"]
    # logits as a model gives them: spread over some tens, the token that came next among the likely ones
    logits = torch.randn(n, vocab, generator=g, device=dev, dtype=dtype).mul_(2.5)
    at = targets.clamp(min=0).long()[:, None]
    logits.scatter_add_(1, at, (7 + 3 * torch.randn(n, 1, generator=g, device=dev)).to(dtype))
    state["logits"] = logits
    if case["op"] in ("score", "step", "backward"):
        state["targets"] = targets
    if case["op"] == "step":                                     # the mean over the scored tokens
        scored = targets >= 0
        state["weights"] = torch.where(scored, -GRAD_SCALE[case["dtype"]] / scored.sum().clamp(min=1), 0.0).float()
    if case["op"] in ("preference", "policy"):
        now = torch.cat([_logprobs(rows.float(), t)[0]
                         for rows, t in zip(logits.split(1024), targets.split(1024))])
        if case["op"] == "preference" or case["reference"]:
            state["reference"] = now + 0.1 * torch.randn(n, generator=g, device=dev)
    if case["op"] == "policy":
        # The old policy's values: the ratio of a token is near 1, some are beyond the bounds.  None is at a bound
        # itself, where the loss has no derivative.
        away = 0.2 * torch.randn(n, generator=g, device=dev)
        for bound in (math.log(1 - LOW), math.log(1 + HIGH)):
            away = torch.where((away - bound).abs() < 2e-3, 0.01, away)
        state["old"] = now - away
        state["advantages"] = torch.randn(n if case["per"] == "token" else len(lens), generator=g, device=dev)
    return state


# ---- the plain form ------------------------------------------------------------------------------------------

def _next_tokens(ids, offsets, first):
    """The token that follows each one in its string; -1 for a string's last one and before a prompt's end."""
    at = torch.arange(1, len(ids) + 1, device=ids.device)
    string = torch.searchsorted(offsets, at - 1, right=True) - 1
    scored = (at < offsets[string + 1]) & (at - offsets[string] >= first[string])
    return torch.where(scored, ids[at.clamp(max=len(ids) - 1)], -1)


def _logprobs(x, targets):
    """(log-probability of each row's target, logarithm of the sum of the row's exponentials); 0 where target < 0."""
    m = x.amax(1, keepdim=True)
    lse = (m + (x - m).exp().sum(1, keepdim=True).log()).squeeze(1)
    lp = x.gather(1, targets.clamp(min=0).long()[:, None]).squeeze(1) - lse
    return torch.where(targets >= 0, lp, 0.0), torch.where(targets >= 0, lse, 0.0)


def _logits_grad(x, targets, lse, weights):
    """The gradient with respect to the logits of the sum of weights x log-probabilities."""
    p = (x - lse[:, None]).exp()
    weights = torch.where(targets >= 0, weights, 0.0)[:, None]
    grad = torch.where(weights != 0, -weights * p, 0.0)
    return grad.scatter_add_(1, targets.clamp(min=0).long()[:, None], weights)


def _by_string(values, offsets):
    """The sum over each string."""
    string = torch.searchsorted(offsets, torch.arange(len(values), device=values.device), right=True) - 1
    return torch.zeros(len(offsets) - 1, device=values.device).index_add_(0, string, values), string


def _run_plain(state):
    case = state["case"]
    op, vocab = case["op"], case["vocab"]
    ids = state["ids"]
    if op == "embed":
        rows = state["weight"][ids.clamp(min=0).long()].float() * SCALE
        return torch.where((ids >= 0)[:, None], rows, 0.0).to(state["weight"].dtype)
    if op == "embed_grad":
        rows = torch.where((ids >= 0)[:, None], state["grad"].float() * SCALE, 0.0)
        total = torch.zeros(vocab, case["dim"], device=ids.device)
        return total.index_add_(0, ids.clamp(min=0).long(), rows).to(TYPES[case["into"]])

    logits, offsets, scale = state["logits"], state["offsets"], GRAD_SCALE[case["dtype"]]
    x = logits.float()
    targets = state["targets"] if "targets" in state else _next_tokens(ids, offsets, state["first"])
    lp, lse = _logprobs(x, targets)
    if op == "score":
        return lp, lse
    if op == "step":
        return lp, _logits_grad(x, targets, lse, state["weights"]).to(logits.dtype)
    if op == "backward":
        return lp, _logits_grad(x, targets, lse, scale * _confidence(lp, targets)).to(logits.dtype)
    scored = targets >= 0
    if op == "preference":
        per_string, string = _by_string(torch.where(scored, lp - state["reference"], 0.0), offsets)
        margins = BETA * (per_string[0::2] - per_string[1::2])
        wins, losses = torch.nn.functional.logsigmoid(margins), torch.nn.functional.logsigmoid(-margins)
        loss = -((1 - SMOOTHING) * wins + SMOOTHING * losses).mean()
        slope = (SMOOTHING * margins.sigmoid() - (1 - SMOOTHING) * (-margins).sigmoid()) * BETA / len(margins)
        weights = scale * torch.stack([slope, -slope], 1).reshape(-1)[string]
        return loss, margins, lp, _logits_grad(x, targets, lse, weights).to(logits.dtype), targets
    counts, string = _by_string(scored.float(), offsets)
    if case["per"] == "string":
        share = (1.0 / (len(counts) * counts.clamp(min=1)))[string]
        advantages = state["advantages"][string]
    else:
        share, advantages = 1.0 / counts.sum().clamp(min=1), state["advantages"]
    ratio = (lp - state["old"]).exp()
    clipped = ratio.clamp(1 - LOW, 1 + HIGH)
    value = -torch.minimum(ratio * advantages, clipped * advantages)
    slope = torch.where(ratio * advantages <= clipped * advantages, -advantages * ratio, 0.0)
    if case["reference"]:
        apart = state["reference"] - lp
        value = value + KL * (apart.exp() - apart - 1)
        slope = slope + KL * (1 - apart.exp())
    loss = torch.where(scored, share * value, 0.0).sum()
    return loss, lp, _logits_grad(x, targets, lse, scale * share * slope).to(logits.dtype), targets


def _confidence(lp, targets):
    """Weights that follow from the log-probabilities: a token counts less the likelier it already was."""
    return (lp.exp() - 1) / (targets >= 0).sum().clamp(min=1)


# ---- the framework's operators -------------------------------------------------------------------------------

def _run_own(state):
    import paper_2507_11941_amd as bpe

    case = state["case"]
    op = case["op"]
    if op == "embed":
        return bpe.embed_tokens(state["weight"], state["ids"], SCALE)
    if op == "embed_grad":
        return bpe.embed_tokens_grad(state["grad"], state["ids"], case["vocab"], SCALE, dtype=TYPES[case["into"]])
    logits, scale = state["logits"], GRAD_SCALE[case["dtype"]]
    if op == "score":
        return bpe.token_logprobs(logits, state["targets"])
    if op == "step":
        lp, _, grad = bpe.token_logprobs_and_grad(logits, state["targets"], state["weights"])
        return lp, grad
    if op == "backward":
        lp, lse = bpe.token_logprobs(logits, state["targets"])
        return lp, bpe.token_logprobs_grad(logits, state["targets"], lse, scale * _confidence(lp, state["targets"]))
    targets = bpe.next_tokens(state["ids"], state["offsets"], state["first"])
    if op == "preference":
        loss, margins, lp, grad = bpe.preference_loss(logits, targets, state["offsets"], state["reference"], BETA, SMOOTHING,
                                                      scale)
        return loss, margins, lp, grad, targets
    loss, lp, grad = bpe.policy_loss(logits, targets, state["offsets"], state["old"], state["advantages"],
                                     state.get("reference"), LOW, HIGH, KL, case["per"], scale)
    return loss, lp, grad, targets


def run(state):
    return _run_own(state) if own else _run_plain(state)


def work(case):
    n, vocab, size = case["tokens"], case["vocab"], SIZES[case["dtype"]]
    if case["op"] == "embed":                                    # each kept row read and each row written
        return {"bytes": n * (4.0 + case["dim"] * size * (2 - case["padded"])), "flops": float(n * case["dim"])}
    if case["op"] == "embed_grad":
        return {"bytes": n * (4.0 + case["dim"] * size * (1 - case["padded"])) + vocab * case["dim"] * SIZES[case["into"]],
                "flops": float(n * case["dim"])}
    lens, first = _lengths(case)
    scored = n if case["op"] == "score" and case["strings"] == 1 else int(np.maximum(lens - np.maximum(first, 1), 0).sum())
    if case["op"] == "score":                                    # each logit once; a maximum, a difference, an exponential, a sum
        return {"bytes": float(scored) * vocab * size + 12.0 * n, "flops": 4.0 * scored * vocab}
    return {"bytes": float(scored + n) * vocab * size + 20.0 * n, "flops": 7.0 * scored * vocab}


# ---- the definitions in 64 bits ------------------------------------------------------------------------------

def exact(case, seed):
    state = prepare(case, seed)
    ids = state["ids"].long()
    n, vocab = case["tokens"], case["vocab"]
    if case["op"] == "embed":
        out = torch.zeros(n, case["dim"], dtype=torch.float64, device=ids.device)
        kept = (ids >= 0).nonzero().squeeze(1)
        out[kept] = state["weight"].double()[ids[kept]] * SCALE
        return out
    if case["op"] == "embed_grad":
        # by sorted tokens: prefix sums of the rows, and their differences where one token's rows end (columns in parts)
        order = torch.argsort(ids, stable=True)
        order = order[(ids < 0).sum():]
        tokens, counts = torch.unique_consecutive(ids[order], return_counts=True)
        ends = counts.cumsum(0)
        out = torch.zeros(vocab, case["dim"], dtype=torch.float64, device=ids.device)
        for c in range(0, case["dim"], 256):
            part = state["grad"][:, c:c + 256].double()[order].cumsum(0)
            sums = torch.cat([torch.zeros_like(part[:1]), part])[torch.cat([torch.zeros_like(ends[:1]), ends])].diff(dim=0)
            out[:, c:c + 256].index_copy_(0, tokens, sums * SCALE)
        return out

    offsets = state["offsets"].tolist()
    if "targets" in state:
        targets = state["targets"].long()
    else:
        targets = torch.full_like(ids, -1)
        for b, e, f in zip(offsets, offsets[1:], state["first"].tolist()):
            lo = b + max(int(f), 1)
            if lo < e:
                targets[lo - 1:e - 1] = ids[lo:e]
    rows = (targets >= 0).nonzero().squeeze(1)
    logits = state["logits"]
    lp = torch.zeros(n, dtype=torch.float64, device=ids.device)
    lse = torch.zeros_like(lp)
    for r in rows.split(512):
        x = logits[r].double()
        lse[r] = torch.logsumexp(x, 1)
        lp[r] = x[torch.arange(len(r), device=x.device), targets[r]] - lse[r]
    if case["op"] == "score":
        return lp, lse

    loss = margins = None
    scale = 1.0 if case["op"] == "step" else GRAD_SCALE[case["dtype"]]
    slope = torch.zeros_like(lp)                                 # of the loss with respect to lp
    if case["op"] == "step":
        slope = state["weights"].double()
    elif case["op"] == "backward":
        slope[rows] = torch.expm1(lp[rows]) / max(1, len(rows))
    elif case["op"] == "preference":
        apart = torch.zeros_like(lp)
        apart[rows] = lp[rows] - state["reference"][rows].double()
        sums = torch.stack([apart[b:e].sum() for b, e in zip(offsets, offsets[1:])])
        margins = BETA * (sums[0::2] - sums[1::2])
        pairs = len(margins)
        loss = ((1 - SMOOTHING) * torch.log1p(torch.exp(-margins)) + SMOOTHING * torch.log1p(torch.exp(margins))).sum() / pairs
        for k in range(pairs):
            d = BETA * (SMOOTHING - 1 + torch.sigmoid(margins[k])) / pairs
            slope[offsets[2 * k]:offsets[2 * k + 1]] = d
            slope[offsets[2 * k + 1]:offsets[2 * k + 2]] = -d
    else:
        loss = torch.zeros((), dtype=torch.float64, device=ids.device)
        for i, (b, e) in enumerate(zip(offsets, offsets[1:])):
            r = b + (targets[b:e] >= 0).nonzero().squeeze(1)
            if not len(r):
                continue
            a = state["advantages"][r].double() if case["per"] == "token" else state["advantages"][i].double().expand(len(r))
            share = 1 / len(rows) if case["per"] == "token" else 1 / (len(offsets) - 1) / len(r)
            ratio = torch.exp(lp[r] - state["old"][r].double())
            free = torch.where(a >= 0, ratio <= 1 + HIGH, ratio >= 1 - LOW)
            value = torch.where(free, -ratio * a, -torch.where(a >= 0, 1 + HIGH, 1 - LOW) * a)
            d = torch.where(free, -ratio * a, 0.0)
            if case["reference"]:
                k = state["reference"][r].double() - lp[r]
                value = value + KL * (torch.expm1(k) - k)
                d = d - KL * torch.expm1(k)
            loss += share * value.sum()
            slope[r] = share * d
    grad = torch.zeros(n, vocab, dtype=torch.float64, device=ids.device)
    for r in rows.split(512):
        p = torch.softmax(logits[r].double(), 1)
        p[torch.arange(len(r), device=p.device), targets[r]] -= 1
        grad[r] = p * (-scale * slope[r, None])
    if case["op"] in ("step", "backward"):
        return lp, grad
    return (loss, margins, lp, grad, None) if case["op"] == "preference" else (loss, lp, grad, None)
