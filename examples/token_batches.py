"""From strings to a trained model and back to their likelihood, without leaving the GPU: a bigram model (an embedding and
a matrix) over the encoder's tokens, trained in three ways.

    python examples/token_batches.py

  1. next-token training: encode, embed, log-probabilities with the logits' gradient, the embedding's gradient
  2. preference training on pairs of strings, against the trained model as the reference
  3. policy training: strings with more of a wanted letter have a higher advantage
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2507_11941_amd as bpe  # noqa: E402
import workloads  # noqa: E402


class Bigram:
    """logits = embed(ids) @ head, trained by plain gradient descent; the weights are kept in 32 bits."""

    def __init__(self, vocab, dim, dev):
        g = torch.Generator().manual_seed(0)
        self.scale = dim ** 0.5
        self.embedding = (torch.randn(vocab, dim, generator=g) / self.scale).to(dev)
        self.head = (torch.randn(dim, vocab, generator=g) * 0.05).to(dev)

    def forward(self, ids):
        self.ids, self.hidden = ids, bpe.embed_tokens(self.embedding, ids, self.scale)
        return self.hidden @ self.head

    def step(self, logits_grad, rate):
        to_hidden = logits_grad @ self.head.t()
        self.head -= rate * (self.hidden.t() @ logits_grad)
        # added onto the weights themselves: -rate times the gradient, and only rows that some token names are touched
        bpe.embed_tokens_grad(to_hidden, self.ids, len(self.embedding), -rate * self.scale, out=self.embedding, accumulate=True)


def encode(table, strings, dev):
    """Packed ids and offsets of some strings, on the GPU."""
    data = torch.frombuffer(bytearray(b"".join(strings)), dtype=torch.uint8).to(dev)
    ends = torch.tensor([0] + [len(s) for s in strings]).cumsum(0).to(dev)
    ids, offsets = bpe.encode_batch(table, data, ends, max(map(len, strings)))
    return ids[:int(offsets[-1])], offsets


def main(steps=60):
    dev = torch.device("cuda:0")
    merges = workloads.load_merges("1k")
    table, vocab = bpe.build_table(merges), 256 + len(merges)
    text = workloads.text(1, 5, 64 * 400).tobytes()
    strings = [text[i:i + 400] for i in range(0, len(text), 400)]
    model = Bigram(vocab, 64, dev)
    losses = {}

    # 1. the mean over the tokens that have a successor
    ids, offsets = encode(table, strings, dev)
    targets = bpe.next_tokens(ids, offsets)
    weights = -(targets >= 0).float() / (targets >= 0).sum()
    for step in range(steps):
        logprobs, _, grad = bpe.token_logprobs_and_grad(model.forward(ids), targets, weights)
        model.step(grad, 1.0)
        losses.setdefault("next token", []).append((weights * logprobs).sum().item())

    # 2. a prompt of two words, then a preferred string and another one: here, the one with more of the letter e
    prompts = [s[:20] for s in strings[:32]]
    pairs = [sorted((p + a[20:200], p + b[20:200]), key=lambda s: -s.count(b"e"))
             for p, a, b in zip(prompts, strings[:32], strings[32:])]
    ids, offsets = encode(table, [s for pair in pairs for s in pair], dev)
    # (tokens need not end where the prompt does: what the two strings of a pair share has no part in their difference)
    targets = bpe.next_tokens(ids, offsets)
    reference, _ = bpe.token_logprobs(model.forward(ids), targets)
    for step in range(steps):
        loss, margins, _, grad = bpe.preference_loss(model.forward(ids), targets, offsets, reference, beta=0.1)
        model.step(grad, 0.02)
        losses.setdefault("preference", []).append(loss.item())

    # 3. the strings are taken to be what the policy has written
    advantages = torch.tensor([float(s.count(b"a")) for s in strings])
    advantages = ((advantages - advantages.mean()) / advantages.std()).to(dev)
    ids, offsets = encode(table, strings, dev)
    first = torch.full((len(strings),), 4, dtype=torch.int32, device=dev)          # four tokens of each are its prompt
    targets = bpe.next_tokens(ids, offsets, first)
    reference, _ = bpe.token_logprobs(model.forward(ids), targets)
    old = reference
    for step in range(steps // 4):
        loss, logprobs, grad = bpe.policy_loss(model.forward(ids), targets, offsets, old, advantages, reference, 0.2, 0.28, 0.01,
                                               per="string")
        model.step(grad, 0.1)
        losses.setdefault("policy", []).append(loss.item())
    return losses


if __name__ == "__main__":
    for name, values in main().items():
        print(f"{name}: {values[0]:.4f} -> {values[-1]:.4f}")
