"""From prompts to answers, without leaving the GPU but to print them: a small model over the encoder's tokens is trained, its
output end is put into 8 bits, and it continues prompts token by token, under penalties for what it has already said, a grammar's masks
and a bias.

    python examples/answer_strings.py

  1. training: encode, embed, a block with a residual, a norm of the sum, log-probabilities with the logits' gradient
  2. 8 bits: the norm writes rows of 8-bit integers, the head's weights are 8-bit integers with a scale for each token
  3. answers: logits, adjusted by each string's history, its bias and the mask of its state; the most likely token; the next state
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2507_11941_amd as bpe  # noqa: E402
import workloads  # noqa: E402


class Model(torch.nn.Module):
    """logits = head(norm(x + block(x))), x the embedding of the last token."""

    def __init__(self, vocab, dim, dev):
        super().__init__()
        g = torch.Generator().manual_seed(0)
        self.embedding = torch.nn.Parameter((torch.randn(vocab, dim, generator=g)).to(dev))
        self.block = torch.nn.Parameter((torch.randn(dim, dim, generator=g) / dim ** 0.5).to(dev))
        self.gain = torch.nn.Parameter(torch.ones(dim, device=dev))
        self.head = torch.nn.Parameter((torch.randn(vocab, dim, generator=g) * 0.05).to(dev))

    def forward(self, ids):
        x = bpe.embed_tokens(self.embedding, ids)
        normed, _, _ = bpe.add_norm(torch.relu(x @ self.block), self.gain, x)
        return normed @ self.head.t()


class Server:
    """The same with an output end in 8 bits."""

    def __init__(self, model):
        self.model = model
        self.head, self.scales = bpe.quantize_rows(model.head.detach())

    @torch.no_grad()
    def logits(self, ids):
        m = self.model
        x = bpe.embed_tokens(m.embedding, ids)
        rows, scales, _ = bpe.add_norm_8bit(torch.relu(x @ m.block), m.gain, x, summed=x)
        return bpe.project_8bit(rows, scales, self.head, self.scales, torch.float32)


def bits(allowed):
    """Masks as adjust_logits takes them: a bit for each token, 32 a word, of a matrix of truth values."""
    states, vocab = allowed.shape
    words = (vocab + 31) // 32
    padded = torch.zeros(states, words * 32, dtype=torch.int64)
    padded[:, :vocab] = allowed
    return (padded.view(states, words, 32) << torch.arange(32)).sum(2).to(torch.int32)


def encode(table, strings, dev):
    data = torch.frombuffer(bytearray(b"".join(strings)), dtype=torch.uint8).to(dev)
    ends = torch.tensor([0] + [len(s) for s in strings]).cumsum(0).to(dev)
    ids, offsets = bpe.encode_batch(table, data, ends, max(map(len, strings)))
    return ids[:int(offsets[-1])], offsets


def main(steps=60, length=24):
    dev = torch.device("cuda:0")
    merges = workloads.load_merges("1k")
    table, vocab = bpe.build_table(merges), 256 + len(merges)
    tokens = [bytes([i]) for i in range(256)]
    for a, b in merges.tolist():
        tokens.append(tokens[a] + tokens[b])
    text = workloads.text(1, 5, 64 * 400).tobytes()
    strings = [text[i:i + 400] for i in range(0, len(text), 400)]
    model = Model(vocab, 64, dev)

    # 1. the mean over the tokens that have a successor
    ids, offsets = encode(table, strings, dev)
    targets = bpe.next_tokens(ids, offsets)
    weights = -(targets >= 0).float() / (targets >= 0).sum()
    optimizer = torch.optim.Adam(model.parameters(), lr=0.01)
    losses = []
    for _ in range(steps):
        optimizer.zero_grad()
        logits = model(ids)
        logprobs, _, grad = bpe.token_logprobs_and_grad(logits.detach(), targets, weights)
        logits.backward(grad)
        optimizer.step()
        losses.append((weights * logprobs).sum().item())

    # 2. and 3. the strings' own buffers: a prompt and the answer so far.  Two states: words (letters and spaces), and the full stop that ends.
    prompts = [s[:12] for s in strings[:8]]
    ids, offsets = encode(table, prompts, dev)
    lengths = offsets.diff()
    n, room = len(prompts), int(lengths.max()) + length
    buffer = torch.full((n, room), -1, dtype=torch.int32, device=dev)
    for i, (b, e) in enumerate(zip(offsets.tolist(), offsets.tolist()[1:])):
        buffer[i, :e - b] = ids[b:e]
    prompt_lengths = lengths.clone()
    words = [all(c in b" abcdefghijklmnopqrstuvwxyz" for c in t) for t in tokens]
    mask = bits(torch.tensor([words, [t == b"." for t in tokens]])).to(dev)
    state = torch.zeros(n, dtype=torch.int32, device=dev)
    begin, rows = torch.arange(n, device=dev) * room, torch.arange(n, device=dev)
    # tokens that begin a word, a little more likely
    spaced = torch.tensor([i for i, t in enumerate(tokens) if t[:1] == b" "], dtype=torch.int32, device=dev)
    bias = (spaced, torch.full((len(spaced),), 0.5, device=dev), torch.zeros(n, dtype=torch.int64, device=dev),
            torch.full((n,), len(spaced), device=dev))
    server = Server(model)
    for step in range(length):
        if step == length - 1:
            state.fill_(1)
        logits = server.logits(buffer[rows, lengths - 1])
        bpe.adjust_logits(logits, buffer.view(-1), begin, begin + lengths, (1.2, 0.5, 0.25), bias, mask, state, out=logits)
        buffer[rows, lengths] = logits.argmax(1).to(torch.int32)
        lengths += 1
    answers = []
    for i in range(n):
        said = buffer[i, int(prompt_lengths[i]):int(lengths[i])].tolist()
        answers.append((prompts[i], b"".join(tokens[t] for t in said)))
    return losses, answers


if __name__ == "__main__":
    losses, answers = main()
    print(f"next token: {losses[0]:.4f} -> {losses[-1]:.4f}")
    for prompt, answer in answers:
        print(prompt.decode(errors="replace"), "|", answer.decode(errors="replace"))
