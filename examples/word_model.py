"""A word-level language model on one GPU that runs the library's calls together, as they would be served.

    embedding -> LSTM whose gate matrix is balanced-sparse -> expert layer in 4 bits (added to its input)
              -> output product in 4 bits -> log probabilities, entropies and the most likely words

``score`` goes over a whole text, ``generate`` makes one word after the other, ``fit_bias`` adapts the output bias to a text
with the gradient of its log probabilities.  Weights are random: the example shows the calls, not a trained model.

    python examples/word_model.py [--words 10000] [--units 1500]
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_1811_00206_amd import binding as bs  # noqa: E402


class WordModel:
    """`units` is the size of embedding and hidden state; `keep` of every `bank` gate weights are kept, `top_k` of `experts` used."""

    def __init__(self, words=10000, units=1500, bank=100, keep=10, experts=8, top_k=2, group=32, seed=0):
        gen = torch.Generator(device="cuda").manual_seed(seed)

        def normal(*shape, scale):
            return torch.randn(shape, generator=gen, device="cuda") * scale

        H = units
        self.units, self.bank, self.group, self.top_k = H, bank, group, top_k
        self.embedding = normal(words, H, scale=1.0)
        self.gates = bs.bs_prune_pack(normal(4 * H, 2 * H, scale=(2 * H * keep / bank) ** -0.5), bank, keep)
        self.gate_bias = torch.zeros(4 * H, device="cuda")
        self.router = normal(experts, H, scale=2 * H**-0.5)
        self.w1 = bs.bs_q4_pack(normal(experts, 2 * H, H, scale=H**-0.5), group)
        self.w2 = bs.bs_q4_pack(normal(experts, H, H, scale=H**-0.5), group)
        self.out = bs.bs_q4_pack(normal(words, H, scale=4 * H**-0.5), group)
        self.out_bias = torch.zeros(words, device="cuda")

    def start(self):
        """State of an empty text: hidden and cell state."""
        return torch.zeros(self.units, device="cuda"), torch.zeros(self.units, device="cuda")

    def logits(self, tokens, state):
        """Rows of logits for the word after each of `tokens`, and the state behind them."""
        h, c = state
        c = c.clone()
        H = bs.bs_lstm_sequence(*self.gates, self.bank, self.embedding[tokens], h, self.gate_bias, c)
        y, ids, weights = bs.bs_q4_moe(H, self.router, *self.w1, *self.w2, self.group, self.top_k)
        return bs.bs_q4_gemv(*self.out, self.group, H + y).add_(self.out_bias), (H[-1].clone(), c)

    def score(self, tokens, top_n=5):
        """Of each word but the first: its log probability, the entropy there, and the most likely words instead of it."""
        logits, _ = self.logits(tokens[:-1], self.start())
        logprob, entropy, _, values, ids = bs.bs_logprobs(logits, tokens[1:], top_n=top_n)
        return logprob, entropy, values, ids

    def generate(self, tokens, n):
        """The n most likely words behind a text, one after the other, and their log probabilities."""
        none = torch.full((1,), -1, dtype=torch.int64, device="cuda")
        logits, state = self.logits(tokens, self.start())
        logits = logits[-1:]
        words, logprobs = [], []
        for i in range(n):
            _, _, _, values, ids = bs.bs_logprobs(logits, none, top_n=1)
            words.append(ids[:, 0].long())
            logprobs.append(values[:, 0])
            if i + 1 < n:
                logits, state = self.logits(words[-1], state)
        return torch.cat(words), torch.cat(logprobs)

    def fit_bias(self, tokens, steps=5, rate=0.5, entropy_weight=0.0):
        """Gradient steps on the output bias: up the mean log probability of a text (and `entropy_weight` times the entropy).
        The mean before each step."""
        logits, _ = self.logits(tokens[:-1], self.start())
        targets, T = tokens[1:], tokens.numel() - 1
        g = torch.full((T,), 1.0 / T, device="cuda")
        means = []
        for _ in range(steps):
            logprob, entropy, lse, _, _ = bs.bs_logprobs(logits, targets)
            means.append(logprob.mean())
            step = rate * bs.bs_logprobs_backward(logits, targets, lse, entropy, g, entropy_weight * g).sum(0)
            self.out_bias += step
            logits += step
        return torch.stack(means)


def main():
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--words", type=int, default=10000)
    p.add_argument("--units", type=int, default=1500)
    a = p.parse_args()
    bs.bs_init()
    model = WordModel(a.words, a.units)
    text = torch.randint(a.words, (200,), generator=torch.Generator().manual_seed(1)).cuda()
    logprob, entropy, values, ids = model.score(text)
    print(f"{text.numel()} words: mean log probability {float(logprob.mean()):.3f}, mean entropy {float(entropy.mean()):.3f}")
    model.generate(text[:20], 5)      # first launches
    torch.cuda.synchronize()
    began = time.perf_counter()
    words, logprobs = model.generate(text[:20], 100)
    torch.cuda.synchronize()
    print(f"100 words behind 20: {(time.perf_counter() - began) * 1e4:.0f} us a word, the first ones {words[:8].tolist()}")
    means = model.fit_bias(text, rate=20.0)
    print("log probability while the output bias is fitted: " + " ".join(f"{m:.3f}" for m in means.tolist()))


if __name__ == "__main__":
    main()
