"""The example that runs the calls together, against the same model in 64 bits on the CPU."""
import importlib.util
import os

import pytest
import torch

from paper_1811_00206_amd import binding as bs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "word_model.py")
    spec = importlib.util.spec_from_file_location("word_model", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def dense(model, packed, K):
    return bs.bs_q4_unpack(*packed, K, model.group).cpu().double()      # exact in fp32: a code has 3 bits, a scale 11


def in_64_bits(model, tokens):
    """Logits for the word after each token, from the same weights."""
    H, bank = model.units, model.bank
    vals, idx = (t.cpu() for t in model.gates)
    W = torch.zeros(4 * H, 2 * H // bank, bank, dtype=torch.float64)
    W.scatter_(-1, idx.long(), vals.double())
    W = W.flatten(-2)
    w1, w2, out = dense(model, model.w1, H), dense(model, model.w2, H), dense(model, model.out, H)
    router, x = model.router.cpu().double(), model.embedding.cpu().double()[tokens.cpu()]
    h = c = torch.zeros(H, dtype=torch.float64)
    rows = []
    for t in range(len(x)):
        i, f, g, o = (W @ torch.cat((x[t], h)) + model.gate_bias.cpu().double()).split(H)
        c = f.sigmoid() * c + i.sigmoid() * g.tanh()
        h = o.sigmoid() * c.tanh()
        top = torch.topk(router @ h, model.top_k)
        y = torch.zeros(H, dtype=torch.float64)
        for p, e in zip(torch.softmax(top.values, 0), top.indices.tolist()):
            a = w1[e] @ h
            y = y + p * (w2[e] @ (torch.nn.functional.silu(a[:H]) * a[H:]))
        rows.append(out @ (h + y) + model.out_bias.cpu().double())
    return torch.stack(rows)


def test_the_calls_together(example):
    bs.bs_init()
    model = example.WordModel(words=997, units=200, bank=50, keep=10, experts=5, top_k=2, seed=3)
    text = torch.randint(997, (70,), generator=torch.Generator().manual_seed(2)).cuda()
    logits = in_64_bits(model, text[:-1])
    logp = torch.log_softmax(logits, -1)
    logprob, entropy, values, ids = model.score(text, top_n=4)
    targets = text[1:].cpu()
    # fp32 states and sums through 69 steps
    assert float((logprob.cpu().double() - logp.gather(1, targets[:, None])[:, 0]).abs().max()) < 1e-3
    assert float((entropy.cpu().double() - torch.special.entr(logp.exp()).sum(-1)).abs().max()) < 1e-3
    assert float((values.cpu().double() - torch.topk(logp, 4).values).abs().max()) < 1e-3
    assert float((values.cpu().double() - logp.gather(1, ids.cpu().long())).abs().max()) < 1e-3

    # the bias: gradient of the mean log probability
    got = model.fit_bias(text, steps=3, rate=0.5, entropy_weight=0.1).cpu().double()
    x, bias = logits, torch.zeros(997, dtype=torch.float64)
    for m in got:
        b = bias.clone().requires_grad_(True)
        logp = torch.log_softmax(x + b, -1)
        mean = logp.gather(1, targets[:, None]).mean()
        assert abs(float(mean.detach()) - float(m)) < 1e-3
        (mean + 0.1 * -(logp.exp() * logp).sum(-1).mean()).backward()
        bias = bias + 0.5 * b.grad
    assert float((model.out_bias.cpu().double() - bias).abs().max()) < 1e-4

    # what is generated is the most likely word at each step, alone and as a whole text
    words, logprobs = model.generate(text[:10], 6)
    whole = torch.cat((text[:10], words))
    again, _, best, _ = model.score(whole, top_n=1)
    assert float((again[9:] - logprobs).abs().max()) < 1e-3 and float((best[9:, 0] - logprobs).abs().max()) < 1e-3
