"""The example's beam search: what it returns is what its own model says of the words it found."""
import importlib.util
import os

import pytest
import torch

from paper_1811_00206_amd import binding as bs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def model():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "word_model.py")
    spec = importlib.util.spec_from_file_location("word_model", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module.WordModel(words=997, units=200, bank=50, keep=10, experts=5, top_k=2, seed=3)


def said(model, text, found):
    """The log probability of the words `found` behind a text, one step after the other."""
    tokens = torch.cat((text, found.long()))
    state, total = model.start(), 0.0
    h, c = state
    for t in range(tokens.numel() - 1):
        c, h = bs.bs_lstm_step(*model.gates, model.bank, model.embedding[tokens[t]], h, model.gate_bias, c)
        if t < text.numel() - 1:
            continue
        y, _, _ = bs.bs_q4_moe(h.view(1, -1), model.router, *model.w1, *model.w2, model.group, model.top_k)
        logits = bs.bs_mx4_gemm(*model.out_mx, h.view(1, -1) + y, bias=model.out_bias)
        total += float(torch.log_softmax(logits[0].double(), -1)[tokens[t + 1]])
    return total


def test_search(model):
    text = torch.randint(997, (12,), generator=torch.Generator().manual_seed(2)).cuda()
    one, score = model.search(text, 6, beams=1)
    assert tuple(one.shape) == (1, 6) and abs(said(model, text, one[0]) - float(score[0])) < 1e-3
    found, scores = model.search(text, 6, beams=5)
    assert tuple(found.shape) == (5, 6) and bool((scores[:-1] >= scores[1:]).all()) and len({tuple(r) for r in found.tolist()}) == 5
    for words, s in zip(found, scores.tolist()):
        assert abs(said(model, text, words) - s) < 1e-3      # fp32 states and sums through 17 steps, two roundings of x to 4 bits alike
    # one word is the most likely ones in order
    first, s = model.search(text, 1, beams=5)
    assert bool((s[:-1] >= s[1:]).all()) and abs(said(model, text, first[0]) - float(s[0])) < 1e-3


def test_an_end_stays(model):
    text = torch.randint(997, (5,), generator=torch.Generator().manual_seed(4)).cuda()
    first = int(model.search(text, 1, beams=3)[0][0, 0])
    found, scores = model.search(text, 7, beams=3, end=first)
    ended = (found == first).any(1)
    for words in found[ended].tolist():
        at = words.index(first)
        assert all(w == first for w in words[at:])
