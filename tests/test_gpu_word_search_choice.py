"""The example's beam search finds what a plain one finds: log probabilities in 64 bits, all continuations in one sorted list, states
gathered one by one.  Both make their logits with the same calls on the same rows, so they choose among the same numbers."""
import math

import pytest
import torch

from paper_1811_00206_amd import binding as bs
from test_gpu_word_search import model, said  # noqa: F401

pytestmark = pytest.mark.gpu


def plain_search(m, text, n, beams, end=-1):
    """Words and 64-bit scores, best first."""
    m.search(text[:1], 1, beams=1)      # which makes the output matrix
    _, (h, c) = m.logits(text[:-1], m.start()) if text.numel() > 1 else (None, m.start())
    found = [([], 0.0, False, int(text[-1]), h, c)]      # words, score, finished, last word, states
    for _ in range(n):
        after = [(bs.bs_lstm_step(*m.gates, m.bank, m.embedding[f[3]], f[4], m.gate_bias, f[5])) for f in found]
        rows = [h for _, h in after] + [torch.zeros_like(h)] * (beams - len(after))      # as many rows as the search multiplies
        H = torch.stack(rows)
        y, _, _ = bs.bs_q4_moe(H, m.router, *m.w1, *m.w2, m.group, m.top_k)
        logits = bs.bs_mx4_gemm(*m.out_mx, H + y, bias=m.out_bias).double().cpu()
        offers = []
        for j, (words, score, done, _, _, _) in enumerate(found):
            if done:
                offers.append((score, j, end))
                continue
            totals = score + torch.log_softmax(logits[j], -1)
            offers += [(float(totals[v]), j, v) for v in totals.argsort(descending=True, stable=True)[:beams + 1].tolist()]
        offers.sort(key=lambda o: (-o[0], o[1], o[2]))
        # The choice has to be one that rounding scores to fp32 does not change.  Equal logits of one beam (products of 4-bit numbers often
        # are) stay equal: their totals move together.
        for a, b in zip(offers[:beams], offers[1:]):
            assert a[0] - b[0] > 1e-4 or (a[:2] == b[:2] and a[2] < b[2]), "choose another text"
        offers = offers[:beams]
        found = [(found[j][0] + [v], score, found[j][2] or v == end, v, after[j][1], after[j][0]) for score, j, v in offers]
    return torch.tensor([f[0] for f in found]), torch.tensor([f[1] for f in found], dtype=torch.float64)


def near(scores, want, n):
    """Each step rounds a score to fp32 once, and the logarithm of a sum in 64 bits is off by 1e-9 at most."""
    return bool(((scores.double().cpu() - want).abs() <= n * (2.0**-24 * want.abs().max() + 1e-9)).all())


def text_of(seed, n):
    return torch.randint(997, (n,), generator=torch.Generator().manual_seed(seed)).cuda()


@pytest.mark.parametrize("beams,n,length,seed", [(1, 8, 5, 1), (5, 1, 12, 2), (5, 6, 12, 2), (3, 7, 1, 3), (8, 5, 9, 4)])
def test_the_best_continuations(model, beams, n, length, seed):  # noqa: F811
    text = text_of(seed, length)
    words, scores = model.search(text, n, beams=beams)
    want, exact = plain_search(model, text, n, beams)
    assert words.cpu().tolist() == want.tolist() and near(scores, exact, n)


def test_one_word(model):  # noqa: F811
    """The most likely words in order, with their log probabilities."""
    text = text_of(2, 12)
    words, scores = model.search(text, 1, beams=5)
    h, c = model.start()
    for t in text.tolist():
        c, h = bs.bs_lstm_step(*model.gates, model.bank, model.embedding[t], h, model.gate_bias, c)
    H = h.expand(5, -1).contiguous()
    y, _, _ = bs.bs_q4_moe(H, model.router, *model.w1, *model.w2, model.group, model.top_k)
    p = torch.log_softmax(bs.bs_mx4_gemm(*model.out_mx, H + y, bias=model.out_bias)[0].double().cpu(), -1)
    best = torch.topk(p, 5)
    assert words[:, 0].tolist() == best.indices.tolist() and near(scores, best.values, 1)


def test_what_ended_keeps_its_words_and_score(model):  # noqa: F811
    text = text_of(4, 5)
    firsts, best = model.search(text, 1, beams=3)
    for place in range(2):      # the most likely first word ends, and the second
        end = int(firsts[place, 0])
        words, scores = model.search(text, 7, beams=3, end=end)
        want, exact = plain_search(model, text, 7, 3, end=end)
        assert words.cpu().tolist() == want.tolist() and near(scores, exact, 7)
        ended = (words == end).any(1)
        assert bool(ended.any())
        at = words.tolist().index([end] * 7)      # that of the first step, which nothing behind it outdoes
        assert float(scores[at]) == float(best[place]) and abs(said(model, text, words[at, :1]) - float(best[place])) < 1e-3
        assert not math.isinf(float(scores.min()))
