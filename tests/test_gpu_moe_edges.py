"""Expert layers where their numbers can go wrong: hidden values that cancel, router logits that are no number, sums that are
larger than what they become; and activations too long for LDS."""
import pytest
import torch

from paper_1811_00206_amd import binding as bs
from test_gpu_moe import BOUND, call, check, definition, layer, values_of
from test_gpu_q4 import TYPES

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("T,E,top_k", [(1, 1, 1), (3, 4, 1), (9, 3, 3), (20, 2, 2), (70, 5, 2)])
def test_hidden_values_that_cancel(T, E, top_k, dtype):
    """Two hidden units, the second 1.5 times the first, of which the outputs take 3 and -2 times: nothing is left.

    The gate rows are equal and all sums of the first product exact (activations are eighths, the codes of the second unit's up row
    stand for 1.5 times the first's), so the hidden values are off by one rounding of the product silu(g) * u, 2^-24 of
    each, beyond what both have in common.  Sums of three parts, scale and weight round at most 8 times more."""
    p = layer(T, 64, 2, E, 32, dtype, 100 * T + E)
    g = torch.Generator().manual_seed(T)
    gate = torch.randint(0, 256, (E, 1, 32), generator=g)
    sign = torch.randint(0, 2, (E, 1, 32), generator=g) * 8 + torch.randint(0, 2, (E, 1, 32), generator=g) * 128
    up = [sign + 0x44, sign + 0x55]                                   # codes 4 and 5: 2 and 3
    p["c1"] = torch.cat((gate, gate, *up), 1).byte().cuda()
    p["s1"] = torch.full((E, 4, 2), 2.0**-4, dtype=torch.float16, device="cuda")
    p["c2"] = torch.zeros((E, 64, 16), dtype=torch.uint8)
    p["c2"][:, :, 0] = 0x5 | 0xC << 4                                 # 3 and -2
    p["c2"] = p["c2"].cuda()
    p["s2"] = torch.ones((E, 64, 1), dtype=torch.float16, device="cuda")
    y, ids, weights = call(p, top_k, True)
    w1 = values_of(p["c1"].reshape(-1, 32), p["s1"].reshape(-1, 2), 64, 32).reshape(E, 4, 64)
    size = torch.zeros(T, dtype=torch.float64)
    for t in range(T):
        for e, weight in zip(ids[t].tolist(), weights[t].tolist()):
            a = w1[e] @ p["x"][t].double()
            h = torch.nn.functional.silu(a[:2]) * a[2:]
            assert float((3 * h[0] - 2 * h[1]).abs()) <= 1e-14 * float(h.abs().sum())
            size[t] += weight * float(3 * h[0].abs() + 2 * h[1].abs())
    assert y.dtype == TYPES[dtype] and float(size.max()) > 0.1
    smallest = 2.0**-25 if dtype == "f16" else 0.0                    # binary16 has no smaller numbers
    off = y.cpu().double().abs().amax(-1)
    assert bool((off <= 10 * 2.0**-24 * size + smallest).all()), float((off / size.clamp(min=1e-30)).max())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,E", [(1, 5), (1, 64), (3, 40), (2, 64), (2, 70), (6, 5), (9, 64), (7, 70)])
def test_logits_that_are_no_number_come_last(T, E, dtype):
    """Behind -inf too, whatever their index: who chooses as many experts as have numbers is not touched by the others."""
    p = layer(T, 64, 40, E, 32, dtype, T + E)
    p["x"] = p["x"].abs() + 0.125
    p["router"] = torch.zeros((E, 64), dtype=TYPES[dtype])
    p["router"][0, 3] = p["router"][3, 60] = float("nan")
    p["router"][2, 7] = p["router"][4, 9] = -float("inf")
    p["router"][5:8, 0] = -1.0
    p["router"][8:, 63] = -float("inf")
    finite = [1, *range(5, min(E, 8))]
    impossible = [2, 4, *range(8, E)]
    order = [*finite, *impossible, 0, 3]
    for top_k in sorted({min(n, 32) for n in (1, 2, len(finite) + 1, E - 2, E - 1, E)}):
        y, ids, weights = call(p, top_k, True)
        assert ids.tolist() == [order[:top_k]] * T
        if top_k <= E - 2:
            want_y, _, want = call(p, min(top_k, len(finite)), True)
            assert not bool(weights[:, len(finite):].any()) and torch.equal(weights[:, :len(finite)], want)
            off = (y.double() - want_y.double()).norm(dim=-1)      # added up in another order
            assert bool((off <= 2 * BOUND[dtype] * want_y.double().norm(dim=-1)).all())
        else:
            assert bool(torch.isnan(weights).all())


@pytest.mark.parametrize("T,D,F,E,top_k", [(1, 11000, 40, 3, 2), (3, 11000, 40, 3, 1), (4, 11003, 33, 5, 2), (9, 11000, 20, 2, 2)])
def test_activations_too_long_to_be_brought_together(T, D, F, E, top_k):
    p = layer(T, D, F, E, 64, "f32", T + D)
    check(call(p, top_k, True), definition(p, top_k, True), "f32")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [1, 5, 20])
def test_hidden_values_near_the_largest_number(T, dtype):
    """Small scales of the second product times large hidden values: finite, though the sum of code times hidden value is not."""
    p = layer(T, 64, 256, 2, 128, dtype, T)
    a = torch.einsum("erd,td->etr", p["w1"], p["x"].double())
    h = a[..., :256].clamp(min=0) * a[..., 256:]
    by = 2.0 ** int((126 - float(h.abs().max().log2())) // 2)
    p["x"], p["router"] = p["x"] * by, p["router"] / by
    p["s2"] = (p["s2"] * 2.0**-7).half()
    p["w2"] = values_of(p["c2"].reshape(128, -1), p["s2"].reshape(128, -1), 256, 128).reshape(2, 64, 256)
    check(call(p, 2, True), definition(p, 2, True), dtype)
