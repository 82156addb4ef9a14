"""Expert layers where their numbers can go wrong: hidden values that cancel."""
import pytest
import torch

from paper_1811_00206_amd import binding as bs
from test_gpu_moe import call, layer, values_of
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
