"""The gradient of log probabilities and entropies for rows that lie far from 0, against the softmax in 64 bits of the logits as they are.

Bounds: the log of a row's sum is off by 1e-5 at most (fp32 roundings of a few hundred additions, of 2^u, and of lse itself), an
entropy by 1e-5 (2 + H); both are factors or terms of p, and the result has its own rounding."""
import pytest
import torch

from paper_1811_00206_amd import binding as bs
from test_gpu_logprobs import ROUNDING, TYPES

pytestmark = pytest.mark.gpu


def check(x, targets, seed, lost=0.0):
    """`lost`: what a rounded lse may cost beside the type's rounding"""
    T, V = x.shape
    g = torch.Generator().manual_seed(seed)
    gl, gh = torch.randn(T, generator=g), torch.randn(T, generator=g)
    _, entropy, lse, _, _ = bs.bs_logprobs(x, targets)
    logp = torch.log_softmax(x.double(), -1).cpu()
    p = logp.exp()
    H = torch.special.entr(p).sum(-1, keepdim=True)
    t = targets.cpu()
    a = torch.where(t < 0, torch.zeros(T), gl).double().unsqueeze(-1)
    smallest = 2.0**-25 if x.dtype == torch.float16 else 2.0**-126
    for gh in (torch.zeros(T), gh):
        b = gh.double().unsqueeze(-1)
        got = bs.bs_logprobs_backward(x, targets, lse, entropy, gl.cuda(), gh.cuda())
        room = x.clone()
        assert torch.equal(bs.bs_logprobs_backward(room, targets, lse, entropy, gl.cuda(), gh.cuda(), out=room), got)
        got = got.cpu().double()
        want = -p * a - b * torch.where(p > 0, p * (logp + H), torch.zeros_like(p))
        row = t >= 0
        want[row.nonzero().squeeze(-1), t[row]] += a[row, 0]
        allowed = p * (1e-5 + lost) * (a.abs() + b.abs() * (2 + 2 * H + torch.where(p > 0, logp.abs(), torch.zeros_like(p))))
        allowed = allowed + ROUNDING[x.dtype] * want.abs() * 1.001 + 2.0**-23 * a.abs() + smallest
        off = (got - want).abs()
        assert bool((off <= allowed).all()), (off / allowed).amax(-1).tolist()
        if x.dtype == torch.float32 and not bool(gh.any()):
            # p adds up to 1: nothing is left of a row but those errors
            left = got.sum(-1).abs()
            assert bool((left <= 1.1e-5 * a.abs().squeeze(-1) + 1e-30).all()), left.tolist()


FAR = {"f32": (0.0, 5e3, -1e4, -65504.0, 1e5, -1e5, 1e6, -1e6, 2.0**20 - 3, -(2.0**20), 2e6), "f16": (0.0, 5e3, -3e4, 6e4), "bf16": (0.0, -1e4, 1e5, 1e6)}


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("V", [3, 200, 1000, 5003, 40000])
def test_rows_far_from_zero(V, dtype):
    """Every lane has another largest logit: steps of the type's own size there, or a spread of 3."""
    rows = []
    for i, at in enumerate(FAR[dtype]):
        x = torch.randn(V, generator=torch.Generator().manual_seed(V + i)).double()
        step = torch.finfo(TYPES[dtype]).eps * abs(at)
        rows.append((at + x * max(3.0, 2 * step)).clamp(-65504, 65504) if dtype == "f16" else at + x * max(3.0, 2 * step))
    x = torch.stack(rows).to(TYPES[dtype])
    targets = torch.randint(-1, V, (len(rows),), generator=torch.Generator().manual_seed(V))
    check(x.cuda(), targets.cuda(), V)


@pytest.mark.parametrize("dtype,lost", [("f32", 0.0), ("f16", 2.0**-15), ("bf16", 2.0**-13)])
@pytest.mark.parametrize("V", [200, 5003, 140000])
def test_rows_as_far_as_lse_is_not_rounded_away(V, dtype, lost):
    """Up to where lse's rounding reaches what the row's sums are off by (a sixteenth of the rounding of a type of 16 bits), and behind it."""
    at = torch.tensor([20.0, -100.0, 240.0, -270.0, 500.0, -1100.0, 2500.0, 4000.0, -4095.0]).unsqueeze(-1)
    x = torch.randn((9, V), generator=torch.Generator().manual_seed(V)) * 3 + at
    targets = torch.randint(-1, V, (9,), generator=torch.Generator().manual_seed(V + 1))
    check(x.to(TYPES[dtype]).cuda(), targets.cuda(), V, lost)


def test_gradient_beside_the_logits_and_on_them():
    """The other half of the logits' rows holds it, or the logits do; a place in between is refused."""
    V = 301
    wide = torch.zeros((5, 2 * V), device="cuda")
    x, targets = torch.randn((5, V), generator=torch.Generator().manual_seed(1)).cuda(), torch.tensor([0, 5, -1, 300, 7]).cuda()
    _, entropy, lse, _, _ = bs.bs_logprobs(x, targets)
    one = torch.ones(5, device="cuda")
    want = bs.bs_logprobs_backward(x, targets, lse, entropy, one, one)
    wide[:, :V] = x
    got = bs.bs_logprobs_backward(wide[:, :V], targets, lse, entropy, one, one, out=wide[:, V:])
    torch.testing.assert_close(got, want, rtol=1e-6, atol=1e-7)
    assert torch.equal(wide[:, :V], x)
    for out in (wide[:, 1:V + 1], wide[:, V - 1:2 * V - 1]):
        with pytest.raises(bs.BsError) as e:
            bs.bs_logprobs_backward(wide[:, :V], targets, lse, entropy, one, one, out=out)
        assert e.value.status == 3
    assert torch.equal(wide[:, :V], x)


@pytest.mark.parametrize("together", [True, False])
def test_small_probabilities_in_fp32(together):
    """Logits that are log probabilities already, lse 0: exp(x) is off by a unit of the power of two's last place and two roundings,
    whatever the size of x.  (Sums of what remains are within a rounding of 1, and lse = 0 is what they have.)"""
    V = 4001
    x = torch.linspace(-87.0, -1e-3, V + 2).unsqueeze(0).cuda()
    x = x[:, 1:V + 1] if not together else x[:, :V].contiguous()
    zero, one = torch.zeros(1, device="cuda"), torch.full((1,), -1.0, device="cuda")
    target = torch.tensor([5], device="cuda")
    got = bs.bs_logprobs_backward(x, target, zero, None, one, None).cpu().double()[0]
    want = x.cpu().double()[0].exp()
    off = ((got - want).abs() / want)
    off[5] = 0.0
    assert float(off.max()) <= 2.0**-21, float(off.max())
