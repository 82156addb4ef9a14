"""Log probabilities, entropies, alternatives and their gradient against the definitions in 64 bits.

Bounds: a sum of exponentials is off by fp32 roundings of a few hundred additions and of 2^u (1e-5 in its logarithm), a
difference of two fp32 numbers by 2^-22 of their sizes.  A gradient carries those in exp(log p), and its own rounding."""
import math

import pytest
import torch

from paper_1811_00206_amd import binding as bs

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
ROUNDING = {torch.float32: 2.0**-24, torch.float16: 2.0**-11, torch.bfloat16: 2.0**-8}
INF = float("inf")


def definition(logits, targets, n):
    x = logits.cpu().double()
    T, V = x.shape
    m = x.amax(-1, keepdim=True)
    m = torch.where(m == -INF, torch.zeros_like(m), m)
    total = (x - m).exp().sum(-1, keepdim=True)
    logp = torch.where(x == -INF, x, (x - m) - total.log())
    lse = (m + total.log()).squeeze(-1)
    entropy = torch.special.entr(logp.exp()).sum(-1)
    t = targets.cpu()
    logprob = torch.where(t < 0, torch.zeros_like(lse), logp.gather(-1, t.clamp(0, V - 1).unsqueeze(-1)).squeeze(-1))
    logprob[t >= V] = math.nan
    ids = torch.sort(x, dim=-1, descending=True, stable=True).indices[:, :n]
    return logprob, entropy, lse, logp.gather(-1, ids), ids, logp


def near(got, want, allowed):
    got = got.cpu().double()
    special = ~torch.isfinite(want)
    assert torch.equal(got[special].nan_to_num(7e77), want[special].nan_to_num(7e77))
    off = (got - want).abs()[~special]
    allowed = allowed[~special]
    assert bool((off <= allowed).all()), float((off / allowed).max())


def check(logits, targets, n):
    got = bs.bs_logprobs(logits, targets, top_n=n)
    logprob, entropy, lse, values, ids, _ = definition(logits, targets, n)
    size = lse.abs().clamp(max=1e38)
    x_t = logits.cpu().double().gather(-1, targets.cpu().clamp(0, logits.shape[1] - 1).unsqueeze(-1)).squeeze(-1).abs()
    near(got[0], logprob, 1e-5 + 2.0**-22 * (x_t + logprob.abs()))
    near(got[1], entropy, 1e-5 * (2 + entropy))
    near(got[2], lse, 1e-5 + 2.0**-22 * size)
    near(got[3], values, 1e-5 + 2.0**-22 * (values.abs() + size.unsqueeze(-1) * (values > -INF)))
    assert got[4].dtype == torch.int32 and torch.equal(got[4].cpu().long(), ids)
    for a, b in zip(got, bs.bs_logprobs(logits, targets, top_n=n)):
        assert torch.equal(a.nan_to_num(7.0), b.nan_to_num(7.0)), "another call, other bits"
    return got


def rows(T, V, dtype, seed, spread=3.0):
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn((T, V), generator=g) * spread).to(TYPES[dtype])
    targets = torch.randint(-1, V, (T,), generator=g)
    return x.cuda(), targets.cuda()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("T,V,n", [(1, 1, 1), (2, 7, 7), (3, 64, 64), (5, 1000, 5), (1, 10000, 20), (70, 10000, 1), (2, 32003, 64),
                                   (600, 4099, 3), (1, 131072, 20), (3, 50001, 0), (1, 262147, 33), (520, 9000, 17)])
def test_rows(T, V, n, dtype):
    check(*rows(T, V, dtype, T + V), n)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("V,n", [(5000, 20), (32003, 5), (70000, 64)])
def test_masked_rows(V, n, dtype):
    """Masks of -inf and of the type's lowest value that leave all words, some, fewer than n, one, or none."""
    lowest = float(torch.finfo(TYPES[dtype]).min)
    x, targets = rows(12, V, dtype, V)
    g = torch.Generator().manual_seed(1)
    for i, (left, mask) in enumerate([(l, m) for l in (V // 2, n - 1, 2, 1, 0) for m in (-INF, lowest)]):
        keep = torch.randperm(V, generator=g)[:left].cuda()
        row = torch.full((V,), mask, dtype=x.dtype, device="cuda")
        row[keep] = x[i, keep]
        x[i] = row
        if left and i % 3 == 0:
            targets[i] = int(keep[0])
    got = check(x, targets, n)
    assert float(got[2][8]) == -INF and float(got[1][8]) == 0.0            # none left of -inf
    assert abs(float(got[1][9]) - math.log(V)) < 1e-4                      # none left of the lowest value: all alike


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("V", [300, 9001, 40000])
def test_rows_that_flood_the_list(V, dtype):
    """Equal logits, rising and falling ones, a few values only, large ones at the end, and signed zeros."""
    up = torch.arange(V).float() * (8.0 / V)
    few = (torch.arange(V) % 7).float()
    late = torch.zeros(V)
    late[-50:] = torch.linspace(1, 2, 50)
    zeros = torch.zeros(V)
    zeros[::2] = -0.0
    x = torch.stack((torch.zeros(V), up, up.flip(0), few, late, zeros, torch.full((V,), -1000.0))).to(TYPES[dtype]).cuda()
    targets = torch.tensor([0, V - 1, 3, -1, V - 1, 1, 2]).cuda()
    for n in (1, 20, 64):
        check(x, targets, n)


@pytest.mark.parametrize("V,n", [(64, 64), (300, 64), (1483, 43), (2049, 64), (9000, 64), (70000, 50)])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_words_that_lie_together(V, n, dtype):
    """Few words that a mask leaves in a row, fewer threads than n that have any, and short rows."""
    x, targets = rows(5, V, dtype, V + n)
    for i, left in enumerate((V, 600, 420, 65, 9)):
        first = (V - left) // 3 if left < V else 0
        x[i, :first] = -INF
        x[i, first + left:] = -INF
        targets[i] = max(0, first)
    check(x, targets, n)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("T,V,n", [(1025, 1, 1), (1100, 7, 7), (2100, 9, 4), (1030, 64, 64), (1105, 1105, 27), (2049, 2051, 64), (2050, 5003, 0),
                                   (2047, 3000, 2), (2048, 9001, 3)])
def test_many_rows(T, V, n, dtype):
    check(*rows(T, V, dtype, T + V), n)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("V,n", [(70, 64), (1500, 20), (9001, 64)])
def test_many_rows_with_masks_and_equals(V, n, dtype):
    """The rows that are hard by themselves, many times over: what each gives alone."""
    x, targets = rows(9, V, dtype, V)
    lowest = float(torch.finfo(TYPES[dtype]).min)
    few = (torch.arange(V) % 7).to(TYPES[dtype]).cuda()
    for i, row in enumerate((0, few, -INF, lowest, -1000.0)):
        x[i] = row
    x[5, V // 3:] = -INF
    x[6, : V - 5] = -INF
    x[7, 3] = math.nan
    x[8] = few * 1e4 - 6e4
    targets[5:7] = torch.tensor([0, V - 1])
    want = bs.bs_logprobs(x, targets, top_n=n)
    many = 2052 // 9 * 9
    got = bs.bs_logprobs(x.repeat(many // 9, 1), targets.repeat(many // 9), top_n=n)
    for a, b in zip(got[:4], want[:4]):
        torch.testing.assert_close(a, b.repeat(many // 9, *(1,) * (b.dim() - 1)), rtol=1e-5, atol=1e-5, equal_nan=True)
    assert torch.equal(got[4], want[4].repeat(many // 9, 1))
    keep = [i for i in range(9) if i != 7]
    check(x[keep], targets[keep], n)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_rows_of_a_wider_tensor(dtype):
    """Rows that start anywhere between the boundaries of loads; what lies beside them is not looked at."""
    V = 1003
    x, targets = rows(9, V, dtype, 4)
    for first in range(9):
        wide = torch.full((9, V + 13), 100.0, dtype=x.dtype, device="cuda")
        wide[:, first:first + V] = x
        part = wide[:, first:first + V]
        for a, b in zip(check(part, targets, 6), bs.bs_logprobs(x, targets, top_n=6)):
            torch.testing.assert_close(a, b, rtol=1e-5, atol=1e-5)
        room = torch.full((9, V + 8), 3.0, dtype=x.dtype, device="cuda")
        check_gradient(part, targets, out=room[:, 2:2 + V])
        assert bool((room[:, :2] == 3).all()) and bool((room[:, 2 + V:] == 3).all())


@pytest.mark.parametrize("V", [900, 70000])
def test_values_that_are_none_and_targets_that_are_none(V):
    x, targets = rows(6, V, "f32", 2)
    want = bs.bs_logprobs(x, targets, top_n=4)
    x[1, 17], x[3, 5] = math.nan, INF
    targets[4], targets[5] = V, -7
    got = bs.bs_logprobs(x, targets, top_n=4)
    for i in (1, 3):
        assert bool(torch.isnan(got[1][i])) and bool(torch.isnan(got[2][i]))
        assert bool(((got[4][i] >= 0) & (got[4][i] < V)).all())
    assert bool(torch.isnan(got[0][4])) and float(got[0][5]) == 0.0
    for i in (0, 2):
        assert all(torch.equal(a[i], b[i]) for a, b in zip(got, want))
    x[0] = math.nan
    got = bs.bs_logprobs(x, targets, top_n=4)
    assert got[4][0].tolist() == [0, 1, 2, 3]


def check_gradient(logits, targets, out=None, entropy_too=True):
    T, V = logits.shape
    g = torch.Generator().manual_seed(T + V)
    gl, gh = torch.randn(T, generator=g), torch.randn(T, generator=g) * entropy_too
    _, entropy, lse, _, _ = bs.bs_logprobs(logits, targets)
    extra = (entropy, gl.cuda(), gh.cuda()) if entropy_too else (None, gl.cuda(), None)
    got = bs.bs_logprobs_backward(logits, targets, lse, *extra, out=out)
    x, t = logits.cpu().double(), targets.cpu()
    logp = x - lse.cpu().double().unsqueeze(-1)
    p = logp.exp()
    H = entropy.cpu().double().unsqueeze(-1)
    a = torch.where(t < 0, torch.zeros(T), gl).double().unsqueeze(-1)
    b = gh.double().unsqueeze(-1)
    inner = torch.where(p > 0, logp + H, torch.zeros_like(p))
    want = -p * a - b * p * inner
    size = p * (a.abs() + b.abs() * (torch.where(p > 0, logp.abs(), torch.zeros_like(p)) + H))
    row = t >= 0
    want[row.nonzero().squeeze(-1), t[row]] += a[row, 0]
    error = 2.0**-20 + 2.0**-22 * (torch.where(p > 0, x.abs(), torch.zeros_like(p)) + lse.cpu().double().abs().unsqueeze(-1))
    allowed = size * error + ROUNDING[logits.dtype] * want.abs() * 1.001 + 2.0**-23 * a.abs() + (2.0**-25 if logits.dtype == torch.float16 else 2.0**-126)
    assert got.dtype == logits.dtype
    off = (got.cpu().double() - want).abs()
    assert bool((off <= allowed).all()), float((off / allowed).max())
    return got


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("T,V", [(1, 1), (2, 9), (35, 1000), (3, 32003), (1, 131072), (300, 517)])
def test_gradient(T, V, dtype):
    x, targets = rows(T, V, dtype, T * V)
    check_gradient(x, targets)
    check_gradient(x, targets, entropy_too=False)
    x[:, ::3] = -INF
    if V > 1:
        targets = torch.where(targets % 3 == 0, targets + 1, targets).clamp(max=V - 1)
        targets = torch.where(targets % 3 == 0, torch.full_like(targets, -1), targets)
        check_gradient(x, targets)


def test_gradient_against_differences():
    T, V, h = 3, 40, 1e-4
    x, _ = rows(T, V, "f32", 7, spread=1.5)
    targets = torch.tensor([4, -1, 39]).cuda()
    gl, gh = torch.tensor([0.7, 1.0, -1.3]), torch.tensor([0.2, -0.5, 1.1])
    _, entropy, lse, _, _ = bs.bs_logprobs(x, targets)
    got = bs.bs_logprobs_backward(x, targets, lse, entropy, gl.cuda(), gh.cuda()).cpu().double()

    def loss(y):
        logprob, H, *_ = definition(y, targets, 1)
        return gl.double() * logprob + gh.double() * H

    for v in range(V):
        up, down = x.cpu().double(), x.cpu().double()
        up[:, v] += h
        down[:, v] -= h
        want = (loss(up) - loss(down)) / (2 * h)
        assert float((got[:, v] - want).abs().max()) <= 1e-6       # h^2 / 6 of third derivatives below 10, and fp32


def test_gradient_in_place_and_of_empty_rows():
    x, targets = rows(4, 2000, "bf16", 1)
    want = check_gradient(x, targets)
    _, entropy, lse, _, _ = bs.bs_logprobs(x, targets)
    g = torch.Generator().manual_seed(2004)
    gl, gh = torch.randn(4, generator=g).cuda(), torch.randn(4, generator=g).cuda()
    assert torch.equal(bs.bs_logprobs_backward(x, targets, lse, entropy, gl, gh, out=x), want) and torch.equal(x, want)
    for mask in (-INF, float(torch.finfo(torch.float32).min)):
        y = torch.full((3, 700), mask, device="cuda")
        t = torch.tensor([5, -1, 0]).cuda()
        _, entropy, lse, _, _ = bs.bs_logprobs(y, t)
        grad = bs.bs_logprobs_backward(y, t, lse, entropy, torch.ones(3).cuda(), torch.ones(3).cuda())
        assert not bool(grad.any())


@pytest.mark.parametrize("dtype,shift", [("f32", 5e4), ("f32", -1e9), ("f32", 1e20), ("f16", -65504.0), ("bf16", -1e9), ("bf16", 3e4)])
def test_gradient_of_rows_whose_lse_is_large(dtype, shift):
    """lse as it is rounded says little of the differences there.  Half of the words are at the shift or a few above, the others
    far below; against the softmax in 64 bits of the logits as they are."""
    V = 9000
    x = torch.full((3, V), shift, device="cuda")
    x[1, ::2] = -INF
    x[2, 5:40] = shift + abs(shift) / 64
    x = x.to(TYPES[dtype])
    targets = torch.tensor([3, 1, 7]).cuda()
    gl, gh = torch.tensor([0.5, -1.0, 2.0]), torch.tensor([0.25, 1.0, -0.5])
    _, entropy, lse, _, _ = bs.bs_logprobs(x, targets)
    got = bs.bs_logprobs_backward(x, targets, lse, entropy, gl.cuda(), gh.cuda()).cpu().double()
    room = x.clone()
    assert torch.equal(bs.bs_logprobs_backward(room, targets, lse, entropy, gl.cuda(), gh.cuda(), out=room).cpu().double(), got)
    logp = torch.log_softmax(x.cpu().double(), -1)
    p = logp.exp()
    H = torch.special.entr(p).sum(-1, keepdim=True)
    want = -p * gl.double().unsqueeze(-1) - gh.double().unsqueeze(-1) * torch.where(p > 0, p * (logp + H), torch.zeros_like(p))
    want[torch.arange(3), targets.cpu()] += gl.double()
    # entropy and log p are each off by 1e-5 of what they are; then the result's own rounding
    allowed = p * 1e-5 * (gl.abs().unsqueeze(-1) + gh.abs().unsqueeze(-1) * (2 + 2 * H + torch.where(p > 0, logp.abs(), torch.zeros_like(p))))
    allowed = allowed + ROUNDING[TYPES[dtype]] * want.abs() * 1.001 + 2.0**-23 * gl.abs().unsqueeze(-1) + (2.0**-25 if dtype == "f16" else 2.0**-126)
    off = (got - want).abs()
    assert bool((off <= allowed).all()), float((off / allowed).max())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [700, 9000, 70000])
def test_rows_of_large_logits(V, dtype):
    """Rows that lie far from 0, words of which are masked with what is large only, and rows across 2^20, where sums are made
    in another way.  An entropy and a log probability do not depend on where the row lies."""
    g = torch.Generator().manual_seed(V)
    rows_ = []
    for at in (-1e9, -1e10, 1e12, -1e30, 2.0**20 - 3, -(2.0**20), 3e6, 1e4):
        x = torch.randint(-8, 9, (V,), generator=g).double()
        step = max(1.0, abs(at) * 2.0**-7 if dtype == "bf16" else abs(at) * 2.0**-23)
        rows_.append((at + x * step).to(TYPES[dtype]))
    some = torch.full((V,), -1e9)
    some[::97] = torch.randn(some[::97].shape, generator=g)
    rows_.append(some.to(TYPES[dtype]))
    x = torch.stack(rows_).cuda()
    targets = torch.randint(0, V, (len(rows_),), generator=g).cuda()
    targets[-1] = 97
    got = check(x, targets, 9)
    logprob, entropy, _, values, _, _ = definition(x, targets, 9)
    near(got[0], logprob, 1e-5 * (1 + logprob.abs()))
    near(got[1], entropy, 1e-5 * (2 + entropy))
    near(got[3], values, 1e-5 * (1 + values.abs()))


def test_gradient_of_a_target_that_is_none():
    x, targets = rows(3, 500, "f32", 9)
    targets[1] = 500
    _, entropy, lse, _, _ = bs.bs_logprobs(x, targets)
    got = bs.bs_logprobs_backward(x, targets, lse, entropy, torch.ones(3).cuda(), torch.ones(3).cuda())
    assert bool(torch.isnan(got[1]).all()) and bool(torch.isfinite(got[[0, 2]]).all())


def test_graph_replays():
    x, targets = rows(2, 50000, "f32", 3)
    bs.bs_init()
    bs.bs_logprobs(x, targets, top_n=5)
    workspace = torch.empty(max(16, bs.bs_logprobs_workspace_bytes(bs.BS_F32, 2, 50000, 5)), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = bs.bs_logprobs(x, targets, top_n=5, workspace=workspace)
    for seed in range(3):
        x.copy_(torch.randn((2, 50000), generator=torch.Generator().manual_seed(seed)))
        eager = bs.bs_logprobs(x, targets, top_n=5)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, eager):
            assert torch.equal(a, b)


def test_refusals():
    x, t = rows(3, 100, "f32", 1)
    one = torch.zeros(3, device="cuda")
    for call, error, status in (
            (lambda: bs.bs_logprobs(x, t, top_n=65), bs.BsError, 3), (lambda: bs.bs_logprobs(x, t, top_n=-1), bs.BsError, 2),
            (lambda: bs.bs_logprobs(x[:, :4], t, top_n=5), bs.BsError, 2), (lambda: bs.bs_logprobs(x[:0], t[:0]), bs.BsError, 1),
            (lambda: bs.bs_logprobs(x, t.int()), TypeError, None), (lambda: bs.bs_logprobs(x, t[:2]), ValueError, None),
            (lambda: bs.bs_logprobs(x.double(), t), TypeError, None), (lambda: bs.bs_logprobs(x.cpu(), t), TypeError, None),
            (lambda: bs.bs_logprobs(x[:1].expand(3, 100), t), ValueError, None), (lambda: bs.bs_logprobs(x.t(), t), ValueError, None),
            (lambda: bs.bs_logprobs_backward(x, t, one, None, one, one), ValueError, None),
            (lambda: bs.bs_logprobs_backward(x, t, one[:2], one, one, one), ValueError, None),
            (lambda: bs.bs_logprobs_backward(x, t, one, one, one, one, out=x.half()), TypeError, None)):
        with pytest.raises(error) as e:
            call()
        if status is not None:
            assert e.value.status == status
    big, t1 = rows(1, 131072, "f32", 1)
    with pytest.raises(bs.BsError) as e:
        bs.bs_logprobs(big, t1, top_n=4, workspace=torch.zeros(16, dtype=torch.uint8, device="cuda"))
    assert e.value.status == 6
