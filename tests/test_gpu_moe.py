"""Mixture-of-experts layers against the definition in 64 bits.  Routers and activations are small whole numbers times a
power of two where the choice of experts is compared, so that logits are exact and their ties are ties.

A result's error in the 2-norm: fp32 sums (1e-5, the library's bound for products), hidden values kept in 16 bits for 16-bit
activations (2^-16), and the result's own rounding (half a unit of its last place, at most 2^-8 / 2^-11 of it)."""
import pytest
import torch

from paper_1811_00206_amd import binding as bs
from test_gpu_q4 import TYPES, packed

pytestmark = pytest.mark.gpu
BOUND = {"f32": 1e-5, "f16": 1e-5 + 2.0**-16 + 2.0**-11, "bf16": 1e-5 + 2.0**-16 + 2.0**-8}


def layer(T, D, F, E, group, dtype, seed, exact_router=True):
    g = torch.Generator().manual_seed(seed)
    x = torch.randint(-8, 9, (T, D), generator=g).float() / 8
    router = torch.randint(-2, 3, (E, D), generator=g).float() / 4
    if not exact_router:
        x, router = torch.randn((T, D), generator=g), torch.randn((E, D), generator=g) * 2 * D**-0.5
    c1, s1, w1 = packed(E * 2 * F, D, group, seed + 1)
    c2, s2, w2 = packed(E * D, F, group, seed + 2)
    s1, s2 = s1 * 0.25 * D**-0.5, s2 * 0.25 * F**-0.5          # rounded to binary16: the values follow
    w1 = values_of(c1, s1, D, group).reshape(E, 2 * F, D)
    w2 = values_of(c2, s2, F, group).reshape(E, D, F)
    return dict(x=x.to(TYPES[dtype]), router=router.to(TYPES[dtype]), c1=c1.reshape(E, 2 * F, -1), s1=s1.reshape(E, 2 * F, -1), w1=w1,
                c2=c2.reshape(E, D, -1), s2=s2.reshape(E, D, -1), w2=w2, group=group)


def values_of(codes, scales, K, group):
    table = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64)
    table = torch.cat((table, -table))
    c = codes.cpu().long()
    v = table[torch.stack((c & 15, c >> 4), -1).flatten(1)][:, :K]
    return v * scales.cpu().double().repeat_interleave(group, 1)[:, :K]


def definition(p, top_k, renormalise):
    x = p["x"].double()
    logits = x @ p["router"].double().t()
    ids = torch.sort(logits, dim=-1, descending=True, stable=True).indices[:, :top_k]
    soft = torch.softmax(logits.gather(1, ids), -1) if renormalise else torch.softmax(logits, -1).gather(1, ids)
    y = torch.zeros_like(x)
    for t in range(x.shape[0]):
        for j in range(top_k):
            e = int(ids[t, j])
            a = p["w1"][e] @ x[t]
            F = a.numel() // 2
            y[t] += soft[t, j] * (p["w2"][e] @ (torch.nn.functional.silu(a[:F]) * a[F:]))
    return y, ids, soft


def call(p, top_k, renormalise, x=None):
    return bs.bs_q4_moe(p["x"].cuda() if x is None else x, p["router"].cuda(), p["c1"], p["s1"], p["c2"], p["s2"], p["group"], top_k,
                        renormalise=renormalise)


def check(got, want, dtype):
    y, ids, weights = got
    wy, wi, ww = want
    assert y.dtype == TYPES[dtype] and ids.dtype == torch.int32 and weights.dtype == torch.float32
    assert torch.equal(ids.cpu().long(), wi)
    assert float((weights.cpu().double() - ww).abs().max()) <= 1e-5
    d = y.cpu().double() - wy
    assert float(d.norm()) <= BOUND[dtype] * float(wy.norm()), float(d.norm() / wy.norm())
    # row by row too: an error in one token does not hide behind the others
    rows = d.norm(dim=-1) / wy.norm(dim=-1).clamp(min=1e-30)
    assert float(rows.max()) <= 2 * BOUND[dtype], rows


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("T,D,F,E,top_k,group,renormalise", [
    (1, 1, 1, 1, 1, 32, True), (1, 64, 32, 4, 2, 32, False), (3, 100, 75, 5, 3, 64, True), (1, 1500, 300, 8, 2, 32, True),
    (5, 129, 257, 3, 3, 128, False), (16, 96, 64, 60, 8, 32, True), (17, 160, 48, 4, 1, 64, False), (9, 256, 130, 300, 4, 128, True),
    (64, 70, 40, 6, 5, 32, True), (40, 48, 33, 40, 32, 64, False), (65, 72, 40, 6, 2, 32, True), (201, 64, 48, 20, 3, 64, False)])
def test_layer(T, D, F, E, top_k, group, renormalise, dtype):
    p = layer(T, D, F, E, group, dtype, T + D + F)
    got = call(p, top_k, renormalise)
    check(got, definition(p, top_k, renormalise), dtype)
    for a, b in zip(got, call(p, top_k, renormalise)):
        assert torch.equal(a, b), "another call, other bits"


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("T,D,F,E,top_k,renormalise", [(1, 300, 70, 300, 5, False), (2, 128, 90, 65, 6, True), (3, 64, 64, 1024, 32, True),
                                                       (3, 700, 40, 64, 8, False), (4, 64, 33, 1000, 32, True), (2, 4096, 48, 16, 2, True)])
def test_few_tokens_of_many_experts(T, D, F, E, top_k, renormalise, dtype):
    """Choices with and without a kernel of their own, of more experts than a wavefront has lanes; equal logits among them."""
    p = layer(T, D, F, E, 32, dtype, T + D + E)
    p["router"][1::3] = p["router"][0]
    got = call(p, top_k, renormalise)
    check(got, definition(p, top_k, renormalise), dtype)
    for a, b in zip(got, call(p, top_k, renormalise)):
        assert torch.equal(a, b), "another call, other bits"


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_all_tokens_of_one_expert_and_ties(dtype):
    """Every token wants the same experts, whose logits are equal: the lower numbers win."""
    p = layer(20, 64, 96, 7, 32, dtype, 3)
    p["router"][:] = p["router"][0]
    check(call(p, 3, True), definition(p, 3, True), dtype)


def test_gaussian_activations():
    p = layer(7, 512, 256, 16, 64, "f32", 11, exact_router=False)
    logits = torch.sort(p["x"].double() @ p["router"].double().t(), dim=-1, descending=True).values
    assert float((logits[:, 3] - logits[:, 4]).min()) > 1e-4       # the choice is not in question
    check(call(p, 4, False), definition(p, 4, False), "f32")


@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_rows_of_a_wider_tensor(dtype):
    p = layer(4, 90, 64, 5, 32, dtype, 21)
    wide = torch.zeros((4, 97), dtype=TYPES[dtype], device="cuda")
    wide[:, 3:93] = p["x"].cuda()
    for a, b in zip(call(p, 2, True), call(p, 2, True, x=wide[:, 3:93])):
        assert torch.equal(a, b)


def test_a_token_that_is_no_number_spoils_no_other():
    p = layer(6, 64, 64, 4, 32, "f32", 5)
    want = call(p, 2, True)
    p["x"][2, 5] = float("nan")
    got = call(p, 2, True)
    keep = [0, 1, 3, 4, 5]
    assert bool(torch.isnan(got[0][2]).all())
    assert bool(((got[1] >= 0) & (got[1] < 4)).all())
    for a, b in zip(got, want):
        assert torch.equal(a[keep], b[keep])


def test_graph_replays():
    p = layer(3, 128, 64, 8, 32, "bf16", 8)
    bs.bs_init()
    x = p["x"].cuda()
    call(p, 2, True, x=x)
    workspace = torch.empty(bs.bs_q4_moe_workspace_bytes(bs.BS_BF16, 3, 128, 64, 8, 2, 32), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    router = p["router"].cuda()
    with torch.cuda.graph(graph):
        out = bs.bs_q4_moe(x, router, p["c1"], p["s1"], p["c2"], p["s2"], 32, 2, workspace=workspace)
    for seed in range(3):
        x.copy_(torch.randint(-8, 9, (3, 128), generator=torch.Generator().manual_seed(seed)) / 8)
        eager = call(p, 2, True, x=x)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, eager):
            assert torch.equal(a, b)


@pytest.mark.parametrize("T,D,F,E,top_k,group,dtype", [(9, 192, 1100, 60, 8, 32, "f32"), (70, 130, 96, 12, 4, 64, "f16")])
def test_graph_replays_of_many_tokens(T, D, F, E, top_k, group, dtype):
    """Choices in a kernel of their own, several workgroups for a tile of outputs, more than 64 tokens: counted anew on every replay."""
    p = layer(T, D, F, E, group, dtype, 18)
    bs.bs_init()
    x, router = p["x"].cuda(), p["router"].cuda()
    size = bs.bs_q4_moe_workspace_bytes(bs._TYPES[TYPES[dtype]], T, D, F, E, top_k, group)
    workspace = torch.full((size,), 255, dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = bs.bs_q4_moe(x, router, p["c1"], p["s1"], p["c2"], p["s2"], group, top_k, workspace=workspace)
    for seed in range(3):
        p["x"] = (torch.randint(-8, 9, (T, D), generator=torch.Generator().manual_seed(seed)) / 8).to(TYPES[dtype])
        x.copy_(p["x"])
        graph.replay()
        torch.cuda.synchronize()
        check(out, definition(p, top_k, True), dtype)
        for a, b in zip(out, call(p, top_k, True)):
            assert torch.equal(a, b)


def test_refusals():
    p = layer(2, 64, 32, 4, 32, "f32", 1)
    x, r = p["x"].cuda(), p["router"].cuda()
    args = lambda **k: {**dict(x=x, router=r, w1=p["c1"], s1=p["s1"], w2=p["c2"], s2=p["s2"], group=32, top_k=2), **k}
    for change, error, status in (
            (dict(top_k=0), bs.BsError, 2), (dict(top_k=5), bs.BsError, 2), (dict(x=x[:0]), bs.BsError, 1),
            (dict(x=torch.zeros((65537, 64), device="cuda")), bs.BsError, 3), (dict(x=x.half()), TypeError, None),
            (dict(x=x[:, :60]), ValueError, None), (dict(router=r[:3]), ValueError, None), (dict(w1=p["c1"][:, 1:].contiguous()), ValueError, None),
            (dict(w2=p["c1"]), ValueError, None), (dict(group=16), ValueError, None), (dict(x=x.cpu()), TypeError, None),
            (dict(workspace=torch.zeros(16, dtype=torch.uint8, device="cuda")), bs.BsError, 6)):
        with pytest.raises(error) as e:
            bs.bs_q4_moe(**args(**change))
        if status is not None:
            assert e.value.status == status, change
