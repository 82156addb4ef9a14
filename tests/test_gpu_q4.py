"""4-bit matrices: packing, unpacking and the product with a few vectors, against definitions in 64 bits.

Codes and scales are compared bit for bit.  A product's error is held to what fp32 sums can lose: an element is the sum
of K exact terms, added 32 at a time and then in at most K / 32 + 64 further steps, each of which loses at most 2^-23 of
the sum of magnitudes; and the result's own rounding."""
import numpy as np
import pytest
import torch

from paper_1811_00206_amd import binding as bs

pytestmark = pytest.mark.gpu
MAGNITUDES = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
ROUNDING = {torch.float32: 2.0**-24, torch.float16: 2.0**-11, torch.bfloat16: 2.0**-8}


def reference_pack(W, group):
    """codes (one a byte) and scales of a float64 matrix, by looking for the nearest number."""
    M, K = W.shape
    G = -(-K // group)
    codes, scales = np.zeros((M, K), np.uint8), np.zeros((M, G), np.float16)
    for g in range(G):
        w = W[:, g * group:(g + 1) * group]
        most = np.abs(w).max(1).astype(np.float32)
        s = np.minimum(most * (np.float32(1) / np.float32(6)), np.float32(65504)).astype(np.float16)
        scales[:, g] = s
        s64 = s.astype(np.float64)[:, None]
        near_s = np.minimum(np.abs(w), 6 * s64)     # beyond the largest number: nearest to it, whatever 64 bits resolve out there
        off = np.abs(near_s[:, :, None] - MAGNITUDES * s64[:, :, None])
        near = off == off.min(-1, keepdims=True)
        even = near[..., ::2]                       # of two that are equally near the even code
        code = np.where(even.any(-1), 2 * even.argmax(-1), near.argmax(-1))
        code = np.where(s[:, None] > 0, code, 0)
        codes[:, g * group:(g + 1) * group] = code | np.where(w < 0, 8, 0)
    return codes, scales


def values(codes, scales, group):
    v = np.concatenate((MAGNITUDES, -MAGNITUDES))[codes]
    return v * np.repeat(scales.astype(np.float64), group, 1)[:, :codes.shape[1]]


def one_a_byte(codes, K):
    c = codes.cpu().numpy()
    both = np.stack((c & 15, c >> 4), -1).reshape(*c.shape[:-1], -1)
    assert not both[..., K:].any(), "codes behind a row's end are 0"
    return both[..., :K]


def matrix(M, K, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    W = torch.randn((M, K), generator=g) * torch.exp2(torch.randint(-6, 7, (M, 1), generator=g).float())
    W[torch.rand((M, K), generator=g) < 0.05] = 0.0
    return W.to(TYPES[dtype])


def packed(M, K, group, seed):
    """A matrix of random codes and scales, and its values."""
    g = torch.Generator().manual_seed(seed)
    codes = torch.randint(0, 256, (M, 16 * -(-K // 32)), generator=g, dtype=torch.int32).to(torch.uint8)
    n = torch.stack((codes & 15, codes >> 4), -1).flatten(1)
    n[:, K:] = 0
    codes = n[:, 0::2] | (n[:, 1::2] << 4)
    scales = (torch.rand((M, -(-K // group)), generator=g) + 0.1).half()
    return codes.cuda(), scales.cuda(), torch.from_numpy(values(n[:, :K].numpy(), scales.numpy(), group))


def check_product(y, W, x):
    K = W.shape[1]
    want, size = x.double() @ W.t(), x.double().abs() @ W.abs().t()
    allowed = 2.0**-23 * (K / 32 + 64) * size + ROUNDING[x.dtype] * want.abs()
    off = (y.cpu().double() - want).abs()
    assert y.dtype == x.dtype and y.shape == want.shape
    assert bool((off <= allowed).all()), float((off / allowed).max())


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("M,K", [(1, 1), (3, 31), (5, 64), (17, 129), (64, 1500), (130, 96), (7, 4096), (33, 1001)])
def test_pack_and_unpack(M, K, group, dtype):
    W = matrix(M, K, dtype, M * 1000 + K)
    codes, scales = bs.bs_q4_pack(W.cuda(), group)
    want, s = reference_pack(W.double().numpy(), group)
    assert scales.dtype == torch.float16 and scales.cpu().numpy().tobytes() == s.tobytes()
    assert np.array_equal(one_a_byte(codes, K), want)
    assert codes.numel() == bs.bs_q4_codes_bytes(M, K) and 2 * scales.numel() == bs.bs_q4_scales_bytes(M, K, group)
    for out in TYPES.values():
        back = bs.bs_q4_unpack(codes, scales, K, group, dtype=out)
        assert torch.equal(back.cpu(), torch.from_numpy(values(want, s, group)).to(out))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_pack_halfway_and_extreme(dtype):
    """Elements halfway between two numbers, groups of zeros, and magnitudes whose scale is subnormal, 0 or cut off."""
    half = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0])
    rows = [torch.cat((half, -half, half * 0.999, half * 1.001)),         # scale 1
            torch.zeros(32), torch.full((32,), -0.0)]
    for most in (6e-8, 2e-7, 1e-5, 6 * 65504.0, 1e30, 3.0):
        rows.append(torch.linspace(-1, 1, 32) * most)
    W = torch.stack(rows)
    if dtype == "f16":
        W = W.clamp(-65504, 65504)
    W = W.to(TYPES[dtype])
    codes, scales = bs.bs_q4_pack(W.cuda(), 32)
    want, s = reference_pack(W.double().numpy(), 32)
    assert scales.cpu().numpy().tobytes() == s.tobytes()
    assert np.array_equal(one_a_byte(codes, 32), want)


def test_pack_of_experts_keeps_leading_dimensions():
    W = matrix(6 * 10, 100, "bf16", 1).reshape(2, 3, 10, 100)
    codes, scales = bs.bs_q4_pack(W.cuda(), 64)
    assert codes.shape == (2, 3, 10, 64) and scales.shape == (2, 3, 10, 2)
    flat = bs.bs_q4_pack(W.reshape(60, 100).cuda(), 64)
    assert torch.equal(codes.reshape(60, 64), flat[0]) and torch.equal(scales.reshape(60, 2), flat[1])
    assert bs.bs_q4_unpack(codes, scales, 100, 64).shape == W.shape


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("M,K,N", [(1, 1, 1), (16, 32, 1), (5, 33, 2), (100, 127, 4), (48, 128, 5), (31, 1500, 1), (257, 640, 16),
                                   (40, 1001, 17), (64, 4100, 3), (20, 25088, 1), (33, 3000, 33), (70, 520, 65), (16, 9000, 13)])
def test_gemv(M, K, N, group, dtype):
    codes, scales, W = packed(M, K, group, M + K + N)
    x = torch.randn((N, K), generator=torch.Generator().manual_seed(N)).to(TYPES[dtype])
    y = bs.bs_q4_gemv(codes, scales, group, x.cuda())
    check_product(y, W, x)
    assert torch.equal(y, bs.bs_q4_gemv(codes, scales, group, x.cuda())), "another call, other bits"
    if N == 1:
        assert torch.equal(y[0], bs.bs_q4_gemv(codes, scales, group, x[0].cuda()))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("N", [1, 3, 20])
def test_gemv_of_slices(N, dtype):
    """Rows of x and of the result inside wider tensors, at odd offsets; what lies between them is left alone."""
    M, K, group = 50, 301, 32
    codes, scales, W = packed(M, K, group, 3)
    wide = torch.randn((N, K + 9), generator=torch.Generator().manual_seed(1)).to(TYPES[dtype])
    for first in (0, 1, 5):
        x = wide.cuda()[:, first:first + K]
        room = torch.full((N, M + 7), 5.0, dtype=TYPES[dtype], device="cuda")
        y = bs.bs_q4_gemv(codes, scales, group, x, out=room[:, 3:3 + M])
        check_product(y, W, wide[:, first:first + K])
        assert bool((room[:, :3] == 5).all()) and bool((room[:, 3 + M:] == 5).all())
        assert torch.equal(y, bs.bs_q4_gemv(codes, scales, group, x.contiguous()))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("N", [2, 18])
def test_gemv_of_extreme_values(N, dtype):
    """Infinities and NaN reach what they belong to and nothing else; large and small magnitudes keep their bits."""
    M, K, group = 40, 200, 64
    codes, scales, W = packed(M, K, group, 9)
    x = torch.randn((N, K), generator=torch.Generator().manual_seed(2))
    x *= torch.exp2(torch.randint(-12, 12, (N, K), generator=torch.Generator().manual_seed(3)).float())
    x = x.to(TYPES[dtype])
    check_product(bs.bs_q4_gemv(codes, scales, group, x.cuda()), W, x)
    x[0, 7], x[1, 9] = float("inf"), float("nan")
    y = bs.bs_q4_gemv(codes, scales, group, x.cuda()).cpu().double()
    want = x.double() @ W.t()
    assert torch.equal(torch.isnan(y), torch.isnan(want)) and torch.equal(torch.isinf(y), torch.isinf(want))
    inf = torch.isinf(want)
    assert torch.equal(y[inf], want[inf])
    check_product(bs.bs_q4_gemv(codes, scales, group, x.cuda())[2:], W, x[2:])
    big = torch.full((N, K), float(torch.finfo(TYPES[dtype]).max)).to(TYPES[dtype])
    y = bs.bs_q4_gemv(codes, scales, group, (big * 2.0**-16).cuda())
    check_product(y, W, big * 2.0**-16)


def test_gemv_on_another_stream_and_in_a_graph():
    M, K, group, N = 300, 1500, 32, 24
    codes, scales, W = packed(M, K, group, 5)
    x = torch.randn((N, K), generator=torch.Generator().manual_seed(4)).cuda()
    want = bs.bs_q4_gemv(codes, scales, group, x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y = bs.bs_q4_gemv(codes, scales, group, x)
    side.synchronize()
    assert torch.equal(y, want)
    bs.bs_init()
    out = torch.empty_like(want)
    workspace = torch.empty(bs.bs_q4_gemv_workspace_bytes(bs.BS_F32, M, K, group, N), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        bs.bs_q4_gemv(codes, scales, group, x, out=out, workspace=workspace)
    for seed in range(3):
        x.copy_(torch.randn((N, K), generator=torch.Generator().manual_seed(seed)))
        eager = bs.bs_q4_gemv(codes, scales, group, x)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager)


@pytest.mark.parametrize("dtype,N", [("f32", 17), ("f32", 24), ("f32", 41), ("f16", 33), ("bf16", 70), ("bf16", 65)])
def test_gemv_whose_last_tiles_have_no_vector(dtype, N):
    """Groups of four tiles, the last of which are empty, in a workspace that ends where it says it does."""
    M, K, group = 70, 1300, 32
    codes, scales, W = packed(M, K, group, N)
    x = torch.randn((N, K), generator=torch.Generator().manual_seed(N)).to(TYPES[dtype])
    need = bs.bs_q4_gemv_workspace_bytes(bs._TYPES[TYPES[dtype]], M, K, group, N)
    room = torch.full((need + 4096,), 255, dtype=torch.uint8, device="cuda")
    y = bs.bs_q4_gemv(codes, scales, group, x.cuda(), workspace=room[:need])
    check_product(y, W, x)
    assert bool((room[need:] == 255).all())


def test_gemv_whose_workgroups_share_k_in_a_graph():
    """Few rows, many columns, several vectors: sums are joined, and counted anew on every replay."""
    M, K, N, group = 40, 12000, 9, 64
    codes, scales, W = packed(M, K, group, 8)
    x = torch.zeros((N, K), dtype=torch.bfloat16, device="cuda")
    bs.bs_init()
    bs.bs_q4_gemv(codes, scales, group, x)
    workspace = torch.full((bs.bs_q4_gemv_workspace_bytes(bs.BS_BF16, M, K, group, N),), 255, dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = bs.bs_q4_gemv(codes, scales, group, x, workspace=workspace)
    for seed in range(3):
        x.copy_(torch.randn((N, K), generator=torch.Generator().manual_seed(seed)))
        want = bs.bs_q4_gemv(codes, scales, group, x)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want)
        check_product(y, W, x.cpu())


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_matrices_that_start_anywhere(dtype):
    """W and scales are only as aligned as their types; what lies beside an unpacked matrix stays."""
    M, K, group = 7, 99, 32
    g = torch.Generator().manual_seed(3)
    W = torch.randn((M, K), generator=g).to(TYPES[dtype]).cuda()
    codes, scales = bs.bs_q4_pack(W, group)
    want = bs.bs_q4_unpack(codes, scales, K, group, dtype=TYPES[dtype])
    x = torch.randn((1, K), generator=g).to(TYPES[dtype]).cuda()
    for first in (1, 2, 3, 5):
        room = torch.zeros(M * K + 8, dtype=W.dtype, device="cuda")
        room[first:first + M * K] = W.flatten()
        c, s = bs.bs_q4_pack(room[first:first + M * K].view(M, K), group)
        assert torch.equal(c, codes) and torch.equal(s, scales)
        wide = torch.zeros(scales.numel() + 8, dtype=torch.float16, device="cuda")
        wide[first:first + scales.numel()] = scales.flatten()
        s = wide[first:first + scales.numel()].view(scales.shape)
        room.fill_(3.0)
        out = bs.bs_q4_unpack(codes, s, K, group, out=room[first:first + M * K].view(M, K))
        assert torch.equal(out, want)
        assert bool((room[:first] == 3).all()) and bool((room[first + M * K:] == 3).all())
        assert torch.equal(bs.bs_q4_gemv(codes, s, group, x), bs.bs_q4_gemv(codes, scales, group, x))


def test_refusals():
    codes, scales, _ = packed(8, 64, 32, 1)
    x = torch.zeros((2, 64), device="cuda")
    for call, error in (
            (lambda: bs.bs_q4_pack(torch.zeros((2, 2), device="cuda", dtype=torch.float64)), TypeError),
            (lambda: bs.bs_q4_pack(torch.zeros((2, 2))), TypeError),
            (lambda: bs.bs_q4_pack(torch.zeros((2, 64), device="cuda"), 48), ValueError),
            (lambda: bs.bs_q4_pack(torch.zeros(64, device="cuda"), 32), ValueError),
            (lambda: bs.bs_q4_pack(torch.zeros((0, 64), device="cuda"), 32), bs.BsError),
            (lambda: bs.bs_q4_pack(torch.zeros((4, 64), device="cuda").t(), 32), ValueError),
            (lambda: bs.bs_q4_unpack(codes, scales, 65, 32), ValueError),
            (lambda: bs.bs_q4_unpack(codes, scales, 64, 64), ValueError),
            (lambda: bs.bs_q4_unpack(codes, scales, 64, 32, dtype=torch.int32), TypeError),
            (lambda: bs.bs_q4_gemv(codes, scales, 32, x[:, :32]), ValueError),
            (lambda: bs.bs_q4_gemv(codes, scales, 33, x), ValueError),
            (lambda: bs.bs_q4_gemv(codes, scales.float(), 32, x), TypeError),
            (lambda: bs.bs_q4_gemv(codes.cpu(), scales, 32, x), TypeError),
            (lambda: bs.bs_q4_gemv(codes, scales, 32, x.double()), TypeError),
            (lambda: bs.bs_q4_gemv(codes, scales, 32, x[:0]), bs.BsError),
            (lambda: bs.bs_q4_gemv(codes, scales, 32, x[:1].expand(2, 64)), ValueError),
            (lambda: bs.bs_q4_gemv(codes, scales, 32, torch.zeros((64, 2), device="cuda").t()), ValueError),
            (lambda: bs.bs_q4_gemv(codes, scales, 32, x, out=torch.zeros((2, 9), device="cuda")), ValueError),
            (lambda: bs.bs_q4_gemv(codes, scales, 32, x, out=torch.zeros((2, 8), device="cuda").half()), TypeError)):
        with pytest.raises(error):
            call()
    many = torch.zeros((20, 64), device="cuda")
    with pytest.raises(bs.BsError) as e:
        bs.bs_q4_gemv(codes, scales, 32, many, workspace=torch.zeros(16, dtype=torch.uint8, device="cuda"))
    assert e.value.status == 6
