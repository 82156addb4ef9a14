"""MX 4-bit matrices and their products against the definition in 64 bits."""
import math

import pytest
import torch

from mx4_reference import packed, quantise, values
from paper_1811_00206_amd import binding as bs

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = (torch.float32, torch.float16, torch.bfloat16)


def _edges(dtype):
    """Rows of 64 elements with everything that a block can hold."""
    tiny = torch.finfo(dtype).smallest_normal
    big = torch.finfo(dtype).max
    g = torch.Generator().manual_seed(3)
    W = torch.randn(24, 64, generator=g)
    W[0] = 0
    W[1, :8] = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 4.0])       # halfway cases
    W[1, 8:] = -0.0
    W[2] = tiny * torch.linspace(-1, 1, 64)
    W[3] = tiny / 2
    W[4, 3] = math.inf
    W[5, 40] = math.nan
    W[6, 1] = -math.inf
    W[7] = big
    W[8, ::2] = -big
    W[9, 5] = 7.99
    W[10] *= 2.0**-10
    W[11, 0], W[11, 1:] = 1.0, 2.0**-6
    W[12, :] = 6.0
    W[13, :32] = torch.arange(32) / 4.0
    W[14, 33] = 1e4
    W[15, :32] = 0
    return W.to(dtype)


def _check_pack(W):
    codes, scales = bs.bs_mx4_pack(W)
    want, want_scales = quantise(W)
    assert torch.equal(scales.cpu().long(), want_scales)
    assert torch.equal(codes.cpu(), packed(want))
    return codes, scales


@pytest.mark.parametrize("dtype", TYPES)
def test_pack_edges(dtype):
    W = _edges(dtype).to(DEV)
    codes, scales = _check_pack(W)
    for out in TYPES:
        got = bs.bs_mx4_unpack(codes, scales, 64, dtype=out).cpu()
        want = values(codes, scales, 64).float().to(out)      # the first rounding is exact, but for what is too large
        assert torch.equal(torch.nan_to_num(got.float(), nan=123.0), torch.nan_to_num(want.float(), nan=123.0))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,K", [(1, 1), (3, 31), (2, 32), (5, 33), (7, 127), (4, 128), (3, 129), (17, 300), (2, 4097), (300, 8)])
def test_pack_shapes(dtype, M, K):
    g = torch.Generator().manual_seed(M * 1000 + K)
    W = (torch.randn(M, K, generator=g) * torch.exp(2 * torch.randn(M, K, generator=g))).to(dtype).to(DEV)
    codes, scales = _check_pack(W)
    wide = torch.full((M, K + 5), 1e9, dtype=torch.float32).to(dtype).to(DEV)
    wide[:, 3:K + 3] = W
    again = bs.bs_mx4_pack(wide[:, 3:K + 3])
    assert torch.equal(codes, again[0]) and torch.equal(scales, again[1])
    out = torch.full((M, K), 9.0, dtype=dtype, device=DEV)
    assert bs.bs_mx4_unpack(codes, scales, K, out=out) is out
    assert torch.equal(out.cpu(), values(codes, scales, K).float().to(dtype))


def test_pack_leading_dimensions_and_every_scale():
    W = torch.randn(2, 3, 70, device=DEV)
    codes, scales = bs.bs_mx4_pack(W)
    assert tuple(codes.shape) == (2, 3, 64) and tuple(scales.shape) == (2, 3, 4)
    flat = bs.bs_mx4_pack(W.view(6, 70))
    assert torch.equal(codes.view(6, -1), flat[0]) and torch.equal(scales.view(6, -1), flat[1])
    # every scale byte with every code
    scales = torch.arange(256, dtype=torch.uint8).view(64, 4).to(DEV)
    codes = torch.arange(256, dtype=torch.uint8).repeat(64, 1)[:, :64].contiguous().to(DEV)
    got = bs.bs_mx4_unpack(codes, scales, 128).cpu().double()
    want = values(codes, scales, 128).float().double()
    assert torch.equal(torch.nan_to_num(got, nan=7.0), torch.nan_to_num(want, nan=7.0))


def _bound(W, X, y, dtype, K, bias):
    """What the matrix unit may be off by: one unit of fp32 of the sum of magnitudes for each of its additions (64 columns each at the least,
    16 for the sums of wavefronts and slices, one for the bias), and half a step of the result's type."""
    steps = -(-K // 64) + 18
    size = X.abs() @ W.abs().t()
    if bias is not None:
        size = size + bias.double().cpu().abs()
    return steps * 2.0**-23 * size + torch.finfo(dtype).eps / 2 * y.abs() + 2.0**-149


def _product(M, K, N, dtype, bias, seed=0, wide=False):
    g = torch.Generator().manual_seed(seed + 7 * M + 3 * K + N)
    W = torch.randn(M, K, generator=g) * torch.exp(torch.randn(M, 1, generator=g))
    x = (torch.randn(N, K, generator=g) * torch.exp(torch.randn(N, 1, generator=g))).to(dtype)
    b = torch.randn(M, generator=g).to(DEV) if bias else None
    codes, scales = bs.bs_mx4_pack(W.to(DEV))
    xd = x.to(DEV)
    if wide:
        room = torch.full((N, K + 3), 1e4, dtype=dtype, device=DEV)
        room[:, 1:K + 1] = xd
        xd = room[:, 1:K + 1]
        place = torch.full((N + 2, M + 7), 3.0, dtype=dtype, device=DEV)
        y = bs.bs_mx4_gemm(codes, scales, xd, bias=b, out=place[1:N + 1, 2:M + 2])
        rest = place.clone()
        rest[1:N + 1, 2:M + 2] = 3.0
        assert bool((rest == 3.0).all())
    else:
        y = bs.bs_mx4_gemm(codes, scales, xd, bias=b)
    xc, xs = quantise(x)
    Xq = values(packed(xc), xs, K)
    Wq = values(codes, scales, K)
    want = Xq @ Wq.t()
    if b is not None:
        want = want + b.double().cpu()
    assert y.dtype == dtype and tuple(y.shape) == (N, M)
    off = (y.double().cpu() - want).abs()
    assert bool((off <= _bound(Wq, Xq, want, dtype, K, b)).all()), float((off / _bound(Wq, Xq, want, dtype, K, b)).max())
    again = bs.bs_mx4_gemm_packed(codes, scales, *bs.bs_mx4_pack(xd), K, dtype=dtype, bias=b)
    assert torch.equal(again, y)


@pytest.mark.parametrize("N", [1, 2, 3, 16, 17, 32, 33, 64, 65, 128, 129, 257])
@pytest.mark.parametrize("M,K", [(1, 1), (16, 128), (33, 40), (64, 257), (130, 500), (300, 1500)])
def test_products(M, K, N):
    for dtype, bias, wide in ((torch.float32, True, False), (torch.float16, False, True), (torch.bfloat16, True, True)):
        _product(M, K, N, dtype, bias, wide=wide)


@pytest.mark.parametrize("M,K,N", [(1000, 3000, 300), (513, 8200, 70), (257, 256, 1025), (2048, 2048, 512), (70, 25088, 5), (64, 25088, 33), (5000, 700, 1),
                                   (31, 16000, 1), (4100, 384, 100), (128, 16384, 256)])
def test_larger_products(M, K, N):
    _product(M, K, N, torch.bfloat16, True)
    _product(M, K, N, torch.float32, False, wide=True)


def test_one_vector():
    W = bs.bs_mx4_pack(torch.randn(50, 96, device=DEV))
    x = torch.randn(96, device=DEV)
    y = bs.bs_mx4_gemm(*W, x)
    assert tuple(y.shape) == (50,) and torch.equal(y, bs.bs_mx4_gemm(*W, x.view(1, 96))[0])
    out = torch.empty(50, device=DEV)
    assert bs.bs_mx4_gemm(*W, x, out=out) is out and torch.equal(out, y)


@pytest.mark.parametrize("N", [1, 2, 5, 40, 200])
def test_what_is_no_number_stays_in_its_row_or_column(N):
    M, K = 150, 300
    W, x = torch.randn(M, K, device=DEV), torch.randn(N, K, device=DEV)
    clean = bs.bs_mx4_gemm(*bs.bs_mx4_pack(W), x)
    W[70, 290], x[N // 2, 7] = math.nan, math.inf
    y = bs.bs_mx4_gemm(*bs.bs_mx4_pack(W), x)
    hit = torch.zeros(N, M, dtype=torch.bool, device=DEV)
    hit[N // 2], hit[:, 70] = True, True
    assert bool(y[hit].isnan().all()) and torch.equal(y[~hit], clean[~hit])


@pytest.mark.parametrize("N", [1, 2, 20, 130])
def test_largest_and_smallest_scales(N):
    """Products of scales outside fp32's range meet others inside it: what is too small adds nothing, what is too large is infinite."""
    M, K = 40, 256
    g = torch.Generator().manual_seed(5)
    codes = torch.randint(0, 256, (M, 128), generator=g, dtype=torch.uint8)
    xc = torch.randint(0, 256, (N, 128), generator=g, dtype=torch.uint8)
    for w_scale, x_scale in ((0, 0), (1, 30), (254, 0), (200, 40), (100, 20), (180, 175)):
        s = torch.full((M, 8), w_scale, dtype=torch.uint8)
        xs = torch.full((N, 8), x_scale, dtype=torch.uint8)
        y = bs.bs_mx4_gemm_packed(codes.to(DEV), s.to(DEV), xc.to(DEV), xs.to(DEV), K).cpu().double()
        Wq, Xq = values(codes, s, K), values(xc, xs, K)
        want = Xq @ Wq.t()
        bound = _bound(Wq, Xq, want, torch.float32, K, None) + 2.0**-149 * 24
        assert bool(((y - want).abs() <= bound).all()), (w_scale, x_scale)
    s, xs = torch.full((M, 8), 254, dtype=torch.uint8), torch.full((N, 8), 254, dtype=torch.uint8)
    codes[:], xc[:] = 0x77, 0x77
    assert bool(bs.bs_mx4_gemm_packed(codes.to(DEV), s.to(DEV), xc.to(DEV), xs.to(DEV), K).isinf().all())


def test_products_are_the_same_every_time():
    for M, K, N in ((4096, 6000, 1), (1000, 25088, 77), (600, 1500, 300)):
        W, x = bs.bs_mx4_pack(torch.randn(M, K, device=DEV)), torch.randn(N, K, device=DEV)
        y = bs.bs_mx4_gemm(*W, x)
        for _ in range(3):
            assert torch.equal(bs.bs_mx4_gemm(*W, x), y)
        # a row's result does not depend on where it lies
        room = torch.empty(N, K + 1, device=DEV)[:, 1:]
        room.copy_(x)
        assert torch.equal(bs.bs_mx4_gemm(*W, room), y)


# one of every kind: rows of W from memory (16 rows of W of a wavefront, 16 rows of x, wavefronts that share K, groups), tiles (rows, columns,
# stages in LDS, whether K is split)
KINDS = [((1, 619, 1), (1, 1, 2, 4)), ((40, 1108, 1), (1, 1, 4, 1)), ((17, 2269, 2), (1, 1, 8, 1)), ((33, 4893, 1), (1, 1, 16, 1)), ((5, 308, 22), (1, 2, 1, 4)),
         ((100, 530, 17), (1, 2, 2, 4)), ((30, 1092, 18), (1, 2, 4, 1)), ((50, 2137, 21), (1, 2, 8, 1)), ((60, 1088, 34), (1, 4, 4, 1)),
         ((90, 2060, 50), (1, 4, 8, 1)), ((17199, 3899, 10), (2, 1, 4, 2)), ((300, 200, 100), (32, 128, 4, False)), ((3, 1480, 66), (32, 128, 4, True)),
         ((134, 2, 4413), (64, 128, 4, False)), ((3, 1541, 2054), (64, 128, 4, True)), ((20052, 4, 67), (96, 128, 4, False)), ((3, 3154, 1812), (96, 128, 4, True)),
         ((19690, 200, 97), (128, 128, 2, False)), ((2, 2648, 2441), (128, 128, 2, True)), ((2139, 849, 1587), (128, 128, 4, False)),
         ((1314, 7772, 527), (128, 128, 4, True)), ((2562, 538, 3608), (256, 256, 2, False)), ((2876, 13468, 1504), (256, 256, 2, True))]


@pytest.mark.parametrize("shape,kind", KINDS)
def test_every_kind_of_product(shape, kind):
    M, K, N = shape
    p = bs.bs_mx4_gemm_plan(M, K, N)
    found = (p["tile_rows"], p["tile_columns"], p["buffers"], p["split"] > 1) if p["tile_rows"] else (p["r"], p["nt"], p["ways"], p["groups"])
    assert found == kind
    _every_type(M, K, N)


# rows of x that every workgroup rounds for itself, 1 to 5 pieces of each thread, and on the other side of that rule
@pytest.mark.parametrize("shape,alone", [((219, 203, 11), True), ((40, 1, 16), True), ((32306, 651, 12), True), ((10000, 1500, 4), True), ((301, 700, 16), True),
                                         ((1100, 3001, 6), True), ((1100, 3001, 7), False), ((77, 8191, 4), True), ((10000, 1500, 8), False), ((200001, 500, 5), False)])
def test_rows_rounded_on_the_way(shape, alone):
    M, K, N = shape
    p = bs.bs_mx4_gemm_plan(M, K, N)
    assert (p["tile_rows"] == 0 and bs.bs_mx4_gemm_workspace_bytes(bs.BS_F32, M, K, N) == 0) == alone
    _every_type(M, K, N)


def _every_type(M, K, N):
    g = torch.Generator().manual_seed(M + K + N)
    x, W = torch.randn(N, K, generator=g).to(DEV), bs.bs_mx4_pack(torch.randn(M, K, generator=g).to(DEV))
    bias = torch.randn(M, generator=g).to(DEV)
    Xq, Wq = bs.bs_mx4_unpack(*bs.bs_mx4_pack(x), K).double(), bs.bs_mx4_unpack(*W, K).double()
    for dtype in TYPES:
        xd = x.to(dtype)
        q = Xq if dtype == torch.float32 else bs.bs_mx4_unpack(*bs.bs_mx4_pack(xd), K).double()
        want = q @ Wq.t() + bias.double()
        y = bs.bs_mx4_gemm(*W, xd, bias=bias)
        size = q.abs() @ Wq.abs().t() + bias.double().abs()
        assert bool(((y.double() - want).abs() <= (-(-K // 64) + 18) * 2.0**-23 * size + torch.finfo(dtype).eps / 2 * want.abs() + 2.0**-149).all())
        # a place whose rows lie further apart, and nothing beside them
        place = torch.full((N + 2, M + 3), 7.0, dtype=dtype, device=DEV)
        bs.bs_mx4_gemm(*W, xd, bias=bias, out=place[1:N + 1, 1:M + 1])
        assert torch.equal(place[1:N + 1, 1:M + 1], y)
        place[1:N + 1, 1:M + 1] = 7.0
        assert bool((place == 7.0).all())
