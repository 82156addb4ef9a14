"""Products with 4-bit matrices of enough rows, or long enough ones, for every way in which the work is split, against the
definition in 64 bits.

Errors as in the tests of small matrices: each of K / 32 + 64 additions loses at most 2^-23 of the sum of magnitudes, then the result's own rounding."""
import functools

import pytest
import torch

from paper_1811_00206_amd import binding as bs
from test_gpu_q4 import ROUNDING, TYPES

pytestmark = pytest.mark.gpu


@functools.lru_cache(maxsize=1)
def matrix(M, K, group):
    """Random codes and scales and their values, all on the GPU."""
    g = torch.Generator(device="cuda").manual_seed(M + K)
    codes = torch.randint(0, 256, (M, 16 * -(-K // 32)), generator=g, device="cuda", dtype=torch.int32).byte()
    n = torch.stack((codes & 15, codes >> 4), -1).flatten(1)
    n[:, K:] = 0
    codes = n[:, 0::2] | n[:, 1::2] << 4
    scales = (torch.rand((M, -(-K // group)), generator=g, device="cuda") + 0.1).half()
    table = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64)
    W = torch.cat((table, -table)).cuda()[n[:, :K].int()]
    return codes, scales, W * scales.double().repeat_interleave(group, 1)[:, :K]


def check(M, K, group, N, dtype, pitch):
    codes, scales, W = matrix(M, K, group)
    room = torch.randn((N, pitch), generator=torch.Generator().manual_seed(N)).to(TYPES[dtype]).cuda()
    x = room[:, pitch - K:]
    y = bs.bs_q4_gemv(codes, scales, group, x)
    X, Wt = x.double(), W.t().contiguous()
    want, size = X @ Wt, X.abs() @ Wt.abs()
    allowed = 2.0**-23 * (K / 32 + 64) * size + ROUNDING[TYPES[dtype]] * want.abs()
    off = (y.double() - want).abs()
    assert y.dtype == TYPES[dtype] and y.shape == (N, M)
    assert bool((off <= allowed).all()), float((off / allowed).max())
    assert torch.equal(y, bs.bs_q4_gemv(codes, scales, group, x)), "another call, other bits"


@pytest.mark.parametrize("pitch", [304, 307], ids=["aligned", "odd"])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("N", [1, 2, 5, 17, 33])
@pytest.mark.parametrize("M,K,group", [(5121, 304, 32), (5121, 297, 64), (16400, 304, 128), (16400, 299, 32)])
def test_many_rows(M, K, group, N, dtype, pitch):
    check(M, K, group, N, dtype, pitch)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("M,K,group,N", [(16400, 4200, 64, 1), (16400, 4200, 64, 4), (16400, 8192, 32, 5), (9409, 22330, 128, 6), (5121, 9000, 64, 20)])
def test_many_rows_that_are_long(M, K, group, N, dtype):
    check(M, K, group, N, dtype, K)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,K,group,N", [(40, 200, 128, 1), (40, 200, 32, 3), (5121, 304, 128, 2), (16400, 304, 128, 1), (33, 9000, 128, 5), (300, 1000, 128, 40)])
def test_activations_near_the_largest_number(M, K, group, N, dtype):
    """Small scales times large activations: finite, though the sum of code times activation is not."""
    codes, scales, W = matrix(M, K, group)
    scales, W = (scales * 2.0**-8).half(), W * 2.0**-8      # exact: scales are 0.1 to 1.1
    x = (torch.randn((N, K), generator=torch.Generator().manual_seed(K)) * 2.0**(125 if K <= 1000 else 122)).to(TYPES[dtype]).cuda()
    y = bs.bs_q4_gemv(codes, scales, group, x)
    X, Wt = x.double(), W.t().contiguous()
    want, size = X @ Wt, X.abs() @ Wt.abs()
    assert float(size.max()) < 3.4e38
    off = (y.double() - want).abs()
    allowed = 2.0**-23 * (K / 32 + 64) * size + ROUNDING[TYPES[dtype]] * want.abs()
    assert bool((off <= allowed).all()), float((off / allowed).max())


@pytest.mark.parametrize("dtype,size_of", [("f32", 2.0**-98), ("bf16", 2.0**-110), ("f16", 2.0**-15)])
@pytest.mark.parametrize("M,K,group,N", [(40, 200, 128, 1), (40, 200, 32, 3), (33, 9000, 128, 5), (300, 1000, 128, 40)])
def test_small_activations(M, K, group, N, dtype, size_of):
    """Products are small numbers, still normal ones, and keep their bits (binary16's own smallest numbers among the activations)."""
    codes, scales, W = matrix(M, K, group)
    x = (torch.randn((N, K), generator=torch.Generator().manual_seed(K)) * size_of).to(TYPES[dtype]).cuda()
    y = bs.bs_q4_gemv(codes, scales, group, x)
    X, Wt = x.double(), W.t().contiguous()
    want, size = X @ Wt, X.abs() @ Wt.abs()
    off = (y.double() - want).abs()
    allowed = 2.0**-23 * (K / 32 + 64) * size + ROUNDING[TYPES[dtype]] * want.abs() + (2.0**-25 if dtype == "f16" else 0.0)
    assert bool((off <= allowed).all()), float((off / allowed).max())
