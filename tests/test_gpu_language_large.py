"""4-bit matrices, expert layers and logits whose offsets pass 32 bits: what lies at the end is as it is by itself."""
import pytest
import torch

from paper_1811_00206_amd import binding as bs

pytestmark = pytest.mark.gpu


def test_matrix_of_more_than_4_gib():
    M, K, last, group = (1 << 18) + 5, 33000, 37, 64      # 8.1 GiB of elements in 16 bits, 4.03 GiB of codes
    W = torch.zeros((M, K), dtype=torch.bfloat16, device="cuda")
    W[-last:] = torch.randn((last, K), generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    assert W.numel() > 2**32 and M * bs.bs_q4_codes_bytes(1, K) > 2**32
    codes, scales = bs.bs_q4_pack(W, group)
    end = bs.bs_q4_pack(W[-last:].clone(), group)
    assert torch.equal(codes[-last:], end[0]) and torch.equal(scales[-last:], end[1])
    assert not bool(codes[:-last].any())
    for dtype, N in ((torch.float32, 1), (torch.bfloat16, 5)):
        x = torch.randn((N, K), generator=torch.Generator().manual_seed(2)).to(dtype).cuda()
        y = bs.bs_q4_gemv(codes, scales, group, x)
        want = bs.bs_q4_gemv(*end, group, x).float()
        torch.testing.assert_close(y[:, -last:].float(), want, rtol=2.0**-7 if dtype == torch.bfloat16 else 1e-5, atol=1e-2 if dtype == torch.bfloat16 else 1e-4)
        assert not bool(y[:, :-last].any())
    W = bs.bs_q4_unpack(codes, scales, K, group, out=W)
    assert torch.equal(W[-last:], bs.bs_q4_unpack(*end, K, group, dtype=torch.bfloat16)) and not bool(W[:-last].any())


def test_experts_of_more_than_4_gib():
    E, D, F, group = 70, 8192, 8200, 64
    w1 = torch.zeros((E, 2 * F, D // 2), dtype=torch.uint8, device="cuda")
    s1 = torch.zeros((E, 2 * F, D // group), dtype=torch.float16, device="cuda")
    w2 = torch.zeros((E, D, 16 * -(-F // 32)), dtype=torch.uint8, device="cuda")
    s2 = torch.zeros((E, D, -(-F // group)), dtype=torch.float16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    w1[-1] = torch.randint(0, 256, w1.shape[1:], generator=g, device="cuda").byte()
    w2[-1, :, :F // 2] = torch.randint(0, 256, (D, F // 2), generator=g, device="cuda").byte()
    s1[-1], s2[-1] = 0.01, 0.01
    assert w1.numel() > 2**32
    router = torch.zeros((E, D), device="cuda")
    router[-1] = 1.0
    x = torch.rand((2, D), generator=g, device="cuda")      # the last expert has the largest logit
    y, ids, weights = bs.bs_q4_moe(x, router, w1, s1, w2, s2, group, 1)
    assert bool((ids == E - 1).all()) and bool((weights == 1).all())
    want, _, _ = bs.bs_q4_moe(x, router[-1:], w1[-1:], s1[-1:], w2[-1:], s2[-1:], group, 1)
    assert bool(want.any()) and float((y - want).norm()) <= 1e-5 * float(want.norm())


def test_logits_of_more_than_2_to_the_32():
    T, V = 140000, 32003
    x = torch.zeros((T, V), dtype=torch.bfloat16, device="cuda")
    assert x.numel() > 2**32
    x[-3:] = torch.randn((3, V), generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    targets = torch.full((T,), V - 1, dtype=torch.int64, device="cuda")
    got = bs.bs_logprobs(x, targets, top_n=3)
    want = bs.bs_logprobs(x[-3:].clone(), targets[-3:], top_n=3)
    for a, b in zip(got, want):
        torch.testing.assert_close(a[-3:], b, rtol=1e-5, atol=1e-5)
        assert torch.equal(a[0], a[T - 4])
    gl, gh = torch.ones(T, device="cuda"), torch.full((T,), 0.5, device="cuda")
    end = bs.bs_logprobs_backward(x[-3:].clone(), targets[-3:], got[2][-3:], got[1][-3:], gl[-3:], gh[-3:])
    grad = bs.bs_logprobs_backward(x, targets, got[2], got[1], gl, gh, out=x)
    assert torch.equal(grad[-3:], end) and torch.equal(grad[0], grad[T - 4])
