"""MX 4-bit matrices from their definition, on the CPU and in 64 bits: what the tests of the calls compare with."""
import torch

MAGNITUDES = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)


def quantise(W):
    """W [M, K] -> (codes [M, 128 * chunks], one a byte, scale bytes [M, 4 * chunks])"""
    X = W.detach().cpu().double()
    M, K = X.shape
    chunks = -(-K // 128)
    G = torch.zeros(M, 128 * chunks, dtype=torch.float64)
    G[:, :K] = X
    G = G.view(M, 4 * chunks, 32)
    a = G.abs()
    bad = ~torch.isfinite(a).all(-1)
    a = torch.where(bad.unsqueeze(-1), 0.0, a)
    most = a.amax(-1)
    e = torch.where(most < 2.0**-126, 0, torch.frexp(most).exponent.long() - 1 + 127)      # the biased exponent as fp32
    s = (e - 2).clamp(min=0)
    q = torch.ldexp(a, (127 - s).unsqueeze(-1))
    off = (q.unsqueeze(-1) - MAGNITUDES).abs()
    off[..., 1::2] *= 1 + 1e-12          # the even code of two that are equally near (anything else is 2^-23 further or nearer)
    codes = off.argmin(-1) | (torch.signbit(G).long() << 3)
    codes[bad] = 0
    s = torch.where(bad, 255, s)
    s[:, -(-K // 32):] = 127
    return codes.view(M, 128 * chunks), s


def packed(codes):
    return (codes[:, 0::2] | (codes[:, 1::2] << 4)).to(torch.uint8)


def values(codes, scales, K):
    """What packed codes and scale bytes stand for, [M, K] in 64 bits."""
    codes, scales = codes.cpu().long(), scales.cpu().long()
    n = torch.stack((codes & 15, codes >> 4), -1).flatten(-2)
    v = MAGNITUDES[n & 7] * torch.where(n >= 8, -1.0, 1.0).double()
    s = torch.where(scales == 255, float("nan"), torch.ldexp(torch.ones(1, dtype=torch.float64), scales - 127))
    return (v.view(*scales.shape, 32) * s.unsqueeze(-1)).flatten(-2)[..., :K]
