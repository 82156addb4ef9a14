"""The two ways from Python to the calls on 4-bit matrices, expert layers and logits give the same bits, on the current stream."""
import pytest
import torch

from paper_1811_00206_amd import binding as bs

pytestmark = pytest.mark.gpu


class Nothing:
    """Native calls that leave everything to the long way."""

    def __getattr__(self, name):
        return lambda *args: None


def calls(dtype):
    g = torch.Generator().manual_seed(5)

    def normal(*shape):
        return torch.randn(shape, generator=g).to(dtype).cuda()

    group, W, w1, w2 = 64, normal(50, 130), normal(6, 80, 70), normal(6, 70, 40)
    x, x1, router, tokens = normal(9, 130), normal(130), normal(6, 70), normal(4, 70)
    logits, targets = normal(3, 40000), torch.tensor([5, -1, 39999]).cuda()
    gl, gh = torch.ones(3).cuda(), torch.full((3,), 0.5).cuda()

    def run():
        c, s = bs.bs_q4_pack(W, group)
        c1, s1 = bs.bs_q4_pack(w1, group)
        c2, s2 = bs.bs_q4_pack(w2, group)
        out = [c, s, c1, s1, bs.bs_q4_unpack(c, s, 130, group), bs.bs_q4_unpack(c1, s1, 70, group, dtype=dtype)]
        out += [bs.bs_q4_gemv(c, s, group, x), bs.bs_q4_gemv(c, s, group, x1), bs.bs_q4_gemv(c, s, group, x[:, :], out=torch.empty((9, 50), dtype=dtype, device="cuda"))]
        for renormalise in (True, False):
            out += bs.bs_q4_moe(tokens, router, c1, s1, c2, s2, group, 2, renormalise)
        lp = bs.bs_logprobs(logits, targets, top_n=7)
        out += lp
        out.append(bs.bs_logprobs_backward(logits, targets, lp[2], lp[1], gl, gh))
        out.append(bs.bs_logprobs_backward(logits, targets, lp[2], None, gl, None, out=torch.empty((3, 40000), dtype=dtype, device="cuda")))
        return out

    return run


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
def test_native_and_long_way(dtype, monkeypatch):
    run = calls(dtype)
    want = run()
    monkeypatch.setattr(bs, "_native", Nothing())
    got = run()
    assert len(want) == len(got)
    for a, b in zip(want, got):
        assert a.dtype == b.dtype and a.shape == b.shape and torch.equal(a, b)


def test_another_stream():
    """Behind work of that stream that the inputs wait for."""
    run = calls(torch.float32)
    want = run()
    x = torch.randn(4096, 4096, device="cuda")
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        for _ in range(3):
            x = x @ x * 1e-3
        got = run()
    stream.synchronize()
    for a, b in zip(want, got):
        assert torch.equal(a, b)
