"""The calls for several hypotheses run together, as a search runs them: products in MX 4-bit, the choice, and the states that follow it;
captured, on another stream, and both ways from Python."""
import pytest
import torch

from mx4_reference import packed, quantise, values
from paper_1811_00206_amd import binding as bs
from test_gpu_beam import reference
from test_gpu_mx4 import _bound

pytestmark = pytest.mark.gpu


class Model:
    """A small recurrent model, and a search over it: h = tanh(A [x ; h]), logits = O h + bias."""

    def __init__(self, words=1003, units=160, beams=4, sequences=3, dtype=torch.float32, seed=0):
        g = torch.Generator().manual_seed(seed)
        self.B, self.W, self.units, self.dtype = sequences, beams, units, dtype
        self.embedding = torch.randn(words, units, generator=g).to(dtype).cuda()
        self.A = bs.bs_mx4_pack((torch.randn(units, 2 * units, generator=g) * units**-0.5).cuda())
        self.O = bs.bs_mx4_pack((torch.randn(words, units, generator=g) * 4 * units**-0.5).cuda())
        self.bias = torch.randn(words, generator=g).cuda()
        self.end = 17

    def start(self):
        B, W = self.B, self.W
        s = {"h": torch.zeros(B * W, self.units, dtype=self.dtype, device="cuda"), "tokens": torch.zeros(B, W, dtype=torch.int32, device="cuda"),
             "scores": torch.full((B, W), -float("inf"), device="cuda"), "finished": torch.zeros(B, W, dtype=torch.bool, device="cuda"),
             "text": torch.zeros(B, W, 20, dtype=torch.int32, device="cuda")}
        s["scores"][:, 0] = 0
        return s

    def step(self, s, t):
        x = torch.cat((self.embedding[s["tokens"].flatten().long()], s["h"]), 1)
        s["h"] = torch.tanh(bs.bs_mx4_gemm(*self.A, x))
        logits = bs.bs_mx4_gemm(*self.O, s["h"], bias=self.bias)
        before = s["scores"], s["finished"]
        s["scores"], s["tokens"], parents, s["finished"] = bs.bs_beam_step(logits, s["scores"], s["finished"], end=self.end)
        text = s["text"].clone()
        bs.bs_beam_reorder([s["h"], s["text"]], parents)
        s["text"][:, :, t] = s["tokens"]
        return x, logits, before, parents, text


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("beams,sequences", [(1, 1), (4, 3), (8, 20)])
def test_a_search(dtype, beams, sequences):
    m = Model(beams=beams, sequences=sequences, dtype=dtype)
    s = m.start()
    O = values(*m.O, m.units)
    for t in range(8):
        h_before = s["h"].clone()
        x, logits, (scores, finished), parents, text = m.step(s, t)
        # the logits are those of the hidden states that were multiplied, the choice that of the logits, the states their parents'
        h = torch.tanh(bs.bs_mx4_gemm(*m.A, x))
        q = values(packed(quantise(h)[0]), quantise(h)[1], m.units)
        want = q @ O.t() + m.bias.double().cpu()
        assert bool(((logits.double().cpu() - want).abs() <= _bound(O, q, want, dtype, m.units, m.bias)).all())
        rows = reference(logits, scores, finished, m.end, beams)
        assert s["tokens"].tolist() == [[r[1] for r in row] for row in rows] and parents.tolist() == [[r[2] for r in row] for row in rows]
        assert s["finished"].tolist() == [[r[3] for r in row] for row in rows]
        at = (parents.long() + beams * torch.arange(sequences, device="cuda").unsqueeze(1)).flatten()
        assert torch.equal(s["h"], h[at]) and torch.equal(s["text"].view(sequences * beams, -1)[:, :t], text.view(sequences * beams, -1)[at][:, :t])
        assert not torch.equal(s["h"], h_before) and bool((s["scores"][:, :-1] >= s["scores"][:, 1:]).all())


def _inputs(dtype=torch.float32, seed=0):
    g = torch.Generator().manual_seed(seed)
    return {"x": torch.randn(12, 1500, generator=g).to(dtype).cuda(), "scores": torch.sort(torch.randn(3, 4, generator=g), -1, descending=True).values.cuda(),
            "state": torch.randn(12, 333, generator=g).cuda(), "text": torch.randint(0, 99, (3, 4, 9), generator=g, dtype=torch.int32).cuda()}


def test_captured_steps_replay():
    """Two graphs that share a workspace, replayed in turns with eager work between them: every replay is the eager result."""
    W, bias = bs.bs_mx4_pack(torch.randn(5000, 1500, device="cuda")), torch.randn(5000, device="cuda")
    need = max(bs.bs_mx4_gemm_workspace_bytes(bs.BS_F32, 5000, 1500, 12), bs.bs_beam_step_workspace_bytes(bs.BS_F32, 3, 4, 5000, 4))
    workspace = torch.empty(need, dtype=torch.uint8, device="cuda")

    def run(i):
        logits = bs.bs_mx4_gemm(*W, i["x"], bias=bias, workspace=workspace)
        out = bs.bs_beam_step(logits, i["scores"], end=5, workspace=workspace)
        bs.bs_beam_reorder([i["state"], i["text"]], out[2])
        return [logits, *out]

    static = [_inputs(seed=n) for n in (1, 2)]
    run(_inputs())      # first launches
    torch.cuda.synchronize()
    graphs, results = [], []
    for i in static:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            results.append(run(i))
        graphs.append(graph)
    for replay in range(3):
        for n, graph in enumerate(graphs):
            fresh = _inputs(seed=10 * replay + n)
            for k in fresh:
                static[n][k].copy_(fresh[k])
            graph.replay()
            want = run(fresh)
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(results[n], want))
            assert torch.equal(static[n]["state"], fresh["state"]) and torch.equal(static[n]["text"], fresh["text"])


class Nothing:
    """Native calls that leave everything to the long way."""

    def __init__(self, native):
        self.native = native

    def __getattr__(self, name):
        return getattr(self.native, name) if name in ("stream", "device") else lambda *args: None


def _calls(dtype):
    g = torch.Generator().manual_seed(5)
    W, W3, x = torch.randn(50, 130, generator=g).to(dtype).cuda(), torch.randn(2, 3, 40, generator=g).to(dtype).cuda(), torch.randn(9, 140, generator=g).to(dtype).cuda()
    bias, logits = torch.randn(50, generator=g).cuda(), torch.randn(12, 700, generator=g).to(dtype).cuda()
    scores, done = torch.randn(3, 4, generator=g).cuda(), torch.rand(3, 4, generator=g).cuda() < 0.3
    states = [torch.randn(12, 33, generator=g).to(dtype).cuda(), torch.randint(0, 9, (3, 4, 5), generator=g).cuda()]

    def run():
        c, s = bs.bs_mx4_pack(W)
        c3, s3 = bs.bs_mx4_pack(W3)
        cs = bs.bs_mx4_pack(x[:, 3:133])
        out = [c, s, c3, s3, *cs, bs.bs_mx4_unpack(c, s, 130), bs.bs_mx4_unpack(c3, s3, 40, dtype=dtype)]
        out += [bs.bs_mx4_gemm(c, s, x[:, 5:135], bias=bias), bs.bs_mx4_gemm(c, s, x[0, :130]), bs.bs_mx4_gemm_packed(c, s, *cs, 130, dtype=dtype)]
        out.append(bs.bs_mx4_gemm(c, s, x[:, :130], out=torch.empty((9, 60), dtype=dtype, device="cuda")[:, 3:53]))
        a = bs.bs_beam_step(logits, scores, done, end=3, n=6)
        out += [*a, *bs.bs_beam_step(logits, scores)]
        moved = [t.clone() for t in states]
        bs.bs_beam_reorder(moved, a[2][:, :4].contiguous())
        return out + moved + bs.bs_beam_reorder(states, a[2][:, 1:5].contiguous(), out=[torch.empty_like(t) for t in states])

    return run


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
def test_native_and_long_way(dtype, monkeypatch):
    run = _calls(dtype)
    want = run()
    monkeypatch.setattr(bs, "_native", Nothing(bs._native))
    got = run()
    assert len(want) == len(got)
    for a, b in zip(want, got):
        assert a.dtype == b.dtype and a.shape == b.shape and torch.equal(a, b)


def test_another_stream():
    """Behind work of that stream that the inputs wait for."""
    run = _calls(torch.float32)
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


# ---- offsets beyond 32 bits: what lies at the end is as it is by itself


@pytest.mark.parametrize("N", [1, 5, 70, 300])
def test_matrix_of_more_than_4_gib(N):
    M, K, last = (1 << 18) + 5, 33000, 37
    codes = torch.zeros((M, 64 * 258), dtype=torch.uint8, device="cuda")
    scales = torch.full((M, 4 * 258), 127, dtype=torch.uint8, device="cuda")
    end = bs.bs_mx4_pack(torch.randn((last, K), generator=torch.Generator().manual_seed(1)).cuda())
    codes[-last:], scales[-last:] = end
    assert codes.numel() > 2**32
    x = torch.randn((N, K), generator=torch.Generator().manual_seed(2)).cuda()
    y = bs.bs_mx4_gemm(codes, scales, x)
    q = values(packed(quantise(x)[0]), quantise(x)[1], K)
    W = values(*end, K)
    want = q @ W.t()
    assert bool(((y[:, -last:].double().cpu() - want).abs() <= _bound(W, q, want, torch.float32, K, None)).all())
    assert not bool(y[:, :-last].any())


def test_many_elements_and_rows():
    M, K = (1 << 18) + 5, 16500      # more than 2^32 elements
    W = torch.zeros((M, K), dtype=torch.bfloat16, device="cuda")
    W[-9:] = torch.randn((9, K), generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    codes, scales = bs.bs_mx4_pack(W)
    end = bs.bs_mx4_pack(W[-9:].clone())
    assert torch.equal(codes[-9:], end[0]) and torch.equal(scales[-9:], end[1]) and not bool(codes[:-9].any())
    W = bs.bs_mx4_unpack(codes, scales, K, out=W)
    assert torch.equal(W[-9:], bs.bs_mx4_unpack(*end, K, dtype=torch.bfloat16)) and not bool(W[:-9].any())
    del W, codes, scales
    # more than 2^32 results, rows of x behind 2^16
    x = torch.zeros((70000, 256), dtype=torch.bfloat16, device="cuda")
    x[-3:] = torch.randn((3, 256), generator=torch.Generator().manual_seed(3)).bfloat16().cuda()
    W = bs.bs_mx4_pack(torch.randn((65000, 256), generator=torch.Generator().manual_seed(4)).cuda())
    y = bs.bs_mx4_gemm(*W, x)
    q, w = values(packed(quantise(x[-3:])[0]), quantise(x[-3:])[1], 256), values(*W, 256)
    want = q @ w.t()
    assert bool(((y[-3:].double().cpu() - want).abs() <= _bound(w, q, want, torch.bfloat16, 256, None)).all()) and not bool(y[:-3].any())


def test_logits_and_states_of_more_than_4_gib():
    B, W, V = 2200, 16, 128000
    logits = torch.zeros((B * W, V), dtype=torch.bfloat16, device="cuda")
    assert logits.numel() > 2**32
    g = torch.Generator().manual_seed(1)
    logits[-W:] = torch.randn((W, V), generator=g).bfloat16().cuda()
    scores = torch.randn((B, W), generator=g).cuda()
    got = bs.bs_beam_step(logits, scores, n=5)
    want = bs.bs_beam_step(logits[-W:].clone(), scores[-1:].clone(), n=5)
    # (many rows go to wavefronts, few to workgroups: their sums are added up in another order)
    assert all(torch.equal(a[-1:], b) for a, b in zip(got[1:], want[1:])) and torch.allclose(got[0][-1:], want[0], rtol=2.0**-23, atol=0)
    best = scores[:-1].argmax(-1)
    assert torch.equal(got[2][:-1, 0].long(), best) and bool((got[1][:-1] == torch.arange(5, device="cuda")).all())
    parents = torch.randint(0, W, (B, W), generator=g, dtype=torch.int32).cuda()
    end = logits[-W:].clone()
    bs.bs_beam_reorder(logits, parents)
    assert torch.equal(logits[-W:], end[parents[-1].long()]) and not bool(logits[:-W].any())
