"""Calls for several hypotheses at the borders of what they take: results beside what is read, and in its place."""
import pytest
import torch

from paper_1811_00206_amd import binding as bs
from test_gpu_beam import check, draw

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = (torch.float32, torch.float16, torch.bfloat16)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,K,N", [(48, 256, 4), (48, 256, 40), (256, 1024, 80)])
def test_products_beside_what_they_read(M, K, N, dtype):
    """All in one piece of memory, each next to the other: y in front of everything, in the middle and behind."""
    g = torch.Generator().manual_seed(M + N)
    W, x = bs.bs_mx4_pack(torch.randn(M, K, generator=g).to(DEV)), torch.randn(N, K, generator=g).to(dtype).to(DEV)
    X, bias = bs.bs_mx4_pack(x), torch.randn(M, generator=g).to(DEV)
    want = bs.bs_mx4_gemm(*W, x, bias=bias)
    parts, size = {"codes": W[0], "scales": W[1], "x": x, "x_codes": X[0], "x_scales": X[1], "bias": bias}, N * M * x.element_size()
    for order in (["y", *parts], ["codes", "x", "x_codes", "y", "scales", "x_scales", "bias"], [*parts, "y"]):
        lengths = {k: v.numel() * v.element_size() for k, v in parts.items()} | {"y": size}
        assert all(n % 16 == 0 for n in lengths.values())
        room, at, placed = torch.zeros(sum(lengths.values()), dtype=torch.uint8, device=DEV), 0, {}
        for k in order:
            like = want if k == "y" else parts[k]
            placed[k] = room[at:at + lengths[k]].view(like.dtype).view(like.shape)
            if k != "y":
                placed[k].copy_(like)
            at += lengths[k]
        y = placed["y"]
        assert torch.equal(bs.bs_mx4_gemm(placed["codes"], placed["scales"], placed["x"], bias=placed["bias"], out=y), want)
        y.zero_()
        assert torch.equal(bs.bs_mx4_gemm_packed(placed["codes"], placed["scales"], placed["x_codes"], placed["x_scales"], K, dtype=dtype, bias=placed["bias"], out=y), want)
        assert all(torch.equal(placed[k], v) for k, v in parts.items())


def test_a_product_over_its_operands_is_refused():
    M, K, N = 128, 512, 8
    codes, scales = bs.bs_mx4_pack(torch.randn(M, K, device=DEV))
    x_codes, x_scales = bs.bs_mx4_pack(torch.randn(N, K, device=DEV))
    kept = [t.clone() for t in (codes, scales, x_codes, x_scales)]
    for over in (codes, x_codes):
        out = over.flatten()[:N * 64 * 4].view(torch.float32)[: N * 16].view(N, 16)
        small = codes[:16], scales[:16]
        with pytest.raises(bs.BsError) as e:
            bs.bs_mx4_gemm_packed(*small, x_codes, x_scales, K, out=out)
        assert e.value.status == 3
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((codes, scales, x_codes, x_scales), kept))


@pytest.mark.parametrize("B,W,V", [(1, 4, 5000), (40, 7, 900), (150, 8, 1500)])
def test_a_step_in_place(B, W, V):
    """Scores and flags over those before: the same results."""
    import ctypes
    lib, g = bs.load_library(), torch.Generator().manual_seed(B)
    logits, scores = torch.randn(B * W, V, generator=g).to(DEV), torch.randn(B, W, generator=g).to(DEV)
    finished = (torch.rand(B, W, generator=g) < 0.3).to(DEV)
    want = bs.bs_beam_step(logits, scores, finished, end=3)
    tokens, parents = (torch.empty((B, W), dtype=torch.int32, device=DEV) for _ in range(2))
    workspace = torch.empty(bs.bs_beam_step_workspace_bytes(bs.BS_F32, B, W, V, W), dtype=torch.uint8, device=DEV)
    p = [ctypes.c_void_p(t.data_ptr()) for t in (logits, scores, finished, tokens, parents, workspace)]
    assert lib.bs_beam_step(p[0], 0, B, W, V, V, p[1], p[2], 3, W, p[1], p[3], p[4], p[2], p[5], workspace.numel(), ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)) == 0
    assert all(torch.equal(a, b) for a, b in zip((scores, tokens, parents, finished), want))


def _best(f):
    """Microseconds of a call in a graph of ten, the best of five replays."""
    f()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for _ in range(10):
            f()
    times = []
    for _ in range(6):
        begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        begin.record()
        graph.replay()
        end.record()
        end.synchronize()
        times.append(begin.elapsed_time(end) * 100)
    return min(times[1:])


@pytest.mark.parametrize("B,W,V,dtype", [(256, 16, 2000, torch.bfloat16), (64, 32, 8003, torch.float32)])
def test_a_few_more_hypotheses_take_little_longer(B, W, V, dtype):
    """Many rows of ordinary logits, as many hypotheses as there are lanes: no walk of the row for each of them."""
    g = torch.Generator(DEV).manual_seed(1)
    logits, scores = (torch.randn(B * W, V, generator=g, device=DEV) * 3).to(dtype), torch.randn(B, W, generator=g, device=DEV)
    workspace = torch.empty(max(bs.bs_beam_step_workspace_bytes(0, B, W, V, n) for n in (48, 64)), dtype=torch.uint8, device=DEV)
    few, many = (_best(lambda: bs.bs_beam_step(logits, scores, n=n, workspace=workspace)) for n in (48, 64))
    assert many < 3 * few, (few, many)      # a third more of a step's lists, and the join grows by their square: 1.8 times at most


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,W,V", [(16, 64, 200), (16, 64, 256), (16, 64, 257), (16, 64, 1000), (16, 64, 2000), (32, 64, 2500)])
def test_as_many_hypotheses_as_lanes(B, W, V, dtype):
    logits, scores = draw(B, W, V, dtype)
    for n in (57, 58, 64):
        check(logits, scores, n=n)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,W,V", [(512, 2, 2000), (1024, 2, 2500)])
def test_floods_of_many_rows(B, W, V, dtype):
    """A wavefront for a row: more words above the bound than its list takes, because all large ones come to few lanes; more or fewer of them
    than it has room for in a second pass."""
    rows, scores = draw(B, W, V, dtype)
    lane = torch.arange(V, device=DEV) // (16 // rows.element_size()) % 64
    for lanes, n in ((39, 40), (20, 21), (3, 5), (55, 57)):
        logits = torch.where(lane < lanes, rows.abs() + 4, -rows.abs())
        check(logits, scores, n=n)
    # a hundred words above many equal ones
    logits = torch.where(torch.arange(V, device=DEV) % 20 == 3, rows.abs() + 1, torch.ones_like(rows))
    check(logits, scores, n=33)
    check(logits, scores, n=57)


@pytest.mark.parametrize("V", [50, 3001, 40000])
def test_words_whose_scores_alone_are_equal(V):
    """Different logits that make the same total in 64 bits: in the order of the logits, not of the words, and cut to n by it; in one slice of a
    row, in several, and for all words where the beams' scores leave nothing of them."""
    logits = torch.full((4, V), -1.0, device=DEV)
    logits[:, V // 2] = 5.0
    small = [7, V // 2 + 1, V - 2, 21, V // 2 - 9]
    for i, at in enumerate(small):
        logits[:, at] = i * 1e-20
    scores = torch.tensor([[-1.0, -1.0], [-2.0, -1.0]], device=DEV)
    for n in (2, 3, 5, 6, 9):
        tokens = check(logits, scores, n=n)[1]
        assert tokens[1].tolist()[2:7] == small[::-1][:max(n - 2, 0)]      # behind both beams' best words, -1 and -2 here and -6 there
    g = torch.Generator().manual_seed(V)
    logits = torch.randn(6, V, generator=g).to(DEV)
    scores = torch.tensor([[-1e30, -1e30, -1e30], [-2e30, -1e30, 1e30]], device=DEV)
    for n in (1, 4, 11):
        tokens, parents = check(logits, scores, n=n)[1:3]
        assert parents.tolist() == [[0] * n, [2] * n]
        assert torch.equal(tokens.long(), torch.topk(logits[[0, 5]], n, -1).indices)
