"""What a language model needs to answer with several hypotheses at once, as cases that can be timed.

``pack``     a dense matrix to MX 4-bit (E2M1 codes, a power of two for every 32 elements), and back to the values the codes stand for
``gemm``     rows of activations, quantised in the call, times such a matrix
``beam``     one step of beam search: the best continuations over all beams and words of each sequence
``reorder``  the states of the beams follow that choice

``run`` makes the library's calls where ``own`` is true and computes the same in elementary torch operations where it is
false; ``exact`` computes it in 64 bits.  The sizes are those of ``paper_1811_00206_amd.workloads`` (a 1500-unit LSTM, a
4096 x 25088 layer, the 16384 x 8192 matrix), of the word-level example and generic ones.

Format of an MX matrix [M, K]: codes uint8 [M, 64 * ceil(K / 128)], element k in the low (k even) or high nibble of byte k // 2; bit 3
the sign, bits 0..2 one of the magnitudes 0, .5, 1, 1.5, 2, 3, 4, 6.  scales uint8 [M, 4 * ceil(K / 128)]: byte s of block k // 32 is
2**(s - 127), 255 no number.  Behind K: codes 0, and scales 127 for the blocks that hold nothing.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}
MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)

# no drawn case moves more bytes or does more operations than the largest listed ones
MAX_BYTES = 650_000_000
MAX_FLOPS = 1_100_000_000_000


def listed():
    return [
        # loading a model: the 1500-unit LSTM's gate matrix (rows of 3000: the last block is a ragged one)
        dict(name="pack_lstm1500", op="pack", M=6000, K=3000, dtype="f32"),
        # loading a large matrix stored in 16 bits
        dict(name="pack_16k_bf16", op="pack", M=16384, K=8192, dtype="bf16"),
        # output product of a word-level model, 10000 words, for one token of a 1500-unit model: latency of one call
        dict(name="gemm_words_f32_n1", op="gemm", M=10000, K=1500, N=1, dtype="f32", bias=True),
        # decoding one token through the largest matrix
        dict(name="gemm_16k_bf16_n1", op="gemm", M=16384, K=8192, N=1, dtype="bf16", bias=False),
        # a long row and a ragged batch of tokens
        dict(name="gemm_fc6_f16_n77", op="gemm", M=4096, K=25088, N=77, dtype="f16", bias=False),
        # one step of 32 sequences with 8 beams each over an odd vocabulary
        dict(name="gemm_beams_bf16_n256", op="gemm", M=32003, K=1500, N=256, dtype="bf16", bias=True),
        # a long prompt through the largest matrix
        dict(name="gemm_16k_bf16_n4096", op="gemm", M=16384, K=8192, N=4096, dtype="bf16", bias=False),
        # one sequence of the word-level model with 4 beams
        dict(name="beam_words_f32", op="beam", B=1, W=4, V=10000, dtype="f32", banned=0.0, ended=0.0),
        # 32 sequences with 8 beams, an odd vocabulary, some words banned, some beams at their end
        dict(name="beam_32x8_bf16", op="beam", B=32, W=8, V=32003, dtype="bf16", banned=0.01, ended=0.1),
        # many sequences with wide beams
        dict(name="beam_256x16_bf16", op="beam", B=256, W=16, V=32003, dtype="bf16", banned=0.0, ended=0.0),
        # the word-level model's hidden and cell state and history, one sequence
        dict(name="reorder_words", op="reorder", B=1, W=4, states=2, width=1500, history=50, dtype="f32"),
        # many sequences of a model of several layers
        dict(name="reorder_256x16", op="reorder", B=256, W=16, states=8, width=2048, history=513, dtype="bf16"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    """One more case: matrices of 64 .. 32768 rows and 64 .. 25088 columns, 1 .. 4096 tokens, vocabularies of 1000 .. 160000 words,
    1 .. 256 sequences with 1 .. 16 beams, up to 8 state tensors a beam, odd sizes throughout, every type."""
    while True:
        op = rng.choice(("pack", "gemm", "gemm", "beam", "reorder"))
        case = {"op": op, "dtype": rng.choice(("f32", "f16", "bf16"))}
        if op in ("pack", "gemm"):
            case |= {"M": _log_int(rng, 64, 32768), "K": _log_int(rng, 64, 25088)}
            if op == "gemm":
                case |= {"N": rng.choice((1, _log_int(rng, 1, 4096), _log_int(rng, 1, 4096))), "bias": rng.random() < 0.5}
        else:
            case |= {"B": _log_int(rng, 1, 256), "W": _log_int(rng, 1, 16)}
            if op == "beam":
                case |= {"V": _log_int(rng, 1000, 160000), "banned": rng.choice((0.0, 0.01)), "ended": rng.choice((0.0, 0.1))}
                if case["B"] * case["W"] * case["V"] > 256 * 16 * 32003:
                    continue
            else:
                case |= {"states": rng.randint(1, 8), "width": _log_int(rng, 64, 4096), "history": _log_int(rng, 1, 1024)}
        w = work(case)
        if w["bytes"] <= MAX_BYTES and w["flops"] <= MAX_FLOPS:
            return case


# ---- the plain forms


def _blocks(x):
    """[.., K] -> fp32 [.., 4 * ceil(K / 128), 32], zeros behind K"""
    return torch.nn.functional.pad(x.float(), (0, -x.shape[-1] % 128)).unflatten(-1, (-1, 32))


def _exponents(G):
    """The scale bytes of blocks [.., 32]: two below the exponent of the largest magnitude."""
    most = G.abs().amax(-1).contiguous()
    s = ((most.view(torch.int32) >> 23) - 2).clamp(min=0)
    return torch.where(most < math.inf, s, torch.full_like(s, 255))


def _times(x, e):
    """x * 2**e in 32 bits, -140 < e < 140: two powers, made of their bits"""
    half = e // 2
    return x * ((half + 127) << 23).view(torch.float32) * ((e - half + 127) << 23).view(torch.float32)


def _levels(G, s):
    """The E2M1 codes of blocks whose scale bytes are s; halfway cases to the even code."""
    a = _times(G.abs(), (127 - s).unsqueeze(-1))
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75).to(torch.uint8) + (a > 1.25).to(torch.uint8) + (a >= 1.75).to(torch.uint8)
            + (a > 2.5).to(torch.uint8) + (a >= 3.5).to(torch.uint8) + (a > 5.0).to(torch.uint8))
    return code | ((G < 0).to(torch.uint8) << 3)


def _quantise(W):
    """codes and scales of a matrix [M, K]"""
    K = W.shape[-1]
    G = _blocks(W)
    s = _exponents(G)
    code = _levels(G, s).flatten(-2)
    s[..., -(-K // 32):] = 127
    return code[..., 0::2] | (code[..., 1::2] << 4), s.to(torch.uint8)


def _scale(s):
    """2**(s - 127) in 32 bits"""
    s = s.int().unsqueeze(-1)
    return torch.where(s == 255, math.nan, _times(1.0, s - 127))


def _values(codes, scales, K):
    """The values that codes and scales stand for, in 32 bits."""
    table = torch.tensor([*MAGNITUDES, *(-m for m in MAGNITUDES)], device=codes.device)
    v = torch.stack((table[(codes & 15).int()], table[(codes >> 4).int()]), -1).flatten(-2)
    return (v.unflatten(-1, (-1, 32)) * _scale(scales)).flatten(-2)[..., :K]


def _rounded(x):
    """The values that x's own MX form stands for, in 32 bits."""
    return _values(*_quantise(x), x.shape[-1])


def _ordered(x):
    """64-bit whole numbers in the order of the logits, the lower index first among equals."""
    i = (x + 0.0).view(torch.int32)
    i = (i ^ ((i >> 31) & 0x7FFFFFFF)).long()
    return i * 2**32 + (2**32 - 1 - torch.arange(x.shape[-1], device=x.device))


def _largest(x, n):
    key = torch.topk(_ordered(x), n, -1).values
    return 2**32 - 1 - (key & (2**32 - 1))


# ---- what is measured


def prepare(case, seed):
    """Weights ~ N(0, 1/sqrt(K)) in MX form, activations ~ N(0, 1) as a norm leaves them, logits of a spread of 3 with a few banned words,
    scores of beams some words into their text, a few of them at their end; states ~ N(0, 1) and the parents that such a step leaves."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    op, dtype = case["op"], DTYPES[case["dtype"]]

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    state = dict(case)
    if op == "pack":
        state["W"] = (normal(case["M"], case["K"]) * case["K"] ** -0.5).to(dtype)
    elif op == "gemm":
        state["codes"], state["scales"] = _quantise(normal(case["M"], case["K"]) * case["K"] ** -0.5)
        state["x"] = normal(case["N"], case["K"]).to(dtype)
        state["b"] = normal(case["M"]) if case["bias"] else None
    elif op == "beam":
        B, W, V = case["B"], case["W"], case["V"]
        logits = normal(B * W, V) * 3.0
        if case["banned"]:
            logits.masked_fill_(torch.rand(V, generator=gen, device="cuda") < case["banned"], -math.inf)
        state["logits"] = logits.to(dtype)
        state["scores"] = torch.sort(-20.0 + 2.0 * normal(B, W), dim=-1, descending=True).values
        state["finished"] = torch.rand((B, W), generator=gen, device="cuda") < case["ended"]
    else:
        B, W = case["B"], case["W"]
        state["tensors"] = [normal(B * W, case["width"]).to(dtype) for _ in range(case["states"])]
        state["tensors"].append(torch.randint(0, 10000, (B * W, case["history"]), generator=gen, device="cuda", dtype=torch.int32))
        state["spare"] = [torch.empty_like(t) for t in state["tensors"]]
        state["parents"] = torch.randint(0, W, (B, W), generator=gen, device="cuda", dtype=torch.int32)
    return state


def run(state):
    return _own(state) if own else _plain(state)


def _own(s):
    from paper_1811_00206_amd import binding as bs
    op = s["op"]
    if op == "pack":
        codes, scales = bs.bs_mx4_pack(s["W"])
        return bs.bs_mx4_unpack(codes, scales, s["K"], dtype=s["W"].dtype)
    if op == "gemm":
        return bs.bs_mx4_gemm(s["codes"], s["scales"], s["x"], bias=s["b"])
    if op == "beam":
        scores, tokens, parents, finished = bs.bs_beam_step(s["logits"], s["scores"], s["finished"], end=0)
        return {"scores": scores, "tokens": tokens, "parents": parents, "finished": finished}
    return bs.bs_beam_reorder(s["tensors"], s["parents"], out=s["spare"])


def _plain(s):
    op = s["op"]
    if op == "pack":
        return _rounded(s["W"]).to(s["W"].dtype)
    if op == "gemm":
        y = _rounded(s["x"]) @ _values(s["codes"], s["scales"], s["K"]).t()
        return (y if s["b"] is None else y + s["b"]).to(s["x"].dtype)
    B, W = s["B"], s["W"]
    if op == "beam":
        # 64 bits for what orders the words of different beams
        x, score, done = s["logits"].float(), s["scores"].double(), s["finished"]
        m = x.amax(-1, keepdim=True).double()
        lse = (m + (x.double() - m).exp().sum(-1, keepdim=True).log())
        word = _largest(x, W)
        total = score.unsqueeze(-1) + (x.gather(-1, word).double() - lse).view(B, W, W)
        word = word.view(B, W, W)
        first = torch.arange(W, device=x.device) == 0
        total = torch.where(done.unsqueeze(-1), torch.where(first, score.unsqueeze(-1), -math.inf), total).flatten(1)
        word = torch.where(done.unsqueeze(-1), 0, word).flatten(1)
        total, at = torch.sort(total, dim=-1, descending=True, stable=True)
        total, at = total[:, :W], at[:, :W]
        token, parent = word.gather(1, at), at // W
        return {"scores": total.float(), "tokens": token.int(), "parents": parent.int(), "finished": done.gather(1, parent) | (token == 0)}
    rows = (s["parents"].long() + W * torch.arange(B, device="cuda").unsqueeze(-1)).flatten()
    return [t[rows] for t in s["tensors"]]


def work(case):
    """Every input read once and every output written once; of the states the parents that beams have on average."""
    op, size = case["op"], SIZE[case["dtype"]]
    if op in ("pack", "gemm"):
        M, K = case["M"], case["K"]
        packed = M * 68 * -(-K // 128)
        if op == "pack":      # packed, and unpacked again
            return {"bytes": 2 * (M * K * size + packed), "flops": 2 * M * K}
        N = case["N"]
        return {"bytes": packed + N * (K + M) * size + (4 * M if case["bias"] else 0), "flops": 2 * M * K * N}
    B, W = case["B"], case["W"]
    if op == "beam":
        live = 1.0 - case["ended"]
        return {"bytes": round(live * B * W * case["V"] * size) + B * W * 18, "flops": round(live * 4 * B * W * case["V"])}
    row = case["states"] * case["width"] * size + 4 * case["history"]
    distinct = W * (1.0 - (1.0 - 1.0 / W) ** W)
    return {"bytes": round(B * (W + distinct) * row) + 4 * B * W, "flops": 0}


# ---- the same from the definitions, in 64 bits


def _power(e):
    """2**e in 64 bits"""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _real(codes, scales, K):
    """Values of an MX matrix in 64 bits: sign, exponent and mantissa bits of each code."""
    n = torch.empty(*codes.shape[:-1], 2 * codes.shape[-1], dtype=torch.uint8, device=codes.device)
    n[..., 0::2], n[..., 1::2] = codes % 16, codes // 16
    n = n[..., :K].int()
    exponent, mantissa = (n // 2) % 4, (n % 2).double()
    size = torch.where(exponent == 0, 0.5 * mantissa, (1 + 0.5 * mantissa) * _power(exponent - 1))
    block = torch.arange(K, device=codes.device) // 32
    return torch.where(n >= 8, -size, size) * _power(scales.int() - 127)[..., block]


def _nearest(x):
    """[M, K] -> the nearest value of each block's format, in 64 bits."""
    X, K = x.double(), x.shape[-1]
    block = torch.arange(K, device=x.device) // 32
    most = torch.zeros(X.shape[0], int(block[-1]) + 1, dtype=torch.float64, device=x.device)
    most = most.scatter_reduce(1, block.expand(X.shape[0], -1), X.abs(), "amax")
    exponent = (torch.frexp(most).exponent - 3).clamp(min=-127)
    scale = _power(torch.where(most == 0, -127, exponent))[:, block]
    out, best = torch.zeros_like(X), X.abs()
    for i in (2, 4, 6, 1, 3, 5, 7):          # even codes first, so that an odd one has to be nearer
        off = (X.abs() - MAGNITUDES[i] * scale).abs()
        nearer = off < best
        out, best = torch.where(nearer, MAGNITUDES[i] * scale, out), torch.where(nearer, off, best)
    return torch.where(X < 0, -out, out)


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "pack":
        return _nearest(s["W"])
    if op == "gemm":
        y = _nearest(s["x"]) @ _real(s["codes"], s["scales"], case["K"]).t()
        return y if s["b"] is None else y + s["b"].double()
    B, W = case["B"], case["W"]
    if op == "beam":
        V, out = case["V"], {"scores": [], "tokens": [], "parents": [], "finished": []}
        for b in range(B):
            total = torch.log_softmax(s["logits"][b * W:(b + 1) * W].double(), -1) + s["scores"][b].double().unsqueeze(-1)
            total[s["finished"][b]] = -math.inf
            total[:, 0] = torch.where(s["finished"][b], s["scores"][b].double(), total[:, 0])
            total, at = torch.sort(total.flatten(), descending=True, stable=True)
            out["scores"].append(total[:W])
            out["tokens"].append((at[:W] % V).int())
            out["parents"].append((at[:W] // V).int())
            out["finished"].append((at[:W] % V == 0) | s["finished"][b][at[:W] // V])
        return {k: torch.stack(v) for k, v in out.items()}
    out = []
    for t in s["tensors"]:
        beams = t.view(B, W, -1)
        index = s["parents"].long().unsqueeze(-1).expand(-1, -1, beams.shape[-1])
        out.append(torch.take_along_dim(beams, index, 1).view_as(t))
    return out
