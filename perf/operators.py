"""The operators of a language model that the library has beside its sparse products, as cases that can be timed.

``pack``      a dense matrix to 4-bit codes (E2M1) with binary16 group scales, and back to the values the codes stand for
``gemv``      such a matrix times one or a few vectors
``moe``       a whole mixture-of-experts layer on 4-bit expert matrices for a few tokens
``logprobs``  log probabilities of given tokens, the entropy of each row and its most likely alternatives
``grad``      the gradient of those log probabilities and entropies with respect to the logits

``run`` makes the library's calls where ``own`` is true and computes the same in elementary torch operations in 32 bits
where it is false; ``exact`` computes it in 64 bits.  The sizes are those of ``paper_1811_00206_amd.workloads`` (a 1500-unit
LSTM, a 4096 x 25088 layer, the 16384 x 8192 matrix) and generic ones.

Format of a 4-bit matrix [M, K]: codes uint8 [M, 16 * ceil(K / 32)], element k in the low (k even) or high nibble of byte
k // 2, zero codes behind K; bit 3 the sign, bits 0..2 one of the magnitudes 0, .5, 1, 1.5, 2, 3, 4, 6; scales float16
[M, ceil(K / group)].
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
MAX_FLOPS = 5_000_000_000


def listed():
    return [
        # loading a model: the 1500-unit LSTM's gate matrix (rows of 3000: the last group is a ragged one)
        dict(name="pack_lstm1500", op="pack", M=6000, K=3000, group=64, dtype="f32"),
        # loading a large matrix stored in 16 bits
        dict(name="pack_16k_bf16", op="pack", M=16384, K=8192, group=128, dtype="bf16"),
        # the smallest product: latency of one call
        dict(name="gemv_256", op="gemv", M=256, K=256, group=32, dtype="f32", N=1),
        # output product of a word-level model, 10000 words, for one token of a 1500-unit model
        dict(name="gemv_words_f32", op="gemv", M=10000, K=1500, group=32, dtype="f32", N=1),
        # decoding one token through the largest matrix
        dict(name="gemv_16k_bf16", op="gemv", M=16384, K=8192, group=64, dtype="bf16", N=1),
        # a long row and a ragged batch of tokens
        dict(name="gemv_fc6_f16_n13", op="gemv", M=4096, K=25088, group=128, dtype="f16", N=13),
        # an expert layer inside the 1500-unit model, one token
        dict(name="moe_1500_t1", op="moe", T=1, D=1500, F=1500, E=8, top_k=2, group=32, dtype="f32", renormalise=True),
        # many small experts, a few sequences decoded together
        dict(name="moe_e64_bf16_t7", op="moe", T=7, D=2048, F=1024, E=64, top_k=6, group=64, dtype="bf16", renormalise=False),
        # one decoded token over a large vocabulary, as a server reports it
        dict(name="logprobs_t1_f32", op="logprobs", T=1, V=131072, dtype="f32", top_n=20, banned=0.0),
        # scoring whole sequences, an odd vocabulary, some words banned
        dict(name="logprobs_4096_bf16", op="logprobs", T=4096, V=32003, dtype="bf16", top_n=5, banned=0.01),
        # one truncated back-propagation of a word-level model
        dict(name="grad_words_f32", op="grad", T=700, V=10000, dtype="f32", banned=0.0),
        # training on long sequences in 16 bits
        dict(name="grad_4096_bf16", op="grad", T=4096, V=32003, dtype="bf16", banned=0.01),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    """One more case: matrices of 64 .. 16384 rows and 64 .. 25088 columns, 1 .. 32 tokens, vocabularies of
    1000 .. 160000 words and 1 .. 4096 rows of logits, odd sizes throughout, every group size and type."""
    while True:
        op = rng.choice(("pack", "gemv", "gemv", "moe", "logprobs", "grad"))
        case = {"op": op, "dtype": rng.choice(("f32", "f16", "bf16"))}
        if op in ("pack", "gemv"):
            case |= {"M": _log_int(rng, 64, 16384), "K": _log_int(rng, 64, 25088), "group": rng.choice((32, 64, 128))}
            if op == "gemv":
                case["N"] = rng.choice((1, _log_int(rng, 1, 32)))
        elif op == "moe":
            E = rng.choice((4, 8, 16, 32, 60, 64))
            case |= {"T": rng.choice((1, _log_int(rng, 1, 16))), "D": _log_int(rng, 256, 4096), "F": _log_int(rng, 128, 4096),
                     "E": E, "top_k": rng.randint(1, min(8, E)), "group": rng.choice((32, 64, 128)),
                     "renormalise": rng.random() < 0.5}
            if 3 * E * case["D"] * case["F"] > 420_000_000:
                continue
        else:
            case |= {"T": _log_int(rng, 1, 4096), "V": _log_int(rng, 1000, 160000), "banned": rng.choice((0.0, 0.01))}
            if op == "logprobs":
                case["top_n"] = rng.choice((0, 1, 5, 20, rng.randint(2, 64)))
            if case["T"] * case["V"] > 4096 * 32003:
                continue
        w = work(case)
        if w["bytes"] <= MAX_BYTES and w["flops"] <= MAX_FLOPS:
            return case


# ---- the plain forms


def _quantise(W, group):
    """codes and scales of a matrix [.., M, K]: s = half(amax / 6), the nearest magnitude times s, halfway cases to the even code."""
    W = W.float()
    K = W.shape[-1]
    pad = -K % group
    G = torch.nn.functional.pad(W, (0, pad)).unflatten(-1, (-1, group))
    scales = (G.abs().amax(-1) / 6.0).clamp(max=65504.0).half()
    s = scales.float().unsqueeze(-1)
    a = G.abs()
    # the middle of two magnitudes times a binary16 scale is exact in 32 bits
    code = ((a > 0.25 * s).to(torch.uint8) + (a >= 0.75 * s).to(torch.uint8) + (a > 1.25 * s).to(torch.uint8)
            + (a >= 1.75 * s).to(torch.uint8) + (a > 2.5 * s).to(torch.uint8) + (a >= 3.5 * s).to(torch.uint8)
            + (a > 5.0 * s).to(torch.uint8))
    code = torch.where(s > 0, code, torch.zeros_like(code)) | ((G < 0).to(torch.uint8) << 3)
    code = code.flatten(-2)[..., :K]
    code = torch.nn.functional.pad(code, (0, -K % 32))
    return code[..., 0::2] | (code[..., 1::2] << 4), scales


def _values(codes, scales, K, group):
    """The values that codes and scales stand for, in 32 bits."""
    table = torch.tensor([*MAGNITUDES, *(-m for m in MAGNITUDES)], device=codes.device)
    v = torch.stack((table[(codes & 15).int()], table[(codes >> 4).int()]), -1).flatten(-2)[..., :K]
    s = scales.float().repeat_interleave(group, -1)[..., :K]
    return v * s


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
    """Weights ~ N(0, 1/sqrt(K)) in 4 bits, activations ~ N(0, 1) as a norm leaves them, router logits of a spread of about 2,
    logits of a spread of 3 with a few banned words and a few rows without a target."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    op, dtype = case["op"], DTYPES[case["dtype"]]

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    state = dict(case)
    if op == "pack":
        state["W"] = (normal(case["M"], case["K"]) * case["K"] ** -0.5).to(dtype)
    elif op == "gemv":
        state["codes"], state["scales"] = _quantise(normal(case["M"], case["K"]) * case["K"] ** -0.5, case["group"])
        state["x"] = normal(case["N"], case["K"]).to(dtype)
    elif op == "moe":
        E, D, F = case["E"], case["D"], case["F"]
        state["router"] = (normal(E, D) * (2.0 * D ** -0.5)).to(dtype)
        state["w1"], state["s1"] = _quantise(normal(E, 2 * F, D) * D ** -0.5, case["group"])
        state["w2"], state["s2"] = _quantise(normal(E, D, F) * F ** -0.5, case["group"])
        state["x"] = normal(case["T"], D).to(dtype)
    else:
        T, V = case["T"], case["V"]
        logits = normal(T, V) * 3.0
        target = torch.randint(0, V, (T,), generator=gen, device="cuda")
        if case["banned"]:
            banned = torch.rand(V, generator=gen, device="cuda") < case["banned"]
            banned[0] = False
            target = torch.where(banned[target], torch.zeros_like(target), target)
            logits.masked_fill_(banned, -math.inf)
        if T > 1:
            target[torch.rand(T, generator=gen, device="cuda") < 0.05] = -1
        state["logits"], state["target"] = logits.to(dtype), target
        if op == "grad":
            x = state["logits"].float()
            state["lse"] = torch.logsumexp(x, -1)
            logp = x - state["lse"].unsqueeze(-1)
            state["entropy"] = -torch.where(logp > -math.inf, logp.exp() * logp, torch.zeros_like(logp)).sum(-1)
            state["g_logprob"], state["g_entropy"] = normal(T) / T, normal(T) * (0.01 / T)
    return state


def run(state):
    return _own(state) if own else _plain(state)


def _own(s):
    from paper_1811_00206_amd import binding as bs
    op = s["op"]
    if op == "pack":
        codes, scales = bs.bs_q4_pack(s["W"], s["group"])
        return bs.bs_q4_unpack(codes, scales, s["K"], s["group"], dtype=s["W"].dtype)
    if op == "gemv":
        return bs.bs_q4_gemv(s["codes"], s["scales"], s["group"], s["x"])
    if op == "moe":
        y, ids, weights = bs.bs_q4_moe(s["x"], s["router"], s["w1"], s["s1"], s["w2"], s["s2"], s["group"], s["top_k"],
                                       renormalise=s["renormalise"])
        return {"y": y, "ids": ids, "weights": weights}
    if op == "logprobs":
        logprob, entropy, lse, values, ids = bs.bs_logprobs(s["logits"], s["target"], top_n=s["top_n"])
        return {"logprob": logprob, "entropy": entropy, "lse": lse, "top_values": values, "top_ids": ids}
    return bs.bs_logprobs_backward(s["logits"], s["target"], s["lse"], s["entropy"], s["g_logprob"], s["g_entropy"])


def _plain(s):
    op = s["op"]
    if op == "pack":
        codes, scales = _quantise(s["W"], s["group"])
        return _values(codes, scales, s["K"], s["group"]).to(s["W"].dtype)
    if op == "gemv":
        K = s["x"].shape[-1]
        return (s["x"].float() @ _values(s["codes"], s["scales"], K, s["group"]).t()).to(s["x"].dtype)
    if op == "moe":
        x, E, F = s["x"].float(), s["E"], s["F"]
        logits = x @ s["router"].float().t()
        ids = _largest(logits, s["top_k"])
        e = (logits - logits.amax(-1, keepdim=True)).exp()
        chosen = e.gather(-1, ids)
        weights = chosen / (chosen if s["renormalise"] else e).sum(-1, keepdim=True)
        dense = torch.zeros_like(logits).scatter(-1, ids, weights)          # [T, E], zero where not chosen
        a = torch.bmm(x.expand(E, -1, -1), _values(s["w1"], s["s1"], s["D"], s["group"]).transpose(1, 2).contiguous())
        g, u = a[..., :F], a[..., F:]
        h = g / (1.0 + (-g).exp()) * u
        y = torch.bmm(h, _values(s["w2"], s["s2"], F, s["group"]).transpose(1, 2).contiguous())
        y = (y * dense.t().unsqueeze(-1)).sum(0)
        return {"y": y.to(s["x"].dtype), "ids": ids.int(), "weights": weights}
    x, target = s["logits"].float(), s["target"]
    none = target < 0
    at = target.clamp(min=0).unsqueeze(-1)
    if op == "logprobs":
        m = x.amax(-1, keepdim=True)
        e = (x - m).exp()
        total = e.sum(-1, keepdim=True)
        lse = m + total.log()
        logp = x - lse
        entropy = -torch.where(e > 0, e / total * logp, torch.zeros_like(e)).sum(-1)
        ids = _largest(x, s["top_n"])
        logprob = torch.where(none, torch.zeros_like(entropy), logp.gather(-1, at).squeeze(-1))
        return {"logprob": logprob, "entropy": entropy, "lse": lse.squeeze(-1), "top_values": logp.gather(-1, ids), "top_ids": ids.int()}
    logp = x - s["lse"].unsqueeze(-1)
    p = logp.exp()
    g = torch.where(none, torch.zeros_like(s["g_logprob"]), s["g_logprob"]).unsqueeze(-1)
    d = -p * g - torch.where(p > 0, s["g_entropy"].unsqueeze(-1) * p * (logp + s["entropy"].unsqueeze(-1)), torch.zeros_like(p))
    return d.scatter_add(-1, at, g).to(s["logits"].dtype)


def work(case):
    """Every input read once and every output written once.  Experts: those that T tokens are expected to choose."""
    op, size = case["op"], SIZE[case["dtype"]]
    if op in ("pack", "gemv"):
        M, K = case["M"], case["K"]
        packed = M * (16 * -(-K // 32) + 2 * -(-K // case["group"]))
        if op == "pack":      # packed, and unpacked again
            return {"bytes": 2 * (M * K * size + packed), "flops": 2 * M * K}
        return {"bytes": packed + case["N"] * (K + M) * size, "flops": 2 * M * K * case["N"]}
    if op == "moe":
        T, D, F, E, k, G = (case[n] for n in ("T", "D", "F", "E", "top_k", "group"))
        active = E * (1.0 - (1.0 - k / E) ** T)
        expert = 2 * F * (16 * -(-D // 32) + 2 * -(-D // G)) + D * (16 * -(-F // 32) + 2 * -(-F // G))
        return {"bytes": round(active * expert) + size * (E * D + 2 * T * D) + 8 * T * k,
                "flops": 2 * T * E * D + 6 * T * k * F * D}
    T, V = case["T"], case["V"]
    if op == "logprobs":
        return {"bytes": T * V * size + T * (20 + 8 * case["top_n"]), "flops": 5 * T * V}
    return {"bytes": 2 * T * V * size + 24 * T, "flops": 6 * T * V}


# ---- the same from the definitions, in 64 bits


def _real(codes, scales, K, group):
    """Values of a 4-bit matrix in 64 bits: sign, exponent and mantissa bits of each code."""
    n = torch.empty(*codes.shape[:-1], 2 * codes.shape[-1], dtype=torch.uint8, device=codes.device)
    n[..., 0::2], n[..., 1::2] = codes % 16, codes // 16
    n = n[..., :K].long()
    exponent, mantissa = (n // 2) % 4, (n % 2).double()
    size = torch.where(exponent == 0, 0.5 * mantissa, (1 + 0.5 * mantissa) * torch.pow(2.0, (exponent - 1).double()))
    column = torch.arange(K, device=codes.device) // group
    return torch.where(n >= 8, -size, size) * scales.double()[..., column]


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "pack":
        W, K, group = s["W"].double(), case["K"], case["group"]
        column = torch.arange(K, device=W.device) // group
        most = torch.zeros(W.shape[0], -(-K // group), dtype=torch.float64, device=W.device)
        most = most.scatter_reduce(1, column.expand(W.shape[0], -1), W.abs(), "amax")
        scale = (most.float() / 6.0).clamp(max=65504.0).half().double()[:, column]     # the scale's own rounding is part of the format
        out, best = torch.zeros_like(W), W.abs()
        for i in (2, 4, 6, 1, 3, 5, 7):          # even codes first, so that an odd one has to be nearer
            off = (W.abs() - MAGNITUDES[i] * scale).abs()
            nearer = (off < best) & (scale > 0)
            out, best = torch.where(nearer, MAGNITUDES[i] * scale, out), torch.where(nearer, off, best)
        return torch.where(W < 0, -out, out)
    if op == "gemv":
        return s["x"].double() @ _real(s["codes"], s["scales"], case["K"], case["group"]).t()
    if op == "moe":
        x, T = s["x"].double(), case["T"]
        logits = x @ s["router"].double().t()
        ids = torch.sort(logits, dim=-1, descending=True, stable=True).indices[:, :case["top_k"]]
        weights = torch.softmax(logits, -1).gather(-1, ids)
        if case["renormalise"]:
            weights = weights / weights.sum(-1, keepdim=True)
        y = torch.zeros(T, case["D"], dtype=torch.float64, device=x.device)
        for e in ids.unique().tolist():
            a = x @ _real(s["w1"][e], s["s1"][e], case["D"], case["group"]).t()
            h = torch.nn.functional.silu(a[:, :case["F"]]) * a[:, case["F"]:]
            y += (h @ _real(s["w2"][e], s["s2"][e], case["F"], case["group"]).t()) * ((ids == e) * weights).sum(-1, keepdim=True)
        return {"y": y, "ids": ids.int(), "weights": weights}
    x = s["logits"].double()
    rows = torch.arange(case["T"], device=x.device)
    if op == "logprobs":
        logp = torch.log_softmax(x, -1)
        lse = torch.logsumexp(x, -1)
        entropy = torch.special.entr(logp.exp()).sum(-1)
        ids = torch.sort(s["logits"], dim=-1, descending=True, stable=True).indices[:, :case["top_n"]]
        logprob = torch.where(s["target"] < 0, 0.0, logp[rows, s["target"].clamp(min=0)])
        return {"logprob": logprob, "entropy": entropy, "lse": lse, "top_values": logp.gather(-1, ids), "top_ids": ids.int()}
    logp = x - s["lse"].double().unsqueeze(-1)
    p = logp.exp()
    gh = s["g_entropy"].double().unsqueeze(-1)
    gl = torch.where(s["target"] < 0, 0.0, s["g_logprob"].double()).unsqueeze(-1)
    d = gh * (torch.special.entr(p) - p * s["entropy"].double().unsqueeze(-1)) - gl * p
    d[rows, s["target"].clamp(min=0)] += gl.squeeze(-1)
    return d
