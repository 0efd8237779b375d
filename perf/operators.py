"""The 8-bit floating-point operators and their work: quantized to e4m3 with a scale for every block of 128, activations
per token, weights per 128 x 128, and multiplied; the linear of one weight, and the one of a mixture of experts
whose rows come sorted by expert.

Three kinds of case:

* ``quant``: the activation quantizer alone, codes and scales.
* ``linear``: one linear: quantize the activations, multiply, scales, bias and activation.
* ``grouped``: the same for rows grouped by expert, with ragged groups, empty ones among them, and rows behind the last
  group that stay as they were.

Weights (quantized and laid out once), biases, workspaces and output buffers are kept as a serving program keeps
them.  Activations are normal with 1 % outlier columns twenty times as large, or post-GELU; weights have a
standard deviation of 0.02, some channel blocks larger than others.  Groups come from a router that prefers some experts.

With ``own`` false the operators are computed from elementary operations in 32 bits.
"""
import math
import random

import torch

own = False

HIDDEN, MLP = 1152, 4608
BLOCK, E4M3_MOST, FLOOR = 128, 448.0, 2.0 ** -64
DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}

# the most a drawn case may hold: the largest listed linear
MOST_MACS = 131072 * HIDDEN * MLP


def _quant(name=None, M=256, K=HIDDEN, x="bf16", post_gelu=False):
    case = {"kind": "quant", "M": M, "K": K, "x": x, "post_gelu": post_gelu}
    return dict(case, name=name) if name else case


def _linear(name=None, M=256, K=HIDDEN, N=HIDDEN, x="bf16", out="bf16", epi="none", bias=True, post_gelu=False):
    case = {"kind": "linear", "M": M, "K": K, "N": N, "x": x, "out": out, "epi": epi, "bias": bias, "post_gelu": post_gelu}
    return dict(case, name=name) if name else case


def _grouped(name=None, M=256, E=8, K=HIDDEN, N=HIDDEN, live=1.0, skew=0.5, empty=0, x="bf16", out="bf16", epi="none", bias=True,
             post_gelu=False):
    """live: share of the buffer's rows that belong to a group; skew: how uneven the router is; empty: experts without rows"""
    case = {"kind": "grouped", "M": M, "E": E, "K": K, "N": N, "live": live, "skew": skew, "empty": empty, "x": x, "out": out,
            "epi": epi, "bias": bias, "post_gelu": post_gelu}
    return dict(case, name=name) if name else case


def listed():
    return [
        # a few hundred rows of no whole blocks: a short video's tokens behind an odd projection
        _quant("quant_ragged_f32", M=333, K=1000, x="f32"),
        # the input of the second MLP linear of a 512 x 512 video: all memory traffic
        _quant("quant_fc2_512", M=65536, K=MLP, post_gelu=True),
        # one conditioning vector per guidance half through the linear that makes a block's modulation vectors: latency
        _linear("modulation_2_tokens", M=2, N=6 * HIDDEN),
        # a text conditioning: a few hundred tokens, in binary32 throughout
        _linear("text_300_f32", M=300, K=MLP, N=HIDDEN, x="f32", out="f32"),
        # nothing a multiple of anything
        _linear("ragged_k1000", M=4099, K=1000, N=1301, out="f32", epi="gelu_erf", bias=False),
        # QKV of a 256 x 256 video
        _linear("qkv_256", M=16384, N=3 * HIDDEN),
        # second MLP linear, 512 x 512 video: the long reduction
        _linear("fc2_512", M=65536, K=MLP, post_gelu=True),
        # first MLP linear with GELU, 512 x 512 video with both halves of the guidance: the largest
        _linear("fc1_gelu_512_cfg", M=131072, N=MLP, epi="gelu_tanh"),
        # four tokens, two experts each, at generation time: weights of few experts and latency
        _grouped("experts_decode", M=8, E=32, N=MLP, skew=0.8, epi="gelu_tanh"),
        # a padded batch: ragged groups, two experts nobody chose, rows behind the last group
        _grouped("experts_padded_ragged", M=3001, E=12, K=1000, N=1301, live=0.8, empty=2, x="f32", out="f32"),
        # first linear of the experts of a 256 x 256 video, two experts a token
        _grouped("experts_fc1_256", M=32768, E=16, N=MLP, epi="gelu_tanh"),
        # second linear of many small experts, a 512 x 512 video
        _grouped("experts_fc2_512", M=65536, E=64, K=MLP, N=HIDDEN, skew=0.4, post_gelu=True),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["quant"] * 2 + ["linear"] * 4 + ["grouped"] * 4)
    x = rng.choice(["bf16", "bf16", "bf16", "f32"])
    # the transformer's widths half of the time, any others otherwise
    K = rng.choice([HIDDEN, HIDDEN, MLP]) if rng.random() < 0.5 else _log_uniform(rng, 24, 2 * MLP)
    N = rng.choice([HIDDEN, 3 * HIDDEN, MLP]) if rng.random() < 0.5 else _log_uniform(rng, 24, 6 * HIDDEN)
    if kind == "quant":
        return _quant(M=min(_log_uniform(rng, 1, 131072), 131072 * MLP // (2 * K)), K=K, x=x, post_gelu=K == MLP)
    args = dict(K=K, N=N, x=x, out=rng.choice(["bf16", "bf16", "bf16", "f32"]), epi=rng.choice(["none", "none", "gelu_tanh", "gelu_erf"]),
                bias=rng.random() < 0.8, post_gelu=K == MLP)
    if kind == "linear":
        return _linear(M=min(_log_uniform(rng, 1, 131072), max(1, MOST_MACS // (K * N))), **args)
    E = min(_log_uniform(rng, 2, 64), max(2, 2 ** 30 // (K * N)))
    return _grouped(M=min(_log_uniform(rng, 1, 65536), max(1, MOST_MACS // (4 * K * N))), E=E, live=rng.choice([1.0, 1.0, rng.uniform(0.5, 1.0)]),
                    skew=rng.uniform(0.0, 0.8), empty=rng.choice([0, 0, 1]), **args)


# ---- inputs --------------------------------------------------------------------------------------

def _activations(g, M, K, dtype, post_gelu):
    x = torch.randn(M, K, generator=g, device="cuda")
    if post_gelu:
        x = torch.nn.functional.gelu(x, approximate="tanh")
    else:
        cols = torch.randperm(K, generator=g, device="cuda")[:max(1, round(0.01 * K))]
        x[:, cols] *= 20.0
    return x.to(dtype)


def _group_sizes(case, seed):
    """Rows of each expert, as a router with preferences deals them out; at most four times their fair share."""
    rng = random.Random(int(seed) * 7919 + case["E"])
    E, rows = case["E"], max(1, round(case["M"] * case["live"]))
    like = [math.exp(case["skew"] * rng.gauss(0.0, 1.0)) for _ in range(E)]
    for e in rng.sample(range(E), min(case["empty"], E - 1)):
        like[e] = 0.0
    total = sum(like)
    like = [min(v, 4.0 * total / E) for v in like]
    total, sizes, dealt, at = sum(like), [], 0, 0.0
    for v in like:
        at += v
        upto = min(rows, int(rows * at / total + 0.5))
        sizes.append(upto - dealt)
        dealt = upto
    sizes[max(range(E), key=lambda e: like[e])] += rows - dealt
    return sizes


def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    data = {"X": _activations(g, case["M"], case["K"], DTYPE[case["x"]], case["post_gelu"])}
    if case["kind"] == "quant":
        return data
    E, N, K = case.get("E", 1), case["N"], case["K"]
    W = torch.randn(E, N, K, generator=g, device="cuda") * 0.02
    blocks = torch.exp(0.3 * torch.randn(E, (N + BLOCK - 1) // BLOCK, 1, generator=g, device="cuda"))
    data["W"] = W.mul_(blocks.repeat_interleave(BLOCK, dim=1)[:, :N])
    data["bias"] = torch.randn(E, N, generator=g, device="cuda") * 0.01 if case["bias"] else None
    # what the buffer of the output holds before: it may have been used
    data["Y"] = torch.randn(case["M"], N, generator=g, device="cuda").to(DTYPE[case["out"]])
    if case["kind"] == "grouped":
        data["sizes"] = _group_sizes(case, seed)
    return data


def prepare(case, seed):
    data = _inputs(case, seed)
    state = {"case": case, "X": data["X"]}
    if case["kind"] == "quant":
        return state
    one = case["kind"] == "linear"
    W, bias = data["W"], data["bias"]
    state.update(Y=data["Y"], bias=bias[0] if one and bias is not None else bias)
    if not one:
        offsets = [0]
        for n in data["sizes"]:
            offsets.append(offsets[-1] + n)
        state.update(offsets=torch.tensor(offsets, dtype=torch.int32, device="cuda"), live=offsets[-1], most=max(data["sizes"]))
    if own:
        from paper_2503_06545_amd import binding as qc
        state["pw"] = qc.pack_weight_fp8_t(W[0] if one else W)
        state["workspace"] = qc.qlinear_fp8_workspace_t(case["M"], case["K"], case["N"])
    else:
        state["Wt"] = _plain_weights(W)
    return state


# ---- the plain forms -----------------------------------------------------------------------------

# Scales and quotients are binary32 ones, divided in 64 bits and rounded: they decide on which side of a border between
# two codes a value falls (and torch divides by a number by multiplying with its reciprocal).

def _plain_scales(largest):
    return (largest.double().clamp_min(FLOOR) / E4M3_MOST).float()


def _plain_cast(x, s):
    return (x.double() / s.double()).float().to(torch.float8_e4m3fn)


def _plain_weights(W):
    """Quantized with a scale for each 128 x 128 and widened again, [E, K, N]"""
    E, N, K = W.shape
    padded = torch.nn.functional.pad(W, (0, -K % BLOCK, 0, -N % BLOCK))
    tiles = padded.view(E, padded.shape[1] // BLOCK, BLOCK, padded.shape[2] // BLOCK, BLOCK)
    s = _plain_scales(tiles.abs().amax(dim=(2, 4), keepdim=True))
    q = _plain_cast(tiles, s).float() * s
    return q.view(padded.shape)[:, :N, :K].transpose(1, 2).contiguous()


def _plain_codes(X):
    M, K = X.shape
    blocks = torch.nn.functional.pad(X.float(), (0, -K % BLOCK)).view(M, -1, BLOCK)
    s = _plain_scales(blocks.abs().amax(dim=2, keepdim=True))
    return _plain_cast(blocks, s), s


def _plain_epilogue(y, bias, epi):
    if bias is not None:
        y = y + bias
    if epi == "gelu_tanh":
        return 0.5 * y * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (y + 0.044715 * y * y * y)))
    if epi == "gelu_erf":
        return 0.5 * y * (1.0 + torch.erf(y * math.sqrt(0.5)))
    return y


def _plain(state):
    case, X = state["case"], state["X"]
    M, K = X.shape
    q, s = _plain_codes(X)
    if case["kind"] == "quant":
        return {"codes": q.view(M, -1)[:, :K].contiguous(), "scales": s.view(M, -1)}
    x = (q.float() * s).view(M, -1)[:, :K]
    if case["kind"] == "linear":
        return _plain_epilogue(x @ state["Wt"][0], state["bias"], case["epi"]).to(state["Y"].dtype)
    # the rows spread out into as many for each expert, one batched product, and gathered again
    live, offsets = state["live"], state["offsets"].long()
    row = torch.arange(live, device="cuda")
    expert = torch.searchsorted(offsets, row, right=True) - 1
    place = row - offsets[expert]
    spread = torch.zeros(case["E"], state["most"], K, device="cuda")
    spread[expert, place] = x[:live]
    y = torch.bmm(spread, state["Wt"])[expert, place]
    bias = None if state["bias"] is None else state["bias"][expert]
    state["Y"][:live] = _plain_epilogue(y, bias, case["epi"]).to(state["Y"].dtype)
    return state["Y"]


# ---- one pass ------------------------------------------------------------------------------------

def run(state):
    if not own:
        return _plain(state)
    from paper_2503_06545_amd import binding as qc
    case = state["case"]
    if case["kind"] == "quant":
        codes, scales = qc.quant_act_fp8_t(state["X"])
        return {"codes": codes, "scales": scales}
    args = dict(bias=state["bias"], epi=case["epi"], out=case["out"], workspace=state["workspace"], Y=state["Y"])
    if case["kind"] == "linear":
        return qc.qlinear_fp8_t(state["X"], state["pw"], **args)
    return qc.qlinear_fp8_grouped_t(state["X"], state["pw"], state["offsets"], **args)


# ---- what a pass cannot do without ---------------------------------------------------------------

def work(case):
    M, K = case["M"], case["K"]
    blocks = (K + BLOCK - 1) // BLOCK
    if case["kind"] == "quant":
        return {"bytes": float(M * K * (SIZE[case["x"]] + 1) + 4 * M * blocks), "flops": 2.0 * M * K}
    N, matrices = case["N"], 1
    if case["kind"] == "grouped":
        M = max(1, round(M * case["live"]))
        matrices = min(case["E"], M)
    weights = N * K + 4 * ((N + BLOCK - 1) // BLOCK) * blocks + (4 * N if case["bias"] else 0)
    return {"bytes": float(M * K * SIZE[case["x"]] + matrices * weights + M * N * SIZE[case["out"]]), "flops": 2.0 * M * N * K}


# ---- the definition in 64 bits -------------------------------------------------------------------
# The quantizer's steps are binary32 ones by definition (its scales and quotients are rounded to binary32 before the
# codes are), which a division in 64 bits, rounded, gives exactly.

def _exact_e4m3(v):
    """The nearest number of 3 fraction bits and an exponent of -6 or more, ties to even"""
    a = v.abs()
    exponent = (torch.frexp(a)[1] - 1).clamp_min(-6)
    step = ((exponent.long() - 3 + 1023) << 52).view(torch.float64)   # two to the power of exponent - 3, exactly
    return torch.sign(v) * torch.round(a / step) * step


def _exact_quantize(v, largest):
    s = (largest.double().clamp_min(FLOOR) / E4M3_MOST).float().double()
    return _exact_e4m3((v.double() / s).float().double()), s


def _exact_rows(X):
    """Codes [M, K] and scales [M, blocks] of rows"""
    codes, scales = [], []
    for k in range(0, X.shape[1], BLOCK):
        part = X[:, k:k + BLOCK]
        q, s = _exact_quantize(part, part.float().abs().amax(dim=1, keepdim=True))
        codes.append(q)
        scales.append(s)
    return torch.cat(codes, dim=1), torch.cat(scales, dim=1)


def _exact_weight(W):
    out = torch.empty(W.shape, dtype=torch.float64, device="cuda")
    for n in range(0, W.shape[0], BLOCK):
        part = W[n:n + BLOCK]
        column = part.abs().amax(dim=0).view(1, 1, -1)
        block = torch.nn.functional.max_pool1d(column, BLOCK, BLOCK, ceil_mode=True).view(-1)
        q, s = _exact_quantize(part, block.repeat_interleave(BLOCK)[:W.shape[1]])
        out[n:n + BLOCK] = q * s
    return out


def _exact_linear(X, W, bias, epi):
    parts = []
    for m in range(0, X.shape[0], 16384):
        q, s = _exact_rows(X[m:m + 16384])
        y = (q * s.repeat_interleave(BLOCK, dim=1)[:, :q.shape[1]]) @ W.t()
        if bias is not None:
            y += bias.double()
        if epi == "gelu_tanh":
            y = y / (1.0 + torch.exp(-2.0 * math.sqrt(2.0 / math.pi) * (y + 0.044715 * y ** 3)))
        elif epi == "gelu_erf":
            y = 0.5 * y * torch.erfc(-y * math.sqrt(0.5))
        parts.append(y)
    return torch.cat(parts)


def exact(case, seed):
    data = _inputs(case, seed)
    if case["kind"] == "quant":
        q, s = _exact_rows(data["X"])
        return {"codes": q, "scales": s}
    bias = data["bias"]
    if case["kind"] == "linear":
        return _exact_linear(data["X"], _exact_weight(data["W"][0]), None if bias is None else bias[0], case["epi"])
    Y, at = data["Y"].double(), 0
    for e, n in enumerate(data["sizes"]):
        if n:
            Y[at:at + n] = _exact_linear(data["X"][at:at + n], _exact_weight(data["W"][e]), None if bias is None else bias[e], case["epi"])
        at += n
    return Y
