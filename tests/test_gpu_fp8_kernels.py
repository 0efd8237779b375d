"""The 8-bit floating-point linears on the GPU, kernel by kernel: each test asks what a call's launches are and asserts it, so
that another choice of kernel cannot leave it without the one that it is for."""
import numpy as np
import pytest
import torch

from paper_2503_06545_amd import binding as qc
from test_gpu_fp8 import KERNELS, which

pytestmark = pytest.mark.gpu

ONE_LAUNCH, RING = [k for k in KERNELS if k[0][3]], [k for k in KERNELS if k[0][0] == "ring"]
DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
# every kernel with every output that it is for: ((kernel, tokens, channels, fused), K, N, output)
EVERY = [(what, K, N, out) for what, K, N, outs in KERNELS for out in ("bf16", "f32")[:outs]]


def rows_for(what, K, N, out, experts=0):
    """The fewest rows that take this kernel and fill more than two of its tiles, else the most that take it."""
    least = 2 * what[1] + 5
    sizes = sorted({least, *range(3, 64), *(int(1.1 ** i) | 1 for i in range(43, 115))})
    found = [M for M in sizes if which(M, K, N, out, experts) == what]
    assert found, (what, K, N, out, experts)
    return next((M for M in found if M >= least), found[-1])


def random_weight(generator, experts, N, K):
    W = torch.randn(experts, N, K, generator=generator, device="cuda") * 0.02
    return qc.pack_weight_fp8_t(W if experts > 1 else W[0])


def generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


# ---- offsets out of order ------------------------------------------------------------------------

@pytest.mark.parametrize("what,K,N,out", EVERY)
def test_disordered_offsets_reach_nothing_outside(what, K, N, out):
    """Falling, negative and too large offsets: what the result is is open, but not where it is."""
    E, guard = 6, 32
    M = rows_for(what, K, N, out, E)
    assert which(M, K, N, out, E) == what
    g = generator(M)
    pw, X = random_weight(g, E, N, K), torch.randn(M, K, generator=g, device="cuda").bfloat16()
    nbytes = qc.qc_qlinear_fp8_workspace_bytes(M, K, N)
    space = torch.full((nbytes + 8192,), 0x5a, dtype=torch.uint8, device="cuda")
    Y = torch.empty(M + 2 * guard, N, dtype=DTYPE[out], device="cuda")
    top = 2 ** 31 - 1
    for offsets in ([0, M, 0, M, 0, M, 0], [-M, -3, M // 2, M // 4, M - 1, 3 * M, top], [M, M - 1, M // 2, M // 3, 2, 1, 0],
                    [-top - 1, top, 1, -1, M + 1, M // 2, M]):
        Y.fill_(5.0)
        off = torch.tensor(offsets, dtype=torch.int32, device="cuda")
        qc.qlinear_fp8_grouped_t(X, pw, off, out=out, workspace=space[4096:4096 + nbytes], Y=Y[guard:guard + M])
        torch.cuda.synchronize()
        assert (Y[:guard] == 5.0).all() and (Y[guard + M:] == 5.0).all(), offsets
        assert (space[:4096] == 0x5a).all() and (space[4096 + nbytes:] == 0x5a).all(), offsets
    if not what[3]:   # in two launches the workspace is what they meet in
        assert (space[4096:4096 + nbytes] != 0x5a).any()


# ---- special values ------------------------------------------------------------------------------

def edge_rows(tokens, M):
    """First and last row, and both sides of the tiles' edges; others are left."""
    rows = sorted({m for m in (0, 15, 16, tokens - 1, tokens, 2 * tokens, M - 1) if 0 <= m < M})
    return rows if len(rows) < M else [0, M - 1]


def spoil(X, rows, first):
    """A NaN or an infinity in each of these rows, in the first and the last column and between."""
    K = X.shape[1]
    for i, m in enumerate(rows):
        X[m, (0, K - 1, K // 2)[(i + first) % 3]] = (float("nan"), float("inf"), -float("inf"))[i % 3]


@pytest.mark.parametrize("x", ["bf16", "f32"])
@pytest.mark.parametrize("grouped", [False, True])
@pytest.mark.parametrize("what,K,N,out", EVERY)
def test_special_values_make_their_tokens_nan_and_no_others(what, K, N, out, grouped, x):
    E = 3 if grouped else 0
    M = rows_for(what, K, N, out, E)
    assert which(M, K, N, out, E) == what
    g = generator(M + K)
    pw = random_weight(g, max(E, 1), N, K)
    X = torch.randn(M, K, generator=g, device="cuda").to(DTYPE[x])
    bias = torch.randn(*([E] if E else []), N, generator=g, device="cuda")
    if grouped:   # one row on either side is of no group
        cut = [1, 1 + (M - 2) // 3, 1 + (M - 2) // 3, M - 1]
        off = torch.tensor(cut, dtype=torch.int32, device="cuda")

    def run(X):
        Y = torch.full((M, N), 7.0, dtype=DTYPE[out], device="cuda")
        if grouped:
            return qc.qlinear_fp8_grouped_t(X, pw, off, bias, "gelu_tanh", out, Y=Y)
        return qc.qlinear_fp8_t(X, pw, bias, "gelu_erf", out, Y=Y)

    clean = run(X)
    assert torch.isfinite(clean).all()
    for first in range(3):
        spoilt = X.clone()
        rows = edge_rows(what[1], M)
        if grouped:   # also the last and the first row of two groups that meet
            rows = sorted({*rows, cut[1] - 1, cut[2]} if M > 8 else {0, 1, M - 1})
        spoil(spoilt, rows, first)
        y = run(spoilt)
        mine = [m for m in rows if not grouped or cut[0] <= m < cut[-1]]
        others = torch.ones(M, dtype=torch.bool, device="cuda")
        others[mine] = False
        assert others.any() and (not mine or torch.isnan(y[mine]).all()), first
        assert torch.equal(y[others], clean[others]), first


@pytest.mark.parametrize("what,K,N,out", EVERY)
def test_zero_rows_and_a_zero_matrix_give_the_bias_in_every_kernel(what, K, N, out):
    M = rows_for(what, K, N, out)
    assert which(M, K, N, out) == what
    g = generator(M + N)
    bias = torch.randn(N, generator=g, device="cuda")
    want = bias.to(DTYPE[out])
    X = torch.randn(M, K, generator=g, device="cuda").bfloat16()
    zero = qc.pack_weight_fp8_t(torch.zeros(N, K, device="cuda"))
    assert (qc.qlinear_fp8_t(X, zero, bias, out=out) == want).all()
    rows = edge_rows(what[1], M)
    X[rows] = 0.0
    y = qc.qlinear_fp8_t(X, random_weight(g, 1, N, K), bias, out=out)
    assert (y[rows] == want).all() and len(rows) < M
    others = torch.ones(M, dtype=torch.bool, device="cuda")
    others[rows] = False
    assert (y[others] != want).any(dim=1).all()


# ---- the calls of a program, through every kernel --------------------------------------------------

@pytest.mark.parametrize("what,K,N,out", EVERY)
def test_captured_and_replayed_through_every_kernel(what, K, N, out):
    """A linear and a grouped one that share a workspace; inputs and group sizes change between the replays."""
    E = 3
    M, G = rows_for(what, K, N, out), rows_for(what, K, N, out, E)
    assert which(M, K, N, out) == which(G, K, N, out, E) == what
    g = generator(M + 1)
    one, pw = random_weight(g, 1, N, K), random_weight(g, E, N, K)
    X = torch.randn(max(M, G), K, generator=g, device="cuda").bfloat16()
    off = torch.tensor([0, G // 3, G // 3, G], dtype=torch.int32, device="cuda")
    ws = qc.qlinear_fp8_workspace_t(max(M, G), K, N)
    Y, Z = torch.empty(M, N, dtype=DTYPE[out], device="cuda"), torch.empty(G, N, dtype=DTYPE[out], device="cuda")

    def step():
        qc.qlinear_fp8_t(X[:M], one, None, "none", out, ws, Y)
        qc.qlinear_fp8_grouped_t(X[:G], pw, off, None, "none", out, ws, Z)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    rng = np.random.default_rng(M)
    for turn in range(4):
        X.copy_(torch.randn(X.shape, generator=g, device="cuda"))
        cut = sorted(int(v) for v in rng.integers(0, G + 1, size=E + 1))   # rows of no group on both sides
        off.copy_(torch.tensor(cut, dtype=torch.int32))
        for t in (Y, Z):
            t.fill_(3.0)
        step()
        torch.cuda.synchronize()
        want = Y.clone(), Z.clone()
        for t in (Y, Z):
            t.fill_(3.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(Y, want[0]) and torch.equal(Z, want[1]), turn
        assert (Z[:cut[0]] == 3.0).all() and (Z[cut[-1]:] == 3.0).all(), turn
        assert not (Y == 3.0).all(dim=1).any(), turn


@pytest.mark.parametrize("what,K,N,outs", RING)
def test_halves_on_the_ring(what, K, N, outs):
    """One input, quantized once, through two linears, the first of them twice: the bits of the whole calls, which take the
    same launches."""
    out = ("bf16", "f32")[outs - 1]
    M = rows_for(what, K, N, out)
    assert which(M, K, N, out) == what and not what[3]
    g = generator(N)
    weights = [random_weight(g, 1, n, K) for n in (N, N + 3)]
    assert which(M, K, N + 3, out) == what
    X = torch.randn(M, K, generator=g, device="cuda").bfloat16()
    ws, stream = qc.qlinear_fp8_workspace_t(M, K, N), torch.cuda.current_stream().cuda_stream
    ws.fill_(0xff)
    assert qc.qc_qlinear_fp8_quant(X.data_ptr(), qc._xdt(X), M, K, ws.data_ptr(), ws.numel(), stream) == qc.QC_OK
    for pw in (weights[0], weights[1], weights[0]):
        bias = torch.randn(pw.N, generator=g, device="cuda")
        Y = torch.full((M, pw.N), float("nan"), dtype=DTYPE[out], device="cuda")
        assert qc.qc_qlinear_fp8_gemm(ws.data_ptr(), ws.numel(), M, K, pw.blob.data_ptr(), pw.scale.data_ptr(), pw.N, bias.data_ptr(),
                                      qc.EPI["gelu_tanh"], Y.data_ptr(), qc.OUT[out], stream) == qc.QC_OK
        assert torch.equal(Y, qc.qlinear_fp8_t(X, pw, bias, "gelu_tanh", out))


@pytest.mark.parametrize("grouped", [False, True])
@pytest.mark.parametrize("place", ["same", "behind", "before"])
@pytest.mark.parametrize("what,K,N,outs", RING)
def test_output_over_its_input_on_the_ring(what, K, N, outs, place, grouped):
    """Y and X begin at the same address, or one some rows into the other: the bits of a call with both apart."""
    out, E = ("bf16", "f32")[outs - 1], 3 if grouped else 0
    M = rows_for(what, K, N, out, E)
    assert which(M, K, N, out, E) == what
    g = generator(K)
    pw = random_weight(g, max(E, 1), N, K)
    size, element = torch.finfo(DTYPE[out]).bits // 8, 2
    far = 16 * K * element * 3 // 16 * 16
    x_at, y_at = (far if place == "before" else 0), (far if place == "behind" else 0)
    both = torch.empty(far + max(M * K * element, M * N * size), dtype=torch.uint8, device="cuda")
    X = both[x_at:x_at + M * K * element].view(torch.bfloat16).view(M, K)
    Y = both[y_at:y_at + M * N * size].view(DTYPE[out]).view(M, N)
    apart = torch.randn(M, K, generator=g, device="cuda").bfloat16()
    X.copy_(apart)
    off = torch.tensor([0, M // 2 + 1, M // 2 + 1, M], dtype=torch.int32, device="cuda")
    if grouped:
        want = qc.qlinear_fp8_grouped_t(apart, pw, off, out=out)
        qc.qlinear_fp8_grouped_t(X, pw, off, out=out, Y=Y)
    else:
        want = qc.qlinear_fp8_t(apart, pw, out=out)
        qc.qlinear_fp8_t(X, pw, out=out, Y=Y)
    assert torch.equal(Y, want)


@pytest.mark.parametrize("grouped", [False, True])
@pytest.mark.parametrize("what,K,N,outs", ONE_LAUNCH)
def test_output_over_its_input_where_apart_it_is_one_launch(what, K, N, outs, grouped):
    """Quantized in a launch of its own then, and the sums in another order: within what the order can change."""
    E = 3 if grouped else 0
    M = rows_for(what, K, N, "f32", E)
    assert which(M, K, N, "f32", E) == what
    g = generator(K + 1)
    pw = random_weight(g, max(E, 1), N, K)
    both = torch.empty(M * max(K, N), device="cuda")
    X, Y = both[:M * K].view(M, K), both[:M * N].view(M, N)
    X.copy_(torch.randn(M, K, generator=g, device="cuda"))
    apart = X.clone()
    off = torch.tensor([0, M // 2, M // 2, M], dtype=torch.int32, device="cuda")
    call = (lambda *a, **k: qc.qlinear_fp8_grouped_t(*a[:2], off, **k)) if grouped else qc.qlinear_fp8_t
    want = call(apart, pw, out="f32")
    # sums of as many magnitudes: the linear of the dequantized operands' absolute values
    q, s = qc.quant_act_fp8_t(apart)
    kb = torch.arange(K, device="cuda") // 128
    x = (q.double() * s.double()[:, kb]).abs()
    codes, nb = qc.unpack_weight_codes_fp8_t(pw), torch.arange(N, device="cuda") // 128
    magnitudes = torch.zeros(M, N, dtype=torch.float64, device="cuda")
    for e, (lo, hi) in enumerate(zip(off.tolist(), off.tolist()[1:]) if grouped else [(0, M)]):
        w = (codes[e].double() * pw.scale[e].double()[nb][:, kb]).abs()
        magnitudes[lo:hi] = x[lo:hi] @ w.t().contiguous()
    call(X, pw, out="f32", Y=Y)
    # a block's products are added alike; of the blocks' sums either order rounds once a block, and each product with its scales twice
    assert bool(((Y.double() - want.double()).abs() <= 2 * (-(-K // 128) + 3) * 2.0 ** -24 * magnitudes).all())


def test_native_helpers_take_every_argument():
    """Calls that succeed, in positions and by name, with a bias of each row: the Python helpers' bits."""
    qc._use_native_helpers()
    g = generator(8)
    for M, N in ((40, 72), (700, 1304)):
        K = 260
        assert which(M, K, N, "bf16")[0] == which(M, K, N, "bf16", 3)[0] == ("few" if M == 40 else "ring")
        X = torch.randn(M, K, generator=g, device="cuda")
        pw, one = random_weight(g, 3, N, K), random_weight(g, 1, N, K)
        off, bias = torch.tensor([0, 11, 11, M], dtype=torch.int32, device="cuda"), torch.randn(3, N, generator=g, device="cuda")
        ws = qc.qlinear_fp8_workspace_t(M, K, N)
        for epi in qc.EPI:
            for out in ("bf16", "f32"):
                for x in (X, X.bfloat16()):
                    outputs = [torch.full((M, N), float("nan"), dtype=DTYPE[out], device="cuda") for _ in range(6)]
                    plain = [f(x, one, bias[1], epi, out, ws, y) for f, y in zip((qc._python_helpers["qlinear_fp8_t"], qc.qlinear_fp8_t), outputs)]
                    plain.append(qc.qlinear_fp8_t(x, one, workspace=ws, bias=bias[1], Y=outputs[2], epi=epi, out=out))
                    grouped = [f(x, pw, off, bias, epi, out, ws, y)
                               for f, y in zip((qc._python_helpers["qlinear_fp8_grouped_t"], qc.qlinear_fp8_grouped_t), outputs[3:])]
                    grouped.append(qc.qlinear_fp8_grouped_t(x, pw, Y=outputs[5], out=out, expert_offsets=off, epi=epi, bias=bias, workspace=ws))
                    assert all(a is b for a, b in zip(plain + grouped, outputs))
                    assert all(torch.isfinite(t).all() and torch.equal(t, ts[0]) for ts in (plain, grouped) for t in ts), (M, epi, out, x.dtype)


@pytest.mark.parametrize("x", ["bf16", "f32"])
@pytest.mark.parametrize("what,K,N,out", EVERY)
def test_calls_that_agree_in_all_but_addresses_give_the_same_bits(what, K, N, out, x):
    """Other buffers, another workspace that held something else, and another stream."""
    M, E = rows_for(what, K, N, out), 3
    G = rows_for(what, K, N, out, E)
    assert which(M, K, N, out) == which(G, K, N, out, E) == what
    g = generator(M + 2)
    one, pw = random_weight(g, 1, N, K), random_weight(g, E, N, K)
    X = torch.randn(max(M, G), K, generator=g, device="cuda").to(DTYPE[x])
    off = torch.tensor([0, G // 3, G // 2, G], dtype=torch.int32, device="cuda")
    want = qc.qlinear_fp8_t(X[:M], one, out=out), qc.qlinear_fp8_grouped_t(X[:G], pw, off, out=out)
    other, again = torch.cuda.Stream(), X.clone()
    ws = qc.qlinear_fp8_workspace_t(max(M, G), K, N)
    other.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(other):
        got = []
        for fill in (0x00, 0xff):
            ws.fill_(fill)
            got += [qc.qlinear_fp8_t(again[:M], one, out=out, workspace=ws), qc.qlinear_fp8_grouped_t(again[:G], pw, off, out=out, workspace=ws)]
    torch.cuda.synchronize()
    assert all(torch.equal(y, want[i % 2]) for i, y in enumerate(got))


# ---- how exact -----------------------------------------------------------------------------------

def whole_numbers(g, rows, K, groups, other):
    """[rows, K] of whole numbers up to 15 times a power of two for each run of 128 columns of a row, or, with `groups`, of 128 rows,
    whose largest magnitude is 448 of them, so that the scales are these powers and the codes the numbers.  The column that holds
    the 448 meets a zero of the other operand; where a run is too short for such columns every value is one."""
    steps = torch.randint(0, 2, (-(-rows // 128) if groups else rows, -(-K // 128)), generator=g, device="cuda")
    v = torch.randint(-15, 16, (rows, K), generator=g, device="cuda").float()
    for b in range(-(-K // 128)):
        at, width = 128 * b, min(128, K - 128 * b)
        if width < 3:
            v[:, at:at + width] = 448.0 * torch.sign(v[:, at:at + width] + 0.5)
        else:
            v[:, at + (5 * b + other) % width], v[:, at + (5 * b + 1 - other) % width] = 448.0, 0.0
    steps = steps.repeat_interleave(128, dim=0)[:rows] if groups else steps
    return v * 2.0 ** steps.repeat_interleave(128, dim=1)[:, :K]


@pytest.mark.parametrize("x", ["bf16", "f32"])
@pytest.mark.parametrize("grouped", [False, True])
@pytest.mark.parametrize("what,K,N,out", EVERY)
def test_whole_numbers_come_out_exactly(what, K, N, out, grouped, x):
    """Every product is a whole number of magnitude 225 at most, seven powers of two above 1, which the e4m3 instruction keeps, or 448 * 448 alone with
    its like, and every sum below 2^24: nothing is rounded before the output.  Each token and each 128 x 128 has scales of its own."""
    E = 3 if grouped else 1
    M = rows_for(what, K, N, out, E if grouped else 0)
    assert which(M, K, N, out, E if grouped else 0) == what
    g = generator(M + N + K)
    X = whole_numbers(g, M, K, False, 0)
    W = torch.stack([whole_numbers(g, N, K, True, 1) for _ in range(E)])
    bias = torch.randint(-100, 101, (E, N), generator=g, device="cuda").float()
    pw = qc.pack_weight_fp8_t(W if grouped else W[0])
    assert bool((torch.log2(pw.scale) == torch.log2(pw.scale).round()).all())
    cut = [1, 1 + M // 2, 1 + M // 2, M - 1] if grouped else [0, M]
    want = torch.full((M, N), 9.0, dtype=torch.float64, device="cuda")
    for e, (lo, hi) in enumerate(zip(cut, cut[1:])):
        want[lo:hi] = X[lo:hi].double() @ W[e].double().t().contiguous() + bias[e].double()
    assert want.abs().max() < 2 ** 24
    Y = torch.full((M, N), 9.0, dtype=DTYPE[out], device="cuda")
    if grouped:
        qc.qlinear_fp8_grouped_t(X.to(DTYPE[x]), pw, torch.tensor(cut, dtype=torch.int32, device="cuda"), bias, out=out, Y=Y)
    else:
        qc.qlinear_fp8_t(X.to(DTYPE[x]), pw, bias[0], out=out, Y=Y)
    assert torch.equal(Y, want.to(DTYPE[out]))


@pytest.mark.parametrize("what,K,N,out", EVERY)
def test_scales_far_from_one(what, K, N, out):
    """Powers of two on either operand come out as their product, as long as the scales' product is a normal number.  (A product of
    codes is below 2^18, a sum of them below 2^24: with the largest powers here outputs stay below 2^124.)"""
    M = rows_for(what, K, N, out)
    assert which(M, K, N, out) == what
    g = generator(M * 2 + K)
    X, W = whole_numbers(g, M, K, False, 0), whole_numbers(g, N, K, True, 1)
    want = X.double() @ W.double().t().contiguous()
    for a, b in ((-50, -60), (-60, -65), (50, 50), (60, -60), (-60, 60), (90, 8), (-60, 100)):
        y = qc.qlinear_fp8_t(X * 2.0 ** a, qc.pack_weight_fp8_t(W * 2.0 ** b), out=out)
        assert torch.equal(y, (want * 2.0 ** (a + b)).to(DTYPE[out])), (a, b)


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("M,K,N,experts", [(3, 100, 2200001, 0), (5, 260, 1100000, 2)])
def test_millions_of_channels(M, K, N, experts, out):
    """More than the rule for few tokens counts, one tile of tokens high."""
    assert which(M, K, N, out, experts)[0] == "ring"
    g = generator(N)
    X = whole_numbers(g, M, K, False, 0)
    W = torch.stack([whole_numbers(g, N, K, True, 1) for _ in range(max(experts, 1))])
    cut = [0, 2, M] if experts else [0, M]
    want = torch.cat([X[lo:hi].double() @ W[e].double().t() for e, (lo, hi) in enumerate(zip(cut, cut[1:]))])
    pw = qc.pack_weight_fp8_t(W if experts else W[0])
    if experts:
        y = qc.qlinear_fp8_grouped_t(X, pw, torch.tensor(cut, dtype=torch.int32, device="cuda"), out=out)
    else:
        y = qc.qlinear_fp8_t(X, pw, out=out)
    assert torch.equal(y, want.to(DTYPE[out]))


def test_weights_beyond_four_gib():
    """The last channels' codes lie past 2^32 bytes; the rows of a few tiles of channels repeated, against those alone."""
    M, K, period, N = 3, 2000, 7 * 128, 2200001
    assert which(M, K, N, "bf16")[0] == "ring" and qc.qc_packed_weight_fp8_bytes(1, N, K) > 2 ** 32
    g = generator(K)
    X, W = whole_numbers(g, M, K, False, 0), whole_numbers(g, period, K, True, 1)
    want = (X.double() @ W.double().t()).bfloat16()
    y = qc.qlinear_fp8_t(X, qc.pack_weight_fp8_t(W.repeat(-(-N // period), 1)[:N]))
    whole = N // period * period
    assert bool((y[:, :whole].reshape(M, -1, period) == want[:, None]).all()) and torch.equal(y[:, whole:], want[:, :N - whole])


def errors_before_rounding(g, what, K, N, values):
    """(errors, sums, sums of magnitudes) of the outputs of one token, all in 64 bits: its bias takes the sums away, so that
    what is left is rounded relative to itself.  All rows are that token."""
    M = rows_for(what, K, N, "bf16")
    assert which(M, K, N, "bf16") == what
    x, W = values(g, 1, K).bfloat16(), values(g, N, K)
    pw = qc.pack_weight_fp8_t(W)
    q, s = qc.quant_act_fp8_t(x)
    kb, nb = torch.arange(K, device="cuda") // 128, torch.arange(N, device="cuda") // 128
    xd = q.double() * s.double()[:, kb]
    wd = qc.unpack_weight_codes_fp8_t(pw)[0].double() * pw.scale[0].double()[nb][:, kb]
    sums, magnitudes = (xd * wd).sum(dim=1), (xd * wd).abs().sum(dim=1)
    bias = -sums.float()
    y = qc.qlinear_fp8_t(x.expand(M, K).contiguous(), pw, bias)
    assert bool((y == y[0]).all())
    return y[0].double() - (sums + bias.double()), sums, magnitudes


def normal(g, rows, K):
    return torch.randn(rows, K, generator=g, device="cuda")


def spread(g, rows, K):   # over twelve powers of two
    return torch.exp2(-12.0 * torch.rand(rows, K, generator=g, device="cuda"))


@pytest.mark.parametrize("what,K,N", [k[:3] for k in KERNELS])
def test_how_far_off_bf16_outputs_are_before_they_are_rounded(what, K, N):
    """The figures that the interface names, 1.4e-5 of normal values' sums and 8e-5 of those of values spread over twelve powers of two (2-norms over
    many channels, one token: their spread is a tenth or so), with a factor of two; and for each output what a group of eight can lose."""
    g = generator(K)
    for values, figure in ((normal, 1.4e-5), (spread, 8e-5)):
        error, sums, magnitudes = errors_before_rounding(g, what, K, N, values)
        assert error.norm() <= 2 * figure * sums.norm(), (values.__name__, float(error.norm() / sums.norm()))
        # beside it the sums in binary32 and the rounding of what is left
        assert bool((error.abs() <= (7 * 2.0 ** -13 + (-(-K // 128) + 3) * 2.0 ** -24) * (1 + 2.0 ** -8) * magnitudes).all()), values.__name__
