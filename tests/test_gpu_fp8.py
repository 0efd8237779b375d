"""The 8-bit floating-point operators on the GPU against the oracle in 64 bits: codes and scales bit for bit, outputs
within what the roundings on their way come to.

An output is a sum of K products and a bias, scaled.  The products are exact (4-bit significands), and whatever the order, a
sum of 128 of them is off by at most 127 steps of 2^-23 (the matrix instruction may cut off instead of rounding), the scaled
sums of the blocks by one each and the scale's two products by one each, all relative to the sum of the magnitudes that
went in.  For bf16 outputs the products of a block are added by an instruction that lines up eight of them, drops what is below
2^-13 of the power of two in the largest (test_what_the_e4m3_instruction_keeps) and so is off by less than 2^-13 of
the largest for each of the other seven: 7 * 2^-13 of the magnitudes at most.  An activation passes an error on at 1.13
at most and adds its own, below 1e-6 of its argument.  bf16 rounds by 2^-8 of the value at most."""
import numpy as np
import pytest
import torch

import oracle
from paper_2503_06545_amd import binding as qc
from paper_2503_06545_amd import synth
from test_gpu_parity import bits_equal, dev, host_f64, random_x

pytestmark = pytest.mark.gpu

EPIS = {"none": oracle.EPI_NONE, "gelu_tanh": oracle.EPI_GELU_TANH, "gelu_erf": oracle.EPI_GELU_ERF}


def weights(rng, N, K):
    W = (rng.standard_normal((N, K)) * 0.02).astype(np.float32)
    return W * np.exp(0.5 * rng.standard_normal((N, 1))).astype(np.float32)


def assert_within(got, ref, K, out, epi):
    steps = 127 + -(-K // 128) + 3
    bound = steps * 2.0 ** -23 * ref["size"]
    if out == "bf16":
        bound = bound + 7 * 2.0 ** -13 * ref["size"]
    if epi != "none":
        bound = 1.13 * bound + 1e-6 * ref["size"]
    if out == "bf16":
        bound = bound * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(ref["y"])
    assert got.shape == ref["y"].shape
    assert np.all(np.isfinite(got)) and np.all(np.abs(got - ref["y"]) <= bound), np.max(np.abs(got - ref["y"]) / bound)


def to_codes(q):
    """A zero's sign is open: x = -0 comes out as a positive zero, because the residual of its quotient, -s (-0) + (-0), is
    +0, and so is what that is added to."""
    return plain_zeros(q.view(torch.uint8).cpu().numpy())


def plain_zeros(codes):
    return np.where(codes == 0x80, 0, codes)


# ---- the quantizers ------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,K", [(1, 1), (3, 3), (5, 7), (9, 8), (1, 127), (2, 128), (7, 129), (33, 130), (8, 144), (31, 255), (40, 384),
                                 (65, 385), (64, 1000), (300, 1152), (17, 4608), (2, 9217), (1, 131072)])
def test_quant_act_is_the_oracles_bit_for_bit(M, K, dtype):
    rng = np.random.default_rng(M * 131 + K)
    x = random_x(rng, M, K, "f32")
    x[M // 2, :200] = 0.0                                  # a block that is zero takes the floor
    x[:, -1] *= 2.0 ** rng.integers(-12, 12, size=M)       # quotients among the smallest codes and below
    if M > 2:
        x[0] *= 1e-30
        x[1] = -np.abs(x[1]) * 1e30
    if dtype == "bf16":
        x = synth.to_bf16_bits(x.astype(np.float32))
    q_ref, s_ref = oracle.quant_act_fp8(x)
    q, s = qc.quant_act_fp8_t(dev(x))
    torch.cuda.synchronize()
    assert q.dtype == torch.float8_e4m3fn and bits_equal(s.cpu().numpy(), s_ref)
    assert np.array_equal(to_codes(q), plain_zeros(q_ref))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_quant_act_on_values_at_the_borders_of_codes(dtype):
    """Every border between two codes times the scale, with neighbours on both sides: the largest is 448 s."""
    table = oracle.E4M3[:127]
    borders = ((table[1:] + table[:-1]) / 2).astype(np.float32)
    for scale in (1.0, 0.37, 3.1e-5):
        row = []
        for b in np.concatenate([borders, -borders]):
            v = np.float32(b) * np.float32(scale)
            row += [v, np.nextafter(v, np.float32(0)), np.nextafter(v, np.float32(np.sign(v) * 1e9))]
        row = np.asarray(row, np.float32)
        row = np.concatenate([row, np.zeros(-len(row) % 127, np.float32)]).reshape(-1, 127)
        x = np.concatenate([row, np.full((len(row), 1), np.float32(448) * np.float32(scale))], axis=1)
        if dtype == "bf16":
            x = synth.to_bf16_bits(x)
        q_ref, s_ref = oracle.quant_act_fp8(x)
        q, s = qc.quant_act_fp8_t(dev(x))
        assert bits_equal(s.cpu().numpy(), s_ref) and np.array_equal(to_codes(q), plain_zeros(q_ref))


# past the caches with and without whole lines of codes, through them where X has none; rows 32 to a block, blocks in eights
@pytest.mark.parametrize("M,K,dtype", [(70003, 1152, "bf16"), (40001, 1152, "f32"), (70003, 1088, "bf16"), (70003, 1001, "bf16"), (50021, 1056, "f32")])
def test_large_inputs_are_the_small_ones_bit_for_bit(M, K, dtype):
    """The rows of a small block repeated, the block against the oracle and every row against the block's."""
    period = 53
    x = random_x(np.random.default_rng(K), period, K, dtype)
    q_ref, s_ref = oracle.quant_act_fp8(x)
    q, s = qc.quant_act_fp8_t(dev(x).repeat(-(-M // period), 1)[:M].contiguous())
    q = q.view(torch.uint8)
    assert bits_equal(s[:period].cpu().numpy(), s_ref) and np.array_equal(to_codes(q[:period]), plain_zeros(q_ref))
    whole = M // period * period
    for t in (q, s):
        assert bool((t[:whole].view(-1, period, t.shape[1]) == t[:period]).all()) and torch.equal(t[whole:], t[:M - whole])


def test_quant_act_into_given_tensors_writes_nothing_else():
    x = random_x(np.random.default_rng(3), 21, 203, "f32")
    codes = torch.full((21 * 203 + 64,), 0x55, dtype=torch.uint8, device="cuda")
    scales = torch.full((21 * 2 + 16,), -7.0, device="cuda")
    q, s = codes[:21 * 203].view(21, 203).view(torch.float8_e4m3fn), scales[:42].view(21, 2)
    assert qc.quant_act_fp8_t(dev(x), q, s)[0] is q
    q_ref, s_ref = oracle.quant_act_fp8(x)
    assert np.array_equal(to_codes(q), plain_zeros(q_ref)) and bits_equal(s.cpu().numpy(), s_ref)
    assert (codes[21 * 203:] == 0x55).all() and (scales[42:] == -7.0).all()


@pytest.mark.parametrize("E,N,K", [(1, 1, 1), (1, 128, 128), (1, 129, 127), (3, 200, 300), (2, 5, 1152)])
def test_weights_are_the_oracles_bit_for_bit(E, N, K):
    rng = np.random.default_rng(E * 1000 + N + K)
    W = np.stack([weights(rng, N, K) for _ in range(E)])
    W[0, :min(N, 128), :min(K, 128)] *= 0.0 if E > 1 else 1.0
    pw = qc.pack_weight_fp8_t(dev(W) if E > 1 else dev(W[0]))
    codes = to_codes(qc.unpack_weight_codes_fp8_t(pw))
    for e in range(E):
        q_ref, s_ref = oracle.quant_weight_fp8(W[e])
        assert np.array_equal(codes[e], plain_zeros(q_ref)) and bits_equal(pw.scale[e].cpu().numpy(), s_ref)


# ---- the linear ----------------------------------------------------------------------------------

def run_linear(rng, M, K, N, x="bf16", out="bf16", epi="none", bias=True, halves=False):
    W, X = weights(rng, N, K), random_x(rng, M, K, x)
    b = (rng.standard_normal(N) * 0.1).astype(np.float32) if bias else None
    ref = oracle.qlinear_fp8(X, *oracle.quant_weight_fp8(W), b, EPIS[epi])
    pw, Xd, bd = qc.pack_weight_fp8_t(dev(W)), dev(X), None if b is None else dev(b)
    ws = qc.qlinear_fp8_workspace_t(M, K, N)
    ws.fill_(0xff)   # NaN as a code and as a scale, no group as a tile
    Y = torch.full((M + 2, N), float("nan"), dtype=torch.float32 if out == "f32" else torch.bfloat16, device="cuda")
    if halves:
        stream = torch.cuda.current_stream().cuda_stream
        assert qc.qc_qlinear_fp8_quant(Xd.data_ptr(), qc._xdt(Xd), M, K, ws.data_ptr(), ws.numel(), stream) == qc.QC_OK
        assert qc.qc_qlinear_fp8_gemm(ws.data_ptr(), ws.numel(), M, K, pw.blob.data_ptr(), pw.scale.data_ptr(), N,
                                      None if bd is None else bd.data_ptr(), qc.EPI[epi], Y.data_ptr(), qc.OUT[out], stream) == qc.QC_OK
    else:
        y = Y[:M] if N else None
        assert qc.qlinear_fp8_t(Xd, pw, bd, epi, out, ws, y) is y
    got = host_f64(Y)
    assert np.isnan(got[M:]).all()   # nothing behind the last row
    assert_within(got[:M], ref, K, out, epi)


SIZES = [(1, 1, 1), (1, 128, 128), (2, 1152, 300), (4, 4608, 136), (15, 129, 17), (16, 7, 5), (17, 130, 129), (33, 256, 1000),
         (64, 1152, 264), (65, 1000, 257), (100, 2304, 40), (128, 384, 384), (129, 1152, 130), (193, 640, 1028), (257, 129, 1301),
         (300, 4608, 72), (513, 1153, 200), (1025, 200, 385)]


@pytest.mark.parametrize("M,K,N", SIZES)
@pytest.mark.parametrize("x,out,epi", [("bf16", "bf16", "none"), ("f32", "f32", "none"), ("bf16", "f32", "gelu_tanh"), ("f32", "bf16", "gelu_erf")])
def test_linear(M, K, N, x, out, epi):
    rng = np.random.default_rng(M * 7 + K * 3 + N)
    run_linear(rng, M, K, N, x, out, epi, bias=(M + N) % 3 != 0)


@pytest.mark.parametrize("M,K,N", [(1, 130, 40), (16, 1152, 300), (40, 1152, 256), (300, 1000, 130), (700, 384, 257)])
def test_linear_in_halves(M, K, N):
    run_linear(np.random.default_rng(M + K), M, K, N, "bf16", "f32", halves=True)


def test_what_the_e4m3_instruction_keeps():
    """Two products of 2^16 that cancel, and one more in their group of eight: what is at most 13 powers of two lower comes
    out exactly, with binary32 output whatever is."""
    M, K = 64, 128
    for low, out in ((3, "bf16"), (-8, "f32")):
        for e in range(15, low - 1, -1):
            a = min(e, 8) if e >= -6 else -6
            X, W = torch.zeros(M, K, device="cuda"), torch.zeros(32, K, device="cuda")
            X[:, 0] = X[:, 1] = W[:, 0] = 256.0
            W[:, 1] = -256.0
            X[:, 127], W[:, 126] = 448.0, 448.0   # both scales one; these two meet zeros
            rows = torch.arange(2, 34, device="cuda")
            X[rows, rows] = 2.0 ** a
            W[:, 2:34] = 2.0 ** (e - a)
            y = qc.qlinear_fp8_t(X, qc.pack_weight_fp8_t(W), out=out).float()
            assert (y[2:34] == 2.0 ** e).all() and (y[34:] == 0).all() and (y[:2] == 0).all(), (out, e)


def which(M, K, N, out, experts=0):
    p = qc.linear_plan_fp8(M, K, N, out, experts)
    return p["kernel"], p["tokens"], p["channels"], p["fused"]


# (kernel, tokens, channels, fused), a ragged reduction and channels, and whether the output may be binary32
KERNELS = [(("few", 16, 16, True), 700, 700, 2), (("few", 16, 32, True), 1153, 2311, 2), (("few", 16, 64, True), 513, 4609, 2),
           (("few", 32, 64, False), 5001, 700, 2), (("ring", 64, 128, False), 260, 1300, 2), (("ring", 128, 128, False), 130, 1301, 2),
           (("ring", 192, 128, False), 257, 701, 1), (("ring", 256, 128, False), 1281, 6901, 1)]


def tokens_for(kernel, K, N, out, experts=0):
    """The fewest tokens of a list, odd ones, for which a linear of these sizes takes this kernel."""
    sizes = sorted({int(1.19 ** i) | 1 for i in range(63)})
    found = [M for M in sizes if which(M, K, N, out, experts) == kernel]
    assert found, (kernel, K, N, out, experts)
    return found[0]


@pytest.mark.parametrize("x,out", [("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32"), ("f32", "f32")])
@pytest.mark.parametrize("kernel", range(len(KERNELS)))
def test_every_kernel_at_ragged_sizes(kernel, x, out):
    what, K, N, outs = KERNELS[kernel]
    if outs == 1 and out == "f32":
        pytest.skip("binary32 outputs have no tiles of this height")
    M = tokens_for(what, K, N, out)
    if M < 10000:
        run_linear(np.random.default_rng(kernel), M, K, N, x, out, bias=kernel % 2 == 0)
    else:
        run_repeated(np.random.default_rng(kernel), M, K, N, x, out)


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("kernel", range(len(KERNELS)))
def test_every_kernel_grouped(kernel, out):
    what, K, N, outs = KERNELS[kernel]
    if outs == 1 and out == "f32":
        pytest.skip("binary32 outputs have no tiles of this height")
    E = 3
    M = tokens_for(what, K, N, out, E)
    rng = np.random.default_rng(kernel)
    if M < 10000:
        cut = sorted(int(v) for v in rng.integers(0, M + 1, size=E))
        run_grouped(rng, M, K, N, [0, *cut], "bf16", out)
    else:
        run_repeated_groups(rng, [M // 3 + 1, 0, M - 2 * (M // 3)], K, N, out)


@pytest.mark.parametrize("blocks", range(1, 14))
def test_every_length_of_the_rings_last_steps(blocks):
    """Six steps to a turn of the ring, and what is left of one.  Tiles of 256 tokens are for four blocks and more."""
    K = 128 * blocks - blocks % 3
    for what, out in ((("ring", 64, 128, False), "f32"), (("ring", 128, 128, False), "bf16"), (("ring", 192, 128, False), "bf16"), (("ring", 256, 128, False), "bf16")):
        N = 6901 if what[1] == 256 else 301
        if what[1] == 256 and blocks < 4:
            continue
        run_repeated(np.random.default_rng(blocks), tokens_for(what, K, N, out), K, N, "bf16", out)


def run_repeated(rng, M, K, N, x="bf16", out="bf16", epi="none"):
    """Many tokens: the rows of a small block repeated, the block against the oracle and every row against the block's."""
    period = min(M, 47)
    W, X = weights(rng, N, K), random_x(rng, period, K, x)
    ref = oracle.qlinear_fp8(X, *oracle.quant_weight_fp8(W), None, EPIS[epi])
    Xd = dev(X).repeat(-(-M // period), 1)[:M].contiguous()
    Y = qc.qlinear_fp8_t(Xd, qc.pack_weight_fp8_t(dev(W)), None, epi, out)
    assert_within(host_f64(Y[:period]), ref, K, out, epi)
    whole = M // period * period
    assert bool((Y[:whole].view(-1, period, N) == Y[:period]).all())
    if M > whole:
        assert torch.equal(Y[whole:], Y[:M - whole])


def run_repeated_groups(rng, sizes, K, N, out="bf16"):
    period = 50
    offsets = np.concatenate([[0], np.cumsum(sizes)]).tolist()
    W = np.stack([weights(rng, N, K) for _ in sizes])
    X = random_x(rng, period, K, "bf16")
    Xd = torch.cat([dev(X).repeat(-(-n // period), 1)[:n] for n in sizes])
    off = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    Y = qc.qlinear_fp8_grouped_t(Xd, qc.pack_weight_fp8_t(dev(W)), off, out=out)
    for e, n in enumerate(sizes):
        if n:
            ref = oracle.qlinear_fp8(X, *oracle.quant_weight_fp8(W[e]))
            y = Y[offsets[e]:offsets[e + 1]]
            assert_within(host_f64(y[:period]), ref, K, out, "none")
            assert torch.equal(y, y[:period].repeat(-(-n // period), 1)[:n])


# the sizes of real layers, sampled
@pytest.mark.parametrize("M,K,N,out,epi", [(16384, 1152, 3456, "bf16", "none"), (20000, 4608, 1152, "f32", "none"), (9000, 1152, 4608, "bf16", "gelu_tanh"),
                                           (40000, 1152, 4608, "bf16", "gelu_tanh"), (4099, 1000, 1301, "f32", "gelu_erf"),
                                           (2500, 9216, 640, "bf16", "none"), (700000, 128, 3200, "bf16", "none"),
                                           (300007, 1152, 20, "bf16", "none")])
def test_large_linears(M, K, N, out, epi):
    run_repeated(np.random.default_rng(M + N), M, K, N, "bf16", out, epi)


def test_codes_and_inputs_beyond_four_gib():
    """The last rows lie past 2^32 bytes of X and of the codes; every row against the first ones'."""
    run_repeated(np.random.default_rng(4), 140000, 31000, 40, "bf16", "bf16")


def test_special_values_stay_in_their_token():
    rng = np.random.default_rng(11)
    M, K, N = 70, 400, 150
    W, X = weights(rng, N, K), random_x(rng, M, K, "f32")
    pw = qc.pack_weight_fp8_t(dev(W))
    clean = qc.qlinear_fp8_t(dev(X), pw, None, "none", "f32").clone()
    for M_used in (M, 3):   # the kernels for many and for few tokens
        bad = X[:M_used].copy()
        bad[0, 5], bad[M_used - 1, 399], bad[1, 130] = np.nan, np.inf, -np.inf
        y = qc.qlinear_fp8_t(dev(bad), pw, None, "none", "f32")
        good = [m for m in range(M_used) if m not in (0, 1, M_used - 1)]
        assert torch.isnan(y[[0, 1, M_used - 1]]).all() and torch.isfinite(y[good]).all()
        if M_used == M:
            assert torch.equal(y[good], clean[good])


def test_zero_rows_and_a_zero_matrix_give_the_bias():
    N, K = 200, 300
    bias = torch.randn(N, device="cuda")
    X = torch.zeros(50, K, device="cuda")
    pw = qc.pack_weight_fp8_t(torch.randn(N, K, device="cuda"))
    zero = qc.pack_weight_fp8_t(torch.zeros(N, K, device="cuda"))
    for M in (1, 50):
        assert torch.equal(qc.qlinear_fp8_t(X[:M], pw, bias, out="f32"), bias.expand(M, N))
        assert torch.equal(qc.qlinear_fp8_t(torch.randn(M, K, device="cuda"), zero, bias, out="f32"), bias.expand(M, N))


@pytest.mark.parametrize("M", [3, 200])
def test_output_over_its_input(M):
    K = N = 256
    rng = np.random.default_rng(M)
    W, X = weights(rng, N, K), random_x(rng, M, K, "f32")
    ref = oracle.qlinear_fp8(X, *oracle.quant_weight_fp8(W))
    Xd = dev(X)
    y = qc.qlinear_fp8_t(Xd, qc.pack_weight_fp8_t(dev(W)), out="f32", Y=Xd)
    assert_within(host_f64(y), ref, K, "f32", "none")


# ---- grouped by expert ---------------------------------------------------------------------------

def run_grouped(rng, M, K, N, offsets, x="bf16", out="bf16", epi="none", bias=True):
    E = len(offsets) - 1
    W, X = np.stack([weights(rng, N, K) for _ in range(E)]), random_x(rng, M, K, x)
    b = (rng.standard_normal((E, N)) * 0.1).astype(np.float32) if bias else None
    pw = qc.pack_weight_fp8_t(dev(W))
    ws = qc.qlinear_fp8_workspace_t(M, K, N)
    ws.fill_(0xff)
    before = torch.randn(M, N, device="cuda").to(torch.float32 if out == "f32" else torch.bfloat16)
    Y = before.clone()
    off = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    assert qc.qlinear_fp8_grouped_t(dev(X), pw, off, None if b is None else dev(b), epi, out, ws, Y) is Y
    got = host_f64(Y)
    for e in range(E):
        lo, hi = offsets[e], offsets[e + 1]
        if hi > lo:
            ref = oracle.qlinear_fp8(X[lo:hi], *oracle.quant_weight_fp8(W[e]), None if b is None else b[e], EPIS[epi])
            assert_within(got[lo:hi], ref, K, out, epi)
    rest = [m for m in range(M) if m < offsets[0] or m >= offsets[-1]]
    assert torch.equal(Y[rest], before[rest])


GROUPS = [
    (1, [0, 1]), (1, [0, 0, 1, 1]), (5, [0, 5]), (5, [0, 0, 0, 0]), (8, [0, 1, 2, 2, 3, 5, 8]), (40, [3, 3, 20, 37]),
    (64, [0, 16, 32, 48, 64]), (65, [0, 64, 65]), (130, [0, 1, 130]), (200, [0, 129, 129, 130, 190]), (300, [0, 300, 300]),
    (333, [10, 75, 140, 333]), (700, [0, 255, 511, 512, 700]), (1200, [0, 600, 600, 1111]),
]


@pytest.mark.parametrize("M,offsets", GROUPS)
@pytest.mark.parametrize("K,N,x,out,epi", [(300, 136, "bf16", "bf16", "none"), (1000, 77, "f32", "f32", "gelu_erf"), (128, 260, "bf16", "f32", "gelu_tanh")])
def test_grouped(M, offsets, K, N, x, out, epi):
    run_grouped(np.random.default_rng(M + K + len(offsets)), M, K, N, offsets, x, out, epi, bias=M % 2 == 1)


@pytest.mark.parametrize("rows_each", [0, 1, 3])
def test_as_many_experts_as_there_may_be(rows_each):
    E = qc.QC_MAX_EXPERTS
    rng = np.random.default_rng(rows_each)
    sizes = rng.integers(0, 2 * rows_each + 1, size=E)
    offsets = [0] + np.cumsum(sizes).tolist()
    run_grouped(rng, max(1, offsets[-1]) + 2, 64, 16, offsets, out="f32", bias=False)


def test_large_groups():
    """Groups of many tiles."""
    run_repeated_groups(np.random.default_rng(2), [5000, 0, 9001, 130, 2700], 1152, 640)


def test_one_group_is_the_linear():
    rng = np.random.default_rng(4)
    for M in (3, 300):
        W, X = weights(rng, 200, 500), random_x(rng, M, 500, "bf16")
        pw, Xd = qc.pack_weight_fp8_t(dev(W)), dev(X)
        off = torch.tensor([0, M], dtype=torch.int32, device="cuda")
        ref = oracle.qlinear_fp8(X, *oracle.quant_weight_fp8(W))
        for y in (qc.qlinear_fp8_t(Xd, pw, out="f32"), qc.qlinear_fp8_grouped_t(Xd, pw, off, out="f32")):
            assert_within(host_f64(y), ref, 500, "f32", "none")


def test_offsets_that_do_not_ascend_touch_nothing_else():
    """What the result is is open, but rows outside the buffer are not reached: offsets below 0, above M, falling."""
    M, K, N, E = 100, 128, 64, 6
    pw = qc.pack_weight_fp8_t(torch.randn(E, N, K, device="cuda"))
    ws = qc.qlinear_fp8_workspace_t(M, K, N)
    guarded = torch.full((ws.numel() + 4096,), 0x5a, dtype=torch.uint8, device="cuda")
    for offsets in ([0, 100, 0, 100, 0, 100, 0], [-50, -3, 20, 10, 90, 400, 2 ** 31 - 1], [100, 80, 60, 40, 20, 10, 0]):
        off = torch.tensor(offsets, dtype=torch.int32, device="cuda")
        for X in (torch.randn(M, K, device="cuda"), torch.randn(4, K, device="cuda")):
            space = torch.full((len(X) + 64, N), 5.0, device="cuda")
            qc.qlinear_fp8_grouped_t(X, pw, off, out="f32", workspace=guarded[:ws.numel()], Y=space[32:32 + len(X)])
            torch.cuda.synchronize()
            assert (space[:32] == 5.0).all() and (space[32 + len(X):] == 5.0).all()
            assert (guarded[ws.numel():] == 0x5a).all()


# ---- as a program uses them ----------------------------------------------------------------------

def test_a_layer_of_experts_from_router_to_sum():
    """Router, rows sorted by expert, both linears of the experts, and the weighted sum, as a model runs them."""
    rng = np.random.default_rng(9)
    T, D, F, E, top = 90, 256, 640, 7, 2
    X = random_x(rng, T, D, "bf16")
    W1, W2 = np.stack([weights(rng, F, D) for _ in range(E)]), np.stack([weights(rng, D, F) for _ in range(E)])
    b1 = (rng.standard_normal((E, F)) * 0.1).astype(np.float32)
    logits = rng.standard_normal((T, E)).astype(np.float32)
    Xd, gate = dev(X), torch.softmax(dev(logits), dim=1)
    share, chosen = gate.topk(top, dim=1)
    order = chosen.view(-1).argsort(stable=True)
    offsets = torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"), torch.bincount(chosen.view(-1), minlength=E).cumsum(0)]).int()
    rows = Xd[order // top]
    p1, p2 = qc.pack_weight_fp8_t(dev(W1)), qc.pack_weight_fp8_t(dev(W2))
    ws = qc.qlinear_fp8_workspace_t(T * top, F, max(D, F))
    h = qc.qlinear_fp8_grouped_t(rows, p1, offsets, dev(b1), "gelu_tanh", "bf16", ws)
    y = qc.qlinear_fp8_grouped_t(h, p2, offsets, None, "none", "f32", ws)
    out = torch.zeros(T, D, device="cuda").index_add_(0, order // top, y * share.view(-1)[order, None])
    order_h, off_h, rows_h = order.cpu().numpy(), offsets.cpu().numpy(), X[(order // top).cpu().numpy()]
    h_bits = h.view(torch.int16).cpu().numpy().view(np.uint16)
    want = np.zeros((T, D))
    size = np.zeros((T, D))
    for e in range(E):
        lo, hi = off_h[e], off_h[e + 1]
        if hi == lo:
            continue
        r1 = oracle.qlinear_fp8(rows_h[lo:hi], *oracle.quant_weight_fp8(W1[e]), b1[e], oracle.EPI_GELU_TANH)
        assert_within(host_f64(h)[lo:hi], r1, D, "bf16", "gelu_tanh")
        r2 = oracle.qlinear_fp8(h_bits[lo:hi], *oracle.quant_weight_fp8(W2[e]))   # on the hidden values that were stored
        g = share.view(-1).double().cpu().numpy()[order_h[lo:hi], None]
        np.add.at(want, order_h[lo:hi] // top, g * r2["y"])
        np.add.at(size, order_h[lo:hi] // top, g * r2["size"])
    # the second linear's roundings and those of the weighted sum
    assert np.all(np.abs(host_f64(out) - want) <= (127 + 5 + 3 + 2 * top) * 2.0 ** -23 * size)


@pytest.mark.parametrize("M", [2, 50, 400])
def test_captured_and_replayed_beside_eager_work(M):
    rng = np.random.default_rng(M)
    K, N, E = 384, 264, 4
    W = np.stack([weights(rng, N, K) for _ in range(E)])
    pw, one = qc.pack_weight_fp8_t(dev(W)), qc.pack_weight_fp8_t(dev(W[0]))
    X = torch.randn(M, K, device="cuda")
    off = torch.tensor([0, M // 3, M // 2, M // 2, M], dtype=torch.int32, device="cuda")
    ws, Y, Z = qc.qlinear_fp8_workspace_t(M, K, N), torch.empty(M, N, device="cuda"), torch.empty(M, N, device="cuda")
    codes, scales = torch.empty(M, K, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(M, 3, device="cuda")

    def step():
        qc.quant_act_fp8_t(X, codes, scales)
        qc.qlinear_fp8_t(X, one, None, "none", "f32", ws, Y)
        qc.qlinear_fp8_grouped_t(X, pw, off, None, "none", "f32", ws, Z)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for turn in range(4):
        X.copy_(torch.randn(M, K, device="cuda"))
        cut = sorted(int(v) for v in rng.integers(0, M + 1, size=3))
        off.copy_(torch.tensor([0, *cut, M], dtype=torch.int32))
        want = [t.clone() for t in (*qc.quant_act_fp8_t(X), qc.qlinear_fp8_t(X, one, out="f32"), qc.qlinear_fp8_grouped_t(X, pw, off, out="f32"))]
        for t in (Y, Z, scales):
            t.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = (codes, scales, Y, Z)
        assert all(torch.equal(g.view(torch.uint8) if g.dtype == torch.float8_e4m3fn else g, w.view(torch.uint8) if w.dtype == torch.float8_e4m3fn else w)
                   for g, w in zip(got, want)), turn


@pytest.mark.parametrize("M", [4, 1500])
def test_on_two_streams_at_once(M):
    K, N = 1152, 512
    pw = qc.pack_weight_fp8_t(torch.randn(N, K, device="cuda") * 0.02)
    Xs = [torch.randn(M, K, device="cuda") for _ in range(2)]
    want = [qc.qlinear_fp8_t(X, pw, out="f32") for X in Xs]
    spaces = [qc.qlinear_fp8_workspace_t(M, K, N) for _ in range(2)]
    out = [[torch.empty(M, N, device="cuda") for _ in range(6)] for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for i in range(6):
        for s in range(2):
            with torch.cuda.stream(streams[s]):
                qc.qlinear_fp8_t(Xs[s], pw, None, "none", "f32", spaces[s], out[s][i])
    torch.cuda.synchronize()
    assert all(torch.equal(y, want[s]) for s in range(2) for y in out[s])


def test_helpers_refuse_tensors_of_other_kinds_on_the_gpu():
    X, pw = torch.zeros(4, 16, device="cuda"), qc.pack_weight_fp8_t(torch.zeros(8, 16, device="cuda"))
    for args in (dict(bias=torch.zeros(7, device="cuda")), dict(bias=torch.zeros(8)), dict(Y=torch.zeros(4, 8, device="cuda")),
                 dict(Y=torch.zeros(3, 8, dtype=torch.bfloat16, device="cuda")), dict(workspace=torch.zeros(4, 4, dtype=torch.uint8, device="cuda"))):
        with pytest.raises((ValueError, TypeError)):
            qc.qlinear_fp8_t(X, pw, **args)
    with pytest.raises(ValueError):
        qc.qlinear_fp8_t(torch.zeros(4, 17, device="cuda"), pw)
    with pytest.raises(KeyError):
        qc.qlinear_fp8_t(X, pw, epi="relu")
    with pytest.raises(KeyError):
        qc.qlinear_fp8_t(X, pw, out="i32")
    with pytest.raises(qc.QcError):
        qc.qlinear_fp8_t(X, pw, workspace=torch.zeros(256, dtype=torch.uint8, device="cuda"))
    with pytest.raises(qc.QcError):
        qc.qlinear_fp8_t(torch.zeros(0, 16, device="cuda"), pw)


def test_a_weight_that_is_not_what_it_says_is_refused():
    """Its blob too short for its sizes, or its scales."""
    X, pw = torch.zeros(4, 128, device="cuda"), qc.pack_weight_fp8_t(torch.zeros(128, 128, device="cuda"))
    off = torch.tensor([0, 2, 4], dtype=torch.int32, device="cuda")
    for bad in (qc.PackedWeightFp8(pw.blob[:-1], pw.scale, 1, 128, 128), qc.PackedWeightFp8(pw.blob, torch.zeros(1, 2, 1, device="cuda"), 1, 256, 128),
                qc.PackedWeightFp8(pw.blob, pw.scale, 1, 129, 128)):
        for helper in (qc.qlinear_fp8_t, qc._python_helpers.get("qlinear_fp8_t", qc.qlinear_fp8_t)):
            with pytest.raises(ValueError, match="blob|scale"):
                helper(X, bad, workspace=qc.qlinear_fp8_workspace_t(4, 128, bad.N), Y=torch.zeros(4, bad.N, dtype=torch.bfloat16, device="cuda"))
        with pytest.raises(ValueError, match="blob|scale"):
            qc.unpack_weight_codes_fp8_t(bad)
    with pytest.raises(ValueError, match="blob"):
        qc.qlinear_fp8_grouped_t(X, qc.PackedWeightFp8(pw.blob, torch.zeros(2, 1, 1, device="cuda"), 2, 128, 128), off)


def test_native_helpers_are_the_python_ones():
    """The same bits, tensors and errors, in any form of the call."""
    qc._use_native_helpers()
    g = torch.Generator(device="cuda").manual_seed(3)
    X = torch.randn(40, 300, generator=g, device="cuda").bfloat16()
    W = torch.randn(3, 70, 300, generator=g, device="cuda")
    pw, one = qc.pack_weight_fp8_t(W), qc.pack_weight_fp8_t(W[0].contiguous())
    off, bias = torch.tensor([0, 11, 11, 40], dtype=torch.int32, device="cuda"), torch.randn(3, 70, generator=g, device="cuda")
    ws = qc.qlinear_fp8_workspace_t(40, 300, 70)

    def Y(dtype=torch.bfloat16):
        return torch.zeros(40, 70, dtype=dtype, device="cuda")

    calls = [("quant_act_fp8_t", (X,), dict), ("quant_act_fp8_t", (X.float(),), lambda: dict(x_scale=torch.empty(40, 3, device="cuda"))),
             ("quant_act_fp8_t", (X, torch.empty(40, 300, dtype=torch.float8_e4m3fn, device="cuda")), dict),
             ("quant_act_fp8_t", (X, torch.empty(40, 299, dtype=torch.float8_e4m3fn, device="cuda")), dict), ("quant_act_fp8_t", (X.t(),), dict),
             ("quant_act_fp8_t", (X.half(),), dict), ("quant_act_fp8_t", (X[:0],), dict), ("quant_act_fp8_t", (X.cpu(),), dict),
             ("qlinear_fp8_t", (X, one), lambda: dict(workspace=ws, Y=Y(), bias=bias[0])), ("qlinear_fp8_t", (X, one), dict),
             ("qlinear_fp8_t", (X, one, bias[1], "gelu_erf", "f32", ws), lambda: dict(Y=Y(torch.float32))),
             ("qlinear_fp8_t", (X, one), lambda: dict(workspace=ws, Y=Y(torch.float32))), ("qlinear_fp8_t", (X, one), lambda: dict(workspace=ws[:64], Y=Y())),
             ("qlinear_fp8_t", (X, pw), lambda: dict(workspace=ws, Y=Y())), ("qlinear_fp8_t", (X, one), lambda: dict(workspace=ws, Y=Y(), bias=bias)),
             ("qlinear_fp8_t", (X, one), lambda: dict(workspace=ws, Y=Y(), epi="relu")), ("qlinear_fp8_t", (X, one), lambda: dict(workspace=ws, Y=Y(), out="i32")),
             ("qlinear_fp8_t", (X[:, :299], one), lambda: dict(workspace=ws, Y=Y())), ("qlinear_fp8_t", (X, None), lambda: dict(workspace=ws, Y=Y())),
             ("qlinear_fp8_grouped_t", (X, pw, off), lambda: dict(workspace=ws, Y=Y(), bias=bias, epi="gelu_tanh")),
             ("qlinear_fp8_grouped_t", (X, pw, off), lambda: dict(workspace=ws)), ("qlinear_fp8_grouped_t", (X, one, off[:2]), lambda: dict(workspace=ws, Y=Y())),
             ("qlinear_fp8_grouped_t", (X, pw, off.long()), lambda: dict(workspace=ws, Y=Y())), ("qlinear_fp8_grouped_t", (X, pw, off[1:]), lambda: dict(workspace=ws, Y=Y())),
             ("qlinear_fp8_grouped_t", (X, pw, off), lambda: dict(workspace=ws, Y=Y(), bias=bias[0]))]

    def outcome(f, args, kwargs):
        try:
            r = f(*args, **kwargs)
        except Exception as e:   # the type and the text are what is compared
            return type(e), str(e)
        return [t.clone() for t in (r if isinstance(r, tuple) else (r,))]

    for name, args, options in calls:
        want, got = outcome(qc._python_helpers[name], args, options()), outcome(getattr(qc, name), args, options())
        if isinstance(want, tuple):
            assert got == want, (name, got, want)
        else:
            assert isinstance(got, list) and all(g.dtype == w.dtype and torch.equal(g.view(torch.uint8), w.view(torch.uint8)) for g, w in zip(got, want)), name
