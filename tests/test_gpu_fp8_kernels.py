"""The 8-bit floating-point linears on the GPU, kernel by kernel: each test asks what a call's launches are and asserts it, so
that another choice of kernel cannot leave it without the one that it is for."""
import numpy as np
import pytest
import torch

from paper_2503_06545_amd import binding as qc
from test_gpu_fp8 import KERNELS, which

pytestmark = pytest.mark.gpu

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
