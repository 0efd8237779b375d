"""The 8-bit floating-point operators without a GPU: the oracle they are compared with, sizes, and everything that is
refused before a launch."""
import numpy as np
import pytest
import torch

import oracle
from paper_2503_06545_amd import binding as qc
from paper_2503_06545_amd import synth


# ---- the oracle ----------------------------------------------------------------------------------

def test_e4m3_values_and_rounding_agree_with_torchs_type():
    codes = np.arange(256, dtype=np.uint8)
    want = torch.from_numpy(codes).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(oracle.e4m3_values(codes), want, equal_nan=True)
    # every bf16 of magnitude 448 at most, both signs, and every midpoint of two neighbours
    bits = np.arange(65536, dtype=np.uint32)
    v = (bits << 16).view(np.float32)
    v = v[np.abs(v) <= 448.0]
    table = oracle.E4M3[:127]
    mid = ((table[1:] + table[:-1]) / 2).astype(np.float32)
    for x in (v, mid, -mid):
        got = oracle.e4m3_codes(x)
        assert np.array_equal(got, torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy())


def test_block_quantizer_brute_force():
    rng = np.random.default_rng(5)
    x = rng.standard_normal((3, 300)).astype(np.float32)
    x[1, 128:256] = 0.0
    q, s = oracle.quant_act_fp8(x)
    assert q.shape == (3, 300) and s.shape == (3, 3)
    for m in range(3):
        for b in range(3):
            part = x[m, 128 * b:128 * b + 128]
            want = np.float32(max(np.abs(part).max(), np.float32(2.0 ** -64))) / np.float32(448)
            assert s[m, b] == want
            back = oracle.e4m3_values(q[m, 128 * b:128 * b + 128]) * float(want)
            # half a step: 2^-4 relative, 2^-10 of a scale below the normal codes; the quotient's rounding beside it
            assert np.all(np.abs(back - part) <= np.maximum(np.abs(part) * 2.0 ** -4, want * 2.0 ** -10) * (1 + 2.0 ** -20))
            if np.abs(part).max() > 0:
                assert np.abs(oracle.e4m3_values(q[m, 128 * b:128 * b + 128])).max() == 448.0
    qw, sw = oracle.quant_weight_fp8(x)
    assert sw.shape == (1, 3) and sw[0, 0] == np.float32(np.abs(x[:, :128]).max()) / np.float32(448)


def test_oracle_linear_is_the_dequantized_product():
    rng = np.random.default_rng(6)
    x, W = rng.standard_normal((5, 200)).astype(np.float32), rng.standard_normal((140, 200)).astype(np.float32)
    qw, sw = oracle.quant_weight_fp8(W)
    ref = oracle.qlinear_fp8(x, qw, sw)
    y = np.zeros((5, 140))
    for m in range(5):
        for n in range(140):
            for b in range(2):
                k = slice(128 * b, 128 * b + 128)
                dot = float(np.dot(oracle.e4m3_values(ref["qx"][m, k]), oracle.e4m3_values(qw[n, k])))
                y[m, n] += float(ref["sx"][m, b]) * float(sw[n // 128, b]) * dot
    assert np.allclose(ref["y"], y, rtol=1e-12, atol=1e-12)
    assert np.abs(ref["y"] - x.astype(np.float64) @ W.T.astype(np.float64)).max() < 2.0   # quantization noise only


# ---- sizes and refusals --------------------------------------------------------------------------

def test_size_queries():
    # a header, whole blocks of 128 x 128, and three more of them that the GEMM runs past the last one
    assert qc.qc_packed_weight_fp8_bytes(1, 3456, 1152) == 256 + 3456 * 1152 + 3 * 16384
    assert qc.qc_packed_weight_fp8_bytes(5, 200, 100) == 256 + 5 * 256 * 128 + 3 * 16384
    for bad in ((0, 8, 8), (1, 0, 8), (1, 8, 0), (qc.QC_MAX_EXPERTS + 1, 8, 8), (1, qc.QC_MAX_N + 1, 8), (1, 8, qc.QC_MAX_K + 1),
                (1024, 1 << 24, 1 << 16)):
        assert qc.qc_packed_weight_fp8_bytes(*bad) == 0
    # codes, one scale per token and block, and a map of the tiles of any grouping of the rows
    got = qc.qc_qlinear_fp8_workspace_bytes(300, 1000, 7)
    assert got >= 320 * 1024 + 320 * 8 * 4 + 300 * 16 and got % 256 == 0
    for bad in ((0, 8, 8), (8, 0, 8), (8, 8, 0), (8, qc.QC_MAX_K + 1, 8)):
        assert qc.qc_qlinear_fp8_workspace_bytes(*bad) == 0


def test_argument_errors_come_before_any_launch():
    A = 0x10000  # a fake, aligned, never dereferenced address: every call below must fail first
    bad, unsupported, workspace = qc.QC_ERR_INVALID_ARG, qc.QC_ERR_UNSUPPORTED, qc.QC_ERR_WORKSPACE
    quant = dict(X=A, xdt=qc.QC_BF16, M=4, K=16, qx=A, x_scale=A)
    for change, want in ((dict(X=None), bad), (dict(xdt=7), bad), (dict(M=0), bad), (dict(K=0), bad), (dict(X=A + 8), bad),
                         (dict(qx=None), bad), (dict(qx=A + 4), bad), (dict(x_scale=None), bad), (dict(x_scale=A + 2), bad),
                         (dict(K=qc.QC_MAX_K + 1), unsupported), (dict(M=1 << 31), unsupported), (dict(M=1 << 30, K=9216), unsupported)):
        assert qc.qc_quant_act_fp8(**{**quant, **change}) == want, change
    pack = dict(W=A, experts=2, N=8, K=16, packed=A, w_scale=A)
    for change, want in ((dict(W=None), bad), (dict(W=A + 4), bad), (dict(experts=0), bad), (dict(N=0), bad), (dict(packed=A + 16), bad),
                         (dict(w_scale=A + 4), bad), (dict(experts=qc.QC_MAX_EXPERTS + 1), unsupported), (dict(N=qc.QC_MAX_N + 1), unsupported)):
        assert qc.qc_pack_weight_fp8(**{**pack, **change}) == want, change
    assert qc.qc_unpack_weight_codes_fp8(None, 1, 8, 16, A) == bad
    assert qc.qc_unpack_weight_codes_fp8(A, 1, 8, qc.QC_MAX_K + 1, A) == unsupported
    linear = dict(X=A, xdt=qc.QC_BF16, M=4, K=16, packed=A, w_scale=A, N=8, bias=None, epi=qc.QC_EPI_NONE, Y=A, ydt=qc.QC_OUT_BF16,
                  workspace=A, workspace_bytes=1 << 30)
    common = ((dict(packed=None), bad), (dict(packed=A + 64), bad), (dict(w_scale=None), bad), (dict(bias=A + 4), bad), (dict(epi=9), bad),
              (dict(ydt=9), bad), (dict(Y=None), bad), (dict(Y=A + 8), bad), (dict(workspace=None), bad), (dict(workspace=A + 16), bad),
              (dict(N=0), bad), (dict(M=0), bad), (dict(K=qc.QC_MAX_K + 1), unsupported), (dict(N=qc.QC_MAX_N + 1), unsupported),
              (dict(ydt=qc.QC_OUT_I32_ACC), unsupported), (dict(M=1 << 31), unsupported), (dict(workspace_bytes=64), workspace),
              (dict(workspace_bytes=qc.qc_qlinear_fp8_workspace_bytes(4, 16, 8) - 1), workspace))
    inputs = ((dict(X=None), bad), (dict(X=A + 2), bad), (dict(xdt=5), bad))
    for change, want in common + inputs:
        assert qc.qc_qlinear_fp8(**{**linear, **change}) == want, change
    halves = {k: v for k, v in linear.items() if k not in ("X", "xdt")}
    for change, want in common:
        assert qc.qc_qlinear_fp8_gemm(**{**halves, **change}) == want, change
    assert qc.qc_qlinear_fp8_quant(A, qc.QC_BF16, 4, 16, A, 64) == workspace
    assert qc.qc_qlinear_fp8_quant(A, qc.QC_BF16, 4, 16, None, 1 << 30) == bad
    assert qc.qc_qlinear_fp8_quant(A, qc.QC_BF16, 4, qc.QC_MAX_K + 1, A, 1 << 40) == unsupported
    grouped = dict(linear, expert_offsets=A, experts=3)
    for change, want in common + inputs + ((dict(expert_offsets=None), bad), (dict(expert_offsets=A + 2), bad), (dict(experts=0), bad),
                                           (dict(experts=qc.QC_MAX_EXPERTS + 1), unsupported)):
        assert qc.qc_qlinear_fp8_grouped(**{**grouped, **change}) == want, change


def test_helpers_refuse_what_is_not_on_the_gpu_or_of_another_kind():
    X, W = torch.zeros(4, 16), torch.zeros(8, 16)
    with pytest.raises(ValueError, match="GPU"):
        qc.quant_act_fp8_t(X)
    with pytest.raises(ValueError, match="GPU"):
        qc.pack_weight_fp8_t(W)
    with pytest.raises(TypeError):
        qc.pack_weight_fp8_t(W.double())
    with pytest.raises(TypeError):
        qc.quant_act_fp8_t(X.half())
    with pytest.raises(ValueError, match="contiguous"):
        qc.quant_act_fp8_t(torch.zeros(16, 4).t())
    with pytest.raises(ValueError):
        qc.quant_act_fp8_t(torch.zeros(16))
    pw = qc.PackedWeightFp8(torch.zeros(256, dtype=torch.uint8), torch.zeros(2, 1, 1), 2, 8, 16)
    with pytest.raises(ValueError, match="grouped"):
        qc.qlinear_fp8_t(X, pw)
    with pytest.raises(TypeError, match="expert_offsets"):
        qc.qlinear_fp8_grouped_t(X, pw, torch.zeros(3, dtype=torch.int64))
    with pytest.raises(ValueError, match="expert_offsets"):
        qc.qlinear_fp8_grouped_t(X, pw, torch.zeros(2, dtype=torch.int32))


def test_bf16_inputs_are_widened_before_the_quantizer():
    x = np.random.default_rng(1).standard_normal((4, 130)).astype(np.float32)
    bits = synth.to_bf16_bits(x)
    for got, want in zip(oracle.quant_act_fp8(bits), oracle.quant_act_fp8(oracle.widen_f32(bits))):
        assert np.array_equal(got, want)


def test_plans():
    """Few tokens go out in one launch, a long reduction of a few hundred through the same kernel from codes, many through the
    ring, on lower tiles the fewer there are; what is refused has no plan."""
    plan = qc.linear_plan_fp8
    assert plan(1, 1152, 6912) == {"kernel": "few", "tokens": 16, "channels": 32, "fused": True}
    assert plan(1, 4608, 1152)["channels"] == 16 and plan(130, 1152, 1152)["channels"] == 64
    assert plan(300, 4608, 1152) == {"kernel": "few", "tokens": 32, "channels": 64, "fused": False}
    assert plan(600, 4608, 1152, "f32")["kernel"] == plan(600, 4608, 1152)["kernel"] == "few" and plan(1200, 4608, 1152)["kernel"] == "ring"
    assert plan(100, 1152, 9000)["kernel"] == "ring" and plan(16, 1152, 4608, experts=32) == {"kernel": "few", "tokens": 16, "channels": 64, "fused": True}
    assert plan(16, 3951, 3456) == plan(16, 3952, 9000) == {"kernel": "few", "tokens": 32, "channels": 64, "fused": False}
    assert plan(131072, 1152, 4608) == {"kernel": "ring", "tokens": 256, "channels": 128, "fused": False}
    assert plan(131072, 1152, 4608, "f32")["tokens"] == 128 and plan(1200, 1152, 1152)["tokens"] == 64
    assert plan(8, 4608, 1152, experts=32)["fused"] and plan(200, 1152, 4608, experts=32)["tokens"] == 64
    assert plan(16000, 1152, 4608, experts=64)["tokens"] == 128
    for bad in ((0, 8, 8), (8, qc.QC_MAX_K + 1, 8), (8, 8, qc.QC_MAX_N + 1)):
        with pytest.raises(qc.QcError):
            plan(*bad)
    with pytest.raises(qc.QcError):
        plan(8, 8, 8, experts=qc.QC_MAX_EXPERTS + 1)
    with pytest.raises(qc.QcError):
        plan(8, 8, 8, "i32")
