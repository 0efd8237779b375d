// C ABI entry points of the 8-bit floating-point linear: argument checks first, then launches on the caller's
// stream.  Nothing here allocates or synchronises.
#include "qc_fp8.h"

using namespace qc;

namespace {

bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

constexpr int64_t kBlocksMost = 0xffffffffLL / 256;   // of 256 threads in a launch

#define QC_TRY(expr)                          \
    do {                                      \
        const qc_status st_ = (expr);         \
        if (st_ != QC_OK) return st_;         \
    } while (0)

qc_status device_status(hipError_t e) { return e == hipSuccess ? QC_OK : QC_ERR_DEVICE; }

// INVALID_ARG (pointers, sizes, enums, alignment), then UNSUPPORTED, then WORKSPACE, as for the integer linears

qc_status check_activation(const void *X, qc_dtype xdt, int64_t M, int64_t K) {
    if (!X || M < 1 || K < 1) return QC_ERR_INVALID_ARG;
    if (xdt != QC_F32 && xdt != QC_BF16) return QC_ERR_INVALID_ARG;
    return aligned(X, 16) ? QC_OK : QC_ERR_INVALID_ARG;
}

qc_status check_weight_side(const void *packed, const float *w_scale, const float *bias, qc_epilogue epi, const void *Y,
                            qc_out ydt, int64_t M, int64_t K, int64_t N) {
    if (!packed || !w_scale || !Y || M < 1 || K < 1 || N < 1) return QC_ERR_INVALID_ARG;
    if (epi != QC_EPI_NONE && epi != QC_EPI_GELU_TANH && epi != QC_EPI_GELU_ERF) return QC_ERR_INVALID_ARG;
    if (ydt != QC_OUT_F32 && ydt != QC_OUT_BF16 && ydt != QC_OUT_I32_ACC) return QC_ERR_INVALID_ARG;
    if (!aligned(packed, 256) || !aligned(w_scale, 16) || !aligned(Y, 16) || (bias && !aligned(bias, 16))) return QC_ERR_INVALID_ARG;
    return QC_OK;
}

qc_status check_quant_supported(int64_t M, int64_t K) {
    return K > QC_MAX_K || M > 0x7fffffffLL || fp8_quant_row_blocks(M) * fp8_blocks(K) >= kBlocksMost ? QC_ERR_UNSUPPORTED : QC_OK;
}

qc_status check_gemm_supported(int64_t M, int64_t K, int64_t N, int64_t experts, qc_out ydt) {
    if (ydt == QC_OUT_I32_ACC || M > 0x7fffffffLL || qc_packed_weight_fp8_bytes(experts, N, K) == 0) return QC_ERR_UNSUPPORTED;
    const int64_t tiles = M / kFp8TokensLeast + experts;
    return tiles * (round_up(N, kTileN) / kTileN) > kBlocksMost ? QC_ERR_UNSUPPORTED : QC_OK;
}

qc_status check_workspace(const void *workspace) { return workspace && aligned(workspace, 256) ? QC_OK : QC_ERR_INVALID_ARG; }

Fp8GemmArgs gemm_args(void *workspace, int64_t M, int64_t K, const void *packed, const float *w_scale, int64_t N, const float *bias,
                      void *Y, const Fp8Plan &plan, int64_t experts, bool grouped) {
    const Fp8Workspace ws = fp8_workspace(M, K);
    uint8_t *const base = (uint8_t *)workspace;
    Fp8GemmArgs a{};
    a.x_tiled = base + ws.codes_offset;
    a.x_scale = (float *)base;
    a.w_codes = (const uint8_t *)packed + kPackedHeaderBytes;
    a.w_scale = w_scale;
    a.bias = bias;
    a.Y = Y;
    a.map = grouped && !plan.few.tokens ? (Fp8Tile *)(base + ws.map_offset) : nullptr;
    a.M = M;
    a.N = N;
    a.Mp = ws.Mp;
    a.w_expert_bytes = fp8_weight_bytes(N, K);
    a.KB = (int)ws.KB;
    a.m_tiles = (int)(grouped ? fp8_tiles_most(M, experts, plan.tokens) : (M + plan.tokens - 1) / plan.tokens);
    a.n_tiles = (int)(round_up(N, kTileN) / kTileN);
    // Token tiles of the patch that the blocks of an XCD work on: eight where there are many channel tiles, else three, as good as
    // two and four there (us at 3 and 8: 131072 x 1152 x 4608 691 678, 32768 x 1152 x 4608 of 16 experts 211 208; 65536 x 4608 x 1152 308 311,
    // of 64 experts 524 566, 12000 x 9216 x 1152 118 121, 40000 x 640 x 1800 65.6 67.1).
    a.group_m = a.n_tiles > 16 ? 8 : 3;
    return a;
}

// the products of codes in the workspace
qc_status gemm(const Fp8GemmArgs &a, int64_t K, const int32_t *offsets, int64_t experts, const Fp8Plan &plan, qc_epilogue epi,
               qc_out ydt, void *stream) {
    if (plan.few.tokens) return device_status(launch_fp8_few(nullptr, QC_F32, K, offsets, (int)experts, a, plan.few, epi, ydt, (hipStream_t)stream));
    return device_status(launch_fp8_gemm(a, plan.tokens, epi, ydt, (hipStream_t)stream));
}

// Both launches of a linear, or the one.  Y may lie over X: in two launches X has been read when the products are
// written; in one launch the blocks that write Y run beside others that still read X.
qc_status linear(const void *X, qc_dtype xdt, int64_t M, int64_t K, const int32_t *offsets, int64_t experts, const void *packed,
                 const float *w_scale, int64_t N, const float *bias, qc_epilogue epi, void *Y, qc_out ydt, void *workspace, void *stream) {
    const size_t x_bytes = (size_t)M * (size_t)K * (xdt == QC_BF16 ? 2 : 4), y_bytes = (size_t)M * (size_t)N * (ydt == QC_OUT_BF16 ? 2 : 4);
    const Fp8Plan plan = fp8_plan(M, N, K, xdt, (int)experts, offsets != nullptr, ydt, !overlap(X, x_bytes, Y, y_bytes));
    const Fp8GemmArgs a = gemm_args(workspace, M, K, packed, w_scale, N, bias, Y, plan, experts, offsets != nullptr);
    if (plan.fused) return device_status(launch_fp8_few(X, xdt, K, offsets, (int)experts, a, plan.few, epi, ydt, (hipStream_t)stream));
    QC_TRY(device_status(launch_fp8_quant(X, xdt, M, K, nullptr, a.x_tiled, a.x_scale, offsets, (int)experts, plan.tokens, a.map, (hipStream_t)stream)));
    return gemm(a, K, offsets, experts, plan, epi, ydt, stream);
}

}  // namespace

extern "C" size_t qc_packed_weight_fp8_bytes(int64_t experts, int64_t N, int64_t K) {
    if (experts < 1 || N < 1 || K < 1 || experts > QC_MAX_EXPERTS || N > QC_MAX_N || K > QC_MAX_K) return 0;
    if (experts * (round_up(N, kTileN) / kTileN) * fp8_blocks(K) > kBlocksMost) return 0;
    return (size_t)kPackedHeaderBytes + (size_t)experts * (size_t)fp8_weight_bytes(N, K) + kFp8WeightSlack;
}

extern "C" qc_status qc_pack_weight_fp8(const float *W, int64_t experts, int64_t N, int64_t K, void *packed, float *w_scale,
                                        void *stream) {
    if (!W || !packed || !w_scale || experts < 1 || N < 1 || K < 1) return QC_ERR_INVALID_ARG;
    if (!aligned(W, 16) || !aligned(packed, 256) || !aligned(w_scale, 16)) return QC_ERR_INVALID_ARG;
    if (qc_packed_weight_fp8_bytes(experts, N, K) == 0) return QC_ERR_UNSUPPORTED;
    return device_status(launch_fp8_pack(W, experts, N, K, (uint8_t *)packed, w_scale, (hipStream_t)stream));
}

extern "C" qc_status qc_unpack_weight_codes_fp8(const void *packed, int64_t experts, int64_t N, int64_t K, uint8_t *codes,
                                                void *stream) {
    if (!packed || !codes || experts < 1 || N < 1 || K < 1 || !aligned(packed, 256)) return QC_ERR_INVALID_ARG;
    if (qc_packed_weight_fp8_bytes(experts, N, K) == 0) return QC_ERR_UNSUPPORTED;
    return device_status(launch_fp8_unpack((const uint8_t *)packed, experts, N, K, codes, (hipStream_t)stream));
}

extern "C" qc_status qc_quant_act_fp8(const void *X, qc_dtype xdt, int64_t M, int64_t K, uint8_t *qx, float *x_scale, void *stream) {
    QC_TRY(check_activation(X, xdt, M, K));
    if (!qx || !x_scale || !aligned(qx, 16) || !aligned(x_scale, 4)) return QC_ERR_INVALID_ARG;
    QC_TRY(check_quant_supported(M, K));
    return device_status(launch_fp8_quant(X, xdt, M, K, qx, nullptr, x_scale, nullptr, 0, 0, nullptr, (hipStream_t)stream));
}

extern "C" size_t qc_qlinear_fp8_workspace_bytes(int64_t M, int64_t K, int64_t N) {
    if (M < 1 || K < 1 || N < 1 || N > QC_MAX_N || check_quant_supported(M, K) != QC_OK) return 0;
    return fp8_workspace(M, K).total_bytes;
}

extern "C" qc_status qc_qlinear_fp8_quant(const void *X, qc_dtype xdt, int64_t M, int64_t K, void *workspace, size_t workspace_bytes,
                                          void *stream) {
    QC_TRY(check_activation(X, xdt, M, K));
    QC_TRY(check_workspace(workspace));
    QC_TRY(check_quant_supported(M, K));
    const Fp8Workspace ws = fp8_workspace(M, K);
    if (workspace_bytes < ws.total_bytes) return QC_ERR_WORKSPACE;
    uint8_t *const base = (uint8_t *)workspace;
    return device_status(launch_fp8_quant(X, xdt, M, K, nullptr, base + ws.codes_offset, (float *)base, nullptr, 0, 0, nullptr,
                                          (hipStream_t)stream));
}

extern "C" qc_status qc_qlinear_fp8_gemm(const void *workspace, size_t workspace_bytes, int64_t M, int64_t K, const void *packed,
                                         const float *w_scale, int64_t N, const float *bias, qc_epilogue epi, void *Y, qc_out ydt,
                                         void *stream) {
    QC_TRY(check_weight_side(packed, w_scale, bias, epi, Y, ydt, M, K, N));
    QC_TRY(check_workspace(workspace));
    QC_TRY(check_gemm_supported(M, K, N, 1, ydt));
    if (workspace_bytes < fp8_workspace(M, K).total_bytes) return QC_ERR_WORKSPACE;
    const Fp8Plan plan = fp8_plan(M, N, K, QC_F32, 1, false, ydt, false);
    return gemm(gemm_args(const_cast<void *>(workspace), M, K, packed, w_scale, N, bias, Y, plan, 1, false), K, nullptr, 1, plan, epi, ydt, stream);
}

extern "C" qc_status qc_qlinear_fp8(const void *X, qc_dtype xdt, int64_t M, int64_t K, const void *packed, const float *w_scale,
                                    int64_t N, const float *bias, qc_epilogue epi, void *Y, qc_out ydt, void *workspace,
                                    size_t workspace_bytes, void *stream) {
    QC_TRY(check_activation(X, xdt, M, K));
    QC_TRY(check_weight_side(packed, w_scale, bias, epi, Y, ydt, M, K, N));
    QC_TRY(check_workspace(workspace));
    QC_TRY(check_quant_supported(M, K));
    QC_TRY(check_gemm_supported(M, K, N, 1, ydt));
    if (workspace_bytes < fp8_workspace(M, K).total_bytes) return QC_ERR_WORKSPACE;
    return linear(X, xdt, M, K, nullptr, 1, packed, w_scale, N, bias, epi, Y, ydt, workspace, stream);
}

extern "C" qc_status qc_qlinear_fp8_grouped(const void *X, qc_dtype xdt, int64_t M, int64_t K, const int32_t *expert_offsets,
                                            int64_t experts, const void *packed, const float *w_scale, int64_t N, const float *bias,
                                            qc_epilogue epi, void *Y, qc_out ydt, void *workspace, size_t workspace_bytes,
                                            void *stream) {
    QC_TRY(check_activation(X, xdt, M, K));
    QC_TRY(check_weight_side(packed, w_scale, bias, epi, Y, ydt, M, K, N));
    if (!expert_offsets || !aligned(expert_offsets, 4) || experts < 1) return QC_ERR_INVALID_ARG;
    QC_TRY(check_workspace(workspace));
    if (experts > QC_MAX_EXPERTS) return QC_ERR_UNSUPPORTED;
    QC_TRY(check_quant_supported(M, K));
    QC_TRY(check_gemm_supported(M, K, N, experts, ydt));
    if (workspace_bytes < fp8_workspace(M, K).total_bytes) return QC_ERR_WORKSPACE;
    return linear(X, xdt, M, K, expert_offsets, experts, packed, w_scale, N, bias, epi, Y, ydt, workspace, stream);
}

extern "C" int qc_debug_linear_plan_fp8(int64_t M, int64_t K, int64_t N, int64_t experts, qc_out ydt, int32_t *plan) {
    if (M < 1 || K < 1 || N < 1 || experts < 0 || !plan || (ydt != QC_OUT_F32 && ydt != QC_OUT_BF16)) return -1;
    const int64_t matrices = experts ? experts : 1;
    if (check_quant_supported(M, K) != QC_OK || check_gemm_supported(M, K, N, matrices, ydt) != QC_OK) return -1;
    const Fp8Plan p = fp8_plan(M, N, K, QC_BF16, (int)matrices, experts != 0, ydt, true);
    plan[0] = p.few.tokens ? kGemmSmall : kGemmRing;
    plan[1] = p.tokens;
    plan[2] = p.few.tokens ? kFragRows * p.few.frags : kTileN;
    plan[3] = p.fused;
    return 0;
}
