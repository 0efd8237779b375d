// The 8-bit floating-point GEMM with a scale for every block of 128 along the reduction, plain and grouped by expert:
//
//   Y[m, n] = act( sum_b sx[m, b] sw[n / 128, b] P_b[m, n] + bias[n] ),   P_b = sum over the 128 k of block b of qx qw
//
// One v_mfma_f32_16x16x128_f8f6f4 covers a block, so P_b comes out of the matrix unit with nothing to add it to, and the
// scales are one fma per output and block on the vector unit, half as many issue cycles as the matrix instruction's.
#include <type_traits>

#include "qc_device.h"
#include "qc_fp8.h"

namespace qc {
namespace {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v8i __attribute__((ext_vector_type(8)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kThreads = 256;

// One operand of 16 rows x 128 k as the matrix unit takes it.  The instructions for e4m3 operands line up eight products with
// the largest of them before they add, and drop what is then too low: the sum of a block comes out 1.5e-5 off (2-norm,
// normal values), where the instruction for bf16 operands is 1e-8 off.  That is enough for outputs that are rounded to bf16
// (2^-9 each), not for binary32 ones.  EXACT widens the codes to bf16, exactly, and takes four instructions of 32 k instead
// of one of 128 (registers only, random operands, TFLOP/s: 4390 and 2260).
template <bool EXACT>
struct Operand;
template <>
struct Operand<false> {
    v8i v;
    __device__ Operand() {}
    __device__ Operand(v4i lo, v4i hi) : v(__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7)) {}
};
template <>
struct Operand<true> {
    bf16x8 v[4];
    __device__ Operand() {}
    __device__ Operand(v4i lo, v4i hi) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int d0 = j < 2 ? lo[2 * j] : hi[2 * j - 4], d1 = j < 2 ? lo[2 * j + 1] : hi[2 * j - 3];
            const bf16x2 p0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(d0, 1.0f, false), p1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(d0, 1.0f, true);
            const bf16x2 p2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(d1, 1.0f, false), p3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(d1, 1.0f, true);
            v[j] = bf16x8{p0[0], p0[1], p1[0], p1[1], p2[0], p2[1], p3[0], p3[1]};
        }
    }
};

__device__ inline f4 product(const Operand<false> &a, const Operand<false> &b) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a.v, b.v, f4{0.0f, 0.0f, 0.0f, 0.0f}, 0, 0, 0, 0, 0, 0);
}
__device__ inline f4 product(const Operand<true> &a, const Operand<true> &b) {
    f4 c = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v[j], b.v[j], c, 0, 0, 0);
    return c;
}

template <int EPI>
__device__ inline float activation(float y) {
    if (EPI == QC_EPI_GELU_TANH) return gelu_tanh_f(y);
    if (EPI == QC_EPI_GELU_ERF) return gelu_erf_f(y);
    return y;
}

// which rows a block's tile has and whose weights it takes
struct Where {
    int64_t row0;
    int rows, expert;
};
__device__ inline Where tile_of(const Fp8GemmArgs &a, int v, int tokens) {
    if (a.map) {
        const Fp8Tile t = a.map[v];
        return {t.row0, t.rows, t.expert};
    }
    const int64_t row0 = (int64_t)v * tokens, rows = a.M - row0;
    return {row0, (int)(rows < tokens ? rows : tokens), 0};
}

// MI x 16 tokens x 128 channels per wavefront, four wavefronts along the tokens
template <int MI, int OUT, int EPI>
__global__ __launch_bounds__(kThreads) void fp8_tile_kernel(Fp8GemmArgs a) {
    constexpr int TM = 64 * MI;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int c = lane & 15, h = lane >> 4;
    const int v = blockIdx.x / (uint32_t)a.n_tiles, nt = blockIdx.x % (uint32_t)a.n_tiles;
    const Where at = tile_of(a, v, TM);
    const int live = at.rows - wave * (16 * MI);   // rows of this wavefront's tile
    if (at.expert < 0 || live <= 0) return;
    const int64_t m0 = at.row0 + wave * (16 * MI);

    const uint8_t *const wsrc = a.w_codes + at.expert * a.w_expert_bytes + (int64_t)nt * a.KB * kFp8TileBytes + lane * 16;
    const float *const ws = a.w_scale + ((int64_t)at.expert * a.n_tiles + nt) * a.KB;
    // rows past the last live one read that one again and are not stored
    const uint8_t *xsrc[MI];
    int64_t xs[MI][4];
#pragma unroll
    for (int i = 0; i < MI; ++i) {
        const int64_t r = m0 + min(16 * i + c, live - 1);
        xsrc[i] = a.x_tiled + fp8_act_offset(r, 16 * h, a.KB);
#pragma unroll
        for (int q = 0; q < 4; ++q) xs[i][q] = m0 + min(16 * i + 4 * h + q, live - 1);
    }
    f4 acc[MI][8];
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int t = 0; t < 8; ++t) acc[i][t] = f4{0.0f, 0.0f, 0.0f, 0.0f};
    for (int b = 0; b < a.KB; ++b) {
        typedef Operand<OUT == QC_OUT_F32> Op;
        Op x[MI];
        float s[MI][4];
        const float sw = ws[b];
#pragma unroll
        for (int i = 0; i < MI; ++i) {
            const v4i *const p = reinterpret_cast<const v4i *>(xsrc[i] + (int64_t)b * (8 * kFragBytes));
            x[i] = Op(p[0], p[64]);
#pragma unroll
            for (int q = 0; q < 4; ++q) s[i][q] = a.x_scale[b * a.Mp + xs[i][q]] * sw;
        }
#pragma unroll
        for (int t = 0; t < 8; ++t) {
            const v4i *const p = reinterpret_cast<const v4i *>(wsrc + (int64_t)b * kFp8TileBytes + 2 * t * kFragBytes);
            const Op w(p[0], p[64]);
#pragma unroll
            for (int i = 0; i < MI; ++i) {
                const f4 p = product(x[i], w);
#pragma unroll
                for (int q = 0; q < 4; ++q) acc[i][t][q] = fmaf(p[q], s[i][q], acc[i][t][q]);
            }
        }
    }

    const int64_t n0 = (int64_t)nt * kTileN + 8 * c;
    if (n0 >= a.N) return;
    const int cols = (int)(a.N - n0 < 8 ? a.N - n0 : 8);
    float bs[8];
#pragma unroll
    for (int t = 0; t < 8; ++t) bs[t] = a.bias && t < cols ? a.bias[at.expert * a.N + n0 + t] : 0.0f;
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if (16 * i + 4 * h + q >= live) continue;
            const int64_t y0 = (m0 + 16 * i + 4 * h + q) * a.N + n0;
            float y[8];
#pragma unroll
            for (int t = 0; t < 8; ++t) y[t] = activation<EPI>(acc[i][t][q] + bs[t]);
            if (OUT == QC_OUT_F32) {
                float *const p = reinterpret_cast<float *>(a.Y) + y0;
                if (cols == 8) __builtin_memcpy(p, y, sizeof(y));
                else for (int t = 0; t < 8; ++t) if (t < cols) p[t] = y[t];
            } else {
                uint16_t *const p = reinterpret_cast<uint16_t *>(a.Y) + y0;
                uint32_t pk[4];
#pragma unroll
                for (int t = 0; t < 4; ++t) pk[t] = pack_bf16x2(y[2 * t], y[2 * t + 1]);
                if (cols == 8) __builtin_memcpy(p, pk, sizeof(pk));
                else
#pragma unroll
                    for (int t = 0; t < 8; ++t) if (t < cols) p[t] = (uint16_t)(t % 2 ? pk[t / 2] >> 16 : pk[t / 2]);
            }
        }
}

template <int OUT>
hipError_t launch_out(const Fp8GemmArgs &a, qc_epilogue epi, hipStream_t stream) {
    const dim3 grid((unsigned)(a.m_tiles * a.n_tiles)), block(kThreads);
    if (epi == QC_EPI_GELU_TANH) fp8_tile_kernel<2, OUT, QC_EPI_GELU_TANH><<<grid, block, 0, stream>>>(a);
    else if (epi == QC_EPI_GELU_ERF) fp8_tile_kernel<2, OUT, QC_EPI_GELU_ERF><<<grid, block, 0, stream>>>(a);
    else fp8_tile_kernel<2, OUT, QC_EPI_NONE><<<grid, block, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace

int fp8_gemm_tokens(int64_t M, int64_t N, int64_t K, int experts) { return 128; }

hipError_t launch_fp8_gemm(const Fp8GemmArgs &args, int tokens, qc_epilogue epi, qc_out ydt, hipStream_t stream) {
    return ydt == QC_OUT_F32 ? launch_out<QC_OUT_F32>(args, epi, stream) : launch_out<QC_OUT_BF16>(args, epi, stream);
}

}  // namespace qc
