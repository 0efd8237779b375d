// Device helpers of the 8-bit floating-point linear: pieces of a row, the cast, operands and products of the matrix unit.
#pragma once

#include "qc_device.h"
#include "qc_fp8.h"

namespace qc {
namespace {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v8i __attribute__((ext_vector_type(8)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// 16 B of a row of K at any alignment, from column col on; zeros past the row's end
template <bool NT = false, typename XT>
__device__ inline uint4 load_piece(const XT *xrow, int64_t col, int64_t K) {
    constexpr int E = 16 / (int)sizeof(XT);
    const int64_t past = col + E - K;   // elements of the piece past the row's end
    if (past <= 0) {
        const u32x4_any *const p = reinterpret_cast<const u32x4_any *>(xrow + col);
        const u32x4_any t = NT ? __builtin_nontemporal_load(p) : *p;
        return make_uint4(t.x, t.y, t.z, t.w);
    }
    if (past >= E) return make_uint4(0, 0, 0, 0);
    if (K >= E) {   // loaded so that it ends with the row, and moved down
        const u32x4_any t = *reinterpret_cast<const u32x4_any *>(xrow + K - E);
        return move_down(make_uint4(t.x, t.y, t.z, t.w), (int)past * (int)(sizeof(XT) / 2));
    }
    uint32_t w[4] = {0, 0, 0, 0};   // a row of less than 16 B
    for (int e = 0; e < (int)(E - past); ++e) {
        if constexpr (sizeof(XT) == 4) w[e] = __float_as_uint(xrow[col + e]);
        else w[e / 2] |= (uint32_t)xrow[col + e] << (16 * (e % 2));
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// four quotients -> four e4m3 codes in a dword, element 0 lowest
__device__ inline uint32_t e4m3x4(float q0, float q1, float q2, float q3) {
    const int w = __builtin_amdgcn_cvt_pk_fp8_f32(q0, q1, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(q2, q3, w, true);
}

// One operand of 16 rows x 128 k as the matrix unit takes it.  The instructions for e4m3 operands line up eight products with
// the largest of them before they add, and cut off what is then too low: the sum of a block comes out 1.4e-5 off (2-norm,
// normal values; 2.2e-5 after GELU, 8e-5 and towards zero for positive values spread over twelve powers of two), where the
// instruction for bf16 operands is 1e-8 off.  That is enough for outputs that are rounded to bf16 (by up to 2^-8 of each), not for binary32 ones.  EXACT widens the codes to bf16, exactly, and takes four instructions of 32 k instead
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

// which rows a block's tile has and whose weights it takes; expert < 0: none
struct Where {
    int64_t row0;
    int rows, expert;
};

}  // namespace
}  // namespace qc
