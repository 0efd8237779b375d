// Internal declarations of the 8-bit floating-point linear: e4m3 codes with one scale for every block of 128 along the
// reduction, per token on the activations' side and per 128 channels on the weights'.
#pragma once

#include "qc_internal.h"

namespace qc {

// ---- data layout of the operands in HBM ---------------------------------------------------
//
// As with the integer operands (qc_internal.h), what a wavefront hands to one matrix instruction is stored lane
// after lane.  v_mfma_f32_16x16x128_f8f6f4 takes 32 bytes a lane: row l % 16 and a quarter of the 128 k.  Which k a
// lane's bytes are is free as long as both operands agree, so the 2 KiB are two halves of 1 KiB that each hold 16
// consecutive k a lane - half hf, lane l: k = 64 hf + 16 (l / 16) .. + 15 - and every copy is a linear one of 16 B/lane.
// With KB = K / 128 rounded up:
//
//   activations, token m:  half ((m / 64) * KB + b) * 8 + (m % 64) / 16 * 2 + hf, row m % 16
//   weights, channel n = 128 G + 8 c + t:  half ((G * KB + b) * 8 + t) * 2 + hf, row c
//       (16 KiB for the 128 x 128 of one scale; a lane ends up with 8 consecutive channels of a token)
//
// The last block's padding holds zeros on both sides: of the other bytes some are NaN.

constexpr int kFp8Block = 128;
constexpr int kFp8TileBytes = kTileN * kFp8Block;   // the weights of one scale
constexpr uint32_t kFp8PackedTag = 0x51433846u;     // "QC8F"
constexpr float kE4m3Most = 448.0f;

__host__ __device__ inline int64_t fp8_blocks(int64_t K) { return (K + kFp8Block - 1) / kFp8Block; }

__host__ __device__ inline int64_t fp8_act_offset(int64_t m, int64_t k, int64_t KB) {
    const int64_t half = ((m / kWaveM) * KB + k / kFp8Block) * 8 + (m % kWaveM) / kFragRows * 2 + k % kFp8Block / kFragK;
    return half * kFragBytes + byte_in_frag(m % kFragRows, k);
}

__host__ __device__ inline int64_t fp8_weight_offset(int64_t n, int64_t k, int64_t KB) {
    const int64_t r = n % kTileN, half = (((n / kTileN) * KB + k / kFp8Block) * 8 + r % 8) * 2 + k % kFp8Block / kFragK;
    return half * kFragBytes + byte_in_frag(r / 8, k);
}

// bytes of one expert's codes
__host__ inline int64_t fp8_weight_bytes(int64_t N, int64_t K) { return round_up(N, kTileN) * fp8_blocks(K) * kFp8Block; }

// A tile of the grouped GEMM's tokens: rows [row0, row0 + rows) of X and Y, of one expert; expert < 0: none.  Those that are any
// come first, `live` of them, in every entry.
struct Fp8Tile {
    int32_t row0, rows, expert, live;
};
constexpr int kFp8TokensLeast = 64;   // of the lowest tile a map is made for

// the tiles that M rows in `experts` groups can come to
__host__ inline int64_t fp8_tiles_most(int64_t M, int64_t experts, int tokens) {
    return M / tokens + (experts < M ? experts : M);
}

// What the GEMM copies or loads past the end of a tile's reduction, and does not use: three blocks of 128 k of the weights,
// one of a panel of 64 tokens (and of the scales, behind which the codes lie).
constexpr int kFp8WeightSlack = 3 * kFp8TileBytes, kFp8ActSlack = kWaveM * kFp8Block;

// workspace: [ scales: KB x Mp floats, token fastest ][ tiled codes: Mp x 128 KB ][ slack ][ map of the grouped GEMM's tiles ]
// Rows M .. Mp - 1 are not written, nor read but as part of the slack.
struct Fp8Workspace {
    int64_t Mp, KB;
    size_t codes_offset, map_offset, total_bytes;
};

__host__ inline Fp8Workspace fp8_workspace(int64_t M, int64_t K) {
    Fp8Workspace w;
    w.Mp = round_up(M, kWaveM);
    w.KB = fp8_blocks(K);
    w.codes_offset = (size_t)round_up(w.Mp * w.KB * 4, 256);
    w.map_offset = w.codes_offset + (size_t)w.Mp * (size_t)w.KB * kFp8Block + kFp8ActSlack;
    w.total_bytes = w.map_offset + (size_t)round_up(fp8_tiles_most(M, QC_MAX_EXPERTS, kFp8TokensLeast) * (int64_t)sizeof(Fp8Tile), 256);
    return w;
}

constexpr int kCus = 256;   // of the chip

// ---- launchers ----------------------------------------------------------------------------

// the quantizer's blocks of threads for each 128 columns, in eights
constexpr int kFp8QuantRows = 32;
__host__ inline int64_t fp8_quant_row_blocks(int64_t M) { return round_up((M + kFp8QuantRows - 1) / kFp8QuantRows, 8); }

// Codes row major with scales [M, KB] (qx), or in the GEMM's order with scales [KB, Mp] (qx_tiled).  offsets: of a grouped
// linear, device int32 [experts + 1]: rows of no group are passed over, and the map of its tiles of `tokens` rows is made if
// there is one.
hipError_t launch_fp8_quant(const void *X, qc_dtype xdt, int64_t M, int64_t K, uint8_t *qx, uint8_t *qx_tiled, float *x_scale,
                            const int32_t *offsets, int experts, int tokens, Fp8Tile *map, hipStream_t stream);

hipError_t launch_fp8_pack(const float *W, int64_t experts, int64_t N, int64_t K, uint8_t *blob, float *w_scale, hipStream_t stream);
hipError_t launch_fp8_unpack(const uint8_t *blob, int64_t experts, int64_t N, int64_t K, uint8_t *codes, hipStream_t stream);

struct Fp8GemmArgs {
    uint8_t *x_tiled;
    float *x_scale;
    const uint8_t *w_codes;
    const float *w_scale;
    const float *bias;
    void *Y;
    Fp8Tile *map;           // grouped; null: one weight, tiles in order
    int64_t M, N, Mp, w_expert_bytes;
    int KB, m_tiles, n_tiles, group_m;
};

// The kernel for few tokens (qc_fp8_few.hip): 16 tokens by 16 times 1, 2 or 4 channels, or 32 by 64
struct Fp8FewTile {
    int tokens, frags;   // tokens 0: not for these sizes
};
// how a linear of these sizes, or a grouped one with so many experts, goes out
struct Fp8Plan {
    bool fused;       // quantization and products in one launch, of the few-token kernel
    Fp8FewTile few;
    int tokens;       // of the tiles, whatever the kernel
};
Fp8Plan fp8_plan(int64_t M, int64_t N, int64_t K, qc_dtype xdt, int experts, bool grouped, qc_out ydt, bool may_fuse);
// X null: from the codes and scales that args names
hipError_t launch_fp8_few(const void *X, qc_dtype xdt, int64_t K, const int32_t *offsets, int experts, const Fp8GemmArgs &args,
                          Fp8FewTile tile, qc_epilogue epi, qc_out ydt, hipStream_t stream);

hipError_t launch_fp8_gemm(const Fp8GemmArgs &args, int tokens, qc_epilogue epi, qc_out ydt, hipStream_t stream);

}  // namespace qc
