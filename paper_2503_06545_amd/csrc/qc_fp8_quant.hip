// Quantizers of the 8-bit floating-point linear: e4m3 codes, one scale for every 128 columns of a token (activations,
// online) or every 128 x 128 (weights, offline).
//
//   s = max(max |x|, 2^-64) / 448,   q = e4m3(x / s)      both divisions IEEE binary32, the cast to nearest even
//
// HBM-bound: every element of X is read once and one code written.  A block of 128 columns is what eight lanes hold of a
// row (see Group in qc_device.h), so a block's maximum is three DPP steps away and nothing has to wait for the rest of the
// row.  The quotient is computed as in qc_quant.hip, from one division per block; values whose quotient is too small for
// that to be exact round to a zero code either way.
#include "qc_fp8_device.h"

namespace qc {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kRowsPerWave = 8;   // eight lanes each
static_assert(kWaves * kRowsPerWave == kFp8QuantRows);

// eight lanes' share of columns col0 .. col0 + 127 of a row of K at any alignment, zeros past its end
template <bool NT, typename XT>
__device__ inline void load_block(Group<XT> &g, const XT *xrow, int64_t col0, int64_t K, int sub) {
    constexpr int E = 16 / (int)sizeof(XT), P = sizeof(g.v) / sizeof(g.v[0]);
#pragma unroll
    for (int j = 0; j < P; ++j) g.v[j] = load_piece<NT>(xrow, col0 + 8 * E * j + E * sub, K);
}

struct QuantArgs {
    const void *X;
    uint8_t *qx, *qx_tiled;
    float *x_scale;
    int64_t M, K, Mp;
    int KB;
    const int32_t *offsets;   // grouped only
    Fp8Tile *map;
    int experts, tokens, map_entries, quant_blocks;
};

// ---- the map of a grouped GEMM's tiles ----------------------------------------------------------
// One block beside those that quantize.  A group is [lo_e, hi_e) with lo_e the largest of offsets 0 .. e and hi_e that of 0 .. e + 1, all
// within 0 .. M: the groups of offsets in order, and for any others still disjoint rows inside the buffer, so that their
// tiles never outnumber fp8_tiles_most().
__device__ void make_map(const QuantArgs &a) {
    __shared__ int32_t lo[QC_MAX_EXPERTS + 1], first[QC_MAX_EXPERTS + 1];
    const int E = a.experts, M = (int)a.M;
    if (threadIdx.x < 64) {   // one wavefront scans, each lane a run of experts
        const int lane = threadIdx.x, per = (E + 64) / 64;   // E + 1 offsets
        const int e0 = lane * per, e1 = min(e0 + per, E + 1);
        int most = 0;
        for (int e = e0; e < e1; ++e) most = max(most, min(a.offsets[e], M));
        int before = most;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int v = __shfl_up(before, d);
            if (lane >= d) before = max(before, v);
        }
        before = __shfl_up(before, 1);
        if (lane == 0) before = 0;
        for (int e = e0; e < e1; ++e) lo[e] = before = max(before, min(a.offsets[e], M));
    }
    __syncthreads();
    if (threadIdx.x < 64) {
        const int lane = threadIdx.x, per = (E + 63) / 64;
        const int e0 = lane * per, e1 = min(e0 + per, E);
        int tiles = 0;
        for (int e = e0; e < e1; ++e) tiles += (lo[e + 1] - lo[e] + a.tokens - 1) / a.tokens;
        int upto = tiles;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int v = __shfl_up(upto, d);
            if (lane >= d) upto += v;
        }
        int at = upto - tiles;
        for (int e = e0; e < e1; ++e) {
            first[e] = at;
            at += (lo[e + 1] - lo[e] + a.tokens - 1) / a.tokens;
        }
        if (lane == 63) first[E] = upto;
    }
    __syncthreads();
    const int total = first[E];
    for (int v = threadIdx.x; v < a.map_entries; v += kThreads) {
        Fp8Tile t{0, 0, -1, total};
        if (v < total) {
            int e = 0, end = E;   // the last expert that begins at or before v: the one with rows
            while (end - e > 1) {
                const int mid = (e + end) / 2;
                if (first[mid] <= v) e = mid;
                else end = mid;
            }
            t.expert = e;
            t.row0 = lo[e] + (v - first[e]) * a.tokens;
            t.rows = min(a.tokens, lo[e + 1] - t.row0);
        }
        a.map[v] = t;
    }
}

// A wavefront takes eight rows x one block of 128 columns: the shorter its chain, the shorter a small call, and the more of
// them there are on the large ones (us at one and three blocks: 16 x 4608 2.6 3.7, 300 x 4608 binary32 4.0 6.6, 16384 x 1152 13.6
// 16.1, 131072 x 1152 80 89, 65536 x 4608 161 169).  Block i runs on XCD i % 8, which takes a row's blocks of columns one after
// another, so that lines that two of them share, of X or of the codes, meet in its L2 (200000 x 1000 267, now 144; 65536 x 4608 167
// 155).  NT, NTS: see streams().
template <typename XT, bool NT, bool NTS>
__global__ __launch_bounds__(kThreads) void fp8_quant_kernel(QuantArgs a) {
    if (a.map && (int)blockIdx.x == a.quant_blocks) {
        make_map(a);
        return;
    }
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int sub = lane & 7;
    const uint32_t of_eight = blockIdx.x % (8u * a.KB);
    const int64_t row_block = blockIdx.x / (8u * a.KB) * 8 + of_eight % 8;
    const int b = of_eight / 8;
    const int64_t row = (row_block * kWaves + wave) * kRowsPerWave + lane / 8;
    if (row >= a.M) return;
    if (a.offsets && (row < a.offsets[0] || row >= a.offsets[a.experts])) return;   // of no group

    Group<XT> g;
    load_block<NT>(g, reinterpret_cast<const XT *>(a.X) + row * a.K, (int64_t)b * kFp8Block, a.K, sub);
    auto running = Group<XT>::no_max();
    g.absmax_into(running);
    const float s = scale_of(max_of_eight(Group<XT>::absmax_value(running)), kE4m3Most);
    const float r = 1.0f / s;
    uint32_t w[4];
#pragma unroll
    for (int d = 0; d < 4; ++d)
        w[d] = e4m3x4(quotient(g.get(4 * d + 0), s, r), quotient(g.get(4 * d + 1), s, r), quotient(g.get(4 * d + 2), s, r),
                      quotient(g.get(4 * d + 3), s, r));
    const uint4 out = Group<XT>::gather_codes(w, sub);
    const u32x4 codes = {out.x, out.y, out.z, out.w};
    const int unit = Group<XT>::unit_of(sub);
    if (a.qx_tiled) {
        const int64_t half = ((row / kWaveM) * a.KB + b) * 8 + (row % kWaveM) / kFragRows * 2 + unit / 4;
        store_piece<false, !NTS>(reinterpret_cast<u32x4 *>(a.qx_tiled + half * kFragBytes + (unit % 4) * 256 + (row % kFragRows) * 16), codes);
        if (sub == 0) a.x_scale[(int64_t)b * a.Mp + row] = s;
    } else {
        const int64_t col = (int64_t)b * kFp8Block + unit * kUnit;
        uint8_t *const p = a.qx + row * a.K + col;
        if (col + kUnit <= a.K) {
            store_piece<true, !NTS>(reinterpret_cast<u32x4 *>(p), codes);
        } else {
            for (int e = 0; e < (int)(a.K - col); ++e) p[e] = (uint8_t)(codes[e / 4] >> (8 * (e % 4)));
        }
        if (sub == 0) a.x_scale[row * a.KB + b] = s;
    }
}

// Which accesses of a call go past the caches.  X: it is not read again, and what it would push out of the last-level cache are codes
// that the products are about to read, from some 32 MB of it on (us, ordinary and non-temporal loads, four inputs in turn: 32 MB 13.6 12.7,
// binary32 22.0 20.0, 604 MB 161 157; but 4 MB binary32 3.9 4.2).  Rows that are no whole lines share some, which it would fetch
// twice (100000 x 1000 72 79, 60000 x 4600 169 184).  Codes for the products only where that cache would not keep them either (the whole
// linear with 1152 channels: 346 MB of codes 597 582, 604 MB 935 909; but 230 MB 367 390, 302 MB 458 462).  Codes that stay row by row,
// with X, from 200 MB of both on (16384 x 4608 40.4 39.0, 65536 x 4608 156 146, 131072 x 4608 309 290; X alone at 38 MB 12.3 13.6).
struct Streams {
    bool x, codes;
};
Streams streams(int64_t M, int64_t K, int64_t element, bool tiled) {
    constexpr int64_t MB = 1 << 20;
    if (K * element % 128) return {false, false};
    if (tiled) return {M * K * element >= 32 * MB, M * K >= 320 * MB};
    const bool large = M * K * (element + 1) >= 200 * MB;
    return {large, large && K % 128 == 0};
}

template <typename XT>
void launch_quant(const QuantArgs &a, Streams past, dim3 grid, hipStream_t stream) {
    if (past.codes) fp8_quant_kernel<XT, true, true><<<grid, kThreads, 0, stream>>>(a);
    else if (past.x) fp8_quant_kernel<XT, true, false><<<grid, kThreads, 0, stream>>>(a);
    else fp8_quant_kernel<XT, false, false><<<grid, kThreads, 0, stream>>>(a);
}

// ---- weights ------------------------------------------------------------------------------------
// A block of threads per 128 x 128 of an expert's matrix: every thread half a row.
__global__ __launch_bounds__(kThreads) void fp8_pack_kernel(const float *__restrict__ W, int64_t experts, int64_t N, int64_t K,
                                                            uint8_t *__restrict__ blob, float *__restrict__ w_scale, int64_t NB,
                                                            int64_t KB, int64_t expert_bytes) {
    __shared__ float wave_max[kWaves];
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        reinterpret_cast<uint32_t *>(blob)[0] = kFp8PackedTag;
        int64_t *const h = reinterpret_cast<int64_t *>(blob + 8);
        h[0] = N; h[1] = K; h[2] = experts;
    }
    const int64_t tile = blockIdx.x, b = tile % KB, G = tile / KB % NB, e = tile / KB / NB;
    const int64_t n = G * kTileN + threadIdx.x / 2, k0 = b * kFp8Block + (threadIdx.x & 1) * kFragK;
    const float *const wrow = W + (e * N + (n < N ? n : 0)) * K;
    float v[kFragK];
    float most = 0.0f;
#pragma unroll
    for (int j = 0; j < kFragK; ++j) {
        v[j] = n < N && k0 + j < K ? wrow[k0 + j] : 0.0f;
        most = fmaxf(most, fabsf(v[j]));
    }
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) most = fmaxf(most, __shfl_xor(most, d));
    if ((threadIdx.x & 63) == 0) wave_max[threadIdx.x >> 6] = most;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) most = fmaxf(most, wave_max[w]);
    const float s = scale_of(most, kE4m3Most);
    if (threadIdx.x == 0) w_scale[tile] = s;
    uint8_t *const codes = blob + kPackedHeaderBytes + e * expert_bytes;
#pragma unroll
    for (int u = 0; u < kFragK / 16; ++u) {
        uint32_t w[4];
#pragma unroll
        for (int d = 0; d < 4; ++d)
            w[d] = e4m3x4(v[16 * u + 4 * d] / s, v[16 * u + 4 * d + 1] / s, v[16 * u + 4 * d + 2] / s, v[16 * u + 4 * d + 3] / s);
        *reinterpret_cast<uint4 *>(codes + fp8_weight_offset(n, k0 + 16 * u, KB)) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

__global__ __launch_bounds__(kThreads) void fp8_unpack_kernel(const uint8_t *__restrict__ codes, int64_t N, int64_t K, int64_t KB,
                                                              int64_t expert_bytes, int64_t total, uint8_t *__restrict__ out) {
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < total; i += (int64_t)gridDim.x * kThreads) {
        const int64_t k = i % K, n = i / K % N, e = i / K / N;
        out[i] = codes[e * expert_bytes + fp8_weight_offset(n, k, KB)];
    }
}

}  // namespace

hipError_t launch_fp8_quant(const void *X, qc_dtype xdt, int64_t M, int64_t K, uint8_t *qx, uint8_t *qx_tiled, float *x_scale,
                            const int32_t *offsets, int experts, int tokens, Fp8Tile *map, hipStream_t stream) {
    QuantArgs a{};
    a.X = X;
    a.qx = qx;
    a.qx_tiled = qx_tiled;
    a.x_scale = x_scale;
    a.M = M;
    a.K = K;
    a.Mp = round_up(M, kWaveM);
    a.KB = (int)fp8_blocks(K);
    a.quant_blocks = (int)(fp8_quant_row_blocks(M) * a.KB);
    a.offsets = offsets;
    a.experts = experts;
    if (map) {
        a.map = map;
        a.tokens = tokens;
        a.map_entries = (int)fp8_tiles_most(M, experts, tokens);
    }
    const dim3 grid((unsigned)(a.quant_blocks + (map ? 1 : 0)));
    const Streams past = streams(M, K, xdt == QC_BF16 ? 2 : 4, qx_tiled != nullptr);
    if (xdt == QC_BF16) launch_quant<uint16_t>(a, past, grid, stream);
    else launch_quant<float>(a, past, grid, stream);
    return hipGetLastError();
}

hipError_t launch_fp8_pack(const float *W, int64_t experts, int64_t N, int64_t K, uint8_t *blob, float *w_scale, hipStream_t stream) {
    const int64_t NB = round_up(N, kTileN) / kTileN, KB = fp8_blocks(K);
    fp8_pack_kernel<<<dim3((unsigned)(experts * NB * KB)), dim3(kThreads), 0, stream>>>(W, experts, N, K, blob, w_scale, NB, KB,
                                                                                       fp8_weight_bytes(N, K));
    return hipGetLastError();
}

hipError_t launch_fp8_unpack(const uint8_t *blob, int64_t experts, int64_t N, int64_t K, uint8_t *codes, hipStream_t stream) {
    const int64_t total = experts * N * K, blocks = (total + kThreads - 1) / kThreads;
    fp8_unpack_kernel<<<dim3((unsigned)(blocks < 65536 ? blocks : 65536)), dim3(kThreads), 0, stream>>>(
        blob + kPackedHeaderBytes, N, K, fp8_blocks(K), fp8_weight_bytes(N, K), total, codes);
    return hipGetLastError();
}

}  // namespace qc
