// The 8-bit floating-point linear on few tokens, or few for each expert: what bounds it is latency - launches, a wavefront's
// chain of loads - and how many CUs pull the weights at once.
//
// A block computes 16 MI tokens x 16 NF channels; its wavefronts deal the blocks of 128 k among themselves, load the
// operands straight into registers and add their scaled sums through LDS in the order of the wavefronts.  Channels are the
// "A" operand here and tokens the "B" operand, so that a lane's results, and the eight or so lanes' worth of activations that
// it quantizes, are one token's: the scale is at hand.  From X (SRC: bf16 or binary32) each wavefront quantizes the k it
// multiplies itself, redundantly over the channel tiles, and the whole linear is one launch; from the workspace (SRC: codes) it
// finds them quantized.
#include "qc_fp8_device.h"

namespace qc {
namespace {

constexpr int kLdsMost = 64 * 1024;

enum Source { kFromF32 = 0, kFromBf16 = 1, kFromCodes = 2 };

// most wavefronts of a block: three to a SIMD where their registers allow it (nine blocks of 128 k are K = 1152), else two or one
template <int SRC, int MI, int NF>
constexpr int kWavesMost = MI * NF <= (SRC == kFromF32 ? 1 : SRC == kFromBf16 ? 2 : 4) ? 12 : 8;

struct FewArgs {
    Fp8GemmArgs g;              // x_tiled and x_scale: from codes only; map: none
    const void *X;
    const int32_t *offsets;     // grouped: the block finds its tile itself
    int64_t K;
    int experts, epi;
};

// Tile v of `tokens` rows of the grouped rows, by every wavefront for itself: 64 experts at a time, the groups as in make_map().
__device__ inline Where find_tile(const int32_t *offsets, int experts, int M, int tokens, int v) {
    const int lane = threadIdx.x & 63;
    int begin = 0, before = 0;   // largest offset and number of tiles so far
    for (int e0 = 0; e0 < experts; e0 += 64) {
        const int e = e0 + lane;
        int lo = e < experts ? min(offsets[e], M) : 0, hi = e < experts ? min(offsets[e + 1], M) : 0;
        if (lane == 0) lo = max(lo, begin);
        lo = max(lo, 0);
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {   // the largest offset up to this one
            const int o = __shfl_up(lo, d);
            if (lane >= d) lo = max(lo, o);
        }
        hi = max(hi, lo);
        const int tiles = e < experts ? (hi - lo + tokens - 1) / tokens : 0;
        int upto = tiles;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int o = __shfl_up(upto, d);
            if (lane >= d) upto += o;
        }
        const int first = before + upto - tiles;
        const uint64_t here = __ballot(v >= first && v < first + tiles);
        if (here) {
            const int l = __builtin_ctzll(here), row0 = __builtin_amdgcn_readlane(lo + (v - first) * tokens, l);
            return {row0, min(tokens, __builtin_amdgcn_readlane(hi, l) - row0), e0 + l};
        }
        before += __builtin_amdgcn_readlane(upto, 63);
        begin = __builtin_amdgcn_readlane(hi, 63);
    }
    return {0, 0, -1};
}

// the largest of lanes l, l ^ 16, l ^ 32, l ^ 48, in each of them
__device__ inline float max_of_quarters(float v) {
    v = fmaxf(v, __shfl_xor(v, 16));
    return fmaxf(v, __shfl_xor(v, 32));
}

// a lane's 32 columns of a block of its token's row, before and after the cast
template <typename XT>
struct Raw {
    static constexpr int E = 16 / (int)sizeof(XT), P = 32 / E;
    uint4 v[P];
    __device__ void load(const XT *xrow, int64_t col0, int64_t K, int h) {
#pragma unroll
        for (int j = 0; j < P; ++j) v[j] = load_piece(xrow, col0 + j / (P / 2) * kFragK + 16 * h + j % (P / 2) * E, K);
    }
    __device__ float get(int i) const {
        const uint4 &u = v[i / E];
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
        if constexpr (sizeof(XT) == 4) return __uint_as_float(w[i % 4]);
        else return i % 2 ? bf16_hi(w[i % 8 / 2]) : bf16_lo(w[i % 8 / 2]);
    }
    __device__ float absmax() const {
        if constexpr (sizeof(XT) == 2) {
            Bf16Max m;
#pragma unroll
            for (int j = 0; j < P; ++j) { m.fold(v[j].x); m.fold(v[j].y); m.fold(v[j].z); m.fold(v[j].w); }
            return m.value();
        } else {
            float m = 0.0f;
#pragma unroll
            for (int i = 0; i < 32; ++i) m = fmaxf(m, fabsf(get(i)));
            return m;
        }
    }
    // the codes, 16 of either half, and their scale
    __device__ float quantize(v4i &lo, v4i &hi) const {
        const float s = scale_of(max_of_quarters(absmax()), kE4m3Most), r = 1.0f / s;
#pragma unroll
        for (int d = 0; d < 8; ++d) {
            const int w = (int)e4m3x4(quotient(get(4 * d), s, r), quotient(get(4 * d + 1), s, r), quotient(get(4 * d + 2), s, r),
                                      quotient(get(4 * d + 3), s, r));
            if (d < 4) lo[d] = w;
            else hi[d - 4] = w;
        }
        return s;
    }
};

// codes and scale from the workspace
struct Stored {
    v4i lo, hi;
    float s;
    __device__ float quantize(v4i &l, v4i &h) const {
        l = lo;
        h = hi;
        return s;
    }
};

template <int NF>
constexpr int kLd = 16 * NF + 4;   // floats of a token's sums in LDS

template <int SRC, int OUT, int MI, int NF>
__global__ __launch_bounds__((64 * kWavesMost<SRC, MI, NF>)) void fp8_few_kernel(FewArgs a) {
    constexpr bool EXACT = OUT == QC_OUT_F32;
    typedef Operand<EXACT> Op;
    typedef std::conditional_t<SRC == kFromF32, float, uint16_t> XT;
    constexpr int TM = 16 * MI;
    extern __shared__ __attribute__((aligned(16))) float sums[];   // [wavefront][16 tokens][channel]

    const Fp8GemmArgs &g = a.g;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    const int c = lane & 15, h = lane >> 4;
    // block b runs on XCD b % 8: the blocks of one XCD take consecutive tiles, token tile fastest, so that they share weights in its L2;
    // grouped they hardly share any, and the tiles without rows, the last ones, come last
    const int nb = gridDim.x, b = blockIdx.x, channel_tiles = g.n_tiles * (8 / NF);
    const int v = (b % 8) * (nb / 8) + min(b % 8, nb % 8) + b / 8;
    const int mt = a.offsets ? b / channel_tiles : v % g.m_tiles, nt = a.offsets ? b % channel_tiles : v / g.m_tiles;
    const int G = nt / (8 / NF), t0 = nt % (8 / NF) * NF;
    if ((int64_t)G * kTileN + t0 >= g.N) return;   // no live channel
    Where at;
    if (a.offsets) {
        at = find_tile(a.offsets, a.experts, (int)g.M, TM, mt);
        if (at.expert < 0) return;
    } else {
        at = {(int64_t)mt * TM, (int)min(g.M - (int64_t)mt * TM, (int64_t)TM), 0};
    }
    const int KB = g.KB;
    const uint8_t *const wsrc = g.w_codes + at.expert * g.w_expert_bytes + (int64_t)G * KB * kFp8TileBytes + t0 * (2 * kFragBytes) + lane * 16;
    const float *const ws = g.w_scale + ((int64_t)at.expert * g.n_tiles + G) * KB;

    struct Piece {
        std::conditional_t<SRC == kFromCodes, Stored, Raw<XT>> x[MI];
        v4i w[NF][2];
        float sw;
    };
    auto load = [&](int kb, Piece &p) {
#pragma unroll
        for (int i = 0; i < MI; ++i) {   // rows past the last live one read that one again
            const int64_t row = at.row0 + min(16 * i + c, at.rows - 1);
            if constexpr (SRC == kFromCodes) {
                const v4i *const x = reinterpret_cast<const v4i *>(g.x_tiled + fp8_act_offset(row, (int64_t)kb * kFp8Block + 16 * h, KB));
                p.x[i].lo = x[0];
                p.x[i].hi = x[64];
                p.x[i].s = g.x_scale[kb * g.Mp + row];
            } else {
                p.x[i].load(reinterpret_cast<const XT *>(a.X) + row * a.K, (int64_t)kb * kFp8Block, a.K, h);
            }
        }
#pragma unroll
        for (int t = 0; t < NF; ++t) {
            const v4i *const w = reinterpret_cast<const v4i *>(wsrc + (int64_t)kb * kFp8TileBytes + t * (2 * kFragBytes));
            p.w[t][0] = w[0];
            p.w[t][1] = w[64];
        }
        p.sw = ws[kb];
    };
    f4 acc[MI][NF];
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int t = 0; t < NF; ++t) acc[i][t] = f4{0.0f, 0.0f, 0.0f, 0.0f};
    auto multiply = [&](const Piece &p) {
        Op x[MI];
        float s[MI];
#pragma unroll
        for (int i = 0; i < MI; ++i) {
            v4i lo, hi;
            s[i] = p.x[i].quantize(lo, hi) * p.sw;
            x[i] = Op(lo, hi);
        }
#pragma unroll
        for (int t = 0; t < NF; ++t) {
            const Op w(p.w[t][0], p.w[t][1]);
#pragma unroll
            for (int i = 0; i < MI; ++i) {
                const f4 r = product(w, x[i]);
#pragma unroll
                for (int q = 0; q < 4; ++q) acc[i][t][q] = fmaf(r[q], s[i], acc[i][t][q]);
            }
        }
    };
    // two pieces in turn, the next one on its way while one is multiplied
    Piece p0, p1;
    int kb = wave;
    if (kb < KB) {
        load(kb, p0);
        for (;;) {
            if (kb + waves < KB) load(kb + waves, p1);
            multiply(p0);
            kb += waves;
            if (kb >= KB) break;
            if (kb + waves < KB) load(kb + waves, p0);
            multiply(p1);
            kb += waves;
            if (kb >= KB) break;
        }
    }

    // Lane (c, h) holds token 16 i + c, channels 8 r + t0 + t with r = 4 h + q.  Sixteen tokens at a time meet in LDS.
    float *const mine = sums + (wave * 16 + c) * kLd<NF> + 4 * h * NF;
#pragma unroll
    for (int i = 0; i < MI; ++i) {
        if (i > 0) {
            if (16 * i >= at.rows) break;
            __syncthreads();   // the sums before have been read
        }
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int t = 0; t < NF; ++t) mine[q * NF + t] = acc[i][t][q];
        __syncthreads();
        for (int o = threadIdx.x; o < 256; o += blockDim.x) {
            const int m = 16 * i + o / 16, r = o % 16;
            const int64_t n0 = (int64_t)G * kTileN + 8 * r + t0;
            if (m >= at.rows || n0 >= g.N) continue;
            float y[NF];
#pragma unroll
            for (int t = 0; t < NF; ++t) y[t] = 0.0f;
            for (int w = 0; w < waves; ++w)
#pragma unroll
                for (int t = 0; t < NF; ++t) y[t] += sums[(w * 16 + o / 16) * kLd<NF> + r * NF + t];
            const int cols = (int)min(g.N - n0, (int64_t)NF);
#pragma unroll
            for (int t = 0; t < NF; ++t) {
                if (g.bias && t < cols) y[t] += g.bias[at.expert * g.N + n0 + t];
                if (a.epi == QC_EPI_GELU_TANH) y[t] = gelu_tanh_f(y[t]);
                else if (a.epi == QC_EPI_GELU_ERF) y[t] = gelu_erf_f(y[t]);
            }
            const int64_t to = (at.row0 + m) * g.N + n0;
            if constexpr (OUT == QC_OUT_F32) {
                float *const p = reinterpret_cast<float *>(g.Y) + to;
                if (cols == NF) __builtin_memcpy(p, y, sizeof(y));
                else
#pragma unroll
                    for (int t = 0; t < NF; ++t) if (t < cols) p[t] = y[t];
            } else {
                uint16_t *const p = reinterpret_cast<uint16_t *>(g.Y) + to;
                uint16_t v16[NF];
#pragma unroll
                for (int t = 0; t < NF; ++t) v16[t] = (uint16_t)pack_bf16x2(y[t], y[t]);
                if (cols == NF) __builtin_memcpy(p, v16, sizeof(v16));
                else
#pragma unroll
                    for (int t = 0; t < NF; ++t) if (t < cols) p[t] = v16[t];
            }
        }
    }
}

template <int SRC, int OUT, int MI, int NF>
hipError_t launch_few_tile(const FewArgs &a, hipStream_t stream) {
    constexpr int kPerWave = 16 * kLd<NF> * (int)sizeof(float), kMost = kLdsMost / kPerWave;
    int waves = a.g.KB < kWavesMost<SRC, MI, NF> ? a.g.KB : kWavesMost<SRC, MI, NF>;
    if (waves > kMost) waves = kMost;
    // Four are as many threads as there are sums to add, and where there are more blocks than CUs two or three such blocks share
    // a CU, whose registers hold one of eight: 16 x 1152 x 4608, eight experts 12.4 us with eight, 10.5 with four; one to a CU 7.2 and 7.9
    const int64_t blocks = (int64_t)a.g.m_tiles * a.g.n_tiles * (8 / NF);   // channel groups whole
    if (waves < 4 || blocks > kCus) waves = 4;
    static_assert(kMost >= 4, "the partial sums of four wavefronts have to fit");
    fp8_few_kernel<SRC, OUT, MI, NF><<<dim3((unsigned)blocks), dim3(64 * waves), waves * kPerWave, stream>>>(a);
    return hipGetLastError();
}

// the tiles that fp8_plan() makes: 32 x 64 from codes, 16 x 16, 32 or 64 from X
template <int SRC, int OUT>
hipError_t launch_few_shape(const FewArgs &a, Fp8FewTile tile, hipStream_t stream) {
    if constexpr (SRC == kFromCodes) {
        return tile.tokens == 32 && tile.frags == 4 ? launch_few_tile<SRC, OUT, 2, 4>(a, stream) : hipErrorInvalidValue;
    } else {
        if (tile.tokens != 16) return hipErrorInvalidValue;
        if (tile.frags == 1) return launch_few_tile<SRC, OUT, 1, 1>(a, stream);
        if (tile.frags == 2) return launch_few_tile<SRC, OUT, 1, 2>(a, stream);
        return launch_few_tile<SRC, OUT, 1, 4>(a, stream);
    }
}

}  // namespace

hipError_t launch_fp8_few(const void *X, qc_dtype xdt, int64_t K, const int32_t *offsets, int experts, const Fp8GemmArgs &args,
                          Fp8FewTile tile, qc_epilogue epi, qc_out ydt, hipStream_t stream) {
    FewArgs a{};
    a.g = args;
    a.X = X;
    a.offsets = offsets;
    a.K = K;
    a.experts = experts;
    a.epi = epi;
    if (!X) return ydt == QC_OUT_F32 ? launch_few_shape<kFromCodes, QC_OUT_F32>(a, tile, stream) : launch_few_shape<kFromCodes, QC_OUT_BF16>(a, tile, stream);
    if (xdt == QC_F32) return ydt == QC_OUT_F32 ? launch_few_shape<kFromF32, QC_OUT_F32>(a, tile, stream) : launch_few_shape<kFromF32, QC_OUT_BF16>(a, tile, stream);
    return ydt == QC_OUT_F32 ? launch_few_shape<kFromBf16, QC_OUT_F32>(a, tile, stream) : launch_few_shape<kFromBf16, QC_OUT_BF16>(a, tile, stream);
}

}  // namespace qc
