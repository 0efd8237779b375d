// The 8-bit floating-point GEMM with a scale for every block of 128 along the reduction, plain and grouped by expert:
//
//   Y[m, n] = act( sum_b sx[m, b] sw[n / 128, b] P_b[m, n] + bias[n] ),   P_b = sum over the 128 k of block b of qx qw
//
// One v_mfma_f32_16x16x128_f8f6f4 covers a block, so P_b comes out of the matrix unit with nothing to add it to, and the
// scales are one fma per output and block on the vector unit, half as many issue cycles as the matrix instruction's.
#include <math.h>

#include "qc_fp8_device.h"

// The copies to LDS name m0, which they set, among what they clobber; the compiler, which keeps it for itself, warns of that.
#pragma clang diagnostic ignored "-Winline-asm"

namespace qc {
namespace {

constexpr int kThreads = 256;

template <int EPI>
__device__ inline float activation(float y) {
    if (EPI == QC_EPI_GELU_TANH) return gelu_tanh_f(y);
    if (EPI == QC_EPI_GELU_ERF) return gelu_erf_f(y);
    return y;
}

__device__ inline Where tile_of(const Fp8GemmArgs &a, int v, int tokens) {
    if (a.map) {
        const Fp8Tile t = a.map[v];
        return {t.row0, t.rows, t.expert};
    }
    const int64_t row0 = (int64_t)v * tokens, rows = a.M - row0;
    return {row0, (int)(rows < tokens ? rows : tokens), 0};
}

constexpr int kSlots = 3;   // of the ring of weights in LDS, a block of 128 k each
constexpr int kRingBytes = kSlots * kFp8TileBytes;

// A block of four wavefronts computes 64 MI tokens x 128 channels, a wavefront 16 MI of the tokens.  The weights, which
// all four use, go HBM -> LDS by linear copies through a ring and are read back 16 B a lane; the activations are
// private to a wavefront and go HBM -> registers, a block of 128 k ahead.  Two blocks fit a CU, so that one's epilogue
// and waits lie under the other's matrix instructions.
//
// Loads, copies and LDS reads are asm so that they stay in flight under counted waits; each wait names the registers that it
// makes valid.  Vector memory operations complete in order, which is the scales and biases, W(0) X(0) W(1) W(2), then X(s + 1)
// at the start and W(s + 3) towards the end of step s, where X are the activations with their scales.  The wait for X(s), after X(s + 1)
// has been requested, leaves that and W(s + 2) in flight, so W(s + 1) has landed with it; the barrier before channel
// block 6 or 7 then makes the next step's weights readable and the slot of this one's free, whose last reads are in registers by then.
// The copies of the last steps run past the reduction and are not used.
//
// What bounds it on large problems is power: 8192 x 8192 x 8192 runs at 1.7 of 2.4 GHz with the matrix units 60 % busy, where a
// loop on registers alone, each product scaled and added, holds 1.9 GHz, 94 % and 3760 TFLOP/s.  us for 131072 x 1152 x 4608,
// 65536 x 4608 x 1152, 8192 x 8192 x 8192: products scaled at once 737 341 498, three products later 729 339 485; scales
// through LDS and copies with scalar addresses 702 326 475, with the channel tile's scales loaded ordinarily, a
// memory round trip ahead of the first copy, 788 329 478; these with tiles of 192 tokens, with 256 680 308 452.
template <int MI, int OUT, int EPI>
__global__ __launch_bounds__(kThreads, 2) void fp8_ring_kernel(Fp8GemmArgs a) {
    constexpr bool EXACT = OUT == QC_OUT_F32;
    typedef Operand<EXACT> Op;
    constexpr int TM = 64 * MI;
    extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];
    float *const lds_bs = reinterpret_cast<float *>(lds + kRingBytes);   // 128 biases
    float *const lds_sw = lds_bs + kTileN;                               // the channel tile's scales, one for each step, in whole 256

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int c = lane & 15, h = lane >> 4;
    int v, nt;
    int blocks = gridDim.x, m_tiles = a.m_tiles;
    if (a.map) {   // The tiles that have rows over all XCDs, blocks without one behind them: dealt out together, they left the last XCD the
                   // empty end (us: 65536 x 4608 x 1152, 64 experts 534, now 514; 3001 x 1000 x 1301, 12 experts 24.3 20.7)
        m_tiles = a.map[0].live;
        blocks = m_tiles * a.n_tiles;
        if ((int)blockIdx.x >= blocks) return;
    }
    tile_of_block(blockIdx.x, blocks, m_tiles, a.n_tiles, a.group_m, v, nt);
    const Where at = tile_of(a, v, TM);
    if (at.expert < 0) return;
    const int first = wave * (16 * MI), live = at.rows - first;   // rows of this wavefront that are stored: may be none
    const int KB = a.KB;

    // Where the next copies come from: scalar addresses that step on, and one 32-bit offset a lane, because vector registers
    // are short and every instruction beside the products counts.  They run up to three steps past the end of the
    // reduction, into the next tile's, or what qc_packed_weight_fp8_bytes() and fp8_workspace() add behind the last.
    const uint8_t *wnext = a.w_codes + at.expert * a.w_expert_bytes + (int64_t)nt * KB * kFp8TileBytes + wave * (4 * kFragBytes);
    const int64_t m0 = at.row0;
    const uint8_t *xnext = a.x_tiled + (m0 / kWaveM) * KB * (8 * kFragBytes);
    const float *snext = a.x_scale + m0;
    const uint32_t lane16 = lane * 16;
    // Rows past the last live one of the tile read that one again.  A lane's place relative to the panel of 64 tokens that
    // the tile begins in.
    uint32_t xoff[MI];
#pragma unroll
    for (int i = 0; i < MI; ++i) {
        const int r = (int)(m0 % kWaveM) + min(first + 16 * i + c, at.rows - 1);
        xoff[i] = (uint32_t)((r / kWaveM) * KB * 8 + r % kWaveM / kFragRows * 2) * kFragBytes + h * 256 + r % kFragRows * 16;
    }
    const uint32_t soff = 4 * min(first + lane, at.rows - 1);

    // LDS: the ring, biases, the channel tile's scales, two steps of 64 token scales for each wavefront
    const uint32_t lds_ring = (uint32_t)(uintptr_t)lds, lds_w = lds_ring + wave * (4 * kFragBytes);
    const uint32_t lds_sx = (uint32_t)(uintptr_t)(lds_sw + round_up(KB, kThreads)) + wave * (4 * kWaveM);
    // Copies to LDS: lane l's piece goes to m0 + offset + its size times l; the offset counts on both sides.  (s_nop: m0 has just been written.)
#define QC_COPY_W(slot)                                                                                        \
    do {                                                                                                       \
        asm volatile("s_add_u32 m0, %0, %3\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2\n\tglobal_load_lds_dwordx4 %1, %2 offset:%4\n\t" \
                     "global_load_lds_dwordx4 %1, %2 offset:%5\n\tglobal_load_lds_dwordx4 %1, %2 offset:%6"    \
                     ::"s"(lds_w), "v"(lane16), "s"(wnext), "n"((slot) * kFp8TileBytes), "n"(kFragBytes), "n"(2 * kFragBytes), \
                     "n"(3 * kFragBytes) : "memory", "scc", "m0");                                                 \
        wnext += kFp8TileBytes;                                                                                \
    } while (0)
#define QC_COPY_4(at_lds, imm, off, base) \
    asm volatile("s_add_u32 m0, %0, %3\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(at_lds), "v"(off), "s"(base), "n"(imm) : "memory", "scc", "m0")
    // the channel tile's scales and biases, without a wait of their own: ahead of the first weights
    for (int b = wave * 64; b < KB; b += kThreads)
        QC_COPY_4((uint32_t)(uintptr_t)(lds_sw + b), 0, 4u * min(b + lane, KB - 1), a.w_scale + ((int64_t)at.expert * a.n_tiles + nt) * KB);
    if (wave < 2) {
        const int n = nt * kTileN + wave * 64;
        if (a.bias) QC_COPY_4((uint32_t)(uintptr_t)(lds_bs + wave * 64), 0, 4u * min(lane, max((int)a.N - 1 - n, 0)), a.bias + (at.expert * a.N + min(n, (int)a.N - 1)));
        else lds_bs[wave * 64 + lane] = 0.0f;
    }

    v4i xq[2][MI][2];
#define QC_LOAD(dst, off, base, imm) asm volatile("global_load_dwordx4 %0, %1, %2 offset:%3" : "=v"(dst) : "v"(off), "s"(base), "n"(imm) : "memory")
#define QC_ISSUE_X(SLOT)                                                        \
    do {                                                                        \
        QC_COPY_4(lds_sx, (SLOT) * (16 * kWaveM), soff, snext);                 \
        _Pragma("unroll") for (int i = 0; i < MI; ++i) {                        \
            QC_LOAD(xq[SLOT][i][0], xoff[i], xnext, 0);                         \
            QC_LOAD(xq[SLOT][i][1], xoff[i], xnext, kFragBytes);                \
        }                                                                       \
        xnext += 8 * kFragBytes;                                                \
        snext += a.Mp;                                                          \
    } while (0)
#define QC_WAIT_X(n, SLOT)                                                                                           \
    do {                                                                                                             \
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(n) : "memory");                                                     \
        _Pragma("unroll") for (int i = 0; i < MI; ++i)                                                               \
            asm volatile("" : "+v"(xq[SLOT][i][0]), "+v"(xq[SLOT][i][1]));                                           \
    } while (0)
    constexpr int kXLoads = 2 * MI + 1;

    // weights: wq[t % TB] the channels 8 c + t of the step; read two ahead, across the end of a step one, or, for want of registers, one
    constexpr int TB = MI == 4 ? 2 : 3;
    v4i wq[TB][2];
    const uint32_t lds_lane = lds_ring + lane16, lds_sx_lane = lds_sx + h * 16;
    uint32_t lds_sw_at = (uint32_t)(uintptr_t)lds_sw;
#define QC_READ_W(slot, t)                                                                                      \
    do {                                                                                                        \
        asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(wq[(t) % TB][0]) : "v"(lds_lane), "n"((slot) * kFp8TileBytes + (t) * 2 * kFragBytes));          \
        asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(wq[(t) % TB][1]) : "v"(lds_lane), "n"((slot) * kFp8TileBytes + ((t) * 2 + 1) * kFragBytes));    \
    } while (0)
#define QC_WAIT_W(n, t) asm volatile("s_waitcnt lgkmcnt(%2)" : "+v"(wq[(t) % TB][0]), "+v"(wq[(t) % TB][1]) : "n"(n))

    constexpr int kDeep = EXACT ? 1 : MI == 4 ? 1 : 3;
    f4 acc[MI][8];
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int t = 0; t < 8; ++t) acc[i][t] = f4{0.0f, 0.0f, 0.0f, 0.0f};

    // step S of six, after which ring and registers are where they were
    auto run_step = [&](auto step_tag) {
        constexpr int S = decltype(step_tag)::value, XS = S % 2, slot = S % kSlots, next = (S + 1) % kSlots;
        f4 sc[MI];
        float sw;
        Op x[MI];
        QC_ISSUE_X(1 - XS);
        QC_WAIT_X(4 + kXLoads, XS);
        asm volatile("ds_read_b32 %0, %1 offset:%2" : "=v"(sw) : "v"(lds_sw_at), "n"(4 * S));
#pragma unroll
        for (int i = 0; i < MI; ++i)
            asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(sc[i]) : "v"(lds_sx_lane), "n"(XS * 16 * kWaveM + 64 * i));
#pragma unroll
        for (int i = 0; i < MI; ++i) x[i] = Op(xq[XS][i][0], xq[XS][i][1]);
        // The products' way through the matrix unit lies under the next ones: one is scaled kDeep products later.
        f4 p[kDeep + 1];
#pragma unroll
        for (int n = 0; n < 8 * MI + kDeep; ++n) {
            const int t = n / MI, i = n % MI;
            if (i == 0 && t < 8) {
                if constexpr (TB == 3) {
                    if (t < 6) QC_READ_W(slot, t + 2);
                    if (t == 0) QC_WAIT_W(2 + MI + 1 + 2, 0);
                    else if (t == 6) {   // blocks 6 and 7 are in registers: this wavefront is done with the slot
                        asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(wq[0][0]), "+v"(wq[0][1]), "+v"(wq[1][0]), "+v"(wq[1][1]));
                        __builtin_amdgcn_s_barrier();
                        asm volatile("" ::: "memory");
                        QC_COPY_W(slot);
                    } else if (t == 7) {
                        QC_READ_W(next, 0);
                    } else {
                        QC_WAIT_W(4, t);
                    }
                } else {
                    if (t < 7) QC_READ_W(slot, t + 1);
                    if (t == 0) QC_WAIT_W(MI + 3, 0);
                    else if (t == 7) {
                        QC_WAIT_W(0, 7);
                        __builtin_amdgcn_s_barrier();
                        asm volatile("" ::: "memory");
                        QC_COPY_W(slot);
                        QC_READ_W(next, 0);
                    } else {
                        QC_WAIT_W(2, t);
                    }
                }
            }
            if (t < 8) p[n % (kDeep + 1)] = product(x[i], Op(wq[t % TB][0], wq[t % TB][1]));
            __builtin_amdgcn_sched_barrier(0);
            if (n == kDeep) {
                asm volatile("s_waitcnt lgkmcnt(2)" : "+v"(sw));
#pragma unroll
                for (int j = 0; j < MI; ++j) {
                    asm volatile("" : "+v"(sc[j]));
                    sc[j] *= sw;
                }
            }
            if (n >= kDeep) {
                const int to = (n - kDeep) / MI, io = (n - kDeep) % MI;
#pragma unroll
                for (int q = 0; q < 4; ++q) acc[io][to][q] = fmaf(p[(n - kDeep) % (kDeep + 1)][q], sc[io][q], acc[io][to][q]);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        if constexpr (TB == 3) QC_READ_W(next, 1);
    };

    // (a vector instruction may have written a scalar address just before, and the compiler sees no memory instruction)
    asm volatile("s_nop 4" ::"s"(wnext), "s"(xnext), "s"(snext));
    QC_COPY_W(0);
    QC_ISSUE_X(0);
    QC_COPY_W(1);
    QC_COPY_W(2);
    QC_WAIT_VMCNT(kXLoads + 8);   // W(0) has landed
    __syncthreads();              // and everybody else's, with the scales
    QC_READ_W(0, 0);
    if constexpr (TB == 3) QC_READ_W(0, 1);
#define QC_STEP(S) run_step(std::integral_constant<int, S>{})
    int left = KB;
    for (; left >= 6; left -= 6) {
        QC_STEP(0);
        QC_STEP(1);
        QC_STEP(2);
        QC_STEP(3);
        QC_STEP(4);
        QC_STEP(5);
        lds_sw_at += 24;
    }
    if (left > 0) QC_STEP(0);
    if (left > 1) QC_STEP(1);
    if (left > 2) QC_STEP(2);
    if (left > 3) QC_STEP(3);
    if (left > 4) QC_STEP(4);
#undef QC_STEP
    // drain what is in flight before its registers are used for anything else
    QC_WAIT_X(0, 0);
    QC_WAIT_X(0, 1);
    asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(wq[0][0]), "+v"(wq[0][1]), "+v"(wq[1][0]), "+v"(wq[1][1]));
#undef QC_WAIT_W
#undef QC_READ_W
#undef QC_WAIT_X
#undef QC_ISSUE_X
#undef QC_LOAD
#undef QC_COPY_4
#undef QC_COPY_W

    // ---- epilogue: lane (c, h) holds channels 8 c .. + 7 of tokens 16 i + 4 h + q
    const int64_t n0 = (int64_t)nt * kTileN + 8 * c;
    constexpr int kOutBytes = OUT == QC_OUT_BF16 ? 2 : 4;
    const bool whole = live >= 16 * MI && (int64_t)(nt + 1) * kTileN <= a.N && a.N % (16 / kOutBytes) == 0;
    float bs[8];
#pragma unroll
    for (int t = 0; t < 8; ++t) bs[t] = lds_bs[8 * c + t];
    auto write_tile = [&](auto checked_tag) {
        constexpr bool CHECKED = decltype(checked_tag)::value;
        if (CHECKED && n0 >= a.N) return;
        const int cols = CHECKED ? (int)(a.N - n0 < 8 ? a.N - n0 : 8) : 8;
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                if (CHECKED && 16 * i + 4 * h + q >= live) continue;
                const int64_t y0 = (m0 + first + 16 * i + 4 * h + q) * a.N + n0;
                float y[8];
#pragma unroll
                for (int t = 0; t < 8; ++t) y[t] = activation<EPI>(acc[i][t][q] + bs[t]);
                if constexpr (OUT == QC_OUT_F32) {
                    float *const p = reinterpret_cast<float *>(a.Y) + y0;
                    if (cols >= 4) store_piece<CHECKED, true>(p, f4{y[0], y[1], y[2], y[3]});
                    if (cols == 8) store_piece<CHECKED, true>(p + 4, f4{y[4], y[5], y[6], y[7]});
                    if (CHECKED && cols < 8) {
#pragma unroll
                        for (int t = 0; t < 8; ++t) if (t >= (cols & 4) && t < cols) p[t] = y[t];
                    }
                } else {
                    uint16_t *const p = reinterpret_cast<uint16_t *>(a.Y) + y0;
                    u32x4 pk;
#pragma unroll
                    for (int t = 0; t < 4; ++t) pk[t] = pack_bf16x2(y[2 * t], y[2 * t + 1]);
                    if (cols == 8) store_piece<CHECKED, CHECKED>(p, pk);
                    else {
#pragma unroll
                        for (int t = 0; t < 8; ++t) if (t < cols) p[t] = (uint16_t)(t % 2 ? pk[t / 2] >> 16 : pk[t / 2]);
                    }
                }
            }
    };
    if (whole) write_tile(std::false_type{});
    else write_tile(std::true_type{});
}

template <int MI, int OUT>
hipError_t launch_tiles(const Fp8GemmArgs &a, qc_epilogue epi, hipStream_t stream) {
    const int bytes = kRingBytes + (int)(kTileN + round_up(a.KB, kThreads) + 2 * 4 * kWaveM) * (int)sizeof(float);
    static_assert(kRingBytes + (kTileN + QC_MAX_K / kFp8Block + 2 * 4 * kWaveM) * sizeof(float) <= 64 * 1024, "dynamic LDS beyond the default limit needs an attribute");
    const dim3 grid((unsigned)(a.m_tiles * a.n_tiles)), block(kThreads);
    if (epi == QC_EPI_GELU_TANH) fp8_ring_kernel<MI, OUT, QC_EPI_GELU_TANH><<<grid, block, bytes, stream>>>(a);
    else if (epi == QC_EPI_GELU_ERF) fp8_ring_kernel<MI, OUT, QC_EPI_GELU_ERF><<<grid, block, bytes, stream>>>(a);
    else fp8_ring_kernel<MI, OUT, QC_EPI_NONE><<<grid, block, bytes, stream>>>(a);
    return hipGetLastError();
}

}  // namespace

// What a CU takes for its share of the ring kernel's tiles of 64 h tokens, `per_cu` of them, in microseconds, with `exact` in hundredths of one for
// each step: read off 3000 drawn linears of 1500 to 60000 tokens, half with 2 to 64 experts, at every height; by it a call takes 0.7 % longer than at
// its best one, at 128 tokens always 3.8 %, at 192 7.2 %.  A step costs a tile the less for each token the higher it is; a CU that has one
// tile or two waits out loads, which a lower one has fewer of; and higher tiles leave more of the last round idle.
// (us at 256 / 192 / 128 / 64 tokens: 300 x 4608 x 1152 - 31.3 25.2 20.2, 5000 x 1152 x 4608 - 41.5 39.8 47.0, 65536 x 4608 x 1152 439 450 464,
// 131072 x 1152 x 4608 739 754 784, 32768 x 1152 x 4608 of 16 experts 211 202 214; binary32, 128 / 64, where the products' widening counts: 300 x 4608 x 1152 46.0 34.7, 4099 x 1000 x 1301
// 31.3 28.8, 10000 x 1152 x 4608 132 144.)
static double ring_cost(int h, double per_cu, int64_t KB, bool grouped, bool exact) {
    if (exact) return h == 1 ? (per_cu <= 1 ? 85 : per_cu <= 2 ? 140 : 68 * per_cu) : per_cu <= 1 ? 115 : per_cu <= 2 ? 210 : 120 * per_cu;
    static const struct {
        double step, tile, last, one, two;   // a step, the rest of a tile, what the last round is short of; one or two tiles to a CU
    } kHeight[] = {{0.36, 0.46, 0.10, 0.12, 1.74}, {0.48, 0.81, 0.07, 1.28, 1.39}, {0.60, 1.53, 0.33, 1.02, 1.58}, {0.76, 2.21, 0.62, 1.60, 2.30}};
    const auto &k = kHeight[h - 1];
    const double t = (double)KB * k.step + k.tile;
    if (per_cu <= 1) return k.one * t;   // nothing is lower than one of the lowest tiles
    if (per_cu <= 2) return k.two * t;
    return (!grouped && per_cu <= 4 ? ceil(per_cu) : per_cu + k.last) * t;
}

static int ring_tokens(int64_t M, int64_t N, int64_t K, int experts, bool grouped, bool exact) {
    const int64_t n_tiles = round_up(N, kTileN) / kTileN;
    int best = 0;
    double least = 0;
    for (int h = exact ? 2 : 4; h >= 1; --h) {
        double per_cu;
        if (grouped) {   // half a tile more than its rows fill for each expert that has any
            const double live = (double)(experts < M ? experts : M), each = (double)M / live / (64 * h) + 0.5;
            per_cu = live * (each > 1 ? each : 1) * (double)n_tiles / kCus;
        } else {
            const int64_t tiles = (M + 64 * h - 1) / (64 * h) * n_tiles;
            per_cu = exact && tiles <= 4 * kCus ? (double)((tiles + kCus - 1) / kCus) : (double)tiles / kCus;
        }
        const double cost = ring_cost(h, per_cu, fp8_blocks(K), grouped, exact);
        if (best == 0 || cost < least) { best = h; least = cost; }
    }
    return 64 * best;
}

// The few-token kernel while its tiles are few, read off 17000 drawn calls of 4 to 700 tokens with one weight and with up to 100
// experts, at every tile and both counts of wavefronts: by it a call takes 2.0 % longer than at its best one.
//
// From X in one launch, tiles of 16 tokens by as few channels as give a CU one at most (us at 16, 32 and 64 channels: 1 x 1152 x 6912 6.7 4.6
// 5.0, 1 x 4608 x 1152 7.6 8.0 8.8, 64 x 1152 x 1152 7.3 4.9 5.6).  Every channel tile casts the same tokens again, so a long
// reduction had better be cast once (tiles of 64 channels up to 24 blocks of 128, others up to 36), and so had bf16 rows that begin at
// odd elements, whose loads are split (16 x 3951 x 3456 14.5, from codes 9.6).  Beyond one tile to a CU short reductions
// gain by it up to two (33 x 577 x 9113 7.4, ring 8.1), and a few rows of many experts, whose tiles are mostly of one row and
// whose upper bound is half empty, up to eight (32 x 2048 x 1408, 64 experts 15.7, ring 17.1; 16 x 1152 x 4608, 32 experts 14.5 15.8).
//
// From codes tiles of 32 x 64 while these are one to a CU (300 x 4608 x 1152 13.5, ring of 64 tokens 20.2; binary32 17.0 34.7), with
// a reduction longer than nine blocks two (200 x 4608 x 4608 17.7, ring 18.7; binary32 21.5 31.8).
Fp8Plan fp8_plan(int64_t M, int64_t N, int64_t K, qc_dtype xdt, int experts, bool grouped, qc_out ydt, bool may_fuse) {
    Fp8Plan p{};
    const int64_t KB = fp8_blocks(K), most = 8 * kCus * 8 * kTileN;   // beyond this the tile counts below need not be made
    if (M <= most && N <= most) {
        const bool odd = xdt == QC_BF16 && K % 2, rows_few = grouped && M <= 96;
        auto tiles = [&](int tokens, int frags) {
            const int64_t m = grouped ? fp8_tiles_most(M, experts, tokens) : (M + tokens - 1) / tokens;
            return m * (round_up(N, kTileN) / kTileN) * (8 / frags);   // a tile's channels lie eight apart: any N has all of a group's
        };
        int frags = 0;
        if (may_fuse && KB <= (odd ? 17 : 36)) {
            if (tiles(16, 1) <= kCus) frags = 1;
            else if (tiles(16, 2) <= kCus) frags = 2;
            else if (tiles(16, 4) <= kCus && (rows_few || KB <= 24)) frags = 4;
            else if (tiles(16, 4) <= (rows_few ? 8 : 2) * kCus && KB <= (odd ? 5 : rows_few ? 36 : 9)) frags = 4;
        }
        p.fused = frags != 0;
        if (p.fused) p.few = {16, frags};
        else if (tiles(32, 4) <= (KB <= 9 ? 1 : rows_few ? 4 : 2) * kCus) p.few = {32, 4};
    }
    p.tokens = p.few.tokens ? p.few.tokens : ring_tokens(M, N, K, experts, grouped, ydt == QC_OUT_F32);
    return p;
}

hipError_t launch_fp8_gemm(const Fp8GemmArgs &args, int tokens, qc_epilogue epi, qc_out ydt, hipStream_t stream) {
    if (ydt == QC_OUT_F32) return tokens == 64 ? launch_tiles<1, QC_OUT_F32>(args, epi, stream) : launch_tiles<2, QC_OUT_F32>(args, epi, stream);
    if (tokens == 64) return launch_tiles<1, QC_OUT_BF16>(args, epi, stream);
    if (tokens == 128) return launch_tiles<2, QC_OUT_BF16>(args, epi, stream);
    if (tokens == 256) return launch_tiles<4, QC_OUT_BF16>(args, epi, stream);
    return launch_tiles<3, QC_OUT_BF16>(args, epi, stream);
}

}  // namespace qc
