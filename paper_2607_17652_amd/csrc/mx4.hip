// Linear layers with MXFP4 weights on the packed live rows: y = W x, W's
// element 2^(scale - 127) E2M1(code), one scale per 32 of K.
//
// An E2M1 value has two significant bits and the scale is a power of two, so
// v_cvt_scalef32_pk_bf16_fp4 turns two codes and their scale into two bf16
// weights exactly, and the products run on v_mfma_f32_16x16x32_bf16: A holds
// 16 columns of the output (rows of W), B 16 tokens, and a lane's result is
// four neighbouring columns of one token.  A dot product does not care which k
// goes into which slot, so lane group g (of four) of a 128-wide chunk of K
// takes the 32 elements k = 32 g ..: one 16-byte read of codes, one scale.
//
// mx4_kernel  a workgroup of eight waves walks K in chunks through a ring of
//             LDS stages, filled by direct global->LDS loads: x (shared by the
//             waves), and each wave's own codes and scales.  A wave owns NT
//             16-column tiles; where the columns are few, KW waves share a
//             tile, take the chunks of a stage in turn and join at the end.
//             Many rows are bound by the matrix cores: 1024 x 16384 x 4096 100-107
//             us, 1.29-1.37 PFLOP/s; 96 x 157184 x 2048 68-72 us, 0.86-0.91 PFLOP/s;
//             1 x 4096 x 4096 5.1 us.  Large bf16 library products reach 1.13
//             (8192^3) and 1.36 PFLOP/s (20416 x 157184 x 2048) on this card.
// mx4_pair_kernel  more rows and a long output: codes two chunks at a time.
// mx4_still_kernel  few rows and a long output: x stays in registers and the
//             weights of whole rows stream by.
#include <type_traits>

#include "internal.h"

namespace fb {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kWaves = 8;
constexpr int kMxThreads = kWaves * 64;
constexpr int kLdsBytes = 160 * 1024;

// What stands in x past K.
__device__ __attribute__((aligned(16))) uint32_t mx4_zeros[4] = {0, 0, 0, 0};

struct MxArgs {
    const uint16_t* x;
    const uint8_t* codes;
    const uint8_t* scales;
    void* y;
    int N, K, row_cap, bf16_out;
};

// Eight weights (one dword of codes) as the MFMA's A operand; the scale is a
// float whose exponent is the E8M0 code.
__device__ inline bf16x8 weights8(uint32_t codes, float scale) {
    union {
        bf16x2 p[4];
        bf16x8 v;
    } w;
    w.p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0);
    w.p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1);
    w.p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2);
    w.p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3);
    return w.v;
}

// Bit i of the result: row r0 + i is live (i < 64 in m0, then m1).
__device__ inline void live_rows(const PackView& pv, int r0, int row_cap, uint64_t& m0,
                                 uint64_t& m1, int n) {
    const int lane = threadIdx.x & 63;
    const int r = r0 + lane;
    m0 = __ballot(lane < n && r < row_cap && pv.row_req[min(r, row_cap - 1)] >= 0);
    m1 = n > 64 ? __ballot(lane + 64 < n && r + 64 < row_cap &&
                           pv.row_req[min(r + 64, row_cap - 1)] >= 0) : 0;
}

// Four neighbouring results; those past N fall away.  Rows of an N that is no multiple
// of four start anywhere: the address unit takes them (900 x 12001 x 608 34.8 us with a
// store for each result, 25.8 so).
__device__ inline void store4(const MxArgs& a, int row, int n, const f32x4& v) {
    const size_t at = (size_t)row * a.N + n;
    if (a.bf16_out) {
        uint16_t* p = static_cast<uint16_t*>(a.y) + at;
        uint16_t h[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) h[i] = __builtin_bit_cast(uint16_t, (__bf16)v[i]);
        if (n + 4 <= a.N) {
            __builtin_memcpy(p, h, 8);
        } else {
#pragma unroll
            for (int i = 0; i < 3; ++i)
                if (n + i < a.N) p[i] = h[i];
        }
    } else {
        float* p = static_cast<float*>(a.y) + at;
        if (n + 4 <= a.N) {
            __builtin_memcpy(p, &v, 16);
        } else {
#pragma unroll
            for (int i = 0; i < 3; ++i)
                if (n + i < a.N) p[i] = v[i];
        }
    }
}

// Direct global->LDS loads; lane l's 16 bytes land at lds + 16 l (its byte,
// widened, at lds + 4 l).
__device__ inline void dma16(uint32_t lds, uint32_t off, const void* base) {
    asm volatile(FB_SET_M0 "global_load_lds_dwordx4 %1, %2"
                 :: "s"(lds), "v"(off), "s"(base) : "memory");
}
__device__ inline void dma16(uint32_t lds, const void* p) {
    asm volatile(FB_SET_M0 "global_load_lds_dwordx4 %1, off"
                 :: "s"(lds), "v"(p) : "memory");
}
__device__ inline void dma4(uint32_t lds, uint32_t off, const void* base) {
    asm volatile(FB_SET_M0 "global_load_lds_dword %1, %2"
                 :: "s"(lds), "v"(off), "s"(base) : "memory");
}
__device__ inline void dma1(uint32_t lds, uint32_t off, const void* base) {
    asm volatile(FB_SET_M0 "global_load_lds_ubyte %1, %2"
                 :: "s"(lds), "v"(off), "s"(base) : "memory");
}

// A NaN scale makes its column NaN: lanes r, r + 16, .. hold the flags of the
// tile's column r, lane group g the columns 4 g ...
template <int TT, int NT>
__device__ inline void spoil(f32x4 (&acc)[TT][NT], int n, bool nan, int g) {
    uint64_t m = __ballot(nan);
    if (!m) return;
    m |= m >> 32;
    m |= m >> 16;
#pragma unroll
    for (int t = 0; t < TT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (m >> (4 * g + i) & 1) acc[t][n][i] = __uint_as_float(0x7fc00000u);
}

// Where row r of 16 has its 16-byte piece p in LDS: at p ^ turn.  A 16-byte read of a
// wave goes in four steps of sixteen lanes, one of them lanes 0-3, 12-15 and 20-27: two
// lane groups g with eight rows each, whose pieces must not share a bank.  Turned by
// the row itself they did, for 12-17% of the cycles: 1024 x 4096 x 4096 49 us, 43 so.
__device__ inline int turn_x(int r) { return r ^ ((r ^ r >> 1) & 4); }   // rows of 256 bytes
__device__ inline int turn_w(int r) { return r & 4 ? 3 : 0; }            // rows of 64 bytes

// TT 16-token tiles, NT 16-column tiles a wave, KW waves to a tile.
// DW: whole chunks (K a multiple of 128) and scales 4-byte aligned, so that a row's
// four scales of a chunk are one dword; a byte a lane otherwise.
template <int TT, int NT, int KW, bool DW>
struct MxShape {
    static constexpr int kX = KW * TT * 4096;               // x of a stage
    static constexpr int kScaleOps = DW ? (NT + 3) / 4 : NT;
    static constexpr int kW = NT * 1024 + kScaleOps * 256;  // a wave's codes and scales
    static constexpr int kStage = kX + kWaves * kW;
    static constexpr int kFit = kLdsBytes / kStage;
    static constexpr int kStages = kFit > 4 ? 4 : kFit;
    static constexpr int kXOps = KW * TT > 2 ? KW * TT / 2 : 1;   // x loads per wave and stage
    static constexpr int kOps = kXOps + NT + kScaleOps;
    static_assert(kStages >= 2 && (kStages - 2) * kOps < 64 && (KW == 1 || NT == 1));
    static_assert(KW == 1 || kWaves * TT * 1024 <= kStages * kStage);
};

template <int TT, int NT, int KW, bool DW>
__global__ void __launch_bounds__(kMxThreads)
mx4_kernel(MxArgs a, PackView pv, int n_groups) {
    using S = MxShape<TT, NT, KW, DW>;
    __shared__ __attribute__((aligned(16))) unsigned char lds[S::kStages * S::kStage];
    const int ng = blockIdx.x % n_groups;
    const int r0 = blockIdx.x / n_groups * (TT * 16);
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    uint64_t m0, m1;
    live_rows(pv, r0, a.row_cap, m0, m1, TT * 16);
    if (!(m0 | m1)) return;   // uniform over the workgroup

    const int kq = wave % KW;
    const int n0 = (ng * (kWaves / KW) + wave / KW) * (NT * 16);
    const int lr = lane & 15, g = lane >> 4;
    const int C = (a.K + 127) / 128;
    const int steps = (C + KW - 1) / KW;
    const uint32_t lds0 = (uint32_t)(uintptr_t)&lds[0];

    // ---- loads ---------------------------------------------------------------
    // codes: four neighbouring lanes take one row's 64 bytes of a chunk.  x: sixteen
    // lanes take one row's 256 bytes.  Their 16-byte pieces are turned by the row.
    const int wr = lane >> 2, wp = (lane & 3) ^ turn_w(wr);
    const int nb = min(n0, a.N - 1);
    const uint8_t* cbase = a.codes + (size_t)nb * (a.K / 2);
    const uint8_t* sbase = a.scales + (size_t)nb * (a.K / 32);
    const int last = a.N - 1 - nb;
    uint32_t c_off[NT], s_off[S::kScaleOps];
#pragma unroll
    for (int n = 0; n < NT; ++n)
        c_off[n] = (uint32_t)min(n * 16 + wr, last) * (uint32_t)(a.K / 2);
#pragma unroll
    for (int o = 0; o < S::kScaleOps; ++o)
        s_off[o] = (uint32_t)min(DW ? min(o * 64 + lane, NT * 16 - 1) : o * 16 + wr, last) *
                   (uint32_t)(a.K / 32);
    const uint16_t* xbase = a.x + (size_t)r0 * a.K;
    uint32_t x_off[S::kXOps];
    int x_cc[S::kXOps];
#pragma unroll
    for (int i = 0; i < S::kXOps; ++i) {
        const int o = (wave * S::kXOps + i) % (KW * TT * 4);
        const int r = (o % (TT * 4)) * 4 + (lane >> 4);
        x_cc[i] = o / (TT * 4);
        x_off[i] = (uint32_t)min(r, a.row_cap - 1 - r0) * (uint32_t)a.K * 2 +
                   ((lane & 15) ^ turn_x(r & 15)) * 16;
    }
    auto issue = [&](int s, int slot) {
        const uint32_t at = lds0 + slot * S::kStage;
#pragma unroll
        for (int i = 0; i < S::kXOps; ++i) {
            const int o = (wave * S::kXOps + i) % (KW * TT * 4);
            const int c = min(s * KW + x_cc[i], C - 1);
            if (DW || c * 128 + 128 <= a.K) {
                dma16(at + o * 1024, x_off[i], xbase + c * 128);
            } else {
                const int r = (o % (TT * 4)) * 4 + (lane >> 4);
                const int k = c * 128 + ((lane & 15) ^ turn_x(r & 15)) * 8;
                const void* p = k < a.K
                    ? static_cast<const void*>(reinterpret_cast<const char*>(xbase + c * 128) + x_off[i])
                    : static_cast<const void*>(mx4_zeros);
                dma16(at + o * 1024, p);
            }
        }
        const int c = min(s * KW + kq, C - 1);
        // a group past K reads the chunk's first one in its place
        const int piece = DW || (4 * c + wp) * 32 < a.K ? wp : 0;
        const int byte = DW || (4 * c + (lane & 3)) * 32 < a.K ? (lane & 3) : 0;
        const uint32_t mine = at + S::kX + wave * S::kW;
#pragma unroll
        for (int n = 0; n < NT; ++n)
            dma16(mine + n * 1024, c_off[n] + piece * 16, cbase + c * 64);
#pragma unroll
        for (int o = 0; o < S::kScaleOps; ++o) {
            if constexpr (DW) dma4(mine + NT * 1024 + o * 256, s_off[o], sbase + c * 4);
            else dma1(mine + NT * 1024 + o * 256, s_off[o] + byte, sbase + c * 4);
        }
    };

    f32x4 acc[TT][NT];
#pragma unroll
    for (int t = 0; t < TT; ++t)
#pragma unroll
        for (int n = 0; n < NT; ++n) acc[t][n] = f32x4{0.f, 0.f, 0.f, 0.f};
    bool nan[NT] = {};
    const bool idle = n0 >= a.N;

    // One barrier a stage: behind it stage s has landed for every wave, and
    // the slot that stage s - 1 was read from is free.
#pragma unroll
    for (int s = 0; s < S::kStages - 1; ++s)
        if (s < steps) issue(s, s);
    int slot = 0;
    for (int s = 0; s < steps; ++s) {
        if (s + S::kStages - 2 < steps) {
            asm volatile("s_waitcnt vmcnt(%0)" :: "n"((S::kStages - 2) * S::kOps) : "memory");
        } else {
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        }
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if (s + S::kStages - 1 < steps)
            issue(s + S::kStages - 1, slot == 0 ? S::kStages - 1 : slot - 1);
        const int c = s * KW + kq;
        if (c < C && !idle) {
            const unsigned char* xs = lds + slot * S::kStage + kq * (TT * 4096);
            const unsigned char* ws = lds + slot * S::kStage + S::kX + wave * S::kW;
            u32x4 q[NT];
            float sc[NT];
            const bool some = (4 * c + g) * 32 < a.K;
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                q[n] = *reinterpret_cast<const u32x4*>(ws + n * 1024 + lr * 64 + (g ^ turn_w(lr)) * 16);
                uint32_t e;
                if constexpr (DW) {
                    e = *reinterpret_cast<const uint32_t*>(ws + NT * 1024 + (n * 16 + lr) * 4);
                    e = e >> (8 * g) & 255;
                } else {
                    e = *reinterpret_cast<const uint32_t*>(ws + NT * 1024 + n * 256 + lr * 16 + g * 4);
                    e = some ? e & 255 : 0;
                }
                nan[n] |= e == 255;
                sc[n] = __uint_as_float(e << 23);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                bf16x8 w[NT];
#pragma unroll
                for (int n = 0; n < NT; ++n) w[n] = weights8(q[n][j], sc[n]);
#pragma unroll
                for (int t = 0; t < TT; ++t) {
                    const bf16x8 b = *reinterpret_cast<const bf16x8*>(
                        xs + (t * 16 + lr) * 256 + ((g * 4 + j) ^ turn_x(lr)) * 16);
#pragma unroll
                    for (int n = 0; n < NT; ++n)
                        acc[t][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[n], b, acc[t][n], 0, 0, 0);
                }
            }
        }
        slot = slot == S::kStages - 1 ? 0 : slot + 1;
    }

#pragma unroll
    for (int n = 0; n < NT; ++n) spoil(acc, n, nan[n], g);
    if constexpr (KW == 1) {
#pragma unroll
        for (int t = 0; t < TT; ++t) {
            const uint64_t m = t < 4 ? m0 >> (16 * t) : m1 >> (16 * (t - 4));
            if (!(m >> lr & 1)) continue;
#pragma unroll
            for (int n = 0; n < NT; ++n)
                store4(a, r0 + t * 16 + lr, n0 + n * 16 + g * 4, acc[t][n]);
        }
    } else {
        // the KW waves of a tile share its token tiles; partials added in order
        f32x4* part = reinterpret_cast<f32x4*>(lds);
        __syncthreads();
#pragma unroll
        for (int t = 0; t < TT; ++t) part[(wave * TT + t) * 64 + lane] = acc[t][0];
        __syncthreads();
        for (int t = kq; t < TT; t += KW) {
            const f32x4* p = part + (wave - kq) * TT * 64 + t * 64 + lane;
            f32x4 v = p[0];
#pragma unroll
            for (int w = 1; w < KW; ++w) v += p[w * TT * 64];
            const uint64_t m = t < 4 ? m0 >> (16 * t) : m1 >> (16 * (t - 4));
            if (m >> lr & 1) store4(a, r0 + t * 16 + lr, n0 + g * 4, v);
        }
    }
}

// Long outputs: as the ring, but a wave reads its codes two chunks at a time, 128
// bytes of a row in one piece (64 bytes are served at 4 TB/s at most).  They go to
// registers when a pair of chunks begins, and their one slot is filled again while
// the pair is multiplied; x has a slot for each chunk of the pair.  K is a multiple
// of 256 and the scales are 4-byte aligned.
template <int TT, int NT>
struct MxPair {
    static constexpr int kX = TT * 4096;                         // x of a chunk
    static constexpr int kScaleOps = (NT + 1) / 2;
    static constexpr int kW = NT * 2048 + kScaleOps * 256;       // a wave's codes and scales
    static constexpr int kXOps = TT / 2;                         // x loads per wave and chunk
    static constexpr int kWOps = 2 * NT + kScaleOps;
    static constexpr int kLds = 2 * kX + kWaves * kW;
    static_assert(TT % 2 == 0 && TT * NT <= 24 && kLds <= kLdsBytes && kWOps < 64);
};

template <int TT, int NT>
__global__ void __launch_bounds__(kMxThreads)
mx4_pair_kernel(MxArgs a, PackView pv, int n_groups) {
    using S = MxPair<TT, NT>;
    __shared__ __attribute__((aligned(16))) unsigned char lds[S::kLds];
    const int ng = blockIdx.x % n_groups;
    const int r0 = blockIdx.x / n_groups * (TT * 16);
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    uint64_t m0, m1;
    live_rows(pv, r0, a.row_cap, m0, m1, TT * 16);
    if (!(m0 | m1)) return;   // uniform over the workgroup
    const int n0 = (ng * kWaves + wave) * (NT * 16);
    const int lr = lane & 15, g = lane >> 4;
    const int pairs = a.K / 256;
    const uint32_t lds0 = (uint32_t)(uintptr_t)&lds[0];
    const uint32_t w_lds = lds0 + 2 * S::kX + wave * S::kW;

    // ---- loads: eight lanes take one row's 128 bytes of codes, two its scales
    const int nb = min(n0, a.N - 1);
    const uint8_t* cbase = a.codes + (size_t)nb * (a.K / 2);
    const uint8_t* sbase = a.scales + (size_t)nb * (a.K / 32);
    const int last = a.N - 1 - nb;
    const int wr = lane >> 3;                                // of the 8 rows of a load
    const int piece = ((lane & 7) ^ (lane >> 4)) * 16;       // turned by the row's half
    const uint16_t* xbase = a.x + (size_t)r0 * a.K;
    uint32_t x_off[S::kXOps];
#pragma unroll
    for (int i = 0; i < S::kXOps; ++i) {
        const int row = (wave * S::kXOps + i) * 4 + (lane >> 4);
        x_off[i] = (uint32_t)min(row, a.row_cap - 1 - r0) * (uint32_t)a.K * 2 +
                   ((lane & 15) ^ turn_x(row & 15)) * 16;
    }
    auto issue_x = [&](int c) {
#pragma unroll
        for (int i = 0; i < S::kXOps; ++i)
            dma16(lds0 + (c & 1) * S::kX + (wave * S::kXOps + i) * 1024, x_off[i], xbase + c * 128);
    };
    auto issue_w = [&](int p) {
#pragma unroll
        for (int o = 0; o < 2 * NT; ++o)
            dma16(w_lds + o * 1024,
                  (uint32_t)(min(o * 8 + wr, last) * (a.K / 2) + (piece ^ (o & 1) * 64)),
                  cbase + p * 128);
#pragma unroll
        for (int o = 0; o < S::kScaleOps; ++o) {
            const int row = min(min(o * 32 + lane / 2, NT * 16 - 1), last);
            dma4(w_lds + NT * 2048 + o * 256, (uint32_t)(row * (a.K / 32) + (lane & 1) * 4),
                 sbase + p * 8);
        }
    };

    f32x4 acc[TT][NT];
#pragma unroll
    for (int t = 0; t < TT; ++t)
#pragma unroll
        for (int n = 0; n < NT; ++n) acc[t][n] = f32x4{0.f, 0.f, 0.f, 0.f};
    bool nan[NT] = {};
    u32x4 q[NT][2];
    uint32_t e[NT][2];
    auto multiply = [&](int c) {
        const unsigned char* xs = lds + c * S::kX;
        float sc[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const uint32_t b = e[n][c] >> (8 * g) & 255;
            nan[n] |= b == 255;
            sc[n] = __uint_as_float(b << 23);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            bf16x8 w[NT];
#pragma unroll
            for (int n = 0; n < NT; ++n) w[n] = weights8(q[n][c][j], sc[n]);
#pragma unroll
            for (int t = 0; t < TT; ++t) {
                const bf16x8 b = *reinterpret_cast<const bf16x8*>(
                    xs + (t * 16 + lr) * 256 + ((g * 4 + j) ^ turn_x(lr)) * 16);
#pragma unroll
                for (int n = 0; n < NT; ++n)
                    acc[t][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[n], b, acc[t][n], 0, 0, 0);
            }
        }
    };

    // A barrier a chunk: behind it the chunk's x has landed for every wave, and the
    // x of the chunk before may be overwritten.
    issue_x(0);
    issue_w(0);
    for (int p = 0; p < pairs; ++p) {
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        issue_x(2 * p + 1);
        const unsigned char* ws = lds + 2 * S::kX + wave * S::kW;
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                q[n][c] = *reinterpret_cast<const u32x4*>(
                    ws + (n * 16 + lr) * 128 + ((c * 4 + g) ^ (lr >> 1)) * 16);
                e[n][c] = *reinterpret_cast<const uint32_t*>(
                    ws + NT * 2048 + ((n * 16 + lr) * 2 + c) * 4);
            }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (p + 1 < pairs) issue_w(p + 1);
        multiply(0);
        if (p + 1 < pairs) {
            // x of the second chunk is older than the codes of the next pair
            asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" :: "n"(S::kWOps) : "memory");
            issue_x(2 * p + 2);
        } else {
            asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        }
        multiply(1);
    }

#pragma unroll
    for (int n = 0; n < NT; ++n) spoil(acc, n, nan[n], g);
#pragma unroll
    for (int t = 0; t < TT; ++t) {
        const uint64_t m = t < 4 ? m0 >> (16 * t) : m1 >> (16 * (t - 4));
        if (!(m >> lr & 1)) continue;
#pragma unroll
        for (int n = 0; n < NT; ++n)
            store4(a, r0 + t * 16 + lr, n0 + n * 16 + g * 4, acc[t][n]);
    }
}

// x stationary: the eight waves of a workgroup split K, each keeps its share of x
// (TT 16-token tiles, CS chunks) in registers for the whole call, and the
// workgroup walks units of NT 16-column tiles.  It reads a tile's rows whole, 16 KB
// in one piece at K = 2048, where the ring above reads 64 bytes of many rows at a
// time (which the memory serves at 4 TB/s at most): 1 x 157184 x 2048 34.6 us, 4.95
// TB/s, and 43 us by the ring.  The partial sums of a tile join in LDS.
// DW: scales in dwords (K a multiple of 128 and scales 4-byte aligned).
template <int TT, int CS, int NT, bool DW>
struct MxStill {
    static constexpr int kCodeOps = NT * CS;
    static constexpr int kScaleOps = DW ? (kCodeOps + 3) / 4 : kCodeOps;
    static constexpr int kUnit = kCodeOps * 1024 + kScaleOps * 256;   // a wave's codes and scales
    static constexpr int kPart = kWaves * TT * NT * 1024;             // the partial sums, twice
    static constexpr int kFit = (kLdsBytes - 2 * kPart) / (kWaves * kUnit);
    static constexpr int kStages = kFit > 6 ? 6 : kFit;
    static constexpr int kOps = kCodeOps + kScaleOps;
    static_assert(kStages >= 2 && kStages * kOps < 64 && TT <= 2 && NT * TT <= kWaves &&
                  (CS == 2 || CS == 4));
};

template <int TT, int CS, int NT, bool DW>
__global__ void __launch_bounds__(kMxThreads)
mx4_still_kernel(MxArgs a, PackView pv, int n_units, int log_run) {
    using S = MxStill<TT, CS, NT, DW>;
    __shared__ __attribute__((aligned(16))) unsigned char
        lds[2 * S::kPart + S::kStages * kWaves * S::kUnit];
    const int walker = blockIdx.x, n_walkers = gridDim.x;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    uint64_t live, none;
    live_rows(pv, 0, a.row_cap, live, none, TT * 16);
    if (!live) return;   // uniform over the workgroup
    const int lr = lane & 15, g = lane >> 4;
    const int c0 = wave * CS;

    // ---- loads: lane l of op o has 16-byte piece i % (4 CS) of row i / (4 CS),
    // i = 64 o + l, turned by the row so that 16 rows' reads cover all banks
    constexpr int P = 4 * CS;
    auto turn = [](int r) { return CS == 2 ? r >> 1 : r; };
    int crow[S::kCodeOps], coff[S::kCodeOps], srow[S::kScaleOps], soff[S::kScaleOps];
#pragma unroll
    for (int o = 0; o < S::kCodeOps; ++o) {
        const int i = o * 64 + lane;
        const int piece = (i % P) ^ (turn(i / P) % P);
        crow[o] = i / P;
        // a piece past K reads the row's first one in its place
        coff[o] = (c0 * 4 + piece) * 32 < a.K ? (c0 * 4 + piece) * 16 : 0;
    }
#pragma unroll
    for (int o = 0; o < S::kScaleOps; ++o) {
        const int i = o * 64 + lane;
        srow[o] = (DW ? i / CS : i / P) % (NT * 16);
        const int group = DW ? (c0 + i % CS) * 4 : c0 * 4 + i % P;
        soff[o] = group * 32 < a.K ? group : 0;
    }
    const uint32_t lds0 = (uint32_t)(uintptr_t)&lds[2 * S::kPart];
    auto issue = [&](int u, int slot) {
        const int n0 = u * (NT * 16);
        const uint8_t* cbase = a.codes + (size_t)n0 * (a.K / 2);
        const uint8_t* sbase = a.scales + (size_t)n0 * (a.K / 32);
        const uint32_t at = lds0 + (slot * kWaves + wave) * S::kUnit;
        const int last = a.N - 1 - n0;
#pragma unroll
        for (int o = 0; o < S::kCodeOps; ++o)
            dma16(at + o * 1024, (uint32_t)(min(crow[o], last) * (a.K / 2) + coff[o]), cbase);
#pragma unroll
        for (int o = 0; o < S::kScaleOps; ++o) {
            const uint32_t off = (uint32_t)(min(srow[o], last) * (a.K / 32) + soff[o]);
            if constexpr (DW) dma4(at + S::kCodeOps * 1024 + o * 256, off, sbase);
            else dma1(at + S::kCodeOps * 1024 + o * 256, off, sbase);
        }
    };

    // ---- the wave's share of x: lane group g is to hold elements 32 g .. of each
    // chunk, which a lane's own loads would fetch as 64 scattered pieces each.  Load j
    // takes the 64 bytes 32 j .. of a row by its four lanes instead, and the 4 x 4
    // transposition between loads and lane groups is two rounds of lane swaps.
    bf16x8 xf[TT][CS][4];
#pragma unroll
    for (int t = 0; t < TT; ++t) {
        const uint16_t* xr = a.x + (size_t)min(t * 16 + lr, a.row_cap - 1) * a.K;
#pragma unroll
        for (int c = 0; c < CS; ++c) {
            u32x4 v[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int k = (c0 + c) * 128 + j * 32;
                v[j] = u32x4{0, 0, 0, 0};
                if (k < a.K) v[j] = *reinterpret_cast<const u32x4*>(xr + k + g * 8);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const u32x2 p = __builtin_amdgcn_permlane32_swap(v[0][i], v[2][i], false, false);
                const u32x2 q = __builtin_amdgcn_permlane32_swap(v[1][i], v[3][i], false, false);
                const u32x2 l = __builtin_amdgcn_permlane16_swap(p[0], q[0], false, false);
                const u32x2 h = __builtin_amdgcn_permlane16_swap(p[1], q[1], false, false);
                v[0][i] = l[0], v[1][i] = l[1], v[2][i] = h[0], v[3][i] = h[1];
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) xf[t][c][j] = __builtin_bit_cast(bf16x8, v[j]);
        }
    }

    // The compiler has to know that x is there: left to itself it waits for x inside
    // the loop, and so for every load of the ring, at each tile.
    __builtin_amdgcn_s_waitcnt(0x0F70);   // vmcnt(0)
    asm volatile("" ::: "memory");

    // the workgroup's units: runs of 2^log_run neighbours, every n_walkers-th run
    const int runs = (n_units + (1 << log_run) - 1) >> log_run;
    int walk = runs > walker ? ((runs - walker + n_walkers - 1) / n_walkers) << log_run : 0;
    if (walk && (runs - 1) % n_walkers == walker) walk -= (runs << log_run) - n_units;
    auto unit = [&](int s) {
        return ((walker + (s >> log_run) * n_walkers) << log_run) + (s & ((1 << log_run) - 1));
    };
    // codes and scales of a unit, from its slot to registers
    u32x4 q[NT][CS];
    uint32_t e[NT][CS];
    auto fetch = [&](int slot) {
        const unsigned char* in = lds + 2 * S::kPart + (slot * kWaves + wave) * S::kUnit;
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int c = 0; c < CS; ++c) {
                const int r = n * 16 + lr;
                q[n][c] = *reinterpret_cast<const u32x4*>(
                    in + r * (CS * 64) + ((c * 4 + g) ^ (turn(r) % P)) * 16);
                e[n][c] = *reinterpret_cast<const uint32_t*>(
                    in + S::kCodeOps * 1024 + (DW ? r * CS + c : r * P + c * 4 + g) * 4);
            }
    };
#pragma unroll
    for (int s = 0; s < S::kStages; ++s)
        if (s < walk) issue(unit(s), s);
    if (S::kStages <= walk)
        asm volatile("s_waitcnt vmcnt(%0)" :: "n"((S::kStages - 1) * S::kOps) : "memory");
    else
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    if (walk) fetch(0);
    int slot = 0;
    for (int s = 0; s < walk; ++s) {
        const int n0 = unit(s) * (NT * 16);
        // the unit is in registers and its slot free (this wave alone reads it)
        if (s == 0) asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (s + S::kStages < walk) issue(unit(s + S::kStages), slot);
        slot = slot == S::kStages - 1 ? 0 : slot + 1;
        f32x4 acc[TT][NT];
#pragma unroll
        for (int t = 0; t < TT; ++t)
#pragma unroll
            for (int n = 0; n < NT; ++n) acc[t][n] = f32x4{0.f, 0.f, 0.f, 0.f};
        bool nan[NT] = {};
#pragma unroll
        for (int c = 0; c < CS; ++c) {
            float sc[NT];
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                uint32_t ee = DW ? e[n][c] >> (8 * g) : e[n][c];
                ee = ((c0 + c) * 4 + g) * 32 < a.K ? ee & 255 : 0;
                nan[n] |= ee == 255;
                sc[n] = __uint_as_float(ee << 23);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const bf16x8 w = weights8(q[n][c][j], sc[n]);
#pragma unroll
                    for (int t = 0; t < TT; ++t)
                        acc[t][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, xf[t][c][j],
                                                                            acc[t][n], 0, 0, 0);
                }
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) spoil(acc, n, nan[n], g);
        // behind the wait the next unit's codes and scales have landed
        if (s + 1 < walk) {
            if (s + S::kStages < walk)
                asm volatile("s_waitcnt vmcnt(%0)" :: "n"((S::kStages - 1) * S::kOps) : "memory");
            else
                asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            fetch(slot);
        }
        f32x4* part = reinterpret_cast<f32x4*>(lds + (s & 1) * S::kPart);
#pragma unroll
        for (int t = 0; t < TT; ++t)
#pragma unroll
            for (int n = 0; n < NT; ++n) part[((wave * TT + t) * NT + n) * 64 + lane] = acc[t][n];
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        // joined in order; the next partials go to the other half, and the barrier
        // after that lies between this read and the next write here
        if (wave < TT * NT) {
            f32x4 v = part[wave * 64 + lane];
#pragma unroll
            for (int w = 1; w < kWaves; ++w) v += part[(w * TT * NT + wave) * 64 + lane];
            const int t = wave / NT, n = wave % NT;
            if (live >> (t * 16 + lr) & 1) store4(a, t * 16 + lr, n0 + n * 16 + g * 4, v);
        }
    }
}

}  // namespace

hipError_t launch_mx4_linear(const void* x, const void* codes, const void* scales, int N, int K,
                             const fb_pack* pack, void* y, int y_dtype, int cu_count,
                             hipStream_t stream) {
    PackView pv = pack_view(pack);
    const int cap = pack->row_cap;
    MxArgs a{static_cast<const uint16_t*>(x), static_cast<const uint8_t*>(codes),
             static_cast<const uint8_t*>(scales), y, N, K, cap, y_dtype == FB_BF16 ? 1 : 0};
    const int tiles = (N + 15) / 16;
    const bool dw = K % 128 == 0 && ((uintptr_t)scales & 3) == 0;
    auto launch = [&](auto tt, auto nt, auto kw) {
        constexpr int T = decltype(tt)::value, M = decltype(nt)::value, W = decltype(kw)::value;
        const int per = kWaves / W * M;
        const int groups = (tiles + per - 1) / per;
        const int rg = (cap + T * 16 - 1) / (T * 16);
        void (*kernel)(MxArgs, PackView, int) =
            dw ? mx4_kernel<T, M, W, true> : mx4_kernel<T, M, W, false>;
        hipLaunchKernelGGL(kernel, dim3((unsigned)groups * rg), dim3(kMxThreads), 0, stream, a, pv,
                           groups);
    };
    using std::integral_constant;
#define FB_C(n) integral_constant<int, n>()
    const int rows16 = (cap + 15) / 16;
    // x stationary: long outputs (16 tiles a CU), where the time to fetch x is small
    // beside the walk, K from 12 chunks to what the registers hold, 32 rows at most.
    // M x N x K, this form and the ring: 1 x 131072 x 4096 55 and 105 us, 32 x 131072 x
    // 4096 66 and 106; 1 x 65536 x 1536 15.1 and 15.0, 1 x 65536 x 2304 22.3 and 21.9.
    // Outside: 1 x 16384 x 2048 7.3 and 6.3, 1 x 65536 x 1408 14.9 and 14.2, 64 x
    // 157184 x 2048 56 and 58.  Two row tiles, and chunks that keep six or seven of the
    // eight waves at work: 24 tiles a CU (32 x 65536 x 1536 18.7 and 18.0, 32 x 65536 x
    // 2304 27.4 and 23.4, but 32 x 100000 x 1536 25.9 and 26.5, 32 x 157184 x 2304 54 and
    // 55; whole, 32 x 65536 x 1920 21.1 and 22.9, 32 x 65536 x 3200 31.5 and 36.5).
    const int C = (K + 127) / 128;
    const bool idle = C < 15 || (C > 16 && C < 23);
    if (C >= 12 && C <= 32 && rows16 <= 2 &&
        tiles >= (rows16 == 2 && idle ? 24 : 16) * cu_count) {
        auto still = [&](auto t, auto c, auto n) {
            constexpr int T = decltype(t)::value, S = decltype(c)::value, M = decltype(n)::value;
            // runs of four tiles, 128 bytes of a row of bf16 results: written by one
            // workgroup, they leave its L2 as whole lines; unless the runs leave the
            // longest walk a tenth longer
            const int units = (tiles + M - 1) / M, log_run = M == 1 ? 2 : 1;
            const int longest = ((((units - 1) >> log_run) + cu_count) / cu_count) << log_run;
            const bool run = longest * 10 <= (units + cu_count - 1) / cu_count * 11;
            void (*kernel)(MxArgs, PackView, int, int) =
                dw ? mx4_still_kernel<T, S, M, true> : mx4_still_kernel<T, S, M, false>;
            hipLaunchKernelGGL(kernel, dim3((unsigned)cu_count), dim3(kMxThreads), 0, stream, a, pv,
                               units, run ? log_run : 0);
        };
        if (C <= 16) {
            if (rows16 == 1) still(FB_C(1), FB_C(2), FB_C(2));
            else still(FB_C(2), FB_C(2), FB_C(2));
        } else {
            if (rows16 == 1) still(FB_C(1), FB_C(4), FB_C(1));
            else still(FB_C(2), FB_C(4), FB_C(1));
        }
        return hipGetLastError();
    }
    // few columns: split K while the waves of a workgroup a CU are not all busy
    const int TT = rows16 <= 1 ? 1 : rows16 <= 2 ? 2 : rows16 <= 4 ? 4 : rows16 <= 6 ? 6 : 8;
    auto units = [&](int tt) { return (long long)tiles * ((rows16 + tt - 1) / tt); };
    const long long want = 8LL * cu_count;     // one tile per wave
    if (units(TT) <= want / 2) {
        // the cheapest of T token tiles and KW waves to a tile: rounds of workgroups x
        // (a start + stages x a stage's time, us: 0.43 at (1, 2) to 1.3 at (8, 2)).  Over
        // nine shapes within 4% of the fastest of the ten pairs.  32 x 4096 x 4096: (1, 4)
        // 6.4 us, (2, 8) 8.2, (4, 2) 14.8; 64 x 4096 x 4096: (2, 4) 8.1, (1, 2) 9.4, (4, 4)
        // 11.6; 96 x 8192 x 4096: (4, 2) 17.7, (1, 2) 21.8, (2, 2) 22.6.
        int t = 1, kw = 2;
        double best = 1e30;
        for (int T : {1, 2, 4, 6, 8})
            for (int W = 2; W <= kWaves && W * T <= 16; W *= 2) {
                const long long groups =
                    (long long)((tiles * W + 7) / 8) * ((rows16 + T - 1) / T);
                const double cost = (double)((groups + cu_count - 1) / cu_count) *
                                    (2.5 + (C + W - 1) / W * (0.3 + 0.045 * T + 0.04 * T * W));
                if (cost < best) {
                    best = cost;
                    t = T;
                    kw = W;
                }
            }
        auto split = [&](auto tt) {
            if (kw == 2) launch(tt, FB_C(1), FB_C(2));
            else if constexpr (decltype(tt)::value <= 4) {
                if (kw == 4) launch(tt, FB_C(1), FB_C(4));
                else if constexpr (decltype(tt)::value <= 2) launch(tt, FB_C(1), FB_C(8));
            }
        };
        if (t == 1) split(FB_C(1));
        else if (t == 2) split(FB_C(2));
        else if (t == 4) split(FB_C(4));
        else if (t == 6) split(FB_C(6));
        else split(FB_C(8));
        return hipGetLastError();
    }
    // tiles per wave: the least (rounds of workgroups) x (tiles + a start)
    int nt = 1;
    double best = 1e30;
    for (int n = 1; n <= (TT == 8 ? 4 : 5); ++n) {
        const long long groups = (tiles + 8 * n - 1) / (8 * n) * ((rows16 + TT - 1) / TT);
        const double cost = (double)((groups + cu_count - 1) / cu_count) * (n + 0.5);
        if (cost < best) {
            best = cost;
            nt = n;
        }
    }
    // Codes two chunks at a time, while they and the sums fit the registers (beyond, at
    // 96 x 157184 x 2048 and five tiles, 70 us and more; the ring 69).  This form and
    // the ring: 64 x 157184 x 2048 52 and 58 us, 128 x 157184 x 2048 89 and 94, 96 x
    // 65536 x 4096 53 and 63, 128 x 65536 x 4096 65 and 74, 512 x 16384 x 4096 60 and 67,
    // 256 x 16384 x 4096 48 and 48.
    if (dw && K % 256 == 0 && TT >= 4 && nt > 1 && TT * nt <= 24) {
        auto pair = [&](auto tt, auto n) {
            constexpr int T = decltype(tt)::value, M = decltype(n)::value;
            const int groups = (tiles + kWaves * M - 1) / (kWaves * M);
            void (*kernel)(MxArgs, PackView, int) = mx4_pair_kernel<T, M>;
            hipLaunchKernelGGL(kernel, dim3((unsigned)(groups * ((rows16 + T - 1) / T))),
                               dim3(kMxThreads), 0, stream, a, pv, groups);
        };
        auto pick = [&](auto tt) {
            constexpr int T = decltype(tt)::value;
            if (nt == 2) pair(tt, FB_C(2));
            else if (nt == 3) pair(tt, FB_C(3));
            else if constexpr (T <= 6) {
                if (nt == 4) pair(tt, FB_C(4));
                else if constexpr (T <= 4) pair(tt, FB_C(5));
            }
        };
        if (TT == 4) pick(FB_C(4));
        else if (TT == 6) pick(FB_C(6));
        else pick(FB_C(8));
        return hipGetLastError();
    }
    auto pick = [&](auto tt) {
        if (nt == 1) launch(tt, FB_C(1), FB_C(1));
        else if (nt == 2) launch(tt, FB_C(2), FB_C(1));
        else if (nt == 3) launch(tt, FB_C(3), FB_C(1));
        else if (nt == 4) launch(tt, FB_C(4), FB_C(1));
        else if constexpr (decltype(tt)::value < 8) launch(tt, FB_C(5), FB_C(1));
    };
    if (TT == 1) pick(FB_C(1));
    else if (TT == 2) pick(FB_C(2));
    else if (TT == 4) pick(FB_C(4));
    else if (TT == 6) pick(FB_C(6));
    else pick(FB_C(8));
#undef FB_C
    return hipGetLastError();
}

}  // namespace fb
