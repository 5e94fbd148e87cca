// Launchers of the quantised cache and of the positions in front of it (each
// returns the launch status), and the elements of the OCP Microscaling formats.
#pragma once

#include "internal.h"

#include "flowblock_cache.h"

namespace fb {

hipError_t launch_rotary(const void* q_in, void* q_out, const void* k_in, void* k_out,
                         const int32_t* positions, const fb_pack* pack, const fb_attn_shape* sh,
                         const fb_rotary* rotary, hipStream_t stream);
// The write's threads count a block's runs of eight channels in 32 bits and step past the
// last one by the grid's width, of at most kMxWriteTall workgroups a block.
constexpr int kMxThreads = 256, kMxWriteTall = 65535;
constexpr long long kMxWriteRuns = (1LL << 31) - (long long)kMxWriteTall * kMxThreads;
hipError_t launch_mx_write(const void* k_new, const void* v_new, const fb_mx_cache* cache,
                           const int32_t* page_table, const fb_pack* pack,
                           const fb_attn_shape* sh, hipStream_t stream);
// `k_out` or `v_out` may be NULL
hipError_t launch_mx_read(const fb_mx_cache* cache, const int32_t* page_table,
                          const int32_t* spans, int T_cap, void* k_out, void* v_out,
                          const fb_pack* pack, const fb_attn_shape* sh, int cu_count,
                          hipStream_t stream);

struct MxAttnSizes {
    int rows;        // query rows of a unit: 128, or 32 where a request has no more
    int wgs;         // workgroups, a multiple of 8
    size_t off_head, off_rec, off_o, off_lse, total;
};
MxAttnSizes mx_attention_sizes(const fb_pack* pack, const fb_attn_shape* sh, int cu_count);
hipError_t launch_mx_attention(const void* q, const fb_mx_cache* cache, const int32_t* page_table,
                               const fb_pack* pack, const fb_attn_shape* sh, void* out, void* ws,
                               const MxAttnSizes& sz, hipStream_t stream);

inline int log2_of(int x) {   // of a power of two
    int s = 0;
    while ((1 << s) < x) ++s;
    return s;
}

namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// A scale byte as the conversions below take it: they read the exponent alone, and make
// NaN of everything where it is 255.
__device__ inline float mx_scale(uint32_t code) { return __uint_as_float(code << 23); }

// Two elements of a dword of codes, as bf16, which holds them exactly (two or
// four significant bits): pair I of four in E2M1, of two in E4M3.
template <int BITS, int I>
__device__ inline bf16x2 mx_pair(uint32_t codes, float scale) {
    if constexpr (BITS == 4) return __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, I);
    else return __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, I);
}

// All elements of a dword of codes.
template <int BITS>
__device__ inline void mx_dword(uint32_t codes, float scale, bf16x2* v) {
    v[0] = mx_pair<BITS, 0>(codes, scale);
    v[1] = mx_pair<BITS, 1>(codes, scale);
    if constexpr (BITS == 4) {
        v[2] = mx_pair<BITS, 2>(codes, scale);
        v[3] = mx_pair<BITS, 3>(codes, scale);
    }
}

// Scales that the write makes end here; in a group of a higher one (255 is NaN) the codes
// whose magnitudes are mx_infinite's or more pass bf16's largest.
template <int BITS>
constexpr uint32_t kMxHighest = BITS == 4 ? 252 : 246;
// E2M1: 4 2^126 and 2 2^127 are 2^128; E4M3: (1 + m/8) 2^(x-7) 2^(scale-127) with x >= 262 - scale
template <int BITS>
__device__ inline uint32_t mx_infinite(uint32_t scale) {
    return BITS == 4 ? (scale == 253 ? 6 : 4) : (262 - scale) << 3;
}

}  // namespace
}  // namespace fb
