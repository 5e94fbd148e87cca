// Keys and values into a quantised paged cache (Eq. 6) and back out of it.
//
// A group of 32 channels x_i has the scale 2^e, e the least integer with
// max|x_i| <= M 2^e (M = 6 in E2M1, 448 in E4M3).  With max|x_i| = m 2^k,
// 1 <= m < 2, and M = m_M 2^(k_M), m_M = 1.5 or 1.75, that is e = k - k_M, one
// more where m > m_M: an addition to the bits of max|x_i| that carries into the
// exponent just there.  Elements are divided by 2^e exactly and rounded to the
// nearest code, ties to even, by the conversion instructions.
//
// mx_write_kernel  a lane takes eight channels of a key and of a value; four
//                  lanes share a group and find its maximum by lane moves.
//                  Bound by memory: 20416 rows of 8 heads of 128 in bf16, 106 MB
//                  in 20.4 us, 5.2 TB/s, a large copy's rate.
// mx_read_kernel   the same eight channels a lane on the way back, four runs at a
//                  time.  Bound by memory, four bytes written to one read in 4
//                  bits: 8 prefixes of 16K .. 32K keys of 8 heads of 128, 980 MB
//                  in 201 us from memory, 4.9 TB/s (231 with whole rows of heads
//                  instead of neighbouring keys to a wave, 240 without the hint on
//                  the stores), 146 where the memory-side cache holds the codes.
#include "cache.h"

namespace fb {
namespace {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x2 __attribute__((ext_vector_type(2)));

struct MxCache {
    uint8_t *kc, *ks, *vc, *vs;
};

MxCache cache_view(const fb_mx_cache* c) {
    return MxCache{static_cast<uint8_t*>(c->k_codes), static_cast<uint8_t*>(c->k_scales),
                   static_cast<uint8_t*>(c->v_codes), static_cast<uint8_t*>(c->v_scales)};
}

template <typename T>
struct Eight {                 // eight elements as loaded
    u32x4 w[sizeof(T) / 2];
    __device__ inline void load(const T* p) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i)
            w[i] = *reinterpret_cast<const u32x4*>(p + i * (16 / sizeof(T)));
    }
    __device__ inline float get(int i) const {
        if constexpr (sizeof(T) == 2)
            return __uint_as_float(i & 1 ? w[0][i / 2] & 0xffff0000u : w[0][i / 2] << 16);
        else return __uint_as_float(w[i / 4][i % 4]);
    }
};

template <int CTRL>
__device__ inline uint32_t quad_move(uint32_t x) {
    return __builtin_amdgcn_update_dpp(0u, x, CTRL, 0xf, 0xf, true);
}

// The codes of a lane's eight elements, and its group's scale byte.
template <typename T, int BITS>
__device__ inline uint32_t quantise8(const Eight<T>& x, uint32_t (&codes)[BITS / 4]) {
    uint32_t top = 0;                           // bits of max |x|, NaN above infinity
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(x.get(i)) & 0x7fffffffu);
    top = max(top, quad_move<0xb1>(top));       // lanes 1 0 3 2
    top = max(top, quad_move<0x4e>(top));       // lanes 2 3 0 1
    constexpr uint32_t kMant = BITS == 4 ? 0x400000u : 0x600000u;   // of 1.5, of 1.75
    constexpr int kExp = BITS == 4 ? 2 : 8;
    constexpr int kLow = BITS == 4 ? 2 : 10, kHigh = BITS == 4 ? 252 : 246;
    int e = (int)((top + (0x7fffffu - kMant)) >> 23) - kExp;
    e = min(max(e, kLow), kHigh);
    const float scale = __uint_as_float((uint32_t)e << 23);
    // E4M3's conversion makes NaN of what is past 464, which is left only where the
    // scale has reached its end; E2M1's ends at 6 by itself
    const float most = 448.0f * scale;
    float f[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        f[i] = x.get(i);
        if constexpr (BITS == 8) f[i] = fminf(fmaxf(f[i], -most), most);
    }
    if constexpr (BITS == 4) {
        uint32_t c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, f[0], f[1], scale, 0);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, f[2], f[3], scale, 1);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, f[4], f[5], scale, 2);
        codes[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, f[6], f[7], scale, 3);
    } else {
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            s16x2 c = {0, 0};
            c = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(c, f[4 * w], f[4 * w + 1], scale, false);
            c = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(c, f[4 * w + 2], f[4 * w + 3], scale, true);
            codes[w] = __builtin_bit_cast(uint32_t, c);
        }
    }
    return top >= 0x7f800000u ? 255u : (uint32_t)e;
}

template <typename T, int BITS>
__global__ void __launch_bounds__(kMxThreads)
mx_write_kernel(const T* __restrict__ k_new, const T* __restrict__ v_new, MxCache cache,
                const int32_t* __restrict__ page_table, PackView pv, int Hkv, int D, int bl,
                int ps_shift, int max_pages, int num_pages) {
    const int t = blockIdx.x;
    if (t >= pv.hdr[kHdrTiles]) return;
    const int32_t* tile = pv.tiles + (size_t)t * kTileInts;
    const int b = tile[kTB], row0 = tile[kTRow0], pos0 = tile[kTPos0];
    const int per_head = D / 8, per_row = Hkv * per_head;
    const int n = bl * per_row;
    const int32_t* pt = page_table + (size_t)b * max_pages;
    for (int e = blockIdx.y * kMxThreads + threadIdx.x; e < n; e += gridDim.y * kMxThreads) {
        // (n is a multiple of four, so the four lanes of a group come together)
        const size_t src = (size_t)row0 * per_row + e;
        Eight<T> k, v;
        k.load(k_new + src * 8);
        v.load(v_new + src * 8);
        const int i = e / per_row, at = e - i * per_row;
        const int c = at / per_head, part = at - c * per_head;
        const int pos = pos0 + i, pidx = pos >> ps_shift;
        const int page = pidx < max_pages ? pt[pidx] : -1;
        uint32_t kq[BITS / 4], vq[BITS / 4];
        const uint32_t ke = quantise8<T, BITS>(k, kq), ve = quantise8<T, BITS>(v, vq);
        if ((unsigned)page >= (unsigned)num_pages) {
            if (at == 0) record_error(pv.hdr, b, FB_DERR_PAGE);
            continue;
        }
        const size_t slot = (((size_t)page * Hkv + c) << ps_shift) + (pos & ((1 << ps_shift) - 1));
        const size_t dst = (slot * per_head + part) * BITS;
        if constexpr (BITS == 4) {
            *reinterpret_cast<uint32_t*>(cache.kc + dst) = kq[0];
            *reinterpret_cast<uint32_t*>(cache.vc + dst) = vq[0];
        } else {
            *reinterpret_cast<u32x2*>(cache.kc + dst) = u32x2{kq[0], kq[1]};
            *reinterpret_cast<u32x2*>(cache.vc + dst) = u32x2{vq[0], vq[1]};
        }
        if (part % 4 == 0) {
            const size_t s = slot * (per_head / 4) + part / 4;
            cache.ks[s] = (uint8_t)ke;
            cache.vs[s] = (uint8_t)ve;
        }
    }
}

// Eight values, past the caches: what is read back is read next by other kernels.
template <int BITS>
__device__ inline void store_values(uint16_t* p, const uint32_t (&codes)[BITS / 4], float scale) {
    union {
        bf16x2 v[4];
        u32x4 w;
    } o;
#pragma unroll
    for (int j = 0; j < BITS / 4; ++j) mx_dword<BITS>(codes[j], scale, o.v + j * (16 / BITS));
    __builtin_nontemporal_store(o.w, reinterpret_cast<u32x4*>(p));
}
template <int BITS>
__device__ inline void store_values(float* p, const uint32_t (&codes)[BITS / 4], float scale) {
    bf16x2 v[4];
#pragma unroll
    for (int j = 0; j < BITS / 4; ++j) mx_dword<BITS>(codes[j], scale, v + j * (16 / BITS));
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const f32x4 f = {(float)v[2 * i][0], (float)v[2 * i][1], (float)v[2 * i + 1][0],
                         (float)v[2 * i + 1][1]};
        __builtin_nontemporal_store(f, reinterpret_cast<f32x4*>(p) + i);
    }
}

template <typename T, int BITS>
__global__ void __launch_bounds__(kMxThreads)
mx_read_kernel(MxCache cache, const int32_t* __restrict__ page_table,
               const int32_t* __restrict__ spans, int T_cap, T* __restrict__ k_out,
               T* __restrict__ v_out, PackView pv, int Hkv, int ph_shift, int ps_shift,
               int max_pages, int num_pages, int wgs) {
    constexpr int U = 4;   // runs of a thread on their way
    const int b = blockIdx.x / wgs, wg = blockIdx.x % wgs;
    const int first = spans[2 * b], n = spans[2 * b + 1];
    if (first < 0 || n < 0 || n > T_cap || (long long)first + n > 0x7fffffffLL ||
        (long long)first + n > ((long long)max_pages << ps_shift)) {
        if (wg == 0 && threadIdx.x == 0) record_error(pv.hdr, b, FB_DERR_SPAN);
        return;
    }
    // Runs of eight channels go head by head of G positions each, so that a wave reads
    // neighbouring keys; a thread's lie wgs kMxThreads apart: dg groups and dat runs.
    constexpr int kG = 2;   // log2 of G
    const int per_row = Hkv << ph_shift, per_group = per_row << kG, ph_mask = (1 << ph_shift) - 1;
    const int stride = wgs * kMxThreads, dg = stride / per_group, dat = stride - dg * per_group;
    const int e0 = wg * kMxThreads + threadIdx.x;
    int grp = e0 / per_group, at = e0 - grp * per_group;
    const int32_t* pt = page_table + (size_t)b * max_pages;
    while (grp << kG < n) {
        int ti[U], ai[U], page[U];   // position, run of its row, page
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int t = (grp << kG) + ((at >> ph_shift) & ((1 << kG) - 1));
            ti[i] = t;
            ai[i] = (at >> (ph_shift + kG) << ph_shift) + (at & ph_mask);
            page[i] = t < n ? pt[(first + t) >> ps_shift] : -1;
            grp += dg, at += dat;
            if (at >= per_group) at -= per_group, ++grp;
        }
        uint32_t kq[U][BITS / 4], vq[U][BITS / 4], ks[U], vs[U];
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const bool good = (unsigned)page[i] < (unsigned)num_pages;
            if (ti[i] < n && !good && ai[i] == 0) record_error(pv.hdr, b, FB_DERR_PAGE);
            if (!good) ti[i] = n;   // nothing is stored
            const int pos = first + ti[i], c = ai[i] >> ph_shift, part = ai[i] & ph_mask;
            const size_t slot = (((size_t)(good ? page[i] : 0) * Hkv + c) << ps_shift) +
                                (pos & ((1 << ps_shift) - 1));
            const size_t src = ((slot << ph_shift) + part) * BITS;
            const size_t s = (slot << (ph_shift - 2)) + part / 4;
#pragma unroll
            for (int j = 0; j < BITS / 4; ++j) {
                if (k_out) kq[i][j] = *reinterpret_cast<const uint32_t*>(cache.kc + src + 4 * j);
                if (v_out) vq[i][j] = *reinterpret_cast<const uint32_t*>(cache.vc + src + 4 * j);
            }
            if (k_out) ks[i] = cache.ks[s];
            if (v_out) vs[i] = cache.vs[s];
        }
#pragma unroll
        for (int i = 0; i < U; ++i) {
            if (ti[i] >= n) continue;
            const size_t dst = (((size_t)b * T_cap + ti[i]) * per_row + ai[i]) * 8;
            if (k_out) store_values<BITS>(k_out + dst, kq[i], mx_scale(ks[i]));
            if (v_out) store_values<BITS>(v_out + dst, vq[i], mx_scale(vs[i]));
        }
    }
}

}  // namespace

hipError_t launch_mx_write(const void* k_new, const void* v_new, const fb_mx_cache* cache,
                           const int32_t* page_table, const fb_pack* pack,
                           const fb_attn_shape* sh, hipStream_t stream) {
    const long long n = (long long)pack->bl * sh->Hkv * (sh->head_dim / 8);
    const long long wgs = (n + kMxThreads - 1) / kMxThreads;
    const dim3 grid(pack->tile_cap, (unsigned)(wgs < kMxWriteTall ? wgs : kMxWriteTall));
    auto go = [&](auto kernel, auto zero) {
        using T = decltype(zero);
        hipLaunchKernelGGL(kernel, grid, dim3(kMxThreads), 0, stream,
                           static_cast<const T*>(k_new), static_cast<const T*>(v_new),
                           cache_view(cache), page_table, pack_view(pack), sh->Hkv, sh->head_dim,
                           pack->bl, log2_of(sh->page_size), sh->max_pages, sh->num_pages);
    };
    const bool four = cache->format == FB_MX4;
    if (sh->dtype == FB_BF16) {
        if (four) go(mx_write_kernel<uint16_t, 4>, uint16_t());
        else go(mx_write_kernel<uint16_t, 8>, uint16_t());
    } else {
        if (four) go(mx_write_kernel<float, 4>, float());
        else go(mx_write_kernel<float, 8>, float());
    }
    return hipGetLastError();
}

hipError_t launch_mx_read(const fb_mx_cache* cache, const int32_t* page_table,
                          const int32_t* spans, int T_cap, void* k_out, void* v_out,
                          const fb_pack* pack, const fb_attn_shape* sh, int cu_count,
                          hipStream_t stream) {
    // eight workgroups a CU over the requests, and no more than the longest span fills
    const long long most =
        ((long long)T_cap * sh->Hkv * (sh->head_dim / 8) + kMxThreads - 1) / kMxThreads;
    long long wgs = (8LL * cu_count + pack->B - 1) / pack->B;
    if (wgs > most) wgs = most;
    auto go = [&](auto kernel, auto zero) {
        using T = decltype(zero);
        hipLaunchKernelGGL(kernel, dim3((unsigned)(pack->B * wgs)), dim3(kMxThreads), 0, stream,
                           cache_view(cache), page_table, spans, T_cap, static_cast<T*>(k_out),
                           static_cast<T*>(v_out), pack_view(pack), sh->Hkv, log2_of(sh->head_dim / 8),
                           log2_of(sh->page_size), sh->max_pages, sh->num_pages, (int)wgs);
    };
    const bool four = cache->format == FB_MX4;
    if (sh->dtype == FB_BF16) {
        if (four) go(mx_read_kernel<uint16_t, 4>, uint16_t());
        else go(mx_read_kernel<uint16_t, 8>, uint16_t());
    } else {
        if (four) go(mx_read_kernel<float, 4>, float());
        else go(mx_read_kernel<float, 8>, float());
    }
    return hipGetLastError();
}

}  // namespace fb
