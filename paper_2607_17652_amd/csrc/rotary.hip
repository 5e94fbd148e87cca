// Rotary positions along several axes: pair j of a head vector, (a, b), becomes
// (a cos - b sin, b cos + a sin) at the angle positions[axis_j][row] freq_j.
//
// rotary_kernel  a workgroup takes R packed rows: their sines and cosines go
//                into LDS once (angles formed and reduced to [-pi, pi] in
//                float64), then every head of q and k is turned by them in runs of
//                eight pairs (halves) or four (neighbours).  Bound by memory: 20416
//                rows of 32 + 8 heads of 128 in bf16, 421 MB in 81 us from memory,
//                5.2 TB/s, a large copy's rate; 71.5 on the same rows again, where
//                it took 112 with plain stores and 87 with one run at a time.  Four
//                rows to a workgroup: two 124, eight 118 (plain stores, of 112).
#include "cache.h"

namespace fb {
namespace {

constexpr int kRotThreads = 256;

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4_at2 __attribute__((ext_vector_type(4), aligned(2)));   // anywhere

struct RotArgs {
    const void *q_in, *k_in;
    void *q_out, *k_out;
    const int32_t* positions;
    int Hq, Hkv, D, row_cap, rows;   // rows: of a workgroup
    fb_rotary r;
};

// Eight consecutive elements; p has the alignment of its type only.
__device__ inline void load8(const uint16_t* p, float (&f)[8]) {
    u32x4 w;
    __builtin_memcpy(&w, p, 16);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        f[2 * j] = __uint_as_float(w[j] << 16);
        f[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
    }
}
__device__ inline void load8(const float* p, float (&f)[8]) { __builtin_memcpy(f, p, 32); }
__device__ inline void store8(uint16_t* p, const float (&f)[8]) {
    uint16_t h[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) h[j] = __builtin_bit_cast(uint16_t, (__bf16)f[j]);
    u32x4 w;
    __builtin_memcpy(&w, h, 16);
    __builtin_nontemporal_store(w, reinterpret_cast<u32x4_at2*>(p));
}
__device__ inline void store8(float* p, const float (&f)[8]) {
    u32x4 w[2];
    __builtin_memcpy(w, f, 32);
    __builtin_nontemporal_store(w[0], reinterpret_cast<u32x4_at2*>(p));
    __builtin_nontemporal_store(w[1], reinterpret_cast<u32x4_at2*>(p + 4));
}
__device__ inline float load1(const uint16_t* p) { return __uint_as_float((uint32_t)*p << 16); }
__device__ inline float load1(const float* p) { return *p; }
__device__ inline void store1(uint16_t* p, float f) { *p = __builtin_bit_cast(uint16_t, (__bf16)f); }
__device__ inline void store1(float* p, float f) { *p = f; }

__device__ inline void turn(float& a, float& b, const float2 cs) {
    const float x = a;
    a = fmaf(x, cs.x, -b * cs.y);
    b = fmaf(b, cs.x, x * cs.y);
}

template <typename T, bool HALVES>
__global__ void __launch_bounds__(kRotThreads)
rotary_kernel(RotArgs a, PackView pv) {
    extern __shared__ __attribute__((aligned(16))) float2 rot_table[];   // [rows][n_pairs]
    const int row0 = blockIdx.x * a.rows;
    const int rows = min(a.rows, a.row_cap - row0);
    const int np = a.r.n_pairs;
    for (int e = threadIdx.x; e < rows * np; e += kRotThreads) {
        const int i = e / np, j = e - i * np;
        if (pv.row_req[row0 + i] < 0) continue;
        const int p = a.positions[(size_t)a.r.axis[j] * a.row_cap + row0 + i];
        const double x = (double)p * a.r.freq[j];
        // 2 pi in two parts, so that angles up to 2^31 keep their last bits
        const double k = rint(x * 0.15915494309189535);
        const double r = fma(-k, 2.4492935982947064e-16, fma(-k, 6.283185307179586, x));
        float s, c;
        sincosf((float)r, &s, &c);
        rot_table[e] = make_float2(c, s);
    }
    __syncthreads();
    const int qh = a.q_in ? a.Hq : 0, heads = qh + (a.k_in ? a.Hkv : 0);
    // element 0 of head rh % heads of row rh / heads, and its table
    struct Head {
        const T* in;
        T* out;
        int table;
    };
    auto head_of = [&](int rh) {
        const int i = rh / heads, h = rh - i * heads, row = row0 + i;
        const size_t at = h < qh ? ((size_t)row * a.Hq + h) * a.D
                                 : ((size_t)row * a.Hkv + (h - qh)) * a.D;
        return Head{static_cast<const T*>(h < qh ? a.q_in : a.k_in) + at,
                    static_cast<T*>(h < qh ? a.q_out : a.k_out) + at,
                    pv.row_req[row] < 0 ? -1 : i * np};
    };
    // Runs of eight pairs (halves) or of four (neighbours; the last one's may be fewer), U
    // of them on their way to a thread.
    constexpr int U = sizeof(T) == 2 ? 2 : 1, N = HALVES ? 2 : 1;
    const int runs = HALVES ? np / 8 : (2 * np + 7) / 8, all = rows * heads * runs;
    for (int e0 = threadIdx.x; e0 < all; e0 += U * kRotThreads) {
        Head hd[U];
        int u[U];
        float f[U][N][8];
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const int e = e0 + k * kRotThreads, rh = e / runs;
            if (e >= all) {
                hd[k].table = -1;
                continue;
            }
            hd[k] = head_of(rh);
            u[k] = e - rh * runs;
            if (hd[k].table < 0) continue;
#pragma unroll
            for (int y = 0; y < N; ++y) load8(hd[k].in + u[k] * 8 + y * np, f[k][y]);
        }
#pragma unroll
        for (int k = 0; k < U; ++k) {
            if (hd[k].table < 0) continue;
            const float2* cs = rot_table + hd[k].table;
            if constexpr (HALVES) {
#pragma unroll
                for (int x = 0; x < 8; ++x) turn(f[k][0][x], f[k][1][x], cs[u[k] * 8 + x]);
            } else {
#pragma unroll
                for (int x = 0; x < 4; ++x)
                    if (u[k] * 4 + x < np) turn(f[k][0][2 * x], f[k][0][2 * x + 1], cs[u[k] * 4 + x]);
            }
#pragma unroll
            for (int y = 0; y < N; ++y) store8(hd[k].out + u[k] * 8 + y * np, f[k][y]);
        }
    }
    // What runs of eight leave over: up to seven pairs (halves), and elements that stay.  (Counted
    // without a sign: four rows' elements may pass 2^31, where heads d < 2^30.)
    const uint32_t pairs = HALVES ? np - runs * 8 : 0;
    const uint32_t rest0 = HALVES ? 2 * np : runs * 8, left = pairs + a.D - rest0;
    const uint32_t over = (uint32_t)rows * heads * left;
    for (uint32_t e = threadIdx.x; e < over; e += kRotThreads) {
        const uint32_t rh = e / left, x = e - rh * left;
        const Head hd = head_of((int)rh);
        if (hd.table < 0) continue;
        if (x < pairs) {
            const uint32_t j = runs * 8 + x;
            float p = load1(hd.in + j), q = load1(hd.in + np + j);
            turn(p, q, rot_table[hd.table + j]);
            store1(hd.out + j, p);
            store1(hd.out + np + j, q);
        } else if (hd.in != hd.out) {
            const uint32_t d = rest0 + x - pairs;
            hd.out[d] = hd.in[d];
        }
    }
}

}  // namespace

hipError_t launch_rotary(const void* q_in, void* q_out, const void* k_in, void* k_out,
                         const int32_t* positions, const fb_pack* pack, const fb_attn_shape* sh,
                         const fb_rotary* rotary, hipStream_t stream) {
    RotArgs a{q_in, k_in, q_out, k_out, positions, sh->Hq, sh->Hkv, sh->head_dim, pack->row_cap,
              4, *rotary};
    const size_t smem = (size_t)a.rows * rotary->n_pairs * sizeof(float2);
    const dim3 grid((pack->row_cap + a.rows - 1) / a.rows);
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, grid, dim3(kRotThreads), smem, stream, a, pack_view(pack));
    };
    const bool halves = rotary->pairing == FB_PAIR_HALVES;
    if (sh->dtype == FB_BF16) {
        if (halves) go(rotary_kernel<uint16_t, true>);
        else go(rotary_kernel<uint16_t, false>);
    } else {
        if (halves) go(rotary_kernel<float, true>);
        else go(rotary_kernel<float, false>);
    }
    return hipGetLastError();
}

}  // namespace fb
