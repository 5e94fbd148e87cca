// Rotary positions along several axes: pair j of a head vector, (a, b), becomes
// (a cos - b sin, b cos + a sin) at the angle positions[axis_j][row] freq_j.
//
// rotary_kernel  a workgroup takes R packed rows: their sines and cosines go
//                into LDS once (angles formed and reduced to [-pi, pi] in
//                float64), then every head of q and k is turned by them, eight
//                pairs (halves) or four (neighbours) a thread.
#include "cache.h"

namespace fb {
namespace {

constexpr int kRotThreads = 256;

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

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
    __builtin_memcpy(p, h, 16);
}
__device__ inline void store8(float* p, const float (&f)[8]) { __builtin_memcpy(p, f, 32); }
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
    // The units of a head: runs of eight pairs (the last one may be shorter), then
    // runs of eight elements that stay.  Neighbours lie four pairs to a run.
    const int turned = HALVES ? (np + 7) / 8 : (2 * np + 7) / 8;
    const int rest0 = HALVES ? 2 * np : turned * 8;      // elements from here on stay
    const int units = turned + (a.D - rest0 + 7) / 8;
    const int heads = (a.q_in ? a.Hq : 0) + (a.k_in ? a.Hkv : 0);
    const int qh = a.q_in ? a.Hq : 0;
    for (int e = threadIdx.x; e < rows * heads * units; e += kRotThreads) {
        const int rh = e / units, u = e - rh * units;
        const int i = rh / heads, h = rh - i * heads;
        const int row = row0 + i;
        if (pv.row_req[row] < 0) continue;
        const bool is_q = h < qh;
        const size_t at = is_q ? ((size_t)row * a.Hq + h) * a.D
                               : ((size_t)row * a.Hkv + (h - qh)) * a.D;
        const T* in = static_cast<const T*>(is_q ? a.q_in : a.k_in) + at;
        T* out = static_cast<T*>(is_q ? a.q_out : a.k_out) + at;
        const float2* cs = rot_table + i * np;
        if (u >= turned) {
            const int d0 = rest0 + (u - turned) * 8;
            if (in == out) continue;
            for (int d = d0; d < min(d0 + 8, a.D); ++d) out[d] = in[d];
        } else if constexpr (HALVES) {
            const int j0 = u * 8;
            if (j0 + 8 <= np) {
                float lo[8], hi[8];
                load8(in + j0, lo);
                load8(in + np + j0, hi);
#pragma unroll
                for (int x = 0; x < 8; ++x) turn(lo[x], hi[x], cs[j0 + x]);
                store8(out + j0, lo);
                store8(out + np + j0, hi);
            } else {
                for (int j = j0; j < np; ++j) {
                    float x = load1(in + j), y = load1(in + np + j);
                    turn(x, y, cs[j]);
                    store1(out + j, x);
                    store1(out + np + j, y);
                }
            }
        } else {
            float f[8];
            load8(in + u * 8, f);
#pragma unroll
            for (int x = 0; x < 4; ++x)
                if (u * 4 + x < np) turn(f[2 * x], f[2 * x + 1], cs[u * 4 + x]);
            store8(out + u * 8, f);
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
