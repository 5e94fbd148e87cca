// The norms around a block, fused with its gate and scaled residual, on the
// packed live rows:  u = rms(y) w_post,  h' = h + a g u,  n = rms(h') w_pre.
//
// residual_norm_kernel  WR waves to a row; a lane holds its share of the row,
//                       at most NC chunks of 16 bytes, in registers, so y and h
//                       are read once and h' never leaves them between its two
//                       uses.  Two sums a row: one over y, one over h'.
#include <type_traits>

#include "internal.h"

namespace fb {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

struct NormArgs {
    const void *y, *h, *gate, *w_post, *w_pre;
    void *h_out, *n_out;
    int D, gate_kind;
    float eps, scale;
};

template <typename T>
struct Chunk {                      // 16 bytes of a row
    static constexpr int N = 16 / sizeof(T);
    // any alignment of the element type: the address unit takes it
    __device__ static inline u32x4 load(const T* p) {
        u32x4 v;
        __builtin_memcpy(&v, p, 16);
        return v;
    }
    __device__ static inline T part(const u32x4& v, int i) {
        if constexpr (sizeof(T) == 2) return (T)(v[i / 2] >> (i % 2 * 16));
        else return __uint_as_float(v[i]);
    }
    __device__ static inline u32x4 load(const T* p, int n) {   // n < N elements
        u32x4 v = u32x4{0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < N - 1; ++i)
            if (i < n) {
                if constexpr (sizeof(T) == 2) v[i / 2] |= (uint32_t)p[i] << (i % 2 * 16);
                else v[i] = __float_as_uint(p[i]);
            }
        return v;
    }
    __device__ static inline void store(T* p, const u32x4& v, int n) {
        if (n >= N) {
            __builtin_memcpy(p, &v, 16);
        } else {
#pragma unroll
            for (int i = 0; i < N - 1; ++i)
                if (i < n) p[i] = part(v, i);
        }
    }
    __device__ static inline void unpack(const u32x4& u, float (&f)[N]) {
        if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                f[2 * j] = __uint_as_float(u[j] << 16);
                f[2 * j + 1] = __uint_as_float(u[j] & 0xffff0000u);
            }
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) f[j] = __uint_as_float(u[j]);
        }
    }
    __device__ static inline u32x4 pack(const float (&f)[N]) {
        u32x4 u;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if constexpr (sizeof(T) == 2) {
                const uint32_t a = __builtin_bit_cast(uint16_t, (__bf16)f[2 * j]);
                const uint32_t b = __builtin_bit_cast(uint16_t, (__bf16)f[2 * j + 1]);
                u[j] = a | b << 16;
            } else {
                u[j] = __float_as_uint(f[j]);
            }
        }
        return u;
    }
};

// Sum over the WR waves of a row, in a fixed order; every lane gets it.
template <int WR>
__device__ inline float row_sum(float v, float* lds) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
    if constexpr (WR > 1) {
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
        __syncthreads();
        v = lds[0];
#pragma unroll
        for (int w = 1; w < WR; ++w) v += lds[w];
    }
    return v;
}

// 1 / sqrt(mean(x^2) + eps) of a row from the lane's sum of squares; all lanes of the row
// get the same.  Where the squares or their sum leave the float range (entries of 1e18
// at D = 1024, say), small_squares() sums them again with the entries taken 2^72 times
// smaller: the largest float squares to 2^112 then, 16384 of them make 2^126, and what
// has to be there for the first sum to overflow is far from underflow.  (Past a root
// mean square of 2^126 the result is subnormal, two bits fewer at most.)
constexpr float kSmall = 0x1p-72f;

template <int WR, typename F>
__device__ inline float inverse_rms(float squares, F&& small_squares, const NormArgs& a,
                                    float (*lds)[WR]) {
    const float q = row_sum<WR>(squares, lds[0]);
    if (q < INFINITY) return 1.f / sqrtf(q / (float)a.D + a.eps);
    const float d = row_sum<WR>(small_squares(), lds[1]);   // infinities and NaN stay
    return kSmall / sqrtf(d / (float)a.D + a.eps * kSmall * kSmall);
}

// RW rows a workgroup, each of WR waves (RW is 1 where WR is more than 1).
// EARLY: before it is known that the row is live it is loaded, and with it (WEIGHTS)
// the weights and the gate, for calls of few rows, whose time is the chain of loads that
// wait for one another.  Rows of more than two chunks a lane leave no registers for the
// weights (96 rows of 16384 in fp32: 9.9 us, 15.1 with 80 registers spilled).
template <typename T, int WR, int RW, int NC, bool EARLY>
__global__ void __launch_bounds__(64 * WR * RW)
residual_norm_kernel(NormArgs a, PackView pv, int row_cap) {
    using V = Chunk<T>;
    constexpr int N = V::N;
    __shared__ float red[4][WR];
    const int row = blockIdx.x * RW + (RW > 1 ? threadIdx.x >> 6 : 0);
    if (RW > 1 && row >= row_cap) return;
    const int req = pv.row_req[row];
    if (!EARLY && req < 0) return;
    const int lane = RW > 1 ? threadIdx.x & 63 : threadIdx.x;
    const size_t at = (size_t)row * a.D;
    const T* h = static_cast<const T*>(a.h) + at;
    const T* y = static_cast<const T*>(a.y);
    if (y) y += at;

    // A row's partial chunk is loaded after all whole ones where its loads are packed
    // and so waited for (bf16): 21216 rows of 4096 130 us, 133 in between; in between
    // in fp32: 4704 rows of 2011 40.1 us, 41.0 last.
    constexpr bool TAIL_LAST = sizeof(T) == 2;
    u32x4 hv[NC], yv[NC];
    int left[NC];      // elements of the lane's chunk that lie in the row
    int pos[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        pos[c] = (c * 64 * WR + lane) * N;
        left[c] = a.D - pos[c];
        hv[c] = yv[c] = u32x4{0, 0, 0, 0};
        if (left[c] >= N) {
            hv[c] = V::load(h + pos[c]);
            if (y) yv[c] = V::load(y + pos[c]);
        } else if (!TAIL_LAST && left[c] > 0) {
            hv[c] = V::load(h + pos[c], left[c]);
            if (y) yv[c] = V::load(y + pos[c], left[c]);
        }
    }
    if constexpr (TAIL_LAST) {
#pragma unroll
        for (int c = 0; c < NC; ++c)
            if (left[c] > 0 && left[c] < N) {
                hv[c] = V::load(h + pos[c], left[c]);
                if (y) yv[c] = V::load(y + pos[c], left[c]);
            }
    }
    auto load = [&](const T* w, int c) {
        if (left[c] >= N) return V::load(w + pos[c]);
        return left[c] > 0 ? V::load(w + pos[c], left[c]) : u32x4{0, 0, 0, 0};
    };
    const T* w_post = static_cast<const T*>(a.w_post);
    const T* w_pre = static_cast<const T*>(a.w_pre);
    const T* g = static_cast<const T*>(a.gate);
    if (a.gate_kind == FB_GATE_REQUEST) g += (size_t)max(req, 0) * a.D;
    if (a.gate_kind == FB_GATE_ROW) g += at;
    constexpr bool WEIGHTS = EARLY && NC <= 2;
    u32x4 early[3][WEIGHTS ? NC : 1];
    if (EARLY && !WEIGHTS) {
        asm volatile("" ::: "memory");   // the loads above stay above
        if (req < 0) return;
    }
    if constexpr (WEIGHTS) {
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            if (w_post) early[0][c] = load(w_post, c);
            if (w_pre) early[2][c] = load(w_pre, c);
        }
        asm volatile("" ::: "memory");   // the loads above stay above
        if (req < 0) return;
#pragma unroll
        for (int c = 0; c < NC; ++c)
            if (g) early[1][c] = load(g, c);
        asm volatile("" ::: "memory");
    }
    auto weight = [&](const T* w, int k, int c, float (&f)[N]) {
        V::unpack(WEIGHTS ? early[k][WEIGHTS ? c : 0] : load(w, c), f);
    };

    float hp[NC][N];
    float s = 0.f;
    if (y) {
        float r = 1.f;
        if (w_post) {
            float q = 0.f;
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                float f[N];
                V::unpack(yv[c], f);
#pragma unroll
                for (int j = 0; j < N; ++j) q = fmaf(f[j], f[j], q);
            }
            r = inverse_rms<WR>(q, [&] {
                float d = 0.f;
#pragma unroll
                for (int c = 0; c < NC; ++c) {
                    float f[N];
                    u32x4 v = yv[c];
                    asm("" : "+v"(v));   // unpacked anew: else it is at the loads, which then wait
                    V::unpack(v, f);
#pragma unroll
                    for (int j = 0; j < N; ++j) d = fmaf(kSmall * f[j], kSmall * f[j], d);
                }
                return d;
            }, a, red);
        }
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            float u[N], f[N];
            V::unpack(yv[c], u);
            if (w_post) {
                weight(w_post, 0, c, f);
#pragma unroll
                for (int j = 0; j < N; ++j) u[j] = u[j] * r * f[j];
            }
            if (a.gate_kind != FB_GATE_NONE) {
                weight(g, 1, c, f);
#pragma unroll
                for (int j = 0; j < N; ++j) u[j] *= f[j];
            }
            V::unpack(hv[c], f);
#pragma unroll
            for (int j = 0; j < N; ++j) {
                hp[c][j] = f[j] + a.scale * u[j];
                s = fmaf(hp[c][j], hp[c][j], s);
            }
            if (left[c] > 0) V::store(static_cast<T*>(a.h_out) + at + pos[c], V::pack(hp[c]), left[c]);
        }
    } else {
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            V::unpack(hv[c], hp[c]);
#pragma unroll
            for (int j = 0; j < N; ++j) s = fmaf(hp[c][j], hp[c][j], s);
        }
    }
    if (!a.n_out) return;
    const float r = inverse_rms<WR>(s, [&] {
        float d = 0.f;
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int j = 0; j < N; ++j) d = fmaf(kSmall * hp[c][j], kSmall * hp[c][j], d);
        return d;
    }, a, red + 2);
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        if (left[c] <= 0) continue;
        float f[N];
        if (w_pre) {
            weight(w_pre, 2, c, f);
#pragma unroll
            for (int j = 0; j < N; ++j) f[j] = hp[c][j] * r * f[j];
        } else {
#pragma unroll
            for (int j = 0; j < N; ++j) f[j] = hp[c][j] * r;
        }
        V::store(static_cast<T*>(a.n_out) + at + pos[c], V::pack(f), left[c]);
    }
}

}  // namespace

hipError_t launch_residual_norm(const void* y, const void* h, const void* gate,
                                const void* w_post, const void* w_pre, void* h_out,
                                void* n_out, const fb_pack* pack, const fb_norm_shape* sh,
                                int cu_count, hipStream_t stream) {
    PackView pv = pack_view(pack);
    NormArgs a{y, h, gate, w_post, w_pre, h_out, n_out, sh->D, sh->gate, sh->eps, sh->res_scale};
    const int cap = pack->row_cap;
    auto go = [&](auto zero, auto wr, auto rw, auto nc, auto early) {
        using T = decltype(zero);
        constexpr int WR = decltype(wr)::value, RW = decltype(rw)::value, NC = decltype(nc)::value;
        hipLaunchKernelGGL((residual_norm_kernel<T, WR, RW, NC, decltype(early)::value>),
                           dim3((cap + RW - 1) / RW), dim3(64 * WR * RW), 0, stream, a, pv, cap);
    };
    // Many rows: two chunks a lane (21216 rows of 4096 in bf16: 131 us = 5.3
    // TB/s, the rate of a large copy; 136 with four chunks, 147 with one).  Few
    // rows, up to two per CU: one chunk a lane and early loads (96 rows of 2048:
    // 3.6 us against 4.5 and, with four chunks, 7.0); over many rows the early
    // loads read dead rows and hold registers (163 us in the first case).
    auto pick = [&](auto zero) {
        using std::integral_constant;
#define FB_GO(wr, rw, nc, early)                                                        \
    go(zero, integral_constant<int, wr>(), integral_constant<int, rw>(),                \
       integral_constant<int, nc>(), integral_constant<bool, early>())
        const int wave_bytes = 64 * 16;
        const int chunks = (int)(((size_t)sh->D * sizeof(zero) + wave_bytes - 1) / wave_bytes);
        if (cap <= 2 * cu_count) {
            if (chunks <= 1) FB_GO(1, 1, 1, true);
            else if (chunks <= 2) FB_GO(2, 1, 1, true);
            else if (chunks <= 4) FB_GO(4, 1, 1, true);
            else if (chunks <= 8) FB_GO(8, 1, 1, true);
            else if (chunks <= 16) FB_GO(16, 1, 1, true);
            else if (chunks <= 32) FB_GO(16, 1, 2, true);
            else FB_GO(16, 1, 4, true);
        } else {
            if (chunks <= 1) FB_GO(1, 4, 1, false);
            else if (chunks <= 2) FB_GO(1, 4, 2, false);
            else if (chunks <= 4) FB_GO(2, 1, 2, false);
            else if (chunks <= 8) FB_GO(4, 1, 2, false);
            else if (chunks <= 16) FB_GO(8, 1, 2, false);
            else if (chunks <= 32) FB_GO(16, 1, 2, false);
            else FB_GO(16, 1, 4, false);
        }
#undef FB_GO
    };
    if (sh->dtype == FB_BF16) pick(uint16_t());
    else pick(float());
    return hipGetLastError();
}

}  // namespace fb
