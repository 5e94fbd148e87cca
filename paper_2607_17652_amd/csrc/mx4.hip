// Linear layers with MXFP4 weights on the packed live rows: y = W x, W's
// element 2^(scale - 127) E2M1(code), one scale per 32 of K.
//
// mx4_kernel  one wave per output column; lanes along K.
#include "internal.h"

namespace fb {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr int kMxThreads = 256;
constexpr int kMxRows = 8;

// Element pair j of a dword of codes, times 2^(scale-127): exact in bf16.
template <int J>
__device__ inline uint32_t weight_pair(uint32_t codes, float scale) {
    const bf16x2 p = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, J);
    return __builtin_bit_cast(uint32_t, p);
}

__device__ inline float lo_f(uint32_t p) { return __uint_as_float(p << 16); }
__device__ inline float hi_f(uint32_t p) { return __uint_as_float(p & 0xffff0000u); }

template <typename T>
__global__ void __launch_bounds__(kMxThreads)
mx4_kernel(const uint16_t* __restrict__ x, const uint8_t* __restrict__ codes,
           const uint8_t* __restrict__ scales, int N, int K, PackView pv, int row_cap,
           T* __restrict__ y) {
    const int n = blockIdx.x * (kMxThreads / 64) + (threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    const int row0 = blockIdx.y * kMxRows;
    if (n >= N) return;
    bool live[kMxRows];
    bool any = false;
#pragma unroll
    for (int i = 0; i < kMxRows; ++i) {
        live[i] = row0 + i < row_cap && pv.row_req[row0 + i] >= 0;
        any |= live[i];
    }
    if (!any) return;
    float acc[kMxRows] = {};
    for (int g = lane; g < K / 32; g += 64) {
        const uint4 c = *reinterpret_cast<const uint4*>(codes + (size_t)n * (K / 2) + g * 16);
        const uint32_t e = scales[(size_t)n * (K / 32) + g];
        const float s = e == 255 ? __uint_as_float(0x7fc00000u) : 1.f;
        const float f = __uint_as_float(e << 23);
        const uint32_t w[4] = {c.x, c.y, c.z, c.w};
        uint32_t p[16];
#pragma unroll
        for (int d = 0; d < 4; ++d) {
            p[4 * d] = weight_pair<0>(w[d], f);
            p[4 * d + 1] = weight_pair<1>(w[d], f);
            p[4 * d + 2] = weight_pair<2>(w[d], f);
            p[4 * d + 3] = weight_pair<3>(w[d], f);
        }
#pragma unroll
        for (int i = 0; i < kMxRows; ++i) {
            if (!live[i]) continue;
            const uint4* xr = reinterpret_cast<const uint4*>(x + (size_t)(row0 + i) * K + g * 32);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const uint4 xv = xr[q];
                const uint32_t xs[4] = {xv.x, xv.y, xv.z, xv.w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    acc[i] = fmaf(lo_f(xs[j]), s * lo_f(p[4 * q + j]), acc[i]);
                    acc[i] = fmaf(hi_f(xs[j]), s * hi_f(p[4 * q + j]), acc[i]);
                }
            }
        }
    }
#pragma unroll
    for (int i = 0; i < kMxRows; ++i) {
        float v = acc[i];
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
        if (lane == 0 && live[i]) {
            T* out = y + (size_t)(row0 + i) * N + n;
            if constexpr (sizeof(T) == 2) {
                const __bf16 r = (__bf16)v;
                *out = __builtin_bit_cast(uint16_t, r);
            } else {
                *out = v;
            }
        }
    }
}

}  // namespace

hipError_t launch_mx4_linear(const void* x, const void* codes, const void* scales, int N, int K,
                             const fb_pack* pack, void* y, int y_dtype, hipStream_t stream) {
    PackView pv = pack_view(pack);
    const dim3 grid((N + 3) / 4, (pack->row_cap + kMxRows - 1) / kMxRows);
    auto go = [&](auto zero) {
        using T = decltype(zero);
        hipLaunchKernelGGL(mx4_kernel<T>, grid, dim3(kMxThreads), 0, stream,
                           static_cast<const uint16_t*>(x), static_cast<const uint8_t*>(codes),
                           static_cast<const uint8_t*>(scales), N, K, pv, pack->row_cap,
                           static_cast<T*>(y));
    };
    if (y_dtype == FB_BF16) go(uint16_t());
    else go(float());
    return hipGetLastError();
}

}  // namespace fb
