// The norms around a block, fused with its gate and scaled residual, on the
// packed live rows:  u = rms(y) w_post,  h' = h + a g u,  n = rms(h') w_pre.
//
// residual_norm_kernel  one workgroup per live row.
#include "internal.h"

namespace fb {
namespace {

constexpr int kNormThreads = 256;

__device__ inline float load1(const uint16_t* p) { return __uint_as_float((uint32_t)*p << 16); }
__device__ inline float load1(const float* p) { return *p; }
__device__ inline void store1(uint16_t* p, float f) {
    const __bf16 v = (__bf16)f;
    *p = __builtin_bit_cast(uint16_t, v);
}
__device__ inline void store1(float* p, float f) { *p = f; }

// Sum over the workgroup, in a fixed order; every thread gets it.
__device__ inline float workgroup_sum(float v, float* lds) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    float s = 0.f;
#pragma unroll
    for (int w = 0; w < kNormThreads / 64; ++w) s += lds[w];
    return s;
}

template <typename T>
__global__ void __launch_bounds__(kNormThreads)
residual_norm_kernel(const T* y, const T* h, const T* gate, const T* w_post, const T* w_pre,
                     T* h_out, T* n_out, PackView pv, int D, int gate_kind, float eps,
                     float scale) {
    extern __shared__ float hs[];   // h' of the row
    __shared__ float red[kNormThreads / 64];
    const int row = blockIdx.x;
    const int req = pv.row_req[row];
    if (req < 0) return;
    const int tid = threadIdx.x;
    const size_t at = (size_t)row * D;
    float r = 1.f;
    if (w_post) {
        float s = 0.f;
        for (int i = tid; i < D; i += kNormThreads) {
            const float v = load1(y + at + i);
            s = fmaf(v, v, s);
        }
        r = 1.f / sqrtf(workgroup_sum(s, red) / (float)D + eps);
    }
    const T* g = gate;
    if (gate_kind == FB_GATE_REQUEST) g += (size_t)req * D;
    if (gate_kind == FB_GATE_ROW) g += at;
    float s = 0.f;
    for (int i = tid; i < D; i += kNormThreads) {
        float v = load1(h + at + i);
        if (y) {
            float u = load1(y + at + i);
            if (w_post) u = u * r * load1(w_post + i);
            if (g) u *= load1(g + i);
            v += scale * u;
        }
        hs[i] = v;
        s = fmaf(v, v, s);
    }
    const float r2 = 1.f / sqrtf(workgroup_sum(s, red) / (float)D + eps);
    for (int i = tid; i < D; i += kNormThreads) {
        const float v = hs[i];
        if (h_out) store1(h_out + at + i, v);
        if (n_out) store1(n_out + at + i, v * r2 * (w_pre ? load1(w_pre + i) : 1.f));
    }
}

}  // namespace

hipError_t launch_residual_norm(const void* y, const void* h, const void* gate,
                                const void* w_post, const void* w_pre, void* h_out,
                                void* n_out, const fb_pack* pack, const fb_norm_shape* sh,
                                hipStream_t stream) {
    PackView pv = pack_view(pack);
    auto go = [&](auto zero) {
        using T = decltype(zero);
        hipLaunchKernelGGL(residual_norm_kernel<T>, dim3(pack->row_cap), dim3(kNormThreads),
                           (size_t)sh->D * sizeof(float), stream, static_cast<const T*>(y),
                           static_cast<const T*>(h), static_cast<const T*>(gate),
                           static_cast<const T*>(w_post), static_cast<const T*>(w_pre),
                           static_cast<T*>(h_out), static_cast<T*>(n_out), pv, sh->D, sh->gate,
                           sh->eps, sh->res_scale);
    };
    if (sh->dtype == FB_BF16) go(uint16_t());
    else go(float());
    return hipGetLastError();
}

}  // namespace fb
