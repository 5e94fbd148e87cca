// Streaming of a row of logits into its running (max, lowest index, scaled
// sum) -- shared by the vocabulary pass and its form under logit rules.
#pragma once

#include "top.h"

namespace fb {

constexpr int kVocabThreads = 512;   // 8 waves per (row, partition): measured 1% faster than 4

// Maximum of the values (logits hold no NaN, so the max needs no quieting
// of its inputs: three-input v_max3 steps instead of fmaxf chains).
template <int N>
__device__ inline float max_of(const float (&f)[N]) {
    if constexpr (N == 1) {
        return f[0];
    } else {
        float m = f[0];
        int j = 1;
        for (; j + 1 < N; j += 2)
            asm("v_max3_f32 %0, %1, %2, %3" : "=v"(m) : "v"(m), "v"(f[j]), "v"(f[j + 1]));
        if (j < N) asm("v_max_f32 %0, %1, %2" : "=v"(m) : "v"(m), "v"(f[j]));
        return m;
    }
}

// What the fold starts from: kLow is no maximum, and -inf logits give exp2(-inf) = 0.
__device__ inline Top top_low() { return Top{kLow, kLowRef, 0.f, 0x7fffffff}; }

// Fold n consecutive values starting at index v into t (values in index order).
template <int N>
__device__ inline void top_fold(Top& t, const float (&f)[N], int v) {
    const float vmax = max_of(f);
    if (vmax > t.m) {
#pragma clang fp contract(off)
        int j0 = N - 1;
#pragma unroll
        for (int j = N - 1; j >= 0; --j)
            if (f[j] == vmax) j0 = j;
        const float nmL = scaled_ref(vmax);
        t.s *= __builtin_amdgcn_exp2f(t.mL - nmL);
        t.m = vmax;
        t.mL = nmL;
        t.idx = v + j0;
    }
    float e[N];
#pragma unroll
    for (int j = 0; j < N; ++j) e[j] = __builtin_amdgcn_exp2f(fmaf(f[j], kLog2e, -t.mL));
#pragma unroll
    for (int w = 1; w < N; w <<= 1)
#pragma unroll
        for (int j = 0; j + w < N; j += 2 * w) e[j] += e[j + w];
    t.s += e[0];
}

// 16-byte load of logits that are read exactly once: the nontemporal hint
// keeps the stream from displacing reusable lines in the caches, which
// measurably raises the achieved HBM read rate of this pass.
template <typename T>
__device__ inline uint4 load_stream16(const T* p) {
    typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
    const u32x4 x = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p));
    return make_uint4(x[0], x[1], x[2], x[3]);
}

template <typename T>
struct VecTraits;
template <>
struct VecTraits<uint16_t> {   // bf16
    static constexpr int N = 8;
    __device__ static inline void unpack(const uint4& u, float (&f)[8]) {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            f[2 * j] = __uint_as_float(w[j] << 16);
            f[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
        }
    }
    __device__ static inline float scalar(const uint16_t* p) {
        return __uint_as_float(((uint32_t)*p) << 16);
    }
};
template <>
struct VecTraits<float> {
    static constexpr int N = 4;
    __device__ static inline void unpack(const uint4& u, float (&f)[4]) {
        f[0] = __uint_as_float(u.x);
        f[1] = __uint_as_float(u.y);
        f[2] = __uint_as_float(u.z);
        f[3] = __uint_as_float(u.w);
    }
    __device__ static inline float scalar(const float* p) { return *p; }
};

// A row's nsplit workgroups take its 16-byte-aligned body in pieces of
// kBatch loads per thread (32 KB), in turn: workgroup k reads pieces k,
// k + nsplit, ...  Neighbouring workgroups then read neighbouring memory,
// which the HBM serves faster than the same bytes in one contiguous share
// per workgroup.
constexpr int kVocabBatch = 4;

}  // namespace fb
