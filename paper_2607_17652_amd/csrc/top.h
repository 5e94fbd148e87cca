// Running (max, lowest index of the max, scaled sum of exponentials) of a
// row's logits, and its merge -- shared by the streaming vocab pass and the
// LM-head epilogue, which both produce 16-byte partials
// {m, s, idx bits, mL} per (row, vocabulary partition).
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>

namespace fb {

constexpr float kLog2e = 1.4426950408889634f;

// Logits down to the type's lowest value stand for masked tokens.  At and below kLow
// rounding m*log2e alone moves an exponent by 64 and more, the product ends as -inf, and
// sums relative to it as infinities and NaN.  So the vocabulary pass takes nothing there
// for a maximum, and what lies there weighs nothing beside others.  A share of nothing
// else is walked again for its maximum and the count of it (below kLow neighbouring
// floats lie 128 apart: whatever is less than the maximum weighs nothing).
constexpr float kLow = -0x1p30f;
constexpr float kLowRef = kLow * kLog2e;   // exact

// Running (max, index, scaled sum).  `s` is relative to mL = round(m*log2e); where a
// share's m is kLow or less it is the count of m, and mL is kLowRef.
struct Top {
    float m;
    float mL;
    float s;
    int idx;
};

__device__ inline Top top_empty() { return Top{-INFINITY, -INFINITY, 0.f, 0x7fffffff}; }

// The reference mL must be the rounded product everywhere it is used: with
// contraction, `x - m*log2e` would become an fma on the exact product and
// every merge would scale the sum by the product's rounding error.
__device__ inline float scaled_ref(float m) {
#pragma clang fp contract(off)
    return m * kLog2e;
}

// Order-independent merge of two partial results (commutative bit for bit); the larger
// mL is the larger m's.
__device__ inline Top top_merge(const Top& a, const Top& b) {
#pragma clang fp contract(off)
    if (a.m == -INFINITY) return b;
    if (b.m == -INFINITY) return a;
    Top r;
    r.m = fmaxf(a.m, b.m);
    r.mL = fmaxf(a.mL, b.mL);
    r.s = a.s * __builtin_amdgcn_exp2f(a.mL - r.mL) + b.s * __builtin_amdgcn_exp2f(b.mL - r.mL);
    r.idx = a.m > b.m ? a.idx : (b.m > a.m ? b.idx : min(a.idx, b.idx));
    return r;
}

// The same for shares, whose s may be counts.
__device__ inline Top top_merge_shares(const Top& a, const Top& b) {
    Top r = top_merge(a, b);
    if (r.m <= kLow) r.s = (a.m == r.m ? a.s : 0.f) + (b.m == r.m ? b.s : 0.f);
    return r;
}

// 1 / sum exp(z - m), m the maximum; 0 if there is none.  s is relative to mL, whose
// rounding is undone exactly.
__device__ inline float top_confidence(const Top& t) {
    if (t.m <= kLow) return t.m == -INFINITY ? 0.f : 1.f / fmaxf(t.s, 1.f);
    return 1.f / (t.s * __builtin_amdgcn_exp2f(-fmaf(t.m, kLog2e, -t.mL)));
}

__device__ inline float4 top_pack(const Top& t) {
    return make_float4(t.m, t.s, __int_as_float(t.idx), t.mL);
}

__device__ inline Top top_unpack(const float4& p) {
    return Top{p.x, p.w, p.y, __float_as_int(p.z)};
}

}  // namespace fb
