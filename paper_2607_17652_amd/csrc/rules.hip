// Penalties for repeated tokens, biases and grammar masks on the live rows'
// logits, in front of the denoise update's reduction.
//
// rules_build_kernel   one workgroup per request turns its committed prefix and
//                      its biases into a bitmap of touched tokens and, at those
//                      tokens only, a count word and a bias.  The dense arrays
//                      are never cleared: an entry is read only where its bit
//                      is set, and every such entry was written by this build.
// vocab_rules_kernel   the vocabulary pass (the same pieces, folds and merges)
//                      on adjusted logits; a group of logits costs one more
//                      byte of bitmap and one of mask, and the gather of counts
//                      and biases only where a bit is set.
// predict_kernel       merges a row's partials into (p, x_hat).
// logits_rules_kernel  the adjusted logits, written.
#include "internal.h"
#include "vocab.h"

namespace fb {
namespace {

constexpr int kBuildThreads = 1024;
constexpr uint32_t kSeen = 0x80000000u;   // count word: seen; the rest is c_v

struct RuleView {
    float4* rec;          // [B] repetition, presence, frequency, 1 if sound
    uint32_t* bits;       // [B][words]
    uint32_t* count;      // [B][words * 32]
    float* bias;          // [B][words * 32]
    int words;
};

inline RuleView rule_view(const RulesSizes& z, void* ws) {
    char* p = static_cast<char*>(ws);
    return RuleView{reinterpret_cast<float4*>(p), reinterpret_cast<uint32_t*>(p + z.off_bits),
                    reinterpret_cast<uint32_t*>(p + z.off_count),
                    reinterpret_cast<float*>(p + z.off_bias), z.words};
}

__device__ inline bool finite(float x) { return fabsf(x) < INFINITY; }

__global__ void __launch_bounds__(kBuildThreads)
rules_build_kernel(fb_logit_rules rules, const fb_req_state* __restrict__ st,
                   const int32_t* __restrict__ tokens, int T_max, int V, PackView pv,
                   RuleView rv) {
    extern __shared__ uint32_t s_bits[];
    __shared__ int s_bad;
    const int b = blockIdx.x;
    const int tid = threadIdx.x;
    if (pv.req_w[b] <= 0) return;   // no live row reads this request's rules
    const int row0 = pv.req_row0[b];
    const int o = min(max(pv.row_pos[row0], 0), T_max);
    const int prompt = st[b].prompt_len;
    const int32_t* tok = tokens + (size_t)b * T_max;
    uint32_t* count = rv.count + (size_t)b * rv.words * 32;
    float* bias = rv.bias + (size_t)b * rv.words * 32;

    float4 rec = make_float4(1.f, 0.f, 0.f, 1.f);
    bool bad = false;
    if (rules.params) {
        const fb_rule_params p = rules.params[b];
        rec = make_float4(p.repetition, p.presence, p.frequency, 1.f);
        bad = !(p.repetition > 0.f) || !finite(p.repetition) || !finite(p.presence) ||
              !finite(p.frequency);
    }
    int lo = 0, hi = 0;
    if (rules.bias_start) {
        lo = rules.bias_start[b];
        hi = rules.bias_start[b + 1];
        if (lo < 0 || lo > hi || hi > rules.n_bias) {
            bad = true;
            lo = hi = 0;
        }
    }
    if (tid == 0) s_bad = 0;
    for (int i = tid; i < rv.words; i += kBuildThreads) s_bits[i] = 0;
    __syncthreads();
    for (int i = lo + tid; i < hi; i += kBuildThreads) {
        const int id = rules.bias_id[i];
        if (id < 0 || id >= V || (i > lo && rules.bias_id[i - 1] > id) ||
            !(rules.bias_val[i] < INFINITY))
            bad = true;
    }
    if (bad) s_bad = 1;
    __syncthreads();
    if (s_bad) {   // uniform
        rec.w = 0.f;
        if (tid == 0) {
            rv.rec[b] = rec;
            record_error(pv.hdr, b, FB_DERR_RULE);
        }
        return;
    }
    // every touched entry is written before it is counted: biased ones as not
    // seen, then the prefix's as seen
    const int n = rules.params ? o : 0;
    for (int i = lo + tid; i < hi; i += kBuildThreads) count[rules.bias_id[i]] = 0;
    __threadfence();
    __syncthreads();
    for (int i = tid; i < n; i += kBuildThreads) {
        const int v = tok[i];
        if (v < 0 || v >= V) continue;
        count[v] = kSeen;
        bias[v] = 0.f;
        atomicOr(&s_bits[v >> 5], 1u << (v & 31));
    }
    __threadfence();
    __syncthreads();
    for (int i = tid; i < n; i += kBuildThreads) {
        const int v = tok[i];
        if (i >= prompt && v >= 0 && v < V) atomicAdd(&count[v], 1u);
    }
    for (int i = lo + tid; i < hi; i += kBuildThreads) {
        const int id = rules.bias_id[i];
        if (i > lo && rules.bias_id[i - 1] == id) continue;
        float s = rules.bias_val[i];
        for (int j = i + 1; j < hi && rules.bias_id[j] == id; ++j) s += rules.bias_val[j];
        bias[id] = s;
        atomicOr(&s_bits[id >> 5], 1u << (id & 31));
    }
    __syncthreads();
    uint32_t* bits = rv.bits + (size_t)b * rv.words;
    for (int i = tid; i < rv.words; i += kBuildThreads) bits[i] = s_bits[i];
    if (tid == 0) rv.rec[b] = rec;
}

// z' of a touched token.
__device__ inline float adjust(float z, uint32_t word, float bias, const float4& rec) {
#pragma clang fp contract(off)
    if (word) z = z > 0.f ? z / rec.x : z * rec.x;
    const float add = bias - ((word & ~kSeen) ? rec.y : 0.f);
    const float times = rec.z * (float)(word & ~kSeen);
    return z + (add - times);
}

// top_fold of logits that may be as low as the type goes (masks of -1e9 or of
// the lowest value).  The sum is kept relative to the rounded m log2 e; where m
// is so large that its rounding alone moves an exponent by more than 4, that
// reference is none.  So where a group's maximum lies below -2^26 its finite
// values count as -2^26: beside any larger logit they weigh nothing either way,
// and a row of nothing else ties.
constexpr float kLowest = -67108864.f;

template <int N>
__device__ inline void fold(Top& t, float (&f)[N], int v) {
    const float vmax = max_of(f);
    if (vmax < kLowest && vmax > -INFINITY) {
#pragma unroll
        for (int j = 0; j < N; ++j) f[j] = f[j] > -INFINITY ? fmaxf(f[j], kLowest) : f[j];
    }
    top_fold<N>(t, f, v);
}

// A row's rules: what the kernels below need to adjust its logits.
struct RowRules {
    float4 rec;
    const uint8_t* bits;      // touched bitmap of the request, NULL if none
    const uint8_t* mask;      // allowed bitmap of the row, NULL if all
    const uint32_t* count;
    const float* bias;
    bool none;                // nothing is allowed

    // N consecutive logits from index v on (v + N <= V).
    template <int N>
    __device__ inline void apply(float (&f)[N], int v) const {
        constexpr uint32_t all = (1u << N) - 1;
        if (bits) {
            const uint32_t t = window(bits, v, N) & all;
            if (t) {
#pragma unroll
                for (int j = 0; j < N; ++j)
                    if (t >> j & 1) f[j] = adjust(f[j], count[v + j], bias[v + j], rec);
            }
        }
        if (mask) {
            const uint32_t a = window(mask, v, N) & all;
#pragma unroll
            for (int j = 0; j < N; ++j) f[j] = a >> j & 1 ? f[j] : -INFINITY;
        }
    }

    // The bits from index v on, at least n <= 8 of them.
    static __device__ inline uint32_t window(const uint8_t* p, int v, int n) {
        const uint32_t w = p[v >> 3] | (uint32_t)p[(v + n - 1) >> 3] << 8;
        return w >> (v & 7);
    }
};

__device__ inline RowRules row_rules(const fb_logit_rules& rules, const RuleView& rv,
                                     const PackView& pv, int row, int req, int mask_words) {
    RowRules r;
    r.rec = rv.rec[req];
    const size_t at = (size_t)req * rv.words;
    r.bits = rules.params || rules.bias_start
                 ? reinterpret_cast<const uint8_t*>(rv.bits + at) : nullptr;
    r.count = rv.count + at * 32;
    r.bias = rv.bias + at * 32;
    r.none = r.rec.w == 0.f;
    r.mask = nullptr;
    if (rules.masks) {
        const int m = rules.row_mask[row];
        if (m < -1 || m >= rules.n_masks) {
            if (threadIdx.x == 0) record_error(pv.hdr, req, FB_DERR_RULE);
            r.none = true;
        } else if (m >= 0) {
            r.mask = reinterpret_cast<const uint8_t*>(rules.masks + (size_t)m * mask_words);
        }
    }
    return r;
}

template <typename T>
__global__ void __launch_bounds__(kVocabThreads)
vocab_rules_kernel(const T* __restrict__ logits, int V, int nsplit, PackView pv,
                   fb_logit_rules rules, RuleView rv, int mask_words,
                   float4* __restrict__ part) {
    using VT = VecTraits<T>;
    constexpr int N = VT::N;
    constexpr int kBatch = kVocabBatch;
    const int row = blockIdx.x / nsplit;
    const int k = blockIdx.x % nsplit;
    const int req = pv.row_req[row];
    if (req < 0) return;
    const int tid = threadIdx.x;
    const RowRules rr = row_rules(rules, rv, pv, row, req, mask_words);
    if (rr.none) {
        if (tid == 0) part[(size_t)row * nsplit + k] = top_pack(top_empty());
        return;
    }
    const T* rp = logits + (size_t)row * V;
    const size_t abs0 = (size_t)row * V;
    int a = (int)((N - (abs0 % N)) % N);
    if (a > V) a = V;
    const int e = a + ((V - a) / N) * N;

    Top t = top_empty();
    if (k == 0 && tid < a) {
        float f[1] = {VT::scalar(rp + tid)};
        rr.template apply<1>(f, tid);
        fold<1>(t, f, tid);
    }
    const int stride = kVocabThreads * N;
    const int piece = kBatch * stride;
    for (int base = a + k * piece + tid * N; base < e; base += nsplit * piece) {
        uint4 raw[kBatch];
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            const int v = base + j * stride;
            raw[j] = v < e ? load_stream16(rp + v) : make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            const int v = base + j * stride;
            if (v < e) {
                float f[N];
                VT::unpack(raw[j], f);
                rr.template apply<N>(f, v);
                fold<N>(t, f, v);
            }
        }
    }
    if (k == 0 && tid < V - e) {
        float f[1] = {VT::scalar(rp + e + tid)};
        rr.template apply<1>(f, e + tid);
        fold<1>(t, f, e + tid);
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) {
        Top o;
        o.m = __shfl_xor(t.m, off, 64);
        o.mL = __shfl_xor(t.mL, off, 64);
        o.s = __shfl_xor(t.s, off, 64);
        o.idx = __shfl_xor(t.idx, off, 64);
        t = top_merge(t, o);
    }
    __shared__ Top wtop[kVocabThreads / 64];
    if ((tid & 63) == 0) wtop[tid >> 6] = t;
    __syncthreads();
    if (tid == 0) {
        Top r = wtop[0];
        for (int w = 1; w < kVocabThreads / 64; ++w) r = top_merge(r, wtop[w]);
        part[(size_t)row * nsplit + k] = top_pack(r);
    }
}

// (p, x_hat) of every live row from its partials, as the update merges them.
constexpr int kPredictThreads = 256;

__global__ void __launch_bounds__(kPredictThreads)
predict_kernel(const float4* __restrict__ part, int nsplit, PackView pv, int row_cap,
               float* __restrict__ conf, int32_t* __restrict__ argmax) {
    const int row = blockIdx.x * kPredictThreads + threadIdx.x;
    if (row >= row_cap || pv.row_req[row] < 0) return;
    Top t = top_unpack(part[(size_t)row * nsplit]);
    for (int k = 1; k < nsplit; ++k)
        t = top_merge(t, top_unpack(part[(size_t)row * nsplit + k]));
    const float resid = fmaf(t.m, kLog2e, -t.mL);
    const bool none = t.m == -INFINITY;
    conf[row] = none ? 0.f : 1.0f / (t.s * __builtin_amdgcn_exp2f(-resid));
    argmax[row] = none ? -1 : t.idx;
}

template <typename T>
__global__ void __launch_bounds__(kVocabThreads)
logits_rules_kernel(const T* logits, T* out, int V, int nsplit, PackView pv,
                    fb_logit_rules rules, RuleView rv, int mask_words) {
    using VT = VecTraits<T>;
    const int row = blockIdx.x / nsplit;
    const int k = blockIdx.x % nsplit;
    const int req = pv.row_req[row];
    if (req < 0) return;
    const RowRules rr = row_rules(rules, rv, pv, row, req, mask_words);
    const T* rp = logits + (size_t)row * V;
    T* wp = out + (size_t)row * V;
    for (int v = k * kVocabThreads + threadIdx.x; v < V; v += nsplit * kVocabThreads) {
        float f[1] = {VT::scalar(rp + v)};
        rr.template apply<1>(f, v);
        if (rr.none) f[0] = -INFINITY;
        if constexpr (sizeof(T) == 2) {
            const __bf16 r = (__bf16)f[0];
            wp[v] = __builtin_bit_cast(uint16_t, r);
        } else {
            wp[v] = f[0];
        }
    }
}

}  // namespace

RulesSizes rules_sizes(const fb_pack* pack, int V) {
    RulesSizes z{};
    z.words = (V + 127) / 128 * 4;
    const size_t B = pack->B;
    z.off_bits = (B * sizeof(float4) + 255) / 256 * 256;
    z.off_count = z.off_bits + (B * z.words * 4 + 255) / 256 * 256;
    z.off_bias = z.off_count + B * z.words * 32 * 4;
    z.total = z.off_bias + B * z.words * 32 * 4;
    return z;
}

hipError_t launch_rules_build(const fb_logit_rules* rules, const fb_req_state* st,
                              const int32_t* tokens, int T_max, int V, const fb_pack* pack,
                              void* ws, const RulesSizes& z, hipStream_t stream) {
    hipLaunchKernelGGL(rules_build_kernel, dim3(pack->B), dim3(kBuildThreads),
                       (size_t)z.words * 4, stream, *rules, st, tokens, T_max, V,
                       pack_view(pack), rule_view(z, ws));
    return hipGetLastError();
}

hipError_t launch_vocab_rules(const void* logits, int V, int dtype, const fb_pack* pack,
                              const fb_logit_rules* rules, const void* rules_ws,
                              const RulesSizes& rz, void* upd_ws, const UpdateSizes& uz,
                              float* conf, int32_t* argmax, hipStream_t stream) {
    PackView pv = pack_view(pack);
    const RuleView rv = rule_view(rz, const_cast<void*>(rules_ws));
    float4* part = static_cast<float4*>(upd_ws);
    auto go = [&](auto zero) {
        using T = decltype(zero);
        hipLaunchKernelGGL(vocab_rules_kernel<T>,
                           dim3((unsigned)pack->row_cap * (unsigned)uz.nsplit),
                           dim3(kVocabThreads), 0, stream, static_cast<const T*>(logits), V,
                           uz.nsplit, pv, *rules, rv, (V + 31) / 32, part);
    };
    if (dtype == FB_BF16) go(uint16_t());
    else go(float());
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || !conf) return e;
    hipLaunchKernelGGL(predict_kernel,
                       dim3((pack->row_cap + kPredictThreads - 1) / kPredictThreads),
                       dim3(kPredictThreads), 0, stream, part, uz.nsplit, pv, pack->row_cap,
                       conf, argmax);
    return hipGetLastError();
}

hipError_t launch_logits_rules(const void* logits, void* out, int V, int dtype,
                               const fb_pack* pack, const fb_logit_rules* rules,
                               const void* rules_ws, const RulesSizes& rz,
                               const UpdateSizes& uz, hipStream_t stream) {
    const RuleView rv = rule_view(rz, const_cast<void*>(rules_ws));
    auto go = [&](auto zero) {
        using T = decltype(zero);
        hipLaunchKernelGGL(logits_rules_kernel<T>,
                           dim3((unsigned)pack->row_cap * (unsigned)uz.nsplit),
                           dim3(kVocabThreads), 0, stream, static_cast<const T*>(logits),
                           static_cast<T*>(out), V, uz.nsplit, pack_view(pack), *rules, rv,
                           (V + 31) / 32);
    };
    if (dtype == FB_BF16) go(uint16_t());
    else go(float());
    return hipGetLastError();
}

}  // namespace fb
