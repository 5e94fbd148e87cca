// Penalties for repeated tokens, biases and grammar masks on the live rows'
// logits, in front of the denoise update's reduction.
//
// rules_build_kernel   turns the committed prefix and the biases of a request
//                      into a bitmap of touched tokens and a list, in token
//                      order, of what is added to each.  A workgroup per slice
//                      of the vocabulary: a slice's list has its own place, so
//                      no workgroup waits for another.
// vocab_rules_kernel   the vocabulary pass on adjusted logits.  A wave takes
//                      windows of 4 KB: its logits fold as in the plain pass,
//                      touched tokens left out; where the window has any, it is
//                      also staged in LDS and its list entries are adjusted and
//                      folded from there, one a lane.
// predict_kernel       merges a row's partials into (p, x_hat).
// logits_rules_kernel  the adjusted logits, written: the list entries patch the
//                      staged window, which is then stored.
#include <type_traits>

#include "internal.h"
#include "vocab.h"

namespace fb {
namespace {

constexpr int kBuildThreads = 1024;
constexpr int kSpan = 1024;               // tokens whose list entries are found by one lookup
constexpr int kSlice = 2 * kSpan;         // slices of the build are multiples of it
constexpr uint32_t kSeen = 0x80000000u;   // beside a count or an id: the token is seen
constexpr uint32_t kDone = 0x40000000u;   // beside an id, within the build: a bias is in

// What fb_rules_build leaves of request b:
//   rec    repetition (NaN if the rules are unsound) and its reciprocal
//   bits   the touched tokens (seen or biased), a bit each
//   spans  per kSpan tokens, first and one past the last of their entries
//   adj    per touched token what is added, and its id, kSeen set if it is seen;
//          the entries of a slice lie together from its first token's place on
struct RuleView {
    float2* rec;          // [B]
    uint32_t* bits;       // [B][words]
    uint2* spans;         // [B][spans]
    uint2* adj;           // [B][words * 32]
    int words, n_spans;
};

inline RuleView rule_view(const RulesSizes& z, void* ws) {
    char* p = static_cast<char*>(ws);
    return RuleView{reinterpret_cast<float2*>(p), reinterpret_cast<uint32_t*>(p + z.off_bits),
                    reinterpret_cast<uint2*>(p + z.off_spans),
                    reinterpret_cast<uint2*>(p + z.off_adj), z.words, z.spans};
}

__device__ inline bool finite(float x) { return fabsf(x) < INFINITY; }

// What is added to a touched token's logit: (bias - [c > 0] p) - f c.
__device__ inline float addend(float bias, uint32_t c, const fb_rule_params& p) {
#pragma clang fp contract(off)
    const float a = bias - (c ? p.presence : 0.f);
    const float b = p.frequency * (float)c;
    return a - b;
}

// Barrier behind which the workgroup sees its own stores to memory, and its
// atomics come after them.  (A device-wide fence would write the L2 back: the
// build of 256 requests took 160 us with two of them, 15 with this.)
__device__ inline void workgroup_sync() {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
}

// What the wave's lanes wrote to LDS before this is what each of them reads after it.
// The hardware keeps a wave's LDS operations in order; the compiler may not, since
// for it another lane's store is another thread's.  No instruction comes of it.
__device__ inline void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// Calls f(i, token - v0) for the tokens of [0, n) that lie in [v0, v0 + nv), the
// loads of eight rounds in flight together: one token a load up to 8192 of them
// (one round trip, every lane at work), four neighbours beyond.
template <typename F>
__device__ inline void each_token(const int32_t* tok, int n, int v0, int nv, F&& f) {
    typedef int i32x4 __attribute__((ext_vector_type(4), aligned(4)));
    constexpr int U = 8, kRound = 4 * kBuildThreads;
    if (n <= U * kBuildThreads) {
        int v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = threadIdx.x + u * kBuildThreads;
            v[u] = i < n ? tok[i] : -1;
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (v[u] >= v0 && v[u] - v0 < nv) f((int)threadIdx.x + u * kBuildThreads, v[u] - v0);
        return;
    }
    for (int i0 = threadIdx.x * 4; i0 < n; i0 += U * kRound) {
        i32x4 v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = i0 + u * kRound;
            v[u] = i32x4{-1, -1, -1, -1};
            if (i + 4 <= n) {
                v[u] = *reinterpret_cast<const i32x4*>(tok + i);
            } else if (i < n) {
                v[u][0] = tok[i];
                if (i + 1 < n) v[u][1] = tok[i + 1];
                if (i + 2 < n) v[u][2] = tok[i + 2];
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (v[u][j] >= v0 && v[u][j] - v0 < nv) f(i0 + u * kRound + j, v[u][j] - v0);
    }
}

// Workgroup (b, s): tokens [s * slice, (s + 1) * slice) of request b.  LDS: the
// slice's bitmap, per word the touched tokens before it, and a count per touched
// token (in adj where there are more than `lds_counts`).
__global__ void __launch_bounds__(kBuildThreads)
rules_build_kernel(fb_logit_rules rules, const fb_req_state* __restrict__ st,
                   const int32_t* __restrict__ tokens, int T_max, int V, PackView pv,
                   RuleView rv, int slice, int n_slices, int lds_counts) {
    extern __shared__ uint32_t s_bits[];
    const int b = blockIdx.x / n_slices;
    const int v0 = blockIdx.x % n_slices * slice;
    const int nv = min(slice, V - v0);
    const int words = (nv + 31) / 32;
    uint32_t* s_rank = s_bits + words;
    uint32_t* s_count = s_rank + words;
    __shared__ int s_bad;
    __shared__ uint32_t s_wave[kBuildThreads / 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    if (pv.req_w[b] <= 0) return;   // no live row reads this request's rules
    const int row0 = pv.req_row0[b];
    const int o = rules.params ? min(max(pv.row_pos[row0], 0), T_max) : 0;
    const int prompt = st[b].prompt_len;
    const int32_t* tok = tokens + (size_t)b * T_max;

    fb_rule_params p{1.f, 0.f, 0.f, 0};
    bool bad = false;
    if (rules.params) {
        p = rules.params[b];
        // a range in which r and 1 / r are normal, for the quotient of adjust()
        bad = !(p.repetition >= 0x1p-40f && p.repetition <= 0x1p40f) || !finite(p.presence) ||
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
    for (int i = tid; i < words; i += kBuildThreads) s_bits[i] = 0;
    __syncthreads();
    for (int i = lo + tid; i < hi; i += kBuildThreads) {
        const int id = rules.bias_id[i];
        if (id < 0 || id >= V || (i > lo && rules.bias_id[i - 1] > id) ||
            !(rules.bias_val[i] < INFINITY))
            bad = true;
        else if (id >= v0 && id - v0 < nv)
            atomicOr(&s_bits[(id - v0) >> 5], 1u << (id & 31));
    }
    if (bad) s_bad = 1;
    // a bit that is set already takes no atomic: frequent tokens would queue for it
    each_token(tok, o, v0, nv, [&](int, int v) {
        const uint32_t m = 1u << (v & 31);
        if (!(s_bits[v >> 5] & m)) atomicOr(&s_bits[v >> 5], m);
    });
    __syncthreads();
    if (s_bad) {   // uniform, and the same in every slice
        if (tid == 0 && v0 == 0) {
            rv.rec[b] = make_float2(NAN, 0.f);
            record_error(pv.hdr, b, FB_DERR_RULE);
        }
        return;
    }

    // ---- ranks: each thread takes `per` neighbouring words
    const int per = (words + kBuildThreads - 1) / kBuildThreads;
    const int w0 = min(tid * per, words), w1 = min(w0 + per, words);
    uint32_t mine = 0;
    for (int i = w0; i < w1; ++i) mine += __popc(s_bits[i]);
    uint32_t x = mine;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const uint32_t y = __shfl_up(x, off, 64);
        if (lane >= off) x += y;
    }
    if (lane == 63) s_wave[wave] = x;
    __syncthreads();
    uint32_t before = 0, total = 0;
#pragma unroll
    for (int w = 0; w < kBuildThreads / 64; ++w) {
        before += w < wave ? s_wave[w] : 0;
        total += s_wave[w];
    }
    uint32_t at = before + x - mine;
    for (int i = w0; i < w1; ++i) {
        s_rank[i] = at;
        at += __popc(s_bits[i]);
    }
    const bool local = total <= (uint32_t)lds_counts;
    if (local)
        for (uint32_t i = tid; i < total; i += kBuildThreads) s_count[i] = 0;
    __syncthreads();

    // ---- the list's ids, the bitmap and the spans
    uint2* adj = rv.adj + (size_t)b * rv.words * 32 + v0;
    uint32_t* bits = rv.bits + (size_t)b * rv.words + v0 / 32;
    uint2* spans = rv.spans + (size_t)b * rv.n_spans + v0 / kSpan;
    for (int i = tid; i < words; i += kBuildThreads) {
        uint32_t k = s_rank[i];
        bits[i] = s_bits[i];
        for (uint32_t m = s_bits[i]; m; m &= m - 1, ++k)
            adj[k] = make_uint2(0, (uint32_t)(v0 + i * 32 + __ffs(m) - 1));
        if (i % (kSpan / 32) == 0) {
            const int next = i + kSpan / 32;
            spans[i / (kSpan / 32)] = make_uint2(v0 + s_rank[i], v0 + (next < words ? s_rank[next] : total));
        }
    }
    workgroup_sync();

    // ---- counts (adj.x holds those that do not fit the LDS)
    auto slot = [&](int v) {
        return s_rank[v >> 5] + __popc(s_bits[v >> 5] & ((1u << (v & 31)) - 1));
    };
    each_token(tok, o, v0, nv, [&](int i, int v) {
        const uint32_t k = slot(v);
        if (!local) {
            if (i >= prompt) atomicAdd(&adj[k].x, 1u);
            else atomicOr(&adj[k].x, kSeen);
        } else if (i >= prompt) {
            atomicAdd(&s_count[k], 1u);
        } else if (!(s_count[k] & kSeen)) {
            atomicOr(&s_count[k], kSeen);
        }
    });
    workgroup_sync();
    // ---- entries without a bias, then those that have one
    for (uint32_t i = tid; i < total; i += kBuildThreads) {
        // counts in memory were added to past the L1
        const uint32_t c = local ? s_count[i]
            : __hip_atomic_load(&adj[i].x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        const uint32_t id = adj[i].y;
        adj[i] = make_uint2(local ? __float_as_uint(addend(0.f, c & ~kSeen, p)) : c,
                            id | (c ? kSeen : 0u));
    }
    workgroup_sync();
    for (int i = lo + tid; i < hi; i += kBuildThreads) {
        const int id = rules.bias_id[i];
        if (id < v0 || id - v0 >= nv || (i > lo && rules.bias_id[i - 1] == id)) continue;
        float bias = rules.bias_val[i];
        for (int j = i + 1; j < hi && rules.bias_id[j] == id; ++j) bias += rules.bias_val[j];
        const uint32_t k = slot(id - v0);
        if (local) adj[k].x = __float_as_uint(addend(bias, s_count[k] & ~kSeen, p));
        else adj[k] = make_uint2(__float_as_uint(addend(bias, adj[k].x & ~kSeen, p)), adj[k].y | kDone);
    }
    if (!local) {
        workgroup_sync();
        for (uint32_t i = tid; i < total; i += kBuildThreads) {
            const uint2 e = adj[i];
            adj[i] = e.y & kDone ? make_uint2(e.x, e.y & ~kDone)
                                 : make_uint2(__float_as_uint(addend(0.f, e.x & ~kSeen, p)), e.y);
        }
    }
    if (tid == 0 && v0 == 0) rv.rec[b] = make_float2(p.repetition, 1.f / p.repetition);
}

// z' of a touched token.  z / r is the correctly rounded quotient: z times the
// rounded reciprocal, corrected once by its exact remainder (Markstein, "Computation
// of elementary functions on the IBM RISC System/6000 processor", 1990).  The remainder
// is exact while its last bit, 2^-47 of z, is a float: from z = 2^-80 on, where the
// quotient is normal too.  Smaller logits, and quotients whose first step overflows, are
// divided.
__device__ inline float adjust(float z, const uint2& adj, const float2& rec) {
#pragma clang fp contract(off)
    const float q = z * rec.y;
    float div = fmaf(fmaf(-q, rec.x, z), rec.y, q);
    if (z > 0.f && (z < 0x1p-80f || !finite(q))) div = z / rec.x;
    const float pen = z > 0.f ? div : z * rec.x;
    return (adj.y & kSeen ? pen : z) + __uint_as_float(adj.x);
}

// A wave's running maximum, its place and the scaled sum (see Top), for logits
// that may be as low as the type goes (masks of -1e9 or of the lowest value).
//
// The maximum is the wave's, not the lane's: among 64 lanes some lane meets a new
// maximum of its own in nearly every group, the wave in few, and a group costs 37
// instructions instead of 70.  A lane keeps the place where it last met it.  Both
// are held apart for the touched tokens and the others (K of fold): the ids of
// either come in ascending order, so the first of equal maxima stays.
//
// The sum is kept relative to the rounded m log2 e; where m is so large that its
// rounding alone moves an exponent by more than 4, that reference is none.  So a
// walk begins at m = -2^26: what lies there or below weighs nothing and is no
// maximum.  A share that ends without a maximum is walked again, its finite values
// counted as -2^26.
constexpr float kLowest = -67108864.f;

struct WaveTop {
    float m[2] = {kLowest, kLowest};               // the wave's maxima
    float mL = scaled_ref(kLowest);                // of the larger one
    float s = 0.f;                                 // the lane's share of the sum
    float at[2] = {-INFINITY, -INFINITY};          // the maximum as the lane last met it
    int idx[2] = {0x7fffffff, 0x7fffffff};         // and its id

    // N logits of ids v ..; lanes that take no part pass -inf
    template <int K, int N>
    __device__ inline void fold(const float (&f)[N], int v) {
#pragma clang fp contract(off)
        const float vmax = max_of(f);
        if (__ballot(vmax > m[K])) {
            if (vmax > m[K]) {
                int j0 = N - 1;
#pragma unroll
                for (int j = N - 1; j >= 0; --j)
                    if (f[j] == vmax) j0 = j;
                at[K] = vmax;
                idx[K] = v + j0;
            }
            float w = vmax;
#pragma unroll
            for (int off = 32; off > 0; off >>= 1) w = fmaxf(w, __shfl_xor(w, off, 64));
            m[K] = w;
            const float nmL = fmaxf(mL, scaled_ref(w));
            s *= __builtin_amdgcn_exp2f(mL - nmL);
            mL = nmL;
        }
        float e[N];
#pragma unroll
        for (int j = 0; j < N; ++j) e[j] = __builtin_amdgcn_exp2f(fmaf(f[j], kLog2e, -mL));
#pragma unroll
        for (int w = 1; w < N; w <<= 1)
#pragma unroll
            for (int j = 0; j + w < N; j += 2 * w) e[j] += e[j + w];
        s += e[0];
    }

    // The wave's Top; every lane gets it.
    __device__ inline Top top() const {
        const float most = fmaxf(m[0], m[1]);
        float sum = s;
        int first = min(at[0] == most ? idx[0] : 0x7fffffff, at[1] == most ? idx[1] : 0x7fffffff);
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) {
            sum += __shfl_xor(sum, off, 64);
            first = min(first, __shfl_xor(first, off, 64));
        }
        return Top{most, mL, sum, first};
    }
};

// A row's rules: what the kernels below need to adjust its logits.
struct RowRules {
    float2 rec;
    const uint8_t* bits;      // touched bitmap of the request, NULL if none
    const uint2* spans;
    const uint2* adj;
    const uint8_t* mask;      // allowed bitmap of the row, NULL if all
    bool none;                // nothing is allowed

    // the bits of the eight tokens from v on (v a multiple of 8)
    __device__ inline uint32_t allowed(int v) const { return mask ? mask[v >> 3] : 255u; }
};

__device__ inline RowRules row_rules(const fb_logit_rules& rules, const RuleView& rv,
                                     const PackView& pv, int row, int req, int mask_words) {
    RowRules r;
    r.rec = rv.rec[req];
    r.bits = rules.params || rules.bias_start
                 ? reinterpret_cast<const uint8_t*>(rv.bits + (size_t)req * rv.words) : nullptr;
    r.spans = rv.spans + (size_t)req * rv.n_spans;
    r.adj = rv.adj + (size_t)req * rv.words * 32;
    r.none = isnan(r.rec.x);
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
__device__ inline float value(T x) {
    if constexpr (sizeof(T) == 2) return __uint_as_float((uint32_t)x << 16);
    else return x;
}
template <typename T>
__device__ inline T minus_inf() {
    if constexpr (sizeof(T) == 2) return (T)0xff80;
    else return -INFINITY;
}

// Rows of a vocabulary that is no multiple of eight start anywhere; the address
// unit takes misaligned 16 bytes.
typedef unsigned Words16 __attribute__((ext_vector_type(4), aligned(2)));

// Eight logits.
template <typename T>
struct Eight {
    static constexpr int Q = sizeof(T) / 2;
    uint4 q[Q];

    __device__ inline void load(const T* p) {
#pragma unroll
        for (int i = 0; i < Q; ++i) {
            const Words16 x = __builtin_nontemporal_load(reinterpret_cast<const Words16*>(p) + i);
            q[i] = make_uint4(x[0], x[1], x[2], x[3]);
        }
    }
    __device__ inline void load(const T* p, int n) {     // n elements, the others -inf
        T t[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) t[i] = i < n ? p[i] : minus_inf<T>();
        __builtin_memcpy(q, t, sizeof t);
    }
    __device__ inline void store(T* p, int n) const {
        if (n >= 8) {
#pragma unroll
            for (int i = 0; i < Q; ++i)
                __builtin_nontemporal_store(Words16{q[i].x, q[i].y, q[i].z, q[i].w},
                                            reinterpret_cast<Words16*>(p) + i);
        } else {
            T t[8];
            __builtin_memcpy(t, q, sizeof t);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < n) p[i] = t[i];
        }
    }
    __device__ inline void unpack(float (&f)[8]) const {
        if constexpr (sizeof(T) == 2) {
            VecTraits<uint16_t>::unpack(q[0], f);
        } else {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                f[4 * i] = __uint_as_float(q[i].x);
                f[4 * i + 1] = __uint_as_float(q[i].y);
                f[4 * i + 2] = __uint_as_float(q[i].z);
                f[4 * i + 3] = __uint_as_float(q[i].w);
            }
        }
    }
    static __device__ inline uint32_t pick(uint32_t m, uint32_t a, uint32_t b) {
        return (m & a) | (~m & b);
    }
    // -inf where a bit of `keep` is 0
    __device__ inline void mask(uint32_t keep) {
        auto bit = [&](int i) { return (uint32_t)__builtin_amdgcn_sbfe(keep, i, 1); };
        if constexpr (sizeof(T) == 2) {
            auto word = [&](int i, uint32_t x) {   // two bits' signs, a half word each
                return pick(__builtin_amdgcn_perm(bit(2 * i + 1), bit(2 * i), 0x05040100u), x,
                            0xff80ff80u);
            };
            q[0] = make_uint4(word(0, q[0].x), word(1, q[0].y), word(2, q[0].z), word(3, q[0].w));
        } else {
            const uint32_t inf = 0xff800000u;
#pragma unroll
            for (int i = 0; i < 2; ++i)
                q[i] = make_uint4(pick(bit(4 * i), q[i].x, inf), pick(bit(4 * i + 1), q[i].y, inf),
                                  pick(bit(4 * i + 2), q[i].z, inf),
                                  pick(bit(4 * i + 3), q[i].w, inf));
        }
    }
};

// A row's workgroups take its pieces of 32 KB in turn; of a piece a wave takes a
// window of 4 KB, a lane kBatch groups of eight logits.
template <typename T>
struct Window {
    static constexpr int kBatch = kVocabBatch * 2 / sizeof(T);
    static constexpr int kTokens = kBatch * 512;
    static constexpr int kPiece = kTokens * (kVocabThreads / 64);
    static_assert(kTokens % kSpan == 0 && kSlice % kTokens == 0);
    typedef T Stage[kTokens];

    Eight<T> raw[kBatch];

    // What lies past the row comes out as -inf.
    __device__ inline void load(const T* rp, int v0, int V) {
        const int base = v0 + (threadIdx.x & 63) * 8;
        if (v0 + kTokens <= V) {   // uniform
#pragma unroll
            for (int j = 0; j < kBatch; ++j) raw[j].load(rp + base + j * 512);
            return;
        }
        fill();
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            const int v = base + j * 512;
            if (v + 8 <= V) raw[j].load(rp + v);
            else if (v < V) raw[j].load(rp + v, V - v);
        }
    }
    __device__ inline void fill() {
        const uint32_t inf = sizeof(T) == 2 ? 0xff80ff80u : 0xff800000u;
#pragma unroll
        for (int j = 0; j < kBatch; ++j)
#pragma unroll
            for (int i = 0; i < Eight<T>::Q; ++i) raw[j].q[i] = make_uint4(inf, inf, inf, inf);
    }
    // the lane's bytes of the row's mask, none past the row
    struct Allowed {
        uint32_t b[kBatch];

        __device__ inline void load(const uint8_t* mask, int v0, int V) {
            if (v0 + kTokens <= V) {   // uniform
#pragma unroll
                for (int j = 0; j < kBatch; ++j)
                    b[j] = (mask + (v0 >> 3))[(threadIdx.x & 63) + j * 64];
                return;
            }
#pragma unroll
            for (int j = 0; j < kBatch; ++j) {
                const int v = v0 + j * 512 + (threadIdx.x & 63) * 8;
                b[j] = v < V ? mask[v >> 3] : 0;
                if (v + 8 > V && v < V) b[j] &= (1u << (V - v)) - 1;
            }
        }
        __device__ inline bool some() const {   // uniform
            uint32_t m = 0;
#pragma unroll
            for (int j = 0; j < kBatch; ++j) m |= b[j];
            return __ballot(m != 0) != 0;
        }
    };
    // -inf where the mask forbids it
    __device__ inline void mask(const Allowed& allowed) {
#pragma unroll
        for (int j = 0; j < kBatch; ++j)
            if (__ballot(allowed.b[j] != 255)) raw[j].mask(allowed.b[j]);
    }
    __device__ inline void stage(Stage& s) const {
#pragma unroll
        for (int j = 0; j < kBatch; ++j)
            __builtin_memcpy(&s[j * 512 + (threadIdx.x & 63) * 8], raw[j].q, sizeof raw[j].q);
    }
    __device__ inline void fetch(const Stage& s) {
#pragma unroll
        for (int j = 0; j < kBatch; ++j)
            __builtin_memcpy(raw[j].q, &s[j * 512 + (threadIdx.x & 63) * 8], sizeof raw[j].q);
    }
};

// The entries of the wave's windows: lane i has the first of its i-th window's,
// lane 32 + i one past the last.  A row of 2^19 float32 logits is 64 pieces, so its
// workgroups have to be two at least; update_sizes makes them two, and the launchers
// refuse what does not fit.
constexpr int kMaxWindows = 32;

template <typename T>
inline bool walk_fits(int V, int nsplit) {
    const int round = nsplit * Window<T>::kPiece;
    return (V + round - 1) / round <= kMaxWindows;
}

template <typename T>
__device__ inline uint32_t window_entries(const RowRules& rr, int first, int stride, int V) {
    if (!rr.bits) return 0;
    const int lane = threadIdx.x & 63;
    const int v0 = first + (lane & (kMaxWindows - 1)) * stride;
    if (v0 >= V) return 0;
    const int last = min((v0 + Window<T>::kTokens) / kSpan, (V + kSpan - 1) / kSpan) - 1;
    return lane < kMaxWindows ? rr.spans[v0 / kSpan].x : rr.spans[last].y;
}

// (p, x_hat) of a row from all of it.
__device__ inline void predict(const Top& t, float* conf, int32_t* argmax) {
    *conf = top_confidence(t);
    *argmax = t.m == -INFINITY ? -1 : t.idx;
}

// `conf` and `argmax`, if not NULL, are written here: nsplit is 1 then.
template <typename T>
__global__ void __launch_bounds__(kVocabThreads, 8)
vocab_rules_kernel(const T* __restrict__ logits, int V, int nsplit, PackView pv,
                   fb_logit_rules rules, RuleView rv, int mask_words,
                   float4* __restrict__ part, float* __restrict__ conf,
                   int32_t* __restrict__ argmax) {
    using W = Window<T>;
    __shared__ __attribute__((aligned(16))) typename W::Stage stages[kVocabThreads / 64];
    __shared__ Top wtop[kVocabThreads / 64];
    __shared__ int s_met[kVocabThreads / 64];
    const int row = blockIdx.x / nsplit;
    const int k = blockIdx.x % nsplit;
    const int req = pv.row_req[row];
    if (req < 0) return;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const RowRules rr = row_rules(rules, rv, pv, row, req, mask_words);
    if (rr.none) {
        if (tid == 0) {
            part[(size_t)row * nsplit + k] = top_pack(top_empty());
            if (conf) predict(top_empty(), conf + row, argmax + row);
        }
        return;
    }
    const T* rp = logits + (size_t)row * V;
    const int first = k * W::kPiece + wave * W::kTokens;
    const int stride = nsplit * W::kPiece;
    const uint32_t entries = window_entries<T>(rr, first, stride, V);
    typename W::Stage& stage = stages[wave];

    WaveTop wt;
    // The mask's bytes come a window ahead: of a window that allows nothing the
    // logits are not read.
    typename W::Allowed allowed, next;
    if (rr.mask) next.load(rr.mask, first, V);
    bool any = false;     // something is allowed
    int i = 0;
    for (int v0 = first; v0 < V; v0 += stride, ++i) {
        if (rr.mask) {    // uniform
            allowed = next;
            const bool some = allowed.some();
            if (v0 + stride < V) next.load(rr.mask, v0 + stride, V);
            if (!some) continue;
        }
        any = true;
        const int e0 = __builtin_amdgcn_readlane(entries, i);
        const int e1 = __builtin_amdgcn_readlane(entries, kMaxWindows + i);
        W w;
        w.load(rp, v0, V);
        uint2 adj = make_uint2(0, (uint32_t)v0);
        if (e0 + lane < e1) adj = rr.adj[e0 + lane];
        if (rr.mask) w.mask(allowed);
        if (e1 > e0) {   // uniform
            // the touched tokens are taken out of the staged window, adjusted and
            // folded one a lane; the rest folds below
            w.stage(stage);
            wave_sync();
            for (int e = e0; e < e1; e += 64) {
                const uint2 a = adj;
                if (e + 64 + lane < e1) adj = rr.adj[e + 64 + lane];
                const int v = (int)(a.y & ~kSeen);
                float f[1] = {-INFINITY};
                if (e + lane < e1) {
                    T& z = stage[v - v0];
                    f[0] = adjust(value(z), a, rr.rec);
                    z = minus_inf<T>();
                }
                wt.fold<1, 1>(f, v);
            }
            wave_sync();
            w.fetch(stage);
        }
#pragma unroll
        for (int j = 0; j < W::kBatch; ++j) {
            float f[8];
            w.raw[j].unpack(f);
            wt.fold<0, 8>(f, v0 + j * 512 + lane * 8);
        }
    }

    Top t = wt.top();
    // the workgroup's partial: its waves' in order, by the first wave
    auto write = [&]() {
        if (lane == 0) wtop[wave] = t;
        __syncthreads();
        if (wave != 0) return;
        t = lane < kVocabThreads / 64 ? wtop[lane] : top_empty();
#pragma unroll
        for (int off = 1; off < kVocabThreads / 64; off <<= 1) {
            Top o;
            o.m = __shfl_xor(t.m, off, 64);
            o.mL = __shfl_xor(t.mL, off, 64);
            o.s = __shfl_xor(t.s, off, 64);
            o.idx = __shfl_xor(t.idx, off, 64);
            t = top_merge(t, o);
        }
        if (lane == 0) {
            part[(size_t)row * nsplit + k] = top_pack(t);
            if (conf) predict(t, conf + row, argmax + row);
        }
    };
    // whether some wave met a maximum, and whether anything is allowed
    if (lane == 0) s_met[wave] = (t.m > kLowest ? 1 : 0) | (any ? 2 : 0);
    write();
    int met = 0;
#pragma unroll
    for (int w = 0; w < kVocabThreads / 64; ++w) met |= s_met[w];
    if (met & 1) return;   // uniform
    t = top_empty();
    if (met & 2) {
        const float each = __builtin_amdgcn_exp2f(fmaf(kLowest, kLog2e, -scaled_ref(kLowest)));
        auto take = [&](int v, float z) {
            if (z > -INFINITY) t = Top{kLowest, scaled_ref(kLowest), t.s + each, min(t.idx, v)};
        };
        i = 0;
        for (int v0 = first; v0 < V; v0 += stride, ++i) {
            const int end = min(v0 + W::kTokens, V);
            for (int v = v0 + lane; v < end; v += 64)
                if ((rr.allowed(v & ~7) >> (v & 7) & 1) &&
                    !(rr.bits && rr.bits[v >> 3] >> (v & 7) & 1))
                    take(v, value(rp[v]));
            const int e1 = __builtin_amdgcn_readlane(entries, kMaxWindows + i);
            for (int e = __builtin_amdgcn_readlane(entries, i) + lane; e < e1; e += 64) {
                const uint2 a = rr.adj[e];
                const int v = (int)(a.y & ~kSeen);
                if (rr.allowed(v & ~7) >> (v & 7) & 1) take(v, adjust(value(rp[v]), a, rr.rec));
            }
        }
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) {
            t.s += __shfl_xor(t.s, off, 64);
            t.idx = min(t.idx, __shfl_xor(t.idx, off, 64));
        }
        if (t.s > 0.f) t = Top{kLowest, scaled_ref(kLowest), t.s, t.idx};
    }
    __syncthreads();
    write();
}

// (p, x_hat) of every live row from its partials, two or more, as the update merges
// them.  (Rows of one partial are predicted by the pass itself.)
constexpr int kPredictThreads = 256;

__global__ void __launch_bounds__(kPredictThreads)
predict_kernel(const float4* __restrict__ part, int nsplit, PackView pv, int row_cap,
               float* __restrict__ conf, int32_t* __restrict__ argmax) {
    const int row = blockIdx.x * kPredictThreads + threadIdx.x;
    if (row >= row_cap) return;
    // loaded together with the row's request
    const float4 first = part[(size_t)row * nsplit], second = part[(size_t)row * nsplit + 1];
    if (pv.row_req[row] < 0) return;
    Top t = top_merge(top_unpack(first), top_unpack(second));
    for (int k = 2; k < nsplit; ++k)
        t = top_merge(t, top_unpack(part[(size_t)row * nsplit + k]));
    predict(t, conf + row, argmax + row);
}

template <typename T>
__global__ void __launch_bounds__(kVocabThreads)
logits_rules_kernel(const T* logits, T* out, int V, int nsplit, PackView pv,
                    fb_logit_rules rules, RuleView rv, int mask_words) {
    using W = Window<T>;
    __shared__ __attribute__((aligned(16))) typename W::Stage stages[kVocabThreads / 64];
    const int row = blockIdx.x / nsplit;
    const int k = blockIdx.x % nsplit;
    const int req = pv.row_req[row];
    if (req < 0) return;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    RowRules rr = row_rules(rules, rv, pv, row, req, mask_words);
    if (rr.none) rr.bits = nullptr;
    const T* rp = logits + (size_t)row * V;
    T* wp = out + (size_t)row * V;
    const int first = k * W::kPiece + wave * W::kTokens;
    const int stride = nsplit * W::kPiece;
    const uint32_t entries = window_entries<T>(rr, first, stride, V);
    typename W::Stage& stage = stages[wave];

    typename W::Allowed allowed, next;
    if (rr.mask) next.load(rr.mask, first, V);
    int i = 0;
    for (int v0 = first; v0 < V; v0 += stride, ++i) {
        bool some = !rr.none;
        if (rr.mask) {    // uniform, and a window ahead as above
            allowed = next;
            some &= allowed.some();
            if (v0 + stride < V) next.load(rr.mask, v0 + stride, V);
        }
        const int e0 = __builtin_amdgcn_readlane(entries, i);
        const int e1 = some ? __builtin_amdgcn_readlane(entries, kMaxWindows + i) : e0;
        W w;
        if (some) w.load(rp, v0, V);
        else w.fill();
        uint2 adj = make_uint2(0, (uint32_t)v0);
        if (e0 + lane < e1) adj = rr.adj[e0 + lane];
        if (some && rr.mask) w.mask(allowed);
        if (e1 > e0) {   // uniform
            w.stage(stage);
            wave_sync();
            for (int e = e0; e < e1; e += 64) {
                const uint2 a = adj;
                if (e + 64 + lane < e1) adj = rr.adj[e + 64 + lane];
                if (e + lane < e1) {
                    T& z = stage[(int)(a.y & ~kSeen) - v0];
                    const float f = adjust(value(z), a, rr.rec);
                    if constexpr (sizeof(T) == 2) z = __builtin_bit_cast(uint16_t, (__bf16)f);
                    else z = f;
                }
            }
            wave_sync();
            w.fetch(stage);
        }
#pragma unroll
        for (int j = 0; j < W::kBatch; ++j) {
            const int v = v0 + j * 512 + lane * 8;
            if (v < V) w.raw[j].store(wp + v, V - v);
        }
    }
}

// Slices of the vocabulary per request: workgroups for about every CU, each of
// at least 8192 tokens (a workgroup reads the whole prefix).
int build_slices(int B, int V, int cu_count) {
    int n = cu_count / B;
    if (n > V / 8192) n = V / 8192;
    return n < 1 ? 1 : n > 32 ? 32 : n;
}

constexpr int kBuildLds = 156 * 1024;

}  // namespace

RulesSizes rules_sizes(const fb_pack* pack, int V) {
    RulesSizes z{};
    z.words = (V + 127) / 128 * 4;
    z.spans = (V + kSpan - 1) / kSpan;
    const size_t B = pack->B;
    z.off_bits = (B * sizeof(float2) + 255) / 256 * 256;
    z.off_spans = z.off_bits + (B * z.words * 4 + 255) / 256 * 256;
    z.off_adj = z.off_spans + (B * z.spans * sizeof(uint2) + 255) / 256 * 256;
    z.total = z.off_adj + B * z.words * 32 * sizeof(uint2);
    return z;
}

hipError_t launch_rules_build(const fb_logit_rules* rules, const fb_req_state* st,
                              const int32_t* tokens, int T_max, int V, const fb_pack* pack,
                              void* ws, const RulesSizes& z, int cu_count, hipStream_t stream) {
    const int n = build_slices(pack->B, V, cu_count);
    const int slice = ((V + n - 1) / n + kSlice - 1) / kSlice * kSlice;
    const int slices = (V + slice - 1) / slice;
    const int words = ((V < slice ? V : slice) + 31) / 32;
    // counts for as many tokens as a prefix and its biases can touch, at most
    // what is left of the LDS
    long long counts = (kBuildLds - words * 8) / 4;
    const long long most = (long long)T_max + rules->n_bias;
    if (counts > most) counts = most;
    if (counts > words * 32) counts = words * 32;
    hipLaunchKernelGGL(rules_build_kernel, dim3(pack->B * slices), dim3(kBuildThreads),
                       (size_t)words * 8 + (size_t)counts * 4, stream, *rules, st, tokens, T_max, V,
                       pack_view(pack), rule_view(z, ws), slice, slices, (int)counts);
    return hipGetLastError();
}

hipError_t launch_vocab_rules(const void* logits, int V, int dtype, const fb_pack* pack,
                              const fb_logit_rules* rules, const void* rules_ws,
                              const RulesSizes& rz, void* upd_ws, const UpdateSizes& uz,
                              float* conf, int32_t* argmax, hipStream_t stream) {
    PackView pv = pack_view(pack);
    const RuleView rv = rule_view(rz, const_cast<void*>(rules_ws));
    float4* part = static_cast<float4*>(upd_ws);
    // one partial a row (V up to 16384): the pass predicts, a launch less
    const bool one = uz.nsplit == 1;
    auto go = [&](auto zero) {
        using T = decltype(zero);
        if (!walk_fits<T>(V, uz.nsplit)) return hipErrorInvalidConfiguration;
        hipLaunchKernelGGL(vocab_rules_kernel<T>,
                           dim3((unsigned)pack->row_cap * (unsigned)uz.nsplit),
                           dim3(kVocabThreads), 0, stream, static_cast<const T*>(logits), V,
                           uz.nsplit, pv, *rules, rv, (V + 31) / 32, part,
                           one ? conf : nullptr, one ? argmax : nullptr);
        return hipGetLastError();
    };
    const hipError_t e = dtype == FB_BF16 ? go(uint16_t()) : go(float());
    if (e != hipSuccess || !conf || one) return e;
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
        if (!walk_fits<T>(V, uz.nsplit)) return hipErrorInvalidConfiguration;
        hipLaunchKernelGGL(logits_rules_kernel<T>,
                           dim3((unsigned)pack->row_cap * (unsigned)uz.nsplit),
                           dim3(kVocabThreads), 0, stream, static_cast<const T*>(logits),
                           static_cast<T*>(out), V, uz.nsplit, pack_view(pack), *rules, rv,
                           (V + 31) / 32);
        return hipGetLastError();
    };
    return dtype == FB_BF16 ? go(uint16_t()) : go(float());
}

}  // namespace fb
