// Windowed block-causal attention (Sec. 4.1; Eq. 5 per packed row) over a
// quantised cache: keys and values in E2M1 or E4M3 with a power-of-two scale per
// 32 channels.
//
// Such a value has at most four significant bits and a power of two, so bf16
// holds it exactly: the products run on v_mfma_f32_32x32x16_bf16 and add up in
// float32.  (The instructions that multiply codes and scales directly were
// measured too: their sums are off by up to 2^-12.5 of the sum of the products'
// magnitudes, where a float32 addition is off by 2^-24.)
//
// Work.  A unit is (request, KV head, group of query rows): the request's rows
// are its window's (position, head of the KV head's group) pairs, position
// major, so a group may span several blocks, which share one pass over the
// prefix; the blocks differ in their last keys only, by a mask per row.  The
// units' key tiles (32 keys), with a few more for a unit's start and end, form
// one line, cut into equal shares, one for each workgroup: no list is made, a
// workgroup finds its place in the line from the requests' windows alone.  A
// unit that a cut divides is merged afterwards.
//   mx_wide_kernel   groups of 128 rows, 32 to a wave; the waves share a key
//                    tile, which they turn into bf16 in LDS.  Bound by the
//                    issue of matrix and vector instructions together: 87
//                    vector instructions (16 of them conversions of codes) to
//                    16 products, the matrix cores busy 46% of the time.  256
//                    requests, 20416 rows over 128 .. 8192 keys, 4 bits: 757 ..
//                    827 us over several boxes, 810 .. 890 TFLOP/s; 8 requests
//                    over 16K .. 32K keys, 8 bits: 421 .. 464 us, 860 .. 950
//                    TFLOP/s
//   mx_few_kernel    requests of at most 32 rows (single tokens among them):
//                    the waves take key tiles in turn, each for all rows, and
//                    join at the end; no tile is shared, so no wave waits.  Bound
//                    by memory where the contexts are long: 64 tokens over 1K ..
//                    32K keys, 639 MB in 4 bits, 141 us, 4.5 TB/s; in 8 bits 1.2
//                    GB in 236 us, 5.2 TB/s
//   mx_merge_kernel  the divided units' pieces, by their log-sum-exps (6 .. 15 us)
//
// S^T = K Q^T leaves in lane l the scores of query row l % 32 and keys
// 8 (x / 4) + 4 (l / 32) + x % 4, x < 16.  The product O^T += V^T P^T takes the
// keys in that order: V is read transposed (ds_read_b64_tr_b16, four keys at a
// time), so P goes from one product into the other without an exchange.
// fp32: queries and weights are split into three bf16 parts, which hold all 24
// bits, so there are three products each.
#include <type_traits>
#include <utility>

#include "cache.h"

namespace fb {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;
constexpr int kKeys = 32;              // of a tile
constexpr int kWideRows = 128, kFewRows = 32;
// Caches that the page table lets hold at most so many keys are walked by one workgroup a
// unit, with no merge, where there are no more units than workgroups.  Divided and whole: 8
// heads, one token, 250 keys 11.9 and 10.1 us, 500 keys 16.6 and 12.1, 1024 keys 18.3 and
// 16.4, 1240 keys 17.7 and 17.2, 1500 keys 18.1 and 18.9.  14 units of 128 rows over heads of
// 64 in 8 bits: 700 keys 19.6 and 18.9, 960 keys 19.5 and 22.5; in float32, whose crossing
// lies lower than this bound, 29.3 and 31.3, 29.3 and 38.0.
constexpr int kWideWholeKeys = 1024, kFewWholeKeys = 1280;
// what a unit's start and end cost, in tiles: of 128 rows, of 32
// (256 requests of windows: 4 780 us, 9 763, 14 782; 64 single tokens: 14 143, 20 142, 40 147)
constexpr int kWideStart = 9, kFewStart = 20;
constexpr int kLeastShare = 8;         // of a workgroup, in tiles
// Workgroups of a CU: as many as their registers let it hold at once.  (Heads of 32 with
// one fewer: 8 long requests 188 us, 180 so; 64 single tokens in 8 bits 76, 66.)
constexpr int per_cu(int D, bool bf16, int rows) {
    return !bf16 ? 2 : rows == kWideRows ? (D == 32 ? 4 : 3) : (D == 32 ? 3 : 2);
}
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kRescaleSlack = 8.0f;  // the running maximum may lag by 2^8

struct MxArgs {
    const void* q;
    void* out;
    int32_t* head;     // [0]: workgroups with a share
    int32_t* rec;      // [wgs][8]: the unit whose first piece the workgroup made
    float* part_o;     // [2 wgs][rows][D]
    float* part_lse;   // [2 wgs][rows]
    int Hq, Hkv, g, bl, B, W_max, row_cap, wgs, ps_shift, max_pages, num_pages;
    int max_keys;      // that the page table reaches
    int whole;         // no unit is divided
    int short_line;    // the line of a full pack has fewer than 2^31 places
    float scale_log2, slack;   // slack: of the running maximum, as a score
};
// What a kernel only reads, apart from its other arguments, so that the compiler may
// use scalar loads.
#define MX_CACHE_PARAMS                                                                  \
    const uint8_t *__restrict__ kc, const uint8_t *__restrict__ ks,                      \
        const uint8_t *__restrict__ vc, const uint8_t *__restrict__ vs,                  \
        const int32_t *__restrict__ page_table
enum RecField { kRRow0 = 0, kRHead, kRFirst, kRRows, kRPieces, kRecInts = 8 };

// ----------------------------------------------------------- the shares ---
// The same value in every lane of the wave, said to the compiler.
__device__ inline int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ inline long long uniform(long long x) {
    return (long long)((uint64_t)(uint32_t)uniform((int)(x >> 32)) << 32 |
                       (uint32_t)uniform((int)x));
}

// A quotient of numbers that are not negative; most fit 32 bits, where a division
// takes a third of the time.
__device__ inline long long div_of(long long x, long long y) {
    return ((x | y) >> 31) == 0 ? (long long)((uint32_t)x / (uint32_t)y) : x / y;
}

// A request's part of the line.
struct Req {
    int b, row0, o, rows, groups;
    long long len;     // of one KV head (65536 groups over 1M keys pass 2^31)
};

// A piece of a unit: key tiles [k0, k1) of kt.
struct Piece {
    int head, group, kt, k0, k1;
    int first, more;   // partial slot (-1: the whole unit), pieces of a unit that begins here
};

template <int ROWS>
constexpr int kStartOf = ROWS == kWideRows ? kWideStart : kFewStart;

template <int ROWS>
__device__ inline int group_tiles(const MxArgs& a, const Req& r, int group) {
    const int last = min((group + 1) * ROWS, r.rows) - 1;
    return (r.o + (last / (a.g * a.bl) + 1) * a.bl + kKeys - 1) / kKeys;
}

// Request b; `report`: an unreachable page is recorded.
template <int ROWS>
__device__ inline Req request(const MxArgs& a, const PackView& pv, int b, bool report) {
    Req r{b, 0, 0, 0, 0, 0};
    const int w = pv.req_w[b], row0 = pv.req_row0[b];
    if (w <= 0 || w > a.W_max || row0 < 0 || row0 > a.row_cap - w * a.bl) return r;
    r.row0 = row0;
    r.o = pv.row_pos[row0];
    if (r.o < 0 || (long long)r.o + (long long)w * a.bl > a.max_keys) {
        if (report) record_error(pv.hdr, b, FB_DERR_PAGE);
        return r;
    }
    r.rows = w * a.bl * a.g;
    r.groups = (r.rows + ROWS - 1) / ROWS;
    for (int i = 0; i < r.groups; ++i) r.len += group_tiles<ROWS>(a, r, i) + kStartOf<ROWS>;
    return r;
}

// The walk of a workgroup along its share, for units of ROWS query rows.
template <int ROWS>
struct Walk {
    static constexpr int kStart = kStartOf<ROWS>;
    long long at, end;    // place in the line of the present unit, end of the share
    long long share;
    int index, head, group, whole;
    int skip;             // place of the share's start in its first unit
    Req r;

    // The cut at place x of a unit of kt tiles, in its tiles: what is left on
    // either side is worth a piece (a 32nd of a share; an eighth costs 2%).
    __device__ inline int least() const { return whole ? 1 << 30 : (int)max(2LL, share / 32); }
    __device__ inline int cut(long long x, int kt) const {
        const int k = (int)max(0LL, min(x - kStart, (long long)kt)), m = least();
        return k < m ? 0 : kt - k < m ? kt : k;
    }

    // Sums of `mine` over the threads up to this one and over all.
    template <typename Int>
    __device__ static inline void scan(Int mine, Int& sum, Int& total) {
        __shared__ Int wave_sum[kThreads / 64];
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        sum = mine;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const Int x = __shfl_up(sum, off, 64);
            if (lane >= off) sum += x;
        }
        if (lane == 63) wave_sum[wave] = sum;
        __syncthreads();
        total = 0;
#pragma unroll
        for (int i = 0; i < kThreads / 64; ++i) {
            if (i < wave) sum += wave_sum[i];
            total += wave_sum[i];
        }
    }

    // All threads of the workgroup; false if it has no share.
    __device__ bool begin(const MxArgs& a, const PackView& pv) {
        __shared__ Req found;
        __shared__ long long found_at;
        whole = a.whole;
        const int tid = threadIdx.x;
        const int per = (a.B + kThreads - 1) / kThreads;
        Req mine_r{};
        long long mine = 0;
        for (int b = tid * per; b < min((tid + 1) * per, a.B); ++b) {
            mine_r = request<ROWS>(a, pv, b, blockIdx.x == 0);
            mine += a.Hkv * mine_r.len;
        }
        long long sum, total;
        if (a.short_line) {
            int s, t;
            scan((int)mine, s, t);
            sum = s, total = uniform(t);
        } else {
            scan(mine, sum, total);
            total = uniform(total);
        }
        share = max(div_of(total + a.wgs - 1, a.wgs), (long long)(kLeastShare + kStart));
        const int busy = (int)div_of(total + share - 1, share);
        // Neighbours in the line read the same keys, so they belong on one XCD: workgroups
        // go to the eight in turn (8 long requests: 426 us, 429 without; 256 requests: 757,
        // 758).
        const int each = (busy + 7) / 8;
        index = blockIdx.x % 8 * each + blockIdx.x / 8;
        if (blockIdx.x == 0 && tid == 0) a.head[0] = busy;
        if (blockIdx.x / 8 >= each || index >= busy) return false;
        const long long p = index * share;
        end = p + share;
        if (sum > p && sum - mine <= p) {
            // the request that holds p is one of this thread's
            long long before = sum - mine;
            for (int b = tid * per; per > 1; ++b) {
                mine_r = request<ROWS>(a, pv, b, false);
                const long long len = a.Hkv * mine_r.len;
                if (before + len > p) break;
                before += len;
            }
            found = mine_r;
            found_at = before;
        }
        __syncthreads();
        r.b = uniform(found.b), r.row0 = uniform(found.row0), r.o = uniform(found.o);
        r.rows = uniform(found.rows), r.groups = uniform(found.groups), r.len = uniform(found.len);
        at = uniform(found_at);
        head = (int)div_of(p - at, r.len);
        at += head * r.len;
        group = 0;
        for (;;) {
            const int len = group_tiles<ROWS>(a, r, group) + kStart;
            if (at + len > p) break;
            at += len;
            ++group;
        }
        skip = (int)(p - at);
        return true;
    }

    // The next piece of the share; false past its last one.
    __device__ bool next(const MxArgs& a, const PackView& pv, Piece& w) {
        for (;;) {
            if (at >= end) return false;
            while (r.len == 0 || head >= a.Hkv) {
                int b = r.b + 1;
                if (r.len == 0) {
                    // (one that has no rows: the next that has, 64 at a look)
                    const int lane = threadIdx.x & 63;
                    uint64_t live = 0;
                    for (; b < a.B; b += 64) {
                        live = __ballot(b + lane < a.B && pv.req_w[min(b + lane, a.B - 1)] > 0);
                        if (live) break;
                    }
                    if (live) b += __ffsll((unsigned long long)live) - 1;
                }
                if (b >= a.B) return false;
                r = request<ROWS>(a, pv, uniform(b), false);
                head = 0;
            }
            w.head = head;
            w.group = group;
            w.kt = group_tiles<ROWS>(a, r, group);
            w.k0 = cut(skip, w.kt);
            const int len = w.kt + kStart;
            w.k1 = end - at >= len ? w.kt : cut(end - at, w.kt);
            w.first = -1;
            w.more = 0;
            if (w.k0 > 0) w.first = 2 * index;
            else if (w.k1 < w.kt && w.k1 > 0) {
                // cuts at m .. kt - m tiles of this unit, this share's end the first
                const long long last = div_of(at + kStart + w.kt - least(), share);
                w.first = 2 * index + 1;
                w.more = (int)(last - index) + 1;
            }
            at += len;
            skip = 0;
            if (++group == r.groups) group = 0, ++head;
            if (w.k0 < w.k1) return true;
        }
    }
};

// ------------------------------------------------------------- operands ---
// The three bf16 parts of a float: two cut off, so that each rest is exact and
// the third holds what is left.
__device__ inline void split3(float x, __bf16 (&p)[3]) {
    const uint32_t hi = __float_as_uint(x) & 0xffff0000u;
    const float r = x - __uint_as_float(hi);
    const uint32_t mid = __float_as_uint(r) & 0xffff0000u;
    p[0] = __builtin_bit_cast(__bf16, (uint16_t)(hi >> 16));
    p[1] = __builtin_bit_cast(__bf16, (uint16_t)(mid >> 16));
    p[2] = (__bf16)(r - __uint_as_float(mid));
}

template <typename T>
constexpr int kParts = sizeof(T) == 2 ? 1 : 3;

// Eight query elements as an operand; zeros where there is no row.
__device__ inline void query8(const uint16_t* p, bool ok, bf16x8 (&f)[1]) {
    f[0] = ok ? *reinterpret_cast<const bf16x8*>(p) : bf16x8{};
}
__device__ inline void query8(const float* p, bool ok, bf16x8 (&f)[3]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        __bf16 s[3];
        split3(ok ? p[i] : 0.f, s);
#pragma unroll
        for (int k = 0; k < 3; ++k) f[k][i] = s[k];
    }
}

__device__ inline void store4(uint16_t* p, float a, float b, float c, float d) {
    const __bf16 v[4] = {(__bf16)a, (__bf16)b, (__bf16)c, (__bf16)d};
    *reinterpret_cast<u32x2*>(p) = *reinterpret_cast<const u32x2*>(v);
}
__device__ inline void store4(float* p, float a, float b, float c, float d) {
    *reinterpret_cast<float4*>(p) = make_float4(a, b, c, d);
}

// Where the 16-byte piece c of row r of a 32-key tile lies in LDS, in elements.
// Rows are padded where tiles are shared, so that the pieces of a row lie at fixed
// distances: sixteen rows' same piece (key operands; a read goes sixteen lanes a
// step) and four neighbouring rows' same 64 bytes (value operands, read transposed)
// then lie in different banks.
template <int D>
struct KeyRows {
    static constexpr int kPitch = D + 8;
    __device__ static inline int at(int r, int c) { return r * kPitch + c * 8; }
};
template <int D>
struct ValueRows {
    static constexpr int kPitch = D == 32 ? 32 : D + 32;
    __device__ static inline int at(int r, int c) { return r * kPitch + c * 8; }
};
// A wave's own values are stored by sixteen rows' same piece too, for which no
// padding serves both: pieces change places by their row's number instead.
template <int D>
struct TurnedRows {
    __device__ static inline int at(int r, int c) {
        const int turn = D == 128 ? (r & 3) << 2 | ((r >> 2) & 3)
                       : D == 64 ? ((r >> 1) & 1) << 2 | ((r >> 2) & 3) : (r >> 2) & 3;
        return r * D + (c ^ turn) * 8;
    }
};

// Values of column l % 16 and four neighbouring rows: lane i of each sixteen
// gives the address of row i / 4, columns 4 (i % 4) ...
__device__ inline s16x4 read_tr(const uint16_t* p) {
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        (__attribute__((address_space(3))) s16x4*)(p));
}

// max over the lanes l and l + 32, which share a query row
__device__ inline float half_max(float x) {
    const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false,
                                                     false);
    float r;   // (plain v_max: the compiler would first make both sides canonical)
    asm("v_max_f32 %0, %1, %2" : "=v"(r) : "v"(__uint_as_float(sw[0])), "v"(__uint_as_float(sw[1])));
    return r;
}

typedef const __attribute__((address_space(1))) uint8_t* GlobalBytes;

// N bytes of codes as dwords.
template <int N>
__device__ inline void load_codes(GlobalBytes p, uint32_t* q) {
#define MX_AT(type, at) (*(const __attribute__((address_space(1))) type*)(p + (at)))
    if constexpr (N == 2) q[0] = MX_AT(uint16_t, 0);
    else if constexpr (N == 4) q[0] = MX_AT(uint32_t, 0);
    else if constexpr (N == 8) {
        const u32x2 x = MX_AT(u32x2, 0);
        q[0] = x[0], q[1] = x[1];
    } else {
#pragma unroll
        for (int j = 0; j < N / 16; ++j) {
            const u32x4 x = MX_AT(u32x4, 16 * j);
#pragma unroll
            for (int i = 0; i < 4; ++i) q[4 * j + i] = x[i];
        }
    }
#undef MX_AT
}

// Eight values from their codes (BITS / 4 dwords).
template <int BITS>
__device__ inline u32x4 eight_values(const uint32_t* q, float scale) {
    bf16x2 v[4];
#pragma unroll
    for (int i = 0; i < BITS / 4; ++i) mx_dword<BITS>(q[i], scale, v + i * (16 / BITS));
    return u32x4{__builtin_bit_cast(uint32_t, v[0]), __builtin_bit_cast(uint32_t, v[1]),
                 __builtin_bit_cast(uint32_t, v[2]), __builtin_bit_cast(uint32_t, v[3])};
}

// Zeros in place of the infinite values of a dword of codes; bits of them where there were
// any.  All codes at once: a magnitude with the sign's bit set, less the first infinite one,
// keeps that bit where it is as large.
template <int BITS>
__device__ inline uint32_t drop_infinite(uint32_t& q, uint32_t scale) {
    constexpr uint32_t kOnes = BITS == 4 ? 0x11111111u : 0x01010101u, kSigns = kOnes << (BITS - 1);
    const uint32_t high = ((q | kSigns) - mx_infinite<BITS>(scale) * kOnes) & kSigns;
    q &= ~((high << 1) - (high >> (BITS - 1)));
    return high;
}

// The lane's number, formed anew where it is asked for: what follows from it behind the
// tiles' loop would else be formed in front of it and take the loop's registers (windows
// over 8 bits 824 us, 836 so).
__device__ inline int late_lane() {
    int lane;
    asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=&v"(lane));
    return lane;
}

// --------------------------------------------------------- online softmax ---
// A wave's 32 query rows: lane l has row l % 32, half of its scores and of its
// result's channels.
template <int D, typename T>
struct Rows {
    static constexpr int KK = D / 16, DT = D / 32, NP = kParts<T>;
    bf16x8 qf[KK][NP];
    floatx16 o[DT];
    float m_sub;      // what the scores are taken relative to, log2 domain
    float thr;        // score above which it moves; -inf: no score above -inf yet
    float l;          // this lane's share of the denominator
    int seen;         // keys that the row sees

    __device__ inline void clear() {
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) o[dt] = floatx16{};
        m_sub = l = 0.f;
        thr = -INFINITY;
    }

    // Keys from `left` on are not seen.
    __device__ inline void mask(floatx16& s, int left) {
        const int h = (threadIdx.x >> 5) & 1;
#pragma unroll
        for (int x = 0; x < 16; ++x)
            if (8 * (x >> 2) + 4 * h + (x & 3) >= left) s[x] = -INFINITY;
    }

    // The running maximum moves when a tile's passes it by 2^8, so that results are
    // seldom rescaled; weights are up to 2^8 then.
    __device__ inline void rescale(float mx, float scale, float slack) {
        const bool need = mx > thr;
        if (__any(need)) {
            const float m_new = need ? mx * scale : m_sub;
            // (the first time there is nothing to scale, and 2^(0 - m) may pass the range)
            const float alpha = thr == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m_sub - m_new);
#pragma unroll
            for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                for (int x = 0; x < 16; ++x) o[dt][x] *= alpha;
            l *= alpha;
            m_sub = m_new;
            if (need) thr = mx + slack;
        }
    }

    // Scores x0 .. x0 + N - 1 into weights.  bf16: they are rounded for the product, as over a
    // bf16 cache, and the denominator sums the rounded ones, so that the rounding cancels where
    // values agree.  (Results are off from float64 by 2.1e-3 of their norm over the measured
    // batches, where their own rounding alone makes 1.66e-3; weights in two parts would be
    // half as many products again.)
    template <int N>
    __device__ inline void weights(const floatx16& s, int x0, float scale, bf16x8 (&pb)[2][NP]) {
#pragma unroll
        for (int x = x0; x < x0 + N; x += 2) {
            float p[2];
#pragma unroll
            for (int i = 0; i < 2; ++i)
                p[i] = __builtin_amdgcn_exp2f(fmaf(s[x + i], scale, -m_sub));
            if constexpr (NP == 1) {
                const bf16x2 pr = {(__bf16)p[0], (__bf16)p[1]};
                const bf16x2 one = {(__bf16)1.0f, (__bf16)1.0f};
                pb[x >> 3][0][x & 7] = pr[0];
                pb[x >> 3][0][(x & 7) + 1] = pr[1];
                l = __builtin_amdgcn_fdot2_f32_bf16(pr, one, l, false);
            } else {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    __bf16 part[3];
                    split3(p[i], part);
#pragma unroll
                    for (int k = 0; k < 3; ++k) pb[x >> 3][k][(x & 7) + i] = part[k];
                    l += p[i];
                }
            }
        }
    }

    // A whole tile's scores into weights, with the running statistics.
    __device__ inline void softmax(floatx16& s, float scale, float slack, bf16x8 (&pb)[2][NP]) {
        float mx = s[0];
#pragma unroll
        for (int x = 1; x < 16; ++x) mx = fmaxf(mx, s[x]);
        rescale(half_max(mx), scale, slack);
        weights<16>(s, 0, scale, pb);
    }

    // The operand V^T of keys 16 t .. 16 t + 15 and channels 32 dt ..: slots 8 h .. hold
    // keys 16 t + 4 h .. + 3, then 16 t + 8 + 4 h .. + 3.
    template <typename L>
    __device__ static inline bf16x8 values(const uint16_t* vt, int t, int dt) {
        const int lane = threadIdx.x & 63, h = lane >> 5;
        const int row = 16 * t + 4 * h + (lane & 15) / 4;
        const int piece = dt * 4 + (lane & 16) / 8 + (lane & 3) / 2, in = (lane & 1) * 4;
        union {
            s16x4 part[2];
            bf16x8 v;
        } f;
        f.part[0] = read_tr(vt + L::at(row, piece) + in);
        f.part[1] = read_tr(vt + L::at(row + 8, piece) + in);
        return f.v;
    }
    __device__ inline void add(const bf16x8& v, int dt, const bf16x8 (&p)[NP]) {
#pragma unroll
        for (int k = 0; k < NP; ++k)
            o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, p[k], o[dt], 0, 0, 0);
    }

    // Values of NaN scales and infinite ones in a tile that not every row sees were staged as
    // zeros: the rows that do see them get their NaN or infinity here.
    template <int BITS>
    __device__ inline void spoil(const MxArgs& a, const uint8_t* vc, const uint8_t* vs,
                                 const int32_t* pt, int head, int key0, int end) {
        const int h = late_lane() >> 5;
        for (int key = key0; key < end; ++key) {
            const int page = pt[key >> a.ps_shift];
            if ((unsigned)page >= (unsigned)a.num_pages) continue;
            const size_t slot = (((size_t)page * a.Hkv + head) << a.ps_shift) +
                                (key & ((1 << a.ps_shift) - 1));
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) {
                const uint32_t s = vs[slot * DT + dt];
                if (s <= kMxHighest<BITS> || key >= seen) continue;
#pragma unroll
                for (int x = 0; x < 16; x += 4) {      // four neighbouring channels
                    const uint8_t* at = vc + (slot * D + dt * 32 + 2 * x + 4 * h) * BITS / 8;
                    const uint32_t four = BITS == 4 ? *reinterpret_cast<const uint16_t*>(at)
                                                    : *reinterpret_cast<const uint32_t*>(at);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t code = four >> i * BITS & ((1u << BITS) - 1);
                        const uint32_t mag = code & ((1u << (BITS - 1)) - 1);
                        if (s == 255 || (BITS == 8 && mag == 127))
                            o[dt][x + i] = __uint_as_float(0x7fc00000u);
                        else if (mag >= mx_infinite<BITS>(s))
                            o[dt][x + i] += mag == code ? INFINITY : -INFINITY;
                    }
                    __builtin_amdgcn_sched_barrier(0);   // (rare: registers count, not time)
                }
            }
        }
    }

    // The rows' results, or their piece's.
    __device__ inline void store(const MxArgs& a, const Req& r, const Piece& w, int row0,
                                 int row_stride) {
        const int lane = late_lane(), h = lane >> 5, r_local = row0 + (lane & 31);
        const float sum = l + __shfl_xor(l, 32, 64);
        const int row = w.group * row_stride + r_local;
        if (row >= r.rows) return;
        // a piece that the row sees nothing of adds nothing to it
        const float inv = w.first >= 0 && sum == 0.f ? 0.f : 1.0f / sum;
        T* dst = static_cast<T*>(a.out) +
                 ((size_t)(r.row0 + row / a.g) * a.Hq + w.head * a.g + row % a.g) * D;
        const size_t slot = (size_t)(w.first < 0 ? 0 : w.first) * row_stride + r_local;
        float* po = a.part_o + slot * D;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int x = 0; x < 16; x += 4) {
                const int d = dt * 32 + x * 2 + h * 4;
                const float v0 = o[dt][x] * inv, v1 = o[dt][x + 1] * inv;
                const float v2 = o[dt][x + 2] * inv, v3 = o[dt][x + 3] * inv;
                if (w.first < 0) store4(dst + d, v0, v1, v2, v3);
                else store4(po + d, v0, v1, v2, v3);
            }
        if (w.first >= 0 && h == 0) a.part_lse[slot] = m_sub + __log2f(sum);
    }
};

__device__ inline void store_record(const MxArgs& a, int index, const Req& r, const Piece& w,
                                    int rows) {
    int32_t* rec = a.rec + (size_t)index * kRecInts;
    rec[kRRow0] = r.row0;
    rec[kRHead] = w.head;
    rec[kRFirst] = w.group * rows;
    rec[kRRows] = min(rows, r.rows - w.group * rows);
    rec[kRPieces] = w.more;
}

// ------------------------------------------------------------- many rows ---
// A step takes a tile's scores, turns them into weights and adds its values; between
// the products of the second half, the codes of the next tile, loaded a step before,
// are turned into bf16 for the other stage.  The three workgroups of a CU have their
// vector and matrix phases beside each other's; taking the next tile's scores beside
// this one's weights within a wave needs registers for two workgroups only and was
// slower (256 requests 850 us, 820 so with two, 780 with three), with 64 keys a step
// too.  The order is held by scheduling barriers: left to the compiler it cost 1-2%.
// PAGED: a page holds a tile, so its loads share one scalar base.
// FULL: every wave of a unit has query rows.
template <int D, int BITS, typename T, bool PAGED, bool FULL>
__global__ void __launch_bounds__(kThreads, per_cu(D, sizeof(T) == 2, kWideRows))
mx_wide_kernel(MxArgs a, MX_CACHE_PARAMS, PackView pv) {
    constexpr int EL = D / 8;             // elements of a thread's run: 8 threads to a key
    constexpr int CB = EL * BITS / 8;     // their code bytes: 2, 4, 8 or 16
    constexpr int CW = (CB + 3) / 4;
    constexpr int KK = D / 16, DT = D / 32, NP = kParts<T>;
    constexpr int kRowBytes = D * BITS / 8;
    using KR = KeyRows<D>;
    using VR = ValueRows<D>;
    using X = Rows<D, T>;
    __shared__ __attribute__((aligned(16))) uint16_t lds_k[2][kKeys * KR::kPitch];
    __shared__ __attribute__((aligned(16))) uint16_t lds_v[2][kKeys * VR::kPitch];

    Walk<kWideRows> walk;
    if (!walk.begin(a, pv)) return;
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, n = lane & 31, h = lane >> 5;
    const int my_key = tid >> 3, my_run = tid & 7;
    const int slot_mask = (1 << a.ps_shift) - 1;
    uint32_t code_at = my_key * kRowBytes + my_run * CB;
    uint32_t scale_at = my_key * DT + my_run * EL / 32;
    const int k_at = KR::at(n, h);        // a key operand's piece 2 kk + h lies 16 kk on
    bool made = false;        // a unit that this share begins and does not end
    Piece w;
    while (walk.next(a, pv, w)) {
        const Req r = walk.r;
        const int32_t* pt = page_table + (size_t)r.b * a.max_pages;
        const int r_local = wave * 32 + n, row = w.group * kWideRows + r_local;
        const bool row_ok = FULL || row < r.rows;
        const bool wave_ok = FULL || uniform(w.group * kWideRows + wave * 32) < r.rows;
        const int ga = a.g * a.bl;
        const int last_row = min((w.group + 1) * kWideRows, r.rows) - 1;
        const int ke = r.o + (last_row / ga + 1) * a.bl;                 // keys of the unit
        const int all = r.o + (w.group * kWideRows / ga + 1) * a.bl;     // that every row sees
        X x;
        x.clear();
        x.seen = r.o + (min(row, last_row) / ga + 1) * a.bl;

        // a thread's run of a tile: key tid / 8, elements (tid % 8) EL ...
        uint32_t kraw[CW], vraw[CW], ksc, vsc;
        bool page_err = false, bad = false;
        // the page of tile t (PAGED), past the piece its last one's
        const int k1 = w.k1;
        auto page_of = [&](int t) {
            return PAGED ? pt[(min(t, k1 - 1) * kKeys) >> a.ps_shift] : 0;
        };
        // Codes of tile t, `page` its page (PAGED).  A bad page id is read as page 0.
        auto load_tile = [&](int t, int page) {
            int p = t * kKeys;
            if constexpr (!PAGED) {
                p = min(p + my_key, ke - 1);
                page = pt[p >> a.ps_shift];
            }
            const bool good = (unsigned)page < (unsigned)a.num_pages;
            page_err |= !good;
            const size_t slot =
                (((size_t)(good ? page : 0) * a.Hkv + w.head) << a.ps_shift) + (p & slot_mask);
            // The compiler would keep the sums of a base and a lane's offset, 64 bits a lane
            // and base: scalar bases and a lane's 32-bit offsets where the lanes share a
            // page; else, where registers are short, one index of codes and one of scales for
            // keys and values (pages of 16 keys, heads of 128: 509 us, 489 so; heads of 64:
            // 290, 310 so).
            size_t ci = slot * kRowBytes + my_run * CB, si = slot * DT + my_run * EL / 32;
            if constexpr (!PAGED && D == 128) asm("" : "+v"(ci), "+v"(si));
            auto run = [&](const uint8_t* codes, const uint8_t* scales, uint32_t* raw, uint32_t& sc) {
                if constexpr (PAGED) {
                    GlobalBytes c0 = (GlobalBytes)(codes + slot * kRowBytes);
                    GlobalBytes s0 = (GlobalBytes)(scales + slot * DT);
                    asm("" : "+s"(c0), "+s"(s0), "+v"(code_at), "+v"(scale_at));
                    load_codes<CB>(c0 + code_at, raw);
                    sc = s0[scale_at];
                } else {
                    load_codes<CB>((GlobalBytes)(codes + ci), raw);
                    sc = scales[si];
                }
            };
            run(kc, ks, kraw, ksc);
            run(vc, vs, vraw, vsc);
        };
        // Piece i of a run into its stage.
        constexpr int NPC = EL < 8 ? 1 : EL / 8;      // pieces of a run
        auto store_piece = [&](auto rows_c, uint16_t* tile, const uint32_t* raw, uint32_t sc, int i) {
            using L = decltype(rows_c);
            const float s = mx_scale(sc);
            if constexpr (EL == 4) {
                bf16x2 v[4];
                if constexpr (BITS == 4) {
                    v[0] = mx_pair<4, 0>(raw[0], s);
                    v[1] = mx_pair<4, 1>(raw[0], s);
                } else {
                    mx_dword<8>(raw[0], s, v);
                }
                *reinterpret_cast<u32x2*>(tile + L::at(my_key, my_run / 2) + my_run % 2 * 4) =
                    u32x2{__builtin_bit_cast(uint32_t, v[0]), __builtin_bit_cast(uint32_t, v[1])};
            } else {
                *reinterpret_cast<u32x4*>(tile + L::at(my_key, my_run * NPC + i)) =
                    eight_values<BITS>(raw + i * (BITS / 4), s);
            }
        };
        // pieces of the next tile: its values', then its keys'
        auto stage = [&](int st, int i) {
            if (i < NPC) store_piece(VR{}, lds_v[st], vraw, vsc, i);
            else store_piece(KR{}, lds_k[st], kraw, ksc, i - NPC);
        };
        // Keys past the unit's last one have no weight, not even as NaN, and neither has a
        // NaN or infinite value for the rows that do not see it: both become zeros before they
        // are stored (those that do see it get it at the end).
        auto zero_tail = [&](int t) {
            if ((t + 1) * kKeys <= all) return;
            const bool past = t * kKeys + my_key >= ke, nan = vsc == 255;
            bad |= nan && !past;
#pragma unroll
            for (int i = 0; i < CW; ++i) {
                kraw[i] = past ? 0 : kraw[i];
                vraw[i] = past || nan ? 0 : vraw[i];
            }
            ksc = past ? 127 : ksc;
            vsc = past || nan ? 127 : vsc;
            if (vsc > kMxHighest<BITS>)
#pragma unroll
                for (int i = 0; i < CW; ++i) bad |= drop_infinite<BITS>(vraw[i], vsc) != 0;
        };

        load_tile(w.k0, page_of(w.k0));
        int page = page_of(w.k0 + 1);        // asked for a step before the tile's codes are
        const T* q = static_cast<const T*>(a.q) +
                     ((size_t)(r.row0 + (row_ok ? row / a.g : 0)) * a.Hq + w.head * a.g +
                      (row_ok ? row % a.g : 0)) * D;
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) query8(q + kk * 16 + h * 8, row_ok, x.qf[kk]);
        zero_tail(w.k0);
#pragma unroll
        for (int i = 0; i < 2 * NPC; ++i) stage(0, i);
        if (w.k0 + 1 < k1) load_tile(w.k0 + 1, page);
        page = page_of(w.k0 + 2);
        // Tile t in stage ST.  NEAR: there may be no tile after it, and rows that do not
        // see all of it or of the next one.
        auto step = [&](int t, auto st_c, auto near_c) __attribute__((always_inline)) {
            constexpr int ST = decltype(st_c)::value;
            constexpr bool NEAR = decltype(near_c)::value;
            constexpr int NX = DT * 2, AHEAD = 2, EVERY = NX / (2 * NPC);
            const uint16_t* kt = lds_k[ST] + k_at;
            auto key = [&](int i) { return *reinterpret_cast<const bf16x8*>(kt + i * 16); };
            auto value = [&](int i) { return X::template values<VR>(lds_v[ST], i / DT, i % DT); };
            __syncthreads();
            bf16x8 pb[2][NP], fr[AHEAD];     // operands are read two products ahead
            if (wave_ok) {
                floatx16 s = floatx16{};
#pragma unroll
                for (int i = 0; i < AHEAD; ++i) fr[i] = key(i);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int i = 0; i < KK; ++i) {
                    const bf16x8 kf = fr[i % AHEAD];
                    fr[i % AHEAD] = i + AHEAD < KK ? key(i + AHEAD) : value(i + AHEAD - KK);
#pragma unroll
                    for (int p = 0; p < NP; ++p)
                        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, x.qf[i][p], s, 0, 0, 0);
                    __builtin_amdgcn_sched_barrier(0);
                }
                if (NEAR && (t + 1) * kKeys > all) x.mask(s, x.seen - t * kKeys);
                x.softmax(s, a.scale_log2, a.slack, pb);
                __builtin_amdgcn_sched_barrier(0);
            }
            const bool more = !NEAR || t + 1 < k1;
            if (NEAR && more) zero_tail(t + 1);
            if (wave_ok) {
#pragma unroll
                for (int i = 0; i < NX; ++i) {
                    const bf16x8 vf = fr[i % AHEAD];
                    if (i + AHEAD < NX) fr[i % AHEAD] = value(i + AHEAD);
                    x.add(vf, i % DT, pb[i / DT]);
                    if (more && i % EVERY == 0) stage(1 - ST, i / EVERY);
                    __builtin_amdgcn_sched_barrier(0);
                }
            } else if (more) {
#pragma unroll
                for (int i = 0; i < 2 * NPC; ++i) stage(1 - ST, i);
            }
            if (!NEAR || t + 2 < k1) load_tile(t + 2, page);
            page = page_of(t + 3);
        };
        using C0 = std::integral_constant<int, 0>;
        using C1 = std::integral_constant<int, 1>;
        // steps whose tile t + 2 is there and whose tile t + 1 every row sees
        const int far = min(k1 - 2, all / kKeys - 1);
        int t = w.k0;
        for (; t + 2 <= far; t += 2) {
            step(t, C0{}, std::false_type{});
            step(t + 1, C1{}, std::false_type{});
        }
        for (; t < k1; t += 2) {
            step(t, C0{}, std::true_type{});
            if (t + 1 < k1) step(t + 1, C1{}, std::true_type{});
        }
        if (page_err) record_error(pv.hdr, r.b, FB_DERR_PAGE);
        // (the barrier also lets the next piece fill the stages)
        if (__syncthreads_or(bad))
            x.template spoil<BITS>(a, vc, vs, pt, w.head, max(w.k0, all / kKeys) * kKeys, min(k1 * kKeys, ke));
        x.store(a, r, w, uniform(wave) * 32, kWideRows);
        if (w.more > 0) {
            made = true;
            if (tid == 0) store_record(a, walk.index, r, w, kWideRows);
        }
    }
    if (!made && tid == 0) a.rec[(size_t)walk.index * kRecInts + kRPieces] = 0;
}

// -------------------------------------------------------------- few rows ---
// What the lanes of a wave wrote to LDS is there for all of them.
__device__ inline void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

template <int D, int BITS, typename T>
__global__ void __launch_bounds__(kThreads, per_cu(D, sizeof(T) == 2, kFewRows))
mx_few_kernel(MxArgs a, MX_CACHE_PARAMS, PackView pv) {
    constexpr int CB = D / 2 * BITS / 8;   // code bytes of half a key: a lane's
    constexpr int CW = CB / 4;
    constexpr int SC = D >= 64 ? D / 64 : 1;
    using R = Rows<D, T>;
    constexpr int KK = R::KK, DT = R::DT, NP = R::NP;
    // each wave's V tile; at a piece's end the results of two waves
    union Lds {
        uint16_t v[4][kKeys * D];
        float4 join[2][DT * 4][64];
    };
    __shared__ __attribute__((aligned(16))) Lds lds;
    __shared__ float stat[2][2][64];
    // fp32: the rows' three parts, the same for every wave; in registers they would spill
    // (64 single tokens over long contexts: 529 us, 234 so)
    constexpr bool kQueryInLds = NP == 3;
    __shared__ __attribute__((aligned(16))) u32x4 lds_q[kQueryInLds ? KK : 1][NP][64];

    Walk<kFewRows> walk;
    if (!walk.begin(a, pv)) return;
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, n = lane & 31, h = lane >> 5;
    const int slot_mask = (1 << a.ps_shift) - 1;
    uint16_t* vt = lds.v[wave];
    bool made = false;
    Piece w;
    while (walk.next(a, pv, w)) {
        const Req r = walk.r;
        const int32_t* pt = page_table + (size_t)r.b * a.max_pages;
        const int row = w.group * kFewRows + n;
        const bool row_ok = row < r.rows;
        const int ga = a.g * a.bl;
        const int last_row = min((w.group + 1) * kFewRows, r.rows) - 1;
        const int ke = r.o + (last_row / ga + 1) * a.bl;
        const int all = r.o + (w.group * kFewRows / ga + 1) * a.bl;
        R x;
        x.clear();
        x.seen = r.o + (min(row, last_row) / ga + 1) * a.bl;
        // lane half h takes channels h D/2 ..; eight of them go to each product
        const T* q = static_cast<const T*>(a.q) +
                     ((size_t)(r.row0 + (row_ok ? row / a.g : 0)) * a.Hq + w.head * a.g +
                      (row_ok ? row % a.g : 0)) * D + h * (D / 2);
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) {
            if constexpr (kQueryInLds) {
                if (kk % 4 != wave) continue;
                bf16x8 f[NP];
                query8(q + kk * 8, row_ok, f);
#pragma unroll
                for (int p = 0; p < NP; ++p) lds_q[kk][p][lane] = __builtin_bit_cast(u32x4, f[p]);
            } else {
                query8(q + kk * 8, row_ok, x.qf[kk]);
            }
        }
        if constexpr (kQueryInLds) __syncthreads();
        auto query = [&](int kk, int p) {
            if constexpr (kQueryInLds) return __builtin_bit_cast(bf16x8, lds_q[kk][p][lane]);
            else return x.qf[kk][p];
        };

        // sets of codes: of the next tile, or of the next two where the registers hold them
        constexpr int SETS = BITS == 4 && NP == 1 ? 2 : 1, STRIDE = 4 * SETS;
        uint32_t kraws[SETS][CW], vraws[SETS][CW], kscs[SETS][SC], vscs[SETS][SC];
        bool page_err = false, bad = false;
        // The page of key n of tile t, past the piece its last tile's.
        auto page_of = [&](int t) {
            return pt[min(min(t, w.k1 - 1) * kKeys + n, ke - 1) >> a.ps_shift];
        };
        // Codes of this lane's half of key n of tile t.  A bad page id is read as page 0.
        auto load_tile = [&](int t, int page, int set) {
            uint32_t(&kraw)[CW] = kraws[set], (&vraw)[CW] = vraws[set];
            uint32_t(&ksc)[SC] = kscs[set], (&vsc)[SC] = vscs[set];
            const int p = min(t * kKeys + n, ke - 1);
            const bool good = (unsigned)page < (unsigned)a.num_pages;
            page_err |= !good;
            const size_t slot =
                (((size_t)(good ? page : 0) * a.Hkv + w.head) << a.ps_shift) + (p & slot_mask);
            load_codes<CB>((GlobalBytes)(kc + slot * (D * BITS / 8) + h * CB), kraw);
            load_codes<CB>((GlobalBytes)(vc + slot * (D * BITS / 8) + h * CB), vraw);
#pragma unroll
            for (int i = 0; i < SC; ++i) {
                ksc[i] = ks[slot * DT + (D >= 64 ? h * SC : 0) + i];
                vsc[i] = vs[slot * DT + (D >= 64 ? h * SC : 0) + i];
            }
        };
        // As in the wide kernel: keys past the unit's last one, and NaN and infinite values that
        // not every row sees, become zeros.
        auto zero_tail = [&](int t, int set) {
            uint32_t(&kraw)[CW] = kraws[set], (&vraw)[CW] = vraws[set];
            uint32_t(&ksc)[SC] = kscs[set], (&vsc)[SC] = vscs[set];
            const bool past = t * kKeys + n >= ke;
#pragma unroll
            for (int i = 0; i < SC; ++i) {
                const bool nan = vsc[i] == 255;
                bad |= nan && !past;
                constexpr int W = CW / SC;
#pragma unroll
                for (int j = 0; j < W; ++j) {
                    kraw[i * W + j] = past ? 0 : kraw[i * W + j];
                    vraw[i * W + j] = past || nan ? 0 : vraw[i * W + j];
                }
                ksc[i] = past ? 127 : ksc[i];
                vsc[i] = past || nan ? 127 : vsc[i];
                if (vsc[i] > kMxHighest<BITS>)
#pragma unroll
                    for (int j = 0; j < W; ++j) bad |= drop_infinite<BITS>(vraw[i * W + j], vsc[i]) != 0;
            }
        };
        const int t0 = w.k0 + wave;
        int page = page_of(t0 + STRIDE);          // asked for a tile before its codes are
        if (t0 < w.k1) load_tile(t0, page_of(t0), 0);
        if (SETS == 2 && t0 + 4 < w.k1) load_tile(t0 + 4, page_of(t0 + 4), SETS - 1);
        auto step = [&](int t, auto set_c) __attribute__((always_inline)) {
            constexpr int SET = decltype(set_c)::value;
            uint32_t(&kraw)[CW] = kraws[SET], (&vraw)[CW] = vraws[SET];
            uint32_t(&ksc)[SC] = kscs[SET], (&vsc)[SC] = vscs[SET];
            const bool masked = (t + 1) * kKeys > all;
            if (masked) zero_tail(t, SET);
            floatx16 s = floatx16{};
#pragma unroll
            for (int kk = 0; kk < KK; ++kk) {
                constexpr int PG = D >= 64 ? 4 : KK;      // pieces of eight to a group
                const u32x4 kf = eight_values<BITS>(kraw + kk * (BITS / 4), mx_scale(ksc[kk / PG]));
#pragma unroll
                for (int p = 0; p < NP; ++p)
                    s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kf),
                                                                query(kk, p), s, 0, 0, 0);
                *reinterpret_cast<u32x4*>(vt + TurnedRows<D>::at(n, h * KK + kk)) =
                    eight_values<BITS>(vraw + kk * (BITS / 4), mx_scale(vsc[kk / PG]));
                __builtin_amdgcn_sched_barrier(0);   // (else every piece is in registers at once)
            }
            if (t + STRIDE < w.k1) load_tile(t + STRIDE, page, SET);
            page = page_of(t + STRIDE + 4);
            wave_sync();
            bf16x8 pb[2][NP];
            if (masked) x.mask(s, x.seen - t * kKeys);
            x.softmax(s, a.scale_log2, a.slack, pb);
            auto value = [&](int i) {
                return R::template values<TurnedRows<D>>(vt, i / DT, i % DT);
            };
            bf16x8 fr[2] = {value(0), value(1)};
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < 2 * DT; ++i) {
                const bf16x8 v = fr[i & 1];
                if (i + 2 < 2 * DT) fr[i & 1] = value(i + 2);
                x.add(v, i % DT, pb[i / DT]);
                __builtin_amdgcn_sched_barrier(0);
            }
            wave_sync();   // the next tile's values go to the same place
        };
        for (int t = t0; t < w.k1; t += STRIDE) {
            step(t, std::integral_constant<int, 0>{});
            if (SETS == 2 && t + 4 < w.k1) step(t + 4, std::integral_constant<int, SETS - 1>{});
        }
        // (each wave gives its rows theirs itself: a key is one wave's)
        if (__any(bad))
            for (int t = w.k0 + wave; t < w.k1; t += 4)
                if ((t + 1) * kKeys > all)
                    x.template spoil<BITS>(a, vc, vs, pt, w.head, t * kKeys, min((t + 1) * kKeys, ke));
        if (page_err) record_error(pv.hdr, r.b, FB_DERR_PAGE);

        // waves 2 and 3 join 0 and 1, then 1 joins 0
#pragma unroll
        for (int from = 2; from >= 1; from >>= 1) {
            __syncthreads();
            const bool gives = wave >= from && wave < 2 * from;
            const int to = wave & (from - 1);
            float4(&j)[DT * 4][64] = lds.join[to];
            if (gives) {
                stat[to][0][lane] = x.thr == -INFINITY ? -INFINITY : x.m_sub;
                stat[to][1][lane] = x.l;
#pragma unroll
                for (int i = 0; i < DT * 4; ++i) {
                    const floatx16& o = x.o[i / 4];
                    const int at = i % 4 * 4;
                    j[i][lane] = make_float4(o[at], o[at + 1], o[at + 2], o[at + 3]);
                }
            }
            __syncthreads();
            if (wave < from) {
                // (a side without a score above -inf has no weight, but its NaN counts)
                const float m0 = x.thr == -INFINITY ? -INFINITY : x.m_sub, m1 = stat[to][0][lane];
                const float m = fmaxf(m0, m1);
                const float f0 = m0 == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m0 - m);
                const float f1 = m1 == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m1 - m);
                if (m > -INFINITY) {
                    x.m_sub = m;
                    x.thr = m;
                }
                x.l = x.l * f0 + stat[to][1][lane] * f1;
#pragma unroll
                for (int i = 0; i < DT * 4; ++i) {
                    floatx16& o = x.o[i / 4];
                    const int at = i % 4 * 4;
                    const float4 v = j[i][lane];
                    o[at] = o[at] * f0 + v.x * f1;
                    o[at + 1] = o[at + 1] * f0 + v.y * f1;
                    o[at + 2] = o[at + 2] * f0 + v.z * f1;
                    o[at + 3] = o[at + 3] * f0 + v.w * f1;
                    if (i % 4 == 3) __builtin_amdgcn_sched_barrier(0);
                }
            }
        }
        if (wave == 0) x.store(a, r, w, 0, kFewRows);
        if (w.more > 0) {
            made = true;
            if (tid == 0) store_record(a, walk.index, r, w, kFewRows);
        }
        __syncthreads();
    }
    if (!made && tid == 0) a.rec[(size_t)walk.index * kRecInts + kRPieces] = 0;
}

// ---------------------------------------------------------------- merge ---
// A workgroup merges R rows of a divided unit: the unit's first piece in slot
// 2 i + 1 of the share i that it began in, the others in slots 2 (i + 1), 2 (i
// + 2), ...  256 / (D / 4) threads to a channel quad: R rows, and PL lanes that
// take the pieces in turn.
template <int D, typename T, int R>
__global__ void __launch_bounds__(kThreads)
mx_merge_kernel(MxArgs a, int rows, int parts) {
    constexpr int Q = D / 4, PL = kThreads / Q / R;
    __shared__ float m_of[PL][R], den_of[PL][R];
    __shared__ float4 acc_of[PL][R][Q];
    const int i = blockIdx.x / parts, part = blockIdx.x % parts;
    if (i >= a.head[0]) return;
    const int32_t* rec = a.rec + (size_t)i * kRecInts;
    const int pieces = rec[kRPieces];
    const int row0 = rec[kRRow0], head = rec[kRHead], first = rec[kRFirst], n = rec[kRRows];
    if (pieces == 0 || part * R >= n) return;
    const int d4 = threadIdx.x % Q, rl = threadIdx.x / Q % R, pl = threadIdx.x / Q / R;
    const int r = min(part * R + rl, n - 1);
    auto slot = [&](int k) {
        return (size_t)(k == 0 ? 2 * i + 1 : 2 * (i + k)) * rows + r;
    };
    float m = -INFINITY, den = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    constexpr int F = 4;   // pieces in flight
    for (int k0 = pl; k0 < pieces; k0 += F * PL) {
        float lse[F];
        float4 v[F];
#pragma unroll
        for (int j = 0; j < F; ++j) {
            const size_t s = slot(min(k0 + j * PL, pieces - 1));
            lse[j] = a.part_lse[s];
            v[j] = *reinterpret_cast<const float4*>(a.part_o + s * D + d4 * 4);
        }
#pragma unroll
        for (int j = 0; j < F; ++j) {
            if (k0 + j * PL >= pieces || lse[j] == -INFINITY) continue;
            const float m_new = fmaxf(m, lse[j]);
            const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - m_new);
            const float x = __builtin_amdgcn_exp2f(lse[j] - m_new);
            den = den * f + x;
            acc.x = acc.x * f + x * v[j].x;
            acc.y = acc.y * f + x * v[j].y;
            acc.z = acc.z * f + x * v[j].z;
            acc.w = acc.w * f + x * v[j].w;
            m = m_new;
        }
    }
    if constexpr (PL > 1) {
        if (d4 == 0) m_of[pl][rl] = m, den_of[pl][rl] = den;
        acc_of[pl][rl][d4] = acc;
        __syncthreads();
        if (pl > 0) return;
#pragma unroll
        for (int p = 1; p < PL; ++p) {
            const float mp = m_of[p][rl];
            const float4 v = acc_of[p][rl][d4];
            if (mp == -INFINITY && den_of[p][rl] == 0.f) continue;
            const float m_new = fmaxf(m, mp);
            const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - m_new);
            const float x = __builtin_amdgcn_exp2f(mp - m_new);
            den = den * f + den_of[p][rl] * x;
            acc.x = acc.x * f + x * v.x;
            acc.y = acc.y * f + x * v.y;
            acc.z = acc.z * f + x * v.z;
            acc.w = acc.w * f + x * v.w;
            m = m_new;
        }
    }
    if (part * R + rl >= n) return;
    const float id = 1.0f / den;
    const int row = first + r;
    T* dst = static_cast<T*>(a.out) +
             ((size_t)(row0 + row / a.g) * a.Hq + head * a.g + row % a.g) * D + d4 * 4;
    store4(dst, acc.x * id, acc.y * id, acc.z * id, acc.w * id);
}

}  // namespace

MxAttnSizes mx_attention_sizes(const fb_pack* pack, const fb_attn_shape* sh, int cu_count) {
    MxAttnSizes z{};
    const long long most = (long long)pack->W_max * pack->bl * (sh->Hq / sh->Hkv);
    z.rows = most <= kFewRows ? kFewRows : kWideRows;
    const int each = per_cu(sh->head_dim, sh->dtype == FB_BF16, z.rows);
    z.wgs = (each * (cu_count > 0 ? cu_count : 256) + 7) / 8 * 8;
    size_t off = 0;
    auto take = [&](size_t bytes) {
        const size_t at = off;
        off += (bytes + 255) & ~(size_t)255;
        return at;
    };
    z.off_head = take(16);
    z.off_rec = take((size_t)z.wgs * kRecInts * sizeof(int32_t));
    z.off_o = take((size_t)2 * z.wgs * z.rows * sh->head_dim * sizeof(float));
    z.off_lse = take((size_t)2 * z.wgs * z.rows * sizeof(float));
    z.total = off;
    return z;
}

hipError_t launch_mx_attention(const void* q, const fb_mx_cache* cache, const int32_t* page_table,
                               const fb_pack* pack, const fb_attn_shape* sh, void* out, void* wsp,
                               const MxAttnSizes& z, hipStream_t stream) {
    const float scale = sh->sm_scale > 0.f ? sh->sm_scale : 1.0f / sqrtf((float)sh->head_dim);
    char* ws = static_cast<char*>(wsp);
    const long long all_rows = (long long)pack->W_max * pack->bl * (sh->Hq / sh->Hkv);
    const long long groups = (all_rows + z.rows - 1) / z.rows;
    const long long most = all_rows < z.rows ? all_rows : z.rows;
    // (positions are 32-bit; the last ones are left out, so that tiles end within them)
    long long max_keys = (long long)sh->max_pages * sh->page_size;
    if (max_keys > 0x7fffffffLL - 4096) max_keys = 0x7fffffffLL - 4096;
    const int whole = (long long)pack->B * sh->Hkv * groups <= z.wgs &&
                      max_keys <= (z.rows == kFewRows ? kFewWholeKeys : kWideWholeKeys);
    const double places = (double)pack->B * sh->Hkv * groups *
                          ((double)max_keys / kKeys + 1 + kFewStart);
    const int short_line = places < 2147483648.0;
    const MxArgs a{q,
                   out,
                   reinterpret_cast<int32_t*>(ws + z.off_head),
                   reinterpret_cast<int32_t*>(ws + z.off_rec),
                   reinterpret_cast<float*>(ws + z.off_o),
                   reinterpret_cast<float*>(ws + z.off_lse),
                   sh->Hq, sh->Hkv, sh->Hq / sh->Hkv, pack->bl, pack->B, pack->W_max,
                   pack->row_cap, z.wgs, log2_of(sh->page_size), sh->max_pages, sh->num_pages,
                   (int)max_keys, whole, short_line,
                   scale * kLog2e, kRescaleSlack / (scale * kLog2e)};
    auto launch = [&](auto d_c, auto bits_c, auto zero) {
        constexpr int D = decltype(d_c)::value, BITS = decltype(bits_c)::value;
        using T = decltype(zero);
        auto go = [&](auto kernel) {
            hipLaunchKernelGGL(kernel, dim3(z.wgs), dim3(kThreads), 0, stream, a,
                               static_cast<const uint8_t*>(cache->k_codes),
                               static_cast<const uint8_t*>(cache->k_scales),
                               static_cast<const uint8_t*>(cache->v_codes),
                               static_cast<const uint8_t*>(cache->v_scales), page_table,
                               pack_view(pack));
        };
        auto merge = [&](auto kernel, int rows) {
            if (a.whole) return;
            const int parts = (int)((most + rows - 1) / rows);   // of the rows that a unit can have
            hipLaunchKernelGGL(kernel, dim3(z.wgs * parts), dim3(kThreads), 0, stream, a, z.rows,
                               parts);
        };
        if (z.rows == kFewRows) {
            go(mx_few_kernel<D, BITS, T>);
            merge(mx_merge_kernel<D, T, 1>, 1);
        } else {
            const bool full = pack->bl * a.g % kWideRows == 0;
            if (sh->page_size < kKeys) go(mx_wide_kernel<D, BITS, T, false, false>);
            else if (full && sizeof(T) == 2) go(mx_wide_kernel<D, BITS, T, true, sizeof(T) == 2>);
            else go(mx_wide_kernel<D, BITS, T, true, false>);
            merge(mx_merge_kernel<D, T, 8>, 8);
        }
    };
    auto of_type = [&](auto d_c, auto bits_c) {
        if (sh->dtype == FB_BF16) launch(d_c, bits_c, uint16_t());
        else launch(d_c, bits_c, float());
    };
    auto of_format = [&](auto d_c) {
        if (cache->format == FB_MX4) of_type(d_c, std::integral_constant<int, 4>{});
        else of_type(d_c, std::integral_constant<int, 8>{});
    };
    if (sh->head_dim == 32) of_format(std::integral_constant<int, 32>{});
    else if (sh->head_dim == 64) of_format(std::integral_constant<int, 64>{});
    else of_format(std::integral_constant<int, 128>{});
    return hipGetLastError();
}

}  // namespace fb
