/*
 * flowblock_cache.h -- a KV cache held in 4 or 8 bits, and positions with
 * several axes in front of it, for callers whose contexts are long or whose
 * tokens stand in images and video.
 *
 *   fb_rotary_axes         rotary positions along several axes, on queries and
 *                          fresh keys (in front of either cache)
 *   fb_mx_write_window_kv  fb_write_window_kv (Eq. 6) into a quantised cache
 *   fb_mx_read_kv          spans of positions read back as dense keys and values
 *   fb_mx_attention        fb_wavefront_attention (Sec. 4.1 / Eq. 5) over the
 *                          quantised cache
 *
 * Every function follows the conventions of flowblock.h (caller-owned device
 * memory, dense row-major arrays, stream-ordered, FB_* status,
 * fb_last_error(), launch shapes that depend on capacities only).  Row
 * arguments are in the pack's row order ([row_cap] rows); rows that are not
 * live are neither read for a result nor written.
 */
#ifndef FLOWBLOCK_CACHE_H
#define FLOWBLOCK_CACHE_H

#include "flowblock.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- rotary positions with several axes ---------------------------------- */

/* Which elements of a head vector turn together. */
#define FB_PAIR_HALVES     0   /* pair j: elements j and n_pairs + j           */
#define FB_PAIR_NEIGHBOURS 1   /* pair j: elements 2j and 2j + 1               */

/* The turning of a head vector (host struct).  Pair j turns by the angle
 * positions[axis[j]][row] * freq[j]; elements from 2 n_pairs on stay as they
 * are.  Sections of pairs for time, height and width, interleaved axes and
 * frequencies that start anew in each section are all a choice of axis and
 * freq; one axis holding the pack's own positions, with freq[j] =
 * base^(-2j/d) over d/2 pairs, is fb_window_prologue's rotation. */
typedef struct fb_rotary {
    int32_t n_axes;      /* rows of positions, 1 .. 8                          */
    int32_t n_pairs;     /* 1 .. head_dim / 2                                  */
    int32_t pairing;     /* FB_PAIR_*                                          */
    int32_t reserved;
    double  freq[64];    /* finite; |position * freq| up to 2^53 (angles past
                            that hold no fraction of a turn)                   */
    uint8_t axis[64];    /* each below n_axes                                  */
} fb_rotary;

/* Turns the live rows' queries and fresh keys; the keys then go to
 * fb_write_window_kv or fb_mx_write_window_kv.  Angles are formed and reduced
 * in float64, their sines and cosines and the products are float32, results
 * are rounded once to the dtype.
 *   q_in, q_out  [row_cap][Hq][d]; may be the same buffer; both NULL: no queries
 *   k_in, k_out  [row_cap][Hkv][d]; the same (not all four NULL)
 *   positions    int32[n_axes][row_cap], any values; not read where a row is
 *                not live
 *   sh           Hq, Hkv, head_dim and dtype are used
 * Outputs that overlap an input without being it, or each other, are refused.
 * Pointers are 16-byte aligned. */
int fb_rotary_axes(const void* q_in, void* q_out, const void* k_in, void* k_out,
                   const int32_t* positions, const fb_pack* pack,
                   const fb_attn_shape* sh, const fb_rotary* rotary, void* stream);

/* ---- the quantised cache ------------------------------------------------- */

/* Codes of a cache: the element types of the OCP Microscaling formats. */
#define FB_MX4 4   /* E2M1: +-{0, 0.5, 1, 1.5, 2, 3, 4, 6}; element 2i in the
                      low half of byte i, 2i + 1 in the high half             */
#define FB_MX8 8   /* E4M3: up to 448, least step 2^-9; one to a byte          */

/* Paged keys and values in codes of 4 or 8 bits with one power-of-two scale
 * (E8M0: 2^(scale - 127)) per 32 channels of a key or value:
 *   *_codes   uint8 [num_pages][Hkv][page_size][d * format / 8]
 *   *_scales  uint8 [num_pages][Hkv][page_size][d / 32]
 * Unlike the bf16 cache's, values stand as keys do (channels innermost).  A
 * token takes 2 Hkv d (format / 8 + 1 / 32) bytes: 27% of the bf16 cache in 4
 * bits, 52% in 8.  Codes are 16-byte aligned, scales need no alignment.
 * Scales of 2 .. 252 (FB_MX4) or 10 .. 246 (FB_MX8) keep every value normal and
 * finite in bf16, and fb_mx_write_window_kv writes no others, but for 255: its
 * 32 values are NaN.  In a cache that others have filled, values under 2^-126 may
 * be taken as 0, values past bf16's largest are infinite, and E4M3's own NaN codes
 * (127, 255), which are not written here, may spoil every row of the request. */
typedef struct fb_mx_cache {
    void* k_codes;
    void* k_scales;
    void* v_codes;
    void* v_scales;
    int32_t format;      /* FB_MX4 or FB_MX8                                   */
    int32_t reserved;
} fb_mx_cache;

/* Device status (fb_pack_read_status): a span of fb_mx_read_kv is ill-formed;
 * its request is skipped. */
#define FB_DERR_SPAN 5

/* Eq. 6 into a quantised cache: the fresh K/V of every live packed row at its
 * absolute position, as fb_write_window_kv stores them, each group of 32
 * channels with a scale 2^e of its own: e is the least integer for which no
 * element passes the largest code (6 or 448) times 2^e, kept within -125 ..
 * 125 (FB_MX4) or -117 .. 119 (FB_MX8).  Elements go to the nearest code, ties
 * to the even one; larger ones than the largest code at the greatest scale go
 * to that code.  A group that holds a NaN or an infinity becomes NaN (scale
 * 255).  Codes depend on nothing but their group, so the same tokens give the
 * same bytes wherever they stand.
 *   k_new, v_new  [row_cap][Hkv][d] (dtype of sh), 16-byte aligned
 *   page_table    int32[B][max_pages]
 *   bl * Hkv * d/8 at most 2^31 - 2^24
 * A page id outside [0, num_pages) or a position past max_pages*page_size is
 * skipped and recorded as FB_DERR_PAGE. */
int fb_mx_write_window_kv(const void* k_new, const void* v_new,
                          const fb_mx_cache* cache, const int32_t* page_table,
                          const fb_pack* pack, const fb_attn_shape* sh,
                          void* stream);

/* Reads positions [first_b, first_b + n_b) of every request back as dense keys
 * and values: position first_b + t goes to row t of request b.  The values that
 * the codes stand for are exact in both dtypes.
 *   spans         int32[B][2]: first_b and n_b, 0 <= first_b, 0 <= n_b <= T,
 *                 first_b + n_b <= max_pages * page_size and below 2^31
 *   T             at most 2^30
 *   k_out, v_out  [B][T][Hkv][d] (dtype of sh), 16-byte aligned; either may be
 *                 NULL, not both; rows from n_b on are not written
 *   pack          its B, and the status word; what it holds is not read
 * An ill-formed span skips its request (FB_DERR_SPAN); a page id outside
 * [0, num_pages) leaves its positions unwritten (FB_DERR_PAGE). */
int fb_mx_read_kv(const fb_mx_cache* cache, const int32_t* page_table,
                  const int32_t* spans, int T, void* k_out, void* v_out,
                  const fb_pack* pack, const fb_attn_shape* sh, void* stream);

/* Workspace bytes for fb_mx_attention with this pack and shape, 0 if the
 * arguments are invalid. */
size_t fb_mx_attention_workspace_bytes(const fb_pack* pack, const fb_attn_shape* sh);

/* fb_wavefront_attention over a quantised cache: a query of window slot s of
 * request b attends to keys [0, o_b + (s+1)*bl) of its KV head,
 *   out[row][h] = sum_j softmax_j(sm_scale * <q[row][h], K[j]>) V[j],
 * K and V the values that the codes stand for, which are exact in bf16.  Call
 * after fb_mx_write_window_kv so the window's own keys are in the cache.  A
 * window of single tokens (bl = 1, W_max = 1) is ordinary decoding.
 * Products and sums are float32.  FB_BF16: the softmax weights are rounded to
 * bf16, the denominator sums the rounded ones.  FB_F32: queries and weights go
 * through the matrix cores in three bf16 parts, which hold all their bits.
 *   q, out  [row_cap][Hq][d] (dtype of sh), 16-byte aligned; out may be q
 *   ws      device workspace of fb_mx_attention_workspace_bytes bytes, 16-byte
 *           aligned
 * Scores sm_scale * <q, K> are below 2^30 in magnitude (the rows of larger ones may
 * be NaN), W_max * bl * Hq/Hkv is at most 2^31 - 128.
 * Deterministic: repeated calls give bit-identical results.  How long contexts
 * are divided among workgroups, and so the rounding of a request's rows, goes
 * by the whole pack; kv_split is not read.  A NaN scale spoils the rows that see
 * its key, no others; an infinite value makes its channel infinite or NaN in
 * those rows, and nothing else.  A page id outside [0, num_pages) is recorded as
 * FB_DERR_PAGE and the rows of its request hold no result; a window that the
 * page table does not reach is recorded too, and its request skipped. */
int fb_mx_attention(const void* q, const fb_mx_cache* cache,
                    const int32_t* page_table, const fb_pack* pack,
                    const fb_attn_shape* sh, void* out, void* ws,
                    size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* FLOWBLOCK_CACHE_H */
