/*
 * flowblock_tail.h -- the tail of the model's forward f_theta (Alg. 1) on the
 * packed live rows: what stands between a block's output and the denoise
 * update, for callers that run their own layers around flowblock.h.
 *
 *   fb_residual_norm       the norms after and before a block, fused with the
 *                          block's gate and scaled residual
 *   fb_mx4_linear          a linear layer with 4-bit weights and group scales
 *                          (projections, LM head)
 *   fb_rules_build         what the committed tokens, biases and penalties of
 *                          each request say about the vocabulary
 *   fb_vocab_reduce_rules  fb_vocab_reduce (Eq. 1's x_hat and p) on logits
 *                          under penalties, biases and grammar masks
 *   fb_logits_rules        the same logits, written whole
 *
 * Every function follows the conventions of flowblock.h (caller-owned device
 * memory, dense row-major arrays, stream-ordered, FB_* status,
 * fb_last_error(), launch shapes that depend on capacities only).  Every row
 * argument is in the pack's row order ([row_cap] rows); rows that are not live
 * are neither read for a result nor written.
 */
#ifndef FLOWBLOCK_TAIL_H
#define FLOWBLOCK_TAIL_H

#include "flowblock.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- norms around a block ------------------------------------------------ */

/* Layouts of the gate of fb_residual_norm. */
#define FB_GATE_NONE    0   /* no gate (1)                                     */
#define FB_GATE_ALL     1   /* [D], the same for every row                     */
#define FB_GATE_REQUEST 2   /* [B][D], a request's rows share theirs           */
#define FB_GATE_ROW     3   /* [row_cap][D]                                    */

typedef struct fb_norm_shape {
    int32_t D;           /* width, 1 .. 16384                                  */
    int32_t dtype;       /* FB_BF16 or FB_F32: every array of the call         */
    int32_t gate;        /* FB_GATE_*                                          */
    float   eps;         /* finite and > 0                                     */
    float   res_scale;   /* a, finite                                          */
    int32_t reserved[3];
} fb_norm_shape;

/* One residual step with the norms on both sides of it, per live row r of
 * request b, over its D elements:
 *   u    = y_r / sqrt(mean(y_r^2) + eps) * w_post     (w_post NULL: u = y_r)
 *   h'   = h_r + a * (g u)                 -> h_out   (y NULL: h' = h_r)
 *   n    = h' / sqrt(mean(h'^2) + eps) * w_pre -> n_out
 * with g the gate (its layout in sh) and a = res_scale.  Everything between
 * the inputs and the two outputs is float32; n is formed from the unrounded h'.
 * The norms hold for every finite y and h', also where the squares or their mean
 * pass float32's range.
 *   y       [row_cap][D], the block's output; NULL for a plain norm of h (then
 *           gate, w_post and h_out are NULL too)
 *   h       [row_cap][D], the residual stream
 *   gate    as sh->gate says (NULL for FB_GATE_NONE)
 *   w_post, w_pre  [D] or NULL (no norm of y; an unweighted norm of h')
 *   h_out   [row_cap][D]; may be h
 *   n_out   [row_cap][D] or NULL (then w_pre is NULL); may be y or h, not h_out
 * Arrays that overlap in another way give undefined results.  Pointers need
 * the alignment of their element type only. */
int fb_residual_norm(const void* y, const void* h, const void* gate,
                     const void* w_post, const void* w_pre, void* h_out,
                     void* n_out, const fb_pack* pack, const fb_norm_shape* sh,
                     void* stream);

/* ---- linear layers with 4-bit weights ------------------------------------ */

/* y_r = W x_r for every live row, W [N][K] in the OCP Microscaling format
 * MXFP4: element (n, k) is E2M1(code[n][k]) * 2^(scale[n][k/32] - 127), the
 * sixteen codes standing for +-{0, 0.5, 1, 1.5, 2, 3, 4, 6} (the top bit is
 * the sign).  The weights are exact in bf16; products are exact and sums are
 * float32, rounded once to y's type.
 *   x       bf16 [row_cap][K], 16-byte aligned
 *   codes   uint8 [N][K/2]: element 2i in the low half of byte i, element
 *           2i + 1 in the high half; 16-byte aligned
 *   scales  uint8 [N][K/32] (E8M0)
 *   y       [row_cap][N], y_dtype FB_BF16 or FB_F32; not x
 *   N 1 .. 2^30; K a positive multiple of 32, at most 65536
 * Scales: 2 .. 252 keep every weight normal in bf16; below, weights under
 * 2^-126 may be taken as 0; above, weights past bf16's largest are infinite;
 * 255 (E8M0's NaN) makes its 32 weights NaN.
 * The order of a sum goes by N, K and the pack's capacity, not by the live
 * rows, so a row's result does not depend on the other rows of the pack. */
int fb_mx4_linear(const void* x, const void* codes, const void* scales, int N,
                  int K, const fb_pack* pack, void* y, int y_dtype, void* stream);

/* ---- penalties, biases and grammar masks on logits ----------------------- */

/* Penalties of one request (device array [B]).  16 bytes. */
typedef struct fb_rule_params {
    float   repetition;   /* r, 2^-40 .. 2^40; 1 is none                      */
    float   presence;     /* p, finite; 0 is none                             */
    float   frequency;    /* f, finite; 0 is none                             */
    int32_t reserved;
} fb_rule_params;

/* The rules of a step (host struct of device pointers).  For a live row of
 * request b, and a token v:
 *   seen_v  v stands in the committed prefix, positions [0, o_b)
 *   c_v     how often it stands at generated positions, [prompt_len, o_b)
 *   z1      = z_v / r if seen_v and z_v > 0, z_v * r if seen_v otherwise, z_v
 *             if not seen
 *   z'_v    = z1 + ((bias_v - (c_v > 0 ? p : 0)) - f * c_v), in float32, no
 *             product contracted; a token neither seen nor biased keeps z_v
 *   z'_v    = -inf where the row's mask does not allow v, whatever z_v is
 * Biases may be -inf (a banned token) but neither +inf nor NaN. */
typedef struct fb_logit_rules {
    const fb_rule_params* params;  /* [B], or NULL: no penalties              */
    const int32_t* bias_start;     /* [B+1] request b's entries of bias_id are
                                      [bias_start[b], bias_start[b+1]); NULL:
                                      no biases                               */
    const int32_t* bias_id;        /* [n_bias] token ids, ascending within a
                                      request; an id that stands there more
                                      than once gets the sum, in order        */
    const float*   bias_val;       /* [n_bias]                                */
    const uint32_t* masks;         /* [n_masks][ceil(V/32)]: bit v % 32 of word
                                      v / 32 set if v is allowed; NULL: none  */
    const int32_t* row_mask;       /* [row_cap] mask of each row, -1: all
                                      allowed; NULL if masks is               */
    int32_t n_bias, n_masks;       /* capacities of the arrays above          */
} fb_logit_rules;

/* Device status (fb_pack_read_status): a request's penalties, bias entries or
 * a row's mask index are out of range.  Nothing is allowed to the request's
 * (the row's) tokens then, as under an empty mask. */
#define FB_DERR_RULE 4

/* Workspace bytes of fb_rules_build for this pack and vocabulary, 0 if the
 * arguments are invalid.  V at most 2^19. */
size_t fb_rules_workspace_bytes(const fb_pack* pack, int V);

/* Writes into `ws` what the rules need of each request: which tokens are seen
 * or biased, how often, by how much.  Reads the committed tokens, never the
 * window's or the logits, so it may run on another stream beside the forward.
 * The two calls below then read ws; the caller orders them after this one and
 * keeps ws untouched in between, the pack and the request states as they were.
 *   st      device fb_req_state[B], as given to fb_pack_wavefronts
 *   tokens  device int32[B][T_max]; ids outside [0, V) are passed over
 *   rules   what masks and row_mask point to is not read
 *   ws      device workspace of fb_rules_workspace_bytes bytes, 16-byte aligned */
int fb_rules_build(const fb_logit_rules* rules, const fb_req_state* st,
                   const int32_t* tokens, int T_max, int V, const fb_pack* pack,
                   void* ws, size_t ws_bytes, void* stream);

/* fb_vocab_reduce on the logits under the rules, which are never written: per
 * live row the partials of x_hat and p go to the update workspace `upd_ws` in
 * the form fb_denoise_apply reads, so fb_rules_build + fb_vocab_reduce_rules
 * + fb_denoise_apply is fb_denoise_update on z'.  A row with nothing left (no
 * z' above -inf) has p = 0 and x_hat = -1; fb_denoise_apply never writes it.
 * Finite z' at or below -2^26 (masks of -1e9 or of the type's lowest value)
 * weigh nothing beside larger ones here, and count as equal, as -2^26, where
 * there are no larger ones; z' are at most 2^26.
 *   logits  [row_cap][V], dtype FB_BF16 or FB_F32, 16-byte aligned; an allowed
 *           entry is neither NaN nor +inf (others may hold anything)
 *   conf, argmax  [row_cap] float32 and int32: p and x_hat of the live rows, or
 *           both NULL
 *   rules_ws  what fb_rules_build wrote for these rules, pack and V
 *   upd_ws  device workspace of fb_update_workspace_bytes(pack, V) bytes,
 *           16-byte aligned */
int fb_vocab_reduce_rules(const void* logits, int V, int dtype, const fb_pack* pack,
                          const fb_logit_rules* rules, const void* rules_ws,
                          size_t rules_ws_bytes, void* upd_ws, size_t upd_ws_bytes,
                          float* conf, int32_t* argmax, void* stream);

/* The logits under the rules, z' rounded once to their type, for samplers of
 * the caller's own.
 *   logits, out  [row_cap][V], dtype FB_BF16 or FB_F32, 16-byte aligned; out
 *           may be logits
 * The other arguments as above. */
int fb_logits_rules(const void* logits, void* out, int V, int dtype,
                    const fb_pack* pack, const fb_logit_rules* rules,
                    const void* rules_ws, size_t rules_ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* FLOWBLOCK_TAIL_H */
