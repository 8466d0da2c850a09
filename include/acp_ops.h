/*
 * acp_ops.h - C ABI of the operators around the attention of acp.h: norms, rotary
 * positions and a paged cache with the attention of new tokens over it.
 *
 * Conventions are those of acp.h (device pointers owned by the caller, host checks
 * before any launch, error codes, `stream`, no allocation, no state), except:
 *   - Tensors described as strided take a pointer to three element strides
 *     {batch, head, position} (paged tensors: {token, head}); the features of a row
 *     are contiguous.  A null stride pointer means contiguous in the order stated.
 *     Strided tensors need only their element's alignment.  A stride is not negative.
 *   - Outputs must not overlap inputs unless said otherwise, nor each other; no two rows
 *     of an output may share memory.
 */
#ifndef ACP_OPS_H
#define ACP_OPS_H

#include "acp.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- Norms -----------------------------------------------------------------------
 * A row x of n features, with m = mean(x) (layer norm; 0 without `center`: RMS norm)
 * and r = 1 / sqrt(mean((x - m)^2) + eps):
 *   y = (x - m) r w + b,
 * evaluated in float32 and rounded once.  The mean is taken first and the squares of
 * the centred row after it.
 * Rows are [B, H, L] of them; `per_head` gives every head its own weight row (QK-norm:
 * x the head-split queries or keys, and gamma of acp_boundary_qknorm the largest |w| of
 * a head, see there for the rounding), otherwise all rows share one.
 *   in : x [B, H, L, n] dt, strided; weight, bias [H, n] or [n] of type wdt (bias may be
 *        null); eps >= 0.
 *   out: y [B, H, L, n] dt, contiguous; mean (with center), rstd [B, H, L] float, or
 *        both null when no backward follows.
 * Supported: 1 <= n <= 16384; H <= 65535; B*H*L <= 2^30; B, H, L >= 0 (no row: nothing is
 * done). */
acp_status acp_norm_fwd(const void* x, const int64_t* x_strides, const void* weight,
                        const void* bias, acp_dtype dt, acp_dtype wdt, int B, int H, int L, int n,
                        int per_head, int center, double eps, void* y, float* mean, float* rstd,
                        void* stream);

/* Gradients of acp_norm_fwd.  With g = dy w and xh = (x - m) r:
 *   dx = r (g - mean(g) [center only] - xh mean(g xh)),
 *   dweight = sum over rows of dy xh,  dbias = sum over rows of dy,
 * the sums in float32, in an order that depends on the shapes alone.
 *   in : dy, x [B, H, L, n] dt, strided; weight as above; mean (null without center),
 *        rstd as acp_norm_fwd left them.
 *   out: dx dt, strided; dweight, dbias (may be null) [H, n] or [n] float, overwritten.
 *        dx may be dy itself (same pointer and strides).
 *   ws : acp_norm_workspace_size() bytes of scratch. */
acp_status acp_norm_workspace_size(int B, int H, int L, int n, int per_head, size_t* bytes);
acp_status acp_norm_bwd(const void* dy, const int64_t* dy_strides, const void* x,
                        const int64_t* x_strides, const void* weight, acp_dtype dt, acp_dtype wdt,
                        int B, int H, int L, int n, int per_head, const float* mean,
                        const float* rstd, void* dx, const int64_t* dx_strides, float* dweight,
                        float* dbias, void* ws, size_t ws_bytes, void* stream);

/* ---- Rotary positions ---------------------------------------------------------------
 * Feature pairs of the first `rot` features of a row at position p are turned by the
 * angle p f_i, i < rot / 2, and scaled:
 *   (a, b) -> amplitude (a cos - b sin, a sin + b cos);
 * the pair is (i, i + rot/2) in the half layout and (2 i, 2 i + 1) interleaved; the
 * features from `rot` on are copied.  Angles are reduced in float64.  A rotation keeps a
 * row's norm, so a bound from QK-norm scales still holds for rotated rows (times
 * amplitude, and up to the rounding described at acp_boundary_qknorm). */
enum { ACP_ROTARY_HALF = 0, ACP_ROTARY_INTERLEAVED = 1 };

/* How frequencies base^(-2 i / rot) are scaled for contexts `factor` times as long:
 *   NONE    not at all
 *   LINEAR  f_i / factor (positions compressed)
 *   BASE    base times factor^(rot / (rot - 2)): the lowest frequency falls by factor
 *   RAMP    by the turns r_i = train_len f_i / (2 pi) that a pair makes over the
 *           training length: f_i where r_i >= fast, f_i / factor where r_i <= slow, and
 *           a linear mix between the two */
enum { ACP_SCALE_NONE = 0, ACP_SCALE_LINEAR = 1, ACP_SCALE_BASE = 2, ACP_SCALE_RAMP = 3 };

/* The rot / 2 frequencies, in turns (f_i / 2 pi) per position, into HOST memory.
 * rot even, 2 <= rot; BASE needs rot >= 4; base > 1; factor >= 1; RAMP needs
 * train_len > 0 and fast > slow >= 0. */
acp_status acp_rotary_table(int rot, double base, int scaling, double factor, double train_len,
                            double slow, double fast, double* turns);

/* q [B, H, L, d] and k [B, Hk, L, d] (either may be null, its outputs with it) turned in
 * one launch.
 *   in : q, k dt, strided; turns [rot / 2] double, DEVICE memory (acp_rotary_table's
 *        values); positions int32 or int64 (pos_bytes 4 or 8) with element strides
 *        pos_strides {batch, position} (0 allowed), or null: position l is start + l.
 *        inverse != 0 turns by the negative angle: the gradient (amplitude included).
 *   out: q_out, k_out dt, strided; each may be its input (same pointer and strides).
 * Supported: even d, rot <= d <= 1024; |position| < 2^31; H + Hk <= 65535;
 * B*L*(d/8 + 2) < 2^32. */
acp_status acp_rotary(const void* q, const int64_t* q_strides, const void* k,
                      const int64_t* k_strides, acp_dtype dt, int B, int H, int Hk, int L, int d,
                      int rot, int layout, int inverse, double amplitude, const double* turns,
                      const void* positions, int pos_bytes, const int64_t* pos_strides,
                      int64_t start, void* q_out, const int64_t* q_out_strides, void* k_out,
                      const int64_t* k_out_strides, void* stream);

/* ---- Paged cache -----------------------------------------------------------------------
 * Keys, values and cumulative gates of many sequences in pages of 64 positions, one
 * buffer:
 *   k, v [P, Hk, 64, d] dt; c [P, H, 64] double (H query heads, Hk key heads, H a
 *   multiple of Hk: query head h reads key head h / (H / Hk); every query head has its
 *   own gates).
 * Position p of sequence s lies in slot p mod 64 of page table[s][p / 64].  c holds the
 * cumulative gate c_p = log f_0 + .. + log f_p as float64, so that c_i - c_j keeps its
 * precision at any length.  A page holds all that its positions need: pages may be moved,
 * shared by sequences with a common prefix (while nobody appends to them), or dropped
 * once no sequence keeps them.  A slot not yet written is never used, whatever it holds.
 *
 * A call names its sequences by
 *   cu [N + 1] int32   sequence s brings the packed rows cu[s] .. cu[s + 1] - 1
 *                      (non-decreasing, cu[0] = 0; equal: no row); rows from cu[N] on
 *                      are left as they are
 *   past [N] int32     positions it holds before them: row cu[s] + r is position past[s] + r
 *   table [N, W] int32 its pages; entries that no position of it needs are not read
 * all device memory.  A page number outside [0, P), or a position beyond 64 W, is not
 * followed: what would be stored is dropped, what would be read is left out, and bit 6
 * of the sequence's flags is set (flags: [N, H] int32, overwritten; null: not reported;
 * bits as in acp.h).  A row outside [0, T) is not touched.
 * Supported: N <= 65535, T*H <= 2^26, N*H <= 2^22. */
typedef struct {
    size_t k;          /* [P,Hk,64,d] dt    */
    size_t v;          /* [P,Hk,64,d] dt    */
    size_t c;          /* [P,H,64] double   */
    size_t total;      /* bytes = acp_paged_cache_size() */
} acp_paged_layout;

/* Supported: d in {64, 128}; P, Hk >= 1; H a multiple of Hk with H / Hk <= 16; H <= 65535. */
acp_status acp_paged_cache_size(int P, int H, int Hk, int d, acp_dtype dt, size_t* bytes);
acp_status acp_paged_offsets(int P, int H, int Hk, int d, acp_dtype dt, acp_paged_layout* out);

/* Stores T new rows: keys and values [T, Hk, d] dt (strided, 16-byte aligned rows) into
 * their slots, and the cumulative gates from log_f [T, H] float (strided) on top of
 * c at position past - 1.  Storing the same rows at the same positions again leaves the
 * same pages.  Flag bit 0: some log f > 0; bit 1: not finite, or c of a new position is not finite
 * or outside the float32 range (a bad gate of an earlier call stays in every later sum);
 * bit 2: some finite |c| reaches 2^32, where float64 holds the differences of later gates to 2^-20
 * and less (a gate of the type's lowest value takes all their bits: the positions after it
 * no longer forget).
 * Two sequences of one call must not store to the same page. */
acp_status acp_paged_append(const void* k, const int64_t* k_strides, const void* v,
                            const int64_t* v_strides, const float* log_f,
                            const int64_t* f_strides, acp_dtype dt, int T, int N, int W, int P,
                            int H, int Hk, int d, const int32_t* cu, const int32_t* past,
                            const int32_t* table, void* cache, size_t cache_bytes, int32_t* flags,
                            void* stream);

/* Attention of the rows of q over the pages, after acp_paged_append of the same rows (the
 * same cu, past and table): the row at position i of head h attends to the positions
 * j <= i of its sequence with logit q.k / sqrt(d) + c_i - c_j.  With ACP (eps > 0) page
 * n < i / 64 is left out where c_i - c_{64 n + 63} < delta, delta = -(2 U + log L_max - log eps),
 * U = gamma_q[h] gamma_k[h / (H / Hk)] sqrt(d) (App. E, App. F: the row-wise block test of
 * fox_attn_decode); eps = 0 leaves nothing out and gamma_q, gamma_k may be null.  The scales
 * must bound the logits, |q.k| / sqrt(d) <= U up to rounding, as those of QK-normed rows do: U also
 * keeps the weights of chunks in bfloat16 in float32's range.  Where it does not (logits some 80 away
 * from what the scales allow) such a row may become infinite, NaN or 0 with lse = -inf; flag bit 8 says
 * that a row of the head did (also where q, k or c is not finite).  Single tokens and float32 do without.
 * The entries of pages that no row keeps any more may be set to -1 (and the pages used anew):
 * with eps > 0 the search for a row's first kept page takes an entry out of range for a page
 * that the test leaves out, and with it the pages before it, and reports neither.  An entry
 * out of range after that page is reported.
 *   in : q [T, H, d] dt (strided, 16-byte aligned rows); gamma_q [H], gamma_k [Hk] float.
 *        max_new bounds cu[s + 1] - cu[s] and max_len past[s] plus that; they choose
 *        the division of the work and size the workspace.  The rows of a sequence with
 *        more than max_new may be left as they are (flag bit 7 says they were); max_len is a
 *        hint, any value from 0 to 2^31: results stay right where it is too small or too large.
 *   out: O [T, H, d] dt, lse [T, H] float, contiguous; a row all of whose keys were
 *        left out by bad pages gets O = 0, lse = -inf; c_i counts as 0 where the row's own
 *        page is bad.
 *   ws : acp_paged_workspace_size() bytes.
 * A value that is not finite reaches the rows that attend to its position, and only them.
 * Flag bit 3: a negative or not finite gamma. */
acp_status acp_paged_workspace_size(int T, int N, int H, int Hk, int d, acp_dtype dt, int max_new,
                                    int64_t max_len, size_t* bytes);
acp_status fox_attn_paged(const void* q, const int64_t* q_strides, acp_dtype dt, int T, int N,
                          int W, int P, int H, int Hk, int d, const int32_t* cu,
                          const int32_t* past, const int32_t* table, const void* cache,
                          size_t cache_bytes, const float* gamma_q, const float* gamma_k,
                          double eps, int64_t L_max, int max_new, int64_t max_len, void* O,
                          float* lse, int32_t* flags, void* ws, size_t ws_bytes, void* stream);

/* The same, for outputs that hold nothing yet: the rows that fox_attn_paged leaves as they are (from
 * cu[N] on, and of a sequence with more than max_new where it says so) get O = 0, lse = -inf. */
acp_status fox_attn_paged_filled(const void* q, const int64_t* q_strides, acp_dtype dt, int T, int N,
                                 int W, int P, int H, int Hk, int d, const int32_t* cu,
                                 const int32_t* past, const int32_t* table, const void* cache,
                                 size_t cache_bytes, const float* gamma_q, const float* gamma_k,
                                 double eps, int64_t L_max, int max_new, int64_t max_len, void* O,
                                 float* lse, int32_t* flags, void* ws, size_t ws_bytes, void* stream);

/* Timing of these operators, as acp_timing_read() of the others: the same switch and
 * reset (acp_timing_enable, acp_timing_reset). */
enum {
    ACP_OP_NORM = 0,        /* acp_norm_fwd                              */
    ACP_OP_NORM_BWD = 1,    /* acp_norm_bwd, the weight's sum included   */
    ACP_OP_ROTARY = 2,
    ACP_OP_APPEND = 3,
    ACP_OP_ATTEND = 4,      /* fox_attn_paged(_filled), the merge of parts included */
    ACP_OP_COUNT = 5
};
typedef struct {
    int64_t launches[ACP_OP_COUNT];
    double ms[ACP_OP_COUNT];
} acp_op_times;
acp_status acp_op_timing_read(acp_op_times* out);

#ifdef __cplusplus
}
#endif

#endif /* ACP_OPS_H */
