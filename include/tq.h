/*
 * tq.h — packed ternary GEMV for AMD Instinct MI355X (gfx950): C ABI.
 *
 * The operation (paper arXiv 2609.09240, section 3, eq. 3, and the footnote
 * to section 3): a linear projection is stored as
 *     W^ = (mu + a0*T0 + a1*T1) (.) M,   T_i in {-1, 0, +1},
 * where every 128-wide group of a row carries plane T0 with an fp16 scale
 * s0, and a selected subset of groups also carries plane T1 with an fp16
 * offset mu and an fp16 scale s1.  On such a two-plane group every weight is
 * mu + s0*t0 + s1*t1; elsewhere it is s0*t0.  Activations stay fp16 (A16,
 * section 3).  The packed format persists the discrete supports losslessly
 * (section 12): five trits per byte as a base-3 code.
 *
 * ------------------------------------------------------------------------
 * Packed format (the paper fixes no byte layout; this is the library's).
 *
 *   Group: 128 trits t[0..127] of one row, input indices 128g .. 128g+127.
 *   Code byte j (j = 0..25) holds trits 5j .. 5j+4:
 *       code = sum_{i=0..4} (t[5j+i] + 1) * 3^i          (0 .. 242)
 *   Byte 25 holds t[125..127] in digits 0..2; its digits 3 and 4 are 1
 *   (trit 0), so a valid last byte lies in 108..134.  Codes 243..255 are
 *   invalid.
 *   A code buffer of n groups is 26*n bytes in the "split" layout: bytes
 *   0..23 of group f at offset 24*f, bytes 24 and 25 of group f at offset
 *   24*n + 2*f.  (Every group body is 8-byte aligned for vector loads.)
 *
 *   A packed linear of N outputs and K inputs (K % 128 == 0, G = K/128):
 *     codes0   uint8  [26*N*G]   plane 0, groups in row-major (r, g) order
 *     scale0   fp16   [N][G]     s0
 *     rowptr1  int32  [N+1]      CSR over rows of the two-plane groups
 *     gidx1    uint16 [nnz1]     group index of each record; strictly
 *                                increasing within a row
 *     codes1   uint8  [26*nnz1]  plane 1 of each record (split layout)
 *     offset1  fp16   [nnz1]     mu
 *     scale1   fp16   [nnz1]     s1
 *
 * ------------------------------------------------------------------------
 * Conventions for every entry point.
 *
 *   - Pointers to data are DEVICE pointers (hipMalloc / torch tensors on
 *     the GPU) unless stated otherwise; tq_matrix itself lives in host
 *     memory and is read only during the call.  The caller owns every
 *     buffer; the library keeps no state and allocates no memory.
 *   - `stream` is a hipStream_t (NULL = the default stream).  Every call is
 *     asynchronous on that stream; nothing synchronises.
 *   - Argument errors (NULL pointers, bad sizes or alignment, group != 128)
 *     are detected on the host before anything is launched and returned
 *     synchronously.  A failed launch returns TQ_ERR_HIP.
 *   - Data errors (invalid trits or codes) are reported asynchronously
 *     through an optional device counter `d_err` (int32, may be NULL),
 *     which is incremented, never reset, by the number of bad bytes.
 *   - tq_gemv, tq_gemv_grouped and tq_gemm_smallbatch do not validate codes:
 *     invalid codes give unspecified (but finite-time, in-bounds) results.
 *     Validate a matrix once with tq_validate when it is loaded.
 *   - Results are deterministic: the same inputs give bit-identical outputs
 *     on every run.
 *   - Fp16 values are passed as their uint16 bit patterns.
 */
#ifndef TQ_H
#define TQ_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define TQ_ABI_VERSION 7
#define TQ_GROUP 128
#define TQ_GROUP_BYTES 26
#define TQ_MAX_GROUPS_PER_ROW 256    /* K <= 32768 */
#define TQ_MAX_GROUPED 8             /* matrices per tq_gemv_grouped call */
#define TQ_MAX_BATCH 64              /* rows of X in tq_gemm_smallbatch */
#define TQ_SELECT_NOALLOC_MAX_GROUPS (1 << 24)  /* n_out * groups_per_row in
                                                   tq_select_two_plane_noalloc */

/* Output element type for tq_gemv / tq_gemm_smallbatch (the `flags` word). */
#define TQ_OUT_FP16 0   /* fp16, rounded to nearest even from fp32 */
#define TQ_OUT_FP32 1   /* the fp32 accumulator, unrounded */

typedef enum {
  TQ_OK = 0,
  TQ_ERR_NULL = 1,        /* a required pointer is NULL */
  TQ_ERR_SHAPE = 2,       /* a size is out of range or inconsistent */
  TQ_ERR_ALIGN = 3,       /* a pointer is not aligned as required */
  TQ_ERR_UNSUPPORTED = 4, /* a valid request this build does not support */
  TQ_ERR_HIP = 5          /* the HIP runtime reported an error */
} tq_status;

/* Non-owning view of one packed linear (layout above).  When nnz1 == 0 the
 * plane-1 pointers are ignored and may be NULL. */
typedef struct tq_matrix {
  int64_t n_out;            /* N >= 1 */
  int64_t n_in;             /* K >= 128, K % 128 == 0, K/128 <= TQ_MAX_GROUPS_PER_ROW;
                               26 * N * K/128 must be below 2^32 (codes of one
                               matrix under 4 GiB) */
  int32_t group;            /* must be 128 */
  int32_t reserved;         /* must be 0 */
  const uint8_t* codes0;    /* 8-byte aligned */
  const uint16_t* scale0;   /* 2-byte aligned */
  int64_t nnz1;             /* 0 <= nnz1 <= N*G */
  const int32_t* rowptr1;   /* 4-byte aligned; rowptr1[0] == 0, rowptr1[N] == nnz1 */
  const uint16_t* gidx1;
  const uint8_t* codes1;    /* 8-byte aligned */
  const uint16_t* offset1;
  const uint16_t* scale1;
  /* Optional (may be NULL): a HOST copy of rowptr1, read during the call
   * only.  With it the GEMV and the small-batch kernels find every
   * workgroup's records on the host and issue their loads with their first
   * batch, instead of reading the device row pointers first (B = 2..4 use
   * the GEMV's decode only when it is present).  It must hold the same
   * values as rowptr1; if it does not, results are unspecified, but every
   * access stays in bounds. */
  const int32_t* rowptr1_host;
  /* Optional (may be NULL; ABI 3): fp16 [N][G] offset mu0 of EVERY group,
   * the paper's representation (eq. 3 gives every masked block an offset).
   * Each weight of group (r, g) is then mu0[r][g] + s0*t0, plus
   * mu + s1*t1 on two-plane groups; the accuracy bound adds |mu0| to the
   * group's coefficient.  2-byte aligned. */
  const uint16_t* offset0;
} tq_matrix;

/* Version of this ABI (TQ_ABI_VERSION). */
int tq_abi_version(void);

/* Static, human-readable name of a status code. */
const char* tq_status_string(tq_status status);

/* Encode trits to lattice codes (section 12: lossless encoding of the
 * discrete supports).
 *   trits   int8 [n_groups][128], values in {-1, 0, +1}
 *   codes   uint8 [26*n_groups], split layout; 8-byte aligned
 *   n_groups >= 0 (0 is a no-op); group must be 128.
 * A code byte whose five trits include a value outside {-1, 0, +1} is
 * written as 0xFF and counted in *d_err. */
tq_status tq_pack(const int8_t* trits, int64_t n_groups, int32_t group,
                  uint8_t* codes, int32_t* d_err, void* stream);

/* Decode lattice codes to trits (inverse of tq_pack; bit-exact).
 *   codes   uint8 [26*n_groups], split layout; 8-byte aligned
 *   trits   int8 [n_groups][128]
 * A code above 242 decodes to five zero trits and is counted in *d_err.
 * The pad digits of byte 25 are not inspected (see tq_validate). */
tq_status tq_unpack(const uint8_t* codes, int64_t n_groups, int32_t group,
                    int8_t* trits, int32_t* d_err, void* stream);

/* Count invalid bytes of a code buffer into *d_err (required here): codes
 * above 242, and last bytes (byte 25) whose pad digits are not both 1.
 * Section 12 makes the packed buffer the lossless carrier of the discrete
 * supports; section 5.4 reports malformed packed tensors that still gave
 * plausible-looking numbers, and section 15 lists such artifact failures.
 * So a loader checks a buffer once with this call; the GEMV does not. */
tq_status tq_validate(const uint8_t* codes, int64_t n_groups, int32_t group,
                      int32_t* d_err, void* stream);

/* Dense fp16 dequantisation of a packed linear (eq. 3).
 *   w  fp16 [N][K] row-major; 16-byte aligned
 * Each weight is evaluated in fp32 in the fixed order
 *     a = +0;  a += mu0;  a += mu;  a += s0*t0;  a += s1*t1
 * (mu0 only with per-group offsets, mu and s1 only on two-plane groups;
 * s*t is exact) and rounded once to fp16, nearest-even, so the result is
 * bit-exact and unique. */
tq_status tq_unpack_fp16(const tq_matrix* m, uint16_t* w, void* stream);

/* y = W^ x for one fp16 activation vector (the decode-time GEMV).
 *   x  fp16 [K]; 16-byte aligned
 *   y  [N], fp16 (flags = TQ_OUT_FP16) or fp32 (TQ_OUT_FP32); 4-byte aligned
 * Accumulates sign-selected fp16 activations in fp32, applies s0 (and
 * mu0*sum(x_g) with per-group offsets) per group and mu*sum(x_g) +
 * s1*sum(t1*x_g) per two-plane group.  Accuracy:
 * |y - exact| <= 2e-3 * sum_g (|s0| + |mu0| + [two-plane](|mu| + |s1|)) *
 * ||x_g||_1 per output (|mu0| only with per-group offsets).  x and y must
 * not overlap the matrix buffers.  Where x_g holds an infinity or NaN the
 * sums above are taken as they stand: a trit of 0 under an infinity makes
 * them, and the output, NaN. */
tq_status tq_gemv(const tq_matrix* m, const uint16_t* x, void* y,
                  int32_t flags, void* stream);

/* Several GEMVs that read the same x in one launch (e.g. q, k and v, or
 * gate and up of one decoder layer).  Section 13 measures the packed decode
 * step of a whole model; in a decoder layer q, k, v read the same normalised
 * input and so do gate and up, so one launch serves each pair or triple.
 *   ms  host array of n matrices (1 <= n <= TQ_MAX_GROUPED), all with the
 *       same K
 *   ys  host array of n device output pointers, ys[i] of N_i elements
 * Each ys[i] equals what tq_gemv(&ms[i], x, ys[i], flags) produces,
 * bit for bit. */
tq_status tq_gemv_grouped(const tq_matrix* ms, int32_t n, const uint16_t* x,
                          void* const* ys, int32_t flags, void* stream);

/* Y = X W^T for a small batch of activations (paper section 18 lists kernel
 * work across batch sizes as the next step).
 *   X  fp16 [B][K] row-major; 16-byte aligned; 1 <= B <= TQ_MAX_BATCH
 *   Y  [B][N] row-major, fp16 or fp32 per flags; 4-byte aligned
 * Same accuracy bound as tq_gemv for every (b, r).  A row's result depends on
 * the row and on B, not on the other rows.
 * B = 1 is tq_gemv.  B = 2..4 take tq_gemv's sums in its order, so that every
 * row equals tq_gemv of that row (+0 and -0 aside), where the matrix has no
 * records or carries rowptr1_host, B rows of x and the records' sums fit in
 * LDS beside the decode table (B * K up to about 40000: K = 12288 at B = 3,
 * not at B = 4) and the outputs fit in 767 workgroups (49000 at K = 4096 and
 * B = 4, fewer at a larger K).  All other calls add on the matrix cores, in
 * another order.
 * Inputs, scales and offsets that are not finite: on the matrix cores the
 * output is what the weights, formed one by one as tq_unpack_fp16 forms them
 * (unrounded), give with X's row (an infinite input times a weight of 0 is
 * NaN, times a weight that an offset makes nonzero +-inf); with tq_gemv's sums
 * a trit of 0 under an infinite input gives NaN whatever the offsets are. */
tq_status tq_gemm_smallbatch(const tq_matrix* m, const uint16_t* X, int32_t B,
                             void* Y, int32_t flags, void* stream);

/* E2M-ATQ ternarisation of 128-weight groups: the planes and scales this
 * format stores, from dense fp16 weights (section 4.2, eqs. 4-6; the
 * representation of section 3, eq. 3).
 *   w          fp16 [n_groups][128], row-major groups; 16-byte aligned
 *   rec_index  int32 [n_groups], or NULL (every group one-plane): -1 for a
 *              one-plane group, k in [0, nnz) for a two-plane group whose
 *              second plane is written as record k (values outside that
 *              range are one-plane).  Records must be distinct: groups
 *              naming the same record, and records no group names, are left
 *              with unspecified contents (always in bounds).
 *   nnz        number of records (rows of t1, offset1, scale1), >= 0
 *   iters      refinement sweeps of every fit that has an offset (two-plane
 *              groups; with offset0 also one-plane groups), 0..1024
 *   t0         int8 [n_groups][128] (16-byte aligned), s0 fp16 [n_groups]
 *   t1         int8 [nnz][128] (16-byte aligned), offset1 and scale1 fp16
 *              [nnz]; may be NULL when nnz == 0
 *   offset0    fp16 [n_groups] or NULL.  Given, every group gets an offset
 *              (the paper's representation, tq_matrix.offset0): one-plane
 *              groups are fitted like the first plane below (mu = mean(w),
 *              then `iters` sweeps of mu <- mean(w - s0*T0),
 *              s0 <- <T0, w - mu>/<T0, T0>), two-plane groups store their mu
 *              here and +0 in offset1.
 *   energy     fp64 [n_groups] or NULL: ||w - mu - s0*T0||^2 of each
 *              group's one-plane fit (mu = 0 without offset0), the ranking
 *              used to choose two-plane groups
 * One-plane groups without offset0: T0 = +1 / -1 where w exceeds
 * +0.75 mean|w| / is below its negation, else 0; s0 = <T0, w> / <T0, T0>
 * (0 on an empty support).
 * Two-plane groups: mu = mean(w); T0, s0 as above on w - mu; T1, s1 the
 * same way on the residual w - mu - s0*T0; then `iters` sweeps updating mu,
 * s0 and s1 in turn with T0, T1 fixed.  Arithmetic is fp64 with every sum
 * in index order; mu, s0, s1 are rounded once to fp16 (nearest even), so
 * results are bit-exact and unique.  All buffers are device memory. */
tq_status tq_ternarize(const uint16_t* w, int64_t n_groups, int32_t group,
                       const int32_t* rec_index, int64_t nnz, int32_t iters,
                       int8_t* t0, uint16_t* s0, int8_t* t1, uint16_t* offset1,
                       uint16_t* scale1, uint16_t* offset0, double* energy,
                       void* stream);

/* Bytes of device workspace tq_select_two_plane needs for n_groups groups
 * (host function; 0 for n_groups < 0). */
size_t tq_select_workspace_bytes(int64_t n_groups);

/* The two-plane groups of a linear and its plane-1 CSR (ABI 5).  Section
 * 4.2 gives a second ternary plane to a minority of blocks; section 3
 * chooses them with salience masks fitted on calibration activations, so
 * without calibration data the ranking is each group's one-plane residual
 * energy (tq_ternarize's `energy`).  The call selects the nnz groups with
 * the largest energy, ties to the lower flat index (groups in row-major
 * (r, g) order); a NaN energy ranks below every number, -0 and +0 tie.
 * Records are numbered in flat order, which is the CSR order by row.
 *   energy          fp64 [n_out * groups_per_row]; 8-byte aligned
 *   n_out >= 1, 1 <= groups_per_row <= TQ_MAX_GROUPS_PER_ROW,
 *   n_out * groups_per_row < 2^31
 *   nnz             0 <= nnz <= n_out * groups_per_row
 *   rec_index       int32 [n_out * groups_per_row] out: the record of each
 *                   group, -1 for one-plane groups (tq_ternarize's input)
 *   rowptr1         int32 [n_out + 1] out (tq_matrix.rowptr1)
 *   gidx1           uint16 [nnz] out (tq_matrix.gidx1); may be NULL when
 *                   nnz == 0
 *   workspace       device scratch of workspace_bytes >=
 *                   tq_select_workspace_bytes(n_out * groups_per_row)
 *                   bytes, 256-byte aligned; its contents on entry do not
 *                   matter and on return are unspecified.  Two calls that
 *                   share a workspace must not overlap in time.
 * All pointers are device memory; 4-byte alignment for rec_index and
 * rowptr1, 2-byte for gidx1.  The result is deterministic and unique. */
tq_status tq_select_two_plane(const double* energy, int64_t n_out, int32_t groups_per_row, int64_t nnz,
                              int32_t* rec_index, int32_t* rowptr1, uint16_t* gidx1,
                              void* workspace, size_t workspace_bytes, void* stream);

/* tq_select_two_plane without a workspace argument (ABI 6), for callers
 * that cannot allocate device memory: code under HIP graph capture, serving
 * loops that must not call hipMalloc, harnesses that forbid it.  Same
 * arguments (less the workspace), same result bit for bit.  The scratch is
 * a static array in the library, one per GPU (about 65 KB, held until the
 * process ends), sized for n_out * groups_per_row <=
 * TQ_SELECT_NOALLOC_MAX_GROUPS; larger requests return TQ_ERR_UNSUPPORTED
 * before anything is launched.  The call allocates nothing.  Every call on
 * one GPU shares that GPU's scratch, so calls that overlap in time on one
 * GPU (other streams, other host threads) race and give unspecified
 * results; order them on one stream. */
tq_status tq_select_two_plane_noalloc(const double* energy, int64_t n_out, int32_t groups_per_row, int64_t nnz,
                                      int32_t* rec_index, int32_t* rowptr1, uint16_t* gidx1, void* stream);

/* ------------------------------------------------------------------------
 * Decode-step chain (ABI 7): a sequence of dependent grouped GEMVs in one
 * launch.  Section 13 runs the packed model's whole decode step; within a
 * decoder layer q, k and v read one input, o the attention output, gate and
 * up the normalised residual and down the activated MLP state, so at batch
 * 1 the step is a chain of GEMVs, each waiting for the one before.  Stage s
 * computes exactly what tq_gemv_grouped(stage s) computes (bit for bit),
 * and reads its x only after every output of stage s - 1 is written, so x
 * may be (or be derived by device code in a later design from) an earlier
 * stage's output.  One launch of one 1024-thread workgroup per CU
 * runs every stage; each workgroup keeps the decode table across stages.
 */
typedef struct tq_stage {
  const tq_matrix* mats;   /* host array of n matrices, all with the same n_in */
  int32_t n;               /* 1 .. TQ_MAX_GROUPED */
  int32_t flags;           /* TQ_OUT_FP16 or TQ_OUT_FP32 */
  const uint16_t* x;       /* device fp16 [n_in]; 16-byte aligned */
  void* const* ys;         /* host array of n device outputs (4-byte aligned) */
} tq_stage;

typedef struct tq_chain_info {
  int32_t n_stages;
  int32_t n_workgroups;    /* one per CU of the device current at planning */
  int32_t lds_bytes;       /* dynamic LDS per workgroup */
  int32_t reserved;
  int64_t plan_bytes;      /* 128 * n_stages * n_workgroups */
  int64_t sync_bytes;      /* 256 + 64 * n_workgroups */
} tq_chain_info;

/* Plan a chain for the current device.  Checks every stage (as tq_gemv_
 * grouped does) and fills *info.  With plan_host != NULL it also writes the
 * plan, a table of info->plan_bytes bytes of device pointers and row
 * ranges, into that HOST buffer (plan_host_bytes >= info->plan_bytes); the
 * caller copies it unchanged to device memory (128-byte aligned) and keeps
 * every buffer the stages name alive while the plan is used.  Record
 * ranges come from the matrices' host row pointers where present.  Returns
 * TQ_ERR_UNSUPPORTED for a stage that does not fit one round of workgroups
 * (more than 6 row passes per workgroup) or the LDS. */
tq_status tq_chain_plan(const tq_stage* stages, int32_t n_stages, tq_chain_info* info,
                        void* plan_host, size_t plan_host_bytes);

/* Zero a sync block (device memory, info->sync_bytes bytes, 256-byte
 * aligned) on `stream`; required once before its first tq_gemv_chain and
 * whenever it is reused for a plan with another stage count.  Layout: word
 * 0 counts completed calls, word 2 (int32 at byte 8) is a sticky error flag
 * that a call sets when one of its waits gave up (after about 0.1 s; the
 * outputs of that call are then unspecified).  The rest is the library's own:
 * the running call's finished workgroups (word 1), its mode (word 16) and
 * tickets (word 32), which every call finds and leaves 0, and behind byte 256
 * one 64-byte slot per work item of a stage.  Nothing but the error flag may
 * be written; a block whose call did not run to its end (a device reset, a
 * copy taken meanwhile) goes through this function again. */
tq_status tq_chain_sync_init(void* sync, const tq_chain_info* info, void* stream);

/* Run every stage of a planned chain on `stream` (one launch).  `plan` is
 * the device copy of the plan, `sync` a sync block of this plan.  Calls on
 * one sync block must not overlap in time. */
tq_status tq_gemv_chain(const void* plan, void* sync, const tq_chain_info* info, void* stream);

/* ------------------------------------------------------------------------
 * The 4-bit side of a decode step: products with 4-bit weights (an output
 * head, a projection kept at 4 bits) and a paged key/value cache held in 4
 * bits with the attention that reads it.  All of it is added to ABI 7;
 * nothing above changed.
 *
 * A value is offset + scale * code, code 0..15, with an fp16 scale and
 * offset per group of 32, 64 or 128 values that lie next to each other.
 * Quantising a group x of fp16 values (tq_q4_quantize, tq_kv_append), in
 * fp32 with every operation rounded to nearest even:
 *     offset = min x;  scale = fp16((max x - min x) / 15);
 *     code   = clamp(rint((x - offset) / scale), 0, 15), 0 where scale is 0.
 * A group that holds an infinity or a NaN gets NaN for scale and offset (its
 * codes are 0), so that its values read back as NaN.
 *
 * Codes lie in 32-bit words of eight: the nibble 0, 4, 1, 5, 2, 6, 3, 7 of
 * the word (nibble 0 the lowest four bits) holds element 0, 1, ..., 7.
 */
#define TQ_Q4_MAX_BATCH 64      /* rows of X in tq_q4_gemm */
#define TQ_Q4_MAX_OUT (1 << 26)  /* outputs and inputs of a 4-bit matrix */
#define TQ_Q4_MAX_IN (1 << 20)
#define TQ_KV_MAX_ROWS 1024     /* rows of a call that changes the page table */
#define TQ_KV_MAX_PAGES (1 << 20)   /* pages of one sequence */
#define TQ_KV_MAX_HEADS 65520       /* query heads in tq_kv_attention */
/* The workspaces of tq_q4_gemm and tq_kv_attention hold counts that every
 * call finds and leaves 0, all of them in the first TQ_WORKSPACE_COUNT_BYTES:
 * only those are to be filled with zeros, once, before a workspace's first
 * call.  One that is large enough serves calls of both. */
#define TQ_WORKSPACE_COUNT_BYTES 16384

/* Non-owning view of a matrix of 4-bit weights.  N and K may be any sizes;
 * the last tile of rows and the last 128 inputs are filled up with codes and
 * parameters of 0 (written by tq_q4_quantize).
 *   codes   words [ceil(N/16)][ceil(K/128)][c 4][row 16][j 4]: the word of
 *           row 16 T + r holds inputs 128 B + 32 j + 8 c + (0..7)
 *   params  fp16 (scale, offset) pairs [ceil(N/16)][128/group * ceil(K/128)]
 *           [row 16] */
typedef struct tq_q4_matrix {
  int64_t n_out;            /* N, 1 .. TQ_Q4_MAX_OUT; at most 2^24 - 1 tiles in all */
  int64_t n_in;             /* K, 1 .. TQ_Q4_MAX_IN */
  int32_t group;            /* 32, 64 or 128 */
  int32_t reserved;         /* must be 0 */
  const uint8_t* codes;     /* 16-byte aligned, tq_q4_code_bytes */
  const uint16_t* params;   /* 16-byte aligned, tq_q4_param_bytes */
} tq_q4_matrix;

/* Bytes of the two buffers of a matrix (host functions; 0 for sizes or
 * groups that are not supported). */
size_t tq_q4_code_bytes(int64_t n_out, int64_t n_in);
size_t tq_q4_param_bytes(int64_t n_out, int64_t n_in, int32_t group);

/* Quantise fp16 weights w [N][K] (rows ldw >= K elements apart) into the
 * buffers of `m` (written through `codes` and `params`, which the caller
 * owns).  A group of the last, shorter kind covers the inputs that are
 * there. */
tq_status tq_q4_quantize(const uint16_t* w, int64_t ldw, const tq_q4_matrix* m,
                         uint8_t* codes, uint16_t* params, void* stream);

/* Dense fp16 w [N][K] of a 4-bit matrix: offset + scale * code in fp32 (one
 * rounding), then rounded to fp16.  w is 2-byte aligned. */
tq_status tq_q4_unpack_fp16(const tq_q4_matrix* m, uint16_t* w, void* stream);

/* Bytes of workspace with which tq_q4_gemm is fastest (host function). */
size_t tq_q4_workspace_bytes(const tq_q4_matrix* m, int32_t B);

/* Y = X W^T for B = 1..TQ_Q4_MAX_BATCH rows of fp16 activations.
 *   X  fp16, rows ldx >= K elements apart; 2-byte aligned
 *   Y  [B][N], fp16 (TQ_OUT_FP16) or fp32 (TQ_OUT_FP32); 4-byte aligned
 *   workspace  NULL, or tq_q4_workspace_bytes of the same arguments (0 for
 *      most), 16-byte aligned: with it K is split among workgroups where more
 *      than 16 rows meet few outputs.  Its counts (TQ_WORKSPACE_COUNT_BYTES)
 *      are filled with zeros once; it serves any calls that do not overlap in
 *      time.
 * scale * sum(code * x) + offset * sum(x) per group, every product exact,
 * sums in fp32; a row's result depends on the row, on the range of B (1 or 2,
 * 3 or 4, 5..16, 17..32, 33..64) and on whether there is a workspace, not on
 * the other rows.  Where that is not finite
 * the output is the fp32 sum of x times the weights formed one by one, so an
 * infinite input under a weight that is not 0 gives an infinity. */
tq_status tq_q4_gemm(const tq_q4_matrix* m, const uint16_t* X, int64_t ldx,
                     int32_t B, void* Y, int32_t flags, void* workspace,
                     size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------------
 * Key/value cache held in 4 bits, in pages.
 *
 * A page holds page_size tokens of one layer, all key/value heads: per head
 * page_size / 32 records of 32 tokens,
 *     key codes    words [half 2][c 4][t 16][j D/32]: channels 32 j + 8 c +
 *                  (0..7) of token 16 half + t
 *     value codes  words [D/64][c 4][ch 16][jd 4]: channel 64 l + 16 jd + ch
 *                  of tokens 4 c + i (nibble i) and 16 + 4 c + i (nibble
 *                  4 + i)
 *     key params   fp16 (scale, offset) [D/group][token 32]
 *     value params likewise
 * so that a wave's 16-byte loads of a record are the operands of its matrix
 * instructions.  Sequences live in slots: `pages` names the pages of a slot
 * in order (the same pages in every layer), `lens` the tokens it holds, and
 * refs[p] how many slots name page p (0: free).  All of the table is device
 * memory that the calls below read and write in stream order; no call waits
 * for the device, and the caller never needs to read it.
 *
 * Calls that take rows work on n_rows slots, seqs[i] (device int32 [n_rows];
 * NULL: slot i).  A slot outside the cache and a slot named twice in a call
 * that changes the table (the first one counts) are left out and counted in
 * *d_err (device int32, may be NULL), like every other request that a call
 * below says it refuses.  Where a table names no page of the pool (-1), its
 * tokens are neither written nor read.
 */
typedef struct tq_kv_cache {
  int32_t n_layers;         /* 1 .. 65535 */
  int32_t n_kv_heads;       /* 1 .. 1024 */
  int32_t head_dim;         /* D: 64, 128 or 256 */
  int32_t group;            /* 32, 64 or 128, at most D */
  int32_t page_size;        /* tokens: 32, 64, 128, 256, 512 or 1024 */
  int32_t n_seqs;           /* slots */
  int32_t max_pages;        /* pages of a slot, 1 .. TQ_KV_MAX_PAGES */
  int32_t reserved;         /* must be 0 */
  int64_t n_pages;          /* pages of the pool, 1 .. 2^30 */
  uint8_t* data;            /* [n_layers][n_pages][tq_kv_page_bytes]; 16-byte aligned */
  int32_t* pages;           /* [n_seqs][max_pages], -1 where there is none */
  int32_t* lens;            /* [n_seqs] */
  int32_t* refs;            /* [n_pages] */
} tq_kv_cache;

/* Rows of fp16 vectors: element d of head h of token t at
 * data[t * token_stride + h * head_stride + d]; 2-byte aligned. */
typedef struct tq_kv_rows {
  const uint16_t* data;
  int64_t token_stride;
  int64_t head_stride;
} tq_kv_rows;

/* Bytes of one page of one layer (host function; 0 for a cache whose sizes
 * are not supported). */
size_t tq_kv_page_bytes(const tq_kv_cache* cache);

/* Room for new tokens.  Row i gets cu_new[i+1] - cu_new[i] tokens (device
 * int32 [n_rows + 1]; NULL: one each): the pages it lacks are taken from the
 * free ones, lowest first, rows in order, its length grows, and starts[i]
 * (device int32 [n_rows]) becomes the length it had.  A row whose pages are
 * not there (more than are free behind the rows before it, or than max_pages)
 * and one whose last page is partly filled and shared keep their length, get
 * starts[i] = -1 and count in *d_err; the pages such a row asked for are not
 * given to later rows of the call. */
tq_status tq_kv_extend(const tq_kv_cache* cache, const int32_t* seqs, const int32_t* cu_new,
                       int32_t n_rows, int32_t* starts, int32_t* d_err, void* stream);

/* Give back every page of the rows' slots (a page is free once no slot
 * names it) and empty them. */
tq_status tq_kv_free(const tq_kv_cache* cache, const int32_t* seqs, int32_t n_rows,
                     int32_t* d_err, void* stream);

/* Bytes of workspace for tq_kv_fork of n_rows rows and for tq_kv_compact
 * (n_rows = 0). */
size_t tq_kv_workspace_bytes(const tq_kv_cache* cache, int32_t n_rows);

/* Slots children[i] become copies of slots parents[i], as those are before
 * the call: full pages are shared, a last page that is partly filled is
 * copied (all layers) into a page of its own, lowest free page first, rows in
 * order.  Refused: a child that holds tokens, is its own parent or comes
 * twice, and a child whose page is not there.  Workspace: 16-byte aligned. */
tq_status tq_kv_fork(const tq_kv_cache* cache, const int32_t* parents, const int32_t* children,
                     int32_t n_rows, int32_t* d_err, void* workspace, size_t workspace_bytes,
                     void* stream);

/* Move pages so that the n pages in use become pages 0 .. n-1: the k-th page
 * in use at or above n moves, in all layers, into the k-th free page below
 * n, and the table and the counts follow.  n_live (device int32 [1], may be
 * NULL) gets n; every byte of data behind page n-1 of a layer is free then.
 * Workspace: 16-byte aligned. */
tq_status tq_kv_compact(const tq_kv_cache* cache, int32_t* n_live, void* workspace,
                        size_t workspace_bytes, void* stream);

/* Copy whole pages src[i] -> dst[i] (device int32 [n], n <= 65535) in all layers; the
 * table stays as it is.  No page may be a destination twice, or a source
 * and a destination.  Pairs with a page outside the pool are refused. */
tq_status tq_kv_copy_pages(const tq_kv_cache* cache, const int32_t* src, const int32_t* dst,
                           int32_t n, int32_t* d_err, void* stream);

/* Quantise new keys and values of one layer into the cache.  Row i's tokens
 * are cu_new[i] .. cu_new[i+1]-1 of k and v (NULL: token i; at most max_new
 * a row, n_tokens in all) and go to positions starts[i], starts[i] + 1, ...
 * of its slot; a row with starts[i] < 0 is left out.  n_rows <= 65535,
 * max_new <= 2^26.  Tokens past max_new,
 * past n_tokens or without a page are left out and the row counts in *d_err
 * (once).  Two rows of a call may not write the same record. */
tq_status tq_kv_append(const tq_kv_cache* cache, int32_t layer, const int32_t* seqs,
                       const int32_t* starts, const int32_t* cu_new, int32_t n_rows,
                       int32_t n_tokens, int32_t max_new, const tq_kv_rows* k,
                       const tq_kv_rows* v, int32_t* d_err, void* stream);

/* The values of cached tokens as fp16 k_out, v_out [n_tokens][n_kv_heads][D]
 * (offset + scale * code in fp32, rounded to fp16; 16-byte aligned), rows and
 * positions as in tq_kv_append.  What has no page, and every token of a row
 * with starts[i] < 0, reads as 0. */
tq_status tq_kv_read(const tq_kv_cache* cache, int32_t layer, const int32_t* seqs,
                     const int32_t* starts, const int32_t* cu_new, int32_t n_rows,
                     int32_t n_tokens, int32_t max_new, uint16_t* k_out, uint16_t* v_out,
                     void* stream);

/* Attention of n_rows rows over their slots' pages of one layer.  Row i's
 * queries are tokens cu_q[i] .. cu_q[i+1]-1 of q (NULL: token i, one a row),
 * the last tokens of its slot: query t of n sits at position p = lens - n +
 * t and attends to the positions j <= p, and j > p - window where window > 0.
 * Query head h reads key/value head h / (n_heads / n_kv_heads).
 *     o = sum_j softmax_j(scale * q . k_j) v_j;   lse = log sum_j exp(scale * q . k_j)
 * A query with nothing to attend to gives o = 0 and lse = -infinity.
 * Positions whose page the table does not name are left out.  Tokens past
 * max_q of a row and past n_tokens are not computed.
 *   max_len  the longest length among the slots, as far as the caller knows
 *            (0: max_pages * page_size).  It decides how the work is split,
 *            not what is read: longer slots are right, and slower.
 *   o        [n_tokens][n_heads][D], fp16 or fp32 per flags; 16-byte aligned
 *   lse      fp32 [n_tokens][n_heads], may be NULL
 * Products are exact, the softmax, its sums and o's are fp32; a probability
 * times the scale of a value enters the matrix instructions as two fp16
 * numbers, 22 bits of it; what lies below 2^-37 of the largest probability
 * times the group's largest scale is rounded off.
 * The workspace (16-byte aligned, tq_kv_attention_workspace_bytes of the same
 * arguments, which may be 0) holds what the parts of a long cache give, and
 * counts of them (TQ_WORKSPACE_COUNT_BYTES, filled with zeros once); it serves
 * any calls that do not overlap in time. */
typedef struct tq_kv_attn {
  int32_t n_rows;           /* >= 1 */
  int32_t n_tokens;         /* tokens of q and o, >= 1 */
  int32_t max_q;            /* queries of a row, >= 1 */
  int32_t n_heads;          /* a multiple of n_kv_heads, up to TQ_KV_MAX_HEADS;
                               n_tokens * n_heads < 2^31 */
  int32_t max_len;
  int32_t window;           /* 0: none */
  float scale;
  int32_t flags;            /* TQ_OUT_FP16 or TQ_OUT_FP32 */
  const int32_t* seqs;
  const int32_t* cu_q;
  tq_kv_rows q;
  void* o;
  float* lse;
  void* workspace;
  size_t workspace_bytes;
} tq_kv_attn;

size_t tq_kv_attention_workspace_bytes(const tq_kv_cache* cache, const tq_kv_attn* a);
tq_status tq_kv_attention(const tq_kv_cache* cache, int32_t layer, const tq_kv_attn* a, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* TQ_H */
