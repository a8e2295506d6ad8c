/*
 * dfa.h - C ABI of the MI355X (gfx950) Dilated Flash Attention forward library.
 *
 * The operation is the attention operator of SAM-Lightening, section 3.1:
 *   - Segmentation + sparsification (Eq. 1): the N tokens of one image are cut into N/w
 *     segments of length w; inside segment i the rows i*w + o + j*r (j = 0 .. w/r-1) of
 *     Q, K and V are kept.  The paper writes o = 0; here o depends on the head
 *     (o = h mod r by default, or an explicit per-head table).
 *   - Per-segment attention (Eq. 2): softmax(scale * Q~_i K~_i^T) V~_i over the kept rows.
 *     Eq. 2 prints no scale factor: pass scale = 1.0f for the literal equation,
 *     1/sqrt(D) for the usual flash-attention convention.
 *   - Recomposition (Eq. 3): results are placed at the token positions they were taken
 *     from in a zero matrix of the input's shape; rows that nothing keeps are 0.
 *   - The paper cuts the sequence into equal-length parts.  The attention entry points also
 *     take other shapes: token n lies in part floor(n / w) and is kept iff
 *     n - floor(n / w) * w - o is a non-negative multiple of r, so the last part is shorter
 *     when w does not divide N (the same as padding the sequence and giving padded keys no
 *     weight), w > N gives a single part, and r need not divide w.  The index map, gather and
 *     placement entry points keep the regular case (w <= N, N % w == 0, w % r == 0).
 *   - Several (w, r) branches are merged with their log-sum-exp weights:
 *     L = log sum_b exp(lse_b), out = sum_b exp(lse_b - L) * out_b over the branches that
 *     keep the row (the paper treats a single branch; nb = 1 reproduces it).
 *
 * Conventions shared by all entry points
 *   - Pointers marked "device" are device memory of the current HIP device, "host" are
 *     ordinary host memory read before the call returns.  The caller owns every buffer.
 *   - Work is enqueued on `stream` (a hipStream_t passed as void*; NULL = default stream)
 *     and the call returns without synchronising, unless stated otherwise.
 *   - Tensors q, k, v are addressed as base + b*stride.b + n*stride.n + h*stride.h + d
 *     (strides in elements, the D elements of one row contiguous).  Every row must start
 *     on a 16-byte boundary.  Outputs are contiguous: out [B, N, H, D], lse [B, H, N].
 *   - D must be 64, and attention is not causal, unless the entry point says otherwise.  No mask, no bias.
 *   - Return value: DFA_OK (0) or a negative dfa_status_t.  Argument errors are found on
 *     the host before anything is enqueued.  No C++ exception crosses this boundary.
 *   - The attention entry points keep a per-process cache of launch plans (tile lists in
 *     device memory, read-only once built, a few hundred KB each), keyed by device and
 *     problem shape.  The first call with a new shape allocates and uploads its plan
 *     (synchronously); later calls with that shape allocate nothing and only enqueue
 *     kernels, so they can be recorded into a HIP graph (call once before capturing).  The
 *     cache holds the 64 most recently used plans (at most 256 MiB); a plan that falls out is
 *     freed (which synchronises its device) once no call is using it.  dfa_release_plans()
 *     empties the cache.  Calls may come from several threads and on several streams at once:
 *     a plan is shared and never written after its upload.
 *   - Workspace.  A bf16 dfa_forward with fewer workgroups than the chip has room for (a single
 *     image, say) is faster when the long key walks are shared out over several workgroups
 *     whose partial results (out in fp16 with a scale per row, lse in fp32) are merged afterwards.
 *     Those partial results live in a workspace that the caller owns: dfa_workspace_bytes() says
 *     how much the shape needs (0 = none; the smallest launches cut the walk inside the workgroup
 *     instead), and each call that may overlap another one needs a workspace of its own.  With
 *     workspace == NULL the call runs unsplit: same results to within rounding, slower for such
 *     shapes.
 */
#ifndef DFA_H
#define DFA_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define DFA_MAX_BRANCHES 8
#define DFA_HEAD_DIM 64

typedef enum {
    DFA_OK = 0,
    DFA_ERR_NULL = -1,      /* a required pointer is NULL                                    */
    DFA_ERR_SHAPE = -2,     /* B, H, N <= 0; D != 64; w < 1; r < 1; head offset outside      */
                            /* [0, r); scale not finite or <= 0; for the index map, gather   */
                            /* and placement also w > N, N % w != 0, w % r != 0; for the     */
                            /* projections sizes that the tiles do not divide; for 8-bit     */
                            /* operands also pitches below the rows they hold, and blocks    */
                            /* and pages of other sizes than the entry point names; for      */
                            /* packed sequences D other than 64 and 128, H not a multiple of */
                            /* Hkv, a scale or an eps outside its range                      */
    DFA_ERR_BRANCHES = -3,  /* nb < 1 or nb > DFA_MAX_BRANCHES                               */
    DFA_ERR_DTYPE = -4,     /* unknown dfa_dtype_t                                           */
    DFA_ERR_ALIGN = -5,     /* a base pointer or stride breaks the 16-byte row alignment     */
    DFA_ERR_LAUNCH = -6,    /* the HIP runtime refused an allocation, copy or launch         */
    DFA_ERR_TOO_LARGE = -7, /* index arithmetic would overflow the kernel's 32-bit counters  */
    DFA_ERR_WORKSPACE = -8  /* a workspace was passed that is smaller than the entry point's ..._workspace_bytes() */
} dfa_status_t;

typedef enum { DFA_BF16 = 0, DFA_F32 = 1 } dfa_dtype_t;

/* One (segment length, sparsification interval) pair of section 3.1. */
typedef struct { int32_t w; int32_t r; } dfa_branch_t;

/* Element strides of a [B, N, H, D]-addressed tensor; D is contiguous. */
typedef struct { int64_t b; int64_t n; int64_t h; } dfa_strides_t;

int dfa_version(void);
const char *dfa_error_string(int code);

/*
 * Kept-row indexer, host (Eq. 1 with the per-head start).
 * out_idx (host, int32 [H][N/r]): out_idx[h][i*(w/r) + j] = i*w + o_h + j*r.
 * head_offsets (host, int32 [H]) or NULL for o_h = h mod r.  Uses no GPU.
 */
int dfa_index_map(int32_t N, int32_t H, dfa_branch_t br, const int32_t *head_offsets,
                  int32_t *out_idx);

/*
 * The same map computed by the device indexer (the routine the gather, scatter and
 * attention kernels address kept rows with), written to d_out_idx (device, int32
 * [H][N/r]).  head_offsets is host memory or NULL.  Asynchronous on `stream`.
 */
int dfa_index_map_device(int32_t N, int32_t H, dfa_branch_t br, const int32_t *head_offsets,
                         int32_t *d_out_idx, void *stream);

/*
 * Bytes of device workspace that dfa_forward / dfa_encoder_stack use for this shape on the current
 * device (section 3.1's operator has no such notion: this is the room for the partial results
 * of a launch whose tiles are each walked by several workgroups, see "Workspace" above).  0 when the
 * shape needs none, for dt = DFA_F32, and for arguments dfa_forward would reject.  Host only: builds
 * the launch plan on the host, allocates nothing on the device; asks the current device for its
 * compute-unit count (the MI355X's when there is no device).
 */
size_t dfa_workspace_bytes(int32_t B, int32_t H, int32_t N, int32_t D, dfa_dtype_t dt,
                           const dfa_branch_t *branches, int32_t nb, const int32_t *head_offsets);

/*
 * Main entry: gather (Eq. 1) + per-segment attention (Eq. 2) + placement (Eq. 3) +
 * log-sum-exp merge of the nb branches, in one fused kernel.
 *   q, k, v       device, dtype dt, strided as described above
 *   branches      host, nb entries; head_offsets host int32 [nb][H] or NULL (o = h mod r)
 *   out           device, dtype dt, contiguous [B, N, H, D]; rows kept by no branch get 0
 *   lse           device, fp32 contiguous [B, H, N], natural log of the sum of
 *                 exp(scale * q.k) over the row's keys (each key counted once per branch
 *                 that pairs it with the row); -inf for rows kept by no branch.  May be NULL.
 *   workspace     device, 16-byte aligned, at least dfa_workspace_bytes() of this shape, written and
 *                 read by this call only (contents need not be kept between calls); or NULL.  Too
 *                 small a non-NULL workspace is DFA_ERR_WORKSPACE.
 * dt = DFA_BF16: bf16 operands on the matrix cores, fp32 accumulation and softmax
 * statistics, probabilities rounded to bf16 before the product with V, result rounded to
 * bf16.  The softmax denominator is the fp32 sum of those rounded probabilities, so out is
 * their exact weighted mean of V rows, and lse is within 2^-8 (3.9e-3) of the exact value
 * in the worst case (one key carrying the row), a few 1e-4 when many keys share the
 * weight.  dt = DFA_F32: fp32 throughout (products of exact three-part splits of the operands, within 2^-23 of each
 * product, 2^-26.7 on average, accumulated in fp32; operands that the parts do not hold exactly, those with bits below 2^-133 and those
 * that are not finite or round up to 2^128, take plain fp32 products, for which a launch takes up to 2.3 times as long; weights below
 * 2^-109 of the row's largest are kept to 2^-133).
 * Keys and values that are not finite make infinities or NaN of the rows that attend to them.  For dt = DFA_F32, for DFA_BF16 launches
 * in 64-row tiles (dfa_launch_describe in dfa_bench.h tells) and for 256-row tiles of one row group each, of no other rows.  256-row
 * tiles that hold several groups of rows (small images in batches) walk the union of their groups' keys: there a key or value that
 * is not finite also makes NaN of the other groups' rows in the tile.
 */
int dfa_forward(const void *q, const void *k, const void *v,
                dfa_strides_t sq, dfa_strides_t sk, dfa_strides_t sv,
                int32_t B, int32_t H, int32_t N, int32_t D, dfa_dtype_t dt, float scale,
                const dfa_branch_t *branches, int32_t nb, const int32_t *head_offsets,
                void *out, float *lse, void *workspace, size_t workspace_bytes, void *stream);

/*
 * dfa_forward with a workspace that is asked for only when the call turns out to need one: alloc(context, bytes) is called at
 * most once, on the calling thread, before anything is enqueued, and returns 16-byte aligned device memory that stays valid for
 * this call's launches, or NULL (the call then runs unsplit).  alloc == NULL: no workspace.  alloc must not throw.
 */
typedef void *(*dfa_alloc_t)(void *context, size_t bytes);
int dfa_forward_alloc(const void *q, const void *k, const void *v,
                      dfa_strides_t sq, dfa_strides_t sk, dfa_strides_t sv,
                      int32_t B, int32_t H, int32_t N, int32_t D, dfa_dtype_t dt, float scale,
                      const dfa_branch_t *branches, int32_t nb, const int32_t *head_offsets,
                      void *out, float *lse, dfa_alloc_t alloc, void *context, void *stream);

/*
 * dfa_forward for callers that cannot allocate device memory (code under HIP graph capture set-up rules,
 * tight serving loops, harnesses that forbid hipMalloc): same arguments without the workspace, same kernels
 * and same results as dfa_forward with a workspace, but it never calls hipMalloc / hipFree or anything else
 * that allocates device memory.  The launch plan and the partial results of a split launch live in a static
 * device array of DFA_STATIC_SCRATCH_BYTES (40 MiB) that each GPU the entry point runs on holds until the
 * process ends; a shape whose plan and partial results do not fit returns DFA_ERR_WORKSPACE before anything
 * is enqueued (every shape that is split fits; the limit is met by plans of some 700 000 workgroups).
 * The first call with a shape other than the previous call's on that GPU synchronises the device and copies
 * the new plan in (not capturable; call once before capturing); calls that repeat the shape only enqueue.
 * All calls on one GPU share the array: calls that overlap on one GPU (two streams, two threads) race on it
 * and must be serialised by the caller.
 */
#define DFA_STATIC_SCRATCH_BYTES ((size_t)40 << 20)
int dfa_forward_static(const void *q, const void *k, const void *v,
                       dfa_strides_t sq, dfa_strides_t sk, dfa_strides_t sv,
                       int32_t B, int32_t H, int32_t N, int32_t D, dfa_dtype_t dt, float scale,
                       const dfa_branch_t *branches, int32_t nb, const int32_t *head_offsets,
                       void *out, float *lse, void *stream);

/*
 * Backward of dfa_forward: gradients with respect to q, k, v for a gradient dout of the merged
 * output (lse takes no gradient).  The paper gives no backward pass; this is the chain rule on
 * Eq. 2 and the branch merge: with P = exp(scale q_n.k_j - lse_n) per (branch, n, j) pair of
 * the definition and delta_n = dout_n . out_n,  dv_j += P dout_n,  ds = P (dout_n . v_j - delta_n),
 * dq_n += scale ds k_j,  dk_j += scale ds q_n.
 *   q, k, v, strides, shapes, dt, scale, branches, head_offsets   exactly as passed to dfa_forward
 *   out, lse       device, what dfa_forward returned (out dtype dt [B, N, H, D], lse fp32 [B, H, N])
 *   dout           device, dtype dt, contiguous [B, N, H, D]
 *   delta_ws       device, fp32 [2][B, H, N] workspace (receives -(dout . out) and lse * log2(e) per row)
 *   dq, dk, dv     device, dtype dt, contiguous [B, N, H, D]; rows kept by no branch get 0
 * dt = DFA_BF16: bf16 operands on the matrix cores, fp32 accumulation, P and dS rounded to bf16
 * before their second products, gradients rounded to bf16.  dt = DFA_F32: fp32 products and sums on
 * the fp32 matrix cores.  Two launches on `stream`; uses the plan cache of dfa_forward.
 */
int dfa_backward(const void *q, const void *k, const void *v, const void *out, const float *lse,
                 const void *dout, dfa_strides_t sq, dfa_strides_t sk, dfa_strides_t sv,
                 int32_t B, int32_t H, int32_t N, int32_t D, dfa_dtype_t dt, float scale,
                 const dfa_branch_t *branches, int32_t nb, const int32_t *head_offsets,
                 float *delta_ws, void *dq, void *dk, void *dv, void *stream);

/*
 * One branch, unmerged (Eq. 1-3 for a single (w, r)): out_b device fp32 [B, N, H, D]
 * (0 on rows the branch does not keep), lse_b device fp32 [B, H, N] (-inf there).
 * head_offsets host int32 [H] or NULL.  Inputs of dtype dt as in dfa_forward.
 */
int dfa_forward_branch(const void *q, const void *k, const void *v,
                       dfa_strides_t sq, dfa_strides_t sk, dfa_strides_t sv,
                       int32_t B, int32_t H, int32_t N, int32_t D, dfa_dtype_t dt, float scale,
                       dfa_branch_t br, const int32_t *head_offsets,
                       float *out_b, float *lse_b, void *stream);

/*
 * Stand-alone log-sum-exp merge of nb unmerged branch results.
 *   out_b device fp32 [nb][B, N, H, D], lse_b device fp32 [nb][B, H, N]
 *   out   device dtype dt [B, N, H, D], lse device fp32 [B, H, N] (may be NULL)
 */
int dfa_merge(const float *out_b, const float *lse_b, int32_t nb,
              int32_t B, int32_t H, int32_t N, int32_t D, dfa_dtype_t dt,
              void *out, float *lse, void *stream);

/*
 * Stand-alone gather (Eq. 1): kept rows of one strided tensor x into a dense
 * xg (device, dtype dt, contiguous [B, H, N/r, D]), rows in index-map order.
 */
int dfa_gather(const void *x, dfa_strides_t sx, int32_t B, int32_t H, int32_t N, int32_t D,
               dfa_dtype_t dt, dfa_branch_t br, const int32_t *head_offsets,
               void *xg, void *stream);

/*
 * Stand-alone placement (the MAP of Eq. 3): dense og (device, dtype dt, [B, H, N/r, D])
 * back to token positions in out (device, dtype dt, contiguous [B, N, H, D]); rows the
 * branch does not keep are written as 0, so out needs no initialisation.
 */
int dfa_scatter(const void *og, int32_t B, int32_t H, int32_t N, int32_t D, dfa_dtype_t dt,
                dfa_branch_t br, const int32_t *head_offsets, void *out, void *stream);

/*
 * Host-side view of the launch plan of plain 256-row tiles (no GPU needed).  Large launches of the bf16 dfa_backward run
 * it as it stands.  The others refine it: the fp32 kernels walk its lists cut into blocks, small launches of either take
 * smaller tiles (dfa_launch_describe in dfa_bench.h gives the plan of a call), the bf16 dfa_forward packs tiles
 * (dfa_plan_describe_forward).  The query rows of each head are grouped by the set of (branch, segment) pairs that keep them and
 * cut into tiles; every tile carries its keys as arithmetic progressions: one per member
 * branch, or, where the member branches keep some keys more than once, the multiset union of
 * those cut into progressions of one multiplicity each (a key kept by m branches is visited
 * once and its softmax weight multiplied by m: the same sum as m visits, section 3.1's merge
 * being a softmax over the multiset union of the branches' keys).
 * Pass NULL arrays to query the sizes only.
 *   n_tiles, n_rows, n_segs, n_items   out, host: entry counts
 *   tiles  host int32 [n_tiles][6] = (h, row_begin, nrows, seg_begin, nseg, 64-key steps of the list)
 *   rows   host int32 [n_rows]     token positions, tile after tile
 *   segs   host int32 [n_segs][4]  = (first key, key stride, key count, multiplicity)
 *   items  host int32 [n_items][2] = (tile or -1 for padding, b) in launch order
 */
int dfa_plan_describe(int32_t B, int32_t H, int32_t N, const dfa_branch_t *branches, int32_t nb,
                      const int32_t *head_offsets, int32_t *n_tiles, int32_t *n_rows,
                      int32_t *n_segs, int32_t *n_items, int32_t *tiles, int32_t *rows,
                      int32_t *segs, int32_t *items);

/*
 * The same view of the plan of 256-row tiles of the bf16 dfa_forward (launches that do not fill the chip may run 64-row
 * tiles instead, see dfa_launch_describe in dfa_bench.h).  It differs from the plain one where row groups fill only part of a
 * 256-row tile (small images: the rows of one window of the narrowest branch fall into several groups by which
 * dilated branches also keep them): groups that share most of their keys are packed into one tile, each group
 * on 32-row blocks of its own (half a wave: the unit with its own softmax state), and the tile walks the union of
 * their key lists once.  A progression then has a multiplicity per block, 0 where that block's rows do not attend
 * to its keys (their scores are masked).
 * Arguments as dfa_plan_describe, with
 *   rows       an entry < 0 is a filler slot between two groups of a packed tile (it holds ~n of a row n of the
 *              group before it; nothing is stored for it)
 *   segs       [n_segs][4] = (first key, key stride, key count, largest multiplicity over the blocks)
 *   block_mult host int32 [n_segs][8]: multiplicity of the progression's keys for the rows of block 0..7
 *              (slots 32k .. 32k+31 of the tile); NULL to skip
 */
int dfa_plan_describe_forward(int32_t B, int32_t H, int32_t N, const dfa_branch_t *branches, int32_t nb,
                              const int32_t *head_offsets, int32_t *n_tiles, int32_t *n_rows,
                              int32_t *n_segs, int32_t *n_items, int32_t *tiles, int32_t *rows,
                              int32_t *segs, int32_t *block_mult, int32_t *items);

/*
 * Projection either side of the operator inside an encoder layer (the ViT self-attention
 * block the paper's encoder is built from, section 3.1): y = x . w^T, one weight ROW per
 * output feature, no bias.  bf16 operands on the matrix cores, fp32 accumulation, y rounded
 * to bf16.
 *   x device bf16 [M][K] with row pitch ldx, w device bf16 [N][K] with row pitch ldw,
 *   y device bf16 [M][N] with row pitch ldy (pitches in elements, each a multiple of 8;
 *   base pointers 16-byte aligned).  M % 256 == 0, N % 128 == 0, K % 64 == 0, else
 *   DFA_ERR_SHAPE.  y must not overlap x or w.  Asynchronous on `stream`.
 */
int dfa_linear(const void *x, const void *w, void *y, int64_t M, int32_t N, int32_t K,
               int64_t ldx, int64_t ldw, int64_t ldy, void *stream);

/*
 * `layers` encoder attention layers back to back (the "encoder attention stack" workload):
 * per layer  qkv = x_l . w_qkv[l]^T  (features ordered [3][H][D]: q heads, k heads, v heads),
 * attn = dfa_forward(q, k, v read in place from qkv through strides),  x_{l+1} = attn . w_o[l]^T.
 * No bias, residual or normalisation.  E = H * D.
 *   x        device bf16 [B][N][E], read only
 *   w_qkv    device bf16 [layers][3E][E];  w_o  device bf16 [layers][E][E]
 *   qkv_ws   device bf16 [B][N][3][H][D]   workspace, holds the last layer's qkv on return
 *   attn_ws  device bf16 [B][N][H][D]      workspace, holds the last layer's attention output
 *   y        device bf16 [B][N][E]         x_layers; also used for every intermediate x_l
 *                                          (y may be the same buffer as x: x is then overwritten)
 *   branches, head_offsets, scale, workspace, workspace_bytes    as in dfa_forward (one workspace
 *                                          serves every layer)
 * (B * N) % 256 == 0 and E % 128 == 0 are required (DFA_ERR_SHAPE otherwise); D must be 64.
 * Every argument is checked before the first launch.  Three launches per layer on `stream` (four
 * where the attention launch is split); allocates only what the plan cache allocates on first use.
 */
int dfa_encoder_stack(const void *x, const void *w_qkv, const void *w_o, int32_t layers,
                      int32_t B, int32_t H, int32_t N, int32_t D, float scale,
                      const dfa_branch_t *branches, int32_t nb, const int32_t *head_offsets,
                      void *qkv_ws, void *attn_ws, void *y, void *workspace, size_t workspace_bytes,
                      void *stream);

/*
 * ---- Products of 8-bit operands --------------------------------------------------------------------------------------------
 * A quantised matrix of `rows` rows of `cols` elements: OCP e4m3 values in blocks that share a power of two, 2^e with the smallest
 * e >= -126 for which the block's largest finite |x| is at most 448 * 2^e.  A value is the e4m3 number nearest to x / 2^e (ties to even); x that is
 * not finite is NaN.  (x of 1.9375 * 2^127 or more is held as 2^128, which fp32 takes as infinite.)  A block is 128 elements of a row
 * (block_rows = 1), or 128 rows by 128 columns (block_rows = 128: the same values for the matrix and its transpose, the form for weights that a
 * backward pass reads too).
 *   values  device, bytes [rows][ld], ld (a multiple of 128) at least cols; columns from cols to the next multiple of 128 hold 0
 *   scales  device, bytes [ld / 128][ld_scales], e + 127 of the block that holds row r and columns 128 c .. 128 c + 127 at
 *           [c][r] (128 equal ones for a 128 x 128 block); ld_scales (a multiple of 16) at least rows
 * Both 16-byte aligned; ld < 2^23.
 */
typedef struct { void *values; void *scales; int64_t ld; int64_t ld_scales; } dfa_quantized_t;

/*
 * Quantises x (device, dtype dt, [rows][cols] with row pitch ldx; rows may start at any element).
 *   q    (host struct or NULL)  receives x: blocks along its columns
 *   q_t  (host struct or NULL)  receives x transposed, [cols][rows]: blocks along x's rows (what a product that contracts over
 *        x's rows reads)
 * Writes values up to the next multiple of 128 columns and scales up to the next multiple of 16 rows.  Asynchronous on `stream`.
 */
int dfa_quantize(const void *x, dfa_dtype_t dt, int64_t rows, int64_t cols, int64_t ldx, int32_t block_rows,
                 const dfa_quantized_t *q, const dfa_quantized_t *q_t, void *stream);

/*
 * y[m][n] = sum_k a[m][k] * b[n][k] of the values that a [M][K] and b [N][K] hold.
 *   dt = DFA_F32   exact products, fp32 sums.  Values below 2^-126, scale included, may count as 0, and one of 2^128 as infinite
 *   dt = DFA_BF16  the matrix instruction adds up the products of 16 neighbouring k (16 j to 16 j + 15) at a time and cuts each of them off at 2^-13 of the
 *                  power of two of the largest: up to 16 * 2^-13 of that product's magnitude for each 16 k (2.3e-5 of the sum of magnitudes, rms, on random
 *                  values; where large terms cancel, what is smaller than that may be lost altogether).  These sums are added up in fp32 and rounded
 *                  once to bf16.  Where that does not do: DFA_F32.
 * This holds for the projection and its gradients below too (dw is always fp32).
 *   y          device, dtype dt, [M][N] with row pitch ldy (elements); must not overlap a or b
 *   workspace  device, 16-byte aligned, dfa_quantized_product_workspace_bytes(dt, M, N, K) (0 = none, NULL allowed): partial sums of
 *              products whose k-steps are shared out over workgroups.  Written and read by this call only: calls that may
 *              overlap need one each.
 * The sums are in a fixed order: equal calls give equal results.  Asynchronous on `stream`; allocates nothing.
 */
size_t dfa_quantized_product_workspace_bytes(dfa_dtype_t dt, int64_t M, int64_t N, int64_t K);
int dfa_quantized_product(dfa_quantized_t a, dfa_quantized_t b, void *y, dfa_dtype_t dt, int64_t M, int64_t N, int64_t K, int64_t ldy,
                          void *workspace, size_t workspace_bytes, void *stream);

/*
 * The projection dfa_linear with a quantised weight: x (device, dtype dt, [M][K] with row pitch ldx) is quantised by the call in blocks
 * of 1 x 128, y[m][n] = sum_k x[m][k] * w[n][k] as above, y of x's dtype and apart from x and w.  Any M, N, K >= 1.  Few rows (64 at
 * most, fewer of long ones) take one launch and no workspace; others quantise into the workspace first.
 */
size_t dfa_quantized_linear_workspace_bytes(dfa_dtype_t dt, int64_t M, int64_t N, int64_t K);
int dfa_quantized_linear(const void *x, dfa_dtype_t dt, int64_t ldx, dfa_quantized_t w, void *y, int64_t M, int64_t N, int64_t K, int64_t ldy,
                         void *workspace, size_t workspace_bytes, void *stream);

/*
 * Gradients of y = x . w^T for a gradient dy [M][N] of y (the quantisation of x and w is passed through as the identity):
 *   dx [M][K] = dy . w    dy in 1 x 128 blocks along N; w_t: w transposed, [K][N] (quantised with block_rows = 128 it holds the forward's
 *                         values)
 *   dw [N][K] = dy^T . x  dy and x in blocks of 128 along M, each column on its own; fp32
 * dy, x and dx have dtype dt; dx and dw overlap none of the operands.  dx or dw may be NULL (not wanted): x is read for dw only, w_t for dx only.
 */
size_t dfa_quantized_linear_backward_workspace_bytes(dfa_dtype_t dt, int64_t M, int64_t N, int64_t K);
int dfa_quantized_linear_backward(const void *dy, int64_t lddy, const void *x, int64_t ldx, dfa_dtype_t dt, dfa_quantized_t w_t, void *dx,
                                  int64_t lddx, float *dw, int64_t lddw, int64_t M, int64_t N, int64_t K, void *workspace, size_t workspace_bytes,
                                  void *stream);

/*
 * ---- Attention over keys and values held in 8 bits -------------------------------------------------------------------------
 * A cache of `pages` pages of `page` tokens (16, 32, 64 or 128) of `heads` heads of D (64 or 128) channels, in e4m3 with one
 * power of two per page and head for the keys and one for the values (format as above: the block is the tokens that the page holds):
 *   k       device, [pages][heads][page][D]       16-byte aligned
 *   v       device, [pages][heads][D][page]       16-byte aligned; a channel's tokens lie side by side
 *   scales  device, bytes [pages][heads][2]       exponent + 127 of the keys and of the values
 * It needs no initialisation.  Sequence b of a call has token n in slot n % page of page table[b * ld_table + n / page]:
 *   table   device, int32 [B][width], width * page tokens at most; entries behind the last token are not used.  A page outside
 *           0 .. pages - 1 is skipped: nothing is written to it, its tokens are attended to by no row.
 *   lengths device, int32 [B]: tokens that sequence b holds, those of this step included
 *   counts  device, int32 [B], or NULL for all: how many of the call's T (or M) rows of sequence b there are, the first ones; the last of
 *           them is token lengths[b] - 1
 */
typedef struct { void *k; void *v; void *scales; int32_t pages; int32_t heads; int32_t page; int32_t D; } dfa_cache_t;

/*
 * Writes rows 0 .. n - 1 (n = counts[b], T without counts) of k and v as tokens lengths[b] - n .. lengths[b] - 1 of every sequence.
 *   k, v   device, dtype dt, [B, T, heads, D] through strides (every row 16-byte aligned)
 * A page's scale holds its new tokens and is not below what its earlier tokens (of this sequence, slots before the first new one) have;
 * where it grows, those move to it: values are rounded to the new scale, a change only below e4m3's normal range.  Slots behind the last new token
 * and pages without new tokens are left as they were.  Tokens before 0 or behind the table's last page are dropped.  No page may
 * take new tokens at two places of the table.  Asynchronous on `stream`; allocates nothing.
 */
int dfa_cache_append(const void *k, const void *v, dfa_strides_t sk, dfa_strides_t sv, dfa_dtype_t dt, int32_t B, int32_t T, dfa_cache_t cache,
                     const int32_t *table, int32_t width, int64_t ld_table, const int32_t *lengths, const int32_t *counts, void *stream);

/*
 * out[b, i, h] = softmax(scale * q[b, i, h] . k) v over tokens of head h / (H / heads) of sequence b, and its lse.
 *   q       device, dtype dt, [B, M, H, D] through strides (every row 16-byte aligned); H a multiple of cache.heads
 *   causal  0: a row attends to all lengths[b] tokens; otherwise row i of the n = counts[b] (M) attends to the first
 *           lengths[b] - (n - 1 - i): the rows are the sequence's last tokens.
 *   out     device, dtype dt, contiguous [B, M, H, D], apart from q;  lse device, fp32 [B, H, M], or NULL
 *           rows that attend to nothing (no tokens, i >= counts[b]) are 0 and -inf; lengths outside 0 .. width * page count as the
 *           nearest of them
 *   max_length  host: no sequence is expected to be longer (longer ones are right, but slower).  It decides how the walk is shared out.
 *   workspace   device, 16-byte aligned, dfa_cache_attention_workspace_bytes() of the same arguments (0 = none, NULL allowed); written and
 *           read by this call only: calls that may overlap, captured ones among them, need one each.
 * dt = DFA_BF16: bf16 operands, probabilities rounded to bf16 before the second product, fp32 sums and statistics; dt = DFA_F32: 24-bit
 * operands throughout (of elements of q below 2^-110 in a row whose largest is 2^-64 or more, bits below 2^-133 count as 0).  Cached values below 2^-126,
 * scale included, may count as 0.  Scores are right at any size as long as q . k, before the scale, and the sums of weighted values are fp32 numbers; what passes
 * fp32's range there counts as infinite, a cached value of 2^128 too.  Keys, values and rows that are not finite reach only the
 * rows that attend to them.  One launch, two where the walk is shared out over workgroups; equal calls give equal results.
 * Asynchronous on `stream`; allocates nothing.
 */
size_t dfa_cache_attention_workspace_bytes(int32_t B, int32_t M, int32_t H, int32_t heads, int32_t D, dfa_dtype_t dt, int64_t max_length);
int dfa_cache_attention(const void *q, dfa_strides_t sq, dfa_dtype_t dt, int32_t B, int32_t M, int32_t H, dfa_cache_t cache, const int32_t *table,
                        int32_t width, int64_t ld_table, const int32_t *lengths, const int32_t *counts, int32_t causal, float scale, int64_t max_length,
                        void *out, float *lse, void *workspace, size_t workspace_bytes, void *stream);

/* Empties the plan cache of every device; a plan is freed (its device synchronised) as soon as no
 * call is using it any more. */
int dfa_release_plans(void);

/*
 * ---- Packed prompts ----------------------------------------------------------------------------------------------------------
 * Sequences that lie one behind the other: rows starts[b] .. starts[b + 1] - 1 of the T rows of a packed tensor are sequence b's, in order.
 *   starts  device, int32 [B + 1], ascending from 0; starts[B] <= T.  Equal neighbours: an empty sequence.  (Other values are read as the nearest that
 *           lie within 0 .. T; starts that do not ascend leave results undefined, but no access leaves the tensors.)
 * Nothing about the lengths is needed on the host: a captured launch serves whatever `starts` holds when it is replayed.
 */

/*
 * out[i, h] = softmax(scale * q[i, h] . k) v over the keys of head h / (H / Hkv) in row i's sequence, and its lse.
 *   q       device, dtype dt, [T, H, D] through strides (b is not used; every row 16-byte aligned; rows less than 2^25 bytes apart); k, v: [T, Hkv, D];
 *           H a multiple of Hkv, D 64 or 128
 *   causal  0: a row attends to its whole sequence; otherwise to the rows before it and itself
 *   out     device, dtype dt, contiguous [T, H, D], apart from q, k and v;  lse device, fp32 [H, T], or NULL
 *           rows of no sequence (from starts[B] on) are 0 and -inf
 * bf16: probabilities are rounded to bf16 before they meet v; sums are fp32.  fp32: products of three bf16 parts a number (24 bits; bits
 * below 2^-133 are lost, and what rounds to 2^128 in bf16 counts as infinite).  scale lies within 2^-100 .. 2^100, and every scale * q . k
 * within 2^127 ln 2 either way.  Keys and values that are not finite reach only the rows that attend to them (an infinite fp32 value may come out as NaN there).
 * (T / 32 + B + 1) H lies below 2^24: a grid holds fewer than 2^32 threads.
 * Sums are in a fixed order: equal calls give equal results.  Asynchronous on `stream`; allocates nothing.
 */
int dfa_prompt_attention(const void *q, const void *k, const void *v, dfa_strides_t sq, dfa_strides_t sk, dfa_strides_t sv, dfa_dtype_t dt, int32_t T,
                         int32_t H, int32_t Hkv, int32_t D, const int32_t *starts, int32_t B, int32_t causal, float scale, void *out, float *lse,
                         void *stream);

/*
 * Gradients of the above for a gradient dout [T, H, D] of out:
 *   dv_j = sum_i P_ij dout_i,  dq_i = scale sum_j dS_ij k_j,  dk_j = scale sum_i dS_ij q_i,  P_ij = exp(scale q_i . k_j - lse_i),
 *   dS_ij = P_ij (dout_i . v_j - dout_i . out_i), the sums of dk and dv over the query heads of a key head too.
 *   out, lse    device, what the forward call returned;  out, dout, dq contiguous [T, H, D], dk and dv contiguous [T, Hkv, D], dtype dt, 16-byte aligned;
 *               H * D elements take less than 2^25 bytes.  dq, dk, dv overlap nothing else.  Rows of no sequence are 0.
 *   workspace   device, 16-byte aligned, ..._workspace_bytes() of the same sizes; written and read by this call only: calls that may overlap, captured
 *               ones among them, need one each.
 * bf16: P and dS are rounded to bf16 before they meet q, k and dout.  A value that is not finite in q, k, v or dout makes all gradients of its
 * sequence and heads undefined, those of others not.  Sums are in a fixed order.  Asynchronous on `stream`; allocates nothing.
 */
size_t dfa_prompt_attention_backward_workspace_bytes(int32_t T, int32_t H, int32_t Hkv, int32_t D, int32_t B);
int dfa_prompt_attention_backward(const void *q, const void *k, const void *v, dfa_strides_t sq, dfa_strides_t sk, dfa_strides_t sv, const void *out,
                                  const float *lse, const void *dout, dfa_dtype_t dt, int32_t T, int32_t H, int32_t Hkv, int32_t D, const int32_t *starts,
                                  int32_t B, int32_t causal, float scale, void *dq, void *dk, void *dv, void *workspace, size_t workspace_bytes,
                                  void *stream);

/*
 * Root-mean-square norm of the rows of x, a residual added first:
 *   h = x + residual (x without one),  r = (mean of h^2 over the row + eps)^(-1/2),  y = h r weight
 * in fp32 from the operands to the one rounding of h and of y (y comes of the unrounded h).
 *   x, residual  device, dtype dt, [M][C] with row pitches (elements; rows may start at any element); residual may be NULL
 *   weight       device, [C], of weight_dt (fp32 rows take fp32 weights, bf16 rows either), or NULL for ones;  eps >= 0
 *   h            device, dtype dt, [M][C] with row pitch ldh, or NULL; may be x or residual itself (same pointer and pitch)
 *   y            device, dtype dt, [M][C] with row pitch ldy, or NULL
 *   q            host struct or NULL: receives y in e4m3, blocks of 128 along the rows, as dfa_quantize does (from the fp32 values, not from
 *                y's rounded ones); one of y and q at least.  Values up to the next multiple of 128 columns (zeros) and scale bytes up to the next multiple of 16
 *                rows are written.
 * h, y and q apart from the operands and each other (but for h as said).  Rows are exact at any size that fp32 holds, subnormal numbers included: sums of squares that
 * overflow, or fall below 1e-30 beside an eps that does, are taken again, scaled, and r, which may then be no fp32 number, is held in two factors.  C is 32768 at most,
 * and M (a grid holds fewer than 2^32 threads) 2^26 - 4 up to 1024 columns, 2^24 - 1 up to 4096, 2^23 - 1 up to 16384 and 2^22 - 1 beyond.
 * Asynchronous on `stream`; allocates nothing.
 */
int dfa_rms_norm(const void *x, int64_t ldx, const void *residual, int64_t ldr, const void *weight, dfa_dtype_t weight_dt, dfa_dtype_t dt, float eps,
                 void *h, int64_t ldh, void *y, int64_t ldy, const dfa_quantized_t *q, int64_t M, int64_t C, void *stream);

/*
 * Gradients of the above for gradients dy of y and dh of h (NULL: none), with g = dy weight and u = h r:
 *   dx = r (g - u mean(g u)) + dh   of x and of the residual alike;  dw = sum over the rows of dy u, fp32 [C], or NULL (not wanted)
 *   h           device, dtype dt, what the forward call stored (x where there was no residual); dy, dh, dx likewise [M][C] with row pitches;
 *               dx may be dy or dh itself (same pointer and pitch), else apart from the operands
 *   workspace   device, 16-byte aligned, ..._workspace_bytes(M, C) (0 = none, NULL allowed; not used without dw): partial sums of dw.  Written and read by this
 *               call only: calls that may overlap, captured ones among them, need one each.
 * Rows of h of any size, as above, and any number of them; g h may overflow (where it falls below 2^-126 it loses bits); a dx that fp32 does not hold is
 * infinite or NaN, and may leave dw so.  Sums are in a fixed order: equal calls give equal results.  Asynchronous on `stream`; allocates nothing.
 */
size_t dfa_rms_norm_backward_workspace_bytes(int64_t M, int64_t C);
int dfa_rms_norm_backward(const void *dy, int64_t lddy, const void *h, int64_t ldh, const void *weight, dfa_dtype_t weight_dt, dfa_dtype_t dt, float eps,
                          const void *dh, int64_t lddh, void *dx, int64_t lddx, float *dw, int64_t M, int64_t C, void *workspace, size_t workspace_bytes,
                          void *stream);

/*
 * Pages for a step's new tokens.  `free_pages` (device, int32 [capacity]) is a stack: its first n_free[0] entries are pages that no sequence
 * holds.  Sequence b holds lengths[b] tokens and gets counts[b] more (0 allowed): it takes ceil(new length / page) - ceil(length / page) pages from the top
 * of the stack, sequence after sequence, page after page, which go into its row of the table behind those it has.
 *   table        device, int32 [B][width] with pitch ld_table; other entries are left as they were
 *   new_lengths  device, int32 [B], lengths + counts; new_n_free device, int32 [1]; may be lengths and n_free themselves (else apart from everything)
 *   starts       device, int32 [B + 1]: where each sequence's new tokens start among the step's packed rows
 *   slots        device, int64 [rows], positions device, int32 [rows]: of every packed row its place in the cache, page number * page + place in the
 *                page, and its place in the sequence; -1 behind the last
 *   refused      device, int32 [1]: 0, or why the step does not fit: 1 too few free pages, 2 a sequence longer than width * page tokens, 4 more than `rows` new
 *                tokens (added up where several hold); 8 a count or length below 0.  A step that does not fit changes nothing: lengths, n_free and
 *                table stay, starts are 0, slots and positions -1.
 * page: 16, 32, 64 or 128.  n_free outside 0 .. capacity counts as the nearest.  One launch for up to 4096 rows, two for more.  Asynchronous on `stream`; allocates
 * nothing.
 */
int dfa_cache_reserve(const int32_t *counts, const int32_t *lengths, int32_t B, int32_t page, int32_t *table, int32_t width, int64_t ld_table,
                      const int32_t *free_pages, int32_t capacity, const int32_t *n_free, int32_t *new_lengths, int32_t *new_n_free, int32_t *starts,
                      int64_t *slots, int32_t *positions, int32_t rows, int32_t *refused, void *stream);

/*
 * Gives the pages of every sequence with done[b] != 0 (device, int32 [B]) back: the first ceil(lengths[b] / page) entries of its row of the table go
 * onto the stack, sequence after sequence, and lengths[b] becomes 0.  refused: 0, or 1 if the stack has no room for them: nothing is changed then.
 */
int dfa_cache_release(const int32_t *done, int32_t *lengths, int32_t B, int32_t page, const int32_t *table, int32_t width, int64_t ld_table,
                      int32_t *free_pages, int32_t capacity, int32_t *n_free, int32_t *refused, void *stream);

/*
 * dfa_cache_append of packed rows: rows starts[b] .. starts[b + 1] - 1 of k and v (device, dtype dt, [T, heads, D] through strides, b not used) are
 * the last tokens of sequence b.  Rows of no sequence are not read.
 */
int dfa_cache_append_packed(const void *k, const void *v, dfa_strides_t sk, dfa_strides_t sv, dfa_dtype_t dt, int32_t T, const int32_t *starts, int32_t B,
                            dfa_cache_t cache, const int32_t *table, int32_t width, int64_t ld_table, const int32_t *lengths, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* DFA_H */
