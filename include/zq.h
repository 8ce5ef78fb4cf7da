/*
 * zq.h -- C ABI of the qwZ / qgZ compression data path for one MI355X (gfx950).
 *
 * Method: arXiv 2501.04266 ("Scaling Large Language Model Training on
 * Frontier with Low-Bandwidth Partitioning").  Its hierarchical ZeRO++
 * partitioning compresses every collective with ZeRO++'s block-based
 * quantisation (Background, ZeRO++ subsection): weights are quantised to
 * INT8 blocks before the weight Allgather and dequantised after it (qwZ;
 * Design, Weight Partitioning: quantiser / dequantiser operators, secondary
 * partition stored quantised), and gradients travel as INT4 blocks through an
 * all-to-all reduce-scatter whose receiver dequantises, sums and requantises
 * the P slices it gets (qgZ; Design, Gradient Partitioning and Communication
 * Volume Analysis).  Each block has its own scale (Evaluations, Model
 * Convergence).  This library is one rank's share of that path, with the P
 * slices of a level already resident in this GPU's memory.
 *
 * Definition implemented (symmetric absmax; the paper gives no formula, these
 * are the readings taken):
 *   block b = elements [b*B, min(n, (b+1)*B)); the last block may be short.
 *   a = max |x_i| over the block;   qmax = 127 (INT8) or 7 (INT4)
 *   a < 2^-119 (incl. all-zero):    scale = +0, every code 0
 *   otherwise: scale = fl(a / qmax), r = fl(qmax / a),
 *              code_i = round-half-even(fl(x_i * r))  (always within +-qmax)
 *   dequant:   y_i = cvt(fl(code_i * scale)), cvt = identity or RNE narrowing
 *   reduce:    acc_i = +0; for p = 0..P-1: acc_i = fl(acc_i + fl(q^p_i * s^p_b))
 *              then INT4-quantise acc (one rounded multiply, then one rounded
 *              add per slice; no fused multiply-add).
 * fl() is one IEEE binary32 operation rounded to nearest even; fp32
 * subnormals are kept.  Results are bit-identical to that definition.
 *
 * Formats:
 *   INT8 codes:  int8_t[n], two's complement.
 *   INT4 codes:  uint8_t[ceil(n/2)]; element 2j in the low nibble of byte j,
 *                element 2j+1 in the high nibble, two's complement; for odd n
 *                the last high nibble is 0.
 *   scales:      float[ceil(n/B)], one per block.
 *   elements:    ZQ_F32 (float), ZQ_F16 (IEEE binary16), ZQ_BF16 (bfloat16).
 *
 * Conventions for every call:
 *   - All array pointers are device pointers (hipMalloc'd or equivalent) in
 *     the caller's ownership; the library allocates nothing and keeps no
 *     state between calls, except the device address table of
 *     qgz_reduce_level_gather_noalloc (a static array per GPU).
 *   - Work is enqueued on `stream` (a hipStream_t; NULL = the default stream)
 *     and returns without synchronising; results are visible after the
 *     stream is synchronised.  Calls from several host threads are safe.
 *   - block must be a power of two in [32, 1024].
 *   - Element and code arrays must be 16-byte aligned, scale arrays 4-byte
 *     aligned.  Outputs must not overlap inputs.
 *   - n == 0 (or m == 0) is a successful no-op; n < 0 is ZQ_E_SIZE.
 *   - Inputs are expected to be finite; non-finite inputs give unspecified
 *     codes (no error is raised, to avoid an extra pass).
 *   - Every argument error is detected on the host before anything is
 *     enqueued, so no output byte is written.  ZQ_E_HIP means a HIP launch
 *     failed (outputs then undefined).
 */
#ifndef ZQ_H
#define ZQ_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef int zq_dtype;
enum { ZQ_F32 = 0, ZQ_F16 = 1, ZQ_BF16 = 2 };
enum { ZQ_I32 = 3, ZQ_I64 = 4 };  /* token ids (embedding calls) */
enum { ZQ_INT4 = 5 };             /* packed INT4 codes with block scales (gradient tables) */
enum { ZQ_INT8 = 6 };             /* INT8 codes with block scales (the weight an AdamW step writes) */
enum { ZQ_F8 = 7 };               /* 8-bit moments of an AdamW step with block scales */

enum {
  ZQ_OK = 0,
  ZQ_E_NULL = -1,   /* a required pointer is NULL (with n > 0) */
  ZQ_E_BLOCK = -2,  /* block not a power of two in [32, 1024] */
  ZQ_E_DTYPE = -3,  /* unknown element dtype */
  ZQ_E_ALIGN = -4,  /* misaligned pointer */
  ZQ_E_SIZE = -5,   /* negative element count, or a size the call does not take */
  ZQ_E_P = -6,      /* slice count outside [1, 1024] */
  ZQ_E_HIP = -7,    /* HIP kernel launch failed */
  ZQ_E_ALIAS = -8   /* an output overlaps an input or another output */
};

/* qwZ quantiser (Background, ZeRO++: quantise the weight shard to INT8 blocks
 * before the Allgather; Design, Weight Partitioning: also the quantised
 * secondary partition).
 *   x       [n] elements of dtype xt (read)
 *   codes   [n] int8 codes (written)
 *   scales  [ceil(n/block)] floats (written) */
int qwz_quantize(const void* x, zq_dtype xt, int64_t n, int32_t block,
                 int8_t* codes, float* scales, void* stream);

/* qwZ dequantiser (Design, Weight Partitioning: dequantise the gathered layer
 * for the forward pass, or the gathered secondary partition for backward).
 *   codes [n], scales [ceil(n/block)] (read) -> y [n] of dtype yt (written) */
int qwz_dequantize(const int8_t* codes, const float* scales, int64_t n, int32_t block,
                   void* y, zq_dtype yt, void* stream);

/* qgZ quantiser (Background, ZeRO++: gradients quantised to INT4 blocks for
 * the all-to-all reduce-scatter).
 *   g [n] of dtype gt (read) -> packed [ceil(n/2)] bytes, scales [ceil(n/block)] */
int qgz_quantize(const void* g, zq_dtype gt, int64_t n, int32_t block,
                 uint8_t* packed, float* scales, void* stream);

/* qgZ reduce level: the receiver side of the quantised all-to-all
 * reduce-scatter (Background, ZeRO++; Design, Communication Volume Analysis:
 * 1-hop all-to-all within the node).  P slices of m elements each, laid out
 * back to back: slice p's bytes at packed_in + p*ceil(m/2), its scales at
 * scales_in + p*ceil(m/block).  They are dequantised, summed in ascending
 * slice order and requantised to one INT4 slice of m elements:
 *   packed_out [ceil(m/2)], scales_out [ceil(m/block)] (written).
 * 1 <= P <= 1024.  The hierarchical scheme applies this once per partition
 * level (Design: GCD pair, node, all ranks). */
int qgz_reduce_level(const uint8_t* packed_in, const float* scales_in, int32_t P, int64_t m,
                     int32_t block, uint8_t* packed_out, float* scales_out, void* stream);

/* qgZ dequantiser: final gradient shard for the optimizer (Design, Gradient
 * Partitioning).  packed [ceil(n/2)], scales [ceil(n/block)] -> y [n] of yt. */
int qgz_dequantize(const uint8_t* packed, const float* scales, int64_t n, int32_t block,
                   void* y, zq_dtype yt, void* stream);

/* Fused last level: the receiver's final reduce level followed by the
 * dequantisation of the resulting gradient shard for the optimizer (Design,
 * Gradient Partitioning; Background, ZeRO++: quantised reduce-scatter).
 * Writes y [m] of dtype yt, bit-identical to qgz_dequantize applied to what
 * qgz_reduce_level would produce from the same slices, without storing and
 * re-reading the INT4 result.  packed_out / scales_out are optional: both NULL,
 * or both given to receive that INT4 result as well.  Slice layout, limits
 * and errors as qgz_reduce_level; y must be 16-byte aligned and overlap no
 * input or output. */
int qgz_reduce_dequantize(const uint8_t* packed_in, const float* scales_in, int32_t P, int64_t m, int32_t block,
                          void* y, zq_dtype yt, uint8_t* packed_out, float* scales_out, void* stream);

/* Reduce level over slices that are not back to back: the receiver reading
 * each peer's INT4 chunk where it lies, without first copying the chunks into
 * one receive buffer (the peer-direct form of the quantised all-to-all
 * reduce-scatter; Background, ZeRO++; Design, Communication Volume Analysis).
 * On one GPU the slices are separate device buffers; on a node they can be
 * the peers' buffers mapped into this GPU's address space.
 *   packed_slices  device array of P pointers; slice p holds ceil(m/2) bytes
 *   scale_slices   device array of P pointers; slice p holds ceil(m/block) floats
 * Same arithmetic, order and output as qgz_reduce_level on the slices laid
 * out back to back (bit-identical).  The two pointer arrays must be 8-byte
 * aligned and stay unchanged until the call completes; when m % 32 == 0 each
 * byte slice must be 16-byte aligned and each scale slice 4-byte aligned.
 * The library cannot read the device-resident pointers on the host, so only
 * the arrays themselves are checked against the outputs for overlap; the
 * slices must not overlap the outputs either.  Other conventions and errors
 * as qgz_reduce_level. */
int qgz_reduce_level_gather(const uint8_t* const* packed_slices, const float* const* scale_slices, int32_t P,
                            int64_t m, int32_t block, uint8_t* packed_out, float* scales_out, void* stream);

/* Allocation-free form of qgz_reduce_level_gather, for callers that cannot
 * allocate device memory (code under HIP graph capture, tight serving loops,
 * harnesses that forbid allocation).  The P slice addresses come in HOST
 * arrays.  Up to 64 slices they travel as arguments of the one kernel launched;
 * for more the library writes them into a static device table of its own (one
 * per GPU, 2048 addresses = 16 KiB, held until the process ends) with small
 * kernels on `stream` whose values travel as kernel arguments, then runs the
 * gathered reduce over them.  Nothing is allocated and nothing synchronises.
 *   packed_slices  host array of P device pointers; slice p holds ceil(m/2) bytes
 *   scale_slices   host array of P device pointers; slice p holds ceil(m/block) floats
 *   packed_out, scales_out as qgz_reduce_level (both required)
 * The host arrays are read before the call returns.  1 <= P <= 1024 (larger P
 * is ZQ_E_P: the table holds 1024 pairs).  Because the addresses are on the
 * host, every slice is checked: non-null (ZQ_E_NULL), 16-byte aligned when
 * m % 32 == 0 and scale slices 4-byte aligned (ZQ_E_ALIGN), no overlap with
 * an output (ZQ_E_ALIAS).  The table belongs to the current device, and
 * `stream` must belong to it too.  Every call of more than 64 slices on one GPU
 * uses the same table: such calls that can overlap on one GPU (different
 * streams, or different host threads without ordering) race on it; calls on one
 * stream are ordered.
 * Results are bit-identical to qgz_reduce_level_gather (and qgz_reduce_level
 * on the slices back to back). */
int qgz_reduce_level_gather_noalloc(const uint8_t* const* packed_slices, const float* const* scale_slices, int32_t P,
                                    int64_t m, int32_t block, uint8_t* packed_out, float* scales_out, void* stream);

/* Dequantise-on-load GEMM: the forward product of a layer whose weight
 * arrives as the gathered INT8 buffer (Design, Weight Partitioning: the
 * Allgathered weights are dequantised for the forward pass), without writing
 * the dequantised weight to memory:
 *   y[m][n] = sum_k x[m][k] * w[n][k],  w[n][k] = cvt(fl(q[n*K + k] * s[(n*K + k) / block]))
 * i.e. w is exactly what qwz_dequantize(codes, scales, N*K, block, ., xt)
 * writes, and the sum is taken in binary32 by the matrix cores in an order of
 * their own, always within 2*K*2^-24 * sum_k |x[m][k] w[n][k]| of the exact
 * value.  When the output tiles alone would leave much of the GPU idle (few
 * rows, or a few hundred rows with few tiles), the K range may be split across
 * workgroups whose partial sums are added into y atomically (after the
 * library zeroes y), so such results can differ between runs in their last
 * bits.
 *   x       [M][K] row-major, xt = ZQ_BF16 or ZQ_F16 (read)
 *   codes   [N][K] int8 row-major (a PyTorch Linear weight, flattened), scales
 *           [ceil(N*K/block)] floats (read)
 *   y       [M][N] float row-major (written)
 * K must be a multiple of 64 (ZQ_E_SIZE otherwise); M, N >= 0 arbitrary; K = 0
 * writes zeros.  x and codes 16-byte aligned, scales and y 4-byte aligned; y
 * must not overlap an input.  Other conventions as above.
 * When to use it: on MI355X this call is faster than qwz_dequantize of the
 * layer followed by a library bf16 GEMM (hipBLASLt) up to about 1,000 rows of
 * x (GPT-20B layer's four GEMMs: 0.12 against 0.54 ms at 16 rows, 0.19 against
 * 0.52 ms at 64, 1.00 against 1.15 ms at 1,024).  With many more rows
 * the separate path wins (6.0 against 5.2 ms at 8,192), so large batches
 * should dequantise the gathered layer once and call a library GEMM. */
int qwz_dequant_gemm(const void* x, zq_dtype xt, const int8_t* codes, const float* scales, int64_t M, int64_t N,
                     int64_t K, int32_t block, float* y, void* stream);

/* ---- The embedding layer --------------------------------------------------
 * Rows of an embedding table by token id, and the table's gradient.  The table is
 * the first weight a rank gathers, and its gradient the largest it sends.
 * For these calls element arrays (table, y, dy, dw) need only the alignment of
 * their elements, ids that of theirs; rows may have any length up to 2^24.  An id
 * that is not in [0, V) names no row: such a token (padding, say as -1) gets a row
 * of zeros and takes no part in the gradient.
 *
 * zq_embedding: y[t][d] = cvt(fl(scale * table[ids[t]][d])).
 *   ids   [T] of type it = ZQ_I32 or ZQ_I64 (read)
 *   table [V][D] of dtype wt (read) -> y [T][D] of dtype yt (written) */
int zq_embedding(const void* ids, zq_dtype it, int64_t T, const void* table, zq_dtype wt, int64_t V, int64_t D,
                 float scale, void* y, zq_dtype yt, void* stream);

/* qwz_embedding: the same from the gathered INT8 table (Design, Weight
 * Partitioning), reading only the rows that occur:
 *   y[t][d] = cvt(fl(scale * fl(codes[f] * scales[f / block]))),  f = ids[t]*D + d,
 * i.e. with scale 1 the rows that qwz_dequantize writes.
 *   codes [V*D], scales [ceil(V*D/block)] (read); block as everywhere. */
int qwz_embedding(const void* ids, zq_dtype it, int64_t T, const int8_t* codes, const float* scales, int64_t V,
                  int64_t D, int32_t block, float scale, void* y, zq_dtype yt, void* stream);

/* zq_embedding_grad: the gradient of the table from the gradient dy of y, dense:
 *   dw[v][d] = cvt(fl(scale * sum_{t: ids[t] = v} dy[t][d]))   zeros where v does not occur
 * with accumulate != 0 added to what dw holds: dw[v][d] = cvt(fl(dw[v][d] + fl(scale *
 * sum))), rows that do not occur untouched.  Sums are taken in binary32 in an order that
 * follows from the ids alone (tokens ascending; where a row has many, 64 at a time, and
 * then these sums ascending), so results are the same in every run.
 *   dy [T][D] of dtype gt (read), dw [V][D] of dtype wt (written)
 *   workspace: device memory of zq_embedding_grad_bytes(T, V, D) bytes or more, 16-byte
 *   aligned, the call's own until it has run (may be NULL where that is 0: few tokens).
 *   T, V <= 2^30, and T * ceil(V / 512) <= 2^41, since every 512 rows look through all
 *   ids (about 2 s for as many): else ZQ_E_SIZE, as is a workspace that is too small. */
int zq_embedding_grad(const void* ids, zq_dtype it, int64_t T, const void* dy, zq_dtype gt, int64_t V, int64_t D,
                      float scale, int accumulate, void* dw, zq_dtype wt, void* workspace, int64_t workspace_bytes,
                      void* stream);
int64_t zq_embedding_grad_bytes(int64_t T, int64_t V, int64_t D); /* -1 for sizes outside the limits */

/* ---- Gradient norm and clipping --------------------------------------------
 * The norm of all of a rank's gradients, and their scaling down to a largest norm,
 * over any number of tensors in one launch each.  A tensor is dense (n elements of
 * dtype ZQ_F32, ZQ_F16 or ZQ_BF16; aligned to its elements) or an INT4 shard as the
 * qgZ calls write it (dtype ZQ_INT4: data the packed codes at any address, scales
 * its block scales), which is read as it is.
 *   out  NULL: clipped in place (an INT4 shard: its scales); else out [n] of
 *        out_dtype receives the clipped elements (an INT4 shard's dequantised)
 * Outputs must not overlap each other or any tensor (in place: the tensor's own
 * memory); a tensor listed twice therefore needs an out for each. */
typedef struct {
  void* data;
  float* scales;     /* ZQ_INT4 only */
  void* out;
  int64_t n;
  int32_t dtype;
  int32_t out_dtype; /* with out */
  int32_t block;     /* ZQ_INT4 only */
  int32_t reserved;
} zq_grad;

/* Sizes of a table of tensors; filled by zq_grad_plan_make. */
typedef struct {
  int64_t bytes;       /* of the table */
  int64_t norm_chunks;
  int64_t clip_chunks;
  int32_t count;
  int32_t reserved;
} zq_grad_plan;

/* Host only.  zq_grad_plan_make checks the tensors (every argument error of the
 * calls below is found here) and fills plan; zq_grad_plan_table writes plan->bytes of
 * table to host memory.  The caller copies them to 16-byte aligned device memory,
 * once for as long as the tensors stay where they are: the calls keep their partial
 * sums in that copy and leave it ready for the next call.  Calls with one table must
 * be ordered (one stream, or events); calls with different tables need not be. */
int zq_grad_plan_make(const zq_grad* grads, int32_t count, zq_grad_plan* plan);
int zq_grad_plan_table(const zq_grad* grads, const zq_grad_plan* plan, void* host_table);

/* norm[0] = |scale| * sqrt(sum of the squares of all elements): squares and sums in
 * binary64, in a fixed order, rounded once; NaN or infinite where an element is.
 * `scale` undoes a loss scale or averages micro-batches.  plan on the host, table
 * and norm (a float) on the device. */
int zq_grad_norm(const zq_grad_plan* plan, void* table, float scale, float* norm, void* stream);

/* Multiplies every element by c = fl(scale * min(1, fl(max_norm / fl(norm[0] + 1e-6)))),
 * which is computed on the device from the norm there; a NaN norm makes every
 * element NaN, an infinite one makes c = 0:
 *   dense  out = cvt(fl(g * c))
 *   INT4   scales = fl(s * c) in place, or out = cvt(fl(q * fl(s * c)))
 * max_norm must be >= 0 (ZQ_E_SIZE).  In place with c = 1 nothing is read or written. */
int zq_grad_clip(const zq_grad_plan* plan, const void* table, const float* norm, float max_norm, float scale,
                 void* stream);

/* ---- Products with an INT4 weight --------------------------------------------
 * The few-row product of qwz_dequant_gemm for a weight in the INT4 format (4-bit
 * codes, one scale a block: a layer, or the output head, kept quantised for
 * generation), without dequantising it to memory:
 *   y[m][n] = sum_k x[m][k] * q[n*K + k] * s[(n*K + k) / block]
 * The weight is not narrowed: the codes' products are exact and summed in binary32 by
 * the matrix cores, each scale multiplies its block's sum (or a part of it), and these
 * are added in binary32, in a fixed order: within (K + 64) * 2^-23 * sum_k |x w| of
 * the exact value, the same bits in every run.  The bound holds where sum_k |x w| is 0
 * or from 2^-122 to the largest binary32 number and every x is 0 or of a magnitude from
 * 2^-110 to below 2^122 (fp16 always is): up to 128 products x * q / 16 are summed before
 * their scale is applied, which overflows beyond, and falls below the normal numbers
 * under it, whatever the scale.
 *   x       [M][K] row-major, xt = ZQ_BF16 or ZQ_F16 (read)
 *   packed  [ceil(N*K/2)] INT4 codes of the N x K weight, row-major, scales
 *           [ceil(N*K/block)] floats (read)
 *   y       [M][N] float row-major (written)
 * K a multiple of 64, at most 2^22 (ZQ_E_SIZE); M, N >= 0 arbitrary; K = 0 writes
 * zeros.  x and packed 16-byte aligned, scales and y 4-byte aligned.  Meant for few
 * rows: the weight is read again for every 64 rows of x.  (Up to 256 rows it is faster
 * than dequantising the weight and a library's product: 24,576 x 6,144, 256 rows 124 us
 * and 186; at 512 rows 235 and 208.)
 *   workspace: device memory of zq_int4_dequant_gemm_bytes(M, N, K) bytes or more, 4-byte
 *   aligned, the call's own until it has run (sums over slices of a long K; may be NULL
 *   where that is 0); one that is too small is ZQ_E_SIZE. */
int zq_int4_dequant_gemm(const void* x, zq_dtype xt, const uint8_t* packed, const float* scales, int64_t M, int64_t N,
                         int64_t K, int32_t block, float* y, void* workspace, int64_t workspace_bytes, void* stream);
int64_t zq_int4_dequant_gemm_bytes(int64_t M, int64_t N, int64_t K); /* -1 for sizes outside the limits */

/* ---- The optimizer's step ------------------------------------------------------
 * One AdamW step over any number of tensors in one launch (two, where only some have 8-bit
 * moments or an INT8 out): the owner's shard of the
 * optimizer states (Design, Optimizer-State Partitioning) updated from the gradient
 * shards as the reduce levels leave them, clipped on the way, and the weight written
 * in the form that is gathered next.  For every element, with t the step, fl() as
 * above, and c = fl(scale * min(1, fl(max_norm / fl(norm[0] + 1e-6)))), or scale
 * where norm is NULL:
 *   g = fl(grad * c)                  an INT4 shard: fl(q * fl(s * c)), as zq_grad_clip
 *   m = fl(fl(b1 * m) + fl(fl(1 - b1) * g))
 *   v = fl(fl(b2 * v) + fl(fl(1 - b2) * fl(g * g)))
 *   d = fl(fl(sqrt(v) * fl(1 / sqrt(1 - b2^t))) + eps)
 *   p = cvt(fl(fl(p * fl(1 - lr * lr_scale * weight_decay))
 *              - fl(fl(lr * lr_scale / (1 - b1^t)) * fl(m / d))))
 * b1, b2 and eps rounded to binary32; what depends on the step or on lr computed in
 * binary64 and rounded once.  A norm that is not finite leaves everything as it is.
 *
 * A tensor:
 *   param  [n] of param_dtype (F32 / F16 / BF16), updated in place
 *   grad   [n] of grad_dtype, or an INT4 shard (ZQ_INT4: packed codes at any address,
 *          grad_scales, grad_block)
 *   m, v   [n] floats (state_dtype ZQ_F32), or ZQ_F8: a byte an element and a float a
 *          block of state_block elements (m_scales, v_scales [ceil(n/state_block)]); m as
 *          e4m3 (OCP: 4 exponent bits of bias 7, 3 mantissa bits, largest 448), v as e5m2
 *          (bias 15, largest 57344; never negative), times their block's scale.  All zero
 *          bytes and scales are a fresh state.
 *   out    NULL, or what receives the new weight beside param: [n] of out_dtype (rounded
 *          from param as stored), or ZQ_INT8: what qwz_quantize of the new param writes
 *          (int8 codes at any address, out_scales, out_block)
 * Writing 8-bit moments: a = largest magnitude of the block, top = 448 or 57344; a below
 * 2^-110: scale 0 and codes 0; else scale = fl(a / top), and fl(|x| * fl(top / a)) is
 * rounded to a neighbouring code, up with the chance of the part cut off (16 bits of it),
 * so that changes smaller than a step are kept on average: nearest rounding would lose
 * every change of v by less than an eighth.  (m's sign is kept, that of a zero too.)  The bits drawn for element i of tensor k are
 * a function of (t, k, i) alone: the same step gives the same result.  With w = mix(key ^
 * (i mod 2^32)), key = mix(mix(mix(t) + k * 0x9E3779B9) + i / 2^32) (the outer mix only
 * where i / 2^32 > 0), mix(x): x ^= x >> 16, x *= 0x6A09E667, x ^= x >> 15, x *=
 * 0x3B67AE85, x ^= x >> 16 on 32 bits: m is rounded by w's low half, v by its high one.
 * Elements that are not finite leave the codes of their block unspecified.
 * Element arrays need the alignment of their elements, scales 4 bytes.  Nothing that is
 * written may overlap anything else of the table. */
typedef struct {
  void* param;
  const void* grad;
  const float* grad_scales; /* ZQ_INT4 only */
  void* m;
  float* m_scales;          /* ZQ_F8 only */
  void* v;
  float* v_scales;          /* ZQ_F8 only */
  void* out;
  float* out_scales;        /* ZQ_INT8 only */
  int64_t n;
  double weight_decay;
  double lr_scale;          /* of this tensor; 1 for the step's lr as it is */
  int32_t param_dtype;
  int32_t grad_dtype;
  int32_t state_dtype;
  int32_t out_dtype;        /* with out */
  int32_t grad_block;       /* ZQ_INT4 only */
  int32_t state_block;      /* ZQ_F8 only */
  int32_t out_block;        /* ZQ_INT8 only */
  int32_t reserved;
} zq_adamw;

/* Sizes of a table of tensors; filled by zq_adamw_plan_make. */
typedef struct {
  int64_t bytes;        /* of the table */
  int64_t pieces;       /* of tensors without blocks of their own */
  int64_t block_pieces; /* of those with 8-bit moments or an INT8 out */
  int32_t count;
  int32_t reserved;
} zq_adamw_plan;

/* A step's numbers.  0 <= beta1, beta2 < 1, eps >= 0, step >= 1, lr finite, and with a
 * norm max_norm >= 0 (else ZQ_E_SIZE). */
typedef struct {
  double lr, beta1, beta2, eps;
  int64_t step;   /* 1 for the first */
  float max_norm; /* with a norm */
  float scale;    /* of the gradients: undoes a loss scale, averages micro-batches */
} zq_adamw_args;

/* As zq_grad_plan_make and zq_grad_plan_table: the checks and the table, host only.  The
 * caller copies the table to 16-byte aligned device memory once for tensors that stay
 * where they are.  Calls with one table must be ordered. */
int zq_adamw_plan_make(const zq_adamw* tensors, int32_t count, zq_adamw_plan* plan);
int zq_adamw_plan_table(const zq_adamw* tensors, const zq_adamw_plan* plan, void* host_table);

/* The step.  plan and args on the host, table on the device.  norm: NULL, or a float on
 * the device (zq_grad_norm's, called with the same scale).  step, lr: NULL, or an
 * int64_t / a float on the device that is read in place of args' when the work runs
 * (one more small launch), for calls captured into a graph; a step below 1 there counts
 * as 1. */
int zq_adamw_step(const zq_adamw_plan* plan, void* table, const zq_adamw_args* args, const int64_t* step,
                  const float* lr, const float* norm, void* stream);

/* ---- RMS norm -------------------------------------------------------------------
 * The root-mean-square norm of T rows of D elements, after the residual's addition:
 *   h    = cvt(fl(x + residual))                     x itself without a residual
 *   rstd = 1 / sqrt(sum_d h[t][d]^2 / D + eps)       in binary64, rounded once
 *   y    = cvt(fl(fl(h * rstd) * weight))            weight NULL: cvt(fl(h * rstd))
 *   x, residual (may be NULL) [T][D] of dtype xt, weight [D] of dtype wt (read)
 *   h     [T][D] of xt: the sum, which is the next residual; required with a residual,
 *         else NULL (nothing is written).  May be residual's or x's own memory.
 *   y     [T][D] of yt, rstd [T] floats (NULL: not wanted) (written)
 * D from 1 to 2^24, eps >= 0 (ZQ_E_SIZE).  Element arrays need the alignment of their
 * elements; outputs overlap nothing but as said.  A row of zeros with eps 0 gives NaN. */
int zq_rms_norm(const void* x, const void* residual, zq_dtype xt, const void* weight, zq_dtype wt, int64_t T,
                int64_t D, double eps, void* h, void* y, zq_dtype yt, float* rstd, void* stream);

/* qwz_rms_norm: the same with y in the INT8 format, the codes and scales that
 * qwz_quantize gives for the binary32 values before the last rounding: an activation
 * kept or sent at half of bf16.  D a multiple of block (ZQ_E_SIZE).
 *   codes [T*D], scales [T*D/block] (written) */
int qwz_rms_norm(const void* x, const void* residual, zq_dtype xt, const void* weight, zq_dtype wt, int64_t T,
                 int64_t D, double eps, void* h, int8_t* codes, float* scales, int32_t block, float* rstd,
                 void* stream);

/* zq_rms_norm_grad: with xh = fl(h * rstd), gw = fl(dy * weight) (dy without a weight),
 *   dx[t][d] = cvt(rstd * (gw - xh * sum_d(gw * xh) / D) + dh[t][d])
 *   dw[d]    = cvt(sum_t dy[t][d] * xh[t][d])        accumulate != 0: added to what dw holds
 * dx is the gradient of x and of residual alike; dh (may be NULL) is the one that reaches
 * h by itself, along the residual's way.  Sums in binary32 in a fixed order that follows
 * from T and D alone: the same bits in every run.
 *   dy [T][D] of gt, h [T][D] of xt, weight [D] of wt (or NULL), rstd [T], dh [T][D] of xt
 *   dx [T][D] of xt (may be dh's own memory), dw [D] of dwt (NULL: not wanted)
 *   workspace: device memory of zq_rms_norm_grad_bytes(T, D) bytes or more, 16-byte
 *   aligned, the call's own until it has run (may be NULL where that is 0) */
int zq_rms_norm_grad(const void* dy, zq_dtype gt, const void* h, zq_dtype xt, const void* weight, zq_dtype wt,
                     const float* rstd, const void* dh, int64_t T, int64_t D, void* dx, int accumulate, void* dw,
                     zq_dtype dwt, void* workspace, int64_t workspace_bytes, void* stream);
int64_t zq_rms_norm_grad_bytes(int64_t T, int64_t D); /* -1 for sizes outside the limits */

/* ---- The loss at the output head ------------------------------------------------
 * Log-probabilities of given tokens, and the clipped policy loss with a KL term and its
 * gradient, from rows of V logits.  Row t of logits starts at element t * ld (ld >= V:
 * heads padded to a wider row), T * ld at most 2^59.  A logit of -infinity names a token
 * that cannot occur: probability and gradient 0.  As the row's own token it has logp
 * -infinity, a ratio of 0 and an infinite KL term, whatever old_logp and ref_logp hold; a
 * loss with that term is infinite, and so is its gradient in the logits whose exponential
 * is above 0 (at least 2^-126).  An id outside [0, V), or a row without any logit above
 * -infinity, names no token: logp 0, no loss, a gradient of zeros.
 *
 * zq_token_logp: logp[t] = scale * (z[a] - max z) - log(sum_v exp(scale * (z[v] - max z))),
 * a = ids[t]; exponentials and sums of 8 neighbours (4 of binary32 logits) in binary32, the
 * rest in binary64, rounded once.  Where a's probability is above a half the sum of its
 * neighbours is binary64 as well: one next to 1 keeps what the others leave of it.
 *   logits of dtype lt, ids [T] of type it = ZQ_I32 or ZQ_I64 (read), logp [T] (written)
 *   scale: 1 / temperature, above 0 and up to 2^127.  V from 1 to 2^24, T <= 2^30
 *   (ZQ_E_SIZE).  Logits whose difference is beyond binary32 count as infinitely far. */
int zq_token_logp(const void* logits, zq_dtype lt, int64_t T, int64_t V, int64_t ld, const void* ids, zq_dtype it,
                  float scale, float* logp, void* stream);

/* What zq_policy_loss takes beside the logits: device arrays of T floats, and numbers. */
typedef struct {
  const float* old_logp;   /* of the policy that drew the tokens */
  const float* advantages;
  const float* weights;    /* of each token in the sums: 0 for one that is masked, whose
                              other values may then be anything; NULL: 1 each */
  const float* ref_logp;   /* of the reference policy; needed where kl != 0 */
  float clip_low, clip_high; /* >= 0; clip_low <= 1 */
  float kl;                /* factor of the KL term, >= 0; 0: none */
  float scale;             /* of the logits: 1 / temperature, above 0 and up to 2^127 */
  float grad_scale;        /* of the gradient: a loss scale, the gradient of the loss */
  int32_t reserved;
} zq_policy;

/* zq_policy_loss: with logp as above, r = exp(logp - old_logp), A = advantages, lo = 1 -
 * clip_low, hi = 1 + clip_high, u = ref_logp - logp:
 *   policy[t] = -min(r * A, clip(r, lo, hi) * A)       KL[t] = exp(u) - u - 1
 *   sums = { sum w (policy + kl * KL), sum w policy, sum w KL, sum w [r is clipped] }
 *   grad[t][v] = grad_scale * w * scale * (kl * (1 - exp(u)) - (r is clipped ? 0 : r * A))
 *                * ((v == ids[t]) - softmax(scale * z)[v])
 * r is clipped where A > 0 and r > hi, or A < 0 and r < lo.  Terms and sums are binary64,
 * in a fixed order; sums[0] is the loss.
 *   sums [4], logp [T] floats (written; logp NULL: not wanted)
 *   grad rows of dtype gt from element t * ldg (ldg >= V; what lies between rows stays as
 *        it is); may be logits itself with gt = lt and ldg = ld; NULL: not wanted
 *   workspace: device memory of zq_policy_loss_bytes(T) bytes or more, 16-byte aligned,
 *   the call's own until it has run */
int zq_policy_loss(const void* logits, zq_dtype lt, int64_t T, int64_t V, int64_t ld, const void* ids, zq_dtype it,
                   const zq_policy* policy, float* sums, float* logp, void* grad, zq_dtype gt, int64_t ldg,
                   void* workspace, int64_t workspace_bytes, void* stream);
int64_t zq_policy_loss_bytes(int64_t T); /* -1 for sizes outside the limits */

/* Size helpers (host only): number of scales ceil(n/block) (-1 on a bad
 * block or n < 0), and INT4 bytes ceil(n/2) (-1 for n < 0). */
int64_t zq_num_scales(int64_t n, int32_t block);
int64_t zq_int4_bytes(int64_t n);

/* Static, human-readable name of a status code. */
const char* zq_status_string(int status);

#ifdef __cplusplus
}
#endif

#endif /* ZQ_H */
