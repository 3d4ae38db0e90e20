/*
 * bpc.h -- C ABI of the two-way error-feedback gradient-compression hot path
 * for one AMD MI355X (gfx950), and of distillation from a teacher's logits that
 * are sent as top-k messages (further down).
 *
 * The library implements, on one GPU, the arithmetic of the paper's gradient
 * aggregation with compression and error feedback (Algorithm 4), its variant
 * without error feedback (Algorithm 3), four compressors C (scaled sign,
 * top-k, random-k, linear dithering; Section 3.2 and Definitions 1-2) plus the
 * identity map, and the moment / parameter update of compressed LANS
 * (Algorithm 5, the lines after the push-pull call; identical to the same
 * lines of Algorithm 2).  Of the other methods the paper's evaluation lists
 * (Section 5.1): natural dithering shares the dithering record, linear
 * dithering goes up to 63 levels (the 5- and 7-bit forms), top-k can send
 * half-precision values, and the FP32 -> FP16 conversion is a kind of its own.
 *
 * Conventions common to every entry point
 * ---------------------------------------
 *  - "device" pointers are HIP device memory of the current device; "host"
 *    pointers are ordinary process memory.  All device buffers are owned by the
 *    caller.  The library allocates no device memory.  What it keeps between
 *    calls, per process: the last HIP error code of each calling thread; per
 *    device, the number of workgroups of each of its kernels that the device
 *    holds at once (found out on the first call that needs it), and, for the
 *    single-pass kernels described under bpc_workspace_check(), the stream of
 *    their last launch plus one event used to order launches on different
 *    streams.
 *  - Work is enqueued on `hip_stream` (a hipStream_t passed as void*; NULL is
 *    the default stream) and the call returns without synchronising, with one
 *    exception: when a single-pass kernel has to be ordered after one launched
 *    on a stream that no longer exists, the call waits for the whole device
 *    (hipDeviceSynchronize) instead.
 *  - A flat gradient of D elements is cut into partitions of `part_elems`
 *    elements (the last one may be shorter, D need not be a multiple).  Every
 *    compressor, scale, norm, k and residual rule applies per partition.
 *    `part_elems` must be a positive multiple of 1024, at most 2^28.
 *  - Every device pointer must be 16-byte aligned.
 *  - Arguments are validated on the host before the first HIP call; a failed
 *    validation touches no device memory and enqueues nothing.
 *  - Behaviour is defined for finite inputs only.
 *  - Calls that share a workspace, a residual or a payload buffer must be
 *    ordered by the caller (same stream or events).
 *  - The calls can be recorded into a HIP graph (stream capture): scratch is
 *    cleared by kernels, and nothing else is enqueued.  The first call of a
 *    kind on a device queries occupancy and sets function attributes, which a
 *    capture does not allow: make each call once eagerly on that device before
 *    capturing it.  Keeping replays of such a graph apart from other bpc calls
 *    running at the same time on the same device is up to the caller (eager
 *    calls on different streams are kept apart by the library).
 *  - TOPK, TOPK16 and RANDK take at most 65535 partitions per call
 *    (BPC_ERR_UNSUPPORTED beyond).
 *
 * Message ("payload") format, one record per partition, records at a fixed
 * stride of bpc_partition_stride() bytes, record p at byte p*stride (unless
 * partitions bypass compression: see bpc_params_t::bypass).  All
 * fields little-endian, 32 bit.  d = elements of that partition, k = its
 * number of kept elements, k_cap = k of a full partition, ru4(x) = x rounded
 * up to a multiple of 4.
 *
 *   IDENTITY  u32 zero[4];            f32 q[d]
 *   SIGN      f32 sigma; u32 zero[3]; u32 bits[ru4(ceil(d/32))]
 *             element j -> word j/32, bit j%32 (LSB first); bit = (q_j < 0);
 *             bits past d are 0.  decode: bit ? -sigma : +sigma.
 *   TOPK      u32 k; u32 zero[3];     i32 idx[ru4(k_cap)]; f32 val[ru4(k_cap)]
 *             first k entries used, idx strictly ascending, partition-local.
 *   TOPK16    u32 k; u32 zero[3];     i32 idx[ru4(k_cap)]; u16 val[2*ru4(ceil(k_cap/2))]
 *             as TOPK, the values as IEEE binary16 (round to nearest even);
 *             half-words past k are 0.  The kept slots of the residual hold
 *             what the rounding dropped.
 *   RANDK     u32 k; u32 zero[3];     f32 val[ru4(k_cap)]
 *             indices are regenerated by the receiver from (seed, stream_id,
 *             partition number): draw t uses word t%4 of Philox4x32-10 block
 *             t/4, idx_t = (word * d) >> 32 (64-bit product).
 *   DITHER    f32 nu; u32 zero[3];    u32 nib[ru4(ceil(d/8))]
 *             element j -> word j/8, bits 4*(j%8)..4*(j%8)+3;
 *             nibble = (q_j < 0 ? 8 : 0) | (level & 7), 0 <= level <= levels;
 *             nibbles past d are 0.
 *             levels > 7 (the 5-bit form up to 15 levels, the 7-bit form up to
 *             63): `planes` = 1, 2 or 3 bit planes follow for levels <= 15, 31,
 *             63.  Plane t starts at word 4 + ru4(ceil(part_elems/8)) +
 *             t*ru4(ceil(part_elems/32)) of the record (fixed by part_elems,
 *             whatever d is) and holds u32 bits[ru4(ceil(d/32))]: element j ->
 *             word j/32, bit j%32 = bit 3+t of its level; bits past d are 0.
 *             decode: +-(nu * level) / levels.
 *   NATDITHER same record as DITHER; decode: level 0 -> 0, else
 *             +-(nu * 2^(level-1)) / 2^(levels-1).
 *
 *   FP16      u32 zero[4];            u16 half[2*ru4(ceil(d/2))]
 *             element j -> IEEE binary16 of q_j, round to nearest even
 *             (past 65504: infinity; a NaN stays a NaN, payload unspecified);
 *             half-words past d are 0.  decode: the half widened (exact).
 *
 * Bytes of a record beyond the fields listed for its own d and k are
 * unspecified.
 *
 * Philox4x32-10 (Salmon et al., SC'11): counter = (block, partition number,
 * stream_id low 32, stream_id high 32), key = (seed low 32, seed high 32).
 */
#ifndef BPC_H_
#define BPC_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  BPC_OK = 0,
  BPC_ERR_INVALID_ARG = 1, /* null pointer, bad size, bad enum, bad ratio ... */
  BPC_ERR_UNSUPPORTED = 2, /* valid in principle, outside what is built */
  BPC_ERR_WORKSPACE = 3,   /* workspace missing or smaller than required */
  BPC_ERR_ALIGNMENT = 4,   /* a device pointer is not 16-byte aligned */
  BPC_ERR_HIP = 5,         /* a HIP call failed; see bpc_last_hip_error() */
  BPC_ERR_WAIT = 6         /* bpc_workspace_check(): a device-side wait gave up */
} bpc_status_t;

typedef enum {
  BPC_IDENTITY = 0, /* C = identity: Algorithms 3/4 reduce to Algorithm 1 */
  BPC_SIGN = 1,     /* scaled sign, C(v) = ||v||_1/d * sign(v) (Definition 2) */
  BPC_TOPK = 2,     /* k largest magnitudes, lowest index wins ties */
  BPC_RANDK = 3,    /* k indices drawn uniformly with replacement */
  BPC_DITHER = 4,   /* linear dithering: stochastic rounding to `levels` steps */
  BPC_NATDITHER = 5, /* natural dithering: stochastic rounding to the power-of-two
                        levels nu * 2^(l-levels), l = 1..levels, and 0 */
  BPC_FP16 = 6,      /* data type conversion FP32 -> FP16 (Section 4.1, the conversion
                        used inside a node; the half-precision method of Section 5.1) */
  BPC_TOPK16 = 7     /* top-k with half-precision values: the 32-bit index + 16-bit value
                        message behind the compression rate quoted in Section 5.2 */
} bpc_kind_t;

/* Gradients are F32 or F16; logits may be BF16 too. */
typedef enum { BPC_F32 = 0, BPC_F16 = 1, BPC_BF16 = 2 } bpc_dtype_t;
typedef enum { BPC_NORM_L2 = 0, BPC_NORM_LINF = 1 } bpc_norm_t;
typedef enum {
  BPC_OPT_LANS = 0, /* Algorithm 5 as printed (block-normalised update) */
  BPC_OPT_ADAM = 1  /* same moments and ratio r, update x -= lr*(r + wd*x) */
} bpc_opt_kind_t;

/* Compressor description.  Plain data, host memory, passed by pointer. */
typedef struct bpc_params {
  int32_t kind;        /* bpc_kind_t */
  int32_t norm;        /* bpc_norm_t; DITHER and NATDITHER only */
  uint64_t part_elems; /* elements per partition, multiple of 1024, <= 2^28 */
  double k_ratio;      /* TOPK/RANDK: k = max(1, floor(k_ratio*d)), 0<k_ratio<=1 */
  uint32_t levels;     /* DITHER: number of intervals s, 1..63; NATDITHER: number of
                          non-zero levels s, 1..7 */
  float value_scale;   /* RANDK decode multiplier; negative means d/k */
  uint64_t seed;       /* Philox key (RANDK, DITHER) */
  uint64_t stream_id;  /* Philox counter words 2,3: caller encodes step/role/worker */
  const float *norm_override; /* device, one f32 per partition, or NULL.  When set,
                          SIGN uses it as sigma and DITHER as nu instead of
                          reducing over the partition (lets a test fix the scale
                          so that every level bit is decided on equal terms). */
  const uint8_t *bypass; /* HOST, one byte per partition of the gradient the call is
                          given, or NULL.  The size threshold of Section 4.2 (tensors
                          under a threshold are not compressed): a partition whose byte
                          is non-zero is carried as it is -- its record is an IDENTITY
                          record, its residual becomes 0 -- whatever `kind` says; the
                          others are compressed by `kind`.  Records then no longer lie
                          at a fixed stride: record p follows record p - 1 directly
                          (bpc_partition_offset()).  A call works through the gradient
                          run by run, a run being a maximal stretch of partitions of
                          one class, with one set of kernel launches per run (FP16: all
                          runs in one launch, but for decode and LANS); at most 64
                          runs (BPC_ERR_UNSUPPORTED beyond).  The mask is read during
                          the call only.  Every params of one bpc_server_aggregate call
                          must mark the same partitions.  LANS with caller-defined
                          blocks does not take a mask with more than one run. */
} bpc_params_t;

/* Optimizer description for bpc_adaptive_update.  Host memory. */
typedef struct bpc_opt {
  int32_t kind;       /* bpc_opt_kind_t */
  float lr;           /* eta_t */
  float beta1, beta2; /* in (0,1) */
  float eps;          /* > 0 */
  float weight_decay; /* lambda */
  float bias_corr1;   /* 1 - beta1^t, computed by the caller in double */
  float bias_corr2;   /* 1 - beta2^t */
  float phi_lo, phi_hi; /* LANS scaling function phi(z) = min(max(z, lo), hi);
                           lo = 0, hi = +inf is the identity */
  uint32_t reserved;
  const uint64_t *block_offsets; /* LANS blocks G_b: device array of n_blocks+1
                           ascending element offsets, first 0, last D; NULL means
                           one block per partition */
  uint64_t n_blocks;  /* ignored when block_offsets is NULL */
} bpc_opt_t;

/* Number of kept elements of a partition with d elements (TOPK, RANDK);
 * 0 for other kinds or invalid parameters. */
uint64_t bpc_partition_k(const bpc_params_t *params, uint64_t d);

/* Byte stride between partition records of a payload; 0 on invalid params. */
size_t bpc_partition_stride(const bpc_params_t *params);

/* Bytes of the payload for a flat gradient of D elements (without a bypass
 * mask: number of partitions * stride); 0 on invalid params or D == 0. */
size_t bpc_payload_bytes(const bpc_params_t *params, uint64_t D);

/* Byte offset of partition p's record in a payload for D elements: p * stride
 * without a bypass mask; with one, the sum of the sizes of the records before it
 * (an IDENTITY record of part_elems elements for a bypassed partition, the kind's
 * stride for the others).  SIZE_MAX on invalid arguments. */
size_t bpc_partition_offset(const bpc_params_t *params, uint64_t D, uint64_t p);

/* Bytes of device workspace that any call with these params and this D may need,
 * bpc_adaptive_update with caller-defined LANS blocks excepted (see below).  n is
 * the number of worker messages (1..64; pass 1 for worker-side calls); it is only
 * validated: the layout has room for 64 messages whatever n is, so one workspace
 * of this size serves the worker, server and update calls of a step.  0 on
 * invalid arguments. */
size_t bpc_workspace_bytes(const bpc_params_t *params, uint64_t D, int n);

/* Bytes of device workspace bpc_adaptive_update needs when opt->block_offsets
 * lists n_blocks caller-defined blocks (n_blocks = 0: blocks are the partitions,
 * the same as bpc_workspace_bytes(params, D, 1)).  Never less than
 * bpc_workspace_bytes(params, D, 1).  0 on invalid arguments. */
size_t bpc_update_workspace_bytes(const bpc_params_t *params, uint64_t D, uint64_t n_blocks);

/* Byte offset, inside a workspace laid out for (params, D), of a u32 status word.  The
 * single-pass kernels synchronise workgroups through the workspace with bounded waits; the
 * word is cleared by every call that uses them and is non-zero afterwards only if a wait
 * gave up (results of that call are then undefined).  SIZE_MAX on invalid params. */
size_t bpc_workspace_status_offset(const bpc_params_t *params, uint64_t D);

/* Waits for `hip_stream` and reads the status word of `ws` (device, laid out for
 * (params, D); NULL: the static workspace of bpc_compress_static_ws on the current
 * device).  The single-pass kernels (SIGN, DITHER, NATDITHER on worker and
 * server, LANS, the fallback form of TOPK and TOPK16 for partitions of more than
 * 2097152 elements) exchange partition-wide sums between
 * workgroups through the workspace and rely on their whole grid being resident
 * on the device; should other work hold the device's compute units for seconds
 * (a replayed graph or another process running beside the call), a bounded wait
 * gives up rather than hang.  TOPK and TOPK16 calls with a k of at most 65536
 * wait too, each workgroup for one key of its partition; they wait only for a
 * workgroup that is running, so other work cannot keep them waiting unless it
 * takes a running workgroup off the device for seconds.  The entry points cannot see that (they do not
 * synchronise) and return BPC_OK; this call returns BPC_ERR_WAIT for it.  After
 * BPC_ERR_WAIT everything the last call on this workspace wrote or updated in
 * place (payload, residual, m, v, param) is undefined and must be restored by
 * the caller.  BPC_OK: no wait gave up since the last call that used `ws`. */
bpc_status_t bpc_workspace_check(const bpc_params_t *params, uint64_t D, const void *ws,
                                 void *hip_stream);

/*
 * Worker side of Algorithm 4 (residual != NULL) or Algorithm 3 (residual ==
 * NULL):  q = grad + residual;  payload = C(q);  residual = q - decode(payload).
 *   grad      device, D elements of `dtype`, read only; fp16 is widened exactly
 *   residual  device, D f32, updated in place, or NULL for no error feedback
 *   payload   device, bpc_payload_bytes() bytes, written
 *   ws        device workspace of ws_bytes >= bpc_workspace_bytes(params, D, 1)
 * D == 0 is a no-op returning BPC_OK.
 */
bpc_status_t bpc_compress(const bpc_params_t *params, const void *grad,
                          bpc_dtype_t dtype, float *residual, uint64_t D,
                          void *payload, void *ws, size_t ws_bytes,
                          void *hip_stream);

/*
 * bpc_compress for callers that cannot allocate device memory, a workspace
 * included (code running under HIP graph capture, tight serving loops,
 * harnesses that forbid hipMalloc): same arguments without `ws`, same kernels,
 * same results.  The workspace is an array of BPC_STATIC_WS_BYTES that is part
 * of the library's device code, so every device the library runs on holds it
 * from the first call there until the process ends.  The first call on a
 * device looks up the array's address (and creates the event that orders
 * single-pass kernels across streams): make it once before capturing.
 *   - BPC_ERR_WORKSPACE if bpc_workspace_bytes(params, D, 1) exceeds
 *     BPC_STATIC_WS_BYTES; nothing is enqueued then.  (4 MiB covers SIGN, DITHER,
 *     NATDITHER, FP16 and IDENTITY up to about 8e8 elements in partitions of
 *     4 MiB of gradient, and the sparse kinds, which keep a dense f32 copy in
 *     the workspace, up to about 5e5 elements.)
 *   - All such calls on one device share the one array: calls that may run at
 *     the same time on a device (different streams, threads or graphs) race and
 *     must be ordered by the caller.  The array keeps the last call's contents;
 *     every call clears what it needs cleared.
 *   - bpc_workspace_check(params, D, NULL, stream) reads this workspace's
 *     status word.
 */
#define BPC_STATIC_WS_BYTES (4u << 20)
bpc_status_t bpc_compress_static_ws(const bpc_params_t *params, const void *grad,
                                    bpc_dtype_t dtype, float *residual, uint64_t D,
                                    void *payload, void *hip_stream);

/*
 * Dense decode of a payload: out = decode(payload), D f32 written (device).
 * This is what a worker does with the pulled message p_t (Section 4.1).
 */
bpc_status_t bpc_decompress(const bpc_params_t *params, const void *payload,
                            uint64_t D, float *out, void *hip_stream);

/*
 * Server side of Algorithm 4 / 3:
 *   Delta = (sum_{i=0..n-1} decode(payloads[i])) * (1/n) + server_residual
 *   out_payload = C(Delta);  server_residual = Delta - decode(out_payload)
 * The sum runs in worker order in f32.
 *   in         host array of n params (same kind, part_elems, k_ratio, levels,
 *              value_scale; stream_id/seed per worker, used by RANDK: if all
 *              workers share one stream their value vectors are summed before
 *              the scatter).  SIGN: if every in[i].norm_override is the same non-NULL
 *              pointer, that states that all workers compressed with that one array
 *              of scales; where the n scales of a partition are then bit-identical
 *              and short (positive, normal, the low six bits of the significand
 *              clear, so that every partial sum m * sigma, |m| <= 64, is exact) the
 *              sum may be formed from bit counts as sigma * (n - 2 c), which is the sum
 *              in worker order to the bit (done for n = 16); elsewhere the additions are made.
 *              The override itself is not read by this call.
 *   payloads   host array of n device pointers (TOPK / TOPK16: the ascending
 *              order of idx is relied on; a record that breaks it gives an
 *              unspecified Delta, never an access outside the buffers)
 *   out        params of the recompression (same kind and part_elems as `in`)
 *   server_residual  device, D f32 in place, or NULL (Algorithm 3: no "+ e~")
 *   ws         >= bpc_workspace_bytes(out, D, n)
 */
bpc_status_t bpc_server_aggregate(const bpc_params_t *in,
                                  const void *const *payloads, int n,
                                  const bpc_params_t *out,
                                  float *server_residual, uint64_t D,
                                  void *out_payload, void *ws, size_t ws_bytes,
                                  void *hip_stream);

/*
 * Algorithm 5, moment and parameter update, fused with the decode of the
 * pulled message:  g = decode(payload), then per element
 *   m = beta1*m + (1-beta1)*g;  v = beta2*v + (1-beta2)*g*g
 *   r = (m/bias_corr1) / (sqrt(v/bias_corr2) + eps);  c = g / (same denominator)
 * LANS:  x -= lr * phi(||x_b||) * (beta1*(r+wd*x)/||r+wd*x||_b
 *                                  + (1-beta1)*(c+wd*x)/||c+wd*x||_b)
 *        with L2 norms over block b; a term whose norm is 0 contributes 0.
 *        (Where partitions are a multiple of 8192 elements the kernels form r
 *        and c with reciprocals, a few ulp from the quotients above, and sum
 *        the squares of 512 elements at a time in f32 (a tree) before the f64
 *        sums of the norms; m and v are exact.)
 * ADAM:  x -= lr * (r + wd*x).
 *   param, m, v  device, D f32 each, updated in place
 *   ws           >= bpc_update_workspace_bytes(params, D, opt->block_offsets ?
 *                opt->n_blocks : 0)
 */
bpc_status_t bpc_adaptive_update(const bpc_params_t *params,
                                 const void *payload, uint64_t D, float *param,
                                 float *m, float *v, const bpc_opt_t *opt,
                                 void *ws, size_t ws_bytes, void *hip_stream);

/*
 * Distillation from a teacher's top logits
 * ----------------------------------------
 * Teachers send students the k largest logits of every row (token, image) as a
 * top-k message instead of the whole row: bpc_logits_topk() makes the messages,
 * bpc_distill_loss(), bpc_distill_grad() and bpc_distill_step() are the
 * student's loss against them and its gradient with respect to the student's
 * logits.
 *
 * Logits are rows of `vocab` elements of `dtype` (F32, F16, BF16), row r at
 * element r * row_stride of a 16-byte aligned buffer; row_stride >= vocab is any
 * number, so rows need not be aligned.  Elements between rows are never written.
 *
 * A message is one record per row, record r at byte r * bpc_logits_stride():
 *   TOPK    u32 n; f32 rest; f32 top; u32 zero;  i32 idx[ru4(k)]; f32 val[ru4(k)]
 *   TOPK16  u32 n; f32 rest; f32 top; u32 zero;  i32 idx[ru4(k)]; u16 val[2*ru4(ceil(k/2))]
 *     n <= k   entries listed: the k largest logits of the row, ties to the lowest
 *              index, a NaN above +inf; -inf (a masked logit) is never listed
 *     top      the row's largest logit (-inf where n = 0)
 *     idx      strictly ascending; -1 from n to k (-0 and +0 are the same number)
 *     val      logit - top (TOPK16: as IEEE binary16, round to nearest even); -inf
 *              from n to k
 *     rest     sum over the logits not listed of exp((logit - top) / temperature)
 *   Bytes of a record past these fields are unspecified.  The student's calls read
 *   n, rest, idx and val; whatever a record says, they read and write inside
 *   their buffers (n is cut to k, entries with idx outside the vocabulary are
 *   skipped; an index that is listed twice gives an unspecified result for its row).
 *
 * With student logits s, c = 1 / temperature, p = softmax(s c), S the listed indices,
 * e_i = exp(val_i c), Q = sum_S e_i (TAIL_DROP) or sum_S e_i + rest (TAIL_REST),
 * q_i = e_i / Q, q_R = rest / Q, p_R = the sum of p outside S:
 *   KL_r   = sum_S q_i log(q_i / p_i)                        (+ q_R log(q_R / p_R) with TAIL_REST)
 *   CE_r   = -log softmax(s)[label_r]                         (at temperature 1)
 *   loss_r = row_weight_r * (soft_weight * KL_r + hard_weight * CE_r)
 *   d loss_r / d s_j = row_weight_r * (soft_weight c (p_j - q_j) + hard_weight (softmax(s)_j - [j = label_r]))
 *            where for j outside S  q_j = q_R p_j / p_R with TAIL_REST, 0 with TAIL_DROP.
 *   (The usual soft weight is alpha * temperature^2.)
 *   - TAIL_DROP renormalises the teacher over its listed words; TAIL_REST compares
 *     the mass of all others as one more word.
 *   - A row of row_weight 0 has loss 0 and a gradient of zeros, its logits are not read.
 *   - A record with n = 0 (or soft_weight 0) gives no soft term, a label outside
 *     [0, vocab) (or labels NULL, or hard_weight 0) no hard term.  A row with neither has
 *     loss 0 and a gradient of zeros, whatever its logits are.
 *   - Masked student logits (-inf) have probability and gradient 0; if the teacher
 *     gives such a word (or, with TAIL_REST, a rest that is masked as a whole) mass,
 *     the loss is +inf and the gradient of the listed words still -q_i.  A label that is
 *     masked gives the loss +inf, too, and its word -1 in place of softmax - 1.
 *   - Logits without a softmax (a NaN or +inf among them, or all of them -inf) make the loss
 *     and the gradient of a row that has either term NaN.  In a teacher's row a NaN or +inf
 *     makes values of its record NaN, and so the student's soft term.
 * Unlike the gradient path these calls take infinities and NaN as described.  Sums are
 * formed in f32 in a fixed order: the same inputs give the same bits (in rows that start
 * elsewhere in their 128-byte line, or of another number, sums may be formed in another order).
 * Limits (BPC_ERR_UNSUPPORTED beyond): vocab <= 2^24, k <= BPC_LOGITS_MAX_K (k may exceed
 * vocab), rows < 2^22.  rows == 0 is a no-op returning BPC_OK.
 * Time: bpc_logits_topk() takes rows of more than 2^18 logits (counted in whole vectors of 16
 * bytes from the first that a row may start in) and rows in which far more than k logits are level
 * with the k-th by a radix select: 4096 rows of 262,080 bf16 logits 0.46 ms, of 262,208 3.6 ms;
 * 4096 equal rows of 50,257 3.1 ms for 0.11.
 */
#define BPC_LOGITS_MAX_K 1024
#define BPC_DISTILL_STATS_BYTES 32
typedef enum { BPC_TAIL_DROP = 0, BPC_TAIL_REST = 1 } bpc_tail_t;
typedef struct bpc_distill {
  int32_t kind;        /* BPC_TOPK: f32 values in the messages, BPC_TOPK16: half */
  int32_t tail;        /* bpc_tail_t */
  uint32_t vocab;      /* logits per row */
  uint32_t k;          /* entries a record has room for */
  float temperature;   /* 1e-30 .. 1e30 */
  float soft_weight, hard_weight;
  uint32_t reserved;
} bpc_distill_t;

/* Byte stride between the records of a message; 0 on invalid arguments. */
size_t bpc_logits_stride(const bpc_distill_t *d);

/* Bytes of the messages of `rows` rows; 0 on invalid arguments or rows == 0. */
size_t bpc_logits_message_bytes(const bpc_distill_t *d, uint64_t rows);

/* Bytes of device workspace that any of the calls below may need for up to `rows`
 * rows of any type (at least 256); 0 on invalid arguments or beyond the limits. */
size_t bpc_distill_workspace_bytes(const bpc_distill_t *d, uint64_t rows);

/*
 * Teacher: the message of `rows` rows of logits.
 *   row_weight  device, f32 per row, or NULL.  Rows of weight 0 are not read and get
 *               the empty record (n = 0, rest = 0, top = -inf).
 *   messages    device, bpc_logits_message_bytes() bytes, written
 *   ws          device workspace of ws_bytes >= bpc_distill_workspace_bytes(d, rows)
 */
bpc_status_t bpc_logits_topk(const bpc_distill_t *d, const void *logits, bpc_dtype_t dtype,
                             uint64_t row_stride, uint64_t rows, const float *row_weight,
                             void *messages, void *ws, size_t ws_bytes, void *hip_stream);

/*
 * Student: loss of each row.
 *   labels      device, i64 per row, or NULL
 *   row_weight  device, f32 per row, or NULL (all 1)
 *   loss        device, f32 per row, written
 *   stats       device, BPC_DISTILL_STATS_BYTES per row, written, or NULL: what
 *               bpc_distill_grad() of the same rows needs (contents unspecified)
 */
bpc_status_t bpc_distill_loss(const bpc_distill_t *d, const void *logits, bpc_dtype_t dtype,
                              uint64_t row_stride, uint64_t rows, const void *messages,
                              const int64_t *labels, const float *row_weight, float *loss,
                              void *stats, void *ws, size_t ws_bytes, void *hip_stream);

/*
 * Student: gradient of the sum of the losses with respect to the logits, from the
 * statistics that bpc_distill_loss() left for the same logits, messages and labels.
 *   row_weight  as above; to carry on a gradient g_r of loss_r, pass row_weight_r * g_r.
 *               A row whose weight was 0 in bpc_distill_loss() has no statistics: its
 *               weight must be 0 here too.  soft_weight and hard_weight may differ from
 *               those of bpc_distill_loss(), except that one that was 0 there must be 0
 *               here; everything else in `d` must be the same.
 *   grad        device, `rows` rows of `vocab` elements of `dtype`, row r at element
 *               r * grad_stride, written; may be the logits themselves
 *               (grad == logits and grad_stride == row_stride), otherwise must not overlap them
 */
bpc_status_t bpc_distill_grad(const bpc_distill_t *d, const void *logits, bpc_dtype_t dtype,
                              uint64_t row_stride, uint64_t rows, const void *messages,
                              const int64_t *labels, const float *row_weight, const void *stats,
                              void *grad, uint64_t grad_stride, void *hip_stream);

/*
 * Student: loss and gradient in one call; the logits are read once where a row stays in
 * registers (rows of up to 32 KB, of up to 128 KB in calls of 512 rows or more), and again
 * while they are in the last-level cache elsewhere.  Arguments as above.
 */
bpc_status_t bpc_distill_step(const bpc_distill_t *d, const void *logits, bpc_dtype_t dtype,
                              uint64_t row_stride, uint64_t rows, const void *messages,
                              const int64_t *labels, const float *row_weight, float *loss,
                              void *grad, uint64_t grad_stride, void *ws, size_t ws_bytes,
                              void *hip_stream);

/*
 * Measurement aid: a plain streaming kernel with the memory traffic of a stage and
 * none of its arithmetic, over n elements, to find what the device's memory
 * system delivers for that access pattern (to be read beside its peak figure).
 *   BPC_PROBE_COPY        c = a                 a, c: n f32        8 B/element
 *   BPC_PROBE_WORKER_MIX  c = widen(a) + b      a: n f16; b, c: n f32   10 B/element
 *                         (gradient and residual in, residual out: the worker
 *                         stage of Algorithm 4 without its message)
 *   BPC_PROBE_UPDATE_MIX  a, b, c <- b, c, a    three f32 arrays read and
 *                         written in place, 24 B/element (m, v, x of the update)
 * All pointers device, 16-byte aligned, arrays distinct; enqueues one kernel.
 */
typedef enum { BPC_PROBE_COPY = 0, BPC_PROBE_WORKER_MIX = 1, BPC_PROBE_UPDATE_MIX = 2 } bpc_probe_t;
bpc_status_t bpc_stream_probe(bpc_probe_t mix, const void *a, const void *b, void *c, uint64_t n,
                              void *hip_stream);

/* Static, never NULL. */
const char *bpc_status_string(bpc_status_t status);

/* hipError_t value of the last failed HIP call made by this thread, 0 if none. */
int bpc_last_hip_error(void);

#ifdef __cplusplus
}
#endif
#endif /* BPC_H_ */
