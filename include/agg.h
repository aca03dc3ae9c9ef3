/*
 * agg -- subsampled global attention (SGA) for VGGT-style models on AMD MI355X (gfx950).
 *
 * C ABI of libagg.so.  The operation is the one the AVGGT paper defines in its
 * Sec. 4.3 ("Subsampling Global Attention") on the token layout of its Sec. 4.1:
 * a sequence is N frames of L = n_special + n_h*n_w tokens; every token is a
 * query; keys/values are all special tokens, all of frame 0 when the reference
 * frame is kept whole, and on every other patch grid the first token of each
 * s_h x s_w window; a query whose own token was dropped also sees its own
 * key/value ("diagonal preservation"); all dropped patches are represented by
 * one mean key/value pair; the three parts share one softmax.
 *
 * Conventions
 *   - Token id inside a sequence: i = f*L + t.  t < n_special is a special token,
 *     otherwise patch p = t - n_special at grid row p / n_w, column p % n_w.
 *   - Q, K, V, O: bf16, device memory, contiguous [B, N*L, H, D] (token-major:
 *     what a fused QKV projection writes and an output projection reads).
 *   - D must be 64.  Pointers to bf16 tensors, to workspaces and to kmean/vmean must be
 *     16-byte aligned; index, count, bitmap and lse pointers 4-byte aligned.
 *   - `hip_stream` is a hipStream_t passed as void* (NULL = the default stream).
 *     Every call only enqueues work on that stream: no allocation, no
 *     synchronisation, no retained pointers.  The caller owns every buffer.
 *   - Results are bit-reproducible from run to run for the same shape.  Sums are formed in an order
 *     that may depend on the shape as a whole: the last bits of one row of O or lse may differ
 *     between calls that hold it with other numbers of queries, batch elements or heads, and those
 *     of kmean and vmean between calls with other B or H.  The error is the same.
 *   - Return value: AGG_OK or a negative agg_status.  All argument validation
 *     happens before the first launch, so every error except AGG_ERR_LAUNCH is
 *     reported without touching the GPU.  Faults inside a kernel surface at the
 *     caller's next synchronisation, as with any HIP launch.
 *
 * Compacted key/value format ("fragment order")
 *   Kc and Vc hold, per (batch, head), the M kept rows padded with zero rows to
 *   M_pad = 64*ceil(M/64), as consecutive 64-row tiles of 4096 bf16 (8 KiB).
 *   Inside a tile the elements are grouped in 16-byte chunks (eight channels of
 *   one key for Kc, eight keys of one channel for Vc) such that a copy into LDS
 *   chunk by chunk lets every wavefront lane fetch its MFMA operand as one
 *   16-byte read:
 *     Kc: row m, channel d  ->  tile m/64, then with km = m%64
 *         ((( (km/32)*4 + d/16 )*2 + (d%16)/8 )*32 + km%32)*8 + d%8
 *     Vc: row m, channel d  ->  tile m/64, then with km = m%64, u = km%16
 *         ((( km/16 )*2 + (u%8)/4 )*64 + d)*8 + (u/8)*4 + u%4
 *   agg_kc_offset()/agg_vc_offset() evaluate these on the host.  Row m of the
 *   compacted set is token idx[m]; idx is ascending.
 */
#ifndef AGG_H_
#define AGG_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct agg_shape {
  int32_t B, N;             /* batch size, frames                       (Sec. 4.1) */
  int32_t n_h, n_w;         /* patch grid                               (Sec. 4.1) */
  int32_t n_special;        /* special tokens per frame, stored before the patches */
  int32_t H, D;             /* heads, head dimension (D = 64)                      */
  int32_t s_h, s_w;         /* window strides; (1,1) = no subsampling   (Sec. 4.3) */
  int32_t keep_first_frame; /* 1: frame 0 kept whole (VGGT); 0: all frames (pi^3)  */
  uint32_t flags;           /* AGG_DIAG | AGG_MEAN                      (Sec. 4.3) */
  float scale;              /* softmax scale, 1/sqrt(D)                            */
  float mean_logit_bias;    /* added to the mean column's logit; 0 = one plain column */
} agg_shape;

enum { AGG_DIAG = 1u, AGG_MEAN = 2u };

typedef enum agg_status {
  AGG_OK = 0,
  AGG_ERR_NULL = -1,        /* a required pointer is NULL                          */
  AGG_ERR_SHAPE = -2,       /* a dimension or stride is < 1, flags unknown, or buffers overlap that may not */
  AGG_ERR_UNSUPPORTED = -3, /* D != 64; rows wider than the call takes              */
  AGG_ERR_ALIGN = -4,       /* a tensor pointer is not 16-byte aligned             */
  AGG_ERR_WORKSPACE = -5,   /* workspace smaller than the matching *_workspace_bytes */
  AGG_ERR_OVERFLOW = -6,    /* N*L, M_pad, a position, a matrix's rows or channels, or a tensor's element count exceeds
                               the index range */
  AGG_ERR_LAUNCH = -7       /* hipGetLastError() after a launch was not hipSuccess */
} agg_status;

const char* agg_status_string(int status);

/* Sec. 4.3 table: sigma in {2,4,6,9} -> (s_h, s_w) = (1,2),(2,2),(2,3),(3,3); sigma 1 -> (1,1).
 * Any other sigma: AGG_ERR_SHAPE. */
int agg_sigma_to_strides(int sigma, int32_t* s_h, int32_t* s_w);

/* Host only.  M = number of kept key/value rows per sequence,
 * n_dropped = number of patch tokens left out (Sec. 4.3).  Either output may be NULL. */
int agg_kv_count(const agg_shape* shape, int64_t* M, int64_t* n_dropped);

/* Host only.  The index set of Sec. 4.3 (special tokens, the reference frame when kept whole,
 * the first patch of every s_h x s_w window), as ascending token ids, into idx[M] (host memory):
 * what agg_kv_subsample writes on the device. */
int agg_kv_indices_host(const agg_shape* shape, int32_t* idx);

/* Host only.  Writes the ascending token ids of the dropped patches (the set the mean
 * component averages, Sec. 4.3) into idx[n_dropped] (host memory). */
int agg_dropped_indices_host(const agg_shape* shape, int32_t* idx);

/* Host only.  Size of ONE compacted tensor (Kc or Vc) in bytes, B*H*M_pad*D*2, and M_pad. */
int agg_kv_compact_bytes(const agg_shape* shape, size_t* bytes, int64_t* M_pad);

/* Host only.  Element offsets inside one (batch, head) block of Kc / Vc (see above). */
int64_t agg_kc_offset(int64_t m, int32_t d);
int64_t agg_vc_offset(int64_t m, int32_t d);

/* Host only.  Scratch bytes agg_kv_subsample needs: the partial sums from which the mean
 * component of Sec. 4.3 (one mean key/value pair over all dropped patches) is formed in a fixed
 * order. */
size_t agg_workspace_bytes(const agg_shape* shape);

/*
 * Sec. 4.3, subsampling + mean component.  Builds on the device:
 *   idx   [M] int32        ascending kept token ids (same for every batch element/head/layer)
 *   Kc,Vc bf16, agg_kv_compact_bytes() each, fragment order, zero padded
 *   kmean,vmean [B,H,D] float32: mean of K resp. V over all dropped patch tokens of the
 *         sequence (zeros when nothing is dropped).  Accumulated in a fixed order:
 *         results are bit-reproducible run to run.
 * K, V: device bf16 [B, N*L, H, D].  workspace: device, >= agg_workspace_bytes().
 * idx may be NULL (not written).  kmean/vmean must be non-NULL.  Kc and Vc may BOTH be NULL:
 * then no compacted copy is made and only idx and the mean terms are produced, which is all
 * that agg_global_attn_fwd_idx needs.
 */
int agg_kv_subsample(const agg_shape* shape, const void* K, const void* V, void* Kc, void* Vc,
                     int32_t* idx, float* kmean, float* vmean, void* workspace,
                     size_t workspace_bytes, void* hip_stream);

/*
 * agg_kv_subsample for callers that cannot allocate device memory and so cannot bring a
 * workspace: code under HIP graph capture, tight serving loops, harnesses that forbid
 * hipMalloc.  Same arguments, same kernels and bit-identical results, minus the workspace: the
 * partial sums of the mean go to a device array that is part of the library (each GPU the
 * library runs on holds agg_static_scratch_bytes() = 32 MiB of it until the process ends).
 * The call allocates nothing.  Shapes whose agg_workspace_bytes() exceeds
 * agg_static_scratch_bytes() are refused with AGG_ERR_WORKSPACE before anything is launched.
 * The first call on a device looks the array's address up (with that device current, which it
 * must be for every call).  All calls on one GPU share the array: two calls whose work may
 * overlap on that GPU (different streams) race; calls on one stream do not.
 */
size_t agg_static_scratch_bytes(void);
int agg_kv_subsample_static(const agg_shape* shape, const void* K, const void* V, void* Kc,
                            void* Vc, int32_t* idx, float* kmean, float* vmean, void* hip_stream);

/*
 * Sec. 4.3, the attention itself.  For every query i of every (batch, head):
 *   softmax over { scale*<q_i, Kc[m]> : m < M }
 *                u { scale*<q_i, k_i> }                    if AGG_DIAG and token i was dropped
 *                u { scale*<q_i, kmean> + mean_logit_bias } if AGG_MEAN and n_dropped > 0
 *   O[i] = sum of the probabilities times the matching value rows (Vc[m], v_i, vmean).
 * Q, K, V: device bf16 [B, N*L, H, D] (K, V are read only for the self terms).
 * Kc, Vc, kmean, vmean: as written by agg_kv_subsample for the same shape.
 * O: device bf16 [B, N*L, H, D].  lse: device float32 [B, H, N*L] (natural-log
 * log-sum-exp of each row's logits) or NULL.
 * With s_h = s_w = 1 nothing is dropped and the result is ordinary global attention.
 */
int agg_global_attn_fwd(const agg_shape* shape, const void* Q, const void* K, const void* V,
                        const void* Kc, const void* Vc, const float* kmean, const float* vmean,
                        void* O, float* lse, void* hip_stream);

/*
 * Sec. 4.3 again, without a compacted copy: the same attention as agg_global_attn_fwd, with the
 * kernel fetching the kept rows of K and V in place through idx (the paper's statement is just
 * that: only a subset of the tokens serves as keys and values).  idx: device int32 [M], the
 * ascending kept token ids as agg_kv_subsample writes them; kmean, vmean: as above.  Results are
 * bit-identical to agg_global_attn_fwd.  Needs N*L < 2^24 and N*L*H*D*2 < 2^32 (rows are
 * addressed with 32-bit offsets inside one batch element's head); otherwise AGG_ERR_OVERFLOW.
 */
int agg_global_attn_fwd_idx(const agg_shape* shape, const void* Q, const void* K, const void* V,
                            const int32_t* idx, const float* kmean, const float* vmean, void* O,
                            float* lse, void* hip_stream);

/*
 * Sec. 4.2: ordinary global attention over the (B, N*L, C) layout -- every token of the
 * sequence is a key -- the s = 1 baseline SGA is measured against.  shape->s_h, s_w,
 * flags and keep_first_frame are ignored.  K and V are read in place (no copy, no workspace).
 */
int agg_dense_global_attn_fwd(const agg_shape* shape, const void* Q, const void* K, const void* V,
                              void* O, float* lse, void* hip_stream);

/*
 * Sec. 4.2, Global-to-Frame conversion: attention applied independently inside every frame,
 * i.e. on the (B*N, L, C) layout -- what an early global block becomes when its rearrangement
 * to (B, N*L, C) is skipped.  Q, K, V, O: the same device tensors as above (a frame's tokens are
 * contiguous in them).  lse: device float32 [B*N, H, L] or NULL.  shape->s_h, s_w, flags and
 * keep_first_frame are ignored.
 */
int agg_frame_attn_fwd(const agg_shape* shape, const void* Q, const void* K, const void* V, void* O,
                       float* lse, void* hip_stream);

/*
 * One global-attention block around the calls above (Sec. 4.2: a converted or subsampled
 * block keeps all its other components and parameters):
 *     y = x + W_o * Attn( Q, K, V ) + b_o,   [Q|K|V] = W_{q,k,v} * LayerNorm(x) + b_{q,k,v}
 * with Attn chosen by `mode`.  x, y: device bf16 [B, N*L, C], C = H*D (y may not alias x).
 * Weights: device memory; w_*: bf16 [C, C], one row per OUTPUT channel (y = x W^T);
 * b_* (may be NULL), ln_gamma, ln_beta: float32 [C].  Q, K, V and the attention output
 * are bf16 tensors in the workspace, as in the calls above.  Rotary embeddings or
 * query/key normalisation, which the paper's text does not describe, are not applied
 * (agg_global_block_ex_fwd below applies them).
 * C may be at most 4096 (64 heads): wider blocks return AGG_ERR_UNSUPPORTED.
 */
typedef struct agg_block_weights {
  const float* ln_gamma;
  const float* ln_beta;
  float ln_eps;
  const void *w_q, *w_k, *w_v, *w_o;
  const float *b_q, *b_k, *b_v, *b_o;
} agg_block_weights;

enum {
  AGG_BLOCK_SGA = 0,   /* subsampled global attention, Sec. 4.3 (shape's strides and flags) */
  AGG_BLOCK_FRAME = 1, /* frame attention: the Global-to-Frame conversion, Sec. 4.2         */
  AGG_BLOCK_DENSE = 2  /* ordinary global attention                                         */
};

/* Host only.  Scratch bytes agg_global_block_fwd needs for `mode` (0 on an invalid shape). */
size_t agg_block_workspace_bytes(const agg_shape* shape, int mode);

int agg_global_block_fwd(const agg_shape* shape, int mode, const agg_block_weights* weights,
                         const void* x, void* y, void* workspace, size_t workspace_bytes,
                         void* hip_stream);

/*
 * ---- Caller-supplied key/value sets (supplementary ablation on the grid strategy) ----
 * The paper compares its fixed choice (first token of each window) with other choices of one
 * token per window: a random one, the one with the highest and the one with the lowest feature
 * magnitude.  These calls run the same attention over ANY list of kept tokens:
 *   list       device int32 [B, M_list]: token ids (0 <= id < N*L) whose K/V rows serve as
 *              keys/values of that batch element, in any order.  Ids outside the range are
 *              clamped into it (memory-safe, meaningless result); a repeated id counts twice.
 *   kept_bits  device uint32 [B, ceil(N*L/32)]: bit t%32 of word t/32 set <=> token t is listed
 *   n_dropped  device int32 [B]: patch tokens (slot >= n_special) that are not listed
 * The self term (AGG_DIAG) applies to every query whose token is not listed, the mean
 * component (AGG_MEAN) averages K resp. V over the unlisted patch tokens and is present when
 * n_dropped[b] > 0.  shape->s_h, s_w, keep_first_frame matter only to agg_select_kv_indices.
 */
enum {
  AGG_SELECT_FIRST = 0,  /* top-left token of each window: the paper's rule (Sec. 4.3)        */
  AGG_SELECT_RANDOM = 1, /* a pseudo-random token of each window                              */
  AGG_SELECT_HIGH = 2,   /* the token of each window with the largest sum of squares of its K */
  AGG_SELECT_LOW = 3     /* ... with the smallest                                             */
};

/*
 * Writes list[B, M] (M of agg_kv_count): row m of batch b is the token chosen for the m-th
 * kept position of the grid rule -- special tokens and (keep_first_frame) frame 0 map to
 * themselves, the m-th window of a subsampled frame to one of its tokens by `rule`:
 *   RANDOM: cell number  mix(mix(s ^ (b*N+frame)*0x85EBCA77) ^ window*0xC2B2AE3D) % cells,
 *           s = (uint32)seed ^ (uint32)(seed>>32)*0x9E3779B1, window = row-major window number
 *           inside the frame, cells counted row-major inside the (possibly clipped) window,
 *           mix(x): x^=x>>16; x*=0x7FEB352D; x^=x>>15; x*=0x846CA68B; x^=x>>16  (32-bit);
 *   HIGH/LOW: magnitude = sum over all H*D channels of K[b, token]^2 in float32; ties go to
 *           the earlier cell.
 * K: device bf16 [B, N*L, H, D]; read only for HIGH/LOW (may be NULL otherwise).
 */
int agg_select_kv_indices(const agg_shape* shape, int rule, uint64_t seed, const void* K,
                          int32_t* list, void* hip_stream);

/*
 * The cell-mean variant of the same ablation: Kc/Vc (agg_kv_compact_bytes each, M rows as for
 * agg_kv_subsample) where the row of a window is the MEAN of the window's tokens (float32
 * accumulation, rounded to bf16 once) instead of its first token; special tokens and a
 * whole-kept frame 0 are copied.  The paper runs this variant without the self term and without
 * the mean component: call agg_global_attn_fwd on the result with flags = 0.
 */
int agg_kv_pool(const agg_shape* shape, const void* K, const void* V, void* Kc, void* Vc,
                void* hip_stream);

/* Host only.  Size of ONE compacted tensor for a list of M_list rows, and its M_pad. */
int agg_list_compact_bytes(const agg_shape* shape, int64_t M_list, size_t* bytes, int64_t* M_pad);

/* Host only.  Scratch bytes agg_kv_subsample_list needs (0 on an invalid shape). */
size_t agg_list_workspace_bytes(const agg_shape* shape);

/* As agg_kv_subsample, for a caller's list: Kc/Vc (agg_list_compact_bytes each; row m of batch
 * b = token list[b, m]), kmean/vmean [B,H,D], kept_bits and n_dropped as defined above. */
int agg_kv_subsample_list(const agg_shape* shape, const int32_t* list, int64_t M_list,
                          const void* K, const void* V, void* Kc, void* Vc, float* kmean,
                          float* vmean, uint32_t* kept_bits, int32_t* n_dropped, void* workspace,
                          size_t workspace_bytes, void* hip_stream);

/* As agg_global_attn_fwd, over what agg_kv_subsample_list wrote for the same shape and M_list. */
int agg_global_attn_fwd_list(const agg_shape* shape, int64_t M_list, const void* Q, const void* K,
                             const void* V, const void* Kc, const void* Vc, const float* kmean,
                             const float* vmean, const uint32_t* kept_bits,
                             const int32_t* n_dropped, void* O, float* lse, void* hip_stream);

/*
 * ---- The other parts of a model's block ----
 * What the models around these attention layers put between projections and attention, and between
 * one block and the next.  Statistics, angles and sums are float32 or better; every output is rounded
 * to bf16 once.  As for every call, the device that holds the tensors must be the current one.
 */
enum {
  AGG_NORM_NONE = 0,  /* y = x                                                          */
  AGG_NORM_LAYER = 1, /* y = (x - mean) / sqrt(var + eps) * gamma + beta                */
  AGG_NORM_RMS = 2    /* y = x / sqrt(mean(x^2) + eps) * gamma + beta                   */
};
typedef struct agg_norm {
  int32_t kind;       /* AGG_NORM_*; NONE: the other fields are ignored                 */
  float eps;          /* > 0                                                            */
  const float* gamma; /* device float32, one per channel, 16-byte aligned; NULL: ones   */
  const float* beta;  /* ... NULL: zeros                                                */
} agg_norm;

/*
 * Rotary positions on three axes.  d_t, d_h, d_w channels of every head turn with the token's time,
 * row and column (each even, together at most D, 0 leaves an axis out); the channels behind them are
 * left as they are.  A pair (x, y) at position p of its axis becomes
 *     (x cos a - y sin a, y cos a + x sin a),   a = p * base^-e:
 *   SECTIONS    an axis's d channels follow each other from channel s; pairs (s+j, s+j+d/2), e = 2j/d
 *   NEIGHBOURS  the same, pairs (s+2j, s+2j+1), e = 2j/d
 *   HEAD        r = d_t+d_h+d_w; pairs (i, i+r/2), e = 2i/r, the first d_t/2 pairs turn with time, the
 *               next d_h/2 with the row, the rest with the column
 * Positions: `pos`, device int32 [B, N*L, 3] (time, row, column), any values; or pos = NULL, the
 * token's place in the sequence: time t0 + frame, row and column counted from patch0 for patches and
 * 0 for special tokens.  a is reduced to one turn in 64-bit integers, so that far positions lose
 * nothing.
 */
enum { AGG_ROPE_SECTIONS = 0, AGG_ROPE_NEIGHBOURS = 1, AGG_ROPE_HEAD = 2 };
typedef struct agg_rope {
  int32_t pairing;       /* AGG_ROPE_* */
  int32_t d_t, d_h, d_w;
  int32_t t0;            /* time of frame 0; t0 + N may not pass 2^31 - 1 */
  int32_t patch0;        /* row and column of a frame's first patch       */
  float base;            /* >= 1, finite                                  */
} agg_rope;

/*
 * Qr = turn(norm(Q)), Kr = turn(norm(K)), head by head: what belongs between the Q/K projections and
 * any of the attention calls.  q_norm, k_norm over a head's D channels (NULL: none); rope NULL: no
 * rotation.  Q, K: device bf16, token t of batch element b at element (b*N*L + t) * stride, stride 0
 * meaning H*D (contiguous), otherwise a multiple of 8 and >= H*D: a fused projection's output is read
 * where it is.  Qr, Kr: [B, N*L, H, D], contiguous.  Qr = Q and Kr = K (contiguous) work in place;
 * other overlaps of an output with an input, its norms' parameters, `pos` or the other output are refused with
 * AGG_ERR_SHAPE.  Q and Qr may both be NULL, or K and Kr.  Of `shape` only B, N, n_h, n_w, n_special, H and D matter.
 */
int agg_rope_fwd(const agg_shape* shape, const agg_rope* rope, const agg_norm* q_norm,
                 const agg_norm* k_norm, const int32_t* pos, const void* Q, int64_t q_stride,
                 const void* K, int64_t k_stride, void* Qr, void* Kr, void* hip_stream);

/*
 * The seam between a branch (attention, token-wise network) and the next one:
 *     h = x + gate * scale * post(branch),     n = pre(h)
 * post: the norm behind the branch, pre: the norm in front of the next branch (of the unrounded h).
 * x, branch, h, n: device bf16 [rows, C].  scale: device float32 [C], 16-byte aligned (NULL: ones).  gate: device bf16
 * [ceil(rows / gate_rows), C], row r uses gate[r / gate_rows] (NULL: ones; gate_rows is then
 * ignored).  branch NULL: h = x.  h may be NULL (not written); n must be given exactly if pre.kind
 * is not NONE.  h = x, h = branch, n = x and n = branch work in place; other overlaps of outputs with x, branch, gate, scale,
 * the norms' parameters or each other are refused with AGG_ERR_SHAPE.  C: a multiple of 8, at most 8192 (AGG_ERR_UNSUPPORTED).  rows = 0: nothing is done.
 */
typedef struct agg_residual {
  agg_norm post, pre;
  const float* scale;
  const void* gate;
  int64_t gate_rows;
} agg_residual;
int agg_residual_norm_fwd(int64_t rows, int32_t C, const agg_residual* residual, const void* x,
                          const void* branch, void* h, void* n, void* hip_stream);

/*
 * ---- Microscaled 4-bit floats ----
 * A matrix [rows, K] in 4 bits: 32 consecutive channels of a row share a scale 2^(s - 127), s one
 * byte; each channel holds a 4-bit float, sign + one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 (codes 0..7, sign
 * in bit 3).  s = 255 makes the 32 values NaN.
 *   codes   [rows, agg_mx4_code_stride(K)] bytes, channel k in byte k/2, low half if k is even
 *   scales  [rows, agg_mx4_scale_stride(K)] bytes, channel k's in byte k/32
 * The strides are K/2 rounded up to 128 and K/32 rounded up to 16, so that rows begin on whole lines;
 * the bytes behind a row's end (and the codes behind K in the last byte run) must be 0, as
 * agg_mx4_quantize leaves them.  Codes and scales are 16-byte aligned.
 *
 * Quantisation: s - 127 = floor(log2(largest magnitude)) - 2, at least -127 (all zeros: s = 0); values
 * are divided by the scale and rounded to the nearest 4-bit float, ties to the even code, magnitudes
 * above 6 to 6.  A block with a NaN or infinity gets s = 255 and codes 0.
 */
int64_t agg_mx4_code_stride(int32_t K);  /* host only; 0 for K < 1 */
int64_t agg_mx4_scale_stride(int32_t K);

/* x: device bf16, row r at element r * x_stride (0: K); K and x_stride multiples of 8.  rows = 0: nothing is done. */
int agg_mx4_quantize(int64_t rows, int32_t K, const void* x, int64_t x_stride, void* codes,
                     void* scales, void* hip_stream);

/* The values that codes and scales stand for, as bf16 [rows, K] (exact; above the type's range
 * infinite).  K a multiple of 8. */
int agg_mx4_dequantize(int64_t rows, int32_t K, const void* codes, const void* scales, void* x,
                       void* hip_stream);

/*
 * Y_i = A W_i^T + bias_i for i < count (1..3, one launch), or with a residual (count = 1)
 *     Y = R + res_scale * (A W^T + bias)
 * A: [rows, K] and W_i: [N, K] in 4 bits; products and sums in float32, one rounding.  bias_i: float32
 * [N], 16-byte aligned, or NULL.  Y_i, R: bf16 [rows, N], contiguous; Y = R works in place, other
 * overlaps of an output with R, A, a W_i, a bias, res_scale or another output are refused with AGG_ERR_SHAPE.  res_scale:
 * like bias_i (NULL: ones; must be NULL without R).
 * K and N are multiples of 8, K at most 2^22 and N at most 2^21.  rows = 0: nothing is done.  The order of a row's sums
 * depends on the call's sizes and the row's place in it, not on the other rows.
 */
typedef struct agg_mx4_matrix {
  const void* codes;
  const void* scales;
} agg_mx4_matrix;
typedef struct agg_mx4_linear {
  int32_t count;
  agg_mx4_matrix w[3];
  const float* bias[3];
  void* y[3];
  const void* residual;
  const float* res_scale;
} agg_mx4_linear;
int agg_mx4_linear_fwd(int64_t rows, int32_t N, int32_t K, const agg_mx4_linear* linear,
                       const void* codes, const void* scales, void* hip_stream);

/*
 * agg_global_block_fwd with the parts above:
 *     [Q|K|V] = W_{q,k,v} first(x) + b_{q,k,v},  Q = turn(q_norm(Q)),  K = turn(k_norm(K)),
 *     y = x + gate * scale * post(W_o Attn(Q, K, V) + b_o),   n = pre(y)
 * weights: as in agg_global_block_fwd, its LayerNorm being `first` (skipped if first_done: x_norm
 * then holds first(x), the n of the block before).  With mx (all four matrices) the projections are
 * products of 4-bit floats: their inputs are quantised, and w_q .. w_o are not read (may be NULL).
 * Everything that is zero or NULL in the options is left out; with all of it left out the result
 * is that of agg_global_block_fwd.  With a norm, a gate or (bf16 weights) a scale behind the output
 * projection, its result is rounded to bf16 before them, as every tensor between the parts is.
 * n: bf16 [B, N*L, C], exactly if residual.pre.kind is not NONE.  y, n, x and x_norm may not overlap, save n = x_norm.
 */
typedef struct agg_block_options {
  const agg_rope* rope;
  const int32_t* pos;
  agg_norm q_norm, k_norm;
  agg_residual residual;
  int32_t first_done;
  const void* x_norm;
  const agg_mx4_matrix* mx; /* host array of 4: q, k, v, o; NULL: the bf16 weights */
} agg_block_options;

/* Host only.  Scratch bytes agg_global_block_ex_fwd needs (0 on an invalid shape). */
size_t agg_block_ex_workspace_bytes(const agg_shape* shape, int mode, const agg_block_options* options);

int agg_global_block_ex_fwd(const agg_shape* shape, int mode, const agg_block_weights* weights,
                            const agg_block_options* options, const void* x, void* y, void* n,
                            void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * ---- Keys and values of another set, and a paged cache of them ----
 * Attention of queries to keys and values of another length: of a few tokens (a pose token, tracked points) to a frame's, of
 * a frame to the frames before it.  For every query i < q_lens[b] of batch element b and every head h
 *     O[b, i, h] = softmax over j < k_lens[b] of scale*<Q[b, i, h], K[b, j, h']>,  times V[b, j, h'],   h' = h / (H / H_kv).
 * A batch element without keys has O = 0 and lse = -infinity.  Keys and values at k_lens[b] and behind it are not
 * looked at, whatever they hold; rows of O and lse at q_lens[b] and behind it are left as they were.
 */
typedef struct agg_cross {
  int32_t B;             /* batch elements                                                           */
  int32_t NQ, NK;        /* most queries and most keys of one; 0: none                               */
  int32_t H, H_kv, D;    /* heads of Q and O; of K and V, which divides H; 64                        */
  float scale;           /* softmax scale                                                            */
  const int32_t* q_lens; /* device int32 [B], clamped to 0 .. NQ; NULL: NQ                           */
  const int32_t* k_lens; /* device int32 [B], clamped to 0 .. NK; NULL: NK                           */
} agg_cross;

/* Host only.  Scratch bytes that the two attention calls below need for this struct (0: none, the pointer may be NULL; 0 too on
 * invalid sizes).  Calls that may overlap in time need a workspace each, as do graphs that are replayed side by side. */
size_t agg_cross_workspace_bytes(const agg_cross* cross);

/*
 * Keys and values where they are: token t of batch element b at element (b*NK + t) * stride of K and of V (queries: (b*NQ + t) *
 * stride of Q), stride 0 meaning contiguous, otherwise a multiple of 8 and at least heads * 64.  Q, K, V: device bf16.
 * O: device bf16 [B, NQ, H, 64], contiguous; lse: device float32 [B, H, NQ] or NULL.  O and lse may overlap nothing else of
 * the call (AGG_ERR_SHAPE).  Logits and sums are float32; a key's probability is rounded to bf16 on its way into the second product, and
 * where a key head serves more than 32 queries the sum may be that of the rounded ones.  Logits may lie anywhere; a row whose logits
 * are all -infinity has O = NaN and lse = -infinity.  Sums of probability times value are float32 too: values beyond 2^100 may overflow them.
 * AGG_ERR_OVERFLOW, beside sizes beyond the index range: calls of more than 2^32 workgroups, and batch elements of more than 2^22
 * workgroups of 128 or 256 rows (tens of GiB of queries each).
 */
int agg_cross_attn_fwd(const agg_cross* cross, const void* Q, int64_t q_stride, const void* K, int64_t k_stride,
                       const void* V, int64_t v_stride, void* O, float* lse, void* workspace,
                       size_t workspace_bytes, void* hip_stream);

/*
 * A cache of keys and values in pages of 64 rows, for frames that arrive one after another.  A pool holds n_pages * H * 4096 bf16
 * (agg_cache_bytes): page p of head h is one 64-row tile in fragment order (above) at element (p*H + h) * 4096.  Row r of sequence
 * b lies in page pages[b, r / 64], row r % 64 of the tile.  The caller hands pages out; sequences may share pages they only
 * read, for instance the frames of a clip, each a sequence of its own length over one row of the table (attention that is
 * causal by frames).  A page number outside the pool is never written, and read as page 0 or the last one.
 */
typedef struct agg_cache {
  int32_t n_pages;        /* pages of a pool                            */
  int32_t H, D;           /* heads of keys and values; 64               */
  int32_t B, max_pages;   /* sequences, and entries of each in `pages`  */
  void *Kc, *Vc;          /* the pools, device bf16, 16-byte aligned    */
  const int32_t* pages;   /* device int32 [B, max_pages]                */
} agg_cache;

/* Host only.  Bytes of ONE pool. */
int agg_cache_bytes(const agg_cache* cache, size_t* bytes);

/*
 * Appends N*L new tokens per sequence, of which the first counts[b] exist (NULL: all): token t of sequence b becomes row start[b] + t
 * of the cache (start NULL: row t).  Keys pass through k_norm and the rotation on the way, and queries, if given, through
 * q_norm and the rotation to Qr, exactly as in agg_rope_fwd, whose conventions (norms, positions by `pos` or by the token's place,
 * strides, Qr = Q in place) hold here; values go as they are.  shape: B, N, n_h, n_w, n_special as there, H the heads of Q, a multiple
 * of cache->H (without Q it does not matter).  Rows before 0 and from 64*max_pages on are not stored.  lens (device int32 [B], may be
 * NULL) receives start[b] + counts[b], clamped to 0 .. 64*max_pages: what k_lens of the next call is.  Everything else in the
 * pools, and Qr of tokens that do not exist, is left as it was.  Two tokens of one call may not share a row.  No output may overlap
 * another operand of the call (AGG_ERR_SHAPE); lens may not be start.  More than 2^32 pieces of 32 rows: AGG_ERR_OVERFLOW.
 */
int agg_cache_append(const agg_cache* cache, const agg_shape* shape, const agg_rope* rope, const agg_norm* q_norm,
                     const agg_norm* k_norm, const int32_t* pos, const void* Q, int64_t q_stride, const void* K,
                     int64_t k_stride, const void* V, int64_t v_stride, const int32_t* start, const int32_t* counts,
                     int32_t* lens, void* Qr, void* hip_stream);

/* agg_cross_attn_fwd over a cache: keys and values of batch element b are the first k_lens[b] rows of its sequence.  cross: B and
 * H_kv are the cache's B and H, NK at most 64*max_pages. */
int agg_cache_attn_fwd(const agg_cache* cache, const agg_cross* cross, const void* Q, int64_t q_stride, void* O,
                       float* lse, void* workspace, size_t workspace_bytes, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* AGG_H_ */
