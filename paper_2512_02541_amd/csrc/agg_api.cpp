// Host side of libagg: argument validation, geometry, counts, index list and
// the extern "C" entry points declared in agg.h.  Nothing here allocates device
// memory or synchronises; every check runs before the first launch.
#include <limits.h>
#include <math.h>
#include <string.h>

#include "agg_internal.h"

namespace agg {

static inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Fills Geom from the caller's shape.  `dense` ignores the subsampling fields
// and treats every token as kept (Sec. 4.2: plain global attention).
int make_geom(const agg_shape* s, Geom* g, bool dense) {
  if (!s || !g) return AGG_ERR_NULL;
  if (s->B < 1 || s->N < 1 || s->n_h < 1 || s->n_w < 1 || s->n_special < 0 || s->H < 1 ||
      s->D < 1)
    return AGG_ERR_SHAPE;
  if (!dense) {
    if (s->s_h < 1 || s->s_w < 1) return AGG_ERR_SHAPE;
    if (s->flags & ~(uint32_t)(AGG_DIAG | AGG_MEAN)) return AGG_ERR_SHAPE;
    if (s->keep_first_frame != 0 && s->keep_first_frame != 1) return AGG_ERR_SHAPE;
  }
  if (!(s->scale > 0.0f) || !(s->scale < 1e30f)) return AGG_ERR_SHAPE;
  if (!(s->mean_logit_bias > -1e30f && s->mean_logit_bias < 1e30f)) return AGG_ERR_SHAPE;
  if (s->D != kHeadDim) return AGG_ERR_UNSUPPORTED;

  int64_t T = (int64_t)s->n_h * s->n_w;
  int64_t L = T + s->n_special;
  if (L > INT32_MAX) return AGG_ERR_OVERFLOW;
  int64_t NQ = (int64_t)s->N * L;
  // token ids and compacted row numbers are int32; tile padding must also fit
  if (NQ > (int64_t)INT32_MAX - 2 * kTileRows) return AGG_ERR_OVERFLOW;
  // element offsets are 64-bit in the kernels, but keep one tensor under 2^62 bytes
  if ((int64_t)s->B * s->H > ((int64_t)1 << 40) / NQ) return AGG_ERR_OVERFLOW;

  g->B = s->B;
  g->N = s->N;
  g->L = (int32_t)L;
  g->P = s->n_special;
  g->n_h = s->n_h;
  g->n_w = s->n_w;
  g->H = s->H;
  g->s_h = dense ? 1 : s->s_h;
  g->s_w = dense ? 1 : s->s_w;
  g->keep_first = dense ? 0 : s->keep_first_frame;
  // a stride larger than the grid keeps one row/column of windows (edge windows count)
  g->kw = (int32_t)ceil_div(s->n_w, g->s_w);
  g->kf = (int32_t)(ceil_div(s->n_h, g->s_h) * g->kw);
  g->rows_sub = g->P + g->kf;
  g->dw = g->n_w - g->kw;
  g->df = (int32_t)(T - g->kf);
  g->NQ = NQ;
  int64_t f0 = g->keep_first ? 1 : 0;
  g->M = f0 * L + ((int64_t)s->N - f0) * g->rows_sub;
  g->M_pad = ceil_div(g->M, kTileRows) * kTileRows;
  g->n_dropped = ((int64_t)s->N - f0) * g->df;
  return AGG_OK;
}

static bool misaligned(const void* p) { return ((uintptr_t)p & 15u) != 0; }

}  // namespace agg

using namespace agg;

extern "C" {

const char* agg_status_string(int status) {
  switch (status) {
    case AGG_OK: return "ok";
    case AGG_ERR_NULL: return "a required pointer is NULL";
    case AGG_ERR_SHAPE: return "invalid shape, stride, scale or flag, or buffers overlap that may not";
    case AGG_ERR_UNSUPPORTED: return "head dimension is not 64, or rows are wider than the call takes";
    case AGG_ERR_ALIGN: return "tensor pointer is not 16-byte aligned";
    case AGG_ERR_WORKSPACE: return "workspace too small";
    case AGG_ERR_OVERFLOW: return "a size or a position exceeds the index range";
    case AGG_ERR_LAUNCH: return "kernel launch failed";
    default: return "unknown status";
  }
}

int agg_sigma_to_strides(int sigma, int32_t* s_h, int32_t* s_w) {
  if (!s_h || !s_w) return AGG_ERR_NULL;
  // Sec. 4.3: sigma = s_h * s_w with the factorisations the paper lists
  static const int table[][3] = {{1, 1, 1}, {2, 1, 2}, {4, 2, 2}, {6, 2, 3}, {9, 3, 3}};
  for (const auto& row : table)
    if (row[0] == sigma) {
      *s_h = row[1];
      *s_w = row[2];
      return AGG_OK;
    }
  return AGG_ERR_SHAPE;
}

int agg_kv_count(const agg_shape* shape, int64_t* M, int64_t* n_dropped) {
  Geom g;
  int rc = make_geom(shape, &g, false);
  if (rc != AGG_OK) return rc;
  if (M) *M = g.M;
  if (n_dropped) *n_dropped = g.n_dropped;
  return AGG_OK;
}

int agg_kv_indices_host(const agg_shape* shape, int32_t* idx) {
  Geom g;
  int rc = make_geom(shape, &g, false);
  if (rc != AGG_OK) return rc;
  if (!idx) return AGG_ERR_NULL;
  for (int64_t m = 0; m < g.M; ++m) idx[m] = (int32_t)kept_row_to_token(g, m);
  return AGG_OK;
}

int agg_dropped_indices_host(const agg_shape* shape, int32_t* idx) {
  Geom g;
  int rc = make_geom(shape, &g, false);
  if (rc != AGG_OK) return rc;
  if (!idx) return AGG_ERR_NULL;
  for (int64_t u = 0; u < g.n_dropped; ++u) idx[u] = (int32_t)dropped_to_token(g, u);
  return AGG_OK;
}

int agg_kv_compact_bytes(const agg_shape* shape, size_t* bytes, int64_t* M_pad) {
  Geom g;
  int rc = make_geom(shape, &g, false);
  if (rc != AGG_OK) return rc;
  if (bytes) *bytes = (size_t)g.B * g.H * g.M_pad * kHeadDim * 2;
  if (M_pad) *M_pad = g.M_pad;
  return AGG_OK;
}

int64_t agg_kc_offset(int64_t m, int32_t d) { return kc_offset(m, d); }
int64_t agg_vc_offset(int64_t m, int32_t d) { return vc_offset(m, d); }

size_t agg_workspace_bytes(const agg_shape* shape) {
  Geom g;
  if (make_geom(shape, &g, false) != AGG_OK) return 0;
  // [B][chunks][2 (K,V)][H*D] float partial sums; never zero so that a valid pointer is required
  size_t n = (size_t)g.B * (size_t)mean_chunks(g) * 2 * g.H * kHeadDim * sizeof(float);
  return n ? n : 256;
}

int agg_kv_subsample(const agg_shape* shape, const void* K, const void* V, void* Kc, void* Vc,
                     int32_t* idx, float* kmean, float* vmean, void* workspace,
                     size_t workspace_bytes, void* hip_stream) {
  Geom g;
  int rc = make_geom(shape, &g, false);
  if (rc != AGG_OK) return rc;
  if (!K || !V || !kmean || !vmean || !workspace) return AGG_ERR_NULL;
  if ((Kc == nullptr) != (Vc == nullptr)) return AGG_ERR_NULL;  // both or neither
  if (misaligned(K) || misaligned(V) || misaligned(Kc) || misaligned(Vc) || misaligned(workspace) ||
      misaligned(kmean) || misaligned(vmean) || ((uintptr_t)idx & 3u))
    return AGG_ERR_ALIGN;
  if (workspace_bytes < agg_workspace_bytes(shape)) return AGG_ERR_WORKSPACE;
  hipStream_t st = (hipStream_t)hip_stream;
  if (launch_subsample(g, K, V, Kc, Vc, idx, kmean, vmean, workspace, st) != hipSuccess)
    return AGG_ERR_LAUNCH;
  return AGG_OK;
}

size_t agg_static_scratch_bytes(void) { return kStaticScratchBytes; }

int agg_kv_subsample_static(const agg_shape* shape, const void* K, const void* V, void* Kc,
                            void* Vc, int32_t* idx, float* kmean, float* vmean, void* hip_stream) {
  Geom g;
  int rc = make_geom(shape, &g, false);
  if (rc != AGG_OK) return rc;
  if (!K || !V || !kmean || !vmean) return AGG_ERR_NULL;
  if ((Kc == nullptr) != (Vc == nullptr)) return AGG_ERR_NULL;  // both or neither
  if (misaligned(K) || misaligned(V) || misaligned(Kc) || misaligned(Vc) || misaligned(kmean) ||
      misaligned(vmean) || ((uintptr_t)idx & 3u))
    return AGG_ERR_ALIGN;
  if (agg_workspace_bytes(shape) > kStaticScratchBytes) return AGG_ERR_WORKSPACE;
  void* ws = nullptr;
  if (static_scratch(&ws) != hipSuccess) return AGG_ERR_LAUNCH;
  hipStream_t st = (hipStream_t)hip_stream;
  if (launch_subsample(g, K, V, Kc, Vc, idx, kmean, vmean, ws, st) != hipSuccess)
    return AGG_ERR_LAUNCH;
  return AGG_OK;
}

int agg_global_attn_fwd(const agg_shape* shape, const void* Q, const void* K, const void* V,
                        const void* Kc, const void* Vc, const float* kmean, const float* vmean,
                        void* O, float* lse, void* hip_stream) {
  Geom g;
  int rc = make_geom(shape, &g, false);
  if (rc != AGG_OK) return rc;
  if (!Q || !K || !V || !Kc || !Vc || !kmean || !vmean || !O) return AGG_ERR_NULL;
  if (misaligned(Q) || misaligned(K) || misaligned(V) || misaligned(Kc) || misaligned(Vc) ||
      misaligned(O) || misaligned(kmean) || misaligned(vmean) || ((uintptr_t)lse & 3u))
    return AGG_ERR_ALIGN;
  hipStream_t st = (hipStream_t)hip_stream;
  if (launch_attn(g, shape->flags, shape->scale, shape->mean_logit_bias, Q, K, V, Kc, Vc, kmean,
                  vmean, O, lse, st) != hipSuccess)
    return AGG_ERR_LAUNCH;
  return AGG_OK;
}

// Whether the in-place row modes of the attention kernel can address this geometry: indexed
// rows use 32-bit byte offsets from the (batch, head) base formed by a 24-bit multiplication.
static bool rows_addressable(const Geom& g) {
  return (uint64_t)g.NQ * g.H * (kHeadDim * 2) <= 0xFFFFFFFFull && g.NQ <= 0xFFFFFF &&
         (uint64_t)g.H * (kHeadDim * 2) <= 0xFFFFFF;
}

int agg_global_attn_fwd_idx(const agg_shape* shape, const void* Q, const void* K, const void* V,
                            const int32_t* idx, const float* kmean, const float* vmean, void* O,
                            float* lse, void* hip_stream) {
  Geom g;
  int rc = make_geom(shape, &g, false);
  if (rc != AGG_OK) return rc;
  if (!Q || !K || !V || !idx || !kmean || !vmean || !O) return AGG_ERR_NULL;
  if (misaligned(Q) || misaligned(K) || misaligned(V) || misaligned(O) || misaligned(kmean) ||
      misaligned(vmean) || ((uintptr_t)idx & 3u) || ((uintptr_t)lse & 3u))
    return AGG_ERR_ALIGN;
  if (!rows_addressable(g)) return AGG_ERR_OVERFLOW;
  if (launch_attn(g, shape->flags, shape->scale, shape->mean_logit_bias, Q, K, V, nullptr, nullptr,
                  kmean, vmean, O, lse, (hipStream_t)hip_stream, nullptr, nullptr, kAttnSrcIndexed,
                  idx, 0) != hipSuccess)
    return AGG_ERR_LAUNCH;
  return AGG_OK;
}

int agg_dense_global_attn_fwd(const agg_shape* shape, const void* Q, const void* K, const void* V,
                              void* O, float* lse, void* hip_stream) {
  Geom g;
  int rc = make_geom(shape, &g, true);
  if (rc != AGG_OK) return rc;
  if (!Q || !K || !V || !O) return AGG_ERR_NULL;
  if (misaligned(Q) || misaligned(K) || misaligned(V) || misaligned(O) || ((uintptr_t)lse & 3u))
    return AGG_ERR_ALIGN;
  // every token is a key: the kernel reads the rows of K and V where they are, no extras
  if (launch_attn(g, 0u, shape->scale, 0.0f, Q, K, V, nullptr, nullptr, nullptr, nullptr, O, lse,
                  (hipStream_t)hip_stream, nullptr, nullptr, kAttnSrcRows) != hipSuccess)
    return AGG_ERR_LAUNCH;
  return AGG_OK;
}

// Frame attention is ordinary attention over B*N independent sequences of one frame each:
// the token-major tensors already hold a frame's L tokens contiguously.
static int frame_shape(const agg_shape* shape, agg_shape* per_frame) {
  if (!shape) return AGG_ERR_NULL;
  if (shape->B < 1 || shape->N < 1) return AGG_ERR_SHAPE;
  if ((int64_t)shape->B * shape->N > INT32_MAX) return AGG_ERR_OVERFLOW;
  *per_frame = *shape;
  per_frame->B = shape->B * shape->N;
  per_frame->N = 1;
  return AGG_OK;
}

int agg_frame_attn_fwd(const agg_shape* shape, const void* Q, const void* K, const void* V, void* O,
                       float* lse, void* hip_stream) {
  agg_shape f;
  int rc = frame_shape(shape, &f);
  if (rc != AGG_OK) return rc;
  return agg_dense_global_attn_fwd(&f, Q, K, V, O, lse, hip_stream);
}

// ---- caller-supplied kept lists ---------------------------------------------------------
// Geometry of the list variants: the grid fields stay (the select kernel needs them), the
// compacted length becomes the list's.
static int list_geom(const agg_shape* shape, int64_t M_list, Geom* g) {
  int rc = make_geom(shape, g, false);
  if (rc != AGG_OK) return rc;
  if (M_list < 1) return AGG_ERR_SHAPE;
  if (M_list > (int64_t)INT32_MAX - 2 * kTileRows) return AGG_ERR_OVERFLOW;
  g->M = M_list;
  g->M_pad = ceil_div(M_list, kTileRows) * kTileRows;
  if ((int64_t)g->B * g->H > ((int64_t)1 << 40) / g->M_pad) return AGG_ERR_OVERFLOW;
  return AGG_OK;
}

int agg_select_kv_indices(const agg_shape* shape, int rule, uint64_t seed, const void* K,
                          int32_t* list, void* hip_stream) {
  Geom g;
  int rc = make_geom(shape, &g, false);
  if (rc != AGG_OK) return rc;
  if (rule < AGG_SELECT_FIRST || rule > AGG_SELECT_LOW) return AGG_ERR_SHAPE;
  const bool needs_k = (rule == AGG_SELECT_HIGH || rule == AGG_SELECT_LOW);
  if (!list || (needs_k && !K)) return AGG_ERR_NULL;
  if ((needs_k && misaligned(K)) || ((uintptr_t)list & 3u)) return AGG_ERR_ALIGN;
  if (launch_select(g, rule, seed, K, list, (hipStream_t)hip_stream) != hipSuccess)
    return AGG_ERR_LAUNCH;
  return AGG_OK;
}

int agg_kv_pool(const agg_shape* shape, const void* K, const void* V, void* Kc, void* Vc,
                void* hip_stream) {
  Geom g;
  int rc = make_geom(shape, &g, false);
  if (rc != AGG_OK) return rc;
  if (!K || !V || !Kc || !Vc) return AGG_ERR_NULL;
  if (misaligned(K) || misaligned(V) || misaligned(Kc) || misaligned(Vc)) return AGG_ERR_ALIGN;
  if (launch_pool(g, K, V, Kc, Vc, (hipStream_t)hip_stream) != hipSuccess) return AGG_ERR_LAUNCH;
  return AGG_OK;
}

int agg_list_compact_bytes(const agg_shape* shape, int64_t M_list, size_t* bytes, int64_t* M_pad) {
  Geom g;
  int rc = list_geom(shape, M_list, &g);
  if (rc != AGG_OK) return rc;
  if (bytes) *bytes = (size_t)g.B * g.H * g.M_pad * kHeadDim * 2;
  if (M_pad) *M_pad = g.M_pad;
  return AGG_OK;
}

size_t agg_list_workspace_bytes(const agg_shape* shape) {
  Geom g;
  if (make_geom(shape, &g, false) != AGG_OK) return 0;
  return list_workspace_bytes(g);
}

int agg_kv_subsample_list(const agg_shape* shape, const int32_t* list, int64_t M_list,
                          const void* K, const void* V, void* Kc, void* Vc, float* kmean,
                          float* vmean, uint32_t* kept_bits, int32_t* n_dropped, void* workspace,
                          size_t workspace_bytes, void* hip_stream) {
  Geom g;
  int rc = list_geom(shape, M_list, &g);
  if (rc != AGG_OK) return rc;
  if (!list || !K || !V || !Kc || !Vc || !kmean || !vmean || !kept_bits || !n_dropped || !workspace)
    return AGG_ERR_NULL;
  if (misaligned(K) || misaligned(V) || misaligned(Kc) || misaligned(Vc) || misaligned(workspace) ||
      misaligned(kmean) || misaligned(vmean) || ((uintptr_t)list & 3u) ||
      ((uintptr_t)kept_bits & 3u) || ((uintptr_t)n_dropped & 3u))
    return AGG_ERR_ALIGN;
  if (workspace_bytes < list_workspace_bytes(g)) return AGG_ERR_WORKSPACE;
  if (launch_subsample_list(g, list, K, V, Kc, Vc, kmean, vmean, kept_bits, n_dropped, workspace,
                            (hipStream_t)hip_stream) != hipSuccess)
    return AGG_ERR_LAUNCH;
  return AGG_OK;
}

int agg_global_attn_fwd_list(const agg_shape* shape, int64_t M_list, const void* Q, const void* K,
                             const void* V, const void* Kc, const void* Vc, const float* kmean,
                             const float* vmean, const uint32_t* kept_bits,
                             const int32_t* n_dropped, void* O, float* lse, void* hip_stream) {
  Geom g;
  int rc = list_geom(shape, M_list, &g);
  if (rc != AGG_OK) return rc;
  if (!Q || !K || !V || !Kc || !Vc || !kmean || !vmean || !kept_bits || !n_dropped || !O)
    return AGG_ERR_NULL;
  if (misaligned(Q) || misaligned(K) || misaligned(V) || misaligned(Kc) || misaligned(Vc) ||
      misaligned(O) || misaligned(kmean) || misaligned(vmean) || ((uintptr_t)lse & 3u) ||
      ((uintptr_t)kept_bits & 3u) || ((uintptr_t)n_dropped & 3u))
    return AGG_ERR_ALIGN;
  if (launch_attn(g, shape->flags, shape->scale, shape->mean_logit_bias, Q, K, V, Kc, Vc, kmean,
                  vmean, O, lse, (hipStream_t)hip_stream, kept_bits, n_dropped) != hipSuccess)
    return AGG_ERR_LAUNCH;
  return AGG_OK;
}

// ---- rotary positions, the seam between branches, 4-bit floats -------------------------------
namespace {

// whether [a, a + na) and [b, b + nb) share a byte (a null pointer shares none)
bool overlap(const void* a, uint64_t na, const void* b, uint64_t nb) {
  if (!a || !b || !na || !nb) return false;
  const uint64_t x = (uint64_t)(uintptr_t)a, y = (uint64_t)(uintptr_t)b;
  return x < y ? y - x < na : x - y < nb;
}

// whether an output shares a byte with the parameters of a norm over C channels
bool overlap_norm(const void* out, uint64_t bytes, const SeamNorm& n, int64_t C) {
  return overlap(out, bytes, n.gamma, (uint64_t)C * 4) || overlap(out, bytes, n.beta, (uint64_t)C * 4);
}

int make_norm(const agg_norm* n, SeamNorm* out) {
  *out = SeamNorm{AGG_NORM_NONE, 1.f, nullptr, nullptr};
  if (!n || n->kind == AGG_NORM_NONE) return AGG_OK;
  if (n->kind != AGG_NORM_LAYER && n->kind != AGG_NORM_RMS) return AGG_ERR_SHAPE;
  if (!(n->eps > 0.0f) || !(n->eps < 1e30f)) return AGG_ERR_SHAPE;
  if (misaligned(n->gamma) || misaligned(n->beta)) return AGG_ERR_ALIGN;
  *out = SeamNorm{n->kind, n->eps, n->gamma, n->beta};
  return AGG_OK;
}

// The pairs of channels that turn, their axes and frequencies (agg.h).
int make_rope(const agg_rope* r, RopeArgs* a) {
  a->pairs = 0;
  for (int c = 0; c < kHeadDim; ++c) a->other[c] = (uint8_t)c;
  if (!r) return AGG_OK;
  if (r->pairing != AGG_ROPE_SECTIONS && r->pairing != AGG_ROPE_NEIGHBOURS && r->pairing != AGG_ROPE_HEAD)
    return AGG_ERR_SHAPE;
  const int32_t d[3] = {r->d_t, r->d_h, r->d_w};
  int turned = 0;
  for (int axis = 0; axis < 3; ++axis) {
    if (d[axis] < 0 || d[axis] > kHeadDim || d[axis] % 2 != 0) return AGG_ERR_SHAPE;
    turned += d[axis];
  }
  if (turned > kHeadDim) return AGG_ERR_SHAPE;
  if (!(r->base >= 1.0f) || !(r->base < INFINITY)) return AGG_ERR_SHAPE;
  a->t0 = r->t0;
  a->patch0 = r->patch0;
  // frequencies in 2^-64 turns per position, each the one before times a constant.  With 64 bits of mantissa all exponents
  // up to 128 are good to 2^-57, and so is a frequency after 32 steps: 2^-28 turns at the farthest position.  (A power for
  // each took the call 10 us, powl for each axis 0.7; this takes 0.3.)
  const long double octaves = -2.0L * log2l((long double)r->base);
  const long double whole = 18446744073709551616.0L / (2 * 3.14159265358979323846264338327950288L);
  long double freq = whole, ratio = 1;
  if (r->pairing == AGG_ROPE_HEAD && turned) ratio = exp2l(octaves / turned);
  int start = 0, p = 0;
  for (int axis = 0; axis < 3; ++axis) {
    if (r->pairing != AGG_ROPE_HEAD && d[axis]) {
      freq = whole;
      ratio = exp2l(octaves / d[axis]);
    }
    for (int j = 0; j < d[axis] / 2; ++j, ++p) {
      const int lo = r->pairing == AGG_ROPE_HEAD ? p : start + (r->pairing == AGG_ROPE_SECTIONS ? j : 2 * j);
      const int hi = lo + (r->pairing == AGG_ROPE_HEAD ? turned / 2 : r->pairing == AGG_ROPE_SECTIONS ? d[axis] / 2 : 1);
      a->freq[p] = (uint64_t)freq;
      freq *= ratio;
      a->axis[p] = (uint8_t)axis;
      a->first[p] = (uint8_t)lo;
      a->second[p] = (uint8_t)hi;
      a->other[lo] = (uint8_t)(hi | 0x80);
      a->other[hi] = (uint8_t)(lo | 0x80);
    }
    start += d[axis];
  }
  a->pairs = p;
  return AGG_OK;
}

// Everything agg_rope_fwd checks; AGG_OK with *a filled in.
int make_rope_args(const agg_shape* shape, const agg_rope* rope, const agg_norm* q_norm,
                   const agg_norm* k_norm, const int32_t* pos, const void* Q, int64_t q_stride,
                   const void* K, int64_t k_stride, void* Qr, void* Kr, RopeArgs* a) {
  Geom g;
  int rc = make_geom(shape, &g, true);
  if (rc != AGG_OK) return rc;
  memset(a, 0, sizeof *a);
  if ((rc = make_rope(rope, a)) != AGG_OK) return rc;
  if ((rc = make_norm(q_norm, &a->norm[0])) != AGG_OK) return rc;
  if ((rc = make_norm(k_norm, &a->norm[1])) != AGG_OK) return rc;
  if ((Q == nullptr) != (Qr == nullptr) || (K == nullptr) != (Kr == nullptr) || (!Q && !K)) return AGG_ERR_NULL;
  if (misaligned(Q) || misaligned(K) || misaligned(Qr) || misaligned(Kr) || ((uintptr_t)pos & 3u))
    return AGG_ERR_ALIGN;
  const int64_t C = (int64_t)g.H * kHeadDim;
  if (!pos && rope) {
    const int64_t side = g.n_h > g.n_w ? g.n_h : g.n_w;
    if ((int64_t)rope->t0 + g.N > INT32_MAX || (int64_t)rope->patch0 + side > INT32_MAX) return AGG_ERR_OVERFLOW;
  }
  a->total = (int64_t)g.B * g.NQ;
  const void* in[2] = {Q, K};
  void* out[2] = {Qr, Kr};
  const int64_t stride[2] = {q_stride, k_stride};
  const uint64_t out_bytes = (uint64_t)a->total * C * 2;
  uint64_t in_bytes[2] = {0, 0};
  for (int t = 0; t < 2; ++t) {
    if (!in[t]) continue;
    const int64_t s = stride[t] ? stride[t] : C;
    if (s < C || s % 8 != 0) return AGG_ERR_SHAPE;
    if (s > ((int64_t)1 << 60) / a->total) return AGG_ERR_OVERFLOW;
    a->in[t] = (const uint16_t*)in[t];
    a->out[t] = (uint16_t*)out[t];
    a->stride[t] = s;
    in_bytes[t] = ((uint64_t)(a->total - 1) * s + C) * 2;
  }
  for (int t = 0; t < 2; ++t) {
    if (!out[t]) continue;
    const bool in_place = in[t] == out[t] && a->stride[t] == C;
    if (!in_place && overlap(in[t], in_bytes[t], out[t], out_bytes)) return AGG_ERR_SHAPE;
    if (overlap(in[1 - t], in_bytes[1 - t], out[t], out_bytes)) return AGG_ERR_SHAPE;
    if (pos && overlap(pos, (uint64_t)a->total * 12, out[t], out_bytes)) return AGG_ERR_SHAPE;
    for (const SeamNorm& n : a->norm)
      if (overlap_norm(out[t], out_bytes, n, kHeadDim)) return AGG_ERR_SHAPE;
  }
  if (overlap(Qr, out_bytes, Kr, out_bytes)) return AGG_ERR_SHAPE;
  a->pos = pos;
  a->NQ = g.NQ;
  a->H = g.H;
  a->L = g.L;
  a->P = g.P;
  a->n_w = g.n_w;
  return AGG_OK;
}

// Everything agg_residual_norm_fwd checks.
int make_seam_args(int64_t rows, int32_t C, const agg_residual* r, const void* x, const void* branch,
                   void* h, void* n, SeamArgs* a) {
  if (!r) return AGG_ERR_NULL;
  if (rows < 0 || C < 1 || C % 8 != 0) return AGG_ERR_SHAPE;
  if (C > 8192) return AGG_ERR_UNSUPPORTED;
  if (rows > ((int64_t)1 << 31)) return AGG_ERR_OVERFLOW;
  int rc;
  memset(a, 0, sizeof *a);
  if ((rc = make_norm(&r->post, &a->post)) != AGG_OK) return rc;
  if ((rc = make_norm(&r->pre, &a->pre)) != AGG_OK) return rc;
  if (r->gate && r->gate_rows < 1) return AGG_ERR_SHAPE;
  if ((n != nullptr) != (a->pre.kind != AGG_NORM_NONE)) return AGG_ERR_NULL;
  if (rows > 0 && (!x || (!h && !n))) return AGG_ERR_NULL;
  if (!branch && (r->gate || r->scale || a->post.kind != AGG_NORM_NONE)) return AGG_ERR_NULL;
  if (misaligned(x) || misaligned(branch) || misaligned(h) || misaligned(n) || misaligned(r->scale) ||
      misaligned(r->gate))
    return AGG_ERR_ALIGN;
  const uint64_t bytes = (uint64_t)rows * C * 2;
  const int64_t groups = r->gate && rows > 0 ? (rows - 1) / r->gate_rows + 1 : 0;
  void* out[2] = {h, n};
  for (void* o : out) {
    if (o != x && overlap(o, bytes, x, bytes)) return AGG_ERR_SHAPE;
    if (o != branch && overlap(o, bytes, branch, bytes)) return AGG_ERR_SHAPE;
    if (overlap(o, bytes, r->gate, (uint64_t)groups * C * 2) || overlap(o, bytes, r->scale, (uint64_t)C * 4) ||
        overlap_norm(o, bytes, a->post, C) || overlap_norm(o, bytes, a->pre, C))
      return AGG_ERR_SHAPE;
  }
  if (overlap(h, bytes, n, bytes)) return AGG_ERR_SHAPE;
  a->x = (const uint16_t*)x;
  a->branch = (const uint16_t*)branch;
  a->gate = (const uint16_t*)r->gate;
  a->scale = r->scale;
  a->h = (uint16_t*)h;
  a->n = (uint16_t*)n;
  a->rows = rows;
  a->gate_rows = r->gate_rows;
  a->C = C;
  return AGG_OK;
}

// rows and channels of a matrix in 4 bits
int check_mx4(int64_t rows, int32_t K) {
  if (rows < 0 || K < 1 || K % 8 != 0) return AGG_ERR_SHAPE;
  // a row's codes are addressed with 32 bits; one tensor stays under 2^60 bytes
  if (K > INT32_MAX - 512 || rows > ((int64_t)1 << 31)) return AGG_ERR_OVERFLOW;
  return AGG_OK;
}

int make_mx4_args(int64_t rows, int32_t N, int32_t K, const agg_mx4_linear* l, const void* codes,
                  const void* scales, Mx4LinearArgs* a) {
  if (!l) return AGG_ERR_NULL;
  int rc = check_mx4(rows, K);
  if (rc != AGG_OK) return rc;
  if (N < 1 || N % 8 != 0 || l->count < 1 || l->count > 3) return AGG_ERR_SHAPE;
  // a tile's rows of codes are addressed with 32 bits, tiles counted with 31
  if (K > (1 << 22) || N > (1 << 21)) return AGG_ERR_OVERFLOW;
  if (rows / 64 + 1 > (int64_t)INT32_MAX / ((N / 64 + 1) * (int64_t)l->count)) return AGG_ERR_OVERFLOW;
  if ((l->residual && l->count != 1) || (l->res_scale && !l->residual)) return AGG_ERR_SHAPE;
  if (rows > 0 && (!codes || !scales)) return AGG_ERR_NULL;
  if (misaligned(codes) || misaligned(scales) || misaligned(l->residual) || misaligned(l->res_scale))
    return AGG_ERR_ALIGN;
  memset(a, 0, sizeof *a);
  const uint64_t y_bytes = (uint64_t)rows * N * 2;
  const uint64_t a_codes = (uint64_t)rows * mx4_code_stride(K), a_scales = (uint64_t)rows * mx4_scale_stride(K);
  for (int i = 0; i < l->count; ++i) {
    if (!l->w[i].codes || !l->w[i].scales || (rows > 0 && !l->y[i])) return AGG_ERR_NULL;
    if (misaligned(l->w[i].codes) || misaligned(l->w[i].scales) || misaligned(l->bias[i]) || misaligned(l->y[i]))
      return AGG_ERR_ALIGN;
    if (overlap(l->y[i], y_bytes, codes, a_codes) || overlap(l->y[i], y_bytes, scales, a_scales))
      return AGG_ERR_SHAPE;
    for (int j = 0; j < i; ++j)
      if (overlap(l->y[i], y_bytes, l->y[j], y_bytes)) return AGG_ERR_SHAPE;
    for (int j = 0; j < l->count; ++j)
      if (overlap(l->y[i], y_bytes, l->w[j].codes, (uint64_t)N * mx4_code_stride(K)) ||
          overlap(l->y[i], y_bytes, l->w[j].scales, (uint64_t)N * mx4_scale_stride(K)) ||
          overlap(l->y[i], y_bytes, l->bias[j], (uint64_t)N * 4))
        return AGG_ERR_SHAPE;
    a->w[i] = Mx4Matrix{(const uint8_t*)l->w[i].codes, (const uint8_t*)l->w[i].scales};
    a->bias[i] = l->bias[i];
    a->y[i] = (uint16_t*)l->y[i];
  }
  if (l->residual != l->y[0] && overlap(l->residual, y_bytes, l->y[0], y_bytes)) return AGG_ERR_SHAPE;
  if (overlap(l->y[0], y_bytes, l->res_scale, (uint64_t)N * 4)) return AGG_ERR_SHAPE;
  a->a = Mx4Matrix{(const uint8_t*)codes, (const uint8_t*)scales};
  a->residual = (const uint16_t*)l->residual;
  a->res_scale = l->res_scale;
  a->rows = rows;
  a->N = N;
  a->K = K;
  a->count = l->count;
  a->code_stride = (int32_t)mx4_code_stride(K);
  a->scale_stride = (int32_t)mx4_scale_stride(K);
  return AGG_OK;
}

}  // namespace

int agg_rope_fwd(const agg_shape* shape, const agg_rope* rope, const agg_norm* q_norm,
                 const agg_norm* k_norm, const int32_t* pos, const void* Q, int64_t q_stride,
                 const void* K, int64_t k_stride, void* Qr, void* Kr, void* hip_stream) {
  RopeArgs a;
  const int rc = make_rope_args(shape, rope, q_norm, k_norm, pos, Q, q_stride, K, k_stride, Qr, Kr, &a);
  if (rc != AGG_OK) return rc;
  return launch_rope(a, (hipStream_t)hip_stream) == hipSuccess ? AGG_OK : AGG_ERR_LAUNCH;
}

int agg_residual_norm_fwd(int64_t rows, int32_t C, const agg_residual* residual, const void* x,
                          const void* branch, void* h, void* n, void* hip_stream) {
  SeamArgs a;
  const int rc = make_seam_args(rows, C, residual, x, branch, h, n, &a);
  if (rc != AGG_OK || rows == 0) return rc;
  return launch_seam(a, (hipStream_t)hip_stream) == hipSuccess ? AGG_OK : AGG_ERR_LAUNCH;
}

int64_t agg_mx4_code_stride(int32_t K) { return K < 1 ? 0 : mx4_code_stride(K); }
int64_t agg_mx4_scale_stride(int32_t K) { return K < 1 ? 0 : mx4_scale_stride(K); }

int agg_mx4_quantize(int64_t rows, int32_t K, const void* x, int64_t x_stride, void* codes,
                     void* scales, void* hip_stream) {
  const int rc = check_mx4(rows, K);
  if (rc != AGG_OK) return rc;
  const int64_t stride = x_stride ? x_stride : K;
  if (stride < K || stride % 8 != 0) return AGG_ERR_SHAPE;
  if (rows == 0) return AGG_OK;
  if (stride > ((int64_t)1 << 60) / rows) return AGG_ERR_OVERFLOW;
  if (!x || !codes || !scales) return AGG_ERR_NULL;
  if (misaligned(x) || misaligned(codes) || misaligned(scales)) return AGG_ERR_ALIGN;
  const uint64_t x_bytes = ((uint64_t)(rows - 1) * stride + K) * 2, c_bytes = (uint64_t)rows * mx4_code_stride(K),
                 s_bytes = (uint64_t)rows * mx4_scale_stride(K);
  if (overlap(x, x_bytes, codes, c_bytes) || overlap(x, x_bytes, scales, s_bytes) ||
      overlap(codes, c_bytes, scales, s_bytes))
    return AGG_ERR_SHAPE;
  return launch_mx4_quantize(x, stride, codes, scales, rows, K, (hipStream_t)hip_stream) == hipSuccess
             ? AGG_OK
             : AGG_ERR_LAUNCH;
}

int agg_mx4_dequantize(int64_t rows, int32_t K, const void* codes, const void* scales, void* x,
                       void* hip_stream) {
  const int rc = check_mx4(rows, K);
  if (rc != AGG_OK || rows == 0) return rc;
  if (!x || !codes || !scales) return AGG_ERR_NULL;
  if (misaligned(x) || misaligned(codes) || misaligned(scales)) return AGG_ERR_ALIGN;
  const uint64_t x_bytes = (uint64_t)rows * K * 2;
  if (overlap(x, x_bytes, codes, (uint64_t)rows * mx4_code_stride(K)) ||
      overlap(x, x_bytes, scales, (uint64_t)rows * mx4_scale_stride(K)))
    return AGG_ERR_SHAPE;
  return launch_mx4_dequantize(codes, scales, x, rows, K, (hipStream_t)hip_stream) == hipSuccess ? AGG_OK
                                                                                               : AGG_ERR_LAUNCH;
}

int agg_mx4_linear_fwd(int64_t rows, int32_t N, int32_t K, const agg_mx4_linear* linear,
                       const void* codes, const void* scales, void* hip_stream) {
  Mx4LinearArgs a;
  const int rc = make_mx4_args(rows, N, K, linear, codes, scales, &a);
  if (rc != AGG_OK || rows == 0) return rc;
  return launch_mx4_linear(a, (hipStream_t)hip_stream) == hipSuccess ? AGG_OK : AGG_ERR_LAUNCH;
}

// ---- one global-attention block --------------------------------------------------------
namespace {

inline size_t align256(size_t n) { return (n + 255) & ~(size_t)255; }

// Workspace layout of agg_global_block_fwd: LayerNorm output, Q, K, V, attention output,
// then whatever the chosen attention needs.
struct BlockPlan {
  size_t act;      // bytes of one [B, N*L, C] bf16 activation
  size_t attn_ws;  // bytes behind the five activations
  size_t compact;  // SGA: bytes of one compacted tensor
  size_t total;
};

int plan_block(const agg_shape* shape, int mode, BlockPlan* p) {
  Geom g;
  int rc = make_geom(shape, &g, mode != AGG_BLOCK_SGA);
  if (rc != AGG_OK) return rc;
  if (mode != AGG_BLOCK_SGA && mode != AGG_BLOCK_FRAME && mode != AGG_BLOCK_DENSE)
    return AGG_ERR_SHAPE;
  p->act = align256((size_t)g.B * g.NQ * g.H * kHeadDim * 2);
  p->compact = 0;
  if (mode == AGG_BLOCK_SGA) {
    p->compact = align256((size_t)g.B * g.H * g.M_pad * kHeadDim * 2);
    const size_t means = align256((size_t)g.B * g.H * kHeadDim * sizeof(float));
    p->attn_ws = 2 * p->compact + 2 * means + align256(agg_workspace_bytes(shape));
  } else {
    p->attn_ws = 0;  // per-frame and ordinary attention read K and V in place
  }
  p->total = 5 * p->act + p->attn_ws;
  return AGG_OK;
}

// A block's attention by mode, on its workspace.
int block_attention(const agg_shape* shape, int mode, const BlockPlan& p, const void* Q, const void* K,
                    const void* V, void* A, char* aws, void* hip_stream) {
  if (mode == AGG_BLOCK_SGA) {
    const size_t means = align256((size_t)shape->B * shape->H * kHeadDim * sizeof(float));
    void* Kc = aws;
    void* Vc = aws + p.compact;
    float* kmean = (float*)(aws + 2 * p.compact);
    float* vmean = (float*)(aws + 2 * p.compact + means);
    void* mws = aws + 2 * p.compact + 2 * means;
    const int rc = agg_kv_subsample(shape, K, V, Kc, Vc, nullptr, kmean, vmean, mws,
                                    agg_workspace_bytes(shape), hip_stream);
    if (rc != AGG_OK) return rc;
    return agg_global_attn_fwd(shape, Q, K, V, Kc, Vc, kmean, vmean, A, nullptr, hip_stream);
  }
  if (mode == AGG_BLOCK_FRAME) return agg_frame_attn_fwd(shape, Q, K, V, A, nullptr, hip_stream);
  return agg_dense_global_attn_fwd(shape, Q, K, V, A, nullptr, hip_stream);
}

}  // namespace

size_t agg_block_workspace_bytes(const agg_shape* shape, int mode) {
  BlockPlan p;
  if (plan_block(shape, mode, &p) != AGG_OK) return 0;
  return p.total;
}

int agg_global_block_fwd(const agg_shape* shape, int mode, const agg_block_weights* w,
                         const void* x, void* y, void* workspace, size_t workspace_bytes,
                         void* hip_stream) {
  BlockPlan p;
  int rc = plan_block(shape, mode, &p);
  if (rc != AGG_OK) return rc;
  if (!w || !x || !y || !workspace || !w->ln_gamma || !w->ln_beta || !w->w_q || !w->w_k ||
      !w->w_v || !w->w_o)
    return AGG_ERR_NULL;
  if (misaligned(x) || misaligned(y) || misaligned(workspace) || misaligned(w->w_q) ||
      misaligned(w->w_k) || misaligned(w->w_v) || misaligned(w->w_o))
    return AGG_ERR_ALIGN;
  if (x == y) return AGG_ERR_SHAPE;
  if (!(w->ln_eps > 0.0f)) return AGG_ERR_SHAPE;
  if (workspace_bytes < p.total) return AGG_ERR_WORKSPACE;
  const int C = shape->H * kHeadDim;
  if (C > 4096) return AGG_ERR_UNSUPPORTED;  // LayerNorm kernel: a row lives in one wavefront's registers
  const int64_t rows = (int64_t)shape->B * shape->N * ((int64_t)shape->n_h * shape->n_w + shape->n_special);
  hipStream_t st = (hipStream_t)hip_stream;
  char* base = (char*)workspace;
  void* xn = base;
  void* Q = base + p.act;
  void* K = base + 2 * p.act;
  void* V = base + 3 * p.act;
  void* A = base + 4 * p.act;  // attention output
  char* aws = base + 5 * p.act;

  if (launch_layernorm(x, w->ln_gamma, w->ln_beta, xn, rows, C, w->ln_eps, st) != hipSuccess)
    return AGG_ERR_LAUNCH;
  const LinearOuts qkv = {{(const uint16_t*)w->w_q, (const uint16_t*)w->w_k, (const uint16_t*)w->w_v},
                          {w->b_q, w->b_k, w->b_v},
                          {(uint16_t*)Q, (uint16_t*)K, (uint16_t*)V},
                          3};
  if (launch_linear(xn, qkv, nullptr, rows, C, C, st) != hipSuccess)
    return AGG_ERR_LAUNCH;
  rc = block_attention(shape, mode, p, Q, K, V, A, aws, hip_stream);
  if (rc != AGG_OK) return rc;
  const LinearOuts out = {{(const uint16_t*)w->w_o, nullptr, nullptr},
                          {w->b_o, nullptr, nullptr},
                          {(uint16_t*)y, nullptr, nullptr},
                          1};
  if (launch_linear(A, out, x, rows, C, C, st) != hipSuccess) return AGG_ERR_LAUNCH;
  return AGG_OK;
}

// ---- the block with the other parts of a model's block ------------------------------------------
namespace {

// agg_global_block_fwd's workspace, then the codes and scales of one activation for 4-bit projections
struct BlockExPlan {
  BlockPlan block;
  size_t codes, scales, total;
};

int plan_block_ex(const agg_shape* shape, int mode, bool mx, BlockExPlan* p) {
  const int rc = plan_block(shape, mode, &p->block);
  if (rc != AGG_OK) return rc;
  p->codes = p->scales = 0;
  if (mx) {
    const size_t rows = (size_t)shape->B * shape->N * ((size_t)shape->n_h * shape->n_w + shape->n_special);
    const int64_t C = (int64_t)shape->H * kHeadDim;
    p->codes = align256(rows * mx4_code_stride(C));
    p->scales = align256(rows * mx4_scale_stride(C));
  }
  p->total = p->block.total + p->codes + p->scales;
  return AGG_OK;
}

}  // namespace

size_t agg_block_ex_workspace_bytes(const agg_shape* shape, int mode, const agg_block_options* o) {
  BlockExPlan p;
  if (!o || plan_block_ex(shape, mode, o->mx != nullptr, &p) != AGG_OK) return 0;
  return p.total;
}

int agg_global_block_ex_fwd(const agg_shape* shape, int mode, const agg_block_weights* w,
                            const agg_block_options* o, const void* x, void* y, void* n,
                            void* workspace, size_t workspace_bytes, void* hip_stream) {
  if (!o) return AGG_ERR_NULL;
  BlockExPlan p;
  int rc = plan_block_ex(shape, mode, o->mx != nullptr, &p);
  if (rc != AGG_OK) return rc;
  if (!w || !x || !y || !workspace) return AGG_ERR_NULL;
  if (o->first_done != 0 && o->first_done != 1) return AGG_ERR_SHAPE;
  if (o->first_done ? !o->x_norm : (!w->ln_gamma || !w->ln_beta)) return AGG_ERR_NULL;
  if (!o->mx && (!w->w_q || !w->w_k || !w->w_v || !w->w_o)) return AGG_ERR_NULL;
  if (misaligned(x) || misaligned(y) || misaligned(n) || misaligned(workspace) ||
      (!o->mx && (misaligned(w->w_q) || misaligned(w->w_k) || misaligned(w->w_v) || misaligned(w->w_o))))
    return AGG_ERR_ALIGN;
  if (o->first_done && misaligned(o->x_norm)) return AGG_ERR_ALIGN;
  if (!o->first_done && !(w->ln_eps > 0.0f)) return AGG_ERR_SHAPE;
  if (workspace_bytes < p.total) return AGG_ERR_WORKSPACE;
  const int C = shape->H * kHeadDim;
  if (shape->H > 4096 / kHeadDim) return AGG_ERR_UNSUPPORTED;
  const int64_t rows = (int64_t)shape->B * shape->N * ((int64_t)shape->n_h * shape->n_w + shape->n_special);
  const uint64_t bytes = (uint64_t)rows * C * 2;
  const void* x_norm = o->first_done ? o->x_norm : nullptr;
  if (overlap(x, bytes, y, bytes) || overlap(x, bytes, n, bytes) || overlap(y, bytes, n, bytes) ||
      overlap(y, bytes, x_norm, bytes) || (n != x_norm && overlap(n, bytes, x_norm, bytes)))
    return AGG_ERR_SHAPE;
  const void* used[4] = {x, y, n, x_norm};
  for (const void* t : used)
    if (overlap(t, bytes, workspace, p.total)) return AGG_ERR_SHAPE;

  const BlockPlan& b = p.block;
  hipStream_t st = (hipStream_t)hip_stream;
  char* base = (char*)workspace;
  void* xn = base;
  void* Q = base + b.act;
  void* K = base + 2 * b.act;
  void* V = base + 3 * b.act;
  void* A = base + 4 * b.act;  // attention output
  char* aws = base + 5 * b.act;
  void* codes = base + b.total;
  void* scales = base + b.total + p.codes;
  void* branch = xn;           // the output projection's result: the projections' input has been read
  const void* first = o->first_done ? o->x_norm : xn;

  // every check of the calls below comes before the first launch
  const bool turn = (o->rope && (o->rope->d_t || o->rope->d_h || o->rope->d_w)) ||
                    o->q_norm.kind != AGG_NORM_NONE || o->k_norm.kind != AGG_NORM_NONE;
  RopeArgs rope;
  rc = make_rope_args(shape, o->rope, &o->q_norm, &o->k_norm, o->pos, Q, 0, K, 0, Q, K, &rope);
  if (rc != AGG_OK) return rc;
  SeamArgs seam;
  rc = make_seam_args(rows, C, &o->residual, x, branch, y, n, &seam);
  if (rc != AGG_OK) return rc;
  // what a projection's own epilogue can add: the residual, and in 4 bits its scale
  const bool seam_apart = seam.post.kind != AGG_NORM_NONE || seam.pre.kind != AGG_NORM_NONE || seam.gate ||
                          (seam.scale && !o->mx);
  Mx4LinearArgs mx_qkv, mx_out;
  if (o->mx) {
    agg_mx4_linear l;
    memset(&l, 0, sizeof l);
    l.count = 3;
    const float* bias[3] = {w->b_q, w->b_k, w->b_v};
    void* out[3] = {Q, K, V};
    for (int i = 0; i < 3; ++i) {
      l.w[i] = o->mx[i];
      l.bias[i] = bias[i];
      l.y[i] = out[i];
    }
    if ((rc = make_mx4_args(rows, C, C, &l, codes, scales, &mx_qkv)) != AGG_OK) return rc;
    memset(&l, 0, sizeof l);
    l.count = 1;
    l.w[0] = o->mx[3];
    l.bias[0] = w->b_o;
    l.y[0] = seam_apart ? branch : y;
    l.residual = seam_apart ? nullptr : x;
    l.res_scale = seam_apart ? nullptr : o->residual.scale;
    if ((rc = make_mx4_args(rows, C, C, &l, codes, scales, &mx_out)) != AGG_OK) return rc;
  }

  if (o->mx) {
    const hipError_t e = o->first_done ? launch_mx4_quantize(o->x_norm, C, codes, scales, rows, C, st)
                                       : launch_layernorm_mx4(x, w->ln_gamma, w->ln_beta, codes, scales, rows, C, w->ln_eps, st);
    if (e != hipSuccess || launch_mx4_linear(mx_qkv, st) != hipSuccess) return AGG_ERR_LAUNCH;
  } else {
    if (!o->first_done && launch_layernorm(x, w->ln_gamma, w->ln_beta, xn, rows, C, w->ln_eps, st) != hipSuccess)
      return AGG_ERR_LAUNCH;
    const LinearOuts qkv = {{(const uint16_t*)w->w_q, (const uint16_t*)w->w_k, (const uint16_t*)w->w_v},
                            {w->b_q, w->b_k, w->b_v},
                            {(uint16_t*)Q, (uint16_t*)K, (uint16_t*)V},
                            3};
    if (launch_linear(first, qkv, nullptr, rows, C, C, st) != hipSuccess) return AGG_ERR_LAUNCH;
  }
  if (turn && launch_rope(rope, st) != hipSuccess) return AGG_ERR_LAUNCH;
  if ((rc = block_attention(shape, mode, b, Q, K, V, A, aws, hip_stream)) != AGG_OK) return rc;
  if (o->mx) {
    if (launch_mx4_quantize(A, C, codes, scales, rows, C, st) != hipSuccess ||
        launch_mx4_linear(mx_out, st) != hipSuccess)
      return AGG_ERR_LAUNCH;
  } else {
    const LinearOuts out = {{(const uint16_t*)w->w_o, nullptr, nullptr},
                            {w->b_o, nullptr, nullptr},
                            {(uint16_t*)(seam_apart ? branch : y), nullptr, nullptr},
                            1};
    if (launch_linear(A, out, seam_apart ? nullptr : x, rows, C, C, st) != hipSuccess) return AGG_ERR_LAUNCH;
  }
  if (seam_apart && launch_seam(seam, st) != hipSuccess) return AGG_ERR_LAUNCH;
  return AGG_OK;
}

}  // extern "C"
