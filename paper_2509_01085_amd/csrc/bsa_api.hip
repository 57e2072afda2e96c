// C-ABI entry points of libbsa: host-side argument validation and dispatch only.
// Every check happens before any launch, so a failed call enqueues nothing.
#include <cmath>

#include "bsa_common.h"

namespace bsa {

static int make_geom(const bsa_shape_t* s, Geom* g, bool limits) {
  if (!s) return BSA_ERR_NULL;
  if (s->dtype != BSA_F32 && s->dtype != BSA_BF16) return BSA_ERR_DTYPE;
  if (s->B <= 0 || s->H <= 0 || s->T <= 0 || s->Hs <= 0 || s->Ws <= 0 || s->Ct <= 0 ||
      s->Ch <= 0 || s->Cw <= 0 || s->d <= 0)
    return BSA_ERR_SHAPE;
  // the paper assumes T/Ct, H/Ch, W/Cw are integers (Sec. 3.2.1)
  if (s->T % s->Ct || s->Hs % s->Ch || s->Ws % s->Cw) return BSA_ERR_SHAPE;
  if (s->d % 8 || s->d > 256) return BSA_ERR_SHAPE;
  const int64_t Bk = (int64_t)s->Ct * s->Ch * s->Cw;
  const int64_t L = (int64_t)s->T * s->Hs * s->Ws;
  if (limits && Bk > 256) return BSA_ERR_SHAPE;
  const int64_t N = L / Bk;
  if (limits && N > 8192) return BSA_ERR_SHAPE;
  const int64_t rows = (int64_t)s->B * s->H * N;
  if (limits && rows * N > 0x7fffffffLL) return BSA_ERR_SHAPE;   // CSR offsets are int32
  if ((int64_t)s->B * s->H * L > 0x3fffffffffLL / s->d) return BSA_ERR_SHAPE;
  g->B = s->B; g->H = s->H; g->T = s->T; g->Hs = s->Hs; g->Ws = s->Ws;
  g->Ct = s->Ct; g->Ch = s->Ch; g->Cw = s->Cw; g->d = s->d;
  g->Nt = s->T / s->Ct; g->Nh = s->Hs / s->Ch; g->Nw = s->Ws / s->Cw;
  g->Bk = (int)Bk; g->N = (int)N; g->L = (int)L; g->rows = (int)rows;
  // windows of the critical-token mechanism must divide the block evenly (Sec. 3.2.2); 0 = the block
  if (s->Wt < 0 || s->Wh < 0 || s->Ww < 0) return BSA_ERR_SHAPE;
  g->Wt = s->Wt ? s->Wt : s->Ct; g->Wh = s->Wh ? s->Wh : s->Ch; g->Ww = s->Ww ? s->Ww : s->Cw;
  if (s->Ct % g->Wt || s->Ch % g->Wh || s->Cw % g->Ww) return BSA_ERR_SHAPE;
  g->Wk = g->Wt * g->Wh * g->Ww;
  g->nwin = g->Bk / g->Wk;
  if (s->layout != BSA_LAYOUT_RASTER && s->layout != BSA_LAYOUT_BLOCK_MAJOR) return BSA_ERR_SHAPE;
  g->tiled = s->layout == BSA_LAYOUT_BLOCK_MAJOR;
  g->dense = 0;
  g->inv_Nw = g->Nw == 1 ? 0u : (uint32_t)(0x100000000ull / (uint32_t)g->Nw) + 1u;
  g->inv_NwNh = g->Nw * g->Nh == 1 ? 0u : (uint32_t)(0x100000000ull / (uint32_t)(g->Nw * g->Nh)) + 1u;
  return BSA_OK;
}

int make_geom(const bsa_shape_t* s, Geom* g) { return make_geom(s, g, true); }

int make_token_geom(const bsa_shape_t* s, Geom* g) {
  if (s && s->T > 0 && s->Hs > 0 && s->Ws > 0 && s->B > 0) {  // B*L < 2^31: token numbers are int32
    const int64_t hw = (int64_t)s->Hs * s->Ws, most = 0x7fffffffLL / s->B;
    if (hw > most || s->T > most / hw) return BSA_ERR_SHAPE;
  }
  return make_geom(s, g, false);
}

// retained tokens per window, ceil(r * Wk); per block it is nwin times that
static int window_quota(const Geom& g, double r) {
  if (!(r > 0.0) || !(r <= 1.0)) return BSA_ERR_RANGE;
  int n = (int)std::ceil(r * g.Wk - 1e-12);
  if (n < 1) n = 1;
  if (n > g.Wk) n = g.Wk;
  return n;
}

static int n_keep_of(const Geom& g, double r) {
  const int kw = window_quota(g, r);
  return kw < 0 ? kw : kw * g.nwin;
}

}  // namespace bsa

using namespace bsa;

extern "C" {

const char* bsa_strerror(int status) {
  switch (status) {
    case BSA_OK: return "ok";
    case BSA_ERR_NULL: return "a required pointer is NULL";
    case BSA_ERR_SHAPE: return "unsupported shape (extents must be positive, the block must divide the grid, d%8==0, d<=256, Bk<=256, N<=8192)";
    case BSA_ERR_RANGE: return "threshold / keep ratio must lie in (0,1], n_keep in [1,Bk], sm_scale > 0, eps > 0 and normal, theta > 0, all finite, stages in 1..7";
    case BSA_ERR_CAPACITY: return "index buffer smaller than rows*N";
    case BSA_ERR_DTYPE: return "dtype must be BSA_F32 or BSA_BF16";
    case BSA_ERR_LAUNCH: return "HIP launch error";
    case BSA_ERR_WORKSPACE: return "workspace missing or too small";
    case BSA_ERR_STATIC_LIMIT: return "shape needs more scratch than the library's built-in buffer holds (BSA_STATIC_SELECT_BYTES)";
    case BSA_ERR_STRIDE: return "strides and addresses (workspaces too) must be multiples of 16 bytes, a rotation table's of 8, strides in [0, 2^40), outputs without overlap";
    default: return "unknown bsa status";
  }
}

int bsa_n_keep(const bsa_shape_t* shape, double keep_ratio) {
  Geom g;
  int rc = make_geom(shape, &g);
  if (rc) return rc;
  return n_keep_of(g, keep_ratio);
}

int bsa_pool_blocks(const bsa_shape_t* shape, const void* X, double* Xbar, void* stream) {
  Geom g;
  int rc = make_geom(shape, &g);
  if (rc) return rc;
  if (!X || !Xbar) return BSA_ERR_NULL;
  return launch_pool(g, shape->dtype, X, Xbar, (hipStream_t)stream);
}

size_t bsa_select_workspace_bytes(const bsa_shape_t* shape) {
  Geom g;
  if (make_geom(shape, &g)) return 0;
  return select_workspace_bytes(g);
}

// use_static: the workspace is this device's copy of the library-owned scratch
static int select_common(const bsa_shape_t* shape, const double* Qbar, const double* Kbar,
                         double threshold, double stat_z, double score_scale, int32_t* q2k_ptr,
                         int32_t* q2k_idx, int64_t idx_capacity, int32_t* k2q_ptr, int32_t* k2q_idx,
                         int64_t* nnz_dev, void* workspace, size_t workspace_bytes, bool use_static,
                         void* stream) {
  Geom g;
  int rc = make_geom(shape, &g);
  if (rc) return rc;
  if (!Qbar || !Kbar || !q2k_ptr || !q2k_idx) return BSA_ERR_NULL;
  if ((k2q_ptr == nullptr) != (k2q_idx == nullptr)) return BSA_ERR_NULL;
  if (!(threshold > 0.0) || !(threshold <= 1.0)) return BSA_ERR_RANGE;
  if (!std::isfinite(score_scale)) return BSA_ERR_RANGE;
  if (idx_capacity < (int64_t)g.rows * g.N) return BSA_ERR_CAPACITY;
  if (use_static) {
    if (select_workspace_bytes(g) > (size_t)BSA_STATIC_SELECT_BYTES) return BSA_ERR_STATIC_LIMIT;
    if ((rc = static_select_scratch(&workspace, &workspace_bytes)) != BSA_OK) return rc;
  }
  if (!workspace || workspace_bytes < select_workspace_bytes(g)) return BSA_ERR_WORKSPACE;
  return launch_select(g, Qbar, Kbar, threshold, stat_z, score_scale, q2k_ptr, q2k_idx, k2q_ptr, k2q_idx,
                       nnz_dev, workspace, (hipStream_t)stream);
}

int bsa_select_kv(const bsa_shape_t* shape, const double* Qbar, const double* Kbar,
                  double threshold, double score_scale, int32_t* q2k_ptr, int32_t* q2k_idx,
                  int64_t idx_capacity, int32_t* k2q_ptr, int32_t* k2q_idx, int64_t* nnz_dev,
                  void* workspace, size_t workspace_bytes, void* stream) {
  return select_common(shape, Qbar, Kbar, threshold, (double)NAN, score_scale, q2k_ptr, q2k_idx,
                       idx_capacity, k2q_ptr, k2q_idx, nnz_dev, workspace, workspace_bytes, false, stream);
}

int bsa_select_kv_static(const bsa_shape_t* shape, const double* Qbar, const double* Kbar,
                         double threshold, double score_scale, int32_t* q2k_ptr, int32_t* q2k_idx,
                         int64_t idx_capacity, int32_t* k2q_ptr, int32_t* k2q_idx, int64_t* nnz_dev,
                         void* stream) {
  return select_common(shape, Qbar, Kbar, threshold, (double)NAN, score_scale, q2k_ptr, q2k_idx,
                       idx_capacity, k2q_ptr, k2q_idx, nnz_dev, nullptr, 0, true, stream);
}

int bsa_select_kv_stat(const bsa_shape_t* shape, const double* Qbar, const double* Kbar,
                       double threshold, double stat_z, double score_scale, int32_t* q2k_ptr,
                       int32_t* q2k_idx, int64_t idx_capacity, int32_t* k2q_ptr, int32_t* k2q_idx,
                       int64_t* nnz_dev, void* workspace, size_t workspace_bytes, void* stream) {
  if (stat_z != stat_z) return BSA_ERR_RANGE;  // NaN
  return select_common(shape, Qbar, Kbar, threshold, stat_z, score_scale, q2k_ptr, q2k_idx,
                       idx_capacity, k2q_ptr, k2q_idx, nnz_dev, workspace, workspace_bytes, false, stream);
}

int bsa_prune_q(const bsa_shape_t* shape, const void* Q, double keep_ratio, int32_t* keep_idx,
                void* stream) {
  Geom g;
  int rc = make_geom(shape, &g);
  if (rc) return rc;
  if (!Q || !keep_idx) return BSA_ERR_NULL;
  const int kw = window_quota(g, keep_ratio);
  if (kw < 0) return kw;
  return launch_prune(g, shape->dtype, Q, kw, keep_idx, (hipStream_t)stream);
}

size_t bsa_fwd_workspace_bytes(const bsa_shape_t* shape, int n_keep) {
  Geom g;
  if (make_geom(shape, &g)) return 0;
  if (n_keep < 1 || n_keep > g.Bk) return 0;
  return mfma_supported(g, shape->dtype, n_keep) ? fwd_workspace_pipe(g, n_keep) : 0;
}

int bsa_attn_fwd(const bsa_shape_t* shape, const void* Q, const void* K, const void* V,
                 const int32_t* q2k_ptr, const int32_t* q2k_idx, const int32_t* keep_idx,
                 int n_keep, float sm_scale, void* O, float* LSE, void* workspace,
                 size_t workspace_bytes, void* stream) {
  Geom g;
  int rc = make_geom(shape, &g);
  if (rc) return rc;
  if (!Q || !K || !V || !q2k_ptr || !q2k_idx || !keep_idx || !O || !LSE) return BSA_ERR_NULL;
  if (n_keep < 1 || n_keep > g.Bk || !(sm_scale > 0.f) || !std::isfinite(sm_scale)) return BSA_ERR_RANGE;
  const size_t need = bsa_fwd_workspace_bytes(shape, n_keep);
  if (need && (!workspace || workspace_bytes < need)) return BSA_ERR_WORKSPACE;
  AttnArgs a{};
  a.fwd_ws = need ? workspace : nullptr;
  a.Q = Q; a.K = K; a.V = V; a.q2k_ptr = q2k_ptr; a.q2k_idx = q2k_idx; a.keep_idx = keep_idx;
  a.n_keep = n_keep; a.sm_scale = sm_scale; a.O_out = O; a.LSE_out = LSE;
  if (mfma_supported(g, shape->dtype, n_keep)) return launch_fwd_pipe(g, a, (hipStream_t)stream);
  return launch_fwd_generic(g, shape->dtype, a, (hipStream_t)stream);
}

size_t bsa_bwd_workspace_bytes(const bsa_shape_t* shape, int n_keep) {
  Geom g;
  if (make_geom(shape, &g)) return 0;
  if (n_keep < 1 || n_keep > g.Bk) return 0;
  if (mfma_supported(g, shape->dtype, n_keep)) return bwd_workspace_pipe(g, n_keep);
  return bwd_workspace_generic(g, n_keep);
}

int bsa_attn_bwd(const bsa_shape_t* shape, const void* Q, const void* K, const void* V,
                 const void* O, const float* LSE, const void* dO, const int32_t* q2k_ptr,
                 const int32_t* q2k_idx, const int32_t* k2q_ptr, const int32_t* k2q_idx,
                 const int32_t* keep_idx, int n_keep, float sm_scale, void* dQ, void* dK, void* dV,
                 void* workspace, size_t workspace_bytes, void* stream) {
  return bsa_attn_bwd_stages(shape, Q, K, V, O, LSE, dO, q2k_ptr, q2k_idx, k2q_ptr, k2q_idx, keep_idx,
                             n_keep, sm_scale, dQ, dK, dV, workspace, workspace_bytes,
                             BSA_BWD_PRE | BSA_BWD_DQ | BSA_BWD_DKV, stream);
}

int bsa_attn_bwd_stages(const bsa_shape_t* shape, const void* Q, const void* K, const void* V,
                        const void* O, const float* LSE, const void* dO, const int32_t* q2k_ptr,
                        const int32_t* q2k_idx, const int32_t* k2q_ptr, const int32_t* k2q_idx,
                        const int32_t* keep_idx, int n_keep, float sm_scale, void* dQ, void* dK,
                        void* dV, void* workspace, size_t workspace_bytes, unsigned stages,
                        void* stream) {
  Geom g;
  int rc = make_geom(shape, &g);
  if (rc) return rc;
  if (!Q || !K || !V || !O || !LSE || !dO || !q2k_ptr || !q2k_idx || !k2q_ptr || !k2q_idx ||
      !keep_idx || !dQ || !dK || !dV)
    return BSA_ERR_NULL;
  if (n_keep < 1 || n_keep > g.Bk || !(sm_scale > 0.f) || !std::isfinite(sm_scale)) return BSA_ERR_RANGE;
  if (!workspace || workspace_bytes < bsa_bwd_workspace_bytes(shape, n_keep)) return BSA_ERR_WORKSPACE;
  AttnArgs a{};
  a.Q = Q; a.K = K; a.V = V; a.O = O; a.LSE_in = LSE; a.dO = dO;
  a.q2k_ptr = q2k_ptr; a.q2k_idx = q2k_idx; a.k2q_ptr = k2q_ptr; a.k2q_idx = k2q_idx;
  a.keep_idx = keep_idx; a.n_keep = n_keep; a.sm_scale = sm_scale;
  a.dQ = dQ; a.dK = dK; a.dV = dV; a.ws = workspace;
  if (stages == 0 || (stages & ~7u)) return BSA_ERR_RANGE;
  a.stages = stages;
  if (mfma_supported(g, shape->dtype, n_keep)) return launch_bwd_pipe(g, a, (hipStream_t)stream);
  return launch_bwd_generic(g, shape->dtype, a, (hipStream_t)stream);
}

// ---- dense baseline (Eq. 1): same kernels, tiles = runs of Bk consecutive tokens, all pairs ----
static int dense_geom(const bsa_shape_t* shape, Geom* g) {
  int rc = make_geom(shape, g);
  if (rc) return rc;
  g->dense = 1;
  g->tiled = 1;
  return BSA_OK;
}

size_t bsa_dense_bwd_workspace_bytes(const bsa_shape_t* shape) {
  Geom g;
  if (dense_geom(shape, &g)) return 0;
  if (mfma_supported(g, shape->dtype, g.Bk)) return bwd_workspace_pipe(g, g.Bk);
  return bwd_workspace_generic(g, g.Bk);
}

int bsa_dense_attn_fwd(const bsa_shape_t* shape, const void* Q, const void* K, const void* V,
                       float sm_scale, void* O, float* LSE, void* stream) {
  Geom g;
  int rc = dense_geom(shape, &g);
  if (rc) return rc;
  if (!Q || !K || !V || !O || !LSE) return BSA_ERR_NULL;
  if (!(sm_scale > 0.f) || !std::isfinite(sm_scale)) return BSA_ERR_RANGE;
  AttnArgs a{};
  a.Q = Q; a.K = K; a.V = V; a.n_keep = g.Bk; a.sm_scale = sm_scale; a.O_out = O; a.LSE_out = LSE;
  if (mfma_supported(g, shape->dtype, g.Bk)) return launch_fwd_pipe(g, a, (hipStream_t)stream);
  return launch_fwd_generic(g, shape->dtype, a, (hipStream_t)stream);
}

int bsa_dense_attn_bwd(const bsa_shape_t* shape, const void* Q, const void* K, const void* V,
                       const void* O, const float* LSE, const void* dO, float sm_scale, void* dQ,
                       void* dK, void* dV, void* workspace, size_t workspace_bytes, void* stream) {
  Geom g;
  int rc = dense_geom(shape, &g);
  if (rc) return rc;
  if (!Q || !K || !V || !O || !LSE || !dO || !dQ || !dK || !dV) return BSA_ERR_NULL;
  if (!(sm_scale > 0.f) || !std::isfinite(sm_scale)) return BSA_ERR_RANGE;
  if (!workspace || workspace_bytes < bsa_dense_bwd_workspace_bytes(shape)) return BSA_ERR_WORKSPACE;
  AttnArgs a{};
  a.Q = Q; a.K = K; a.V = V; a.O = O; a.LSE_in = LSE; a.dO = dO; a.n_keep = g.Bk;
  a.sm_scale = sm_scale; a.dQ = dQ; a.dK = dK; a.dV = dV; a.ws = workspace;
  a.stages = BSA_BWD_PRE | BSA_BWD_DQ | BSA_BWD_DKV;
  if (mfma_supported(g, shape->dtype, g.Bk)) return launch_bwd_pipe(g, a, (hipStream_t)stream);
  return launch_bwd_generic(g, shape->dtype, a, (hipStream_t)stream);
}

}  // extern "C"

// ---- the operators around the attention: tensors with strides ----
namespace bsa {

static bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }
static bool aligned8(const void* p) { return ((uintptr_t)p & 7) == 0; }  // cosine and sine are one load

// Partial results and row statistics move in 16 bytes.
static int fit_workspace(const void* p, size_t bytes, size_t need) {
  if (!need) return BSA_OK;
  if (!p || bytes < need) return BSA_ERR_WORKSPACE;
  return aligned16(p) ? BSA_OK : BSA_ERR_STRIDE;
}

// Multiples of 16 bytes in range; the stride of an extent of 1 becomes 0.
static int fit_strides(bsa_strides_t* s, int64_t b, int64_t l, int64_t h, int dtype) {
  const int64_t n[3] = {b, l, h}, unit = dtype == BSA_F32 ? 4 : 8;
  int64_t* v[3] = {&s->b, &s->l, &s->h};
  for (int i = 0; i < 3; ++i) {
    if (n[i] == 1) *v[i] = 0;
    if (*v[i] < 0 || *v[i] >= (1LL << 40) || *v[i] % unit) return BSA_ERR_STRIDE;
  }
  return BSA_OK;
}

// The same for a tensor that is written: along the indexes by rising stride, each step leaves what is below it behind.
static int fit_out_strides(bsa_strides_t* s, int64_t b, int64_t l, int64_t h, int d, int dtype) {
  const int rc = fit_strides(s, b, l, h, dtype);
  if (rc) return rc;
  int64_t n[3] = {b, l, h}, v[3] = {s->b, s->l, s->h};
  for (int i = 0; i < 2; ++i)
    for (int j = 0; j < 2 - i; ++j)
      if (v[j] > v[j + 1]) {
        const int64_t tv = v[j], tn = n[j];
        v[j] = v[j + 1]; v[j + 1] = tv;
        n[j] = n[j + 1]; n[j + 1] = tn;
      }
  int64_t span = d;
  for (int i = 0; i < 3; ++i) {
    if (n[i] == 1) continue;
    if (v[i] < span) return BSA_ERR_STRIDE;
    if (n[i] - 1 > ((1LL << 60) - span) / v[i]) return BSA_ERR_STRIDE;
    span += (n[i] - 1) * v[i];
  }
  return BSA_OK;
}

static int rope_of(const Geom& g, const bsa_rope_t* rope, RopeArgs* a) {
  a->nt = a->nh = a->nw = a->halves = 0;
  if (!rope) return BSA_OK;
  if (rope->dt < 0 || rope->dh < 0 || rope->dw < 0 || rope->dt > g.d || rope->dh > g.d || rope->dw > g.d) return BSA_ERR_SHAPE;
  if (rope->dt % 2 || rope->dh % 2 || rope->dw % 2) return BSA_ERR_SHAPE;
  const int n = rope->dt + rope->dh + rope->dw;
  if (n > g.d || n % 8) return BSA_ERR_SHAPE;
  if (rope->style != BSA_ROPE_PAIRS && rope->style != BSA_ROPE_HALVES) return BSA_ERR_SHAPE;
  a->nt = rope->dt / 2; a->nh = rope->dh / 2; a->nw = rope->dw / 2;
  a->halves = rope->style == BSA_ROPE_HALVES;
  return BSA_OK;
}

static int rope_args(const bsa_shape_t* shape, const bsa_rope_t* rope, const float* table, float eps, Geom* g, RopeArgs* a) {
  int rc = make_token_geom(shape, g);
  if (rc) return rc;
  if ((rc = rope_of(*g, rope, a)) != BSA_OK) return rc;
  if (!rope_fits(*g)) return BSA_ERR_SHAPE;
  if (a->nt + a->nh + a->nw) {
    if (!table) return BSA_ERR_NULL;
    if (!aligned8(table)) return BSA_ERR_STRIDE;
  }
  if (!(eps > 0.f) || !std::isnormal(eps)) return BSA_ERR_RANGE;  // (v_rsq_f32 takes a subnormal number for zero)
  a->table = table;
  a->eps = eps;
  return BSA_OK;
}

static int cross_args(const bsa_cross_shape_t* s, CrossArgs* a) {
  if (!s) return BSA_ERR_NULL;
  if (s->dtype != BSA_F32 && s->dtype != BSA_BF16) return BSA_ERR_DTYPE;
  if (s->B <= 0 || s->H <= 0 || s->Hkv <= 0 || s->Lq <= 0 || s->S <= 0 || s->d <= 0) return BSA_ERR_SHAPE;
  if (s->H % s->Hkv || s->d % 8 || s->d > 256) return BSA_ERR_SHAPE;
  const int G = s->H / s->Hkv;
  if ((int64_t)G * s->Lq > 0x7fffff00LL || s->Lq > 0x7fffff00 || s->S > 0x7fffff00) return BSA_ERR_SHAPE;
  // tiles of 32 queries by 32 keys, heads and batch: the kernels count them in 32 bits
  const int64_t tiles = (int64_t)((s->Lq + 31) / 32) * ((s->S + 31) / 32), heads = (int64_t)s->B * s->H;
  if (heads > 0x3fffffffLL / ((s->Lq + 31) / 32 + (s->S + 31) / 32) || tiles > 0x3fffffffLL / heads) return BSA_ERR_SHAPE;
  if ((((int64_t)G * s->Lq + 127) / 128) * s->B * s->Hkv >= 1 << 23) return BSA_ERR_SHAPE;  // units: a launch has fewer than 2^32 threads
  a->B = s->B; a->H = s->H; a->Hkv = s->Hkv; a->G = G; a->Lq = s->Lq; a->M = G * s->Lq; a->S = s->S; a->d = s->d; a->dtype = s->dtype;
  return BSA_OK;
}

static int cross_strides(const bsa_cross_shape_t* s, CrossArgs* a, bool backward) {
  a->q = s->q; a->k = s->k; a->v = s->v; a->o = s->o;
  int rc;
  if ((rc = fit_strides(&a->q, s->B, s->Lq, s->H, s->dtype)) || (rc = fit_strides(&a->k, s->B, s->S, s->Hkv, s->dtype)) ||
      (rc = fit_strides(&a->v, s->B, s->S, s->Hkv, s->dtype)))
    return rc;
  return backward ? fit_strides(&a->o, s->B, s->Lq, s->H, s->dtype) : fit_out_strides(&a->o, s->B, s->Lq, s->H, s->d, s->dtype);
}

}  // namespace bsa

extern "C" {

size_t bsa_rope_table_bytes(const bsa_shape_t* shape, const bsa_rope_t* rope) {
  Geom g;
  RopeArgs a{};
  if (make_token_geom(shape, &g) || rope_of(g, rope, &a)) return 0;
  return ((size_t)g.T * a.nt + (size_t)g.Hs * a.nh + (size_t)g.Ws * a.nw) * 2 * sizeof(float);
}

int bsa_rope_table(const bsa_shape_t* shape, const bsa_rope_t* rope, double theta, int64_t t0, int64_t h0, int64_t w0,
                   float* table, void* stream) {
  Geom g;
  RopeArgs a{};
  int rc = make_token_geom(shape, &g);
  if (rc) return rc;
  if ((rc = rope_of(g, rope, &a)) != BSA_OK) return rc;
  if (!rope || !table) return BSA_ERR_NULL;
  if (!aligned8(table)) return BSA_ERR_STRIDE;
  if (!(theta > 0.0) || !std::isfinite(theta)) return BSA_ERR_RANGE;
  const double origin[3] = {(double)t0, (double)h0, (double)w0};
  return launch_rope_table(g, a, theta, origin, table, (hipStream_t)stream);
}

int bsa_qk_norm_rope_fwd(const bsa_shape_t* shape, const bsa_rope_t* rope, const float* table, const void* Xq,
                         const void* Xk, const void* Xv, const bsa_strides_t* x, const float* wq, const float* wk,
                         float eps, void* Q, void* K, void* V, void* stream) {
  Geom g;
  RopeArgs a{};
  int rc = rope_args(shape, rope, table, eps, &g, &a);
  if (rc) return rc;
  const void* in[3] = {Xq, Xk, Xv};
  void* out[3] = {Q, K, V};
  if (!x || (!Xq && !Xk && !Xv)) return BSA_ERR_NULL;
  for (int i = 0; i < 3; ++i) {
    if (!in[i] != !out[i]) return BSA_ERR_NULL;
    if (!aligned16(in[i]) || !aligned16(out[i])) return BSA_ERR_STRIDE;
    a.X[i] = in[i]; a.Y[i] = out[i];
  }
  a.x = *x;
  if ((rc = fit_strides(&a.x, g.B, g.L, g.H, shape->dtype)) != BSA_OK) return rc;
  a.w[0] = wq; a.w[1] = wk;
  return launch_rope_fwd(g, shape->dtype, a, (hipStream_t)stream);
}

size_t bsa_qk_norm_rope_bwd_workspace_bytes(const bsa_shape_t* shape) {
  Geom g;
  if (make_token_geom(shape, &g)) return 0;
  return rope_bwd_workspace(g);
}

int bsa_qk_norm_rope_bwd(const bsa_shape_t* shape, const bsa_rope_t* rope, const float* table, const void* Xq,
                         const void* Xk, const bsa_strides_t* x, const float* wq, const float* wk, float eps,
                         const void* dQ, const void* dK, const void* dV, void* dXq, void* dXk, void* dXv,
                         const bsa_strides_t* dx, float* dwq, float* dwk, void* workspace, size_t workspace_bytes,
                         void* stream) {
  Geom g;
  RopeArgs a{};
  int rc = rope_args(shape, rope, table, eps, &g, &a);
  if (rc) return rc;
  const void* in[2] = {Xq, Xk};
  const void* dy[3] = {dQ, dK, dV};
  void* out[3] = {dXq, dXk, dXv};
  float* dw[2] = {dwq, dwk};
  if (!dx || (!dQ && !dK && !dV) || (!x && (Xq || Xk))) return BSA_ERR_NULL;
  for (int i = 0; i < 3; ++i) {
    if (!dy[i] != !out[i]) return BSA_ERR_NULL;
    if (i < 2 && (!in[i] != !out[i] || (!in[i] && dw[i]))) return BSA_ERR_NULL;
    if ((i < 2 && !aligned16(in[i])) || !aligned16(dy[i]) || !aligned16(out[i])) return BSA_ERR_STRIDE;
    if (i < 2) { a.X[i] = in[i]; a.dw[i] = dw[i]; }
    a.dY[i] = dy[i]; a.dX[i] = out[i];
  }
  if (x) {
    a.x = *x;
    if ((rc = fit_strides(&a.x, g.B, g.L, g.H, shape->dtype)) != BSA_OK) return rc;
  }
  a.dx = *dx;
  if ((rc = fit_out_strides(&a.dx, g.B, g.L, g.H, g.d, shape->dtype)) != BSA_OK) return rc;
  if ((rc = fit_workspace(workspace, workspace_bytes, rope_bwd_workspace(g))) != BSA_OK) return rc;
  a.w[0] = wq; a.w[1] = wk;
  a.part = static_cast<float*>(workspace);
  return launch_rope_bwd(g, shape->dtype, a, (hipStream_t)stream);
}

size_t bsa_cross_attn_fwd_workspace_bytes(const bsa_cross_shape_t* shape) {
  CrossArgs a{};
  return cross_args(shape, &a) ? 0 : cross_fwd_workspace(a);
}

int bsa_cross_attn_fwd(const bsa_cross_shape_t* shape, const void* Q, const void* K, const void* V, const int32_t* kv_len,
                       const uint8_t* kv_mask, float sm_scale, void* O, float* LSE, void* workspace,
                       size_t workspace_bytes, void* stream) {
  CrossArgs a{};
  int rc = cross_args(shape, &a);
  if (rc) return rc;
  if (!Q || !K || !V || !O || !LSE) return BSA_ERR_NULL;
  if (!(sm_scale > 0.f) || !std::isfinite(sm_scale)) return BSA_ERR_RANGE;
  if (!aligned16(Q) || !aligned16(K) || !aligned16(V) || !aligned16(O)) return BSA_ERR_STRIDE;
  if ((rc = cross_strides(shape, &a, false)) != BSA_OK) return rc;
  if ((rc = fit_workspace(workspace, workspace_bytes, cross_fwd_workspace(a))) != BSA_OK) return rc;
  a.Q = Q; a.K = K; a.V = V; a.kv_len = kv_len; a.kv_mask = kv_mask; a.sm_scale = sm_scale;
  a.O_out = O; a.LSE_out = LSE; a.ws = workspace; a.ws_bytes = workspace ? workspace_bytes : 0;
  return launch_cross_fwd(a, (hipStream_t)stream);
}

size_t bsa_cross_attn_bwd_workspace_bytes(const bsa_cross_shape_t* shape) {
  CrossArgs a{};
  return cross_args(shape, &a) ? 0 : cross_bwd_workspace(a);
}

int bsa_cross_attn_bwd(const bsa_cross_shape_t* shape, const void* Q, const void* K, const void* V, const void* O,
                       const float* LSE, const void* dO, const int32_t* kv_len, const uint8_t* kv_mask, float sm_scale,
                       void* dQ, void* dK, void* dV, const bsa_strides_t* grads, void* workspace,
                       size_t workspace_bytes, void* stream) {
  CrossArgs a{};
  int rc = cross_args(shape, &a);
  if (rc) return rc;
  if (!Q || !K || !V || !O || !LSE || !dO || !dQ || !dK || !dV) return BSA_ERR_NULL;
  if (!(sm_scale > 0.f) || !std::isfinite(sm_scale)) return BSA_ERR_RANGE;
  for (const void* p : {Q, K, V, O, dO, (const void*)dQ, (const void*)dK, (const void*)dV})
    if (!aligned16(p)) return BSA_ERR_STRIDE;
  if ((int64_t)((a.S + 63) / 64) * a.B * a.Hkv >= 1 << 23) return BSA_ERR_SHAPE;
  if ((rc = cross_strides(shape, &a, true)) != BSA_OK) return rc;
  a.go = grads ? grads[0] : shape->o;
  a.gq = grads ? grads[1] : shape->q;
  a.gk = grads ? grads[2] : shape->k;
  a.gv = grads ? grads[3] : shape->v;
  const int t = shape->dtype;
  if ((rc = fit_strides(&a.go, a.B, a.Lq, a.H, t)) || (rc = fit_out_strides(&a.gq, a.B, a.Lq, a.H, a.d, t)) ||
      (rc = fit_out_strides(&a.gk, a.B, a.S, a.Hkv, a.d, t)) || (rc = fit_out_strides(&a.gv, a.B, a.S, a.Hkv, a.d, t)))
    return rc;
  if ((rc = fit_workspace(workspace, workspace_bytes, cross_bwd_workspace(a))) != BSA_OK) return rc;
  a.Q = Q; a.K = K; a.V = V; a.O = O; a.LSE_in = LSE; a.dO = dO; a.kv_len = kv_len; a.kv_mask = kv_mask;
  a.sm_scale = sm_scale; a.dQ = dQ; a.dK = dK; a.dV = dV; a.ws = workspace; a.ws_bytes = workspace_bytes;
  return launch_cross_bwd(a, (hipStream_t)stream);
}

}  // extern "C"
