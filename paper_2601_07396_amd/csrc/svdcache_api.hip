// C ABI of libsvdcache: argument validation and dispatch.  See include/svdcache.h.
#include <stdint.h>

#include <mutex>

#include "eight_bit.h"
#include "svdc_internal.h"

using namespace svdc;

// Workspace of svdcache_fit_basis_static: one array per GPU, part of the loaded code object, so the entry point
// never allocates.  In host code this name is only a handle for hipGetSymbolAddress; the device address it resolves
// to (per device) is what kernels get.
static __device__ __align__(256) unsigned char scratch[SVDC_STATIC_SCRATCH_BYTES];

namespace {

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

int32_t check_shape(const svdc_shape* s) {
  if (!s) return SVDC_E_NULL;
  if (s->dtype != SVDC_F32 && s->dtype != SVDC_BF16) return SVDC_E_DTYPE;
  if (s->precision != SVDC_PRECISE && s->precision != SVDC_FAST) return SVDC_E_PARAM;
  if (s->B < 1 || s->B > 65535 || s->N < 1 || s->D < 1 || s->k < 1) return SVDC_E_SHAPE;
  if (s->N > (1 << 30) || s->D > (1 << 30)) return SVDC_E_SHAPE;   // tile counts such as (N + 31) / 32 stay in int
  if (s->k > s->N || s->k > s->D || s->k > 1024) return SVDC_E_SHAPE;
  // At most 2^48 elements from the first to the last block: more than any device holds, and small enough
  // that no offset or byte count computed from these strides leaves the int64 range.
  constexpr int64_t kMaxElems = int64_t(1) << 48;
  if (s->ldf < s->D || s->ldf > kMaxElems / s->N) return SVDC_E_SHAPE;
  if (s->block_stride < (int64_t)(s->N - 1) * s->ldf + s->D || s->block_stride > kMaxElems / s->B) return SVDC_E_SHAPE;
  const int64_t unit = s->dtype == SVDC_BF16 ? 8 : 4;
  if (s->D % unit || s->ldf % unit || s->block_stride % unit) return SVDC_E_ALIGN;
  return SVDC_OK;
}

// Limits of the operators in 8 bits: rows and row strides (a stride is checked where its tensor is given)
constexpr int32_t kMaxColumns8 = 1 << 20, kMaxOutputs8 = 1 << 24;
bool rows8_ok(int64_t rows, int32_t D) { return rows >= 0 && rows <= INT32_MAX && D >= 1 && D <= kMaxColumns8; }
bool stride8_ok(int64_t rows, int32_t D, int64_t ld) { return ld >= D && ld <= (int64_t(1) << 48) / (rows > 0 ? rows : 1); }
bool plain_dtype(int32_t dtype) { return dtype == SVDC_F32 || dtype == SVDC_BF16; }
size_t dtype_size(int32_t dtype) { return dtype == SVDC_F32 ? 4 : dtype == SVDC_BF16 ? 2 : 1; }

int32_t check_matmul8(const svdc_matmul8* p) {
  if (!p) return SVDC_E_NULL;
  if (!plain_dtype(p->dtype) && p->dtype != SVDC_E4M3) return SVDC_E_DTYPE;
  if (p->act != SVDC_ACT_NONE && p->act != SVDC_ACT_GELU && p->act != SVDC_ACT_SWIGLU) return SVDC_E_PARAM;
  if (!rows8_ok(p->M, p->K) || p->N < 1 || p->N > kMaxOutputs8) return SVDC_E_SHAPE;
  if (p->dtype != SVDC_E4M3 && !stride8_ok(p->M, p->N, p->ldo)) return SVDC_E_SHAPE;
  if (p->dtype == SVDC_E4M3 && p->N > kMaxColumns8) return SVDC_E_SHAPE;   // the result is a matrix in 8 bits itself
  return SVDC_OK;
}

// Limits of the operators around the attention.  With rows up to 2^31 and the strides' limits no offset leaves 2^62.
constexpr int32_t kMaxHeadDim = 256, kMaxHeads = 1 << 16, kMaxTurned = 128;
constexpr int64_t kMaxRowStride = int64_t(1) << 22, kMaxStride = int64_t(1) << 40, kMaxAttentionRows = int64_t(1) << 30;
bool heads_ok(const svdc_heads& s, bool seq = true) {
  return s.row >= 0 && s.row <= kMaxRowStride && s.head >= 0 && s.head <= kMaxStride && (!seq || (s.seq >= 0 && s.seq <= kMaxStride));
}
bool same_heads(const svdc_heads& a, const svdc_heads& b) { return a.seq == b.seq && a.row == b.row && a.head == b.head; }
bool batch_rows_ok(int64_t batch, int64_t rows) {
  return batch >= 0 && batch <= INT32_MAX && rows >= 0 && rows <= INT32_MAX && batch * rows <= INT32_MAX;
}

int32_t check_attention(const svdc_attention* p, bool q_span, bool k_span) {
  if (!p) return SVDC_E_NULL;
  if (!plain_dtype(p->dtype)) return SVDC_E_DTYPE;
  if (!(p->scale > 0.f && p->scale <= 1e38f) || p->reserved != 0) return SVDC_E_PARAM;
  if (p->batch > 65535 || p->q_rows > kMaxAttentionRows || p->k_rows > kMaxAttentionRows || !batch_rows_ok(p->batch, p->q_rows) || !batch_rows_ok(p->batch, p->k_rows) || p->heads < 1 || p->heads > kMaxHeads || p->kv_heads < 1 ||
      p->heads % p->kv_heads != 0 || p->head_dim < 1 || p->head_dim > kMaxHeadDim)
    return SVDC_E_SHAPE;
  // units of work, each at most 64 workgroups
  if (p->batch * p->heads * ((p->q_rows + 127) / 128) > (1 << 23)) return SVDC_E_SHAPE;
  if (q_span && (p->q_total < 0 || p->q_total > INT32_MAX)) return SVDC_E_SHAPE;
  if (k_span && (p->k_total < 0 || p->k_total > INT32_MAX)) return SVDC_E_SHAPE;
  if (!heads_ok(p->q, !q_span) || !heads_ok(p->o, !q_span) || !heads_ok(p->k, !k_span) || !heads_ok(p->v, !k_span)) return SVDC_E_SHAPE;
  return SVDC_OK;
}

constexpr int kMaxDevices = 64;
void* g_scratch_ptr[kMaxDevices];   // device address of `scratch` on each device, resolved on first use
std::mutex g_scratch_mutex;

// Address of the current device's copy of `scratch` (looked up once per device, with that device current).
int32_t static_scratch(void** out) {
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= kMaxDevices) return SVDC_E_HIP;
  std::lock_guard<std::mutex> lock(g_scratch_mutex);
  if (!g_scratch_ptr[dev]) {
    void* p = nullptr;
    if (hipGetSymbolAddress(&p, HIP_SYMBOL(scratch)) != hipSuccess || !p) return SVDC_E_HIP;
    g_scratch_ptr[dev] = p;
  }
  *out = g_scratch_ptr[dev];
  return SVDC_OK;
}

__global__ void copy_status_kernel(const int32_t* __restrict__ src, int32_t* __restrict__ dst, int n) {
  const int i = blockIdx.x * blockDim.x + threadIdx.x;
  if (i < n) dst[i] = src[i];
}

}  // namespace

extern "C" {

int32_t svdcache_version(void) { return 500; }   // 0.5.0: operators around a block's attention

const char* svdcache_strerror(int32_t status) {
  switch (status) {
    case SVDC_OK: return "ok";
    case SVDC_E_NULL: return "a required pointer is NULL";
    case SVDC_E_SHAPE: return "shape, stride or rank out of the supported range";
    case SVDC_E_DTYPE: return "unknown dtype";
    case SVDC_E_ALIGN: return "pointer or stride not aligned as documented";
    case SVDC_E_PARAM: return "parameter out of range";
    case SVDC_E_WORKSPACE: return "workspace or packed-basis buffer too small";
    case SVDC_E_HIP: return "HIP runtime call or kernel launch failed";
    default: return "unknown status";
  }
}

size_t svdcache_fit_workspace_bytes(const svdc_shape* shape, const svdc_fit_params* params) {
  FitPlan plan;
  if (check_shape(shape) != SVDC_OK || !make_fit_plan(*shape, params, &plan)) return 0;
  return plan.total;
}

size_t svdcache_workspace_bytes(const svdc_shape* shape, const svdc_fit_params* params) {
  return svdcache_fit_workspace_bytes(shape, params);
}

size_t svdcache_fit_status_offset(const svdc_shape* shape, const svdc_fit_params* params) {
  FitPlan plan;
  if (check_shape(shape) != SVDC_OK || !make_fit_plan(*shape, params, &plan)) return 0;
  return plan.off_info;
}

size_t svdcache_packed_basis_bytes(const svdc_shape* shape) {
  if (check_shape(shape) != SVDC_OK || !mfma_shape_supported(*shape)) return 0;
  return mfma_packed_bytes(*shape);
}

int32_t svdcache_has_mfma_path(const svdc_shape* shape) {
  return check_shape(shape) == SVDC_OK && mfma_shape_supported(*shape) ? 1 : 0;
}

int32_t svdcache_fit_basis(const svdc_shape* shape, const svdc_fit_params* params, const void* F, float* V,
                           float* sigma, float* fro2, void* workspace, size_t workspace_bytes, void* stream) {
  int32_t rc = check_shape(shape);
  if (rc != SVDC_OK) return rc;
  if (!F || !V || !sigma || !workspace) return SVDC_E_NULL;
  if (!aligned(F, 16) || !aligned(V, 16) || !aligned(workspace, 256)) return SVDC_E_ALIGN;
  FitPlan plan;
  if (shape->k > 256) return SVDC_E_SHAPE;
  if (!make_fit_plan(*shape, params, &plan)) return SVDC_E_PARAM;
  if (workspace_bytes < plan.total) return SVDC_E_WORKSPACE;
  return run_fit(*shape, plan, F, V, sigma, fro2, workspace, (hipStream_t)stream);
}

int32_t svdcache_fit_basis_static(const svdc_shape* shape, const svdc_fit_params* params, const void* F, float* V,
                                  float* sigma, float* fro2, int32_t* status, void* stream) {
  int32_t rc = check_shape(shape);
  if (rc != SVDC_OK) return rc;
  if (!F || !V || !sigma) return SVDC_E_NULL;
  if (!aligned(F, 16) || !aligned(V, 16) || (status && !aligned(status, 4))) return SVDC_E_ALIGN;
  FitPlan plan;
  if (shape->k > 256) return SVDC_E_SHAPE;
  if (!make_fit_plan(*shape, params, &plan)) return SVDC_E_PARAM;
  if (plan.total > (size_t)SVDC_STATIC_SCRATCH_BYTES) return SVDC_E_WORKSPACE;
  void* ws = nullptr;
  rc = static_scratch(&ws);
  if (rc != SVDC_OK) return rc;
  // the fit clears what must start at zero (accumulators, status words) with fill kernels of its own
  rc = run_fit(*shape, plan, F, V, sigma, fro2, ws, (hipStream_t)stream);
  if (rc != SVDC_OK || !status) return rc;
  copy_status_kernel<<<(shape->B + 255) / 256, 256, 0, (hipStream_t)stream>>>(
      reinterpret_cast<const int32_t*>(static_cast<const char*>(ws) + plan.off_info), status, shape->B);
  return launch_status();
}

int32_t svdcache_pack_basis(const svdc_shape* shape, const float* V, void* packed, size_t packed_bytes,
                            void* stream) {
  int32_t rc = check_shape(shape);
  if (rc != SVDC_OK) return rc;
  if (!V || !packed) return SVDC_E_NULL;
  if (!mfma_shape_supported(*shape)) return SVDC_E_SHAPE;
  if (!aligned(V, 16) || !aligned(packed, 256)) return SVDC_E_ALIGN;
  if (packed_bytes < mfma_packed_bytes(*shape)) return SVDC_E_WORKSPACE;
  return launch_pack_basis(*shape, V, packed, (hipStream_t)stream);
}

int32_t svdcache_full_step(const svdc_shape* shape, const void* F, const float* V, const void* packed, void* R,
                           float* S, float* C, float alpha, int32_t init, void* stream) {
  int32_t rc = check_shape(shape);
  if (rc != SVDC_OK) return rc;
  if (!F || !V || !R || !S) return SVDC_E_NULL;
  if (!(alpha > 0.f && alpha <= 1.f)) return SVDC_E_PARAM;
  if (!aligned(F, 16) || !aligned(R, 16) || !aligned(V, 16) || !aligned(S, 16) || (C && !aligned(C, 16)))
    return SVDC_E_ALIGN;
  if (packed && mfma_shape_supported(*shape)) {
    if (!aligned(packed, 256)) return SVDC_E_ALIGN;
    return launch_full_step_mfma(*shape, F, packed, R, S, C, alpha, init != 0, ResidualEma{}, (hipStream_t)stream);
  }
  return launch_full_step_general(*shape, F, V, R, S, C, alpha, init != 0, ResidualEma{}, (hipStream_t)stream);
}

int32_t svdcache_full_step_residual_ema(const svdc_shape* shape, const void* F, const float* V, const void* packed,
                                        const void* R_prev, void* R, float* S, float* C, float alpha,
                                        float alpha_r, int32_t init, void* stream) {
  int32_t rc = check_shape(shape);
  if (rc != SVDC_OK) return rc;
  if (!F || !V || !R || !S) return SVDC_E_NULL;
  if (!(alpha > 0.f && alpha <= 1.f) || !(alpha_r > 0.f && alpha_r <= 1.f)) return SVDC_E_PARAM;
  ResidualEma re;
  if (init == 0 && alpha_r < 1.f) {
    if (!R_prev) return SVDC_E_NULL;
    // the previous residual is read while the new one is written: it may be the output buffer (updated in
    // place) but then the output cannot also be the feature buffer
    if (R_prev == F) return SVDC_E_PARAM;
    if (!aligned(R_prev, 16)) return SVDC_E_ALIGN;
    re.prev = R_prev;
    re.alpha_r = alpha_r;
  }
  if (!aligned(F, 16) || !aligned(R, 16) || !aligned(V, 16) || !aligned(S, 16) || (C && !aligned(C, 16)))
    return SVDC_E_ALIGN;
  if (packed && mfma_shape_supported(*shape)) {
    if (!aligned(packed, 256)) return SVDC_E_ALIGN;
    return launch_full_step_mfma(*shape, F, packed, R, S, C, alpha, init != 0, re, (hipStream_t)stream);
  }
  return launch_full_step_general(*shape, F, V, R, S, C, alpha, init != 0, re, (hipStream_t)stream);
}

int32_t svdcache_forecast(const svdc_shape* shape, const float* S, const float* V, const void* packed,
                          const void* R, void* Fhat, void* stream) {
  int32_t rc = check_shape(shape);
  if (rc != SVDC_OK) return rc;
  if (!S || !V || !R || !Fhat) return SVDC_E_NULL;
  if (!aligned(R, 16) || !aligned(Fhat, 16) || !aligned(V, 16) || !aligned(S, 16)) return SVDC_E_ALIGN;
  if (packed && mfma_shape_supported(*shape)) {
    if (!aligned(packed, 256)) return SVDC_E_ALIGN;
    return launch_forecast_mfma(*shape, S, packed, R, Fhat, (hipStream_t)stream);
  }
  CoefStates cs{};
  cs.s[0] = S;
  cs.w[0] = 1.f;
  cs.m = 1;
  return launch_forecast_general(*shape, cs, V, R, nullptr, Fhat, (hipStream_t)stream);
}

size_t svdcache_packed_state_bytes(const svdc_shape* shape) {
  if (check_shape(shape) != SVDC_OK || !mfma_shape_supported(*shape)) return 0;
  return mfma_packed_state_bytes(*shape);
}

int32_t svdcache_pack_state(const svdc_shape* shape, const float* S, void* S_packed, size_t S_packed_bytes,
                            void* stream) {
  int32_t rc = check_shape(shape);
  if (rc != SVDC_OK) return rc;
  if (!S || !S_packed) return SVDC_E_NULL;
  if (!mfma_shape_supported(*shape)) return SVDC_E_SHAPE;
  if (!aligned(S, 16) || !aligned(S_packed, 256)) return SVDC_E_ALIGN;
  if (S_packed_bytes < mfma_packed_state_bytes(*shape)) return SVDC_E_WORKSPACE;
  return launch_pack_state(*shape, S, S_packed, (hipStream_t)stream);
}

int32_t svdcache_full_step_packed(const svdc_shape* shape, const void* F, const float* V, const void* packed, void* R,
                                  float* S, float* C, void* S_packed, size_t S_packed_bytes, float alpha,
                                  int32_t init, void* stream) {
  int32_t rc = check_shape(shape);
  if (rc != SVDC_OK) return rc;
  if (!F || !V || !R || !S || !packed || !S_packed) return SVDC_E_NULL;
  if (!(alpha > 0.f && alpha <= 1.f)) return SVDC_E_PARAM;
  if (!mfma_shape_supported(*shape)) return SVDC_E_SHAPE;
  if (!aligned(F, 16) || !aligned(R, 16) || !aligned(V, 16) || !aligned(S, 16) || (C && !aligned(C, 16)) ||
      !aligned(packed, 256) || !aligned(S_packed, 256))
    return SVDC_E_ALIGN;
  if (S_packed_bytes < mfma_packed_state_bytes(*shape)) return SVDC_E_WORKSPACE;
  ResidualEma re;
  re.packed_state = S_packed;
  return launch_full_step_mfma(*shape, F, packed, R, S, C, alpha, init != 0, re, (hipStream_t)stream);
}

int32_t svdcache_forecast_packed(const svdc_shape* shape, const void* S_packed, const void* packed, const void* R,
                                 void* Fhat, void* stream) {
  int32_t rc = check_shape(shape);
  if (rc != SVDC_OK) return rc;
  if (!S_packed || !packed || !R || !Fhat) return SVDC_E_NULL;
  if (!mfma_shape_supported(*shape)) return SVDC_E_SHAPE;
  if (!aligned(R, 16) || !aligned(Fhat, 16) || !aligned(packed, 256) || !aligned(S_packed, 256)) return SVDC_E_ALIGN;
  return launch_forecast_packed_mfma(*shape, S_packed, packed, R, Fhat, (hipStream_t)stream);
}

int32_t svdcache_select_rank(int32_t B, int32_t k, const float* sigma, const float* fro2, float tau,
                             int32_t* k_star, int32_t* reached, void* stream) {
  if (!sigma || !fro2 || !k_star) return SVDC_E_NULL;
  if (B < 1 || k < 1 || k > 1024) return SVDC_E_SHAPE;
  if (!(tau > 0.f && tau <= 1.f)) return SVDC_E_PARAM;
  return launch_select_rank(B, k, sigma, fro2, tau, k_star, reached, (hipStream_t)stream);
}

int32_t svdcache_truncate_basis(const svdc_shape* shape, float* V, float* sigma, const int32_t* k_star,
                                void* stream) {
  int32_t rc = check_shape(shape);
  if (rc != SVDC_OK) return rc;
  if (!V || !k_star) return SVDC_E_NULL;
  return launch_truncate_basis(*shape, V, sigma, k_star, (hipStream_t)stream);
}

int32_t svdcache_extrapolation_weights(int32_t order, double offset, double interval, float* weights) {
  if (!weights) return SVDC_E_NULL;
  const auto finite = [](double v) { return v - v == 0.0; };   // false for NaN and for +-inf
  if (order < 0 || order >= SVDC_MAX_STATES || interval == 0.0 || !finite(interval) || !finite(offset))
    return SVDC_E_PARAM;
  // Lagrange weights at x = offset / interval for the nodes 0, -1, ..., -order
  const double x = offset / interval;
  for (int m = 0; m <= order; ++m) {
    double w = 1.0;
    for (int i = 0; i <= order; ++i)
      if (i != m) w *= (x + i) / (double)(i - m);
    weights[m] = (float)w;
  }
  return SVDC_OK;
}

int32_t svdcache_forecast_combine(const svdc_shape* shape, int32_t num_states, const float* const* S_list,
                                  const float* weights, const float* V, const void* packed, const void* R,
                                  const void* X, void* Out, void* stream) {
  int32_t rc = check_shape(shape);
  if (rc != SVDC_OK) return rc;
  if (!S_list || !weights || !V || !R || !Out) return SVDC_E_NULL;
  if (num_states < 1 || num_states > SVDC_MAX_STATES) return SVDC_E_PARAM;
  CoefStates cs{};
  cs.m = num_states;
  for (int m = 0; m < num_states; ++m) {
    if (!S_list[m]) return SVDC_E_NULL;
    if (!aligned(S_list[m], 16)) return SVDC_E_ALIGN;
    if (!(weights[m] == weights[m])) return SVDC_E_PARAM;   // NaN
    cs.s[m] = S_list[m];
    cs.w[m] = weights[m];
  }
  if (!aligned(R, 16) || !aligned(Out, 16) || !aligned(V, 16) || (X && !aligned(X, 16))) return SVDC_E_ALIGN;
  if (packed && mfma_shape_supported(*shape)) {
    if (!aligned(packed, 256)) return SVDC_E_ALIGN;
    return launch_forecast_combine_mfma(*shape, cs, packed, R, X, Out, (hipStream_t)stream);
  }
  return launch_forecast_general(*shape, cs, V, R, X, Out, (hipStream_t)stream);
}

int32_t svdcache_basis_overlap(const svdc_shape* shape, const float* V_old, const float* V_new, float* M,
                               void* stream) {
  int32_t rc = check_shape(shape);
  if (rc != SVDC_OK) return rc;
  if (!V_old || !V_new || !M) return SVDC_E_NULL;
  if (!rebase_rank_supported(shape->k)) return SVDC_E_SHAPE;
  return launch_basis_overlap(*shape, V_old, V_new, M, (hipStream_t)stream);
}

int32_t svdcache_rebase_state(const svdc_shape* shape, const float* M, const float* S_in, float* S_out,
                              void* stream) {
  int32_t rc = check_shape(shape);
  if (rc != SVDC_OK) return rc;
  if (!M || !S_in || !S_out) return SVDC_E_NULL;
  if (!rebase_rank_supported(shape->k)) return SVDC_E_SHAPE;
  return launch_rebase_state(*shape, M, S_in, S_out, (hipStream_t)stream);
}

int32_t svdcache_basis_similarity(const svdc_shape* shape, const float* V_a, const float* sigma_a,
                                  const float* V_b, const float* sigma_b, float* sim_dir, float* sim_sigma,
                                  void* stream) {
  int32_t rc = check_shape(shape);
  if (rc != SVDC_OK) return rc;
  if (!V_a || !V_b || !sim_dir) return SVDC_E_NULL;
  if (sim_sigma && (!sigma_a || !sigma_b)) return SVDC_E_NULL;
  return launch_basis_similarity(*shape, V_a, sigma_a, V_b, sigma_b, sim_dir, sim_sigma, (hipStream_t)stream);
}

size_t svdcache_q8_bytes(int64_t rows, int32_t D) {
  return rows8_ok(rows, D) ? (size_t)(rows * q8_row_bytes(D)) : 0;
}

size_t svdcache_q8_scale_bytes(int64_t rows, int32_t D, int32_t block_rows) {
  if (!rows8_ok(rows, D) || (block_rows != 1 && block_rows != kScaleBlock)) return 0;
  return (size_t)((rows + block_rows - 1) / block_rows * q8_scale_row_bytes(D));
}

int32_t svdcache_rms_norm8(const svdc_norm8* p, const void* X, const void* F, const float* gain, void* H, void* Y, void* Q, void* scales,
                           void* stream) {
  if (!p) return SVDC_E_NULL;
  if (!plain_dtype(p->dtype) || (F && !plain_dtype(p->dtype_f))) return SVDC_E_DTYPE;
  if (!(p->eps >= 0.f && p->eps <= 3.402823466e38f)) return SVDC_E_PARAM;
  if (!rows8_ok(p->rows, p->D) || !stride8_ok(p->rows, p->D, p->ldx) || (F && !stride8_ok(p->rows, p->D, p->ldf)) ||
      (H && !stride8_ok(p->rows, p->D, p->ldh)) || (Y && !stride8_ok(p->rows, p->D, p->ldy)))
    return SVDC_E_SHAPE;
  if (p->rows == 0) return SVDC_OK;
  if (!X || (!Y && !Q) || (Q == nullptr) != (scales == nullptr)) return SVDC_E_NULL;
  const size_t unit = dtype_size(p->dtype);
  if (!aligned(X, unit) || (F && !aligned(F, dtype_size(p->dtype_f))) || (gain && !aligned(gain, 4)) || (H && !aligned(H, unit)) ||
      (Y && !aligned(Y, unit)) || (Q && !aligned(Q, 16)) || (scales && !aligned(scales, 4)))
    return SVDC_E_ALIGN;
  // a row is written where another one is still read, if the buffers are the same and the strides are not
  if (H && ((H == X && p->ldh != p->ldx) || (F && H == F && (p->ldh != p->ldf || p->dtype != p->dtype_f)))) return SVDC_E_PARAM;
  if (Y && (Y == X || Y == F || Y == H)) return SVDC_E_PARAM;
  return launch_rms_norm8(*p, X, F, gain, H, Y, Q, scales, (hipStream_t)stream);
}

int32_t svdcache_quantize8(const svdc_quant8* p, const void* X, void* Q, void* scales, void* stream) {
  if (!p) return SVDC_E_NULL;
  if (!plain_dtype(p->dtype)) return SVDC_E_DTYPE;
  if ((p->block_rows != 1 && p->block_rows != kScaleBlock) || p->reserved != 0) return SVDC_E_PARAM;
  if (!rows8_ok(p->rows, p->D) || !stride8_ok(p->rows, p->D, p->ldx)) return SVDC_E_SHAPE;
  if (p->rows == 0) return SVDC_OK;
  if (!X || !Q || !scales) return SVDC_E_NULL;
  if (!aligned(X, dtype_size(p->dtype)) || !aligned(Q, 16) || !aligned(scales, 4)) return SVDC_E_ALIGN;
  return launch_quantize8(*p, X, Q, scales, (hipStream_t)stream);
}

size_t svdcache_matmul8_workspace_bytes(const svdc_matmul8* p) { return check_matmul8(p) == SVDC_OK ? matmul8_workspace_bytes(*p) : 0; }

int32_t svdcache_matmul8(const svdc_matmul8* p, const void* A, const void* A_scales, const void* W, const void* W_scales, const float* bias,
                         void* Out, void* Out_scales, void* workspace, size_t workspace_bytes, void* stream) {
  const int32_t rc = check_matmul8(p);
  if (rc != SVDC_OK) return rc;
  if (p->M == 0) return SVDC_OK;
  if (!A || !A_scales || !W || !W_scales || !Out || (p->dtype == SVDC_E4M3 && !Out_scales)) return SVDC_E_NULL;
  if (!aligned(A, 16) || !aligned(A_scales, 4) || !aligned(W, 16) || !aligned(W_scales, 4) || (bias && !aligned(bias, 4)) ||
      !aligned(Out, p->dtype == SVDC_E4M3 ? 16 : dtype_size(p->dtype)) || (p->dtype == SVDC_E4M3 && !aligned(Out_scales, 4)))
    return SVDC_E_ALIGN;
  const size_t need = matmul8_workspace_bytes(*p);
  if (need && !workspace) return SVDC_E_NULL;
  if (need && !aligned(workspace, 256)) return SVDC_E_ALIGN;
  if (need > workspace_bytes) return SVDC_E_WORKSPACE;
  return launch_matmul8(*p, A, A_scales, W, W_scales, bias, Out, Out_scales, need ? workspace : nullptr, (hipStream_t)stream);
}

int32_t svdcache_rotary_table(const svdc_rotary* p, const void* pos, float* table, void* stream) {
  if (!p) return SVDC_E_NULL;
  if (p->rows < 0 || p->rows > INT32_MAX || p->axes < 1 || p->axes > SVDC_MAX_AXES || p->ld < p->axes || p->ld > (1 << 24)) return SVDC_E_SHAPE;
  if (p->whole != 0 && p->whole != 1) return SVDC_E_PARAM;
  int64_t columns = 0;
  for (int a = 0; a < p->axes; ++a) {
    if (p->dims[a] < 2 || p->dims[a] % 2 || p->dims[a] > 2 * kMaxTurned) return SVDC_E_SHAPE;
    if (!(p->theta[a] > 0.0 && p->theta[a] <= 1.7976931348623157e308)) return SVDC_E_PARAM;
    columns += p->dims[a];
  }
  if (columns > 2 * kMaxTurned) return SVDC_E_SHAPE;
  if (p->rows == 0) return SVDC_OK;
  if (!pos || !table) return SVDC_E_NULL;
  if (!aligned(pos, 4) || !aligned(table, 8)) return SVDC_E_ALIGN;
  return launch_rotary_table(*p, pos, table, (hipStream_t)stream);
}

int32_t svdcache_norm_rotate(const svdc_norm_rotate* p, const void* Q, const void* K, const void* V, const float* gain_q, const float* gain_k,
                             const float* table, void* Qo, void* Ko, void* Vo, void* stream) {
  if (!p) return SVDC_E_NULL;
  if (!plain_dtype(p->dtype) || !plain_dtype(p->dtype_out)) return SVDC_E_DTYPE;
  if (!(p->eps >= 0.f && p->eps <= 3.402823466e38f) || (p->norm != 0 && p->norm != 1) || p->reserved != 0 ||
      (p->layout != SVDC_PAIRS_NEIGHBOURS && p->layout != SVDC_PAIRS_HALVES))
    return SVDC_E_PARAM;
  if (!batch_rows_ok(p->batch, p->rows) || p->heads < 1 || p->heads > kMaxHeads || p->kv_heads < 1 || p->kv_heads > kMaxHeads || p->head_dim < 1 ||
      p->head_dim > kMaxHeadDim || p->pairs < 0 || 2 * p->pairs > p->head_dim || p->table_seq < 0 || p->table_seq > kMaxStride)
    return SVDC_E_SHAPE;
  if ((Q && (!heads_ok(p->q) || !heads_ok(p->qo))) || (K && (!heads_ok(p->k) || !heads_ok(p->ko))) || (V && (!heads_ok(p->v) || !heads_ok(p->vo)))) return SVDC_E_SHAPE;
  if (p->batch == 0 || p->rows == 0) return SVDC_OK;
  if ((!Q && !K && !V) || (Q == nullptr) != (Qo == nullptr) || (K == nullptr) != (Ko == nullptr) || (V == nullptr) != (Vo == nullptr) || (p->pairs && (Q || K) && !table))
    return SVDC_E_NULL;
  const size_t in = dtype_size(p->dtype), out = dtype_size(p->dtype_out);
  if (!aligned(Q, in) || !aligned(K, in) || !aligned(V, in) || !aligned(Qo, out) || !aligned(Ko, out) || !aligned(Vo, out) || (p->pairs && !aligned(table, 8)) ||
      (p->norm && (!aligned(gain_q, 4) || !aligned(gain_k, 4))))
    return SVDC_E_ALIGN;
  // in place: a head is written where it was read
  const bool types = p->dtype == p->dtype_out;
  if ((Q && Qo == Q && !(types && same_heads(p->q, p->qo))) || (K && Ko == K && !(types && same_heads(p->k, p->ko))) || (V && Vo == V && !(types && same_heads(p->v, p->vo))))
    return SVDC_E_PARAM;
  // one buffer for two of the outputs, or one that is another's input
  if ((Qo && (Qo == Ko || Qo == Vo || Qo == K || Qo == V)) || (Ko && (Ko == Vo || Ko == Q || Ko == V)) || (Vo && (Vo == Q || Vo == K))) return SVDC_E_PARAM;
  return launch_norm_rotate(*p, Q, K, V, gain_q, gain_k, table, Qo, Ko, Vo, (hipStream_t)stream);
}

size_t svdcache_attention_workspace_bytes(const svdc_attention* p) {
  // valid for a call with some of the spans: what that call does not read may hold anything
  for (const bool q_span : {false, true})
    for (const bool k_span : {false, true})
      if (check_attention(p, q_span, k_span) == SVDC_OK) return attention_workspace_bytes(*p);
  return 0;
}

int32_t svdcache_attention(const svdc_attention* p, const void* Q, const void* K, const void* V, const int32_t* q_span, const int32_t* k_span,
                           const uint8_t* key_mask, void* Out, void* workspace, size_t workspace_bytes, void* stream) {
  const int32_t rc = check_attention(p, q_span != nullptr, k_span != nullptr);
  if (rc != SVDC_OK) return rc;
  if (p->batch == 0 || p->q_rows == 0 || (q_span && p->q_total == 0)) return SVDC_OK;
  const bool keys = p->k_rows && !(k_span && p->k_total == 0);   // else results are zeros
  if (!Q || !Out || (keys && (!K || !V))) return SVDC_E_NULL;
  const size_t unit = dtype_size(p->dtype);
  if (!aligned(Q, unit) || !aligned(K, unit) || !aligned(V, unit) || !aligned(Out, unit) || !aligned(q_span, 8) || !aligned(k_span, 8)) return SVDC_E_ALIGN;
  if (Out == Q || (keys && (Out == K || Out == V))) return SVDC_E_PARAM;
  const size_t need = attention_workspace_bytes(*p);
  if (need && !workspace) return SVDC_E_NULL;
  if (need && !aligned(workspace, 256)) return SVDC_E_ALIGN;
  if (need > workspace_bytes) return SVDC_E_WORKSPACE;
  return launch_attention(*p, Q, K, V, q_span, k_span, key_mask, Out, need ? workspace : nullptr, (hipStream_t)stream);
}

}  // extern "C"
