// C ABI of the operators of a transformer block: argument checks and launches.
// The kernels are in k_norm.hip, k_attention.hip and k_dropout.hip;
// dbw_group_linear is in lm_api.cpp, beside the product it extends.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "dbw.h"
#include "dbw_internal.h"
#include "lm_ops.h"

#define DBW_API extern "C" __attribute__((visibility("default")))

using dbw::aligned;
using dbw::set_free_error;

namespace {

constexpr int64_t kMostRows = int64_t{1} << 31;
constexpr int64_t kMostStride = int64_t{1} << 32;

bool known(int32_t dtype) { return dtype == DBW_F32 || dtype == DBW_BF16 || dtype == DBW_F16; }

// What the calls over [T] rows have in common.
dbw_status check_rows(const char* call, int32_t n, int64_t T, int32_t d, int32_t most_d, int32_t dtype,
                      const int32_t* offsets) {
  if (n < 1 || n > DBW_MAX_N) return set_free_error(DBW_EINVAL, "%s: n=%d outside [1, %d]", call, n, DBW_MAX_N);
  if (T < 0 || T >= kMostRows) return set_free_error(DBW_EINVAL, "%s: T=%lld outside [0, 2^31)", call, (long long)T);
  if (d < 1) return set_free_error(DBW_EINVAL, "%s: %d columns", call, d);
  if (d > most_d) return set_free_error(DBW_EUNSUPPORTED, "%s: %d columns, at most %d", call, d, most_d);
  if (!known(dtype)) return set_free_error(DBW_EINVAL, "%s: unknown dtype %d", call, dtype);
  if (!offsets) return set_free_error(DBW_EINVAL, "%s: a device pointer is NULL", call);
  if (!aligned(offsets, 4)) return set_free_error(DBW_EINVAL, "%s: a pointer is not aligned to its elements", call);
  return DBW_OK;
}

// An array of T rows of d values.
struct Rows {
  const void* p;
  int64_t ld;
  bool needed;
};
dbw_status check_array(const char* call, const Rows& r, int64_t T, int32_t d, size_t bytes) {
  if (!r.p) return r.needed && T > 0 ? set_free_error(DBW_EINVAL, "%s: a device pointer is NULL", call) : DBW_OK;
  if (!aligned(r.p, bytes)) return set_free_error(DBW_EINVAL, "%s: a pointer is not aligned to its elements", call);
  if (r.ld < d) return set_free_error(DBW_EINVAL, "%s: a row stride is below its row", call);
  if (r.ld >= kMostStride) return set_free_error(DBW_EUNSUPPORTED, "%s: a row stride reaches 2^32", call);
  return DBW_OK;
}

dbw_status check_workspace(const char* call, int64_t need, const void* workspace, int64_t given) {
  if (need > 0 && (!workspace || given < need || !aligned(workspace, 16)))
    return set_free_error(DBW_EINVAL, "%s: needs %lld bytes of workspace, 16-byte aligned (%lld given)", call,
                          (long long)need, (long long)given);
  return DBW_OK;
}

dbw_status launched(const char* call, hipError_t e) {
  return e == hipSuccess ? DBW_OK : set_free_error(DBW_EHIP, "%s: launch failed: %s", call, hipGetErrorString(e));
}

dbw_status overlap(const char* call) {
  return set_free_error(DBW_EINVAL, "%s: an output must not overlap another array", call);
}

bool good_eps(double eps) { return eps >= 1e-30 && eps <= 1e30; }

}  // namespace

// ---------------------------------------------------------------------------
DBW_API dbw_status dbw_layer_norm(int32_t n, int64_t T, int32_t d, int32_t dtype, const int32_t* offsets, const void* X,
                                  int64_t ld_X, const float* gamma, const float* beta, double eps, void* Y,
                                  int64_t ld_Y, void* stream) {
  const char* call = "dbw_layer_norm";
  if (dbw_status s = check_rows(call, n, T, d, dbw::kNormMost, dtype, offsets); s != DBW_OK) return s;
  const size_t e = dbw::elem_bytes(dtype);
  for (const Rows& r : {Rows{X, ld_X, true}, Rows{Y, ld_Y, true}})
    if (dbw_status s = check_array(call, r, T, d, e); s != DBW_OK) return s;
  if (!gamma || !aligned(gamma, 4) || !aligned(beta, 4))
    return set_free_error(DBW_EINVAL, "%s: gamma is NULL, or a pointer is not aligned to its elements", call);
  if (!good_eps(eps)) return set_free_error(DBW_EINVAL, "%s: eps lies in [1e-30, 1e30]", call);
  if (Y && (Y == X || Y == gamma || Y == beta || Y == offsets)) return overlap(call);
  dbw::NormArgs a{};
  a.n = n; a.d = d; a.T = T; a.dtype = dtype; a.offsets = offsets; a.X = X; a.ld_X = ld_X;
  a.gamma = gamma; a.beta = beta; a.eps = static_cast<float>(eps); a.out = Y; a.ld_out = ld_Y;
  return launched(call, dbw::launch_layer_norm(a, static_cast<hipStream_t>(stream)));
}

DBW_API int64_t dbw_layer_norm_workspace(int32_t n, int64_t T, int32_t d) {
  if (n < 1 || n > DBW_MAX_N || T < 0 || T >= kMostRows || d < 1 || d > dbw::kNormMost) return -1;
  return dbw::norm_workspace(n, T, d);
}

DBW_API dbw_status dbw_layer_norm_grad(int32_t n, int64_t T, int32_t d, int32_t dtype, const int32_t* offsets,
                                       const void* dY, int64_t ld_dY, const void* X, int64_t ld_X, const float* gamma,
                                       double eps, void* dX, int64_t ld_dX, float* dgamma, int64_t ld_dgamma,
                                       float* dbeta, int64_t ld_dbeta, void* workspace, int64_t workspace_bytes,
                                       void* stream) {
  const char* call = "dbw_layer_norm_grad";
  if (dbw_status s = check_rows(call, n, T, d, dbw::kNormMost, dtype, offsets); s != DBW_OK) return s;
  const size_t e = dbw::elem_bytes(dtype);
  for (const Rows& r : {Rows{dY, ld_dY, true}, Rows{X, ld_X, true}, Rows{dX, ld_dX, true}})
    if (dbw_status s = check_array(call, r, T, d, e); s != DBW_OK) return s;
  for (const Rows& r : {Rows{dgamma, ld_dgamma, false}, Rows{dbeta, ld_dbeta, false}})
    if (dbw_status s = check_array(call, r, T, d, 4); s != DBW_OK) return s;
  if (!gamma || !dgamma || !aligned(gamma, 4))
    return set_free_error(DBW_EINVAL, "%s: gamma or dgamma is NULL, or a pointer is not aligned to its elements", call);
  if (!good_eps(eps)) return set_free_error(DBW_EINVAL, "%s: eps lies in [1e-30, 1e30]", call);
  if (dX && (dX == dY || dX == X || dX == gamma || dX == dgamma || dX == dbeta || dX == offsets)) return overlap(call);
  for (const void* g : {static_cast<const void*>(dgamma), static_cast<const void*>(dbeta)})
    if (g && (g == dY || g == X || g == gamma || g == offsets)) return overlap(call);
  if (dgamma == dbeta) return overlap(call);
  if (dbw_status s = check_workspace(call, dbw::norm_workspace(n, T, d), workspace, workspace_bytes); s != DBW_OK)
    return s;
  dbw::NormArgs a{};
  a.n = n; a.d = d; a.T = T; a.dtype = dtype; a.offsets = offsets; a.dY = dY; a.ld_dY = ld_dY; a.X = X; a.ld_X = ld_X;
  a.gamma = gamma; a.eps = static_cast<float>(eps); a.out = dX; a.ld_out = ld_dX;
  a.dgamma = dgamma; a.ld_dgamma = ld_dgamma; a.dbeta = dbeta; a.ld_dbeta = ld_dbeta;
  a.parts = static_cast<float*>(workspace);
  return launched(call, dbw::launch_layer_norm_grad(a, static_cast<hipStream_t>(stream)));
}

// ---------------------------------------------------------------------------
DBW_API int64_t dbw_linear_grad_workspace(int32_t n, int64_t T, int32_t C) {
  if (n < 1 || n > DBW_MAX_N || T < 0 || T >= kMostRows || C < 1 || C > (1 << 20)) return -1;
  return dbw::linear_grad_workspace(n, T, C);
}

DBW_API dbw_status dbw_linear_grad(int32_t n, int64_t T, int32_t C, int32_t dtype, int32_t activation,
                                   const int32_t* offsets, const void* dY, int64_t ld_dY, const void* Z, int64_t ld_Z,
                                   void* dZ, int64_t ld_dZ, float* dbias, int64_t ld_dbias, void* workspace,
                                   int64_t workspace_bytes, void* stream) {
  const char* call = "dbw_linear_grad";
  if (dbw_status s = check_rows(call, n, T, C, 1 << 20, dtype, offsets); s != DBW_OK) return s;
  if (activation < DBW_ACT_NONE || activation > DBW_ACT_SILU)
    return set_free_error(DBW_EINVAL, "%s: unknown activation %d", call, activation);
  const bool acts = activation != DBW_ACT_NONE;
  const size_t e = dbw::elem_bytes(dtype);
  for (const Rows& r : {Rows{dY, ld_dY, true}, Rows{Z, ld_Z, acts}, Rows{dZ, ld_dZ, acts}})
    if (dbw_status s = check_array(call, r, T, C, e); s != DBW_OK) return s;
  if (dbw_status s = check_array(call, Rows{dbias, ld_dbias, false}, T, C, 4); s != DBW_OK) return s;
  if (!dZ && !dbias && T > 0) return set_free_error(DBW_EINVAL, "%s: neither dZ nor dbias is given", call);
  if (dZ && (dZ == dY || dZ == Z || dZ == dbias || dZ == offsets)) return overlap(call);
  if (dbias && (dbias == dY || dbias == Z || dbias == static_cast<const void*>(offsets))) return overlap(call);
  if (dbias)
    if (dbw_status s = check_workspace(call, dbw::linear_grad_workspace(n, T, C), workspace, workspace_bytes); s != DBW_OK)
      return s;
  dbw::LinearGradArgs a{};
  a.n = n; a.C = C; a.T = T; a.dtype = dtype; a.act = activation; a.offsets = offsets; a.dY = dY; a.ld_dY = ld_dY;
  a.Z = acts ? Z : nullptr; a.ld_Z = ld_Z; a.dZ = dZ; a.ld_dZ = ld_dZ; a.dbias = dbias; a.ld_dbias = ld_dbias;
  a.parts = static_cast<float*>(workspace);
  return launched(call, dbw::launch_linear_grad(a, static_cast<hipStream_t>(stream)));
}

// ---------------------------------------------------------------------------
DBW_API dbw_status dbw_dropout(int32_t n, int64_t T, int32_t d, int32_t dtype, const int32_t* offsets, const void* X,
                               int64_t ld_X, double p, uint64_t seed, const int64_t* step, const void* R, int64_t ld_R,
                               void* Y, int64_t ld_Y, void* stream) {
  const char* call = "dbw_dropout";
  if (dbw_status s = check_rows(call, n, T, d, 1 << 20, dtype, offsets); s != DBW_OK) return s;
  const size_t e = dbw::elem_bytes(dtype);
  for (const Rows& r : {Rows{X, ld_X, true}, Rows{R, ld_R, false}, Rows{Y, ld_Y, true}})
    if (dbw_status s = check_array(call, r, T, d, e); s != DBW_OK) return s;
  if (!(p >= 0.0 && p <= 1.0)) return set_free_error(DBW_EINVAL, "%s: p lies in [0, 1]", call);
  if (!aligned(step, 8)) return set_free_error(DBW_EINVAL, "%s: step is not aligned", call);
  if (Y && ((Y == X && ld_Y != ld_X) || (Y == R && ld_Y != ld_R)))
    return set_free_error(DBW_EINVAL, "%s: Y in the place of an input needs its row stride", call);
  if (Y && (Y == static_cast<const void*>(step) || Y == offsets)) return overlap(call);
  dbw::DropoutArgs a{};
  a.n = n; a.d = d; a.T = T; a.dtype = dtype; a.offsets = offsets; a.X = X; a.ld_X = ld_X; a.R = R; a.ld_R = ld_R;
  a.Y = Y; a.ld_Y = ld_Y; a.seed = seed; a.step = step;
  a.cut = static_cast<uint32_t>(std::nearbyint(65536.0 * p));
  a.scale = a.cut < 65536 ? static_cast<float>(65536.0 / (65536 - a.cut)) : 0.f;
  return launched(call, dbw::launch_dropout(a, static_cast<hipStream_t>(stream)));
}

DBW_API uint32_t dbw_dropout_bits(uint64_t seed, int64_t step, int64_t t, int32_t c) {
  uint32_t x[4] = {static_cast<uint32_t>(c) / 8, static_cast<uint32_t>(t), static_cast<uint32_t>(step),
                   static_cast<uint32_t>(static_cast<uint64_t>(step) >> 32)};
  dbw::lm_philox(x, static_cast<uint32_t>(seed), static_cast<uint32_t>(seed >> 32));
  const uint32_t k = static_cast<uint32_t>(c) % 8;
  return x[k / 2] >> (16 * (k % 2)) & 0xffffu;
}

// ---------------------------------------------------------------------------
namespace {

dbw_status check_attention(const char* call, const dbw_attention_shape* p) {
  if (!p) return set_free_error(DBW_EINVAL, "%s: shape is NULL", call);
  if (p->dtype == DBW_F32) return set_free_error(DBW_EUNSUPPORTED, "%s: arrays are bf16 or fp16, not fp32", call);
  if (p->dtype != DBW_BF16 && p->dtype != DBW_F16)
    return set_free_error(DBW_EINVAL, "%s: unknown dtype %d", call, p->dtype);
  if (p->n < 1 || p->n > 65536) return set_free_error(DBW_EINVAL, "%s: n=%d outside [1, 65536]", call, p->n);
  if (p->T < 0 || p->T >= kMostRows)
    return set_free_error(DBW_EINVAL, "%s: T=%lld outside [0, 2^31)", call, (long long)p->T);
  if (p->heads < 1 || p->kv_heads < 1 || p->heads % p->kv_heads)
    return set_free_error(DBW_EINVAL, "%s: heads=%d is not a multiple of kv_heads=%d", call, p->heads, p->kv_heads);
  if (p->heads > 1024) return set_free_error(DBW_EUNSUPPORTED, "%s: heads=%d above 1024", call, p->heads);
  if (p->D < 1) return set_free_error(DBW_EINVAL, "%s: D=%d < 1", call, p->D);
  if (p->D > 128 || p->D % 8) return set_free_error(DBW_EUNSUPPORTED, "%s: D=%d is not a multiple of 8 up to 128", call, p->D);
  if (!(p->scale >= 1e-20 && p->scale <= 1e20)) return set_free_error(DBW_EINVAL, "%s: scale lies in [1e-20, 1e20]", call);
  // (a launch holds fewer than 2^32 threads)
  if ((p->T / dbw::kAttentionKeys + p->n) * p->heads >= (int64_t{1} << 23))
    return set_free_error(DBW_EUNSUPPORTED, "%s: 2^23 tiles or more", call);
  return DBW_OK;
}

dbw_status check_heads(const char* call, const char* name, const dbw_heads* h, int64_t T, int32_t heads, int32_t D,
                       bool out) {
  if (!h) return set_free_error(DBW_EINVAL, "%s: %s is NULL", call, name);
  if (T == 0) return DBW_OK;
  if (!h->data) return set_free_error(DBW_EINVAL, "%s: %s: a device pointer is NULL", call, name);
  if (h->token < 0 || h->head < 0) return set_free_error(DBW_EINVAL, "%s: %s: a stride is below 0", call, name);
  if (!aligned(h->data, 16) || h->token % 8 || h->head % 8)
    return set_free_error(DBW_EUNSUPPORTED, "%s: %s: rows do not start at multiples of 16 bytes", call, name);
  if (h->token >= (int64_t{1} << 21) || h->head >= (int64_t{1} << 40))
    return set_free_error(DBW_EUNSUPPORTED, "%s: %s: a stride reaches 2^21 (tokens) or 2^40 (heads)", call, name);
  const bool heads_inside = (heads == 1 || h->head >= D) && (T == 1 || h->token >= (heads - 1) * h->head + D);
  const bool tokens_inside = (T == 1 || h->token >= D) && (heads == 1 || h->head >= (T - 1) * h->token + D);
  if (out && !heads_inside && !tokens_inside) return set_free_error(DBW_EINVAL, "%s: rows of %s overlap", call, name);
  return DBW_OK;
}

dbw::HeadRows rows_of(const dbw_heads& h) { return {static_cast<char*>(h.data), h.token, h.head}; }

dbw::AttentionArgs attention_args(const dbw_attention_shape& p, const int32_t* offsets) {
  dbw::AttentionArgs a{};
  a.n = p.n; a.heads = p.heads; a.kv_heads = p.kv_heads; a.D = p.D; a.T = p.T; a.dtype = p.dtype;
  a.scale = static_cast<float>(p.scale); a.offsets = offsets;
  return a;
}

}  // namespace

DBW_API dbw_status dbw_attention(const dbw_attention_shape* shape, const int32_t* offsets, const dbw_heads* Q,
                                 const dbw_heads* K, const dbw_heads* V, const dbw_heads* O, float* lse, void* stream) {
  const char* call = "dbw_attention";
  if (dbw_status s = check_attention(call, shape); s != DBW_OK) return s;
  const dbw_attention_shape& p = *shape;
  if (!offsets || !aligned(offsets, 4) || !aligned(lse, 4))
    return set_free_error(DBW_EINVAL, "%s: offsets is NULL, or a pointer is not aligned to its elements", call);
  if (dbw_status s = check_heads(call, "Q", Q, p.T, p.heads, p.D, false); s != DBW_OK) return s;
  if (dbw_status s = check_heads(call, "K", K, p.T, p.kv_heads, p.D, false); s != DBW_OK) return s;
  if (dbw_status s = check_heads(call, "V", V, p.T, p.kv_heads, p.D, false); s != DBW_OK) return s;
  if (dbw_status s = check_heads(call, "O", O, p.T, p.heads, p.D, true); s != DBW_OK) return s;
  if (p.T == 0) return DBW_OK;
  for (const dbw_heads* in : {Q, K, V})
    if (O->data == in->data || (lse && lse == in->data)) return overlap(call);
  if (O->data == offsets || (lse && (lse == O->data || lse == static_cast<const void*>(offsets)))) return overlap(call);
  dbw::AttentionArgs a = attention_args(p, offsets);
  a.Q = rows_of(*Q); a.K = rows_of(*K); a.V = rows_of(*V); a.O = rows_of(*O); a.lse = lse;
  return launched(call, dbw::launch_attention(a, static_cast<hipStream_t>(stream)));
}

namespace {
// delta, lse and maximum of every query; and the parts' sums
int64_t delta_bytes(const dbw_attention_shape& p) { return (int64_t{12} * p.heads * p.T + 15) / 16 * 16; }
int64_t sum_bytes(const dbw_attention_shape& p) {
  const int64_t parts = dbw::attention_parts(p.n, p.T, p.heads, p.kv_heads);
  return parts > 1 ? parts * 8 * p.T * p.kv_heads * p.D : 0;
}
}  // namespace

DBW_API int64_t dbw_attention_workspace(const dbw_attention_shape* shape) {
  if (check_attention("dbw_attention_workspace", shape) != DBW_OK) return -1;
  return delta_bytes(*shape) + sum_bytes(*shape);
}

DBW_API dbw_status dbw_attention_grad(const dbw_attention_shape* shape, const int32_t* offsets, const dbw_heads* dO,
                                      const dbw_heads* Q, const dbw_heads* K, const dbw_heads* V, const dbw_heads* O,
                                      const float* lse, const dbw_heads* dQ, const dbw_heads* dK, const dbw_heads* dV,
                                      void* workspace, int64_t workspace_bytes, void* stream) {
  const char* call = "dbw_attention_grad";
  if (dbw_status s = check_attention(call, shape); s != DBW_OK) return s;
  const dbw_attention_shape& p = *shape;
  if (!offsets || (!lse && p.T > 0) || !aligned(offsets, 4) || !aligned(lse, 4))
    return set_free_error(DBW_EINVAL, "%s: offsets or lse is NULL, or a pointer is not aligned to its elements", call);
  const struct {
    const char* name;
    const dbw_heads* h;
    int32_t heads;
    bool out;
  } arrays[] = {{"dO", dO, p.heads, false},  {"Q", Q, p.heads, false},  {"K", K, p.kv_heads, false},
                {"V", V, p.kv_heads, false}, {"O", O, p.heads, false},  {"dQ", dQ, p.heads, true},
                {"dK", dK, p.kv_heads, true}, {"dV", dV, p.kv_heads, true}};
  for (const auto& x : arrays)
    if (dbw_status s = check_heads(call, x.name, x.h, p.T, x.heads, p.D, x.out); s != DBW_OK) return s;
  if (p.T == 0) return DBW_OK;
  for (const auto& x : arrays)
    for (const auto& y : arrays)
      if (x.out && &x != &y && x.h->data == y.h->data) return overlap(call);
  for (const auto& x : arrays)
    if (x.out && (x.h->data == lse || x.h->data == offsets)) return overlap(call);
  if (dbw_status s = check_workspace(call, delta_bytes(p) + sum_bytes(p), workspace, workspace_bytes); s != DBW_OK) return s;
  dbw::AttentionArgs a = attention_args(p, offsets);
  a.Q = rows_of(*Q); a.K = rows_of(*K); a.V = rows_of(*V); a.O = rows_of(*O); a.dO = rows_of(*dO);
  a.dQ = rows_of(*dQ); a.dK = rows_of(*dK); a.dV = rows_of(*dV);
  a.lse = const_cast<float*>(lse); a.delta = static_cast<float*>(workspace);
  a.parts = dbw::attention_parts(p.n, p.T, p.heads, p.kv_heads);
  a.sums = reinterpret_cast<float*>(static_cast<char*>(workspace) + delta_bytes(p));
  return launched(call, dbw::launch_attention_grad(a, static_cast<hipStream_t>(stream)));
}
