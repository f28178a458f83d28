// C ABI of the products, the token loss and AdamW: argument checks, plans and
// launches.  The kernels are in k_group.hip, k_token.hip and k_adamw.hip.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <new>
#include <vector>

#include "dbw.h"
#include "dbw_internal.h"
#include "lm_ops.h"

#define DBW_API extern "C" __attribute__((visibility("default")))

using dbw::set_free_error;

namespace {

using dbw::aligned;

// Makes `dev` the current device for a scope.
struct OnDevice {
  int prev = -1;
  explicit OnDevice(int dev) {
    if (hipGetDevice(&prev) == hipSuccess && prev != dev) (void)hipSetDevice(dev);
    else prev = -1;
  }
  ~OnDevice() {
    if (prev >= 0) (void)hipSetDevice(prev);
  }
};

// ---------------------------------------------------------------------------
dbw_status check_shape(const dbw_group_shape* p, const char* call) {
  if (!p) return set_free_error(DBW_EINVAL, "%s: shape is NULL", call);
  if (p->form != DBW_GROUP_FORWARD && p->form != DBW_GROUP_INPUT_GRAD && p->form != DBW_GROUP_WEIGHT_GRAD)
    return set_free_error(DBW_EINVAL, "%s: unknown form %d", call, p->form);
  if (p->dtype == DBW_F32) return set_free_error(DBW_EUNSUPPORTED, "%s: inputs are bf16 or fp16, not fp32", call);
  if (p->dtype != DBW_BF16 && p->dtype != DBW_F16)
    return set_free_error(DBW_EINVAL, "%s: unknown dtype %d", call, p->dtype);
  if (p->out_dtype != p->dtype && p->out_dtype != DBW_F32)
    return set_free_error(DBW_EINVAL, "%s: the output has the inputs' type or fp32", call);
  if (p->n < 1 || p->n > DBW_MAX_N)
    return set_free_error(DBW_EINVAL, "%s: n=%d outside [1, %d]", call, p->n, DBW_MAX_N);
  if (p->d < 1 || p->C < 1) return set_free_error(DBW_EINVAL, "%s: d=%d or C=%d < 1", call, p->d, p->C);
  if (p->d > (1 << 20) || p->C > (1 << 20))
    return set_free_error(DBW_EUNSUPPORTED, "%s: d=%d or C=%d above 2^20", call, p->d, p->C);
  if (p->T < 0 || p->T >= (int64_t{1} << 31))
    return set_free_error(DBW_EINVAL, "%s: T=%lld outside [0, 2^31)", call, (long long)p->T);
  if (p->ld_d < p->d || p->ld_C < p->C || p->ld_W < p->C)
    return set_free_error(DBW_EINVAL, "%s: a row stride is below its row", call);
  const int64_t most = int64_t{1} << 21;
  if (p->ld_d >= most || p->ld_C >= most || p->ld_W >= most)
    return set_free_error(DBW_EUNSUPPORTED, "%s: a row stride reaches 2^21", call);
  const int64_t whole = (p->d - 1) * p->ld_W + p->C;   // elements of one W
  const bool shared = p->st_W == 0 && p->form != DBW_GROUP_WEIGHT_GRAD;
  if (p->n > 1 && !shared && p->st_W < whole)
    return set_free_error(DBW_EINVAL, "%s: W_%d would overlap W_0 (st_W=%lld)", call, 1, (long long)p->st_W);
  if (p->st_W >= (int64_t{1} << 40))
    return set_free_error(DBW_EUNSUPPORTED, "%s: st_W reaches 2^40", call);
  // (a launch holds fewer than 2^32 threads: fewer than 2^24 workgroups, which
  // are twice the plan's where lines at odd addresses take the smaller tile, and
  // up to 255 more for whole runs)
  if (dbw::group_plan(*p).blocks > (int64_t{1} << 23) - 128 - 1)
    return set_free_error(DBW_EUNSUPPORTED, "%s: 2^23 output tiles or more", call);
  return DBW_OK;
}

}  // namespace

DBW_API dbw_status dbw_group_workspace(const dbw_group_shape* shape, int64_t* bytes) {
  if (dbw_status s = check_shape(shape, "dbw_group_workspace"); s != DBW_OK) return s;
  if (!bytes) return set_free_error(DBW_EINVAL, "dbw_group_workspace: bytes is NULL");
  const dbw::GroupPlan plan = dbw::group_plan(*shape);
  *bytes = plan.splits > 1 ? plan.splits * plan.part * static_cast<int64_t>(sizeof(float)) : 0;
  return DBW_OK;
}

namespace {
// Checks of a product's pointers, and the product.
dbw_status group_call(const char* call, const dbw_group_shape* shape, const dbw_linear_epilogue* epilogue,
                      const int32_t* offsets, const void* a, const void* b, void* out, void* workspace,
                      int64_t workspace_bytes, void* stream) {
  int64_t need = 0;
  if (dbw_status s = dbw_group_workspace(shape, &need); s != DBW_OK) return s;
  const bool grad = shape->form == DBW_GROUP_WEIGHT_GRAD;
  // without rows, the arrays of T rows may be empty
  const bool rows = shape->T > 0;
  if (!offsets || (!a && rows) || (!b && (!grad || rows)) || (!out && (grad || rows)))
    return set_free_error(DBW_EINVAL, "%s: a device pointer is NULL", call);
  if (!aligned(offsets, 4) || !aligned(a, 2) || !aligned(b, 2) || !aligned(out, dbw::elem_bytes(shape->out_dtype)))
    return set_free_error(DBW_EINVAL, "%s: a pointer is not aligned to its elements", call);
  if (need > 0 && (!workspace || workspace_bytes < need || !aligned(workspace, 16)))
    return set_free_error(DBW_EINVAL, "%s: needs %lld bytes of workspace, 16-byte aligned (%lld given)", call,
                          (long long)need, (long long)workspace_bytes);
  if (out && (out == a || out == b))
    return set_free_error(DBW_EINVAL, "%s: out must not overlap the inputs", call);
  const dbw::GroupPlan plan = dbw::group_plan(*shape);
  const hipError_t e = dbw::launch_group(*shape, plan, offsets, a, b, out, static_cast<float*>(workspace), epilogue,
                                         static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return set_free_error(DBW_EHIP, "%s: launch failed: %s", call, hipGetErrorString(e));
  return DBW_OK;
}
}  // namespace

DBW_API dbw_status dbw_group_product(const dbw_group_shape* shape, const int32_t* offsets, const void* a,
                                     const void* b, void* out, void* workspace, int64_t workspace_bytes,
                                     void* stream) {
  const char* call = "dbw_group_product";
  if (dbw_status s = check_shape(shape, call); s != DBW_OK) return s;
  return group_call(call, shape, nullptr, offsets, a, b, out, workspace, workspace_bytes, stream);
}

DBW_API dbw_status dbw_group_linear(const dbw_group_shape* shape, const dbw_linear_epilogue* epilogue,
                                    const int32_t* offsets, const void* X, const void* W, void* Y, void* workspace,
                                    int64_t workspace_bytes, void* stream) {
  const char* call = "dbw_group_linear";
  if (dbw_status s = check_shape(shape, call); s != DBW_OK) return s;
  if (shape->form != DBW_GROUP_FORWARD) return set_free_error(DBW_EINVAL, "%s: the form is FORWARD", call);
  if (!epilogue) return set_free_error(DBW_EINVAL, "%s: epilogue is NULL", call);
  dbw_linear_epilogue e = *epilogue;
  if (e.activation < DBW_ACT_NONE || e.activation > DBW_ACT_SILU)
    return set_free_error(DBW_EINVAL, "%s: unknown activation %d", call, e.activation);
  if (!aligned(e.bias, 4) || !aligned(e.residual, dbw::elem_bytes(shape->out_dtype)) || !aligned(e.pre, 2))
    return set_free_error(DBW_EINVAL, "%s: a pointer is not aligned to its elements", call);
  if (!e.bias || shape->n == 1) e.st_bias = 0;
  if (e.st_bias && e.st_bias < shape->C)
    return set_free_error(DBW_EINVAL, "%s: b_1 would overlap b_0 (st_bias=%lld)", call, (long long)e.st_bias);
  if (e.st_bias && shape->st_W == 0)
    return set_free_error(DBW_EINVAL, "%s: groups that share W share its bias", call);
  if (e.st_bias >= (int64_t{1} << 40)) return set_free_error(DBW_EUNSUPPORTED, "%s: st_bias reaches 2^40", call);
  if ((e.residual && e.ld_residual < shape->C) || (e.pre && e.ld_pre < shape->C))
    return set_free_error(DBW_EINVAL, "%s: a row stride is below its row", call);
  const int64_t most = int64_t{1} << 21;
  if ((e.residual && e.ld_residual >= most) || (e.pre && e.ld_pre >= most))
    return set_free_error(DBW_EUNSUPPORTED, "%s: a row stride reaches 2^21", call);
  if (e.residual && e.residual == Y && e.ld_residual != shape->ld_C)
    return set_free_error(DBW_EINVAL, "%s: Y in the place of R needs its row stride", call);
  if (e.pre && (e.pre == Y || e.pre == X || e.pre == W || e.pre == e.residual))
    return set_free_error(DBW_EINVAL, "%s: Z must not overlap other arrays", call);
  for (const void* in : {static_cast<const void*>(e.bias), static_cast<const void*>(offsets)})
    if (in && (in == Y || in == e.pre))
      return set_free_error(DBW_EINVAL, "%s: an output must not overlap the bias or the offsets", call);
  return group_call(call, shape, &e, offsets, X, W, Y, workspace, workspace_bytes, stream);
}

// ---------------------------------------------------------------------------
namespace {
constexpr int64_t align256(int64_t b) { return (b + 255) / 256 * 256; }
}  // namespace

DBW_API int64_t dbw_token_workspace(int32_t n, int64_t T) {
  if (n < 1 || n > DBW_MAX_N || T < 0 || T >= (int64_t{1} << 31)) return -1;
  return int64_t{12} * n * dbw::kTokenParts + 4 * T;
}

DBW_API dbw_status dbw_token_loss(int32_t n, int64_t T, int32_t C, int32_t dtype, const int32_t* offsets,
                                  const void* Z, int64_t ld_Z, const int32_t* y, double scale, void* dZ,
                                  int64_t ld_dZ, float* loss, void* workspace, int64_t workspace_bytes,
                                  void* stream) {
  const char* call = "dbw_token_loss";
  if (n < 1 || n > DBW_MAX_N) return set_free_error(DBW_EINVAL, "%s: n=%d outside [1, %d]", call, n, DBW_MAX_N);
  if (T < 0 || T >= (int64_t{1} << 31))
    return set_free_error(DBW_EINVAL, "%s: T=%lld outside [0, 2^31)", call, (long long)T);
  if (C < 1) return set_free_error(DBW_EINVAL, "%s: C=%d < 1", call, C);
  if (C > (1 << 24)) return set_free_error(DBW_EUNSUPPORTED, "%s: C=%d above 2^24", call, C);
  if (dtype != DBW_F32 && dtype != DBW_BF16 && dtype != DBW_F16)
    return set_free_error(DBW_EINVAL, "%s: unknown dtype %d", call, dtype);
  if (!offsets || !loss || !workspace || (T > 0 && (!Z || !y)))
    return set_free_error(DBW_EINVAL, "%s: a device pointer is NULL", call);
  const size_t e = dbw::elem_bytes(dtype);
  if (!aligned(offsets, 4) || !aligned(y, 4) || !aligned(loss, 4) || !aligned(Z, e) || !aligned(dZ, e))
    return set_free_error(DBW_EINVAL, "%s: a pointer is not aligned to its elements", call);
  if (ld_Z < C || (dZ && ld_dZ < C)) return set_free_error(DBW_EINVAL, "%s: a row stride is below C=%d", call, C);
  if (ld_Z >= (int64_t{1} << 32) || (dZ && ld_dZ >= (int64_t{1} << 32)))
    return set_free_error(DBW_EUNSUPPORTED, "%s: a row stride reaches 2^32", call);
  if (dZ == Z && dZ && ld_dZ != ld_Z)
    return set_free_error(DBW_EINVAL, "%s: dZ in the place of Z needs its row stride", call);
  if (!std::isfinite(scale) || !std::isfinite(static_cast<float>(scale)))
    return set_free_error(DBW_EINVAL, "%s: scale is not finite", call);
  const int64_t need = dbw_token_workspace(n, T);
  if (workspace_bytes < need || !aligned(workspace, 16))
    return set_free_error(DBW_EINVAL, "%s: needs %lld bytes of workspace, 16-byte aligned (%lld given)", call,
                          (long long)need, (long long)workspace_bytes);
  dbw::TokenArgs a{};
  a.n = n; a.C = C; a.T = T; a.dtype = dtype; a.offsets = offsets;
  a.Z = Z; a.ld_Z = ld_Z; a.y = y; a.scale = static_cast<float>(scale);
  a.dZ = dZ; a.ld_dZ = ld_dZ; a.loss = loss;
  a.sums = static_cast<double*>(workspace);
  a.counts = reinterpret_cast<int32_t*>(a.sums + n * dbw::kTokenParts);
  a.row_loss = reinterpret_cast<float*>(a.counts + n * dbw::kTokenParts);
  const hipError_t err = dbw::launch_token_loss(a, static_cast<hipStream_t>(stream));
  if (err != hipSuccess) return set_free_error(DBW_EHIP, "%s: launch failed: %s", call, hipGetErrorString(err));
  return DBW_OK;
}

// ---------------------------------------------------------------------------
struct dbw_adamw {
  int device = 0;
  dbw_adamw_config cfg{};
  int64_t nchunks = 0;
  char* pool = nullptr;   // step, parts, tensors, chunks
  dbw::AdamStep* step = nullptr;
  double* parts = nullptr;
  dbw::AdamTensor* tensors = nullptr;
  dbw::AdamChunk* chunks = nullptr;
  std::vector<dbw_adamw_tensor> list;   // the caller's description
};

dbw_status dbw::adamw_place(const dbw_adamw* o, int device, const float* g, int64_t P, const float** w,
                            std::string* why) {
  if (o->device != device) {
    *why = "the plan is on another device";
    return DBW_EINVAL;
  }
  if (o->cfg.g_dtype != DBW_F32) {
    *why = "the context's gradient is fp32, the plan's are not";
    return DBW_EINVAL;
  }
  *w = nullptr;
  for (size_t i = 0; i < o->list.size(); ++i) {
    const dbw_adamw_tensor& t = o->list[i];
    if (!t.count) continue;
    const float* tg = static_cast<const float*>(t.g);
    const bool inside = tg >= g && t.count <= P && tg - g <= P - t.count;
    const float* base = inside ? t.w - (tg - g) : nullptr;
    if (!inside || (*w && base != *w)) {
      *why = "tensor " + std::to_string(i) + (inside ? ": its w has another place than its gradient in g"
                                                     : ": its gradient is not in the context's g");
      return DBW_EINVAL;
    }
    *w = base;
  }
  return DBW_OK;
}

dbw_status dbw::adamw_check(const dbw_adamw_hyper& h, std::string* why) {
  if (!(h.lr >= 0.0) || !std::isfinite(h.lr)) *why = "lr is finite and >= 0";
  else if (!(h.beta1 >= 0.0 && h.beta1 < 1.0 && h.beta2 >= 0.0 && h.beta2 < 1.0)) *why = "beta1 and beta2 lie in [0, 1)";
  else if (!(h.eps >= 1e-30) || !std::isfinite(h.eps)) *why = "eps is at least 1e-30";
  else if (!std::isfinite(h.grad_scale)) *why = "grad_scale is not finite";
  else if (!(h.max_norm >= 0.0) || !std::isfinite(h.max_norm)) *why = "max_norm is finite and >= 0";
  else return DBW_OK;
  return DBW_EINVAL;
}

namespace {
// A tensor one of whose arrays overlaps another that a step writes (a tensor
// listed twice, a state of two tensors), or -1.  In the order of their starts,
// an array is compared with the farthest ends before it, of all and of the
// written ones.
int32_t overlapping(const dbw_adamw_config& cfg, const dbw_adamw_tensor* tensors, size_t state) {
  struct Array {
    uintptr_t first, end;
    int32_t tensor;
    bool written;
  };
  std::vector<Array> all;
  all.reserve(static_cast<size_t>(cfg.tensors) * 7);
  for (int32_t i = 0; i < cfg.tensors; ++i) {
    const dbw_adamw_tensor& t = tensors[i];
    if (!t.count) continue;
    const auto add = [&](const void* p, int64_t bytes, bool written) {
      const uintptr_t first = reinterpret_cast<uintptr_t>(p);
      all.push_back(Array{first, first + static_cast<uintptr_t>(bytes), i, written});
    };
    add(t.w, t.count * 4, true);
    add(t.g, t.count * dbw::elem_bytes(cfg.g_dtype), false);
    add(t.m, t.count * static_cast<int64_t>(state), true);
    add(t.v, t.count * static_cast<int64_t>(state), true);
    if (t.w_low) add(t.w_low, t.count * 2, true);
    if (cfg.state_bits == 8) {
      const int64_t blocks = (t.count + dbw::kAdamBlock - 1) / dbw::kAdamBlock;
      add(t.m_scale, blocks, true);
      add(t.v_scale, blocks, true);
    }
  }
  std::sort(all.begin(), all.end(), [](const Array& a, const Array& b) { return a.first < b.first; });
  uintptr_t end = 0, end_written = 0;
  for (const Array& a : all) {
    if (a.first < (a.written ? end : end_written)) return a.tensor;
    end = std::max(end, a.end);
    if (a.written) end_written = std::max(end_written, a.end);
  }
  return -1;
}
}  // namespace

DBW_API dbw_status dbw_adamw_create(const dbw_adamw_config* cfg, const dbw_adamw_tensor* tensors, dbw_adamw** out) {
  const char* call = "dbw_adamw_create";
  if (!cfg || !tensors || !out) return set_free_error(DBW_EINVAL, "%s: a pointer is NULL", call);
  *out = nullptr;
  if (cfg->state_bits != 8 && cfg->state_bits != 32)
    return set_free_error(DBW_EINVAL, "%s: state_bits=%d is neither 8 nor 32", call, cfg->state_bits);
  if (cfg->g_dtype != DBW_F32 && cfg->g_dtype != DBW_BF16 && cfg->g_dtype != DBW_F16)
    return set_free_error(DBW_EINVAL, "%s: unknown g_dtype %d", call, cfg->g_dtype);
  if (cfg->low_dtype != DBW_BF16 && cfg->low_dtype != DBW_F16)
    return set_free_error(DBW_EINVAL, "%s: low_dtype is DBW_BF16 or DBW_F16", call);
  if (cfg->tensors < 1 || cfg->tensors > 65536)
    return set_free_error(DBW_EINVAL, "%s: tensors=%d outside [1, 65536]", call, cfg->tensors);
  if (cfg->t < 0) return set_free_error(DBW_EINVAL, "%s: t=%lld < 0", call, (long long)cfg->t);
  const size_t state = cfg->state_bits == 32 ? 4 : 1;
  int64_t nchunks = 0;
  for (int32_t i = 0; i < cfg->tensors; ++i) {
    const dbw_adamw_tensor& t = tensors[i];
    if (t.count < 0) return set_free_error(DBW_EINVAL, "%s: tensor %d: count < 0", call, i);
    if (!std::isfinite(t.lr_scale) || !std::isfinite(t.weight_decay) || t.lr_scale < 0.0 || t.weight_decay < 0.0)
      return set_free_error(DBW_EINVAL, "%s: tensor %d: lr_scale and weight_decay are finite and >= 0", call, i);
    if (!t.count) continue;
    if (!t.w || !t.g || !t.m || !t.v || (cfg->state_bits == 8 && (!t.m_scale || !t.v_scale)))
      return set_free_error(DBW_EINVAL, "%s: tensor %d: a device pointer is NULL", call, i);
    if (!aligned(t.w, 4) || !aligned(t.g, dbw::elem_bytes(cfg->g_dtype)) || !aligned(t.m, state) ||
        !aligned(t.v, state) || !aligned(t.w_low, 2))
      return set_free_error(DBW_EINVAL, "%s: tensor %d: a pointer is not aligned to its elements", call, i);
    if (t.count > (int64_t{1} << 40))
      return set_free_error(DBW_EUNSUPPORTED, "%s: tensor %d: count above 2^40", call, i);
    nchunks += (t.count + dbw::kAdamChunk - 1) / dbw::kAdamChunk;
  }
  if (nchunks > (int64_t{1} << 26))
    return set_free_error(DBW_EUNSUPPORTED, "%s: more than 2^26 chunks of %d values", call, dbw::kAdamChunk);
  try {
    if (const int32_t i = overlapping(*cfg, tensors, state); i >= 0)
      return set_free_error(DBW_EINVAL, "%s: tensor %d: an array overlaps another, and a step writes one of them", call, i);
  } catch (const std::exception&) {
    return set_free_error(DBW_EHIP, "%s: out of host memory", call);
  }
  dbw_adamw* o = new (std::nothrow) dbw_adamw;
  if (!o) return set_free_error(DBW_EHIP, "%s: out of host memory", call);
  o->cfg = *cfg;
  o->nchunks = nchunks;
  hipError_t e = hipGetDevice(&o->device);
  const int64_t at_parts = align256(sizeof(dbw::AdamStep));
  const int64_t at_tensors = at_parts + align256(sizeof(double) * dbw::kAdamNormParts);
  const int64_t at_chunks = at_tensors + align256(sizeof(dbw::AdamTensor) * cfg->tensors);
  const int64_t all = at_chunks + align256(sizeof(dbw::AdamChunk) * (nchunks ? nchunks : 1));
  std::vector<char> host;
  try {
    host.resize(all);
    o->list.assign(tensors, tensors + cfg->tensors);
  } catch (const std::exception&) {
    delete o;
    return set_free_error(DBW_EHIP, "%s: out of host memory", call);
  }
  dbw::AdamStep first{};
  first.t = cfg->t;
  *reinterpret_cast<dbw::AdamStep*>(host.data()) = first;
  auto* ht = reinterpret_cast<dbw::AdamTensor*>(host.data() + at_tensors);
  auto* hc = reinterpret_cast<dbw::AdamChunk*>(host.data() + at_chunks);
  int64_t c = 0;
  for (int32_t i = 0; i < cfg->tensors; ++i) {
    const dbw_adamw_tensor& t = tensors[i];
    ht[i] = dbw::AdamTensor{t.w, t.g, t.m, t.v, t.m_scale, t.v_scale, t.w_low, t.count, t.lr_scale, t.weight_decay};
    const int64_t mine = (t.count + dbw::kAdamChunk - 1) / dbw::kAdamChunk;
    for (int64_t q = 0; q < mine; ++q) hc[c++] = dbw::AdamChunk{i, static_cast<uint32_t>(q)};
  }
  if (e == hipSuccess) e = hipMalloc(reinterpret_cast<void**>(&o->pool), all);
  if (e == hipSuccess) e = hipMemcpy(o->pool, host.data(), all, hipMemcpyHostToDevice);
  if (e != hipSuccess) {
    if (o->pool) (void)hipFree(o->pool);
    (void)hipGetLastError();   // not the next launch's
    delete o;
    return set_free_error(DBW_EHIP, "%s: the plan's %lld bytes: %s", call, (long long)all, hipGetErrorString(e));
  }
  o->step = reinterpret_cast<dbw::AdamStep*>(o->pool);
  o->parts = reinterpret_cast<double*>(o->pool + at_parts);
  o->tensors = reinterpret_cast<dbw::AdamTensor*>(o->pool + at_tensors);
  o->chunks = reinterpret_cast<dbw::AdamChunk*>(o->pool + at_chunks);
  *out = o;
  return DBW_OK;
}

DBW_API void dbw_adamw_destroy(dbw_adamw* o) {
  if (!o) return;
  OnDevice on(o->device);
  (void)hipFree(o->pool);   // waits for the steps that still use it
  delete o;
}

DBW_API dbw_status dbw_adamw_step(dbw_adamw* o, const dbw_adamw_hyper* h, float* norm, void* stream) {
  const char* call = "dbw_adamw_step";
  if (!o || !h) return set_free_error(DBW_EINVAL, "%s: a pointer is NULL", call);
  std::string why;
  if (dbw_status st = dbw::adamw_check(*h, &why); st != DBW_OK)
    return set_free_error(st, "%s: %s", call, why.c_str());
  if (!aligned(norm, 4)) return set_free_error(DBW_EINVAL, "%s: norm is not aligned", call);
  OnDevice on(o->device);
  dbw::AdamArgs a{};
  a.tensors = o->tensors; a.chunks = o->chunks; a.nchunks = o->nchunks; a.step = o->step; a.parts = o->parts;
  a.bits = o->cfg.state_bits; a.g_dtype = o->cfg.g_dtype; a.low_dtype = o->cfg.low_dtype; a.h = *h; a.norm = norm;
  const hipError_t e = dbw::launch_adamw(a, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return set_free_error(DBW_EHIP, "%s: launch failed: %s", call, hipGetErrorString(e));
  return DBW_OK;
}

DBW_API dbw_status dbw_adamw_export(dbw_adamw* o, int64_t* t) {
  const char* call = "dbw_adamw_export";
  if (!o || !t) return set_free_error(DBW_EINVAL, "%s: a pointer is NULL", call);
  OnDevice on(o->device);
  hipError_t e = hipDeviceSynchronize();
  if (e == hipSuccess) e = hipMemcpy(t, &o->step->t, sizeof *t, hipMemcpyDeviceToHost);
  if (e != hipSuccess) return set_free_error(DBW_EHIP, "%s: %s", call, hipGetErrorString(e));
  return DBW_OK;
}

DBW_API dbw_status dbw_adamw_import(dbw_adamw* o, int64_t t) {
  const char* call = "dbw_adamw_import";
  if (!o) return set_free_error(DBW_EINVAL, "%s: the plan is NULL", call);
  if (t < 0) return set_free_error(DBW_EINVAL, "%s: t=%lld < 0", call, (long long)t);
  OnDevice on(o->device);
  hipError_t e = hipDeviceSynchronize();
  if (e == hipSuccess) e = hipMemcpy(&o->step->t, &t, sizeof t, hipMemcpyHostToDevice);
  if (e != hipSuccess) return set_free_error(DBW_EHIP, "%s: %s", call, hipGetErrorString(e));
  return DBW_OK;
}

DBW_API uint32_t dbw_adamw_bits(uint32_t seed, int64_t t, int32_t tensor, int64_t index) {
  const uint32_t key = dbw::adam_mix(dbw::adam_mix(dbw::adam_mix(seed) + static_cast<uint32_t>(t)) +
                                     static_cast<uint32_t>(tensor));
  return dbw::adam_mix(dbw::adam_index(index) + key);
}
