// C ABI of the layer operators: validation, planning and launch order (see include/stripe.h).
#include <algorithm>
#include <cmath>
#include <cstdio>
#include <cstring>
#include <memory>

#include "layers_host.hpp"

using namespace stripe;

namespace stripe {

stripe_status_t Workspace::set(void* ptr, size_t bytes, int64_t need) {
  if (ptr && (uintptr_t)ptr % 256) return api_fail(STRIPE_ERR_INVALID_DESC, "the workspace must be 256-byte aligned");
  if (ptr && (int64_t)bytes < need)
    return api_fail(STRIPE_ERR_NOMEM, "the workspace holds " + std::to_string(bytes) + " bytes, the handle needs " + std::to_string((long long)need));
  std::lock_guard<std::mutex> lock(mutex_);
  caller_ = ptr;
  return STRIPE_OK;
}

stripe_status_t Workspace::get(int64_t need, hipStream_t stream, unsigned char** out) {
  *out = nullptr;
  if (need == 0) return STRIPE_OK;
  std::lock_guard<std::mutex> lock(mutex_);
  if (caller_) {
    *out = (unsigned char*)caller_;
    return STRIPE_OK;
  }
  int dev = -1;
  if (const hipError_t e = hipGetDevice(&dev); e != hipSuccess) return api_fail(STRIPE_ERR_HIP, hipGetErrorString(e));
  for (const auto& d : owned_)
    if (d.first == dev) {
      *out = (unsigned char*)d.second;
      return STRIPE_OK;
    }
  hipStreamCaptureStatus capturing = hipStreamCaptureStatusNone;
  if (stream && hipStreamIsCapturing(stream, &capturing) == hipSuccess && capturing != hipStreamCaptureStatusNone)
    return api_fail(STRIPE_ERR_NOMEM, "no workspace yet, and none can be allocated under graph capture: set one, or run the handle once before");
  owned_.reserve(owned_.size() + 1);
  void* p = nullptr;
  if (hipMalloc(&p, (size_t)need) != hipSuccess) {
    (void)hipGetLastError();
    return api_fail(STRIPE_ERR_NOMEM, "out of device memory for the handle's workspace");
  }
  owned_.emplace_back(dev, p);
  *out = (unsigned char*)p;
  return STRIPE_OK;
}

}  // namespace stripe

namespace {

constexpr int64_t kMaxLinearRows = (int64_t)1 << 28, kMaxNormRows = (int64_t)1 << 30;

}  // namespace

struct stripe_linear {
  stripe_linear_desc_t d;
  Access best = kAny;                   // with 16-byte aligned buffers
  Access otherwise = kAny;
  ProductPlan plan[3][3];               // [Access][ProductKind]
  int64_t dz_bytes = 0, sums_bytes = 0, partial_bytes = 0;
  Workspace ws;
  int64_t ws_bytes() const { return dz_bytes + sums_bytes + partial_bytes; }
};

struct stripe_norm {
  stripe_norm_desc_t d;
  int blocks = 0;
  int64_t ws_bytes = 0;
  Workspace ws;
};

namespace {

stripe_status_t linear_create(const stripe_linear_desc_t* desc, stripe_linear_t** out) {
  if (!desc || !out) return api_fail(STRIPE_ERR_NULL, "desc or out is NULL");
  *out = nullptr;
  stripe_linear_desc_t d = *desc;
  if (d.rows < 0 || d.rows > kMaxLinearRows || d.in_features < 1 || d.in_features > kMaxFeatures || d.out_features < 1 || d.out_features > kMaxFeatures)
    return api_fail(STRIPE_ERR_INVALID_DESC, "a linear layer has 0 .. 2^28 rows and 1 .. 2^24 features on either side");
  if (d.groups < 0 || d.groups > kMaxGroups) return api_fail(STRIPE_ERR_INVALID_DESC, "groups is 0 (one matrix) or 1 .. 4096");
  if (d.dtype != STRIPE_BF16 && d.dtype != STRIPE_F32) return api_fail(STRIPE_ERR_UNSUPPORTED, "a linear layer computes in bf16 or f32");
  if (d.activation < STRIPE_ACT_NONE || d.activation > STRIPE_ACT_SILU) return api_fail(STRIPE_ERR_INVALID_DESC, "unknown activation");
  if (!d.x_row) d.x_row = d.in_features;
  if (!d.w_row) d.w_row = d.in_features;
  if (!d.y_row) d.y_row = d.out_features;
  if (d.x_row < d.in_features || d.x_row > kMaxStride || d.w_row < d.in_features || d.w_row > kMaxStride || d.y_row < d.out_features || d.y_row > kMaxStride)
    return api_fail(STRIPE_ERR_INVALID_DESC, "a row stride is shorter than its row (or beyond 2^40 elements)");
  if (beyond(d.rows, d.x_row) || beyond(d.rows, d.y_row) || beyond(d.out_features, d.w_row))
    return api_fail(STRIPE_ERR_INVALID_DESC, "a buffer spans more than 2^56 elements");
  const int64_t matrix = (d.out_features - 1) * d.w_row + d.in_features;
  if (!d.w_group) d.w_group = d.out_features * d.w_row;
  if (d.groups && d.w_group < matrix) return api_fail(STRIPE_ERR_INVALID_DESC, "w_group is shorter than a matrix");
  if (beyond(d.groups, d.w_group)) return api_fail(STRIPE_ERR_INVALID_DESC, "a buffer spans more than 2^56 elements");
  // a launch holds fewer than 2^32 lanes: 2^24 workgroups of 256, counted in tiles of 64 x 64 outputs, the smallest
  auto tiles = [](__int128 images, int64_t m, int64_t n) { return (images + m / 64 + 1) * (n / 64 + 1); };
  if (tiles(d.groups, d.rows, d.out_features) >= 1 << 24 || tiles(d.groups, d.rows, d.in_features) >= 1 << 24 ||
      tiles(0, d.out_features, d.in_features) * (d.groups ? d.groups : 1) >= 1 << 24)
    return api_fail(STRIPE_ERR_UNSUPPORTED, "more than 2^24 tiles of outputs");
  auto lin = std::make_unique<stripe_linear>();
  lin->d = d;
  const int64_t v = 16 / elem_size(d.dtype);
  // the kernels that load into LDS have 32-bit offsets: a tile's rows, at most 256, span less than 2^31 bytes
  const int64_t most = (int64_t)1 << 20;
  const bool near = d.x_row <= most && d.w_row <= most && d.y_row <= most;
  lin->otherwise = near && d.dtype == STRIPE_F32 ? kWords : kAny;
  lin->best = near && d.in_features % v == 0 && d.out_features % v == 0 && d.x_row % v == 0 && d.w_row % v == 0 && d.y_row % v == 0 &&
                      (!d.groups || d.w_group % v == 0) ? kPieces : lin->otherwise;
  for (const Access access : {lin->best, lin->otherwise})
    for (int k = 0; k < 3; ++k) {
      lin->plan[access][k] = plan_product((ProductKind)k, d.dtype, d.rows, d.in_features, d.out_features, d.groups, access, d.w_row * elem_size(d.dtype) % 4 != 0);
      lin->partial_bytes = std::max(lin->partial_bytes, round_up_256(lin->plan[access][k].ws_bytes));
    }
  if (d.activation != STRIPE_ACT_NONE) {
    const int64_t row = (d.out_features + v - 1) / v * v;    // dz's rows start at 16-byte boundaries
    lin->dz_bytes = round_up_256(d.rows * row * elem_size(d.dtype));
  }
  const int64_t slots = dz_slots(d.rows, d.groups);
  if (slots > 1) lin->sums_bytes = round_up_256(slots * d.out_features * 4);
  *out = lin.release();
  return STRIPE_OK;
}

stripe_status_t check_offsets(const stripe_linear_t* lin, const int32_t* offsets) {
  if (lin->d.groups && !offsets) return api_fail(STRIPE_ERR_NULL, "a layer with groups needs its offsets");
  if (!lin->d.groups && offsets) return api_fail(STRIPE_ERR_INVALID_DESC, "offsets without groups");
  if (misaligned(offsets, 4)) return api_fail(STRIPE_ERR_MISALIGNED, "offsets are not aligned to 4 bytes");
  return STRIPE_OK;
}

stripe_status_t linear_run(stripe_linear_t* lin, const void* x, const void* w, const float* bias, const void* residual, const int32_t* offsets, void* y,
                           void* pre, void* hip_stream) {
  if (!lin) return api_fail(STRIPE_ERR_NULL, "lin is NULL");
  const stripe_linear_desc_t& d = lin->d;
  if (d.rows && (!x || !w || !y)) return api_fail(STRIPE_ERR_NULL, "x, w or y is NULL");
  if (const stripe_status_t st = check_offsets(lin, offsets); st != STRIPE_OK) return st;
  const int64_t e = elem_size(d.dtype), v = 16 / e;
  if (misaligned(x, e) || misaligned(w, e) || misaligned(residual, e) || misaligned(y, e) || misaligned(pre, e) || misaligned(bias, 4))
    return api_fail(STRIPE_ERR_MISALIGNED, "a buffer is not aligned to its element type");
  if (!d.rows) return STRIPE_OK;
  if (shared({y, pre}, {x, w, bias, offsets}) || (pre && pre == residual)) return api_fail(STRIPE_ERR_INVALID_DESC, "y or pre is an input, or one another");
  const Access access = misaligned(x, 16) || misaligned(w, 16) ? lin->otherwise : lin->best;
  const ProductPlan& plan = lin->plan[access][kForward];
  unsigned char* ws = nullptr;
  if (plan.ws_bytes)
    if (const stripe_status_t st = lin->ws.get(lin->ws_bytes(), (hipStream_t)hip_stream, &ws); st != STRIPE_OK) return st;
  ProductParams p = {};
  p.a = x; p.b = w; p.c = y; p.bias = bias; p.residual = residual; p.pre = pre; p.offsets = offsets;
  p.partial = ws ? (float*)(ws + lin->dz_bytes + lin->sums_bytes) : nullptr;
  p.a_ld = d.x_row; p.b_ld = d.w_row; p.c_ld = d.y_row; p.b_group = d.w_group;
  p.rows = p.M = (int32_t)d.rows; p.N = (int32_t)d.out_features; p.K = (int32_t)d.in_features;
  p.groups = d.groups; p.act = d.activation;
  p.vec = d.y_row % v == 0 && !misaligned(y, 16) && !misaligned(residual, 16) && !misaligned(pre, 16);
  return launched(launch_product(kForward, d.dtype, plan, access, p, (hipStream_t)hip_stream));
}

stripe_status_t linear_backward(stripe_linear_t* lin, const void* dy, const void* x, const void* w, const void* pre, const int32_t* offsets, void* dx, void* dw,
                                float* dbias, void* hip_stream) {
  if (!lin) return api_fail(STRIPE_ERR_NULL, "lin is NULL");
  const stripe_linear_desc_t& d = lin->d;
  const hipStream_t stream = (hipStream_t)hip_stream;
  const bool act = d.activation != STRIPE_ACT_NONE;
  if (!dx && !dw && !dbias) return STRIPE_OK;
  if (d.rows && (!dy || (act && !pre) || (dx && !w) || (dw && !x))) return api_fail(STRIPE_ERR_NULL, "dy, or what a gradient reads (pre, w, x), is NULL");
  if (const stripe_status_t st = check_offsets(lin, offsets); st != STRIPE_OK) return st;
  const int64_t e = elem_size(d.dtype), v = 16 / e;
  if (misaligned(dy, e) || misaligned(x, e) || misaligned(w, e) || misaligned(pre, e) || misaligned(dx, e) || misaligned(dw, e) || misaligned(dbias, 4))
    return api_fail(STRIPE_ERR_MISALIGNED, "a buffer is not aligned to its element type");
  if (d.rows && shared({dx, dw, dbias}, {dy, x, w, pre, offsets})) return api_fail(STRIPE_ERR_INVALID_DESC, "a gradient's buffer is an input's or another's");
  const bool dy_off = !act && misaligned(dy, 16);
  const Access w_access = dy_off || misaligned(w, 16) ? lin->otherwise : lin->best, x_access = dy_off || misaligned(x, 16) ? lin->otherwise : lin->best;
  const ProductPlan &in_plan = lin->plan[w_access][kInputGrad], &w_plan = lin->plan[x_access][kWeightGrad];
  const int64_t slots = dz_slots(d.rows, d.groups);
  const bool need_dz = act && (dx || dw);
  unsigned char* ws = nullptr;
  if (need_dz || (dbias && slots > 1) || (dx && in_plan.ws_bytes) || (dw && w_plan.ws_bytes))
    if (const stripe_status_t st = lin->ws.get(lin->ws_bytes(), stream, &ws); st != STRIPE_OK) return st;
  const int64_t dz_row = act ? (d.out_features + v - 1) / v * v : d.y_row;
  const void* dz = act ? (const void*)ws : dy;
  if (need_dz || dbias) {
    DzParams p = {};
    p.dy = dy; p.z = act ? pre : nullptr; p.dz = need_dz ? ws : nullptr; p.db = dbias; p.partial = ws ? (float*)(ws + lin->dz_bytes) : nullptr;
    p.offsets = offsets;
    p.y_row = d.y_row; p.dz_row = dz_row;
    p.rows = (int32_t)d.rows; p.out = (int32_t)d.out_features; p.groups = d.groups; p.act = d.activation; p.slots = (int32_t)slots;
    if (const stripe_status_t st = launched(launch_dz(d.dtype, p, stream)); st != STRIPE_OK) return st;
  }
  ProductParams p = {};
  p.offsets = offsets;
  p.partial = ws ? (float*)(ws + lin->dz_bytes + lin->sums_bytes) : nullptr;
  p.rows = (int32_t)d.rows; p.groups = d.groups;
  p.a = dz; p.a_ld = dz_row;
  if (dx && d.rows) {
    p.b = w; p.b_ld = d.w_row; p.b_group = d.w_group;
    p.c = dx; p.c_ld = d.x_row;
    p.M = (int32_t)d.rows; p.N = (int32_t)d.in_features; p.K = (int32_t)d.out_features;
    p.vec = d.x_row % v == 0 && !misaligned(dx, 16);
    if (const stripe_status_t st = launched(launch_product(kInputGrad, d.dtype, in_plan, w_access, p, stream)); st != STRIPE_OK) return st;
  }
  if (dw) {
    p.b = x; p.b_ld = d.x_row; p.b_group = 0;
    p.c = dw; p.c_ld = d.w_row; p.c_group = d.w_group;
    p.M = (int32_t)d.out_features; p.N = (int32_t)d.in_features; p.K = (int32_t)d.rows;
    p.vec = d.w_row % v == 0 && (!d.groups || d.w_group % v == 0) && !misaligned(dw, 16);
    if (const stripe_status_t st = launched(launch_product(kWeightGrad, d.dtype, w_plan, x_access, p, stream)); st != STRIPE_OK) return st;
  }
  return STRIPE_OK;
}

stripe_status_t norm_create(const stripe_norm_desc_t* desc, stripe_norm_t** out) {
  if (!desc || !out) return api_fail(STRIPE_ERR_NULL, "desc or out is NULL");
  *out = nullptr;
  stripe_norm_desc_t d = *desc;
  if (d.rows < 0 || d.rows > kMaxNormRows || d.features < 1 || d.features > kMaxFeatures)
    return api_fail(STRIPE_ERR_INVALID_DESC, "a layer norm has 0 .. 2^30 rows of 1 .. 2^24 features");
  if (d.dtype != STRIPE_BF16 && d.dtype != STRIPE_F32) return api_fail(STRIPE_ERR_UNSUPPORTED, "a layer norm reads and writes bf16 or f32");
  if (!(d.eps >= 0) || !std::isfinite((float)d.eps)) return api_fail(STRIPE_ERR_INVALID_DESC, "eps is a finite number, at least 0");
  if (!d.x_row) d.x_row = d.features;
  if (!d.y_row) d.y_row = d.features;
  if (d.x_row < d.features || d.x_row > kMaxStride || d.y_row < d.features || d.y_row > kMaxStride)
    return api_fail(STRIPE_ERR_INVALID_DESC, "a row stride is shorter than its row (or beyond 2^40 elements)");
  if ((__int128)d.rows * std::max(d.x_row, d.y_row) > (__int128)1 << 56) return api_fail(STRIPE_ERR_INVALID_DESC, "a buffer spans more than 2^56 elements");
  auto norm = std::make_unique<stripe_norm>();
  norm->d = d;
  norm->blocks = norm_backward_blocks(d.rows, d.features, d.dtype);
  norm->ws_bytes = norm->blocks > 1 ? round_up_256((int64_t)norm->blocks * 2 * d.features * 4) : 0;
  *out = norm.release();
  return STRIPE_OK;
}

NormParams norm_params(const stripe_norm_t* norm) {
  NormParams p = {};
  p.x_row = norm->d.x_row; p.y_row = norm->d.y_row;
  p.rows = (int32_t)norm->d.rows; p.features = (int32_t)norm->d.features;
  p.blocks = norm->blocks;
  p.eps = (float)norm->d.eps;
  return p;
}

stripe_status_t norm_run(stripe_norm_t* norm, const void* x, const float* gamma, const float* beta, void* y, float* mean, float* rstd, void* hip_stream) {
  if (!norm) return api_fail(STRIPE_ERR_NULL, "norm is NULL");
  if (norm->d.rows && (!x || !y)) return api_fail(STRIPE_ERR_NULL, "x or y is NULL");
  const int64_t e = elem_size(norm->d.dtype);
  if (misaligned(x, e) || misaligned(y, e) || misaligned(gamma, 4) || misaligned(beta, 4) || misaligned(mean, 4) || misaligned(rstd, 4))
    return api_fail(STRIPE_ERR_MISALIGNED, "a buffer is not aligned to its element type");
  if (!norm->d.rows) return STRIPE_OK;
  if (shared({y, mean, rstd}, {gamma, beta}) || x == mean || x == rstd || (x == y && norm->d.rows > 1 && norm->d.x_row != norm->d.y_row))
    return api_fail(STRIPE_ERR_INVALID_DESC, "an output is an input or another output, or y is x with other row strides");
  NormParams p = norm_params(norm);
  p.x = x; p.gamma = gamma; p.beta = beta; p.y = y; p.mean = mean; p.rstd = rstd;
  return launched(launch_norm(norm->d.dtype, p, (hipStream_t)hip_stream));
}

stripe_status_t norm_backward(stripe_norm_t* norm, const void* dy, const void* x, const float* gamma, const float* mean, const float* rstd, void* dx,
                              float* dgamma, float* dbeta, void* hip_stream) {
  if (!norm) return api_fail(STRIPE_ERR_NULL, "norm is NULL");
  if (!dx && !dgamma && !dbeta) return STRIPE_OK;
  if (norm->d.rows && (!dy || !x || !mean || !rstd)) return api_fail(STRIPE_ERR_NULL, "dy, x, mean or rstd is NULL");
  const int64_t e = elem_size(norm->d.dtype);
  if (misaligned(x, e) || misaligned(dy, e) || misaligned(dx, e) || misaligned(gamma, 4) || misaligned(mean, 4) || misaligned(rstd, 4) ||
      misaligned(dgamma, 4) || misaligned(dbeta, 4))
    return api_fail(STRIPE_ERR_MISALIGNED, "a buffer is not aligned to its element type");
  if (norm->d.rows && shared({dx, dgamma, dbeta}, {dy, x, gamma, mean, rstd}))
    return api_fail(STRIPE_ERR_INVALID_DESC, "a gradient's buffer is an input's or another's");
  unsigned char* ws = nullptr;
  if (norm->ws_bytes && (dgamma || dbeta))
    if (const stripe_status_t st = norm->ws.get(norm->ws_bytes, (hipStream_t)hip_stream, &ws); st != STRIPE_OK) return st;
  NormParams p = norm_params(norm);
  p.x = x; p.dy = dy; p.gamma = gamma; p.mean_in = mean; p.rstd_in = rstd; p.dx = dx; p.dgamma = dgamma; p.dbeta = dbeta;
  p.partial = (float*)ws;
  return launched(launch_norm_backward(norm->d.dtype, p, (hipStream_t)hip_stream));
}

}  // namespace

extern "C" {

stripe_status_t stripe_linear_create(const stripe_linear_desc_t* desc, stripe_linear_t** out) {
  return guarded([&] { return linear_create(desc, out); });
}

stripe_status_t stripe_linear_run(stripe_linear_t* lin, const void* x, const void* w, const float* bias, const void* residual, const int32_t* offsets,
                                  void* y, void* pre, void* hip_stream) {
  return guarded([&] { return linear_run(lin, x, w, bias, residual, offsets, y, pre, hip_stream); });
}

stripe_status_t stripe_linear_backward(stripe_linear_t* lin, const void* dy, const void* x, const void* w, const void* pre, const int32_t* offsets, void* dx,
                                       void* dw, float* dbias, void* hip_stream) {
  return guarded([&] { return linear_backward(lin, dy, x, w, pre, offsets, dx, dw, dbias, hip_stream); });
}

stripe_status_t stripe_linear_workspace_size(const stripe_linear_t* lin, size_t* bytes) {
  return guarded([&]() -> stripe_status_t {
    if (!lin || !bytes) return api_fail(STRIPE_ERR_NULL, "lin or bytes is NULL");
    *bytes = (size_t)lin->ws_bytes();
    return STRIPE_OK;
  });
}

stripe_status_t stripe_linear_set_workspace(stripe_linear_t* lin, void* device_ptr, size_t bytes) {
  return guarded([&] { return lin ? lin->ws.set(device_ptr, bytes, lin->ws_bytes()) : api_fail(STRIPE_ERR_NULL, "lin is NULL"); });
}

stripe_status_t stripe_linear_query(const stripe_linear_t* lin, stripe_linear_info_t* info) {
  return guarded([&]() -> stripe_status_t {
    if (!lin || !info) return api_fail(STRIPE_ERR_NULL, "lin or info is NULL");
    std::memset(info, 0, sizeof *info);
    char* names[3] = {info->forward, info->input_grad, info->weight_grad};
    for (int k = 0; k < 3; ++k)
      std::snprintf(names[k], sizeof info->forward, "%s", product_name((ProductKind)k, lin->d.dtype, lin->plan[lin->best][k], lin->best).c_str());
    info->workspace_bytes = lin->ws_bytes();
    return STRIPE_OK;
  });
}

void stripe_linear_destroy(stripe_linear_t* lin) { delete lin; }

stripe_status_t stripe_norm_create(const stripe_norm_desc_t* desc, stripe_norm_t** out) {
  return guarded([&] { return norm_create(desc, out); });
}

stripe_status_t stripe_norm_run(stripe_norm_t* norm, const void* x, const float* gamma, const float* beta, void* y, float* mean, float* rstd,
                                void* hip_stream) {
  return guarded([&] { return norm_run(norm, x, gamma, beta, y, mean, rstd, hip_stream); });
}

stripe_status_t stripe_norm_backward(stripe_norm_t* norm, const void* dy, const void* x, const float* gamma, const float* mean, const float* rstd, void* dx,
                                     float* dgamma, float* dbeta, void* hip_stream) {
  return guarded([&] { return norm_backward(norm, dy, x, gamma, mean, rstd, dx, dgamma, dbeta, hip_stream); });
}

stripe_status_t stripe_norm_workspace_size(const stripe_norm_t* norm, size_t* bytes) {
  return guarded([&]() -> stripe_status_t {
    if (!norm || !bytes) return api_fail(STRIPE_ERR_NULL, "norm or bytes is NULL");
    *bytes = (size_t)norm->ws_bytes;
    return STRIPE_OK;
  });
}

stripe_status_t stripe_norm_set_workspace(stripe_norm_t* norm, void* device_ptr, size_t bytes) {
  return guarded([&] { return norm ? norm->ws.set(device_ptr, bytes, norm->ws_bytes) : api_fail(STRIPE_ERR_NULL, "norm is NULL"); });
}

void stripe_norm_destroy(stripe_norm_t* norm) { delete norm; }

}  // extern "C"
