// C ABI of the gated unit, the cross entropy of a linear head and AdamW: validation, planning and launch order (see include/stripe.h).
#include <cmath>
#include <cstdio>
#include <cstring>
#include <memory>

#include "kernels.hpp"
#include "layers_host.hpp"

using namespace stripe;

struct stripe_gated {
  stripe_gated_desc_t d;
  Access best = kAny, otherwise = kAny;      // with W and x aligned to 16 bytes, and else
  ProductPlan plan[3][3];                    // [Access][forward, dx, dW]
  int64_t dz_row = 0, dz_bytes = 0, partial_bytes = 0;
  bool copies[3] = {false, false, false};    // this product reads copies of W and x (forward), of W (dx), of x (dW) in whole pieces
  int64_t copy_row = 0, w_bytes = 0, x_bytes = 0;
  Workspace ws;
  int64_t ws_bytes() const { return dz_bytes + partial_bytes + w_bytes + x_bytes; }
};

struct stripe_xent {
  stripe_xent_desc_t d;
  Access best = kAny, otherwise = kAny;      // with W aligned to 16 bytes, and else
  Access copies = kAny;                      // of products that read the workspace only
  bool w_copy[2] = {false, false};           // forward, backward: W is copied to rows of whole pieces
  int64_t w_bytes = 0;
  ProductPlan logits[3], dx[3], dw;          // [Access]
  int64_t piece = 0, pieces = 0;             // classes of a piece of the backward pass
  int64_t x_ld = 0, dz_ld = 0;
  // the workspace: rows' numbers and values, x's rows; then, forward: the tiles' sums, backward: dz, dx in fp32; partial images
  int64_t count_bytes = 0, row_bytes = 0, x_bytes = 0, stats_bytes = 0, dz_bytes = 0, sum_bytes = 0, partial_bytes = 0;
  Workspace ws;
  int64_t ws_bytes() const { return 256 + 256 + count_bytes + 6 * row_bytes + x_bytes + std::max(stats_bytes, dz_bytes + sum_bytes) + partial_bytes + w_bytes; }
};

struct stripe_adamw {
  stripe_dtype_t grad = STRIPE_F32;
  bool eight = false, bound = false;
  double beta1 = 0, beta2 = 0;
  std::vector<int64_t> elements;
  std::vector<double> decay;
  std::vector<AdamWParams> launches;         // without a step's values
  std::vector<std::vector<int32_t>> members; // the tensors of each launch
};

namespace {

constexpr int64_t kMaxLayerRows = (int64_t)1 << 28, kMaxXentRows = (int64_t)1 << 24, kMaxXentFeatures = (int64_t)1 << 20;
constexpr int64_t kNear = (int64_t)1 << 20;      // row strides up to which a tile's rows span less than 2^31 bytes
// dz of a piece: what the products that follow read again is still in the 256 MB of the last level cache (8192 rows, 2048 -> 65536 bf16 with gradients: 8
// pieces of 128 MB 6.47 ms, 2 of them 6.61, 4 6.49, 16 6.82).
constexpr int64_t kPieceBytes = (int64_t)128 << 20, kMaxPiece = (int64_t)1 << 19;
constexpr int64_t kMaxElements = (int64_t)1 << 34;
constexpr int64_t kFewRows = 64;

// Rows of bf16 that are no whole pieces go through registers, on the smallest tiles.  Where the estimates say so they are copied first: a launch, and the bytes
// read and written (a gated unit of 8192 rows, 4095 -> 4096: 986 us forward and 2095 backward through registers, 430 and 845; the cross entropy of 4096 rows,
// 1324 -> 15104: 293 and 760, 175 and 473).
constexpr int64_t kMostCopied = (int64_t)2 << 30;
double copy_time(int64_t bytes) { return 4 + 2 * (double)bytes / 4.5e6; }
// (STRIPE_TUNE's layers_copy: 0 never, 1 wherever it can be)
bool copy_pays(double with, double without) {
  const int forced = tune_int("layers_copy", -1);
  return forced < 0 ? with < without : forced != 0;
}

// a launch holds fewer than 2^32 lanes: 2^24 workgroups of 256, counted in tiles of 64 x 64 outputs, the smallest
bool too_many_tiles(int64_t images, int64_t m, int64_t n) { return ((__int128)images + m / 64 + 1) * (n / 64 + 1) >= 1 << 24; }

stripe_status_t check_type(stripe_dtype_t dtype, const char* what) {
  return dtype == STRIPE_BF16 || dtype == STRIPE_F32 ? STRIPE_OK : api_fail(STRIPE_ERR_UNSUPPORTED, std::string(what) + " computes in bf16 or f32");
}

// ---- gated unit -----------------------------------------------------------------
stripe_status_t gated_create(const stripe_gated_desc_t* desc, stripe_gated_t** out) {
  if (!desc || !out) return api_fail(STRIPE_ERR_NULL, "desc or out is NULL");
  *out = nullptr;
  stripe_gated_desc_t d = *desc;
  if (d.rows < 0 || d.rows > kMaxLayerRows || d.in_features < 1 || d.in_features > kMaxFeatures || d.out_features < 1 || d.out_features > kMaxFeatures / 2)
    return api_fail(STRIPE_ERR_INVALID_DESC, "a gated unit has 0 .. 2^28 rows, 1 .. 2^24 features in and 1 .. 2^23 out");
  if (d.groups < 0 || d.groups > kMaxGroups) return api_fail(STRIPE_ERR_INVALID_DESC, "groups is 0 (one matrix) or 1 .. 4096");
  if (const stripe_status_t st = check_type(d.dtype, "a gated unit"); st != STRIPE_OK) return st;
  if (d.activation < STRIPE_ACT_NONE || d.activation > STRIPE_ACT_SILU) return api_fail(STRIPE_ERR_INVALID_DESC, "unknown activation");
  const int64_t both = 2 * d.out_features, e = elem_size(d.dtype), v = 16 / e;
  if (!d.x_row) d.x_row = d.in_features;
  if (!d.w_row) d.w_row = d.in_features;
  if (!d.y_row) d.y_row = d.out_features;
  if (!d.pre_row) d.pre_row = both;
  if (d.x_row < d.in_features || d.x_row > kMaxStride || d.w_row < d.in_features || d.w_row > kMaxStride || d.y_row < d.out_features || d.y_row > kMaxStride ||
      d.pre_row < both || d.pre_row > kMaxStride)
    return api_fail(STRIPE_ERR_INVALID_DESC, "a row stride is shorter than its row (or beyond 2^40 elements)");
  if (beyond(d.rows, d.x_row) || beyond(d.rows, d.y_row) || beyond(d.rows, d.pre_row) || beyond(both, d.w_row))
    return api_fail(STRIPE_ERR_INVALID_DESC, "a buffer spans more than 2^56 elements");
  if (!d.w_group) d.w_group = both * d.w_row;
  if (d.groups && d.w_group < (both - 1) * d.w_row + d.in_features) return api_fail(STRIPE_ERR_INVALID_DESC, "w_group is shorter than a matrix");
  if (beyond(d.groups, d.w_group)) return api_fail(STRIPE_ERR_INVALID_DESC, "a buffer spans more than 2^56 elements");
  if (too_many_tiles(d.groups, d.rows, both) || too_many_tiles(d.groups, d.rows, d.in_features) || (d.rows + 15) / 16 * (d.out_features / 256 + 1) >= 1 << 24 ||
      ((__int128)both / 64 + 1) * (d.in_features / 64 + 1) * std::max(1, d.groups) >= 1 << 24)
    return api_fail(STRIPE_ERR_UNSUPPORTED, "more than 2^24 tiles of outputs");
  auto gated = std::make_unique<stripe_gated>();
  gated->d = d;
  gated->dz_row = (both + v - 1) / v * v;
  const bool near = d.x_row <= kNear && d.w_row <= kNear && gated->dz_row <= kNear;
  gated->otherwise = near && d.dtype == STRIPE_F32 ? kWords : kAny;
  // (dz's rows end in zeros, and the rows of pre and y are only stored: out_features may be anything)
  gated->best = near && d.in_features % v == 0 && d.x_row % v == 0 && d.w_row % v == 0 && (!d.groups || d.w_group % v == 0) ? kPieces : gated->otherwise;
  const bool odd = d.w_row * e % 4 != 0;
  for (const Access access : {gated->best, gated->otherwise})
    for (int k = 0; k < 3; ++k) {
      gated->plan[access][k] = plan_product((ProductKind)k, d.dtype, d.rows, d.in_features, both, d.groups, access, odd, kHalves);
      gated->partial_bytes = std::max(gated->partial_bytes, round_up_256(gated->plan[access][k].ws_bytes));
    }
  gated->dz_bytes = round_up_256(d.rows * gated->dz_row * e);
  gated->copy_row = (d.in_features + v - 1) / v * v;
  const int64_t matrices = std::max(1, d.groups) * both, w_bytes = round_up_256(matrices * gated->copy_row * e), x_bytes = round_up_256(d.rows * gated->copy_row * e);
  if (d.rows && d.dtype == STRIPE_BF16 && gated->best == kAny && gated->copy_row <= kNear && gated->dz_row <= kNear && w_bytes + x_bytes <= kMostCopied) {
    for (int k = 0; k < 3; ++k) {
      const ProductPlan plan = plan_product((ProductKind)k, d.dtype, d.rows, d.in_features, both, d.groups, kPieces, odd, kHalves);
      const int64_t bytes = k == kForward ? w_bytes + x_bytes : k == kInputGrad ? w_bytes : x_bytes;
      if (plan.few || !copy_pays(plan.us + copy_time(bytes) + (k == kForward ? 4 : 0), gated->plan[kAny][k].us)) continue;
      gated->copies[k] = true;
      gated->plan[kPieces][k] = plan;
      gated->partial_bytes = std::max(gated->partial_bytes, round_up_256(plan.ws_bytes));
      if (k != kWeightGrad) gated->w_bytes = w_bytes;
      if (k != kInputGrad) gated->x_bytes = x_bytes;
    }
  }
  *out = gated.release();
  return STRIPE_OK;
}

stripe_status_t check_offsets(int groups, const int32_t* offsets) {
  if (groups && !offsets) return api_fail(STRIPE_ERR_NULL, "a layer with groups needs its offsets");
  if (!groups && offsets) return api_fail(STRIPE_ERR_INVALID_DESC, "offsets without groups");
  if (misaligned(offsets, 4)) return api_fail(STRIPE_ERR_MISALIGNED, "offsets are not aligned to 4 bytes");
  return STRIPE_OK;
}

// A copy of x or of W in whole pieces, which the product is to read.
stripe_status_t gated_copy(const stripe_gated_t* gated, const void* x, const void* w, unsigned char* ws, ProductParams& p, hipStream_t stream) {
  const stripe_gated_desc_t& d = gated->d;
  unsigned char* const w_copy = ws + gated->dz_bytes + gated->partial_bytes;
  PadParams c = {};
  c.to_row = gated->copy_row; c.cols = (int32_t)d.in_features;
  if (w) {
    c.from = w; c.to = w_copy;
    c.each = 2 * d.out_features; c.rows = std::max(1, d.groups) * c.each; c.from_row = d.w_row; c.from_matrix = d.w_group;
    p.b = c.to; p.b_ld = c.to_row; p.b_group = c.each * c.to_row;
  } else {
    c.from = x; c.to = w_copy + gated->w_bytes;
    c.each = c.rows = d.rows; c.from_row = d.x_row;
    p.a = c.to; p.a_ld = c.to_row;
  }
  return launched(launch_pad(c, stream));
}

stripe_status_t gated_run(stripe_gated_t* gated, const void* x, const void* w, const int32_t* offsets, void* y, void* pre, void* hip_stream) {
  if (!gated) return api_fail(STRIPE_ERR_NULL, "gated is NULL");
  const stripe_gated_desc_t& d = gated->d;
  if (d.rows && (!x || !w || !y)) return api_fail(STRIPE_ERR_NULL, "x, w or y is NULL");
  if (const stripe_status_t st = check_offsets(d.groups, offsets); st != STRIPE_OK) return st;
  const int64_t e = elem_size(d.dtype), v = 16 / e;
  if (misaligned(x, e) || misaligned(w, e) || misaligned(y, e) || misaligned(pre, e))
    return api_fail(STRIPE_ERR_MISALIGNED, "a buffer is not aligned to its element type");
  if (!d.rows) return STRIPE_OK;
  if (shared({y, pre}, {x, w, offsets})) return api_fail(STRIPE_ERR_INVALID_DESC, "y or pre is an input, or one another");
  const bool copies = gated->copies[kForward];
  const Access access = copies ? kPieces : misaligned(x, 16) || misaligned(w, 16) ? gated->otherwise : gated->best;
  const ProductPlan& plan = gated->plan[access][kForward];
  unsigned char* ws = nullptr;
  if (plan.ws_bytes || copies)
    if (const stripe_status_t st = gated->ws.get(gated->ws_bytes(), (hipStream_t)hip_stream, &ws); st != STRIPE_OK) return st;
  ProductParams p = {};
  p.a = x; p.b = w; p.c = y; p.pre = pre; p.offsets = offsets;
  p.partial = ws ? (float*)(ws + gated->dz_bytes) : nullptr;
  p.a_ld = d.x_row; p.b_ld = d.w_row; p.c_ld = d.y_row; p.pre_ld = d.pre_row; p.b_group = d.w_group;
  if (copies) {
    if (const stripe_status_t st = gated_copy(gated, x, nullptr, ws, p, (hipStream_t)hip_stream); st != STRIPE_OK) return st;
    if (const stripe_status_t st = gated_copy(gated, nullptr, w, ws, p, (hipStream_t)hip_stream); st != STRIPE_OK) return st;
  }
  p.half = d.out_features * p.b_ld;
  p.rows = p.M = (int32_t)d.rows; p.N = (int32_t)d.out_features; p.K = (int32_t)d.in_features;
  p.groups = d.groups; p.act = d.activation;
  p.vec = d.y_row % v == 0 && !misaligned(y, 16);
  p.vec_pre = d.pre_row % v == 0 && d.out_features % v == 0 && !misaligned(pre, 16);
  return launched(launch_gated(d.dtype, plan, access, p, (hipStream_t)hip_stream));
}

stripe_status_t gated_backward(stripe_gated_t* gated, const void* dy, const void* x, const void* w, const void* pre, const int32_t* offsets, void* dx, void* dw,
                               void* hip_stream) {
  if (!gated) return api_fail(STRIPE_ERR_NULL, "gated is NULL");
  const stripe_gated_desc_t& d = gated->d;
  const hipStream_t stream = (hipStream_t)hip_stream;
  if (!dx && !dw) return STRIPE_OK;
  if (d.rows && (!dy || !pre || (dx && !w) || (dw && !x))) return api_fail(STRIPE_ERR_NULL, "dy, pre, or what a gradient reads (w, x), is NULL");
  if (const stripe_status_t st = check_offsets(d.groups, offsets); st != STRIPE_OK) return st;
  const int64_t e = elem_size(d.dtype), v = 16 / e;
  if (misaligned(dy, e) || misaligned(x, e) || misaligned(w, e) || misaligned(pre, e) || misaligned(dx, e) || misaligned(dw, e))
    return api_fail(STRIPE_ERR_MISALIGNED, "a buffer is not aligned to its element type");
  if (d.rows && shared({dx, dw}, {dy, x, w, pre, offsets})) return api_fail(STRIPE_ERR_INVALID_DESC, "a gradient's buffer is an input's or another's");
  unsigned char* ws = nullptr;
  if (d.rows)
    if (const stripe_status_t st = gated->ws.get(gated->ws_bytes(), stream, &ws); st != STRIPE_OK) return st;
  const Access w_access = gated->copies[kInputGrad] ? kPieces : misaligned(w, 16) ? gated->otherwise : gated->best;
  const Access x_access = gated->copies[kWeightGrad] ? kPieces : misaligned(x, 16) ? gated->otherwise : gated->best;
  if (d.rows) {
    GatedGradParams p = {};
    p.dy = dy; p.pre = pre; p.dz = ws;
    p.y_row = d.y_row; p.pre_row = d.pre_row; p.dz_row = gated->dz_row;
    p.rows = (int32_t)d.rows; p.out = (int32_t)d.out_features; p.act = d.activation;
    if (const stripe_status_t st = launched(launch_gated_grad(d.dtype, p, stream)); st != STRIPE_OK) return st;
  }
  ProductParams p = {};
  p.offsets = offsets;
  p.partial = ws ? (float*)(ws + gated->dz_bytes) : nullptr;
  p.rows = (int32_t)d.rows; p.groups = d.groups;
  p.a = ws; p.a_ld = gated->dz_row;
  if (dx && d.rows) {
    p.b = w; p.b_ld = d.w_row; p.b_group = d.w_group;
    if (gated->copies[kInputGrad])
      if (const stripe_status_t st = gated_copy(gated, nullptr, w, ws, p, stream); st != STRIPE_OK) return st;
    p.c = dx; p.c_ld = d.x_row;
    p.M = (int32_t)d.rows; p.N = (int32_t)d.in_features; p.K = (int32_t)(2 * d.out_features);
    p.vec = d.x_row % v == 0 && !misaligned(dx, 16);
    if (const stripe_status_t st = launched(launch_product(kInputGrad, d.dtype, gated->plan[w_access][kInputGrad], w_access, p, stream)); st != STRIPE_OK) return st;
  }
  if (dw) {
    p.b = x; p.b_ld = d.x_row;
    if (gated->copies[kWeightGrad] && d.rows) {
      ProductParams copy = {};
      if (const stripe_status_t st = gated_copy(gated, x, nullptr, ws, copy, stream); st != STRIPE_OK) return st;
      p.b = copy.a; p.b_ld = copy.a_ld;
    }
    p.b_group = 0;
    p.c = dw; p.c_ld = d.w_row; p.c_group = d.w_group;
    p.M = (int32_t)(2 * d.out_features); p.N = (int32_t)d.in_features; p.K = (int32_t)d.rows;
    p.vec = d.w_row % v == 0 && (!d.groups || d.w_group % v == 0) && !misaligned(dw, 16);
    if (const stripe_status_t st = launched(launch_product(kWeightGrad, d.dtype, gated->plan[x_access][kWeightGrad], x_access, p, stream)); st != STRIPE_OK) return st;
  }
  return STRIPE_OK;
}

// ---- cross entropy of a linear head -------------------------------------------------
stripe_status_t xent_create(const stripe_xent_desc_t* desc, stripe_xent_t** out) {
  if (!desc || !out) return api_fail(STRIPE_ERR_NULL, "desc or out is NULL");
  *out = nullptr;
  stripe_xent_desc_t d = *desc;
  if (d.rows < 0 || d.rows > kMaxXentRows || d.in_features < 1 || d.in_features > kMaxXentFeatures || d.classes < 1 || d.classes > kMaxFeatures)
    return api_fail(STRIPE_ERR_INVALID_DESC, "a cross entropy has 0 .. 2^24 rows of 1 .. 2^20 features, and 1 .. 2^24 classes");
  if (const stripe_status_t st = check_type(d.dtype, "a cross entropy"); st != STRIPE_OK) return st;
  const int64_t e = elem_size(d.dtype), v = 16 / e;
  if (!d.x_row) d.x_row = d.in_features;
  if (!d.w_row) d.w_row = d.in_features;
  if (d.x_row < d.in_features || d.x_row > kMaxStride || d.w_row < d.in_features || d.w_row > kMaxStride)
    return api_fail(STRIPE_ERR_INVALID_DESC, "a row stride is shorter than its row (or beyond 2^40 elements)");
  if (beyond(d.rows, d.x_row) || beyond(d.classes, d.w_row)) return api_fail(STRIPE_ERR_INVALID_DESC, "a buffer spans more than 2^56 elements");
  if (too_many_tiles(1, d.rows, d.classes) || too_many_tiles(1, d.rows, d.in_features) || too_many_tiles(1, d.classes, d.in_features))
    return api_fail(STRIPE_ERR_UNSUPPORTED, "more than 2^24 tiles of outputs");
  auto xent = std::make_unique<stripe_xent>();
  xent->d = d;
  // pieces of equal size, whole tiles of classes
  const int64_t most = std::min(kMaxPiece, std::max<int64_t>(256, kPieceBytes / e / std::max<int64_t>(1, d.rows) / 256 * 256));
  xent->pieces = (d.classes + most - 1) / most;
  if (const int forced = tune_int("xent_pieces", 0); forced > 0) xent->pieces = std::max<int64_t>(forced, (d.classes + kMaxPiece - 1) / kMaxPiece);
  xent->piece = std::min(d.classes, ((d.classes + xent->pieces - 1) / xent->pieces + 255) / 256 * 256);
  xent->pieces = (d.classes + xent->piece - 1) / xent->piece;
  xent->x_ld = (d.in_features + v - 1) / v * v;
  xent->dz_ld = (xent->piece + 7) / 8 * 8;
  const bool near = d.w_row <= kNear;
  xent->otherwise = near && d.dtype == STRIPE_F32 ? kWords : kAny;
  xent->best = near && d.in_features % v == 0 && d.w_row % v == 0 ? kPieces : xent->otherwise;
  xent->copies = kPieces;
  const bool odd = d.w_row * e % 4 != 0;
  xent->dw = plan_product(kWeightGrad, d.dtype, d.rows, d.in_features, xent->piece, 0, xent->copies, odd);
  xent->partial_bytes = xent->dw.ws_bytes;
  for (const Access access : {xent->best, xent->otherwise}) {
    xent->logits[access] = plan_product(kForward, d.dtype, d.rows, d.in_features, d.classes, 0, access, odd, kLogits);
    xent->dx[access] = plan_product(kInputGrad, d.dtype, d.rows, d.in_features, xent->piece, 0, access, odd);
    // (a piece's logits in slices: its classes end in zeros up to a multiple of 8)
    const int64_t slices = xent->logits[access].splits > 1 ? xent->logits[access].splits * d.rows * xent->dz_ld * 4 : 0;
    xent->partial_bytes = std::max({xent->partial_bytes, xent->dx[access].ws_bytes, xent->logits[access].ws_bytes, slices});
    const int64_t bn = tile_columns(xent->logits[access]);
    xent->stats_bytes = std::max(xent->stats_bytes, round_up_256(std::max((d.classes + bn - 1) / bn, (int64_t)xent_slice_blocks(d.classes)) * d.rows * 8));
  }
  const int64_t w_bytes = round_up_256(d.classes * xent->x_ld * e);
  if (d.rows && d.dtype == STRIPE_BF16 && xent->best == kAny && w_bytes <= kMostCopied) {
    const ProductPlan logits = plan_product(kForward, d.dtype, d.rows, d.in_features, d.classes, 0, kPieces, odd, kLogits);
    const ProductPlan dx = plan_product(kInputGrad, d.dtype, d.rows, d.in_features, xent->piece, 0, kPieces, odd);
    const double any = xent->logits[kAny].us, pieces = (double)xent->pieces;
    // An eighth less at least: a copy costs the same however few rows count, and the estimates of large copies beside few rows favour it (157 rows, 3790 -> 30841 with
    // dx: 227 us by the estimate and 246 through registers, measured 248 and 199; 205 rows, 1023 -> 50001: 122 and 158, 116 and 144).
    xent->w_copy[0] = copy_pays(logits.us + copy_time(w_bytes), 0.875 * any);
    xent->w_copy[1] = copy_pays(logits.us + dx.us * pieces + copy_time(w_bytes), 0.875 * (any + xent->dx[kAny].us * pieces));
    if (xent->w_copy[0] || xent->w_copy[1]) {
      xent->w_bytes = w_bytes;
      xent->logits[kPieces] = logits;
      xent->dx[kPieces] = dx;
      const int64_t bn = tile_columns(logits);
      xent->stats_bytes = std::max(xent->stats_bytes, round_up_256(std::max((d.classes + bn - 1) / bn, (int64_t)xent_slice_blocks(d.classes)) * d.rows * 8));
      xent->partial_bytes = std::max({xent->partial_bytes, dx.ws_bytes, logits.ws_bytes, logits.splits > 1 ? logits.splits * d.rows * xent->dz_ld * 4 : 0});
    }
  }
  xent->partial_bytes = round_up_256(xent->partial_bytes);
  xent->row_bytes = round_up_256(d.rows * 4);
  xent->count_bytes = round_up_256(d.rows / 1024 * 8 + 8);
  xent->x_bytes = round_up_256(d.rows * xent->x_ld * e);
  xent->dz_bytes = round_up_256(d.rows * xent->dz_ld * e);
  xent->sum_bytes = xent->pieces > 1 ? round_up_256(d.rows * d.in_features * 4) : 0;
  *out = xent.release();
  return STRIPE_OK;
}

// The parts of the workspace, and the rows that count copied into it.
struct XentParts {
  XentRowsParams rows = {};
  float* target_z;
  unsigned char* rest;
};
XentParts xent_parts(const stripe_xent_t* xent, unsigned char* ws) {
  XentParts parts;
  XentRowsParams& p = parts.rows;
  auto take = [&](int64_t bytes) { return ws += bytes, ws - bytes; };
  p.span = (int32_t*)take(256);
  p.scale = (float*)take(256);
  p.counts = (int32_t*)take(xent->count_bytes);
  p.index = (int32_t*)take(xent->row_bytes);
  p.row_target = (int32_t*)take(xent->row_bytes);
  p.row_lse = (float*)take(xent->row_bytes);
  p.row_all = (float*)take(xent->row_bytes);
  p.row_loss = (float*)take(xent->row_bytes);
  parts.target_z = (float*)take(xent->row_bytes);
  p.rows_x = take(xent->x_bytes);
  parts.rest = ws;
  p.x_row = xent->d.x_row; p.x_ld = xent->x_ld;
  p.rows = (int32_t)xent->d.rows; p.features = (int32_t)xent->d.in_features; p.classes = (int32_t)xent->d.classes;
  return parts;
}

ProductParams xent_logits(const stripe_xent_t* xent, const XentParts& parts, const void* w) {
  ProductParams p = {};
  p.a = parts.rows.rows_x; p.b = w; p.offsets = parts.rows.span; p.targets = parts.rows.row_target;
  p.a_ld = xent->x_ld; p.b_ld = xent->d.w_row;
  p.rows = p.M = (int32_t)xent->d.rows; p.K = (int32_t)xent->d.in_features;
  p.groups = 1;
  return p;
}

// A copy of W in whole pieces in its place.
stripe_status_t xent_copy(const stripe_xent_t* xent, const XentParts& parts, const void** w, int64_t* w_row, hipStream_t stream) {
  PadParams c = {};
  c.from = *w; c.to = parts.rest + std::max(xent->stats_bytes, xent->dz_bytes + xent->sum_bytes) + xent->partial_bytes;
  c.rows = c.each = xent->d.classes; c.from_row = xent->d.w_row; c.to_row = xent->x_ld; c.cols = (int32_t)xent->d.in_features;
  *w = c.to;
  *w_row = c.to_row;
  return launched(launch_pad(c, stream));
}

stripe_status_t xent_run(stripe_xent_t* xent, const void* x, const void* w, const int32_t* targets, float* loss, float* lse, void* hip_stream) {
  if (!xent) return api_fail(STRIPE_ERR_NULL, "xent is NULL");
  const stripe_xent_desc_t& d = xent->d;
  const hipStream_t stream = (hipStream_t)hip_stream;
  if (!loss && !lse) return STRIPE_OK;
  if (d.rows && (!x || !w || !targets)) return api_fail(STRIPE_ERR_NULL, "x, w or targets is NULL");
  const int64_t e = elem_size(d.dtype);
  if (misaligned(x, e) || misaligned(w, e) || misaligned(targets, 4) || misaligned(loss, 4) || misaligned(lse, 4))
    return api_fail(STRIPE_ERR_MISALIGNED, "a buffer is not aligned to its element type");
  if (!d.rows) return STRIPE_OK;
  if (shared({loss, lse}, {x, w, targets})) return api_fail(STRIPE_ERR_INVALID_DESC, "loss or lse is an input, or one another");
  unsigned char* ws = nullptr;
  if (const stripe_status_t st = xent->ws.get(xent->ws_bytes(), stream, &ws); st != STRIPE_OK) return st;
  XentParts parts = xent_parts(xent, ws);
  // Rows that fit one tile: leaving some out would save nothing, so x is read where it lies (a launch less: 16 rows, 4096 -> 32768 bf16 64.0 us, 58.9).  Not by
  // fp32 in parts, which computes a tile again if any of its rows does not end finite: the others' last bits would hang on rows that do not count.
  const bool copied = xent->w_copy[0];
  Access access = copied ? kPieces : misaligned(w, 16) ? xent->otherwise : xent->best;
  const Access there = misaligned(x, 16) || d.x_row % (16 / e) ? xent->otherwise : access;
  const bool in_place = !copied && d.rows <= kFewRows && d.x_row <= kNear && !xent->logits[there].parts;
  if (in_place) access = there;
  int64_t w_row = d.w_row;
  if (copied)
    if (const stripe_status_t st = xent_copy(xent, parts, &w, &w_row, stream); st != STRIPE_OK) return st;
  if (!in_place) {
    parts.rows.x = x; parts.rows.targets = targets; parts.rows.loss = loss; parts.rows.lse = lse; parts.rows.scale = nullptr;
    if (const stripe_status_t st = launched(launch_xent_rows(d.dtype, parts.rows, stream)); st != STRIPE_OK) return st;
  }
  const ProductPlan& plan = xent->logits[access];
  ProductParams p = xent_logits(xent, parts, w);
  p.b_ld = w_row;
  p.N = (int32_t)d.classes;
  if (in_place) p.a = x, p.a_ld = d.x_row, p.targets = targets, p.offsets = nullptr, p.groups = 0;
  p.stats = (float*)parts.rest; p.target_z = parts.target_z;
  p.partial = (float*)(parts.rest + std::max(xent->stats_bytes, xent->dz_bytes + xent->sum_bytes));
  if (const stripe_status_t st = launched(launch_xent(kLogSum, d.dtype, plan, access, p, stream)); st != STRIPE_OK) return st;
  XentJoinParams j = {};
  j.stats = p.stats; j.target_z = p.target_z;
  if (plan.splits > 1) j.partial = p.partial, j.splits = plan.splits;
  j.targets = p.targets;
  if (!in_place) j.index = parts.rows.index, j.span = parts.rows.span;
  j.classes = (int32_t)d.classes;
  j.loss = loss; j.lse = lse;
  j.rows = (int32_t)d.rows;
  j.tiles = plan.splits > 1 ? xent_slice_blocks(d.classes) : (int32_t)((d.classes + tile_columns(plan) - 1) / tile_columns(plan));
  return launched(launch_xent_join(j, stream));
}

stripe_status_t xent_backward(stripe_xent_t* xent, const void* x, const void* w, const int32_t* targets, const float* lse, const float* dloss, const float* dlse,
                              void* dx, void* dw, void* hip_stream) {
  if (!xent) return api_fail(STRIPE_ERR_NULL, "xent is NULL");
  const stripe_xent_desc_t& d = xent->d;
  const hipStream_t stream = (hipStream_t)hip_stream;
  if (!dx && !dw) return STRIPE_OK;
  if (d.rows && (!x || !w || !targets || !lse)) return api_fail(STRIPE_ERR_NULL, "x, w, targets or lse is NULL");
  const int64_t e = elem_size(d.dtype), v = 16 / e;
  if (misaligned(x, e) || misaligned(w, e) || misaligned(dx, e) || misaligned(dw, e) || misaligned(targets, 4) || misaligned(lse, 4) || misaligned(dloss, 4) ||
      misaligned(dlse, 4))
    return api_fail(STRIPE_ERR_MISALIGNED, "a buffer is not aligned to its element type");
  if (d.rows && shared({dx, dw}, {x, w, targets, lse, dloss, dlse})) return api_fail(STRIPE_ERR_INVALID_DESC, "a gradient's buffer is an input's or another's");
  const bool vec_w = d.w_row % v == 0 && !misaligned(dw, 16);
  if (!d.rows) {      // dW = 0
    if (!dw) return STRIPE_OK;
    ProductParams p = {};
    p.c = dw; p.c_ld = d.w_row; p.a_ld = p.b_ld = 8;
    p.M = (int32_t)d.classes; p.N = (int32_t)d.in_features;
    p.vec = vec_w;
    return launched(launch_product(kWeightGrad, d.dtype, xent->dw, xent->copies, p, stream));
  }
  unsigned char* ws = nullptr;
  if (const stripe_status_t st = xent->ws.get(xent->ws_bytes(), stream, &ws); st != STRIPE_OK) return st;
  XentParts parts = xent_parts(xent, ws);
  XentRowsParams& r = parts.rows;
  r.x = x; r.targets = targets; r.lse_in = lse; r.dloss = dloss; r.dlse = dlse; r.dx = dx;
  if (const stripe_status_t st = launched(launch_xent_rows(d.dtype, r, stream)); st != STRIPE_OK) return st;
  void* const dz = parts.rest;
  float* const sum = (float*)(parts.rest + xent->dz_bytes);
  float* const partial = (float*)(parts.rest + std::max(xent->stats_bytes, xent->dz_bytes + xent->sum_bytes));
  const Access access = xent->w_copy[1] ? kPieces : misaligned(w, 16) ? xent->otherwise : xent->best;
  int64_t w_row = d.w_row;
  if (xent->w_copy[1])
    if (const stripe_status_t st = xent_copy(xent, parts, &w, &w_row, stream); st != STRIPE_OK) return st;
  for (int64_t first = 0; first < d.classes; first += xent->piece) {
    const int64_t count = std::min(xent->piece, d.classes - first);
    const void* const rows = (const char*)w + first * w_row * e;
    ProductParams p = xent_logits(xent, parts, rows);
    p.b_ld = w_row;
    p.c = dz; p.c_ld = xent->dz_ld;
    p.N = (int32_t)((count + 7) / 8 * 8); p.class0 = (int32_t)first; p.classes = (int32_t)count;
    p.row_lse = r.row_lse; p.row_all = r.row_all; p.row_loss = r.row_loss; p.scale = r.scale;
    p.vec = 1; p.partial = partial;
    if (const stripe_status_t st = launched(launch_xent(kLossGrad, d.dtype, xent->logits[access], access, p, stream)); st != STRIPE_OK) return st;
    p = {};
    p.a = dz; p.a_ld = xent->dz_ld; p.offsets = r.span; p.groups = 1; p.partial = partial; p.scale = r.scale;
    p.rows = (int32_t)d.rows; p.N = (int32_t)d.in_features;
    if (dx) {
      p.b = rows; p.b_ld = w_row;
      p.c = dx; p.c_ld = d.x_row;
      p.M = (int32_t)d.rows; p.K = (int32_t)count;
      p.sum = xent->pieces > 1 ? sum : nullptr; p.index = r.index; p.first = first == 0; p.last = first + count == d.classes;
      p.vec = d.x_row % v == 0 && !misaligned(dx, 16);
      if (const stripe_status_t st = launched(launch_xent(kSumGrad, d.dtype, xent->dx[access], access, p, stream)); st != STRIPE_OK) return st;
    }
    if (dw) {
      p.b = r.rows_x; p.b_ld = xent->x_ld;
      p.c = (char*)dw + first * d.w_row * e; p.c_ld = d.w_row;
      p.M = (int32_t)count; p.K = (int32_t)d.rows;
      p.vec = vec_w;
      if (const stripe_status_t st = launched(launch_xent(kLossWeight, d.dtype, xent->dw, xent->copies, p, stream)); st != STRIPE_OK) return st;
    }
  }
  return STRIPE_OK;
}

// ---- AdamW ---------------------------------------------------------------------------
stripe_status_t adamw_create(const stripe_adamw_desc_t* desc, stripe_adamw_t** out) {
  if (!desc || !out) return api_fail(STRIPE_ERR_NULL, "desc or out is NULL");
  *out = nullptr;
  const stripe_adamw_desc_t& d = *desc;
  if (d.tensors < 0 || d.tensors > 1 << 20) return api_fail(STRIPE_ERR_INVALID_DESC, "an optimizer has 0 .. 2^20 tensors");
  if (d.tensors && !d.elements) return api_fail(STRIPE_ERR_NULL, "elements is NULL");
  if (d.grad_dtype != STRIPE_BF16 && d.grad_dtype != STRIPE_F32) return api_fail(STRIPE_ERR_UNSUPPORTED, "gradients are bf16 or f32");
  if (d.state_dtype != STRIPE_F32 && d.state_dtype != STRIPE_I8) return api_fail(STRIPE_ERR_UNSUPPORTED, "states are f32 or i8");
  if (!(d.beta1 >= 0 && d.beta1 < 1 && d.beta2 >= 0 && d.beta2 < 1)) return api_fail(STRIPE_ERR_INVALID_DESC, "beta1 and beta2 are at least 0 and less than 1");
  // (below, the reciprocal of what divides a state of 0 is infinite)
  if (!(d.eps == 0 || d.eps >= 0x1p-126) || !std::isfinite((float)d.eps)) return api_fail(STRIPE_ERR_INVALID_DESC, "eps is a finite number, 0 or at least 2^-126");
  auto adamw = std::make_unique<stripe_adamw>();
  adamw->grad = d.grad_dtype;
  adamw->eight = d.state_dtype == STRIPE_I8;
  adamw->beta1 = d.beta1;
  adamw->beta2 = d.beta2;
  AdamWParams p = {};
  p.b1 = (float)d.beta1; p.c1 = (float)(1 - d.beta1); p.b2 = (float)d.beta2; p.c2 = (float)(1 - d.beta2); p.eps = (float)d.eps;
  std::vector<int32_t> members;
  auto close = [&] {
    p.count = (int32_t)members.size();
    if (!p.count) return;
    adamw->launches.push_back(p);
    adamw->members.push_back(members);
    members.clear();
  };
  for (int32_t i = 0; i < d.tensors; ++i) {
    const int64_t n = d.elements[i];
    if (n < 0 || n > kMaxElements) return api_fail(STRIPE_ERR_INVALID_DESC, "a tensor has 0 .. 2^34 elements");
    const double wd = d.weight_decay ? d.weight_decay[i] : 0;
    if (!std::isfinite((float)wd)) return api_fail(STRIPE_ERR_INVALID_DESC, "a weight decay is a finite number");
    adamw->elements.push_back(n);
    adamw->decay.push_back(wd);
    if (!n) continue;
    const uint32_t chunks = adamw_chunks(n);
    if (members.size() == kAdamWTensors || (!members.empty() && (uint64_t)p.through[members.size() - 1] + chunks >= 1 << 24)) close();
    const size_t at = members.size();
    p.tensor[at] = {};
    p.tensor[at].elements = n;
    p.tensor[at].number = (uint32_t)i;
    p.through[at] = (at ? p.through[at - 1] : 0) + chunks;
    members.push_back(i);
  }
  close();
  *out = adamw.release();
  return STRIPE_OK;
}

stripe_status_t adamw_bind(stripe_adamw_t* adamw, const stripe_adamw_tensor_t* tensors) {
  if (!adamw) return api_fail(STRIPE_ERR_NULL, "adamw is NULL");
  if (!adamw->elements.empty() && !tensors) return api_fail(STRIPE_ERR_NULL, "tensors is NULL");
  const int64_t g = elem_size(adamw->grad), s = adamw->eight ? 1 : 4;
  std::vector<const void*> outs, ins;
  for (size_t i = 0; i < adamw->elements.size(); ++i) {
    if (!adamw->elements[i]) continue;
    const stripe_adamw_tensor_t& t = tensors[i];
    if (!t.p || !t.grad || !t.m || !t.v || (adamw->eight && (!t.m_scale || !t.v_scale)))
      return api_fail(STRIPE_ERR_NULL, "tensor " + std::to_string(i) + ": p, grad, a state or its factors are NULL");
    if (!adamw->eight && (t.m_scale || t.v_scale)) return api_fail(STRIPE_ERR_INVALID_DESC, "states of f32 have no factors");
    if (misaligned(t.p, 4) || misaligned(t.grad, g) || misaligned(t.m, s) || misaligned(t.v, s) || misaligned(t.m_scale, 4) || misaligned(t.v_scale, 4) ||
        misaligned(t.copy, 2))
      return api_fail(STRIPE_ERR_MISALIGNED, "tensor " + std::to_string(i) + ": a buffer is not aligned to its element type");
    for (const void* o : {(const void*)t.p, (const void*)t.m, (const void*)t.v, (const void*)t.m_scale, (const void*)t.v_scale, (const void*)t.copy})
      if (o) outs.push_back(o);
    ins.push_back(t.grad);
  }
  std::sort(outs.begin(), outs.end());
  const bool twice = std::adjacent_find(outs.begin(), outs.end()) != outs.end();
  if (twice || std::any_of(ins.begin(), ins.end(), [&](const void* q) { return std::binary_search(outs.begin(), outs.end(), q); }))
    return api_fail(STRIPE_ERR_INVALID_DESC, "a buffer that a step writes is bound twice");
  for (size_t l = 0; l < adamw->launches.size(); ++l)
    for (size_t k = 0; k < adamw->members[l].size(); ++k) {
      const stripe_adamw_tensor_t& t = tensors[adamw->members[l][k]];
      AdamWTensor& to = adamw->launches[l].tensor[k];
      to.p = t.p; to.grad = t.grad; to.m = t.m; to.v = t.v; to.m_scale = t.m_scale; to.v_scale = t.v_scale; to.copy = t.copy;
    }
  adamw->bound = true;
  return STRIPE_OK;
}

stripe_status_t adamw_run(stripe_adamw_t* adamw, const stripe_adamw_step_t* step, void* hip_stream) {
  if (!adamw || !step) return api_fail(STRIPE_ERR_NULL, "adamw or step is NULL");
  if (!adamw->bound && !adamw->launches.empty()) return api_fail(STRIPE_ERR_NULL, "no tensors are bound");
  if (misaligned(step->control, 4)) return api_fail(STRIPE_ERR_MISALIGNED, "control is not aligned to 4 bytes");
  if (!step->control && (step->step < 1 || step->step > (int64_t)1 << 53)) return api_fail(STRIPE_ERR_INVALID_DESC, "steps are counted from 1");
  if (!step->control && (!std::isfinite((float)step->lr) || !std::isfinite((float)step->factor)))
    return api_fail(STRIPE_ERR_INVALID_DESC, "lr and factor are finite numbers");
  for (size_t l = 0; l < adamw->launches.size(); ++l) {
    AdamWParams p = adamw->launches[l];
    for (size_t k = 0; k < adamw->members[l].size(); ++k) {
      const double wd = adamw->decay[adamw->members[l][k]];
      p.tensor[k].keep = step->control ? (float)wd : (float)(1 - step->lr * wd);
    }
    p.control = (const float*)step->control;
    if (!step->control) {
      p.rate = (float)(step->lr / (1 - std::pow(adamw->beta1, (double)step->step)));
      p.spread = (float)(1 / std::sqrt(1 - std::pow(adamw->beta2, (double)step->step)));
      p.factor = (float)step->factor;
      p.seed = step->seed;
    }
    if (const stripe_status_t st = launched(launch_adamw(adamw->grad, adamw->eight, p, (hipStream_t)hip_stream)); st != STRIPE_OK) return st;
  }
  return STRIPE_OK;
}

stripe_status_t adamw_read(stripe_adamw_t* adamw, float* const* m, float* const* v, void* hip_stream) {
  if (!adamw) return api_fail(STRIPE_ERR_NULL, "adamw is NULL");
  if (!adamw->eight) return api_fail(STRIPE_ERR_UNSUPPORTED, "states of f32 are their values");
  if (!adamw->bound && !adamw->launches.empty()) return api_fail(STRIPE_ERR_NULL, "no tensors are bound");
  std::vector<const void*> outs;
  std::vector<const void*> ins;
  for (size_t l = 0; l < adamw->launches.size(); ++l)
    for (size_t k = 0; k < adamw->members[l].size(); ++k) {
      const int32_t i = adamw->members[l][k];
      for (float* q : {m ? m[i] : nullptr, v ? v[i] : nullptr}) {
        if (misaligned(q, 4)) return api_fail(STRIPE_ERR_MISALIGNED, "tensor " + std::to_string(i) + ": an output is not aligned to 4 bytes");
        if (q) outs.push_back(q);
      }
      const AdamWTensor& t = adamw->launches[l].tensor[k];
      ins.insert(ins.end(), {t.m, t.v, t.m_scale, t.v_scale});
    }
  std::sort(outs.begin(), outs.end());
  if (std::adjacent_find(outs.begin(), outs.end()) != outs.end() ||
      std::any_of(ins.begin(), ins.end(), [&](const void* q) { return std::binary_search(outs.begin(), outs.end(), q); }))
    return api_fail(STRIPE_ERR_INVALID_DESC, "an output is a state or another output");
  for (size_t l = 0; l < adamw->launches.size(); ++l) {
    AdamWParams p = adamw->launches[l];
    for (size_t k = 0; k < adamw->members[l].size(); ++k) {
      const int32_t i = adamw->members[l][k];
      p.tensor[k].p = m ? m[i] : nullptr;
      p.tensor[k].copy = v ? v[i] : nullptr;
    }
    if (const stripe_status_t st = launched(launch_adamw_read(p, (hipStream_t)hip_stream)); st != STRIPE_OK) return st;
  }
  return STRIPE_OK;
}

}  // namespace

extern "C" {

stripe_status_t stripe_gated_create(const stripe_gated_desc_t* desc, stripe_gated_t** out) {
  return guarded([&] { return gated_create(desc, out); });
}

stripe_status_t stripe_gated_run(stripe_gated_t* gated, const void* x, const void* w, const int32_t* offsets, void* y, void* pre, void* hip_stream) {
  return guarded([&] { return gated_run(gated, x, w, offsets, y, pre, hip_stream); });
}

stripe_status_t stripe_gated_backward(stripe_gated_t* gated, const void* dy, const void* x, const void* w, const void* pre, const int32_t* offsets, void* dx,
                                      void* dw, void* hip_stream) {
  return guarded([&] { return gated_backward(gated, dy, x, w, pre, offsets, dx, dw, hip_stream); });
}

stripe_status_t stripe_gated_workspace_size(const stripe_gated_t* gated, size_t* bytes) {
  return guarded([&]() -> stripe_status_t {
    if (!gated || !bytes) return api_fail(STRIPE_ERR_NULL, "gated or bytes is NULL");
    *bytes = (size_t)gated->ws_bytes();
    return STRIPE_OK;
  });
}

stripe_status_t stripe_gated_set_workspace(stripe_gated_t* gated, void* device_ptr, size_t bytes) {
  return guarded([&] { return gated ? gated->ws.set(device_ptr, bytes, gated->ws_bytes()) : api_fail(STRIPE_ERR_NULL, "gated is NULL"); });
}

stripe_status_t stripe_gated_query(const stripe_gated_t* gated, stripe_linear_info_t* info) {
  return guarded([&]() -> stripe_status_t {
    if (!gated || !info) return api_fail(STRIPE_ERR_NULL, "gated or info is NULL");
    std::memset(info, 0, sizeof *info);
    char* names[3] = {info->forward, info->input_grad, info->weight_grad};
    for (int k = 0; k < 3; ++k) {
      const Access access = gated->copies[k] ? kPieces : gated->best;
      std::snprintf(names[k], sizeof info->forward, "%s%s%s", k ? "" : "gated_", product_name((ProductKind)k, gated->d.dtype, gated->plan[access][k], access).c_str(),
                    gated->copies[k] ? "_copied" : "");
    }
    info->workspace_bytes = gated->ws_bytes();
    return STRIPE_OK;
  });
}

void stripe_gated_destroy(stripe_gated_t* gated) { delete gated; }

stripe_status_t stripe_xent_create(const stripe_xent_desc_t* desc, stripe_xent_t** out) {
  return guarded([&] { return xent_create(desc, out); });
}

stripe_status_t stripe_xent_run(stripe_xent_t* xent, const void* x, const void* w, const int32_t* targets, float* loss, float* lse, void* hip_stream) {
  return guarded([&] { return xent_run(xent, x, w, targets, loss, lse, hip_stream); });
}

stripe_status_t stripe_xent_backward(stripe_xent_t* xent, const void* x, const void* w, const int32_t* targets, const float* lse, const float* dloss,
                                     const float* dlse, void* dx, void* dw, void* hip_stream) {
  return guarded([&] { return xent_backward(xent, x, w, targets, lse, dloss, dlse, dx, dw, hip_stream); });
}

stripe_status_t stripe_xent_workspace_size(const stripe_xent_t* xent, size_t* bytes) {
  return guarded([&]() -> stripe_status_t {
    if (!xent || !bytes) return api_fail(STRIPE_ERR_NULL, "xent or bytes is NULL");
    *bytes = xent->d.rows ? (size_t)xent->ws_bytes() : 0;
    return STRIPE_OK;
  });
}

stripe_status_t stripe_xent_set_workspace(stripe_xent_t* xent, void* device_ptr, size_t bytes) {
  return guarded([&] { return xent ? xent->ws.set(device_ptr, bytes, xent->d.rows ? xent->ws_bytes() : 0) : api_fail(STRIPE_ERR_NULL, "xent is NULL"); });
}

stripe_status_t stripe_xent_query(const stripe_xent_t* xent, stripe_linear_info_t* info) {
  return guarded([&]() -> stripe_status_t {
    if (!xent || !info) return api_fail(STRIPE_ERR_NULL, "xent or info is NULL");
    std::memset(info, 0, sizeof *info);
    const int dtype = xent->d.dtype;
    auto name = [&](char* to, ProductKind kind, const ProductPlan* plans, bool copied) {
      const Access access = copied ? kPieces : xent->best;
      std::snprintf(to, sizeof info->forward, "%s%s", product_name(kind, dtype, plans[access], access).c_str(), copied ? "_copied" : "");
    };
    name(info->forward, kForward, xent->logits, xent->w_copy[0]);
    name(info->input_grad, kInputGrad, xent->dx, xent->w_copy[1]);
    std::snprintf(info->weight_grad, sizeof info->weight_grad, "%s", product_name(kWeightGrad, dtype, xent->dw, xent->copies).c_str());
    info->workspace_bytes = xent->d.rows ? xent->ws_bytes() : 0;
    return STRIPE_OK;
  });
}

void stripe_xent_destroy(stripe_xent_t* xent) { delete xent; }

stripe_status_t stripe_adamw_create(const stripe_adamw_desc_t* desc, stripe_adamw_t** out) {
  return guarded([&] { return adamw_create(desc, out); });
}

stripe_status_t stripe_adamw_bind(stripe_adamw_t* adamw, const stripe_adamw_tensor_t* tensors) {
  return guarded([&] { return adamw_bind(adamw, tensors); });
}

stripe_status_t stripe_adamw_run(stripe_adamw_t* adamw, const stripe_adamw_step_t* step, void* hip_stream) {
  return guarded([&] { return adamw_run(adamw, step, hip_stream); });
}

stripe_status_t stripe_adamw_read(stripe_adamw_t* adamw, float* const* m, float* const* v, void* hip_stream) {
  return guarded([&] { return adamw_read(adamw, m, v, hip_stream); });
}

void stripe_adamw_destroy(stripe_adamw_t* adamw) { delete adamw; }

}  // extern "C"
