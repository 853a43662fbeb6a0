// Launch records and launchers of the layer operators (linear layer, rows sorted by expert, layer norm).
#pragma once

#include <hip/hip_runtime.h>

#include <mutex>
#include <string>
#include <utility>
#include <vector>

#include "../../include/stripe.h"

namespace stripe {

stripe_status_t api_fail(stripe_status_t st, const std::string& msg);

// A handle's device workspace: the caller's, else memory the handle allocates once per device and keeps until it is destroyed (a
// graph captured on one device stays valid when the handle runs on another).
class Workspace {
 public:
  ~Workspace() {
    for (auto& d : owned_) (void)hipFree(d.second);
  }
  stripe_status_t set(void* ptr, size_t bytes, int64_t need);
  stripe_status_t get(int64_t need, hipStream_t stream, unsigned char** out);

 private:
  std::mutex mutex_;
  void* caller_ = nullptr;
  std::vector<std::pair<int, void*>> owned_;
};

// ---- products of the linear layer (product.hip) -----------------------------
// C[m, n] = sum over k of A(m, k) B(k, n) in one of three layouts:
//   kForward      A [m][k] = x,   B [n][k] = W      y  = act(x W^T + b) + r
//   kInputGrad    A [m][k] = dz,  B [k][n] = W      dx = dz W
//   kWeightGrad   A [k][m] = dz,  B [k][n] = x      dW = dz^T x
// and, of the operators around it,
//   kGated        kForward, W's rows in two halves      y  = act(g) u                    (gated.hip)
//   kLogSum       kForward                              each tile's part of log sum exp  (xent.hip)
//   kLossGrad     kForward                              gradient of the logits
//   kSumGrad      kInputGrad                            added to an fp32 image; the last product's total goes to the rows that `index` names
//   kLossWeight   kWeightGrad                           the gradients of kLossGrad come divided by `scale`: the outputs times it (kSumGrad's too)
enum ProductKind { kForward = 0, kInputGrad = 1, kWeightGrad = 2, kGated = 3, kLogSum = 4, kLossGrad = 5, kSumGrad = 6, kLossWeight = 7 };
// A is [k][m], the reduction goes over rows
constexpr bool over_rows(int kind) { return kind == kWeightGrad || kind == kLossWeight; }
// B is [k][n]
constexpr bool reduces_rows(int kind) { return kind == kInputGrad || kind == kSumGrad || over_rows(kind); }

struct ProductParams {
  const void *a, *b;
  void* c;
  const float* bias;
  const void* residual;
  void* pre;
  const int32_t* offsets;   // rows of group g: offsets[g] .. offsets[g+1] - 1
  float* partial;           // splits > 1: fp32 images of the output, one per slice of the reduction
  int64_t a_ld, b_ld, c_ld; // row strides in elements
  int64_t b_group;          // kForward, kInputGrad: elements between the matrices of two groups
  int64_t c_group;          // kWeightGrad: the same of the output
  int32_t rows;             // rows of x (the range of offsets)
  int32_t M, N, K;          // kForward, kInputGrad with groups: M = rows; kWeightGrad: K = rows
  int32_t groups;           // 0: dense
  int32_t tiles_m, tiles_n; // kForward, kInputGrad: tiles_m is an upper bound of the row tiles with groups
  int32_t splits;
  int32_t act;
  int32_t vec;              // rows of c, residual and pre start at 16-byte boundaries
  // kGated: N outputs from 2 N rows of W
  int64_t half, pre_ld;     // elements from a gate row to its up row; row stride of pre, [rows][2 N]
  int32_t vec_pre;          // as vec, of both halves of pre
  // kLogSum, kLossGrad
  int32_t class0, classes;  // kLossGrad: the first class of this piece, and how many it has (N: with the zeros behind them)
  const int32_t* targets;   // [rows]
  const float *row_lse, *row_all, *row_loss;   // kLossGrad: lse, dloss + dlse, dloss
  const float* scale;       // kLossGrad, kSumGrad, kLossWeight
  float *stats, *target_z;  // kLogSum: [tiles_n][M] pairs; [rows]
  // kSumGrad
  float* sum;               // [M][N], nullptr: one product is all
  const int32_t* index;     // [rows]
  int32_t first, last;
  int32_t tile_rows, most_slices;   // of an output tile; of a reduction that is split
};

struct ProductPlan {
  int tile = 0;             // index into the tile table
  int splits = 1;
  bool parts = false;       // fp32 in three bf16 parts
  bool few = false;         // kForward: the kernel for few rows (product_rows.hip)
  int64_t ws_bytes = 0;     // partial images
  double us = 0;            // estimated time
};
// How a product's operands can be fetched: element by element at their rims; in whole 16-byte pieces (addresses, strides and contiguous extents are
// multiples of them); in 4-byte words (fp32).  The latter two also want a tile's rows to span less than 2^31 bytes.
enum Access { kAny = 0, kPieces = 1, kWords = 2 };
// What a forward product is for: kLogits are made on tiles, in slices only where they are few; kHalves is a gated unit's, `out` both halves.
enum ProductUse { kLayer, kHalves, kLogits };
ProductPlan plan_product(ProductKind kind, int dtype, int64_t rows, int64_t in, int64_t out, int groups, Access access, bool odd_rows, ProductUse use = kLayer);
int tile_columns(const ProductPlan& plan);
std::string product_name(ProductKind kind, int dtype, const ProductPlan& plan, Access access);
hipError_t launch_product(ProductKind kind, int dtype, const ProductPlan& plan, Access access, ProductParams p, hipStream_t stream);

hipError_t launch_product_rows(ProductKind kind, int dtype, ProductParams p, hipStream_t stream);     // kForward, kGated

// dz = dy act'(z) (dz == nullptr: not stored; act none: not needed) and db = sums of dz over each group's rows (db == nullptr: not
// computed).  partial: fp32, dz_slots(rows, groups) x out, unused if db is nullptr or there is one slot.
struct DzParams {
  const void *dy, *z;
  void* dz;
  float *db, *partial;
  const int32_t* offsets;
  int64_t y_row, dz_row;
  int32_t rows, out, groups, act, slots;
};
int64_t dz_slots(int64_t rows, int groups);
hipError_t launch_dz(int dtype, const DzParams& p, hipStream_t stream);

// ---- gated unit (gated.hip) ---------------------------------------------------
// [dg | du] from dy and [g | u], rows `dz_row` apart, zeros behind column 2 out up to it.
struct GatedGradParams {
  const void *dy, *pre;
  void* dz;
  int64_t y_row, pre_row, dz_row;
  int32_t rows, out, act;
};
// Rows of bf16 that start anywhere, copied to rows of whole 16-byte pieces, zeros behind column `cols`.  Row r comes from matrix r / each, row r % each.
struct PadParams {
  const void* from;
  void* to;
  int64_t rows, each, from_row, from_matrix, to_row;
  int32_t cols;
};
hipError_t launch_pad(const PadParams& p, hipStream_t stream);
hipError_t launch_gated(int dtype, const ProductPlan& plan, Access access, ProductParams p, hipStream_t stream);
hipError_t launch_gated_grad(int dtype, const GatedGradParams& p, hipStream_t stream);

// ---- cross entropy of a linear head (xent.hip) ---------------------------------
// The rows that count, i.e. whose target is a class, are copied to the front, in their order: index[i] is the i-th of them, span = {0, their
// number}.  Arrays of the others: all [rows].  What the outputs hold for rows that do not count is written here.
struct XentRowsParams {
  const void* x;
  const int32_t* targets;
  const float *lse_in, *dloss, *dlse;        // nullptr: no gradient; ones; zeros
  void* rows_x;                              // [rows][x_ld], zeros behind column `features`
  int32_t *index, *span, *row_target;
  int32_t* counts;                           // of many rows: those that count of each block of them, and the largest weight of each
  float *row_lse, *row_all, *row_loss, *scale;
  float *loss, *lse;                         // forward: 0 where a row does not count
  void* dx;                                  // backward: the same
  int64_t x_row, x_ld;
  int32_t rows, features, classes;
};
hipError_t launch_xent_rows(int dtype, const XentRowsParams& p, hipStream_t stream);
// loss and lse from the tiles' parts
struct XentJoinParams {
  float *stats, *target_z;                   // [tiles][rows] pairs, [rows]
  const float* partial;                      // [splits][rows][classes]: slices of the logits, from which stats and target_z are made first
  const int32_t *index, *span;               // nullptr: the rows are where they were, `targets` says which of them count
  const int32_t* targets;
  int32_t classes, splits;
  float *loss, *lse;
  int32_t rows, tiles;
};
int xent_slice_blocks(int64_t classes);     // `tiles` of logits in slices
hipError_t launch_xent_join(const XentJoinParams& p, hipStream_t stream);
hipError_t launch_xent(ProductKind kind, int dtype, const ProductPlan& plan, Access access, ProductParams p, hipStream_t stream);

// ---- AdamW (adamw.hip) ----------------------------------------------------------
constexpr int kAdamWBlock = 256;             // elements that share a factor (states in 8 bits)
constexpr int kAdamWTensors = 40;            // of a launch: their records are kernel arguments
struct AdamWTensor {
  float* p;
  const void* grad;
  void *m, *v;
  float *m_scale, *v_scale;
  void* copy;
  int64_t elements;
  float keep;                                // 1 - lr wd; with control: wd
  uint32_t number;
};
struct AdamWParams {
  AdamWTensor tensor[kAdamWTensors];
  uint32_t through[kAdamWTensors];           // chunks of the tensors up to and with it
  int32_t count;
  float b1, c1, b2, c2, eps;
  float rate, spread, factor;                // lr / (1 - b1^t); 1 / sqrt(1 - b2^t); of the gradients
  uint32_t seed;
  const float* control;                      // nullptr: the values above; else {lr, 1 / (1 - b1^t), 1 / sqrt(1 - b2^t), factor, seed's bits}
};
uint32_t adamw_chunks(int64_t elements);     // workgroups of a tensor
hipError_t launch_adamw(int grad_dtype, bool eight, const AdamWParams& p, hipStream_t stream);
hipError_t launch_adamw_read(const AdamWParams& p, hipStream_t stream);

// ---- layer norm (norm.hip) ----------------------------------------------------
struct NormParams {
  const void *x, *dy;
  const float *gamma, *beta, *mean_in, *rstd_in;
  void *y, *dx;
  float *mean, *rstd, *dgamma, *dbeta, *partial;
  int64_t x_row, y_row;
  int32_t rows, features, blocks;    // blocks: of the backward pass, each of which leaves one row of partial sums
  float eps;
};
int norm_backward_blocks(int64_t rows, int64_t features, int dtype);
hipError_t launch_norm(int dtype, const NormParams& p, hipStream_t stream);
hipError_t launch_norm_backward(int dtype, const NormParams& p, hipStream_t stream);

}  // namespace stripe
