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
enum ProductKind { kForward = 0, kInputGrad = 1, kWeightGrad = 2 };

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
};

struct ProductPlan {
  int tile = 0;             // index into the tile table
  int splits = 1;
  bool parts = false;       // fp32 in three bf16 parts
  bool few = false;         // kForward: the kernel for few rows (product_rows.hip)
  int64_t ws_bytes = 0;     // partial images
};
// How a product's operands can be fetched: element by element at their rims; in whole 16-byte pieces (addresses, strides and contiguous extents are
// multiples of them); in 4-byte words (fp32).  The latter two also want a tile's rows to span less than 2^31 bytes.
enum Access { kAny = 0, kPieces = 1, kWords = 2 };
ProductPlan plan_product(ProductKind kind, int dtype, int64_t rows, int64_t in, int64_t out, int groups, Access access, bool odd_rows);
std::string product_name(ProductKind kind, int dtype, const ProductPlan& plan, Access access);
hipError_t launch_product(ProductKind kind, int dtype, const ProductPlan& plan, Access access, ProductParams p, hipStream_t stream);

hipError_t launch_product_rows(int dtype, ProductParams p, hipStream_t stream);

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
