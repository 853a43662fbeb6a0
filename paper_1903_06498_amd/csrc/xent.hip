// Softmax cross entropy of a linear head, z = x W^T, forward and backward, without keeping z (gfx950).
//
// Forward: one product whose epilogue keeps, of each row of a tile, the largest logit and the sum of the exponentials of the distances from it;
// a second launch joins the tiles.  Backward, a piece of the vocabulary at a time: the same product again with dz = exp(z - lse) (dloss + dlse) -
// [target] dloss as its epilogue, rounded to the operands' type for the matrix instructions; dx += dz W (an fp32 image, written out by the last piece);
// the piece's rows of dW = dz^T x.  A bf16 dz is divided by a scale for its rounding, by which dx and dW are multiplied.
// Rows that do not count are taken out before: the kernels see the others, one after the other, as the one group of rows [0, their number), a number
// that stays on the device.
#include "product_tiles.hpp"

namespace stripe {
namespace {

constexpr int kCountBlock = 1024;      // rows of a count
constexpr int kRowsEach = 4;           // rows of a workgroup that copies
constexpr int64_t kManyRows = 16384;   // more of them are counted in blocks before

__device__ __forceinline__ bool counts(const XentRowsParams& p, int64_t row) { return (uint32_t)p.targets[row] < (uint32_t)p.classes; }
// What a row's dz is divided by at most: the larger of its dloss and dloss + dlse, where they are finite.
__device__ __forceinline__ float weight(const XentRowsParams& p, int64_t row) {
  if (!counts(p, row)) return 0.f;
  const float one = p.dloss ? p.dloss[row] : 1.f, all = p.dlse ? one + p.dlse[row] : one, w = fmaxf(__builtin_fabsf(one), __builtin_fabsf(all));
  return w < __builtin_inff() ? w : 0.f;
}
// A workgroup's total, and its largest value.
__device__ __forceinline__ int block_sum(int v, int* shared) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) v += __shfl_xor(v, d);
  if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = v;
  __syncthreads();
  v = shared[0] + shared[1] + shared[2] + shared[3];
  __syncthreads();
  return v;
}
__device__ __forceinline__ float block_largest(float v, int* shared) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) v = fmaxf(v, __shfl_xor(v, d));
  float* const f = (float*)shared;
  if ((threadIdx.x & 63) == 0) f[threadIdx.x >> 6] = v;
  __syncthreads();
  v = fmaxf(fmaxf(f[0], f[1]), fmaxf(f[2], f[3]));
  __syncthreads();
  return v;
}

__global__ __launch_bounds__(256) void xent_count_kernel(const XentRowsParams p) {
  __shared__ int shared[4];
  int n = 0;
  float top = 0.f;
#pragma unroll
  for (int i = 0; i < kCountBlock / 256; ++i) {
    const int64_t row = (int64_t)blockIdx.x * kCountBlock + i * 256 + threadIdx.x;
    if (row >= p.rows) break;
    n += counts(p, row);
    if (p.scale) top = fmaxf(top, weight(p, row));
  }
  n = block_sum(n, shared);
  top = block_largest(top, shared);
  if (threadIdx.x == 0) p.counts[2 * blockIdx.x] = n, p.counts[2 * blockIdx.x + 1] = __builtin_bit_cast(int, top);
}

// A few rows a workgroup, a wavefront copies one at a time: its place is the number of rows before it that count, which every workgroup counts for itself
// (8192 x 2048 bf16: 17 us; counted by one workgroup in a launch of its own before, 12 and 15).  The first workgroup finds the scale, the last one the number of all.
template <typename T>
__global__ __launch_bounds__(256) void xent_rows_kernel(const XentRowsParams p) {
  constexpr int VEC = kVec<T>, ROWS = kRowsEach, AHEAD = 4;
  __shared__ int shared[4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t row0 = (int64_t)blockIdx.x * ROWS;
  const bool many = p.rows > kManyRows;
  int n = 0;
  if (many)
    for (int64_t b = threadIdx.x; b < row0 / kCountBlock; b += 256) n += p.counts[2 * b];
#pragma unroll 8
  for (int64_t r = (many ? row0 / kCountBlock * kCountBlock : 0) + threadIdx.x; r < row0; r += 256) n += counts(p, r);
  int before = block_sum(n, shared);
  const bool mine = lane < ROWS && row0 + lane < p.rows && counts(p, row0 + lane);
  const uint64_t all = __ballot(mine);      // of the workgroup's rows, in every wavefront
  if (threadIdx.x == 0 && row0 + ROWS >= p.rows) p.span[0] = 0, p.span[1] = before + __builtin_popcountll(all);
  if (p.scale && blockIdx.x == 0) {
    // bf16: dz is divided by the largest weight, so that a target's dz, the value that matters most, lies in the upper half of a power of two, where
    // rounding is half as coarse (equal weights and unsure targets: dz = -1 + p)
    float top = 0.f;
    if (sizeof(T) == 2) {
      if (many)
        for (int64_t b = threadIdx.x; b < (p.rows + kCountBlock - 1) / kCountBlock; b += 256) top = fmaxf(top, __builtin_bit_cast(float, p.counts[2 * b + 1]));
      else
#pragma unroll 4
        for (int64_t r = threadIdx.x; r < p.rows; r += 256) top = fmaxf(top, weight(p, r));
    }
    top = block_largest(top, shared);
    if (threadIdx.x == 0) *p.scale = top > 0x1p-100f ? top : 1.f;
  }
  for (int i = wave; i < ROWS && row0 + i < p.rows; i += 4) {
    const int64_t row = row0 + i;
    if (!(all >> i & 1)) {
      if (lane == 0) {
        if (p.loss) p.loss[row] = 0.f;
        if (p.lse) p.lse[row] = 0.f;
      }
      if (p.dx)
        for (int64_t c = lane * VEC; c < p.features; c += 64 * VEC) store_piece<T>((T*)p.dx + row * p.x_row + c, (u32x4){0, 0, 0, 0}, (int)(p.features - c));
      continue;
    }
    const int64_t at = before + __builtin_popcountll(all & (((uint64_t)1 << i) - 1));
    const T* const x = (const T*)p.x + row * p.x_row;
    T* const to = (T*)p.rows_x + at * p.x_ld;
    int64_t c = lane * VEC;
    for (; c + (AHEAD - 1) * 64 * VEC + VEC <= p.features; c += AHEAD * 64 * VEC) {
      u32x4 v[AHEAD];
#pragma unroll
      for (int k = 0; k < AHEAD; ++k) __builtin_memcpy(&v[k], x + c + k * 64 * VEC, 16);
#pragma unroll
      for (int k = 0; k < AHEAD; ++k) *(u32x4*)(to + c + k * 64 * VEC) = v[k];
    }
    for (; c < p.features; c += 64 * VEC) *(u32x4*)(to + c) = load_piece<T>(x + c, (int)(p.features - c));
    if (lane == 0) {
      p.index[at] = (int)row;
      p.row_target[at] = p.targets[row];
      if (p.lse_in) {
        const float one = p.dloss ? p.dloss[row] : 1.f;
        p.row_lse[at] = p.lse_in[row];
        p.row_loss[at] = one;
        p.row_all[at] = p.dlse ? one + p.dlse[row] : one;
      }
    }
  }
}

// From the largest logit of row `row` of those that the products saw, the sum of the exponentials of the distances from it, and the target's logit.
__device__ __forceinline__ void store_loss(const XentJoinParams& p, int row, float top, float sum, float target_z) {
  const int at = p.index ? p.index[row] : row;
  const bool counts = (uint32_t)p.targets[row] < (uint32_t)p.classes, finite = __builtin_fabsf(top) < __builtin_inff();
  const float rest = logf(sum);
  if (p.lse) p.lse[at] = counts ? finite ? top + rest : rest : 0.f;
  if (p.loss) p.loss[at] = counts ? finite ? top - target_z + rest : rest - target_z : 0.f;
}

// A row's lse and loss from the tiles' parts: 16 rows a workgroup, 16 threads to a row, four tiles of each on their way at a time.
__global__ __launch_bounds__(256) void xent_join_kernel(const XentJoinParams p) {
  __shared__ float2 part[16][17];
  const int r = threadIdx.x & 15, slice = threadIdx.x >> 4, count = p.span ? p.span[1] : p.rows;
  const int row = (int)blockIdx.x * 16 + r;
  if ((int)blockIdx.x * 16 >= count) return;
  float top = -__builtin_inff(), sum = 0.f;
  auto add = [&](const float2* s, int n) {
    float high = top;
    for (int i = 0; i < n; ++i) high = fmaxf(high, s[i].x);
    const float from = __builtin_fabsf(high) < __builtin_inff() ? high : 0.f;
    sum *= __builtin_amdgcn_exp2f((top - from) * kLog2E);
    for (int i = 0; i < n; ++i) sum += s[i].y * __builtin_amdgcn_exp2f((s[i].x - from) * kLog2E);
    top = high;
  };
  if (row < count) {
    for (int t = slice; t < p.tiles; t += 64) {
      float2 s[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) s[i] = t + 16 * i < p.tiles ? ((const float2*)p.stats)[(int64_t)(t + 16 * i) * p.rows + row] : make_float2(-__builtin_inff(), 0.f);
      add(s, 4);
    }
  }
  part[slice][r] = make_float2(top, sum);
  __syncthreads();
  if (slice || row >= count) return;
  top = -__builtin_inff(), sum = 0.f;
  float2 s[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) s[i] = part[i][r];
  add(s, 16);
  store_loss(p, row, top, sum, p.target_z[row]);
}

// The same parts from logits in slices of the reduction, 1024 classes of a row a workgroup (one workgroup for a row: 4 rows, 1024 -> 15324 bf16 16.0 us in all, 11.3
// here); lse and loss, where there are no more.
constexpr int kSliceClasses = 1024;
__global__ __launch_bounds__(256) void xent_slices_kernel(const XentJoinParams p) {
  constexpr int EACH = kSliceClasses / 256;
  __shared__ float tops[4], sums[4], target_z;
  const int block = (int)(blockIdx.x % (unsigned)p.tiles), row = (int)(blockIdx.x / (unsigned)p.tiles), lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (row >= (p.span ? p.span[1] : p.rows)) return;
  const int target = p.targets[row], first = block * kSliceClasses + (int)threadIdx.x;
  float z[EACH], top = -__builtin_inff(), sum = 0.f;
#pragma unroll
  for (int i = 0; i < EACH; ++i) z[i] = 0.f;
#pragma unroll 4
  for (int s = 0; s < p.splits; ++s) {
    const float* from = p.partial + ((int64_t)s * p.rows + row) * p.classes;
#pragma unroll
    for (int i = 0; i < EACH; ++i) z[i] += first + 256 * i < p.classes ? from[first + 256 * i] : 0.f;
  }
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    if (first + 256 * i >= p.classes) z[i] = -__builtin_inff();
    else if (first + 256 * i == target) target_z = p.target_z[row] = z[i];
    top = fmaxf(top, z[i]);
  }
#pragma unroll
  for (int d = 1; d < 64; d *= 2) top = fmaxf(top, __shfl_xor(top, d));
  if (lane == 0) tops[wave] = top;
  __syncthreads();
  top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
  const float from = __builtin_fabsf(top) < __builtin_inff() ? top : 0.f;
#pragma unroll
  for (int i = 0; i < EACH; ++i) sum += __builtin_amdgcn_exp2f((z[i] - from) * kLog2E);
  sum = wave_sum(sum);
  if (lane == 0) sums[wave] = sum;
  __syncthreads();
  if (threadIdx.x) return;
  sum = (sums[0] + sums[1]) + (sums[2] + sums[3]);
  if (p.tiles == 1) store_loss(p, row, top, sum, target_z);
  else ((float2*)p.stats)[(int64_t)block * p.rows + row] = make_float2(top, sum);
}

template <typename T>
hipError_t launch_xent_type(ProductKind kind, const ProductPlan& plan, Access access, ProductParams& p, hipStream_t stream) {
  switch (kind) {
    case kLogSum: return launch_kind<T, kLogSum>(plan, access, p, stream);
    case kLossGrad: return launch_kind<T, kLossGrad>(plan, access, p, stream);
    case kSumGrad: return launch_kind<T, kSumGrad>(plan, access, p, stream);
    default: return launch_kind<T, kLossWeight>(plan, access, p, stream);
  }
}

}  // namespace

hipError_t launch_xent_rows(int dtype, const XentRowsParams& p, hipStream_t stream) {
  if (p.rows > kManyRows) xent_count_kernel<<<dim3((unsigned)((p.rows + kCountBlock - 1) / kCountBlock)), dim3(256), 0, stream>>>(p);
  const dim3 grid((unsigned)(((int64_t)p.rows + kRowsEach - 1) / kRowsEach));
  if (dtype == STRIPE_F32) xent_rows_kernel<float><<<grid, dim3(256), 0, stream>>>(p);
  else xent_rows_kernel<__bf16><<<grid, dim3(256), 0, stream>>>(p);
  return hipGetLastError();
}

int xent_slice_blocks(int64_t classes) { return (int)((classes + kSliceClasses - 1) / kSliceClasses); }

hipError_t launch_xent_join(const XentJoinParams& p, hipStream_t stream) {
  if (p.partial) {
    xent_slices_kernel<<<dim3((unsigned)((int64_t)p.rows * p.tiles)), dim3(256), 0, stream>>>(p);
    if (p.tiles == 1) return hipGetLastError();
  }
  xent_join_kernel<<<dim3((unsigned)(((int64_t)p.rows + 15) / 16)), dim3(256), 0, stream>>>(p);
  return hipGetLastError();
}

hipError_t launch_xent(ProductKind kind, int dtype, const ProductPlan& plan, Access access, ProductParams p, hipStream_t stream) {
  return dtype == STRIPE_F32 ? launch_xent_type<float>(kind, plan, access, p, stream) : launch_xent_type<__bf16>(kind, plan, access, p, stream);
}

}  // namespace stripe
