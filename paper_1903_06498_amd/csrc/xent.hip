// Softmax cross entropy of a linear head, z = x W^T, forward and backward, without keeping z (gfx950).
//
// Forward: one product whose epilogue keeps, of each row of a tile, the largest logit and the sum of the exponentials of the distances from it;
// a second launch joins the tiles.  Backward, a piece of the vocabulary at a time: the same product again with dz = exp(z - lse) (dloss + dlse) -
// [target] dloss as its epilogue, rounded to the operands' type for the matrix instructions; dx += dz W (an fp32 image, written out by the last piece);
// the piece's rows of dW = dz^T x.
// Rows that do not count are taken out before: the kernels see the others, one after the other, as the one group of rows [0, their number), a number
// that stays on the device.
#include "product_tiles.hpp"

namespace stripe {
namespace {

// Which rows count: one workgroup, a run of rows for each thread.
__global__ __launch_bounds__(1024) void xent_index_kernel(const XentRowsParams p) {
  __shared__ int waves[16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t each = (p.rows + 1023) / 1024, first = threadIdx.x * each, last = first + each < p.rows ? first + each : p.rows;
  int mine = 0;
  for (int64_t r = first; r < last; ++r) mine += (uint32_t)p.targets[r] < (uint32_t)p.classes;
  int through = mine;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int o = __shfl_up(through, d);
    if (lane >= d) through += o;
  }
  if (lane == 63) waves[wave] = through;
  __syncthreads();
  int before = through - mine;
  for (int w = 0; w < wave; ++w) before += waves[w];
  if (threadIdx.x == 1023) p.span[0] = 0, p.span[1] = before + mine;
  for (int64_t r = first; r < last; ++r)
    if ((uint32_t)p.targets[r] < (uint32_t)p.classes) p.index[before++] = (int)r;
}

// A row of the copies, and of the outputs where a row does not count: a wavefront each.
template <typename T>
__global__ __launch_bounds__(256) void xent_rows_kernel(const XentRowsParams p) {
  constexpr int VEC = kVec<T>;
  const int lane = threadIdx.x & 63;
  const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (row >= p.rows) return;
  if ((uint32_t)p.targets[row] >= (uint32_t)p.classes) {
    if (lane == 0) {
      if (p.loss) p.loss[row] = 0.f;
      if (p.lse) p.lse[row] = 0.f;
    }
    if (p.dx)
      for (int64_t c = lane * VEC; c < p.features; c += 64 * VEC) store_piece<T>((T*)p.dx + row * p.x_row + c, (u32x4){0, 0, 0, 0}, (int)(p.features - c));
  }
  if (row >= p.span[1]) return;
  const int64_t from = p.index[row];
  const T* const x = (const T*)p.x + from * p.x_row;
  T* const to = (T*)p.rows_x + row * p.x_ld;
  for (int64_t c = lane * VEC; c < p.features; c += 64 * VEC) *(u32x4*)(to + c) = load_piece<T>(x + c, (int)(p.features - c));
  if (lane == 0) {
    p.row_target[row] = p.targets[from];
    if (p.lse_in) {
      const float one = p.dloss ? p.dloss[from] : 1.f;
      p.row_lse[row] = p.lse_in[from];
      p.row_loss[row] = one;
      p.row_all[row] = p.dlse ? one + p.dlse[from] : one;
    }
  }
}

// A row's lse and loss: 64 rows, four wavefronts that share the tiles out.
__global__ __launch_bounds__(256) void xent_join_kernel(const XentJoinParams p) {
  __shared__ float2 part[4][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, count = p.span[1];
  const int row = (int)blockIdx.x * 64 + lane;
  if ((int)blockIdx.x * 64 >= count) return;
  float top = -__builtin_inff(), sum = 0.f;
  auto add = [&](float2 s) {
    const float high = fmaxf(top, s.x), from = __builtin_fabsf(high) < __builtin_inff() ? high : 0.f;
    sum = sum * expf(top - from) + s.y * expf(s.x - from);
    top = high;
  };
  if (row < count) {
#pragma unroll 4
    for (int t = wave; t < p.tiles; t += 4) add(((const float2*)p.stats)[(int64_t)t * p.rows + row]);
  }
  part[wave][lane] = make_float2(top, sum);
  __syncthreads();
  if (wave || row >= count) return;
  for (int w = 1; w < 4; ++w) add(part[w][lane]);
  const float lse = (__builtin_fabsf(top) < __builtin_inff() ? top : 0.f) + logf(sum);
  const int at = p.index[row];
  if (p.lse) p.lse[at] = lse;
  if (p.loss) p.loss[at] = lse - p.target_z[row];
}

template <typename T>
hipError_t launch_xent_type(ProductKind kind, const ProductPlan& plan, Access access, ProductParams& p, hipStream_t stream) {
  switch (kind) {
    case kLogSum: return launch_kind<T, kLogSum>(plan, access, p, stream);
    case kLossGrad: return launch_kind<T, kLossGrad>(plan, access, p, stream);
    default: return launch_kind<T, kSumGrad>(plan, access, p, stream);
  }
}

}  // namespace

hipError_t launch_xent_rows(int dtype, const XentRowsParams& p, hipStream_t stream) {
  xent_index_kernel<<<dim3(1), dim3(1024), 0, stream>>>(p);
  const dim3 grid((unsigned)(((int64_t)p.rows + 3) / 4));
  if (dtype == STRIPE_F32) xent_rows_kernel<float><<<grid, dim3(256), 0, stream>>>(p);
  else xent_rows_kernel<__bf16><<<grid, dim3(256), 0, stream>>>(p);
  return hipGetLastError();
}

hipError_t launch_xent_join(const XentJoinParams& p, hipStream_t stream) {
  xent_join_kernel<<<dim3((unsigned)(((int64_t)p.rows + 63) / 64)), dim3(256), 0, stream>>>(p);
  return hipGetLastError();
}

hipError_t launch_xent(ProductKind kind, int dtype, const ProductPlan& plan, Access access, ProductParams p, hipStream_t stream) {
  return dtype == STRIPE_F32 ? launch_xent_type<float>(kind, plan, access, p, stream) : launch_xent_type<__bf16>(kind, plan, access, p, stream);
}

}  // namespace stripe
