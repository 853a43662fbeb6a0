// The linear layer's forward product with few rows, dense or in each group (gfx950): what bounds it is reading W once.
//
// A workgroup owns 16 columns (rows of W) and up to 16 rows of x of one group.  Its eight wavefronts share the reduction out in pieces of
// 128 bytes of every row (together 1 KB of each row of W per step) and add their sums through LDS: 4096 columns are 256 workgroups, with up to
// sixteen 16-byte loads of W per lane in flight.  Nothing is staged: a lane's 16 bytes along k are a matrix instruction's fragment as they
// are, for both operands; x comes from L2.  Rows of W and x beyond the last repeat it; their results are not stored.
// A gated unit's workgroup owns 8 outputs: 8 rows of W's gate half and the 8 that belong to them in its up half.
#include <algorithm>

#include "layers_device.hpp"

namespace stripe {
namespace {

constexpr int kWaves = 8, kCols = 16;

template <typename T>
__device__ __forceinline__ f32x4 mma16(u32x4 a, u32x4 b, f32x4 c) {
  if constexpr (sizeof(T) == 2) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  } else {
    const f32x4 x = __builtin_bit_cast(f32x4, a), y = __builtin_bit_cast(f32x4, b);
#pragma unroll
    for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(x[i], y[i], c, 0, 0, 0);
    return c;
  }
}

template <typename T, int UNROLL, bool GATED>
__global__ __launch_bounds__(64 * kWaves) void product_rows_kernel(const ProductParams p) {
  constexpr int VEC = kVec<T>, STEP = kWaves * 128 / (int)sizeof(T);      // elements of a row that the workgroup takes at a time
  __shared__ float part[kWaves][16][kCols];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, idx = lane & 15;
  const int slot = (int)(blockIdx.x / (unsigned)p.tiles_n), n0 = (int)(blockIdx.x % (unsigned)p.tiles_n) * (GATED ? kCols / 2 : kCols);
  RowTile r = {0, slot * 16, 0};
  if (p.groups) {
    r = find_row_tile(p.offsets, p.groups, p.rows, 16, slot);
    if (r.rows <= 0) return;
  } else {
    const int left = p.M - r.row0;
    r.rows = left < 16 ? left : 16;
  }
  // the output of this thread: its bias and residual are asked for before the reduction
  const int om = (int)threadIdx.x >> 4, on = n0 + ((int)threadIdx.x & 15);
  const bool stores = om < r.rows && on < p.N && (!GATED || (threadIdx.x & 15) < kCols / 2);
  const int64_t at = (int64_t)(r.row0 + om) * p.c_ld + on;
  float bias = 0.f, residual = 0.f;
  if (stores && p.bias) bias = p.bias[(int64_t)r.group * p.N + on];
  if (stores && p.residual) residual = (float)((const T*)p.residual)[at];

  const int k0 = wave * (STEP / kWaves) + (lane >> 4) * VEC;
  const int wc = GATED ? n0 + (idx & 7) : n0 + idx, wr = wc < p.N ? wc : p.N - 1;
  const T* w = (const T*)p.b + (int64_t)r.group * p.b_group + (int64_t)wr * p.b_ld + k0 + (GATED && idx >= 8 ? p.half : 0);
  const T* x = (const T*)p.a + (int64_t)(r.row0 + (idx < r.rows ? idx : r.rows - 1)) * p.a_ld + k0;
  f32x4 acc[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};      // two chains
  const int whole = p.K / STEP;      // steps in which every piece exists
  int s = 0;
  auto steps = [&](auto count) {
    constexpr int U = decltype(count)::value;
    u32x4 b[2 * U], a[2 * U];
#pragma unroll
    for (int u = 0; u < 2 * U; ++u) __builtin_memcpy(&b[u], w + (s + u / 2) * STEP + (u & 1) * 4 * VEC, 16);
#pragma unroll
    for (int u = 0; u < 2 * U; ++u) __builtin_memcpy(&a[u], x + (s + u / 2) * STEP + (u & 1) * 4 * VEC, 16);
    __builtin_amdgcn_sched_barrier(0);      // all loads of these steps are on their way before the first is waited for
#pragma unroll
    for (int u = 0; u < 2 * U; ++u) acc[u & 1] = mma16<T>(b[u], a[u], acc[u & 1]);
    s += U;
  };
  while (s + UNROLL <= whole) steps(std::integral_constant<int, UNROLL>{});
  if constexpr (UNROLL > 4)
    if (s + 4 <= whole) steps(std::integral_constant<int, 4>{});
  if constexpr (UNROLL > 2)
    if (s + 2 <= whole) steps(std::integral_constant<int, 2>{});
  if (s < whole) steps(std::integral_constant<int, 1>{});
  // the last, partial step
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int k = whole * STEP + u * 4 * VEC, n = p.K - k - k0;
    if (p.K - k - wave * (STEP / kWaves) <= 0) break;      // of the whole wavefront
    acc[u] = mma16<T>(load_piece<T>(w + k, n), load_piece<T>(x + k, n), acc[u]);
  }
  // element e of a lane: column (lane >> 4) * 4 + e, row lane & 15
  *(f32x4*)&part[wave][idx][(lane >> 4) * 4] = acc[0] + acc[1];
  __syncthreads();
  if (!stores) return;
  float v = 0.f;
#pragma unroll
  for (int g = 0; g < kWaves; ++g) v += part[g][om][threadIdx.x & 15];
  if constexpr (GATED) {
    float u = 0.f;
#pragma unroll
    for (int g = 0; g < kWaves; ++g) u += part[g][om][8 + (threadIdx.x & 7)];
    if (p.pre) {
      T* const pre = (T*)p.pre + (int64_t)(r.row0 + om) * p.pre_ld + on;
      pre[0] = (T)v;
      pre[p.N] = (T)u;
    }
    ((T*)p.c)[at] = (T)(activate<T>(v, p.act) * u);
    return;
  }
  v += bias;
  if (p.pre) ((T*)p.pre)[at] = (T)v;
  v = activate<T>(v, p.act) + residual;
  ((T*)p.c)[at] = (T)v;
}

template <typename T, bool GATED>
hipError_t launch_rows(const ProductParams& p, unsigned grid, hipStream_t stream) {
  // no more steps at once than there are
  const int64_t steps = (int64_t)p.K * (int64_t)sizeof(T) / (kWaves * 128);
  const dim3 wg(64 * kWaves);
  if (steps >= 8) product_rows_kernel<T, 8, GATED><<<dim3(grid), wg, 0, stream>>>(p);
  else if (steps >= 4) product_rows_kernel<T, 4, GATED><<<dim3(grid), wg, 0, stream>>>(p);
  else product_rows_kernel<T, 2, GATED><<<dim3(grid), wg, 0, stream>>>(p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_product_rows(ProductKind kind, int dtype, ProductParams p, hipStream_t stream) {
  const int cols = kind == kGated ? kCols / 2 : kCols;
  p.tiles_n = (p.N + cols - 1) / cols;
  const int64_t slots = p.groups ? p.M / 16 + std::min<int64_t>(p.groups, p.M) : (p.M + 15) / 16;
  const unsigned grid = (unsigned)(slots * p.tiles_n);
  if (kind == kGated) return dtype == STRIPE_F32 ? launch_rows<float, true>(p, grid, stream) : launch_rows<__bf16, true>(p, grid, stream);
  return dtype == STRIPE_F32 ? launch_rows<float, false>(p, grid, stream) : launch_rows<__bf16, false>(p, grid, stream);
}

}  // namespace stripe
