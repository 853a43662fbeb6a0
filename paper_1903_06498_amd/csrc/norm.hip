// Layer norm, forward and backward (gfx950).
//
// Each row is read once into registers: 64, 256 or 1024 lanes share a row, at most 32 elements each (longer rows are read again for
// each sum).  Mean first, then the mean of the squared distances from it -- not E[x^2] - E[x]^2, which loses
// what the mean's square has more digits than.  The backward pass keeps its columns' sums of dy h and dy in registers over all the
// rows that its workgroup takes, leaves one row of partial sums per workgroup and adds those in a second launch in a fixed order.
#include <algorithm>
#include <type_traits>

#include "layers_device.hpp"

namespace stripe {
namespace {

// Sum over the TPR lanes that share a row; all of them get it.
template <int TPR>
__device__ __forceinline__ float row_sum(float v, float* shared) {
#pragma unroll
  for (int d = 32; d; d /= 2) v += __shfl_xor(v, d);
  if constexpr (TPR > 64) {
    const int wave = threadIdx.x >> 6;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) shared[wave] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int w = 0; w < TPR / 64; ++w) v += shared[w];
  }
  return v;
}
template <int TPR>
__device__ __forceinline__ void row_sums(float& a, float& b, float* shared) {
#pragma unroll
  for (int d = 32; d; d /= 2) {
    a += __shfl_xor(a, d);
    b += __shfl_xor(b, d);
  }
  if constexpr (TPR > 64) {
    const int wave = threadIdx.x >> 6;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) shared[2 * wave] = a, shared[2 * wave + 1] = b;
    __syncthreads();
    a = b = 0.f;
#pragma unroll
    for (int w = 0; w < TPR / 64; ++w) a += shared[2 * w], b += shared[2 * w + 1];
  }
}

template <int VEC>
__device__ __forceinline__ void load_floats(const float* q, int n, float dflt, float (&f)[VEC]) {
#pragma unroll
  for (int i = 0; i < VEC; ++i) f[i] = dflt;
  if (!q) return;
  if (n >= VEC) {
    __builtin_memcpy(f, q, VEC * 4);
  } else {
#pragma unroll
    for (int i = 0; i < VEC; ++i)
      if (i < n) f[i] = q[i];
  }
}

template <typename T, int TPR, int V>
__global__ __launch_bounds__(TPR > 256 ? TPR : 256) void norm_kernel(const NormParams p) {
  constexpr int VEC = kVec<T>, RPB = TPR >= 256 ? 1 : 256 / TPR;
  __shared__ float shared[32];
  const int sub = RPB == 1 ? 0 : (int)threadIdx.x / TPR, t = (int)threadIdx.x % TPR;
  // (a row's lanes stay together: barriers only where a workgroup takes one row at a time)
  for (int64_t row = (int64_t)blockIdx.x * RPB + sub; row < p.rows; row += (int64_t)gridDim.x * RPB) {
  const T* x = (const T*)p.x + row * p.x_row;
  float f[V][VEC], sum = 0.f;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int c = (v * TPR + t) * VEC;
    unpack<T>(load_piece<T>(x + c, p.features - c), f[v]);
#pragma unroll
    for (int i = 0; i < VEC; ++i) sum += f[v][i];
  }
  const float mean = row_sum<TPR>(sum, shared) / (float)p.features;
  float sq = 0.f;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int c = (v * TPR + t) * VEC;
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      f[v][i] -= mean;
      sq += c + i < p.features ? f[v][i] * f[v][i] : 0.f;
    }
  }
  const float rstd = 1.f / sqrtf(row_sum<TPR>(sq, shared) / (float)p.features + p.eps);
  T* y = (T*)p.y + row * p.y_row;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int c = (v * TPR + t) * VEC, n = p.features - c;
    if (n <= 0) continue;
    float g[VEC], b[VEC];
    load_floats<VEC>(p.gamma ? p.gamma + c : nullptr, n, 1.f, g);
    load_floats<VEC>(p.beta ? p.beta + c : nullptr, n, 0.f, b);
#pragma unroll
    for (int i = 0; i < VEC; ++i) g[i] = f[v][i] * rstd * g[i] + b[i];
    store_piece<T>(y + c, pack<T>(g), n);
  }
  if (t == 0) {
    if (p.mean) p.mean[row] = mean;
    if (p.rstd) p.rstd[row] = rstd;
  }
  }
}

template <typename T, int TPR, int V>
__global__ __launch_bounds__(TPR > 256 ? TPR : 256) void norm_backward_kernel(const NormParams p) {
  constexpr int VEC = kVec<T>, RPB = TPR >= 256 ? 1 : 256 / TPR;
  __shared__ float shared[64];
  __shared__ float sums[RPB > 1 ? 2 * V * TPR * VEC : 1];
  const int sub = RPB == 1 ? 0 : (int)threadIdx.x / TPR, t = (int)threadIdx.x % TPR;
  float dg[V][VEC], db[V][VEC], gamma[V][VEC];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int c = (v * TPR + t) * VEC;
    load_floats<VEC>(p.gamma ? p.gamma + c : nullptr, p.features - c, 1.f, gamma[v]);
#pragma unroll
    for (int i = 0; i < VEC; ++i) dg[v][i] = db[v][i] = 0.f;
  }
  const float over = 1.f / (float)p.features;
  for (int64_t row = (int64_t)blockIdx.x * RPB + sub; row < p.rows; row += (int64_t)gridDim.x * RPB) {
    const T *x = (const T*)p.x + row * p.x_row, *dy = (const T*)p.dy + row * p.y_row;
    u32x4 xv[V], dv[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int c = (v * TPR + t) * VEC;
      xv[v] = load_piece<T>(x + c, p.features - c);
      dv[v] = load_piece<T>(dy + c, p.features - c);
    }
    const float mean = p.mean_in[row], rstd = p.rstd_in[row];
    float s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      float h[VEC], d[VEC];
      unpack<T>(xv[v], h);
      unpack<T>(dv[v], d);
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        h[i] = (h[i] - mean) * rstd;
        const float g = d[i] * gamma[v][i];
        s1 += g;
        s2 += g * h[i];
        dg[v][i] += d[i] * h[i];
        db[v][i] += d[i];
      }
    }
    if (!p.dx) continue;     // uniform
    row_sums<TPR>(s1, s2, shared);
    s1 *= over;
    s2 *= over;
    T* dx = (T*)p.dx + row * p.x_row;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int c = (v * TPR + t) * VEC;
      if (c >= p.features) continue;
      float h[VEC], d[VEC];
      unpack<T>(xv[v], h);
      unpack<T>(dv[v], d);
#pragma unroll
      for (int i = 0; i < VEC; ++i) d[i] = rstd * (d[i] * gamma[v][i] - s1 - (h[i] - mean) * rstd * s2);
      store_piece<T>(dx + c, pack<T>(d), p.features - c);
    }
  }
  if (!p.dgamma && !p.dbeta) return;
  // one row of sums per workgroup: its wavefronts' in turn
  if constexpr (RPB > 1) {
    for (int w = 0; w < RPB; ++w) {
      if (sub == w) {
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
          for (int i = 0; i < VEC; ++i) {
            float* at = sums + ((v * TPR + t) * VEC + i) * 2;
            at[0] = w ? at[0] + dg[v][i] : dg[v][i];
            at[1] = w ? at[1] + db[v][i] : db[v][i];
          }
      }
      __syncthreads();
    }
    if (sub) return;
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        const float* at = sums + ((v * TPR + t) * VEC + i) * 2;
        dg[v][i] = at[0];
        db[v][i] = at[1];
      }
  }
  float* to_g = p.blocks > 1 ? p.partial + (int64_t)blockIdx.x * 2 * p.features : p.dgamma;
  float* to_b = p.blocks > 1 ? p.partial + ((int64_t)blockIdx.x * 2 + 1) * p.features : p.dbeta;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int c = (v * TPR + t) * VEC;
#pragma unroll
    for (int i = 0; i < VEC; ++i)
      if (c + i < p.features) {
        if (to_g) to_g[c + i] = dg[v][i];
        if (to_b) to_b[c + i] = db[v][i];
      }
  }
}

// The workgroups' rows of sums, added in their order: 64 columns of dgamma or dbeta (blockIdx.y), four wavefronts.
__global__ __launch_bounds__(256) void norm_sums_kernel(const float* __restrict__ partial, float* __restrict__ dgamma, float* __restrict__ dbeta, int features,
                                                        int blocks) {
  __shared__ float part[4][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t c = (int64_t)blockIdx.x * 64 + lane;
  float* to = blockIdx.y ? dbeta : dgamma;
  if (!to) return;
  float s = 0.f;
  if (c < features) {
#pragma unroll 8
    for (int b = wave; b < blocks; b += 4) s += partial[((int64_t)b * 2 + blockIdx.y) * features + c];
  }
  part[wave][lane] = s;
  __syncthreads();
  if (wave == 0 && c < features) to[c] = (part[0][lane] + part[1][lane]) + (part[2][lane] + part[3][lane]);
}

// ---- rows longer than a workgroup's registers: one workgroup to a row, read again for each sum ----
template <typename T>
__global__ __launch_bounds__(1024) void norm_long_kernel(const NormParams p) {
  constexpr int VEC = kVec<T>;
  __shared__ float shared[32];
  for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
  const T* x = (const T*)p.x + row * p.x_row;
  T* y = (T*)p.y + row * p.y_row;
  float sum = 0.f;
  for (int c = threadIdx.x * VEC; c < p.features; c += 1024 * VEC) {
    float f[VEC], part = 0.f;
    unpack<T>(load_piece<T>(x + c, p.features - c), f);
#pragma unroll
    for (int i = 0; i < VEC; ++i) part += f[i];
    sum += part;
  }
  const float mean = row_sum<1024>(sum, shared) / (float)p.features;
  float sq = 0.f;
  for (int c = threadIdx.x * VEC; c < p.features; c += 1024 * VEC) {
    float f[VEC], part = 0.f;
    unpack<T>(load_piece<T>(x + c, p.features - c), f);
#pragma unroll
    for (int i = 0; i < VEC; ++i) part += c + i < p.features ? (f[i] - mean) * (f[i] - mean) : 0.f;
    sq += part;
  }
  const float rstd = 1.f / sqrtf(row_sum<1024>(sq, shared) / (float)p.features + p.eps);
  for (int c = threadIdx.x * VEC; c < p.features; c += 1024 * VEC) {
    const int n = p.features - c;
    float f[VEC], g[VEC], b[VEC];
    unpack<T>(load_piece<T>(x + c, n), f);
    load_floats<VEC>(p.gamma ? p.gamma + c : nullptr, n, 1.f, g);
    load_floats<VEC>(p.beta ? p.beta + c : nullptr, n, 0.f, b);
#pragma unroll
    for (int i = 0; i < VEC; ++i) f[i] = (f[i] - mean) * rstd * g[i] + b[i];
    store_piece<T>(y + c, pack<T>(f), n);
  }
  if (threadIdx.x == 0) {
    if (p.mean) p.mean[row] = mean;
    if (p.rstd) p.rstd[row] = rstd;
  }
  }
}

template <typename T>
__global__ __launch_bounds__(1024) void norm_long_backward_kernel(const NormParams p) {
  constexpr int VEC = kVec<T>;
  __shared__ float shared[64];
  for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
  const T *x = (const T*)p.x + row * p.x_row, *dy = (const T*)p.dy + row * p.y_row;
  T* dx = (T*)p.dx + row * p.x_row;
  const float mean = p.mean_in[row], rstd = p.rstd_in[row];
  float s1 = 0.f, s2 = 0.f;
  for (int c = threadIdx.x * VEC; c < p.features; c += 1024 * VEC) {
    float h[VEC], d[VEC], g[VEC], a = 0.f, b = 0.f;
    unpack<T>(load_piece<T>(x + c, p.features - c), h);
    unpack<T>(load_piece<T>(dy + c, p.features - c), d);
    load_floats<VEC>(p.gamma ? p.gamma + c : nullptr, p.features - c, 1.f, g);
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      a += d[i] * g[i];
      b += d[i] * g[i] * (h[i] - mean) * rstd;
    }
    s1 += a;
    s2 += b;
  }
  row_sums<1024>(s1, s2, shared);
  s1 /= (float)p.features;
  s2 /= (float)p.features;
  for (int c = threadIdx.x * VEC; c < p.features; c += 1024 * VEC) {
    float h[VEC], d[VEC], g[VEC];
    unpack<T>(load_piece<T>(x + c, p.features - c), h);
    unpack<T>(load_piece<T>(dy + c, p.features - c), d);
    load_floats<VEC>(p.gamma ? p.gamma + c : nullptr, p.features - c, 1.f, g);
#pragma unroll
    for (int i = 0; i < VEC; ++i) d[i] = rstd * (d[i] * g[i] - s1 - (h[i] - mean) * rstd * s2);
    store_piece<T>(dx + c, pack<T>(d), p.features - c);
  }
  }
}

// Column sums of long rows: a lane's columns over the rows of its workgroup row (blockIdx.y).
template <typename T>
__global__ __launch_bounds__(256) void norm_long_sums_kernel(const NormParams p) {
  constexpr int VEC = kVec<T>;
  const int64_t c = ((int64_t)blockIdx.x * 256 + threadIdx.x) * VEC;
  if (c >= p.features) return;
  const int n = (int)(p.features - c);
  float dg[VEC], db[VEC];
#pragma unroll
  for (int i = 0; i < VEC; ++i) dg[i] = db[i] = 0.f;
  for (int64_t row = blockIdx.y; row < p.rows; row += p.blocks) {
    float h[VEC], d[VEC];
    unpack<T>(load_piece<T>((const T*)p.x + row * p.x_row + c, n), h);
    unpack<T>(load_piece<T>((const T*)p.dy + row * p.y_row + c, n), d);
    const float mean = p.mean_in[row], rstd = p.rstd_in[row];
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      dg[i] += d[i] * ((h[i] - mean) * rstd);
      db[i] += d[i];
    }
  }
  float* to_g = p.blocks > 1 ? p.partial + (int64_t)blockIdx.y * 2 * p.features : p.dgamma;
  float* to_b = p.blocks > 1 ? p.partial + ((int64_t)blockIdx.y * 2 + 1) * p.features : p.dbeta;
#pragma unroll
  for (int i = 0; i < VEC; ++i)
    if (i < n) {
      if (to_g) to_g[c + i] = dg[i];
      if (to_b) to_b[c + i] = db[i];
    }
}

// A launch holds fewer than 2^32 lanes: workgroups beyond these many rows take several.
unsigned row_blocks(int64_t rows) { return (unsigned)(rows < (1 << 20) ? rows : 1 << 20); }

// Elements a lane holds, features beyond which a row is read several times.  A lane of 1024 has 128 registers, which its sums of the
// backward pass would fill by themselves.
constexpr int kPerLane = 32, kLong = 1024 * kPerLane, kLongBackward = kLong / 2;

int lanes_of(int64_t features) { return features <= 64 * kPerLane ? 64 : features <= 256 * kPerLane ? 256 : 1024; }

template <typename T, typename F>
void with_shape(int64_t features, F&& go) {
  const int lanes = lanes_of(features), pieces = (int)((features + lanes * kVec<T> - 1) / (lanes * kVec<T>));
  auto with_lanes = [&](auto tpr) {
    constexpr int TPR = decltype(tpr)::value;
    if (pieces <= 1) go(std::integral_constant<int, TPR>{}, std::integral_constant<int, 1>{});
    else if (pieces <= 2) go(std::integral_constant<int, TPR>{}, std::integral_constant<int, 2>{});
    else if (sizeof(T) == 2 || pieces <= 4) go(std::integral_constant<int, TPR>{}, std::integral_constant<int, 4>{});
    else if constexpr (sizeof(T) == 4) go(std::integral_constant<int, TPR>{}, std::integral_constant<int, 8>{});
  };
  if (lanes == 64) with_lanes(std::integral_constant<int, 64>{});
  else if (lanes == 256) with_lanes(std::integral_constant<int, 256>{});
  else with_lanes(std::integral_constant<int, 1024>{});
}

template <typename T>
hipError_t forward_t(const NormParams& p, hipStream_t stream) {
  if (p.features > kLong) {
    norm_long_kernel<T><<<dim3(row_blocks(p.rows)), dim3(1024), 0, stream>>>(p);
    return hipGetLastError();
  }
  with_shape<T>(p.features, [&](auto tpr, auto v) {
    constexpr int TPR = decltype(tpr)::value, V = decltype(v)::value, RPB = TPR >= 256 ? 1 : 256 / TPR;
    norm_kernel<T, TPR, V><<<dim3(row_blocks((p.rows + RPB - 1) / RPB)), dim3(TPR > 256 ? TPR : 256), 0, stream>>>(p);
  });
  return hipGetLastError();
}

template <typename T>
hipError_t backward_t(const NormParams& p, hipStream_t stream) {
  if (p.features > kLongBackward) {
    if (p.dx && p.rows) norm_long_backward_kernel<T><<<dim3(row_blocks(p.rows)), dim3(1024), 0, stream>>>(p);
    if (p.dgamma || p.dbeta)
      norm_long_sums_kernel<T><<<dim3((unsigned)((p.features + 256 * kVec<T> - 1) / (256 * kVec<T>)), (unsigned)p.blocks), dim3(256), 0, stream>>>(p);
  } else {
    with_shape<T>(p.features, [&](auto tpr, auto v) {
      constexpr int TPR = decltype(tpr)::value, V = TPR == 1024 ? std::min(decltype(v)::value, kLongBackward / 1024 / kVec<T>) : decltype(v)::value;
      norm_backward_kernel<T, TPR, V><<<dim3((unsigned)p.blocks), dim3(TPR > 256 ? TPR : 256), 0, stream>>>(p);
    });
  }
  if ((p.dgamma || p.dbeta) && p.blocks > 1)
    norm_sums_kernel<<<dim3((unsigned)((p.features + 63) / 64), 2), dim3(256), 0, stream>>>(p.partial, p.dgamma, p.dbeta, p.features, p.blocks);
  return hipGetLastError();
}

}  // namespace

int norm_backward_blocks(int64_t rows, int64_t features, int dtype) {
  (void)dtype;
  const int64_t at_once = lanes_of(features) == 64 ? 4 : 1, groups = (rows + at_once - 1) / at_once;
  return (int)(groups < 1 ? 1 : groups < 512 ? groups : 512);
}

hipError_t launch_norm(int dtype, const NormParams& p, hipStream_t stream) {
  return dtype == STRIPE_F32 ? forward_t<float>(p, stream) : forward_t<__bf16>(p, stream);
}

hipError_t launch_norm_backward(int dtype, const NormParams& p, hipStream_t stream) {
  return dtype == STRIPE_F32 ? backward_t<float>(p, stream) : backward_t<__bf16>(p, stream);
}

}  // namespace stripe
