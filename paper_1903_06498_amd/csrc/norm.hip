// Layer norm, forward and backward (gfx950).  What bounds it is memory: 16384 x 4096 bf16 51 us forward (5.25 TB/s; a plain copy of 1 GiB: 4.5), 79 us
// backward (5.1); 8192 x 8192 51 and 85.
//
// Each row is read once into registers: 64, 256 or 512 lanes share a row, at most 32 elements each (longer rows are read again for
// each sum).  Mean first, then the mean of the squared distances from it -- not E[x^2] - E[x]^2, which loses
// what the mean's square has more digits than -- together with the mean distance, which is the first mean's rounding error, up to n 2^-24 |x| for its n
// additions: without it, 16384 equal fp32 values 1000.1 came out as 0.1 gamma + beta (1000 of them: 0.04).  Rows of bf16 do without it where they stay in
// registers (16384 x 4096 takes 6 % longer with it, 32768 x 512 13 %; fp32 up to 2 %): where their spread is small beside their mean, the values are
// multiples of 2^-9 of the largest, and sums of up to 2^15 of them are exact in fp32.  The backward pass keeps its columns' sums of dy h and dy in registers over all the
// rows that its workgroup takes, leaves one row of partial sums per workgroup and adds those in a second launch in a fixed order.
#include <algorithm>

#include "layers_device.hpp"

namespace stripe {
namespace {

// Sums over the TPR lanes that share a row; all of them get them.  `shared`: 2 x 32 floats, which consecutive calls of a workgroup take in turn (a
// wavefront that is one call ahead writes the other half; two ahead it cannot be, as each call has a barrier).
template <int TPR>
__device__ __forceinline__ void row_sums(float& a, float& b, float (*shared)[32], int turn) {
  a = wave_sum(a);
  b = wave_sum(b);
  if constexpr (TPR > 64) {
    constexpr int W = TPR / 64;
    const int wave = threadIdx.x >> 6;
    float* s = shared[turn & 1];
    if ((threadIdx.x & 63) == 0) s[2 * wave] = a, s[2 * wave + 1] = b;
    __syncthreads();
    a = b = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w) a += s[2 * w], b += s[2 * w + 1];
  }
}
template <int TPR>
__device__ __forceinline__ float row_sum(float a, float (*shared)[32], int turn) {
  a = wave_sum(a);
  if constexpr (TPR > 64) {
    float* s = shared[turn & 1];
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = a;
    __syncthreads();
    a = 0.f;
#pragma unroll
    for (int w = 0; w < TPR / 64; ++w) a += s[w];
  }
  return a;
}

// s from the sums of the squared distances from the first mean and of the distances themselves, and the mean without its error.  (Where the squares do
// not end finite -- infinities, NaN, distances from 2^64 on -- both stay what they are without a correction.)
__device__ __forceinline__ float inverse_spread(float sq, float off, int features, float eps, float& mean) {
  const float v = sq / (float)features, o = v < __builtin_inff() ? off / (float)features : 0.f, var = v - o * o;
  mean += o;
  return 1.f / sqrtf((var < 0.f ? 0.f : var) + eps);
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

// A workgroup takes rows one grid apart, gamma and beta stay in registers (they are fp32, twice or four times a bf16 row: read for each row again they
// were what 16384 x 4096 waited for, 74 us), and the next row is on its way while one is summed.
template <typename T, int TPR, int V>
__global__ __launch_bounds__(TPR > 256 ? TPR : 256) void norm_kernel(const NormParams p) {
  constexpr int VEC = kVec<T>, RPB = TPR >= 256 ? 1 : 256 / TPR;
  constexpr bool CORRECT = sizeof(T) == 4;
  __shared__ float shared[2][32];
  const int sub = RPB == 1 ? 0 : (int)threadIdx.x / TPR, t = (int)threadIdx.x % TPR;
  const int64_t step = (int64_t)gridDim.x * RPB;
  int64_t row = (int64_t)blockIdx.x * RPB + sub;
  u32x4 next[V];
  auto load = [&](int64_t r) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int c = (v * TPR + t) * VEC;
      next[v] = load_piece<T>((const T*)p.x + r * p.x_row + c, p.features - c);
    }
  };
  if (row < p.rows) load(row);
  float gamma[V][VEC], beta[V][VEC];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int c = (v * TPR + t) * VEC;
    load_floats<VEC>(p.gamma ? p.gamma + c : nullptr, p.features - c, 1.f, gamma[v]);
    load_floats<VEC>(p.beta ? p.beta + c : nullptr, p.features - c, 0.f, beta[v]);
  }
  // (a row's lanes stay together: barriers only where a workgroup takes one row at a time)
  int turn = 0;
  for (; row < p.rows; row += step) {
    u32x4 now[V];
    float sum = 0.f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      now[v] = next[v];
      float f[VEC];
      unpack<T>(now[v], f);
#pragma unroll
      for (int i = 0; i < VEC; ++i) sum += f[i];
    }
    if (row + step < p.rows) load(row + step);
    float mean = row_sum<TPR>(sum, shared, turn++) / (float)p.features;
    float sq = 0.f, off = 0.f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int c = (v * TPR + t) * VEC;
      float f[VEC];
      unpack<T>(now[v], f);
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        const float d = f[i] - mean;
        sq += c + i < p.features ? d * d : 0.f;
        if constexpr (CORRECT) off += c + i < p.features ? d : 0.f;
      }
    }
    float rstd;
    if constexpr (CORRECT) {
      row_sums<TPR>(sq, off, shared, turn++);
      rstd = inverse_spread(sq, off, p.features, p.eps, mean);
    } else {
      rstd = 1.f / sqrtf(row_sum<TPR>(sq, shared, turn++) / (float)p.features + p.eps);
    }
    T* y = (T*)p.y + row * p.y_row;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int c = (v * TPR + t) * VEC;
      if (c >= p.features) continue;
      float f[VEC];
      unpack<T>(now[v], f);
#pragma unroll
      for (int i = 0; i < VEC; ++i) f[i] = (f[i] - mean) * rstd * gamma[v][i] + beta[v][i];
      store_piece<T>(y + c, pack<T>(f), p.features - c);
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
  __shared__ float shared[2][32];
  __shared__ float sums[RPB > 1 ? 2 * V * TPR * VEC : 1];
  const int sub = RPB == 1 ? 0 : (int)threadIdx.x / TPR, t = (int)threadIdx.x % TPR;
  float dg[V][VEC], db[V][VEC], gamma[V][VEC];
  const float over = 1.f / (float)p.features;
  const int64_t step = (int64_t)gridDim.x * RPB;
  int64_t row = (int64_t)blockIdx.x * RPB + sub;
  u32x4 next_x[V], next_d[V];
  float next_mean = 0.f, next_rstd = 0.f;
  auto load = [&](int64_t r) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int c = (v * TPR + t) * VEC;
      next_x[v] = load_piece<T>((const T*)p.x + r * p.x_row + c, p.features - c);
      next_d[v] = load_piece<T>((const T*)p.dy + r * p.y_row + c, p.features - c);
    }
    next_mean = p.mean_in[r];
    next_rstd = p.rstd_in[r];
  };
  if (row < p.rows) load(row);
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int c = (v * TPR + t) * VEC;
    load_floats<VEC>(p.gamma ? p.gamma + c : nullptr, p.features - c, 1.f, gamma[v]);
#pragma unroll
    for (int i = 0; i < VEC; ++i) dg[v][i] = db[v][i] = 0.f;
  }
  int turn = 0;
  for (; row < p.rows; row += step) {
    u32x4 xv[V], dv[V];
#pragma unroll
    for (int v = 0; v < V; ++v) xv[v] = next_x[v], dv[v] = next_d[v];
    const float mean = next_mean, rstd = next_rstd;
    if (row + step < p.rows) load(row + step);
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
    row_sums<TPR>(s1, s2, shared, turn++);
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

// The workgroups' rows of sums, added in their order: 64 columns of dgamma or dbeta (blockIdx.y), sixteen wavefronts.
__global__ __launch_bounds__(1024) void norm_sums_kernel(const float* __restrict__ partial, float* __restrict__ dgamma, float* __restrict__ dbeta, int features,
                                                         int blocks) {
  __shared__ float part[16][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t c = (int64_t)blockIdx.x * 64 + lane;
  float* to = blockIdx.y ? dbeta : dgamma;
  if (!to) return;
  float s = 0.f;
  if (c < features) {
#pragma unroll 16
    for (int b = wave; b < blocks; b += 16) s += partial[((int64_t)b * 2 + blockIdx.y) * features + c];
  }
  part[wave][lane] = s;
  __syncthreads();
  if (wave || c >= features) return;
  s = 0.f;
#pragma unroll
  for (int w = 0; w < 16; ++w) s += part[w][lane];
  to[c] = s;
}

// ---- rows longer than a workgroup's registers: one workgroup to a row, read again for each sum ----
template <typename T>
__global__ __launch_bounds__(1024) void norm_long_kernel(const NormParams p) {
  constexpr int VEC = kVec<T>;
  __shared__ float shared[2][32];
  int turn = 0;
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
    float mean = row_sum<1024>(sum, shared, turn++) / (float)p.features;
    float sq = 0.f, off = 0.f;
    for (int c = threadIdx.x * VEC; c < p.features; c += 1024 * VEC) {
      float f[VEC], part = 0.f, part_off = 0.f;
      unpack<T>(load_piece<T>(x + c, p.features - c), f);
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        const float d = c + i < p.features ? f[i] - mean : 0.f;
        part_off += d;
        part += d * d;
      }
      off += part_off;
      sq += part;
    }
    row_sums<1024>(sq, off, shared, turn++);
    const float rstd = inverse_spread(sq, off, p.features, p.eps, mean);
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
  __shared__ float shared[2][32];
  int turn = 0;
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
    row_sums<1024>(s1, s2, shared, turn++);
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

// Features beyond which a row is read several times; the lanes that share a shorter one: a lane holds up to 32 elements, in the backward pass, whose
// sums take twice as many registers again, 16 where 512 lanes suffice for that.
constexpr int kLong = 16384;

int lanes_of(int64_t features, bool backward) {
  if (backward) return features <= 1024 ? 64 : features <= 4096 ? 256 : 512;
  return features <= 2048 ? 64 : features <= 8192 ? 256 : 512;
}

template <typename T, typename F>
void with_shape(int64_t features, bool backward, F&& go) {
  const int lanes = lanes_of(features, backward), pieces = (int)((features + lanes * kVec<T> - 1) / (lanes * kVec<T>));
  auto with_lanes = [&](auto tpr) {
    constexpr int TPR = decltype(tpr)::value;
    if (pieces <= 1) go(std::integral_constant<int, TPR>{}, std::integral_constant<int, 1>{});
    else if (pieces <= 2) go(std::integral_constant<int, TPR>{}, std::integral_constant<int, 2>{});
    else if (sizeof(T) == 2 || pieces <= 4) go(std::integral_constant<int, TPR>{}, std::integral_constant<int, 4>{});
    else if constexpr (sizeof(T) == 4) go(std::integral_constant<int, TPR>{}, std::integral_constant<int, 8>{});
  };
  if (lanes == 64) with_lanes(std::integral_constant<int, 64>{});
  else if (lanes == 256) with_lanes(std::integral_constant<int, 256>{});
  else with_lanes(std::integral_constant<int, 512>{});
}

template <typename T>
hipError_t forward_t(const NormParams& p, hipStream_t stream) {
  if (p.features > kLong) {
    norm_long_kernel<T><<<dim3(row_blocks(p.rows)), dim3(1024), 0, stream>>>(p);
    return hipGetLastError();
  }
  with_shape<T>(p.features, false, [&](auto tpr, auto v) {
    constexpr int TPR = decltype(tpr)::value, V = decltype(v)::value, RPB = TPR >= 256 ? 1 : 256 / TPR;
    // as many workgroups as stay on the chip, where a lane holds 32 elements two for each CU (8192 x 8192 bf16: 51 us, 56 with four), else four
    // (16384 x 4096: 51, 62 with two)
    const int64_t blocks = (p.rows + RPB - 1) / RPB, most = V * kVec<T> > 16 ? 512 : 1024;
    norm_kernel<T, TPR, V><<<dim3((unsigned)(blocks < most ? blocks : most)), dim3(TPR > 256 ? TPR : 256), 0, stream>>>(p);
  });
  return hipGetLastError();
}

template <typename T>
hipError_t backward_t(const NormParams& p, hipStream_t stream) {
  if (p.features > kLong) {
    if (p.dx && p.rows) norm_long_backward_kernel<T><<<dim3(row_blocks(p.rows)), dim3(1024), 0, stream>>>(p);
    if (p.dgamma || p.dbeta)
      norm_long_sums_kernel<T><<<dim3((unsigned)((p.features + 256 * kVec<T> - 1) / (256 * kVec<T>)), (unsigned)p.blocks), dim3(256), 0, stream>>>(p);
  } else {
    with_shape<T>(p.features, true, [&](auto tpr, auto v) {
      constexpr int TPR = decltype(tpr)::value, V = decltype(v)::value;
      norm_backward_kernel<T, TPR, V><<<dim3((unsigned)p.blocks), dim3(TPR > 256 ? TPR : 256), 0, stream>>>(p);
    });
  }
  if ((p.dgamma || p.dbeta) && p.blocks > 1)
    norm_sums_kernel<<<dim3((unsigned)((p.features + 63) / 64), 2), dim3(1024), 0, stream>>>(p.partial, p.dgamma, p.dbeta, p.features, p.blocks);
  return hipGetLastError();
}

}  // namespace

// Each workgroup leaves 8 bytes for each feature, to be read again: one for each CU; two where rows are short and there are many (8192 x 8192 bf16: 85 us,
// 95 with two; 32768 x 512: 31 and 26; 1537 x 1000 fp32: 10.9 and 13.2).  Rows too long for registers are summed in strips of 256 lanes, by as many
// workgroups to a strip as make about 1024 of all strips: the sums take at most 16 MB, and the two launches
// 23.5 us at 300 x 20000 bf16 (38 with 256 to a strip; 16.3 with half as many), 222 at 16384 x 20000 (256; 268), 190 at 512 x 2^18 fp32 (405;
// 215), 235 at 256 x 2^20 bf16 (1735 and 2 GB of sums; 204).
int norm_backward_blocks(int64_t rows, int64_t features, int dtype) {
  if (features > kLong) {
    const int64_t lane = dtype == STRIPE_F32 ? 4 : 8, strips = (features + 256 * lane - 1) / (256 * lane);
    return (int)std::max<int64_t>(1, std::min<int64_t>(rows, 1024 / strips));
  }
  const int64_t at_once = lanes_of(features, true) == 64 ? 4 : 1, groups = (rows + at_once - 1) / at_once;
  const int64_t most = features * (dtype == STRIPE_F32 ? 4 : 2) <= 4096 && groups >= 16 * 512 ? 512 : 256;
  return (int)(groups < 1 ? 1 : groups < most ? groups : most);
}

hipError_t launch_norm(int dtype, const NormParams& p, hipStream_t stream) {
  return dtype == STRIPE_F32 ? forward_t<float>(p, stream) : forward_t<__bf16>(p, stream);
}

hipError_t launch_norm_backward(int dtype, const NormParams& p, hipStream_t stream) {
  return dtype == STRIPE_F32 ? backward_t<float>(p, stream) : backward_t<__bf16>(p, stream);
}

}  // namespace stripe
