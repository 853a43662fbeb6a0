// Device helpers that the layer operators' kernels share: elements, activations, rows sorted by group.
#pragma once

#include <hip/hip_runtime.h>

#include <type_traits>

#include "layers.hpp"

namespace stripe {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// ---- 16-byte pieces of a row -------------------------------------------------
template <typename T>
constexpr int kVec = 16 / sizeof(T);

// The first n of the elements at q as a 16-byte piece, zeros behind them.  Rows may start at any element: a whole piece is
// one 16-byte load at whatever address.
template <typename T>
__device__ __forceinline__ u32x4 load_piece(const T* q, int n) {
  u32x4 v = {0, 0, 0, 0};
  if (n >= kVec<T>) {
    __builtin_memcpy(&v, q, 16);
  } else {
    T e[kVec<T>];
#pragma unroll
    for (int i = 0; i < kVec<T>; ++i) e[i] = i < n ? q[i] : (T)0.f;
    __builtin_memcpy(&v, e, 16);
  }
  return v;
}
template <typename T>
__device__ __forceinline__ void store_piece(T* q, u32x4 v, int n) {
  if (n >= kVec<T>) {
    __builtin_memcpy(q, &v, 16);
  } else {
    T e[kVec<T>];
    __builtin_memcpy(e, &v, 16);
#pragma unroll
    for (int i = 0; i < kVec<T>; ++i)
      if (i < n) q[i] = e[i];
  }
}
template <typename T>
__device__ __forceinline__ void unpack(u32x4 v, float (&f)[kVec<T>]) {
  T e[kVec<T>];
  __builtin_memcpy(e, &v, 16);
#pragma unroll
  for (int i = 0; i < kVec<T>; ++i) f[i] = (float)e[i];
}
// fp32 to the element type: bf16 to nearest even, NaN kept
template <typename T>
__device__ __forceinline__ u32x4 pack(const float (&f)[kVec<T>]) {
  T e[kVec<T>];
#pragma unroll
  for (int i = 0; i < kVec<T>; ++i) e[i] = (T)f[i];
  u32x4 v;
  __builtin_memcpy(&v, e, 16);
  return v;
}

// ---- sums over a wavefront -------------------------------------------------------
// In the same order in every call; every lane gets the total.  Six additions whose second operand comes through the lanes' crossbar (a shuffle
// through LDS hardware takes ten times as long).
__device__ __forceinline__ float wave_sum(float v) {
  auto from = [](float x, auto ctrl, auto rows) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), decltype(ctrl)::value, decltype(rows)::value, 0xf, true));
  };
  using std::integral_constant;
  v += from(v, integral_constant<int, 0xb1>{}, integral_constant<int, 0xf>{});       // lane ^ 1
  v += from(v, integral_constant<int, 0x4e>{}, integral_constant<int, 0xf>{});       // lane ^ 2
  v += from(v, integral_constant<int, 0x141>{}, integral_constant<int, 0xf>{});      // mirrored within 8
  v += from(v, integral_constant<int, 0x140>{}, integral_constant<int, 0xf>{});      // mirrored within 16
  v += from(v, integral_constant<int, 0x142>{}, integral_constant<int, 0xa>{});      // rows 0 and 2 of 16 lanes into rows 1 and 3
  v += from(v, integral_constant<int, 0x143>{}, integral_constant<int, 0xc>{});      // the lower half into the upper
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
}

// ---- activations ---------------------------------------------------------------
// In a bf16 pipeline the hardware's exponential and reciprocal (2 ulp of fp32) are far inside the result's rounding.  Results below 2^-118 in size may come
// out as 0: exp(-z) overflows, or its reciprocal is subnormal.
template <typename T>
__device__ __forceinline__ float exp_of(float v) {
  if constexpr (sizeof(T) == 2) return __builtin_amdgcn_exp2f(v * 1.44269504f);
  else return expf(v);
}
template <typename T>
__device__ __forceinline__ float inv(float v) {
  if constexpr (sizeof(T) == 2) return __builtin_amdgcn_rcpf(v);
  else return 1.f / v;
}

constexpr float kGeluA = 0.7978845608f, kGeluB = 0.044715f;   // sqrt(2/pi)

// The normal distribution function; *density: exp(-z^2 / 2).  fp32: the library's erfc.  bf16 (2048 x 4096 outputs: 36 us of a forward pass less):
// exp(-z^2 / 2) g(|z|) on the negative side, 1 - that on the other, g(a) = exp(a^2 / 2) erfc(a / sqrt(2)) / 2.  g falls like 1 / a, and so does
// t = 1 / (1 + 0.2928 a): a polynomial of degree 6 in t without a constant, fitted (by linear programming, to the smallest largest deviation on
// 0 .. 14) for what is left to be at most 7e-8 of 1 and at most 2^-14 of g itself, so that the small values of the tail are within bf16's rounding too.
template <typename T>
__device__ __forceinline__ float normal_cdf(float z, float* density) {
  *density = exp_of<T>(-0.5f * z * z);
  if constexpr (sizeof(T) == 2) {
    const float t = __builtin_amdgcn_rcpf(1.f + 0.292774067f * __builtin_fabsf(z));
    const float tail = t * (0.117673576f + t * (0.105071628f + t * (0.167696047f + t * (-0.0698138839f + t * (0.265270169f + t * -0.0858976065f))))) * *density;
    return z < 0.f ? tail : 1.f - tail;
  } else {
    return 0.5f * erfcf(-0.70710678f * z);
  }
}

template <typename T>
__device__ __forceinline__ float activate(float z, int act) {
  switch (act) {
    case STRIPE_ACT_RELU: return z > 0.f ? z : (z != z ? z : 0.f);
    case STRIPE_ACT_GELU: {
      float density;
      return z * normal_cdf<T>(z, &density);
    }
    case STRIPE_ACT_GELU_TANH: return z * inv<T>(1.f + exp_of<T>(-2.f * kGeluA * (z + kGeluB * z * z * z)));
    case STRIPE_ACT_SILU: return z * inv<T>(1.f + exp_of<T>(-z));
    default: return z;
  }
}
template <typename T>
__device__ __forceinline__ float slope(float z, int act) {
  switch (act) {
    case STRIPE_ACT_RELU: return z > 0.f ? 1.f : 0.f;
    case STRIPE_ACT_GELU: {
      float density;
      const float p = normal_cdf<T>(z, &density);
      return p + z * 0.3989422804f * density;
    }
    case STRIPE_ACT_GELU_TANH: {
      const float s = inv<T>(1.f + exp_of<T>(-2.f * kGeluA * (z + kGeluB * z * z * z)));
      const float c = __builtin_amdgcn_fmed3f(z, -100.f, 100.f);      // beyond, s (1 - s) is 0, and z^2 may overflow
      return s + c * s * (1.f - s) * 2.f * kGeluA * (1.f + 3.f * kGeluB * c * c);
    }
    case STRIPE_ACT_SILU: {
      const float s = inv<T>(1.f + exp_of<T>(-z));
      return s * (1.f + z * (1.f - s));
    }
    default: return 1.f;
  }
}

// Several values: one branch for all of them.
template <typename F>
__device__ __forceinline__ void with_activation(int act, F&& go) {
  switch (act) {
    case STRIPE_ACT_RELU: return go(std::integral_constant<int, STRIPE_ACT_RELU>{});
    case STRIPE_ACT_GELU: return go(std::integral_constant<int, STRIPE_ACT_GELU>{});
    case STRIPE_ACT_GELU_TANH: return go(std::integral_constant<int, STRIPE_ACT_GELU_TANH>{});
    case STRIPE_ACT_SILU: return go(std::integral_constant<int, STRIPE_ACT_SILU>{});
    default: return;
  }
}
template <typename T>
__device__ __forceinline__ void activate8(float (&v)[8], int act) {
  with_activation(act, [&](auto a) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = activate<T>(v[e], decltype(a)::value);
  });
}
template <typename T, int N>
__device__ __forceinline__ void times_slope(float (&d)[N], const float (&z)[N], int act) {
  with_activation(act, [&](auto a) {
#pragma unroll
    for (int e = 0; e < N; ++e) d[e] *= slope<T>(z[e], decltype(a)::value);
  });
}

// ---- rows sorted by group -------------------------------------------------------
// Rows of group g: bound(g) .. bound(g + 1) - 1, bound(i) = the running maximum of offsets[0 .. i], limited to 0 .. rows.
// The lanes of a wavefront look at 64 groups at a time.
struct GroupChunk {
  int start, end;     // of this lane's group (empty beyond the last)
  int tiles, through; // its tiles of `height` rows, and those of all groups up to and with it
};
__device__ __forceinline__ int limited(int v, int rows) { return v < 0 ? 0 : v > rows ? rows : v; }

__device__ __forceinline__ GroupChunk group_chunk(const int32_t* offsets, int groups, int rows, int base, int carry_end, int carry_tiles, int height) {
  const int lane = threadIdx.x & 63, g = base + lane;
  int end = g < groups ? limited(offsets[g + 1], rows) : 0;
  end = end > carry_end ? end : carry_end;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int o = __shfl_up(end, d);
    if (lane >= d && o > end) end = o;
  }
  GroupChunk c;
  c.end = end;
  const int before = __shfl_up(end, 1);
  c.start = lane ? before : carry_end;
  c.tiles = (c.end - c.start + height - 1) / height;
  int sum = c.tiles;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int o = __shfl_up(sum, d);
    if (lane >= d) sum += o;
  }
  c.through = carry_tiles + sum;
  return c;
}
__device__ __forceinline__ int lane_value(int v, int lane) { return __builtin_amdgcn_readlane(v, lane); }

struct RowTile {
  int group, row0, rows;   // first row, rows of the tile (at most height)
};
// Of a chunk of groups from number `base` on, the tile number t if it is among them.
__device__ __forceinline__ bool tile_in_chunk(const GroupChunk& c, int base, int height, int t, RowTile* r) {
  const uint64_t past = __ballot(c.through > t);
  if (!past) return false;
  const int at = __builtin_ctzll(past);
  const int first = t - (lane_value(c.through, at) - lane_value(c.tiles, at));
  r->group = base + at;
  r->row0 = lane_value(c.start, at) + first * height;
  const int left = lane_value(c.end, at) - r->row0;
  r->rows = left < height ? left : height;
  return true;
}
// All groups' tiles of `height` rows.
__device__ __forceinline__ int count_row_tiles(const int32_t* offsets, int groups, int rows, int height) {
  int end = limited(offsets[0], rows), tiles = 0;
  for (int base = 0; base < groups; base += 64) {
    const GroupChunk c = group_chunk(offsets, groups, rows, base, end, tiles, height);
    end = lane_value(c.end, 63);
    tiles = lane_value(c.through, 63);
  }
  return tiles;
}
// The tile number `t`; no rows if there are not that many.
__device__ __forceinline__ RowTile find_row_tile(const int32_t* offsets, int groups, int rows, int height, int t) {
  int end = limited(offsets[0], rows), tiles = 0;
  RowTile r = {0, 0, 0};
  for (int base = 0; base < groups; base += 64) {
    const GroupChunk c = group_chunk(offsets, groups, rows, base, end, tiles, height);
    if (tile_in_chunk(c, base, height, t, &r)) return r;
    end = lane_value(c.end, 63);
    tiles = lane_value(c.through, 63);
  }
  return r;
}
// Rows of one group, and the number of tiles of the groups before it.
__device__ __forceinline__ void group_rows(const int32_t* offsets, int groups, int rows, int group, int height, int* start, int* end_out, int* tiles_before) {
  int end = limited(offsets[0], rows), tiles = 0;
  for (int base = 0;; base += 64) {
    const GroupChunk c = group_chunk(offsets, groups, rows, base, end, tiles, height);
    if (group < base + 64) {
      const int at = group - base;
      *start = lane_value(c.start, at);
      *end_out = lane_value(c.end, at);
      *tiles_before = lane_value(c.through, at) - lane_value(c.tiles, at);
      return;
    }
    end = lane_value(c.end, 63);
    tiles = lane_value(c.through, 63);
  }
}

// The group of a row, -1 where it is none's.
__device__ __forceinline__ int group_of_row(const int32_t* offsets, int groups, int rows, int row) {
  int end = limited(offsets[0], rows);
  for (int base = 0; base < groups; base += 64) {
    const GroupChunk c = group_chunk(offsets, groups, rows, base, end, 0, 1);
    const uint64_t in = __ballot(c.start <= row && row < c.end);
    if (in) return base + __builtin_ctzll(in);
    end = lane_value(c.end, 63);
  }
  return -1;
}

// Logical number of workgroup b when `total` of the grid's workgroups (a multiple of 8, at least total) have work: hardware numbers
// go round the 8 XCDs, each XCD gets a contiguous run of logical ones.  false: nothing to do.
__device__ __forceinline__ bool logical_number(unsigned b, unsigned total, unsigned* l) {
  const unsigned x = b & 7u, i = b >> 3, q = total >> 3, r = total & 7u;
  if (i >= q + (x < r ? 1u : 0u)) return false;
  *l = x * q + (x < r ? x : r) + i;
  return true;
}

}  // namespace
}  // namespace stripe
