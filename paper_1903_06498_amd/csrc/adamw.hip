// AdamW over many tensors in few launches (gfx950).  What bounds it is memory.
//
//   g = factor grad,  m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2,  p = p (1 - lr wd) - lr (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps)
//
// The tensors' records are kernel arguments: nothing is copied to the device before, and a captured launch holds them.  A wavefront takes blocks of 256
// consecutive elements, four a lane.
//
// States in 8 bits: per block, m = q c |c| with c = -127 .. 127 and sqrt(v) = q c^2 with c = 0 .. 255; the squares spend the codes on small values as well (the
// smallest but 0 are 2^-14 and 2^-16 of the block's largest).  An update changes sqrt(v) by 2^-11 of itself where the codes are 2^-7 apart: rounded to nearest,
// a state would stand still but for the factor q.  So c is one of its value's two neighbours at random, such that the value's mean is kept, from a hash
// of (seed, tensor, element).  sqrt(v) > 0 is never rounded to 0: m / eps would be the step.
// Every operation is rounded by itself (no contraction), so that codes are a function of the formula and not of the compiler.
//
// What is read and written goes past the caches, but for the loads of codes, 4 bytes a lane (95 M elements, bf16 gradients and copies: 28 bytes each with fp32
// states 514 us through the caches, 494 with such stores, 437 with such loads too, 6.1 TB/s; 16 bytes with 8-bit states, and read back with 10: 550, 458, 414; codes
// too: 481).
#include "layers_device.hpp"

namespace stripe {
namespace {

constexpr int kEach = 2, kChunk = 4 * kEach * kAdamWBlock;      // blocks of a wavefront, elements of a workgroup

// MurmurHash3's finalizer.
__device__ __forceinline__ uint32_t mix(uint32_t x) {
  x ^= x >> 16;
  x *= 0x85ebca6bu;
  x ^= x >> 13;
  x *= 0xc2b2ae35u;
  return x ^ (x >> 16);
}

// The largest of a wavefront's values, as bits of floats that are not negative: NaN is above all.
__device__ __forceinline__ float wave_largest(uint32_t v) {
  auto from = [&](auto ctrl, auto rows) {
    const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, decltype(ctrl)::value, decltype(rows)::value, 0xf, true);
    v = v > o ? v : o;
  };
  using std::integral_constant;
  from(integral_constant<int, 0xb1>{}, integral_constant<int, 0xf>{});
  from(integral_constant<int, 0x4e>{}, integral_constant<int, 0xf>{});
  from(integral_constant<int, 0x141>{}, integral_constant<int, 0xf>{});
  from(integral_constant<int, 0x140>{}, integral_constant<int, 0xf>{});
  from(integral_constant<int, 0x142>{}, integral_constant<int, 0xa>{});
  from(integral_constant<int, 0x143>{}, integral_constant<int, 0xc>{});
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane((int)v, 63));
}

// Four neighbouring elements, the first n of which exist.
template <typename T>
__device__ __forceinline__ void load4(const T* q, int n, T (&to)[4]) {
  if (n >= 4) {
    typedef T vec __attribute__((ext_vector_type(4), aligned(sizeof(T))));
    vec v;
    if constexpr (sizeof(T) == 1) v = *(const vec*)q;
    else v = __builtin_nontemporal_load((const vec*)q);
    __builtin_memcpy(to, &v, 4 * sizeof(T));
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) to[i] = i < n ? q[i] : (T)0;
  }
}
template <typename T>
__device__ __forceinline__ void store4(T* q, int n, const T (&from)[4]) {
  if (n >= 4) {
    typedef T vec __attribute__((ext_vector_type(4), aligned(sizeof(T))));
    vec v;
    __builtin_memcpy(&v, from, 4 * sizeof(T));
    __builtin_nontemporal_store(v, (vec*)q);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < n) q[i] = from[i];
  }
}

// Codes of a block's values (not negative), and the factor of their squares.  The instruction's root gives the codes of an exact one: a floor that is one too
// large, which it has for values just below a square, is taken back by `past` and `place`, and one that is too small does not occur (looked at on gfx950 for every
// fp32 value up to 2^16, and all random bits where the floors differ).
template <int MOST, bool KEEPS>
__device__ __forceinline__ float encode(const float (&value)[4], const uint32_t (&bits)[4], float (&code)[4]) {
#pragma clang fp contract(off)
  uint32_t high = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t b = __builtin_bit_cast(uint32_t, value[i]);
    high = high > b ? high : b;
  }
  const float top = wave_largest(high);
  if (!(top < __builtin_inff())) {      // not finite: the block is NaN from here on
#pragma unroll
    for (int i = 0; i < 4; ++i) code[i] = 1.f;
    return __builtin_nanf("");
  }
  const bool fine = top > 1e-30f;
  const float inverse = fine ? 1.f / top * (float)(MOST * MOST) : 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float t = value[i] * inverse, low = floorf(__builtin_amdgcn_sqrtf(t)), past = t - low * low, place = (float)bits[i] * 0x1p-16f * (2.f * low + 1.f);
    float c = low + (past > place ? 1.f : 0.f);
    c = fminf(c, (float)MOST);
    if (KEEPS) c = t > 0.f ? fmaxf(c, 1.f) : c;
    code[i] = c;
  }
  return fine ? top * (float)(1.0 / (MOST * MOST)) : 0.f;
}

__device__ __forceinline__ int find_tensor(const uint32_t* through, int count, uint32_t chunk) {
  const int lane = threadIdx.x & 63;
  const uint64_t past = __ballot(lane < count && through[lane < count ? lane : 0] > chunk);
  return (int)__builtin_ctzll(past);
}

template <typename G, bool EIGHT>
__global__ __launch_bounds__(256) void adamw_kernel(const AdamWParams p) {
#pragma clang fp contract(off)
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int at = find_tensor(p.through, p.count, blockIdx.x);
  const AdamWTensor& x = p.tensor[at];
  const int64_t chunk = (int64_t)(blockIdx.x - (at ? p.through[at - 1] : 0u)), first = chunk * kChunk + wave * (kEach * kAdamWBlock);
  float keep = x.keep, rate = p.rate, spread = p.spread, factor = p.factor;
  uint32_t seed = p.seed;
  if (p.control) {
    const float lr = p.control[0];
    keep = 1.f - lr * keep;
    rate = lr * p.control[1];
    spread = p.control[2];
    factor = p.control[3];
    seed = __builtin_bit_cast(uint32_t, p.control[4]);
  }
  const uint32_t key = EIGHT ? mix(seed + x.number) : 0;

  float pv[kEach][4], mv[kEach][4], vv[kEach][4], mq[kEach], vq[kEach];
  G gv[kEach][4];
  int8_t mc[kEach][4];
  uint8_t vc[kEach][4];
#pragma unroll
  for (int b = 0; b < kEach; ++b) {
    const int64_t i = first + b * kAdamWBlock + 4 * lane;
    const int n = x.elements - i < 4 ? (x.elements > i ? (int)(x.elements - i) : 0) : 4;
    load4<float>(x.p + i, n, pv[b]);
    load4<G>((const G*)x.grad + i, n, gv[b]);
    if constexpr (EIGHT) {
      const int64_t block = (first + b * kAdamWBlock) / kAdamWBlock;
      const bool there = block * kAdamWBlock < x.elements;
      load4<int8_t>((const int8_t*)x.m + i, n, mc[b]);
      load4<uint8_t>((const uint8_t*)x.v + i, n, vc[b]);
      mq[b] = there ? x.m_scale[block] : 0.f;
      vq[b] = there ? x.v_scale[block] : 0.f;
    } else {
      load4<float>((const float*)x.m + i, n, mv[b]);
      load4<float>((const float*)x.v + i, n, vv[b]);
    }
  }
#pragma unroll
  for (int b = 0; b < kEach; ++b) {
    const int64_t i = first + b * kAdamWBlock + 4 * lane;
    const int n = x.elements - i < 4 ? (x.elements > i ? (int)(x.elements - i) : 0) : 4;
    float m[4], v[4], r[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float g = (float)gv[b][e] * factor;
      if constexpr (EIGHT) {
        const float c = (float)mc[b][e], k = (float)vc[b][e], s = k * k * vq[b];
        m[e] = c * __builtin_fabsf(c) * mq[b];
        v[e] = s * s;
      } else {
        m[e] = mv[b][e];
        v[e] = vv[b][e];
      }
      m[e] = m[e] * p.b1 + g * p.c1;
      v[e] = v[e] * p.b2 + g * g * p.c2;
      r[e] = sqrtf(v[e]);
      pv[b][e] = pv[b][e] * keep - m[e] * rate * __builtin_amdgcn_rcpf(r[e] * spread + p.eps);      // (the reciprocal is off by 1 ulp at most)
    }
    store4<float>(x.p + i, n, pv[b]);
    if (x.copy) {
      __bf16 copy[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) copy[e] = (__bf16)pv[b][e];
      store4<__bf16>((__bf16*)x.copy + i, n, copy);
    }
    if constexpr (EIGHT) {
      const int64_t block = (first + b * kAdamWBlock) / kAdamWBlock;
      float size[4];
      uint32_t low[4], high[4];
      float code[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t bits = mix(key + (uint32_t)(i + e));
        low[e] = bits & 0xffffu;
        high[e] = bits >> 16;
        size[e] = e < n ? __builtin_fabsf(m[e]) : 0.f;
        r[e] = e < n ? r[e] : 0.f;
      }
      const float mscale = encode<127, false>(size, low, code);
#pragma unroll
      for (int e = 0; e < 4; ++e) mc[b][e] = (int8_t)(int)(m[e] < 0.f ? -code[e] : code[e]);
      const float vscale = encode<255, true>(r, high, code);
#pragma unroll
      for (int e = 0; e < 4; ++e) vc[b][e] = (uint8_t)(int)code[e];
      store4<int8_t>((int8_t*)x.m + i, n, mc[b]);
      store4<uint8_t>((uint8_t*)x.v + i, n, vc[b]);
      if (lane == 0 && block * kAdamWBlock < x.elements) {
        x.m_scale[block] = mscale;
        x.v_scale[block] = vscale;
      }
    } else {
      store4<float>((float*)x.m + i, n, m);
      store4<float>((float*)x.v + i, n, v);
    }
  }
}

// The values that states in 8 bits stand for: m to `p`, v to `copy`.  A lane's loads are 4 bytes: those of four chunks are on their way together.
constexpr int kReadChunks = 4;
__global__ __launch_bounds__(256) void adamw_read_kernel(const AdamWParams p) {
#pragma clang fp contract(off)
  constexpr int N = kReadChunks * kEach;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  float *mto[N], *vto[N], mq[N], vq[N];
  int left[N];
  int8_t mc[N][4];
  uint8_t vc[N][4];
#pragma unroll
  for (int c = 0; c < kReadChunks; ++c) {
    uint32_t number = blockIdx.x * kReadChunks + c;
    const bool there = number < p.through[p.count - 1];
    number = there ? number : 0;
    const int at = find_tensor(p.through, p.count, number);
    const AdamWTensor& x = p.tensor[at];
    const int64_t chunk = (int64_t)(number - (at ? p.through[at - 1] : 0u)), first = chunk * kChunk + wave * (kEach * kAdamWBlock);
#pragma unroll
    for (int b = 0; b < kEach; ++b) {
      const int k = c * kEach + b;
      const int64_t i = first + b * kAdamWBlock + 4 * lane, block = i / kAdamWBlock;
      left[k] = !there || x.elements <= i ? 0 : x.elements - i < 4 ? (int)(x.elements - i) : 4;
      load4<int8_t>((const int8_t*)x.m + i, left[k], mc[k]);
      load4<uint8_t>((const uint8_t*)x.v + i, left[k], vc[k]);
      mq[k] = left[k] ? x.m_scale[block] : 0.f;
      vq[k] = left[k] ? x.v_scale[block] : 0.f;
      mto[k] = x.p ? x.p + i : nullptr;
      vto[k] = x.copy ? (float*)x.copy + i : nullptr;
    }
  }
#pragma unroll
  for (int k = 0; k < N; ++k) {
    float m[4], v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float c = (float)mc[k][e], d = (float)vc[k][e], s = d * d * vq[k];
      m[e] = c * __builtin_fabsf(c) * mq[k];
      v[e] = s * s;
    }
    if (mto[k]) store4<float>(mto[k], left[k], m);
    if (vto[k]) store4<float>(vto[k], left[k], v);
  }
}

}  // namespace

uint32_t adamw_chunks(int64_t elements) { return (uint32_t)((elements + kChunk - 1) / kChunk); }

hipError_t launch_adamw(int grad_dtype, bool eight, const AdamWParams& p, hipStream_t stream) {
  const dim3 grid(p.through[p.count - 1]);
  if (eight) {
    if (grad_dtype == STRIPE_F32) adamw_kernel<float, true><<<grid, dim3(256), 0, stream>>>(p);
    else adamw_kernel<__bf16, true><<<grid, dim3(256), 0, stream>>>(p);
  } else {
    if (grad_dtype == STRIPE_F32) adamw_kernel<float, false><<<grid, dim3(256), 0, stream>>>(p);
    else adamw_kernel<__bf16, false><<<grid, dim3(256), 0, stream>>>(p);
  }
  return hipGetLastError();
}

hipError_t launch_adamw_read(const AdamWParams& p, hipStream_t stream) {
  adamw_read_kernel<<<dim3((p.through[p.count - 1] + kReadChunks - 1) / kReadChunks), dim3(256), 0, stream>>>(p);
  return hipGetLastError();
}

}  // namespace stripe
