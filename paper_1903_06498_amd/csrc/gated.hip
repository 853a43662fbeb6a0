// Gated unit, y = act(g) u with [g | u] = x W^T, and the gradient of [g | u] (gfx950).
//
// Forward: the linear layer's product kernels on tiles whose columns are, for each wavefront, half gate and half up, so that a lane's registers hold
// g and u of the same outputs and nothing but y (and what a backward pass asks for) is written.  The gradients dx and dW are ordinary products of
// dz = [dg | du], because W's halves follow one another; dz itself is one pass over dy, g and u.
#include "product_tiles.hpp"

namespace stripe {
namespace {

// 16 rows by 64 pieces of 16 bytes, four rows a wavefront, all loads on their way before the first is used.  They go past the caches, where dz is to stay
// for the two products behind (8192 x 4096 bf16: 75 us, 66; with the products 688 and 680).
constexpr int kGradRows = 16;

template <typename T>
__global__ __launch_bounds__(256) void gated_grad_kernel(const GatedGradParams p, int strips) {
  constexpr int VEC = kVec<T>, EACH = kGradRows / 4;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t row0 = (int64_t)(blockIdx.x / (unsigned)strips) * kGradRows + wave * EACH;
  const int c = ((int)(blockIdx.x % (unsigned)strips) * 64 + lane) * VEC, n = p.out - c;
  if (n <= 0) return;
  u32x4 dy[EACH], g[EACH], u[EACH];
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    const int64_t row = row0 + i < p.rows ? row0 + i : p.rows - 1;
    const T* const pre = (const T*)p.pre + row * p.pre_row + c;
    if (n >= VEC) {
      typedef u32x4 any __attribute__((aligned(2)));
      dy[i] = __builtin_nontemporal_load((const any*)((const T*)p.dy + row * p.y_row + c));
      g[i] = __builtin_nontemporal_load((const any*)pre);
      u[i] = __builtin_nontemporal_load((const any*)(pre + p.out));
    } else {
      dy[i] = load_piece<T>((const T*)p.dy + row * p.y_row + c, n);
      g[i] = load_piece<T>(pre, n);
      u[i] = load_piece<T>(pre + p.out, n);
    }
  }
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    if (row0 + i >= p.rows) return;
    float d[VEC], gf[VEC], uf[VEC], dg[VEC], du[VEC];
    unpack<T>(dy[i], d);
    unpack<T>(g[i], gf);
    unpack<T>(u[i], uf);
#pragma unroll
    for (int e = 0; e < VEC; ++e) dg[e] = d[e] * uf[e];
    times_slope<T>(dg, gf, p.act);
#pragma unroll
    for (int e = 0; e < VEC; ++e) du[e] = gf[e];
    if (p.act != STRIPE_ACT_NONE) {
      with_activation(p.act, [&](auto a) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) du[e] = activate<T>(du[e], decltype(a)::value);
      });
    }
#pragma unroll
    for (int e = 0; e < VEC; ++e) du[e] *= d[e];
    T* const dz = (T*)p.dz + (row0 + i) * p.dz_row + c;
    store_piece<T>(dz, pack<T>(dg), n);
    store_piece<T>(dz + p.out, pack<T>(du), n);
    if (n <= VEC)      // the row's last piece: zeros behind it
      for (int64_t k = 2 * (int64_t)p.out; k < p.dz_row; ++k) ((T*)p.dz)[(row0 + i) * p.dz_row + k] = (T)0.f;
  }
}

// A thread copies four pieces, a workgroup's pieces one after the other.
__global__ __launch_bounds__(256) void pad_kernel(const PadParams p) {
  const unsigned pieces = (unsigned)(p.to_row / 8);
  const int64_t total = p.rows * pieces, first = (int64_t)blockIdx.x * 1024 + threadIdx.x;
  u32x4 v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t at = first + 256 * i;
    if (at >= total) break;
    const int64_t row = at / pieces, c = (at - row * pieces) * 8, m = row / p.each;
    v[i] = load_piece<__bf16>((const __bf16*)p.from + m * p.from_matrix + (row - m * p.each) * p.from_row + c, (int)(p.cols - c));
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (first + 256 * i < total) *(u32x4*)((__bf16*)p.to + (first + 256 * i) * 8) = v[i];
}

}  // namespace

hipError_t launch_pad(const PadParams& p, hipStream_t stream) {
  const int64_t total = p.rows * (p.to_row / 8);
  pad_kernel<<<dim3((unsigned)((total + 1023) / 1024)), dim3(256), 0, stream>>>(p);
  return hipGetLastError();
}

hipError_t launch_gated(int dtype, const ProductPlan& plan, Access access, ProductParams p, hipStream_t stream) {
  if (plan.few) return launch_product_rows(kGated, dtype, p, stream);
  return dtype == STRIPE_F32 ? launch_kind<float, kGated>(plan, access, p, stream) : launch_kind<__bf16, kGated>(plan, access, p, stream);
}

hipError_t launch_gated_grad(int dtype, const GatedGradParams& p, hipStream_t stream) {
  const int width = 64 * (dtype == STRIPE_F32 ? 4 : 8), strips = (p.out + width - 1) / width;
  const dim3 grid((unsigned)((p.rows + kGradRows - 1) / kGradRows * (int64_t)strips));
  if (dtype == STRIPE_F32) gated_grad_kernel<float><<<grid, dim3(256), 0, stream>>>(p, strips);
  else gated_grad_kernel<__bf16><<<grid, dim3(256), 0, stream>>>(p, strips);
  return hipGetLastError();
}

}  // namespace stripe
