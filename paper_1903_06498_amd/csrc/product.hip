// Products of the linear layer on the gfx950 matrix cores, dense or with rows sorted by group (see ProductKind for the three
// layouts).
//
// A workgroup of four wavefronts (2 x 2) computes a tile of BM x BN outputs, in 32 x 32 fragments.  K tiles are 64 bytes deep (32 bf16 or
// 16 fp32) and lie in a ring of four LDS stages:
//   an operand whose reduction index is contiguous in memory ([row][k]): 64 bytes per row, 16-byte piece c of row r in slot
//   c ^ ((r >> 2) & 3); a fragment is one 16-byte read;
//   one whose row index is contiguous ([k][row]): as it lies in memory, a row of BM or BN elements per k, pieces swizzled by k; a bf16
//   fragment is two transposing reads, an fp32 one four 4-byte reads.
// Everything beyond the reduction's end is zero in both operands; rows and columns beyond the output repeat valid ones, whose sums are
// never stored.
#include <algorithm>
#include <type_traits>

#include "layers_device.hpp"

namespace stripe {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr int kStages = 4, kDepthBytes = 64;

template <typename T>
__device__ __forceinline__ f32x16 mma(u32x4 a, u32x4 b, f32x16 c) {
  if constexpr (sizeof(T) == 2) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  } else {
    const f32x4 x = __builtin_bit_cast(f32x4, a), y = __builtin_bit_cast(f32x4, b);
#pragma unroll
    for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_32x32x2f32(x[i], y[i], c, 0, 0, 0);
    return c;
  }
}

// One operand's part of a tile: WIDTH rows (or columns) of it.  STRIDED: stored [k][row].
template <typename T, int WIDTH, bool STRIDED>
struct Operand {
  static constexpr int VEC = kVec<T>, DEPTH = kDepthBytes / (int)sizeof(T);
  static constexpr int ROW = STRIDED ? WIDTH * (int)sizeof(T) : kDepthBytes;   // bytes of an LDS row
  static constexpr int STAGE = WIDTH * kDepthBytes, LOADS = STAGE / 4096;      // 16-byte pieces per lane and K tile
  static __device__ __forceinline__ int key(int r) {
    if constexpr (!STRIDED) return (r >> 2) & 3;
    else if constexpr (sizeof(T) == 4) return 8 * ((r >> 2) & 1);              // the wavefront's halves read k and k + 4
    else return ROW >= 256 ? 4 * (r & 3) : 4 * ((r >> 1) & 1);                 // a transposing read takes four rows of k
  }
  // where piece `u` of this lane comes from
  const T* src[LOADS];
  int k[LOADS], left[LOADS];      // its first k; elements of it inside the rows' range (strided) -- else a constant
  int64_t step;                   // elements from one K tile to the next

  // base: element (row0, k = 0); rows: valid rows from row0 on; ld: row stride
  __device__ __forceinline__ void init(const T* base, int rows, int64_t ld) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int u = 0; u < LOADS; ++u) {
      const int at = (u * 4 + wave) * 1024 + lane * 16, r = at / ROW, piece = (at % ROW / 16) ^ key(r);
      if constexpr (!STRIDED) {
        k[u] = piece * VEC;
        left[u] = 0;
        src[u] = base + (int64_t)(r < rows ? r : rows - 1) * ld + k[u];
      } else {
        k[u] = r;
        left[u] = rows - piece * VEC;
        src[u] = base + (int64_t)r * ld + piece * VEC;
      }
    }
    step = STRIDED ? DEPTH * ld : DEPTH;
  }
  // elements of piece u of K tile kt that exist
  __device__ __forceinline__ int valid(int u, int kt, int K) const {
    const int n = K - (k[u] + kt * DEPTH);
    if constexpr (!STRIDED) return n;
    else return n > 0 ? left[u] : 0;
  }
  __device__ __forceinline__ void fetch(u32x4 (&to)[LOADS], int kt, int K) const {
#pragma unroll
    for (int u = 0; u < LOADS; ++u) to[u] = load_piece<T>(src[u] + (int64_t)kt * step, valid(u, kt, K));
  }
  static __device__ __forceinline__ void put(unsigned char* stage, const u32x4 (&from)[LOADS]) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int u = 0; u < LOADS; ++u) *(u32x4*)(stage + (u * 4 + wave) * 1024 + lane * 16) = from[u];
  }
  // fragment of rows row0 .. row0 + 31 (row0 a multiple of 32), matrix-instruction step s (half a K tile): lane l holds row l & 31 and the
  // 16 bytes of k with number 2 s + (l >> 5)
  static __device__ __forceinline__ u32x4 fragment(const unsigned char* stage, int row0, int s) {
    const int lane = threadIdx.x & 63, fr = lane & 31, fh = lane >> 5;
    if constexpr (!STRIDED) {
      return *(const u32x4*)(stage + (row0 + fr) * ROW + (((2 * s + fh) ^ key(fr)) << 4));
    } else if constexpr (sizeof(T) == 2) {
      // within 16 lanes, lane p points at 4 consecutive values of one k; lane i gets, for j = 0 .. 3, value i & 3 of what lane
      // (i >> 2) + 4 j points at: four k of row i
      typedef __attribute__((address_space(3))) s16x4* lptr;
      const int g = lane >> 4, q = lane & 15, kr = 8 * (g >> 1) + (q >> 2), piece = row0 / 8 + 2 * (g & 1) + ((q & 3) >> 1);
      const unsigned char* at = stage + (16 * s + kr) * ROW + ((piece ^ key(kr)) << 4) + (q & 1) * 8;
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lptr)at), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lptr)(at + 4 * ROW));
      return __builtin_bit_cast(u32x4, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    } else {
      const unsigned char* at = stage + (8 * s + 4 * fh) * ROW + ((((row0 + fr) >> 2) ^ key(4 * fh)) << 4) + (fr & 3) * 4;
      u32x4 v;
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = *(const uint32_t*)(at + j * ROW);
      return v;
    }
  }
};

// What a tile is: its place in the output and its part of the reduction.
struct Tile {
  int group, m0, m, n0;         // first output row (kForward, kInputGrad: of all rows), rows, first column
  int k0, k;                    // kWeightGrad: first row of the reduction, and its length
};

// Tiles in patches of PATCH row tiles by all column tiles: neighbouring numbers (one XCD's) share panels of both operands.
template <int KIND, int BM, int BN>
__device__ __forceinline__ bool place(const ProductParams& p, Tile* t) {
  constexpr unsigned PATCH = BM >= 256 ? 4 : 8;
  unsigned row_tiles = (unsigned)p.tiles_m, total, l;
  if (KIND != kWeightGrad && p.groups) row_tiles = (unsigned)count_row_tiles(p.offsets, p.groups, p.rows, BM);
  total = row_tiles * (unsigned)p.tiles_n;
  if (KIND == kWeightGrad && p.groups) total *= (unsigned)p.groups;
  if (!logical_number(blockIdx.x, total, &l)) return false;
  t->group = 0;
  if (KIND == kWeightGrad && p.groups) {
    const unsigned each = row_tiles * (unsigned)p.tiles_n;
    t->group = (int)(l / each);
    l %= each;
  }
  const unsigned per = PATCH * (unsigned)p.tiles_n, patch = l / per, w = l % per;
  const unsigned high = row_tiles - patch * PATCH < PATCH ? row_tiles - patch * PATCH : PATCH;
  const int tm = (int)(patch * PATCH + w % high), tn = (int)(w / high);
  t->n0 = tn * BN;
  t->k0 = 0;
  t->k = p.K;
  if (KIND != kWeightGrad && p.groups) {
    const RowTile r = find_row_tile(p.offsets, p.groups, p.rows, BM, tm);
    t->group = r.group;
    t->m0 = r.row0;
    t->m = r.rows;
  } else {
    t->m0 = tm * BM;
    t->m = p.M - t->m0 < BM ? p.M - t->m0 : BM;
    if (KIND == kWeightGrad && p.groups) {
      int end, unused;
      group_rows(p.offsets, p.groups, p.rows, t->group, 1, &t->k0, &end, &unused);
      t->k = end - t->k0;
    }
  }
  return true;
}

// Four neighbouring outputs of a row: the epilogue in fp32, then one rounding.
template <typename T, int KIND>
__device__ __forceinline__ void finish4(const ProductParams& p, int group, int64_t row, int col, f32x4 v) {
  const int n = p.N - col < 4 ? p.N - col : 4;
  const int64_t at = row * p.c_ld + col + (KIND == kWeightGrad ? group * p.c_group : 0);
  T* c = (T*)p.c + at;
  typedef T t4 __attribute__((ext_vector_type(4)));
  if constexpr (KIND == kForward) {
    if (p.bias) {
      const float* b = p.bias + (int64_t)group * p.N + col;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (e < n) v[e] += b[e];
    }
    if (p.pre) {
      T* z = (T*)p.pre + at;
      if (p.vec) {
        *(t4*)z = __builtin_convertvector(v, t4);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (e < n) z[e] = (T)v[e];
      }
    }
    if (p.act != STRIPE_ACT_NONE) {
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = activate<T>(v[e], p.act);
    }
    if (p.residual) {
      const T* r = (const T*)p.residual + at;
      if (p.vec) {
        v += __builtin_convertvector(*(const t4*)r, f32x4);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (e < n) v[e] += (float)r[e];
      }
    }
  }
  if (p.vec) {
    *(t4*)c = __builtin_convertvector(v, t4);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < n) c[e] = (T)v[e];
  }
}

template <typename T, int KIND, int FM, int FN>
__global__ __launch_bounds__(256) void product_kernel(const ProductParams p) {
  constexpr int BM = 64 * FM, BN = 64 * FN;
  using A = Operand<T, BM, KIND == kWeightGrad>;
  using B = Operand<T, BN, KIND != kForward>;
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  unsigned char *const lds_a = lds, *const lds_b = lds + kStages * A::STAGE;
  Tile t;
  if (!place<KIND, BM, BN>(p, &t)) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm = wave >> 1, wn = wave & 1;

  A a;
  B b;
  if constexpr (KIND == kWeightGrad) {
    a.init((const T*)p.a + (int64_t)t.k0 * p.a_ld + t.m0, t.m, p.a_ld);
    b.init((const T*)p.b + (int64_t)t.k0 * p.b_ld + t.n0, p.N - t.n0, p.b_ld);
  } else {
    const T* w = (const T*)p.b + (int64_t)t.group * p.b_group;
    a.init((const T*)p.a + (int64_t)t.m0 * p.a_ld, t.m, p.a_ld);
    b.init(KIND == kForward ? w + (int64_t)t.n0 * p.b_ld : w + t.n0, p.N - t.n0, p.b_ld);
  }
  // this workgroup's K tiles
  int kt0 = 0, kt1 = (t.k + A::DEPTH - 1) / A::DEPTH;
  if (p.splits > 1) {
    const int per = (kt1 + p.splits - 1) / p.splits;
    kt0 = (int)blockIdx.y * per < kt1 ? (int)blockIdx.y * per : kt1;
    kt1 = kt0 + per < kt1 ? kt0 + per : kt1;
  }

  f32x16 acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.f;

  u32x4 ra[A::LOADS], rb[B::LOADS];
  a.fetch(ra, kt0, t.k);
  b.fetch(rb, kt0, t.k);
  for (int kt = kt0; kt < kt1; ++kt) {
    const int stage = kt & 1;
    A::put(lds_a + stage * A::STAGE, ra);
    B::put(lds_b + stage * B::STAGE, rb);
    __syncthreads();          // (the stage that the next turn writes was read before this barrier's turn)
    a.fetch(ra, kt + 1, t.k);
    b.fetch(rb, kt + 1, t.k);
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      u32x4 fa[FM], fb[FN];
#pragma unroll
      for (int i = 0; i < FM; ++i) fa[i] = A::fragment(lds_a + stage * A::STAGE, (wm * FM + i) * 32, s);
#pragma unroll
      for (int j = 0; j < FN; ++j) fb[j] = B::fragment(lds_b + stage * B::STAGE, (wn * FN + j) * 32, s);
#pragma unroll
      for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = mma<T>(fa[i], fb[j], acc[i][j]);
    }
  }

  // Element v of lane l of a fragment is row 8 (v / 4) + 4 (l >> 5) + v % 4, column l & 31.  Each fragment goes through 4 KB of the idle ring
  // that are the wavefront's own, pieces swizzled by the row, and leaves with four neighbouring columns per lane.
  __syncthreads();
  unsigned char* buf = lds + wave * 4096;
  const int fr = lane & 31, fh = lane >> 5, sp = lane >> 3, sc = lane & 7;
  const int64_t image = KIND == kWeightGrad ? (int64_t)t.group * p.M : 0;
  const int64_t images = KIND == kWeightGrad && p.groups ? (int64_t)p.groups * p.M : p.M;
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j) {
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        const int row = 8 * (v / 4) + 4 * fh + v % 4;
        *(float*)(buf + row * 128 + (((fr >> 2) ^ (row & 7)) << 4) + (fr & 3) * 4) = acc[i][j][v];
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int r8 = 0; r8 < 4; ++r8) {
        const f32x4 v = *(const f32x4*)(buf + (8 * r8 + sp) * 128 + ((sc ^ sp) << 4));
        const int row = (wm * FM + i) * 32 + 8 * r8 + sp, col = t.n0 + (wn * FN + j) * 32 + 4 * sc;
        if (row >= t.m || col >= p.N) continue;
        if (p.splits > 1) {
          float* to = p.partial + ((int64_t)blockIdx.y * images + image + t.m0 + row) * p.N + col;
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (col + e < p.N) to[e] = v[e];
        } else {
          finish4<T, KIND>(p, t.group, (int64_t)t.m0 + row, col, v);
        }
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
}

// ---- dz = dy act'(z), and the bias gradient -------------------------------------
// A workgroup takes up to 64 rows of one group (a "slot") by 64 pieces of 16 bytes, a row per wavefront at a time.
constexpr int kSlot = 64;

template <typename T>
__global__ __launch_bounds__(256) void dz_kernel(const DzParams p, int strips) {
  constexpr int VEC = kVec<T>;
  __shared__ float part[4][64 * VEC];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int slot = (int)(blockIdx.x / (unsigned)strips), strip = (int)(blockIdx.x % (unsigned)strips);
  RowTile r = {0, slot * kSlot, 0};
  if (p.groups) {
    if (slot >= count_row_tiles(p.offsets, p.groups, p.rows, kSlot)) return;
    r = find_row_tile(p.offsets, p.groups, p.rows, kSlot, slot);
  } else {
    const int left = p.rows - r.row0;
    r.rows = left < kSlot ? left : kSlot;
  }
  const int c = (strip * 64 + lane) * VEC, n = p.out - c;
  float sum[VEC];
#pragma unroll
  for (int i = 0; i < VEC; ++i) sum[i] = 0.f;
  if (n > 0) {
#pragma unroll 4
    for (int q = wave; q < r.rows; q += 4) {
      const int64_t row = (int64_t)r.row0 + q;
      float d[VEC];
      unpack<T>(load_piece<T>((const T*)p.dy + row * p.y_row + c, n), d);
      if (p.z) {
        float z[VEC];
        unpack<T>(load_piece<T>((const T*)p.z + row * p.y_row + c, n), z);
#pragma unroll
        for (int i = 0; i < VEC; ++i) d[i] *= slope<T>(z[i], p.act);
        if (p.dz) store_piece<T>((T*)p.dz + row * p.dz_row + c, pack<T>(d), n);
      }
#pragma unroll
      for (int i = 0; i < VEC; ++i) sum[i] += d[i];
    }
  }
  if (!p.db) return;
#pragma unroll
  for (int i = 0; i < VEC; ++i) part[wave][lane * VEC + i] = sum[i];
  __syncthreads();
  float* to = p.slots > 1 ? p.partial + (int64_t)slot * p.out : p.db;
  for (int i = threadIdx.x; i < 64 * VEC; i += 256) {
    const int col = strip * 64 * VEC + i;
    if (col < p.out) to[col] = (part[0][i] + part[1][i]) + (part[2][i] + part[3][i]);
  }
}

// Each group's slots added in their order: 64 columns, four wavefronts.
__global__ __launch_bounds__(256) void db_kernel(const DzParams p, int strips) {
  __shared__ float part[4][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int group = (int)(blockIdx.x / (unsigned)strips), c = (int)(blockIdx.x % (unsigned)strips) * 64 + lane;
  int first = 0, count = p.slots;
  if (p.groups) {
    int start, end;
    group_rows(p.offsets, p.groups, p.rows, group, kSlot, &start, &end, &first);
    count = (end - start + kSlot - 1) / kSlot;
  }
  float s = 0.f;
  if (c < p.out) {
#pragma unroll 8
    for (int i = wave; i < count; i += 4) s += p.partial[(int64_t)(first + i) * p.out + c];
  }
  part[wave][lane] = s;
  __syncthreads();
  if (wave == 0 && c < p.out) p.db[(int64_t)group * p.out + c] = (part[0][lane] + part[1][lane]) + (part[2][lane] + part[3][lane]);
}

// ---- host ---------------------------------------------------------------------
struct TileShape {
  int fm, fn;
};
constexpr TileShape kTiles[] = {{2, 2}};

template <typename T, int KIND>
hipError_t launch_kind(const ProductPlan& plan, ProductParams& p, hipStream_t stream) {
  const TileShape s = kTiles[plan.tile];
  const int bm = 64 * s.fm, bn = 64 * s.fn;
  p.tiles_n = (p.N + bn - 1) / bn;
  p.tiles_m = (p.M + bm - 1) / bm;
  p.splits = plan.splits;
  int64_t total = (int64_t)p.tiles_m * p.tiles_n;
  if (p.groups) {
    // every group's last tile may be part of one
    if (KIND == kWeightGrad) total *= p.groups;
    else total = ((int64_t)p.M / bm + std::min<int64_t>(p.groups, p.M)) * p.tiles_n;
  }
  const dim3 grid((unsigned)((total + 7) / 8 * 8), (unsigned)plan.splits);
  product_kernel<T, KIND, 2, 2><<<grid, dim3(256), kStages * (bm + bn) * kDepthBytes, stream>>>(p);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_type(ProductKind kind, const ProductPlan& plan, ProductParams& p, hipStream_t stream) {
  switch (kind) {
    case kForward: return launch_kind<T, kForward>(plan, p, stream);
    case kInputGrad: return launch_kind<T, kInputGrad>(plan, p, stream);
    default: return launch_kind<T, kWeightGrad>(plan, p, stream);
  }
}

}  // namespace

ProductPlan plan_product(ProductKind kind, int dtype, int64_t rows, int64_t in, int64_t out, int groups, bool aligned) {
  (void)kind, (void)dtype, (void)rows, (void)in, (void)out, (void)groups, (void)aligned;
  return {};
}

std::string product_name(ProductKind kind, int dtype, const ProductPlan& plan, bool aligned) {
  (void)aligned;
  const TileShape s = kTiles[plan.tile];
  return std::string("product_") + (kind == kForward ? "nt_" : kind == kInputGrad ? "nn_" : "tn_") + (dtype == STRIPE_F32 ? "f32_" : "bf16_") +
         std::to_string(64 * s.fm) + "x" + std::to_string(64 * s.fn);
}

hipError_t launch_product(ProductKind kind, int dtype, const ProductPlan& plan, bool aligned, ProductParams p, hipStream_t stream) {
  (void)aligned;
  return dtype == STRIPE_F32 ? launch_type<float>(kind, plan, p, stream) : launch_type<__bf16>(kind, plan, p, stream);
}

// (one more with groups: a single empty group's zeros come from db_kernel)
int64_t dz_slots(int64_t rows, int groups) { return groups ? rows / kSlot + groups + 1 : std::max<int64_t>(1, (rows + kSlot - 1) / kSlot); }

hipError_t launch_dz(int dtype, const DzParams& p, hipStream_t stream) {
  const int vec = dtype == STRIPE_F32 ? 4 : 8, strips = (p.out + 64 * vec - 1) / (64 * vec), sums = (p.out + 63) / 64;
  const dim3 grid((unsigned)((int64_t)p.slots * strips));
  if (dtype == STRIPE_F32) dz_kernel<float><<<grid, dim3(256), 0, stream>>>(p, strips);
  else dz_kernel<__bf16><<<grid, dim3(256), 0, stream>>>(p, strips);
  if (p.db && p.slots > 1) db_kernel<<<dim3((unsigned)((int64_t)std::max(1, p.groups) * sums)), dim3(256), 0, stream>>>(p, sums);
  return hipGetLastError();
}

}  // namespace stripe
