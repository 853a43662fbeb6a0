// The linear layer's products, dz and the bias gradient; which tile and how many slices a product gets (gfx950).  Kernels: product_tiles.hpp.
#include <algorithm>
#include <cmath>

#include "product_tiles.hpp"

namespace stripe {
namespace {

// ---- dz = dy act'(z), and the bias gradient -------------------------------------
// A workgroup takes up to 32 rows of one group (a "slot") by 64 pieces of 16 bytes, a row per wavefront at a time.  (64 rows: too few
// workgroups for 4096 x 2048 in 16 groups; 16: twice the partial sums.)
constexpr int kSlot = 32;

template <typename T>
__global__ __launch_bounds__(256) void dz_kernel(const DzParams p, int strips) {
  constexpr int VEC = kVec<T>;
  __shared__ float part[4][64 * VEC];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int slot = (int)(blockIdx.x / (unsigned)strips), strip = (int)(blockIdx.x % (unsigned)strips);
  RowTile r = {0, slot * kSlot, 0};
  if (p.groups) {
    r = find_row_tile(p.offsets, p.groups, p.rows, kSlot, slot);
    if (r.rows <= 0) return;      // behind the last one
  } else {
    const int left = p.rows - r.row0;
    r.rows = left < kSlot ? left : kSlot;
  }
  const int c = (strip * 64 + lane) * VEC, n = p.out - c;
  float sum[VEC];
#pragma unroll
  for (int i = 0; i < VEC; ++i) sum[i] = 0.f;
  const T *dy = (const T*)p.dy + (int64_t)r.row0 * p.y_row + c, *z = (const T*)p.z + (int64_t)r.row0 * p.y_row + c;
  T* dz = (T*)p.dz + (int64_t)r.row0 * p.dz_row + c;
  auto use = [&](int64_t row, u32x4 dv, u32x4 zv, int n) {
    float d[VEC];
    unpack<T>(dv, d);
    if (p.z) {
      float zf[VEC];
      unpack<T>(zv, zf);
      times_slope<T>(d, zf, p.act);
      if (p.dz) store_piece<T>(dz + row * p.dz_row, pack<T>(d), n);
    }
#pragma unroll
    for (int i = 0; i < VEC; ++i) sum[i] += d[i];
  };
  if (n >= VEC && r.rows > 0) {      // (a layer without rows has a last row no more than a first)
    // all of a wavefront's rows are on their way before the first is used (8192 x 8192 bf16, 403 MB: 112 -> 97 us); rows behind the last repeat it
    constexpr int EACH = kSlot / 4;
    u32x4 dv[EACH], zv[EACH];
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      const int q = 4 * i + wave;
      const int64_t row = q < r.rows ? q : r.rows - 1;
      __builtin_memcpy(&dv[i], dy + row * p.y_row, 16);
      if (p.z) __builtin_memcpy(&zv[i], z + row * p.y_row, 16);
    }
#pragma unroll
    for (int i = 0; i < EACH; ++i)
      if (4 * i + wave < r.rows) use(4 * i + wave, dv[i], zv[i], VEC);
  } else if (n > 0) {
    for (int64_t q = wave; q < r.rows; q += 4) use(q, load_piece<T>(dy + q * p.y_row, n), p.z ? load_piece<T>(z + q * p.y_row, n) : (u32x4){0, 0, 0, 0}, n);
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
// Estimated times, in us: of a K tile where workgroups are alone on their CU and few on the chip; where they fill it; the same of what else
// a workgroup does.
struct TileTime {
  double k_few, k_full, store_few, store_full;
};
// parts: fp32 split into three bf16 parts, which is faster where the matrix instructions are what a CU waits for (2048^3: 124 us with fp32
// instructions, 106), and slower where it is the way through the registers (512^3: 12.4 and 14.2).
TileTime tile_time(int tile, int dtype, Access access, bool parts) {
  if (dtype == STRIPE_F32) {
    if (parts) return {0.95, 1.55, 5, 7};
    if (access == kWords) return tile == kLeastTile ? TileTime{0.58, 0.97, 2, 4} : TileTime{1.05, 1.95, 3, 5};
    return tile == kLeastTile ? TileTime{0.5, 1.0, 2, 4} : TileTime{0.95, 1.95, 3, 5};
  }
  if (access != kPieces) return {0.75, 1.1, 3, 5};
  constexpr TileTime t[] = {{1.03, 1.36, 6, 9}, {0.56, 0.76, 4, 5}, {0.28, 0.5, 3, 5}, {0.22, 0.35, 2, 4}};
  return t[tile];
}


template <typename T>
hipError_t launch_type(ProductKind kind, const ProductPlan& plan, Access access, ProductParams& p, hipStream_t stream) {
  switch (kind) {
    case kForward: return launch_kind<T, kForward>(plan, access, p, stream);
    case kInputGrad: return launch_kind<T, kInputGrad>(plan, access, p, stream);
    default: return launch_kind<T, kWeightGrad>(plan, access, p, stream);
  }
}

// Few rows, which read W once for every 16 rows of a group, 16 columns a workgroup: a launch, and for each workgroup of a CU its bytes at the rate that one
// reaches; bf16 rows at odd addresses take three times as long (4095 -> 4095, 16 rows: 26.7 us, 18.4 on tiles).  floor: what the tiles take at least once
// they are more than one to a CU, W from memory.  The groups that have rows are taken to be as many as if rows were dealt out at random.
// Measured, this kernel and the tiles, us: 4096 -> 4096 bf16 1 row 8.3 and 10.8, 16 10.5 and 10.6, 32 18.3 and 11.3; 1024 -> 1024 6.3 and 6.5 up to 64 rows;
// 8192 -> 2048 1 row 12 and 12, 16 16.8 and 11.3; fp32 4096 -> 4096 16 rows 20.5 and 23, 32 36.9 and 23.5; 2048 -> 1024 of 64 groups 16 rows 14.2 and 11.2,
// 64 35 and 42, 256 53 and 55; of 8 groups 64 rows 9.5 and 12.6; 1024 -> 4096 of 64 groups 64 rows 71 and 62.
struct RowsTime {
  double us, floor;
};
RowsTime rows_time(int dtype, int64_t rows, int64_t in, int64_t out, int groups, bool odd_rows) {
  const double all = groups, used = groups ? all * (1 - std::exp(-(double)rows / all)) : 1;
  const double slots = used * std::ceil((double)rows / (16 * used)), each = 16.0 * (double)in * (dtype == STRIPE_F32 ? 4 : 2);
  const double rate = odd_rows ? 6e3 : 20e3;      // bytes per us
  const double workgroups = slots * (double)((out + 15) / 16);
  return {3.5 + std::max(1.0, workgroups / 256) * (each / rate + 0.15), 4 + used * (double)in * (double)out * (dtype == STRIPE_F32 ? 4 : 2) / 5.2e6};
}

}  // namespace

// Logits that are made in slices of the reduction are in memory as a whole, for a moment: 4 MB for each slice at most.  With more of them there are tiles enough.
constexpr int64_t kFewLogits = (int64_t)1 << 20;

// The tile and the slices of the reduction with the smallest estimated time: the workgroups of the CU that has most of them one after the other,
// or in pairs where two fit.
ProductPlan plan_product(ProductKind kind, int dtype, int64_t rows, int64_t in, int64_t out, int groups, Access access, bool odd_rows, ProductUse use) {
  ProductPlan plan;
  plan.tile = kSmallTile;
  if (!rows) return plan;
  const int64_t m = kind == kWeightGrad ? out : rows, n = kind == kForward ? out : in, k = kind == kForward ? in : kind == kInputGrad ? out : rows;
  const int64_t images = kind == kWeightGrad ? std::max(1, groups) : 1, depth = dtype == STRIPE_F32 ? 32 : 64;
  const double depth_of = kind == kWeightGrad && groups ? (double)k / groups : (double)k;
  const int64_t k_tiles = std::max<int64_t>(1, (int64_t)std::ceil(depth_of / (double)depth));
  double best = __builtin_huge_val(), best_workgroups = 0;
  const int forced_tile = tune_int("product_tile", -1), forced_splits = tune_int("product_splits", 0);
  const bool f32 = dtype == STRIPE_F32;
  // A gated unit's few rows read W from memory at the same rate on every tile, but for what its slices cost: 16 rows, 4096 -> 2 x 8192 bf16, tiles 0 to 3 33.4 (four
  // slices), 30.9 (four), 37.9 (two) and 30.6 us; 8192 -> 2 x 8192 71.3, 68.9, 64.3, 60.5; 2048 -> 2 x 4096 16.8, 14.7, 12.5, 9.9.
  const bool streams = use == kHalves && kind == kForward && !groups && !f32 && access == kPieces && rows <= 64 && n >= 128 * 64 && forced_tile < 0 && !forced_splits;
  for (int variant = 0; variant < kTileCount; ++variant) {
    // loads into LDS: bf16 any tile, fp32 the small ones; the kernel for any alignment has the small one's shape, for fp32 in parts (variant 1)
    const bool parts = f32 && variant == 1;
    const int tile = parts ? kSmallTile : variant;
    if (access == kAny ? (f32 ? !parts : tile != kSmallTile) : (f32 && variant == 0) || (forced_tile >= 0 && forced_tile != variant)) continue;
    if (streams && tile != kLeastTile) continue;
    const TileShape s = kTiles[tile];
    const TileTime t = tile_time(tile, dtype, access, parts);
    const int64_t bm = 64 * s.fm, bn = 64 * s.fn;
    const double row_tiles = kind == kWeightGrad ? (double)((m + bm - 1) / bm * images)
                             : groups            ? (double)m / (double)bm + 0.5 * std::min<double>(groups, (double)m)
                                                 : (double)((m + bm - 1) / bm);
    const double tiles = row_tiles * (double)((n + bn - 1) / bn);
    for (int splits = 1; splits <= (streams || (use == kLogits && m * n > kFewLogits) ? 1 : 16); ++splits) {
      if (splits > 1 && (k_tiles < 2 * splits || (forced_splits && splits != forced_splits))) continue;
      const int64_t bytes = splits > 1 ? splits * images * m * n * 4 : 0;
      if (bytes > (64 << 20)) continue;
      const double workgroups = std::max(1.0, tiles * splits), most = std::ceil(workgroups / 256), full = std::min(1.0, workgroups / 256);
      const double kt = std::ceil((double)k_tiles / splits);
      double us = 4;
      if (s.resident == 1) us += most * (kt * (t.k_few + (t.k_full - t.k_few) * full) + t.store_few + (t.store_full - t.store_few) * full);
      else us += std::floor(most / 2) * (kt * t.k_full + t.store_full) + std::fmod(most, 2) * (kt * t.k_few + t.store_few);
      if (use == kLogits) {
        // Few rows read W from memory, a workgroup with a stage less a half of its tile on its way, about 2.2 us each.  16 rows, 4096 -> 32768 bf16 (268 MB): tiles 0
        // to 3 106, 64, 62 and 54 us; by this 102, 64, 64 and 57.
        const double way = (s.stages - 0.5) * (double)bn * 128, held = std::min(256.0, workgroups) * (workgroups > 256 ? s.resident : 1) * way / 2.2;
        us = std::max(us, 6 + (double)n * (double)k * (f32 ? 4 : 2) / std::min(5.3e6, held));
      }
      // the join: a launch, and its bytes written and read (300^3 fp32: 8.9 us in one piece, 9.6 in the five that would win without the launch;
      // 1000 x 777 x 1283's dW: 40.9 in one, 34.8 in three)
      if (splits > 1) us += 3.2 + (double)bytes * 1.5 / 4e6;
      if (forced_splits && splits != forced_splits) us += 1e9;      // one piece, only where that many cannot be made
      if (us < best) {
        best = us;
        plan.tile = tile;
        plan.parts = parts;
        plan.splits = splits;
        plan.ws_bytes = bytes;
        best_workgroups = workgroups;
        plan.us = us;
      }
    }
  }
  if (kind == kForward && use != kLogits && rows <= (groups ? 8 * (int64_t)groups : 64)) {
    const RowsTime few = rows_time(dtype, rows, in, out, groups, odd_rows);
    if (best_workgroups > 256 || use == kHalves) best = std::max(best, few.floor);
    // A gated unit, 4096 -> 2 x 8192 bf16, 1, 4, 8 and 16 rows: here 29.9, 31.5, 34.1 and 39.7 us, as every workgroup reads x, on tiles 3 30.5 to 30.7.
    const double x_us = use == kHalves ? std::max(1.0, (double)((out + 15) / 16) / 256) * (double)std::min<int64_t>(rows, 16) * (double)in * (f32 ? 4 : 2) / 52e3 : 0;
    plan.few = few.us + x_us <= 1.05 * best;
    if (plan.few) plan.us = few.us + x_us;
  }
  if (const int forced = tune_int("product_few", -1); forced >= 0 && kind == kForward && use != kLogits) plan.few = forced != 0;
  if ((groups ? rows / 16 + std::min<int64_t>(groups, rows) : (rows + 15) / 16) * ((out + 15) / 16) >= 1 << 23) plan.few = false;      // 2^32 lanes
  if (plan.few) plan.splits = 1, plan.ws_bytes = 0;
  return plan;
}

int tile_columns(const ProductPlan& plan) { return 64 * kTiles[plan.tile].fn; }

std::string product_name(ProductKind kind, int dtype, const ProductPlan& plan, Access access) {
  if (plan.few) return std::string("product_rows_") + (dtype == STRIPE_F32 ? "f32_" : "bf16_") + "16x16";
  const TileShape s = kTiles[plan.tile];
  return std::string(access != kAny && !plan.parts ? "product_stream_" : "product_") + (kind == kForward ? "nt_" : kind == kInputGrad ? "nn_" : "tn_") + (dtype == STRIPE_F32 ? "f32_" : "bf16_") +
         std::to_string(64 * s.fm) + "x" + std::to_string(64 * s.fn) + (plan.parts ? "_parts" : access != kAny ? "_s" + std::to_string(s.stages) : "") + (access == kWords && !plan.parts ? "_words" : "") +
         (plan.splits > 1 ? "_k" + std::to_string(plan.splits) : "");
}

hipError_t launch_product(ProductKind kind, int dtype, const ProductPlan& plan, Access access, ProductParams p, hipStream_t stream) {
  if (plan.few) return launch_product_rows(kind, dtype, p, stream);
  return dtype == STRIPE_F32 ? launch_type<float>(kind, plan, access, p, stream) : launch_type<__bf16>(kind, plan, access, p, stream);
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
