// Products of the layers on the gfx950 matrix cores, dense or with rows sorted by group (see ProductKind for the layouts and what follows a product):
// kernels and their launches, which product.hip, gated.hip and xent.hip instantiate for the kinds that they have.
//
// A workgroup of four or eight wavefronts (2 x 2, 2 x 4) computes a tile of BM x BN outputs, in 16 x 16 fragments (32 x 32 ones do as many operations
// per cycle, but draw more power for each: the chip's clock gives way, 4096^3 bf16 on N(0,1) 113 us where 16 x 16 take 99).  K tiles are 128 bytes deep (64 bf16
// or 32 fp32: whole cache lines of a row, where halves of them cost the L2 as much) and lie in a ring of LDS stages:
//   an operand whose reduction index is contiguous in memory ([row][k]): 128 bytes per row, 16-byte piece c of row r in slot
//   c ^ ((r >> 1) & 7); a fragment is one 16-byte read;
//   one whose row index is contiguous ([k][row]): as it lies in memory, a row of BM or BN elements per k, pieces swizzled by k; a bf16
//   fragment is two transposing reads, an fp32 one four 4-byte reads.
// Everything beyond the reduction's end is zero in both operands; rows and columns beyond the output are zeros or repeat valid ones, and their sums
// are never stored.
#pragma once

#include <algorithm>
#include <atomic>

#include "kernels.hpp"
#include "layers_device.hpp"

namespace stripe {
namespace {

typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr int kDepthBytes = 128;      // two matrix-instruction steps

// c[j] += b[j] a^T over 64 bytes of k: lane l holds row l & 15 of a and of b[j], 16-byte piece l >> 4; element v of its c[j] is row l & 15 of a's, row
// 4 (l >> 4) + v of b[j]'s.  (In this order: neighbouring instructions add to different registers, each in place.)
template <typename T, int C>
__device__ __forceinline__ void mma_row(u32x4 a, const u32x4 (&b)[C], f32x4 (&c)[C]) {
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int j = 0; j < C; ++j) c[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, b[j]), __builtin_bit_cast(bf16x8, a), c[j], 0, 0, 0);
  } else {
    const f32x4 x = __builtin_bit_cast(f32x4, a);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < C; ++j) c[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(__builtin_bit_cast(f32x4, b[j])[i], x[i], c[j], 0, 0, 0);
  }
}

// A wavefront's LDS-direct load: lane i's PIECE bytes from offset `from` of the buffer land at lds_off + PIECE i; beyond the buffer: zeros.  Written
// as assembly because the compiler, which cannot tell a load into one ring stage from fragment reads of another, would wait for all of them
// before every LDS read; the kernels wait by count.  M0 is written here and nowhere else (no register array is indexed dynamically,
// nothing else reads M0).
template <int PIECE>
__device__ __forceinline__ void load_to_lds(u32x4 buffer, unsigned from, unsigned lds_off) {
  static_assert(PIECE == 16 || PIECE == 4, "what a lane can load into LDS");
  if constexpr (PIECE == 16)
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" : : "v"(from), "s"(buffer), "s"(lds_off) : "memory", "m0");
  else
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dword %0, %1, 0 offen lds" : : "v"(from), "s"(buffer), "s"(lds_off) : "memory", "m0");
}
template <int N>
__device__ __forceinline__ void wait_loads() {      // until at most N of the wavefront's loads are outstanding
  static_assert(N >= 0 && N < 64, "the counter's range");
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
constexpr uint32_t kOutside = 0x80000000u, kRecords = 0x7fffffffu;      // an offset beyond the buffer, and its size

// One operand's part of a tile: WIDTH rows (or columns) of it.  STRIDED: stored [k][row].
template <typename T, int WIDTH, bool STRIDED, int WAVES = 4>
struct Operand {
  static constexpr int VEC = kVec<T>, DEPTH = kDepthBytes / (int)sizeof(T);
  static constexpr int ROW = STRIDED ? WIDTH * (int)sizeof(T) : kDepthBytes;   // bytes of an LDS row
  static constexpr int STAGE = WIDTH * kDepthBytes, LOADS = STAGE / (1024 * WAVES);   // 16-byte pieces per lane and K tile
  static __device__ __forceinline__ int key(int r) {
    if constexpr (!STRIDED) return (r >> 1) & 7;
    else if constexpr (sizeof(T) == 4) return 4 * ((r >> 2) & 3);              // the wavefront's quarters read k, k + 4, k + 8, k + 12
    else if constexpr (ROW >= 256) return 2 * ((r & 3) | ((r >> 1) & 4));      // half a transposing read takes k = 0 .. 3 and 8 .. 11, 32 bytes of each
    else return 2 * (((r >> 1) & 1) | ((r >> 2) & 2));
  }
  // Fragment i (rows row0 + 16 i .. + 15) of matrix-instruction step s: lane l holds row l & 15 and the 16 bytes of k with number 4 s + (l >> 4).  The
  // swizzles only flip address bits that i and s set, so that one register, first(row0), serves all fragments of a wavefront's rows
  // (row0 a multiple of their number).
  static __device__ __forceinline__ unsigned first(int row0) {
    const int lane = threadIdx.x & 63, fr = lane & 15, fq = lane >> 4;
    if constexpr (!STRIDED) {
      return (row0 + fr) * ROW + ((fq ^ key(fr)) << 4);
    } else if constexpr (sizeof(T) == 2) {
      // within 16 lanes, lane p points at 4 consecutive values of one k; lane i gets, for j = 0 .. 3, value i & 3 of what lane
      // (i >> 2) + 4 j points at: four k of row i
      const int kr = 8 * fq + (fr >> 2);
      return kr * ROW + (((row0 / 8 + ((fr & 3) >> 1)) ^ key(kr)) << 4) + (fr & 1) * 8;
    } else {
      return 4 * fq * ROW + ((((row0 + fr) >> 2) ^ key(4 * fq)) << 4) + (fr & 3) * 4;
    }
  }
  static __device__ __forceinline__ u32x4 fragment(const unsigned char* lds, unsigned first, int i, int s) {
    if constexpr (!STRIDED) {
      return *(const u32x4*)(lds + (first ^ (s << 6)) + i * 16 * ROW);
    } else if constexpr (sizeof(T) == 2) {
      typedef __attribute__((address_space(3))) s16x4* lptr;
      const unsigned char* at = lds + (first ^ (i << 5)) + 32 * s * ROW;
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lptr)at), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lptr)(at + 4 * ROW));
      return __builtin_bit_cast(u32x4, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    } else {
      const unsigned char* at = lds + (first ^ (i << 6)) + 16 * s * ROW;
      u32x4 v;
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = *(const uint32_t*)(at + j * ROW);
      return v;
    }
  }
};

// Where the pieces of an operand come from: any alignment.  Every piece of a K tile that exists as a whole is one 16-byte load without a condition -- a
// load beside a branch would make the compiler wait for all loads at each use, prefetched tiles included.  A strided operand's piece that hangs over the
// last row lies back as far as it hangs over and is shifted when it is used.
template <typename T, int WIDTH, bool STRIDED>
struct Fetch : Operand<T, WIDTH, STRIDED> {
  using Operand<T, WIDTH, STRIDED>::VEC;
  using Operand<T, WIDTH, STRIDED>::DEPTH;
  using Operand<T, WIDTH, STRIDED>::ROW;
  using Operand<T, WIDTH, STRIDED>::LOADS;
  using Operand<T, WIDTH, STRIDED>::key;
  const T* src[LOADS];
  int k[LOADS];                   // its first k
  int back[LOADS];                // elements that the piece lies back (strided)
  int64_t step;                   // elements from one K tile to the next
  int few;                        // strided, fewer rows in all than a piece has elements: their number, else 0
  bool hangs;                     // some piece lies back

  // base: element (row0, k = 0); rows: valid rows from row0 on, behind `before` others; ld: row stride
  __device__ __forceinline__ void init(const T* base, int rows, int before, int64_t ld) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    few = STRIDED && rows + before < VEC ? rows : 0;      // (then row0 = 0)
    hangs = STRIDED && rows < WIDTH && !few;
#pragma unroll
    for (int u = 0; u < LOADS; ++u) {
      const int at = (u * 4 + wave) * 1024 + lane * 16, r = at / ROW, piece = (at % ROW / 16) ^ key(r);
      back[u] = 0;
      if constexpr (!STRIDED) {
        k[u] = piece * VEC;
        src[u] = base + (int64_t)(r < rows ? r : rows - 1) * ld + k[u];
      } else {
        k[u] = r;
        const int over = (piece + 1) * VEC - rows;
        if (hangs && over > 0) back[u] = over;
        src[u] = base + (int64_t)r * ld + piece * VEC - back[u];
      }
    }
    step = STRIDED ? DEPTH * ld : DEPTH;
  }
  // whether K tile kt consists of whole pieces
  __device__ __forceinline__ bool whole(int kt, int K) const { return !few && (kt + 1) * DEPTH <= K; }
  template <bool WHOLE>
  __device__ __forceinline__ void fetch(u32x4 (&to)[LOADS], int kt, int K) const {
    if constexpr (WHOLE) {
#pragma unroll
      for (int u = 0; u < LOADS; ++u) __builtin_memcpy(&to[u], src[u] + (int64_t)kt * step, 16);
    } else {
#pragma unroll
      for (int u = 0; u < LOADS; ++u) {
        const int n = K - (k[u] + kt * DEPTH), left = few - (int)(threadIdx.x % (ROW / 16) ^ key(k[u])) * VEC;
        to[u] = (u32x4){0, 0, 0, 0};
        if (!STRIDED || few) to[u] = load_piece<T>(src[u] + (int64_t)kt * step, !STRIDED ? n : n > 0 ? left : 0);
        else if (n > 0) __builtin_memcpy(&to[u], src[u] + (int64_t)kt * step, 16);
      }
    }
  }
  __device__ __forceinline__ void shift(u32x4 (&v)[LOADS]) const {
    if (!STRIDED || !hangs) return;
#pragma unroll
    for (int u = 0; u < LOADS; ++u) {
      u32x4 x = v[u];
      if constexpr (sizeof(T) == 2) {
        const u32x4 half = {x[0] >> 16 | x[1] << 16, x[1] >> 16 | x[2] << 16, x[2] >> 16 | x[3] << 16, x[3] >> 16};
        x = back[u] & 1 ? half : x;
      }
      const int words = back[u] * (int)sizeof(T) / 4;
      const u32x4 one = {x[1], x[2], x[3], 0};
      x = words & 1 ? one : x;
      const u32x4 two = {x[2], x[3], 0, 0};
      v[u] = words & 2 ? two : x;
    }
  }
  static __device__ __forceinline__ void put(unsigned char* stage, const u32x4 (&from)[LOADS]) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int u = 0; u < LOADS; ++u) *(u32x4*)(stage + (u * 4 + wave) * 1024 + lane * 16) = from[u];
  }
};

// fp32 on the bf16 matrix instructions: v = hi + mid + lo, three bf16 values that hold all 24 bits (each is the rounding of what the ones before it left,
// and the remainders are exact), and a b = lo hi + mid mid + hi lo + mid hi + hi mid + hi hi up to 2^-25 of it.  Six instructions of 16 cycles take the
// place of eight of 32, the fp32 rate's.  LDS holds a plane of each part, a K tile of 32:
//   [row][k]: 64 bytes per row, 16-byte piece c of row r in slot c ^ ((r >> 2) & 3);
//   [k][row]: as a bf16 operand's.
template <int WIDTH, bool STRIDED>
struct Split : Operand<__bf16, WIDTH, STRIDED> {
  using Half = Operand<__bf16, WIDTH, STRIDED>;
  using From = Fetch<float, WIDTH, STRIDED>;
  static constexpr int PLANE = WIDTH * 64, STAGE = 3 * PLANE;
  static __device__ __forceinline__ void split(const u32x4 (&from)[From::LOADS], u32x2 (&part)[From::LOADS][3]) {
#pragma unroll
    for (int u = 0; u < From::LOADS; ++u) {
      f32x4 v = __builtin_bit_cast(f32x4, from[u]);
#pragma unroll
      for (int p = 0; p < 3; ++p) {
        part[u][p] = __builtin_bit_cast(u32x2, __builtin_convertvector(v, bf16x4));
        if (p < 2) {
          const uint32_t x = part[u][p].x, y = part[u][p].y;
          v -= __builtin_bit_cast(f32x4, (u32x4){x << 16, x & 0xffff0000u, y << 16, y & 0xffff0000u});
        }
      }
    }
  }
  static __device__ __forceinline__ void put(unsigned char* stage, const u32x2 (&part)[From::LOADS][3]) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int u = 0; u < From::LOADS; ++u) {
      const int at = (u * 4 + wave) * 1024 + lane * 16, r = at / From::ROW, piece = (at % From::ROW / 16) ^ From::key(r);      // as fetched
      unsigned to;
      if constexpr (!STRIDED) to = r * 64 + (((piece >> 1) ^ ((r >> 2) & 3)) << 4) + (piece & 1) * 8;
      else to = r * Half::ROW + (((piece >> 1) ^ Half::key(r)) << 4) + (piece & 1) * 8;
#pragma unroll
      for (int p = 0; p < 3; ++p) *(u32x2*)(stage + p * PLANE + to) = part[u][p];
    }
  }
  static __device__ __forceinline__ unsigned first(int row0) {
    if constexpr (STRIDED) {
      return Half::first(row0);
    } else {
      const int lane = threadIdx.x & 63, fr = lane & 15;
      return (row0 + fr) * 64 + (((lane >> 4) ^ ((fr >> 2) & 3)) << 4);
    }
  }
  static __device__ __forceinline__ u32x4 fragment(const unsigned char* plane, unsigned first, int i) {
    if constexpr (STRIDED) return Half::fragment(plane, first, i, 0);
    else return *(const u32x4*)(plane + first + i * 16 * 64);
  }
};

// The same as LDS-direct loads of consecutive K tiles, PIECE bytes per lane: 16, which wants operands in whole pieces, or 4 -- four times as many loads, which
// fp32's long matrix instructions hide -- for fp32 at any address.  The buffer's base moves from K tile to K tile (scalar additions); a
// lane's offsets within it stay, 32 bits each (the host has checked that a tile's rows span less than 2^31 bytes).
template <typename T, int WIDTH, bool STRIDED, int WAVES, int PIECE>
struct Stream : Operand<T, WIDTH, STRIDED, WAVES> {
  using Operand<T, WIDTH, STRIDED, WAVES>::VEC;
  using Operand<T, WIDTH, STRIDED, WAVES>::DEPTH;
  using Operand<T, WIDTH, STRIDED, WAVES>::ROW;
  using Operand<T, WIDTH, STRIDED, WAVES>::key;
  static constexpr int LOADS = Operand<T, WIDTH, STRIDED, WAVES>::LOADS * 16 / PIECE, BLOCK = 64 * PIECE;      // bytes of a wavefront's load
  uint64_t base, step;            // of the next K tile, bytes to the one after it
  uint32_t from[LOADS];

  // row of the LDS image that load u of this lane goes to, and its first element there
  static __device__ __forceinline__ void place(int u, int* r, int* e) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, at = (u * WAVES + wave) * BLOCK + lane * PIECE;
    *r = at / ROW;
    *e = ((at % ROW / 16) ^ key(*r)) * VEC + at % 16 / (int)sizeof(T);
  }
  __device__ __forceinline__ void init(const T* at0, int rows, int, int64_t ld) {
#pragma unroll
    for (int u = 0; u < LOADS; ++u) {
      int r, e;
      place(u, &r, &e);
      from[u] = (STRIDED ? e : r) < rows ? (uint32_t)(r * (uint32_t)ld + e) * (uint32_t)sizeof(T) : kOutside;
    }
    const uint64_t b = (uint64_t)(uintptr_t)at0;
    base = (uint64_t)__builtin_amdgcn_readfirstlane((int)(b >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)b);
    step = (STRIDED ? (uint64_t)DEPTH * (uint64_t)ld : (uint64_t)DEPTH) * sizeof(T);
  }
  // From here on only `left` (< DEPTH) of a K tile's depth exist: the reduction's last tile, or none of those behind it.
  __device__ __forceinline__ void cut(int u, int left) {
    int r, e;
    place(u, &r, &e);
    if ((STRIDED ? r : e) >= left) from[u] = kOutside;
  }
  __device__ __forceinline__ void load(int u, unsigned stage) const {
    const u32x4 buffer = {(uint32_t)base, (uint32_t)(base >> 32), kRecords, 0x00020000u};
    load_to_lds<PIECE>(buffer, from[u], stage + u * (BLOCK * WAVES));
  }
};

// The weights of a gated unit: each wavefront's columns of a tile are H rows of W's gate half, then the H rows of its up half that belong to them,
// `half` elements on.  A load of one wavefront lies in one half.
template <typename T, int WIDTH, int H>
struct FetchHalves : Fetch<T, WIDTH, false> {
  using Base = Fetch<T, WIDTH, false>;
  __device__ __forceinline__ void init_halves(const T* base, int rows, int64_t half, int64_t ld) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    this->few = 0;
    this->hangs = false;
#pragma unroll
    for (int u = 0; u < Base::LOADS; ++u) {
      const int at = (u * 4 + wave) * 1024 + lane * 16, r = at / Base::ROW, piece = (at % Base::ROW / 16) ^ Base::key(r), c = r / (2 * H) * H + r % H;
      this->back[u] = 0;
      this->k[u] = piece * Base::VEC;
      this->src[u] = base + (r / H & 1 ? half : 0) + (int64_t)(c < rows ? c : rows - 1) * ld + this->k[u];
    }
    this->step = Base::DEPTH;
  }
};
template <typename T, int WIDTH, int H, int WAVES, int PIECE>
struct StreamHalves : Stream<T, WIDTH, false, WAVES, PIECE> {
  using Base = Stream<T, WIDTH, false, WAVES, PIECE>;
  static_assert(H * kDepthBytes % Base::BLOCK == 0, "a wavefront's load lies in one half");
  uint64_t up;                    // bytes from a gate row to its up row
  int wave;
  __device__ __forceinline__ void init_halves(const T* at0, int rows, int64_t half, int64_t ld) {
    Base::init(at0, 1, 0, ld);
    wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    up = (uint64_t)half * sizeof(T);
#pragma unroll
    for (int u = 0; u < Base::LOADS; ++u) {
      int r, e;
      Base::place(u, &r, &e);
      const int c = r / (2 * H) * H + r % H;
      this->from[u] = c < rows ? (uint32_t)(c * (uint32_t)ld + e) * (uint32_t)sizeof(T) : kOutside;
    }
  }
  __device__ __forceinline__ void load(int u, unsigned stage) const {
    const uint64_t b = this->base + ((u * WAVES + wave) * Base::BLOCK / (H * kDepthBytes) & 1 ? up : 0);
    const u32x4 buffer = {(uint32_t)b, (uint32_t)(b >> 32), kRecords, 0x00020000u};
    load_to_lds<PIECE>(buffer, this->from[u], stage + u * (Base::BLOCK * WAVES));
  }
};

// A tile's second operand; COLS: columns of a wavefront.
template <typename T, int KIND, int WIDTH, int COLS>
using FetchOf = std::conditional_t<KIND == kGated, FetchHalves<T, WIDTH, COLS / 2>, Fetch<T, WIDTH, reduces_rows(KIND)>>;
template <typename T, int KIND, int WIDTH, int COLS, int WAVES, int PIECE>
using StreamOf = std::conditional_t<KIND == kGated, StreamHalves<T, WIDTH, COLS / 2, WAVES, PIECE>, Stream<T, WIDTH, reduces_rows(KIND), WAVES, PIECE>>;

// What a tile is: its place in the output and its part of the reduction.
struct Tile {
  int group, m0, m, n0;         // first output row (kForward, kInputGrad: of all rows), rows, first column
  int k0, k;                    // kWeightGrad: first row of the reduction, and its length
  int slice, slices;            // of a split reduction
  int64_t images;               // rows of a slice's partial image
};

// The slices of kSumGrad's reduction where `count` of its rows count, a number that the host does not know: p.splits are planned for all rows, and the
// workgroups and partial images that all would take make more slices for those that count.  The pass with the logits, all rows and half of them: 512 rows, 50001 -> 4096
// bf16 426 and 249 us (always four slices: 442, 322; always eight: 441, 247); 1500 rows 1085 and 650 (always two: 1169, 827; four: 1177, 672); 512 rows, 32768 -> 2048
// 134 and 109 (always eight: 135, 112; sixteen: 148, 120); 1000 rows, 10007 -> 333 fp32 140 and 90 (always ten: 140, 107).
__device__ __forceinline__ int sum_slices(const ProductParams& p, int count) {
  if (p.splits == 1 || count <= 0) return p.splits;
  const unsigned tiles = (unsigned)((count + p.tile_rows - 1) / p.tile_rows * p.tiles_n), all = (unsigned)(p.tiles_m * p.tiles_n);
  const unsigned workgroups = (all + 7u) / 8u * 8u * (unsigned)p.splits / ((tiles + 7u) / 8u * 8u), images = (unsigned)p.splits * (unsigned)p.M / (unsigned)count;
  const unsigned most = workgroups < images ? workgroups : images;
  return (int)(most < (unsigned)p.most_slices ? most : (unsigned)p.most_slices);
}

// Whether every XCD takes its share of every group's tiles: shares of 4 of a matrix's tiles at least, and no more workgroups than a launch holds.
__host__ __device__ constexpr bool spread(uint64_t tiles, uint64_t groups) { return tiles >= 32 && tiles * groups < 1 << 22; }

// Tiles in patches of PATCH row tiles by all column tiles: neighbouring numbers (one XCD's) share panels of both operands.
template <int KIND, int BM, int BN>
__device__ __forceinline__ bool place(const ProductParams& p, Tile* t) {
  constexpr unsigned PATCH = BM >= 256 ? 4 : 8;
  unsigned row_tiles = (unsigned)p.tiles_m, total, l;
  GroupChunk chunk;      // of up to 64 groups: all of them
  const bool one = KIND >= kLogSum && p.groups;      // a cross entropy's rows are one group, which needs no search
  int start = 0, end = p.M;
  if (one) {
    start = limited(p.offsets[0], p.rows);
    end = limited(p.offsets[1], p.rows);
    end = end > start ? end : start;
  }
  if (!over_rows(KIND) && p.groups) {
    if (one) {
      row_tiles = (unsigned)((end - start + BM - 1) / BM);
    } else if (p.groups <= 64) {
      chunk = group_chunk(p.offsets, p.groups, p.rows, 0, limited(p.offsets[0], p.rows), 0, BM);
      row_tiles = (unsigned)lane_value(chunk.through, 63);
    } else {
      row_tiles = (unsigned)count_row_tiles(p.offsets, p.groups, p.rows, BM);
    }
  }
  total = row_tiles * (unsigned)p.tiles_n;
  t->group = 0;
  t->slice = (int)blockIdx.y;
  t->slices = p.splits;
  t->images = over_rows(KIND) && p.groups ? (int64_t)p.groups * p.M : p.M;
  unsigned number = blockIdx.x;
  if (KIND == kSumGrad) {      // its slices' workgroups follow one another
    const unsigned each = (total + 7u) / 8u * 8u;
    if (!total) return false;
    t->slices = sum_slices(p, end);
    t->images = end;
    t->slice = (int)(number / each);
    if (t->slice >= t->slices) return false;
    number %= each;
  }
  if (over_rows(KIND) && p.groups) {
    unsigned own = total, first = 0;
    if (spread(total, (unsigned)p.groups)) {
      // An eighth of every group's tiles to each XCD: the groups' reductions are of very different lengths (8192 rows in 16 uneven groups, 1024 x 4096 features: 137 us
      // where an XCD had whole groups, 100 here).
      const unsigned x = blockIdx.x & 7u;
      first = total * x >> 3;
      own = (total * (x + 1) >> 3) - first;
      l = blockIdx.x >> 3;
      if (l >= own * (unsigned)p.groups) return false;
    } else if (!logical_number(number, total * (unsigned)p.groups, &l)) {
      return false;
    }
    t->group = (int)(l / own);
    l = first + l % own;
  } else if (!logical_number(number, total, &l)) {
    return false;
  }
  const unsigned per = PATCH * (unsigned)p.tiles_n, patch = l / per, w = l % per;
  const unsigned high = row_tiles - patch * PATCH < PATCH ? row_tiles - patch * PATCH : PATCH;
  const int tm = (int)(patch * PATCH + w % high), tn = (int)(w / high);
  t->n0 = tn * (KIND == kGated ? BN / 2 : BN);
  t->k0 = 0;
  t->k = p.K;
  if (!over_rows(KIND) && one) {
    t->m0 = start + tm * BM;
    t->m = end - t->m0 < BM ? end - t->m0 : BM;
  } else if (!over_rows(KIND) && p.groups) {
    RowTile r = {0, 0, 0};
    if (p.groups <= 64) tile_in_chunk(chunk, 0, BM, tm, &r);
    else r = find_row_tile(p.offsets, p.groups, p.rows, BM, tm);
    t->group = r.group;
    t->m0 = r.row0;
    t->m = r.rows;
  } else {
    t->m0 = tm * BM;
    t->m = p.M - t->m0 < BM ? p.M - t->m0 : BM;
    if (over_rows(KIND) && p.groups) {
      int unused;
      if (one) t->k0 = start;
      else group_rows(p.offsets, p.groups, p.rows, t->group, 1, &t->k0, &end, &unused);
      t->k = end - t->k0;
    }
  }
  return true;
}

// Eight neighbouring outputs of a row: the epilogue in fp32, then one rounding.  at: their place in y, residual and pre (or dx, dW); n: how many of
// them there are; r: the residual's, loaded before.
template <typename T>
struct Eight {
  u32x4 v[sizeof(T) / 2];
  __device__ __forceinline__ void load(const T* q, int n, bool whole) {
    if (whole) {
#pragma unroll
      for (int i = 0; i < (int)sizeof(T) / 2; ++i) v[i] = *(const u32x4*)(q + i * kVec<T>);
    } else {
#pragma unroll
      for (int i = 0; i < (int)sizeof(T) / 2; ++i) v[i] = load_piece<T>(q + i * kVec<T>, n - i * kVec<T>);
    }
  }
  // PAST: past the caches, for what is read again much later if at all (a vocabulary's dW, 50001 x 4096 bf16 of
  // 205 rows: 208 us, 199, and the next product that reads W 140 us, 115).
  template <bool PAST = false>
  __device__ __forceinline__ void store(T* q, int n, bool whole) const {
    if (whole) {
#pragma unroll
      for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
        if constexpr (PAST) __builtin_nontemporal_store(v[i], (u32x4*)(q + i * kVec<T>));
        else *(u32x4*)(q + i * kVec<T>) = v[i];
      }
    } else {
#pragma unroll
      for (int i = 0; i < (int)sizeof(T) / 2; ++i) store_piece<T>(q + i * kVec<T>, v[i], n - i * kVec<T>);
    }
  }
  __device__ __forceinline__ void get(float (&f)[8]) const {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
      float e[kVec<T>];
      unpack<T>(v[i], e);
#pragma unroll
      for (int k = 0; k < kVec<T>; ++k) f[i * kVec<T> + k] = e[k];
    }
  }
  __device__ __forceinline__ void set(const float (&f)[8]) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
      float e[kVec<T>];
#pragma unroll
      for (int k = 0; k < kVec<T>; ++k) e[k] = f[i * kVec<T> + k];
      v[i] = pack<T>(e);
    }
  }
};

constexpr bool scaled(int kind) { return kind == kSumGrad || kind == kLossWeight; }

template <typename T, int KIND>
__device__ __forceinline__ void finish(const ProductParams& p, float scale, int row, int col, int64_t at, int n, float (&v)[8], const float (&bias)[8], const Eight<T>& r) {
  const bool whole = p.vec && n >= 8;
  Eight<T> out;
  if constexpr (KIND == kSumGrad) {
    if (p.sum) {
      Eight<float> sum;
      float* const to = p.sum + (int64_t)row * p.N + col;
      if (!p.first) {
        float f[8];
        sum.load(to, n, false);
        sum.get(f);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += f[e];
      }
      if (!p.last) {
        sum.set(v);
        sum.store(to, n, false);
        return;
      }
    }
    at = (int64_t)p.index[row] * p.c_ld + col;
  }
  if constexpr (scaled(KIND)) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] *= scale;
  }
  if constexpr (KIND == kForward) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] += bias[e];
    if (p.pre) {
      out.set(v);
      out.store((T*)p.pre + at, n, whole);
    }
    activate8<T>(v, p.act);
    if (p.residual) {
      float f[8];
      r.get(f);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += f[e];
    }
  }
  out.set(v);
  out.template store<KIND == kLossWeight>((T*)p.c + at, n, whole);
}

// B's fragments are the matrix instruction's first operand, so that a lane holds four neighbouring columns of a row: 4 (l >> 4) .. + 3 of row l & 15.
// A wavefront lays 64 (or its 32) columns at a time into a part of the idle ring, 16-byte pieces swizzled by the row, and takes them out again
// eight neighbouring columns per lane, eight (16) rows at a time: 128 contiguous bytes of a bf16 row.  A loop and not 256 copies of the
// epilogue: the residual's loads of four turns are on their way together, two sets of them.
template <typename T, int KIND, int FM, int C, int WAVES>
__device__ __forceinline__ void store_tile(const ProductParams& p, const Tile& t, unsigned char* lds, const f32x4 (&acc)[2 * FM][C]) {
  constexpr int PARTS = WAVES / 4, ROWS = FM * 32 / PARTS;                     // a wavefront's rows at a time
  constexpr int COLS = C >= 4 ? 64 : 32, LANES = COLS / 8, HIGH = 64 / LANES;  // lanes to a row, rows of a turn
  constexpr int TURNS = ROWS / HIGH, SET = TURNS < 4 ? TURNS : 4;
  static_assert(C * 16 % COLS == 0 && TURNS % SET == 0, "whole turns");
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm = wave / (WAVES / 2), wn = wave % (WAVES / 2);
  unsigned char* buf = lds + wave * (ROWS * COLS * 4);
  const int fr = lane & 15, fq = lane >> 4, sp = lane / LANES, sc = lane % LANES;
  const int64_t image = over_rows(KIND) ? (int64_t)t.group * p.M : 0;
  const int64_t base = (over_rows(KIND) ? t.group * p.c_group : 0) + (int64_t)t.m0 * p.c_ld;
  auto key = [](int row) { return COLS == 64 ? row & 15 : (row >> 1) & 7; };
  const float scale = scaled(KIND) ? *p.scale : 1.f;
#pragma unroll
  for (int jp = 0; jp < C * 16 / COLS; ++jp) {
    const int col = t.n0 + wn * C * 16 + jp * COLS + 8 * sc, n = p.N - col;
    float bias[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) bias[e] = 0.f;
    const bool residual = KIND == kForward && p.residual && p.splits == 1;
    if constexpr (KIND == kForward)
      if (p.bias && p.splits == 1) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (e < n) bias[e] = p.bias[(int64_t)t.group * p.N + col + e];
      }
    auto load = [&](Eight<T> (&r)[SET], int first) {      // the residual of a set of turns, from the wavefront's row `first` on
#pragma unroll
      for (int q = 0; q < SET; ++q) {
        const int row = wm * FM * 32 + first + q * HIGH + sp;
        if (residual && row < t.m && n > 0) r[q].load((const T*)p.residual + base + (int64_t)row * p.c_ld + col, n, p.vec && n >= 8);
      }
    };
    Eight<T> now[SET], ahead[SET];
    load(now, 0);
    if (jp == 0) __syncthreads();      // every wavefront is done with the ring
#pragma unroll
    for (int part = 0; part < PARTS; ++part) {
#pragma unroll
      for (int i = 0; i < ROWS / 16; ++i)
#pragma unroll
        for (int j = 0; j < COLS / 16; ++j)
          *(f32x4*)(buf + (16 * i + fr) * (COLS * 4) + (((4 * j + fq) ^ key(fr)) << 4)) = acc[part * (ROWS / 16) + i][jp * (COLS / 16) + j];
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
#pragma unroll 1
      for (int turn = 0; turn < TURNS; turn += SET) {
        const int first = part * ROWS + turn * HIGH;
        if (first + SET * HIGH < FM * 32) load(ahead, first + SET * HIGH);
#pragma unroll
        for (int q = 0; q < SET; ++q) {
          const int local = (turn + q) * HIGH + sp, row = wm * FM * 32 + part * ROWS + local;
          float v[8];
          *(f32x4*)v = *(const f32x4*)(buf + local * (COLS * 4) + (((2 * sc) ^ key(local)) << 4));
          *(f32x4*)(v + 4) = *(const f32x4*)(buf + local * (COLS * 4) + (((2 * sc + 1) ^ key(local)) << 4));
          if (row < t.m && n > 0) {
            if (p.splits > 1) {
              Eight<float> out;
              out.set(v);
              out.store(p.partial + (t.slice * t.images + image + t.m0 + row) * p.N + col, n, false);
            } else {
              finish<T, KIND>(p, scale, t.m0 + row, col, base + (int64_t)row * p.c_ld + col, n, v, bias, now[q]);
            }
          }
        }
#pragma unroll
        for (int q = 0; q < SET; ++q) now[q] = ahead[q];
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
  }
}

// Eight neighbouring outputs of a gated unit.
template <typename T>
__device__ __forceinline__ void finish_gated(const ProductParams& p, int64_t row, int col, int n, float (&g)[8], const float (&u)[8]) {
  Eight<T> out;
  if (p.pre) {
    const bool whole = p.vec_pre && n >= 8;
    T* const pre = (T*)p.pre + row * p.pre_ld + col;
    out.set(g);
    out.store(pre, n, whole);
    out.set(u);
    out.store(pre + p.N, n, whole);
  }
  activate8<T>(g, p.act);
#pragma unroll
  for (int e = 0; e < 8; ++e) g[e] *= u[e];
  out.set(g);
  out.store((T*)p.c + row * p.c_ld + col, n, p.vec && n >= 8);
}

// A gated unit's tile: as above, but a wavefront's columns are H of the gate and the same H of up, which a lane takes out together.
template <typename T, int FM, int C, int WAVES>
__device__ __forceinline__ void store_gated(const ProductParams& p, const Tile& t, unsigned char* lds, const f32x4 (&acc)[2 * FM][C]) {
  constexpr int PARTS = WAVES / 4, ROWS = FM * 32 / PARTS;
  constexpr int COLS = 16 * C, H = COLS / 2, LANES = H / 8, HIGH = 64 / LANES, TURNS = ROWS / HIGH;
  static_assert(COLS <= 64 && ROWS % HIGH == 0, "whole turns");
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm = wave / (WAVES / 2), wn = wave % (WAVES / 2);
  unsigned char* buf = lds + wave * (ROWS * COLS * 4);
  const int fr = lane & 15, fq = lane >> 4, sp = lane / LANES, sc = lane % LANES;
  const int col = t.n0 + wn * H + 8 * sc, n = p.N - col;
  auto key = [](int row) { return COLS == 64 ? row & 15 : (row >> 1) & 7; };
  __syncthreads();      // every wavefront is done with the ring
#pragma unroll
  for (int part = 0; part < PARTS; ++part) {
#pragma unroll
    for (int i = 0; i < ROWS / 16; ++i)
#pragma unroll
      for (int j = 0; j < C; ++j) *(f32x4*)(buf + (16 * i + fr) * (COLS * 4) + (((4 * j + fq) ^ key(fr)) << 4)) = acc[part * (ROWS / 16) + i][j];
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
#pragma unroll 1
    for (int turn = 0; turn < TURNS; ++turn) {
      const int local = turn * HIGH + sp, row = wm * FM * 32 + part * ROWS + local;
      float g[8], u[8];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        *(f32x4*)(g + 4 * e) = *(const f32x4*)(buf + local * (COLS * 4) + (((2 * sc + e) ^ key(local)) << 4));
        *(f32x4*)(u + 4 * e) = *(const f32x4*)(buf + local * (COLS * 4) + (((H / 4 + 2 * sc + e) ^ key(local)) << 4));
      }
      if (row < t.m && n > 0) {
        if (p.splits > 1) {
          Eight<float> out;
          float* const to = p.partial + (t.slice * t.images + t.m0 + row) * (2 * (int64_t)p.N) + col;
          out.set(g);
          out.store(to, n, false);
          out.set(u);
          out.store(to + p.N, n, false);
        } else {
          finish_gated<T>(p, t.m0 + row, col, n, g, u);
        }
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
}

// Of each row of a tile of logits: the largest, and the sum of the exponentials of their distances from it (from 0 where it is infinite, so that the sum is
// 0, infinite or NaN as the formula has it); the target's logit where it lies in this tile.  NaN is in the sum only.  The distance is taken first and scaled
// then: its error is half an ulp of the distance, whatever the logits' size, and a part whose largest logit is a mask's -1e30 has the sum 1 or more, as any
// other.  Only tiles at the last class look at each column, only fragments with a target look for it.
constexpr float kLog2E = 1.44269504f;

template <int FM, int C, int WAVES>
__device__ __forceinline__ void store_log_sums(const ProductParams& p, const Tile& t, unsigned char* lds, f32x4 (&acc)[2 * FM][C]) {
  constexpr int R = 2 * FM, WN = WAVES / 2, BM = 64 * FM, BN = 16 * C * WN;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm = wave / WN, wn = wave % WN, fr = lane & 15;
  const int col = t.n0 + wn * C * 16 + 4 * (lane >> 4);      // the lane's first column
  float2* const sums = (float2*)lds;
  int target[R];
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int row = wm * R * 16 + 16 * i + fr;
    target[i] = row < t.m ? (int)((uint32_t)p.targets[t.m0 + row] - (uint32_t)col) : -1;      // (may be none of the classes)
  }
  if (t.n0 + BN > p.N) {
#pragma unroll
    for (int j = 0; j < C; ++j)
#pragma unroll
      for (int v = 0; v < 4; ++v)
        if (col + 16 * j + v >= p.N) {
#pragma unroll
          for (int i = 0; i < R; ++i) acc[i][j][v] = -__builtin_inff();
        }
  }
  __syncthreads();      // every wavefront is done with the ring
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int row = wm * R * 16 + 16 * i + fr;
    if (__any((unsigned)target[i] < 16u * C)) {
#pragma unroll
      for (int j = 0; j < C; ++j)
#pragma unroll
        for (int v = 0; v < 4; ++v)
          if (target[i] == 16 * j + v) p.target_z[t.m0 + row] = acc[i][j][v];      // (of a column behind the last class: nobody reads it)
    }
    float top = acc[i][0][0];
#pragma unroll
    for (int j = 0; j < C; ++j)
#pragma unroll
      for (int v = 0; v < 4; ++v) top = fmaxf(top, acc[i][j][v]);
    top = fmaxf(top, __shfl_xor(top, 16));
    top = fmaxf(top, __shfl_xor(top, 32));
    const float from = __builtin_fabsf(top) < __builtin_inff() ? top : 0.f;
    float sum = 0.f;
#pragma unroll
    for (int j = 0; j < C; ++j)
#pragma unroll
      for (int v = 0; v < 4; ++v) sum += __builtin_amdgcn_exp2f((acc[i][j][v] - from) * kLog2E);
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);
    if (lane < 16) sums[row * WN + wn] = make_float2(top == top ? top : -__builtin_inff(), sum);
  }
  __syncthreads();
  for (int row = threadIdx.x; row < BM && row < t.m; row += 64 * WAVES) {
    float2 s[WN];
    float top = -__builtin_inff(), sum = 0.f;
#pragma unroll
    for (int w = 0; w < WN; ++w) s[w] = sums[row * WN + w], top = fmaxf(top, s[w].x);
    const float from = __builtin_fabsf(top) < __builtin_inff() ? top : 0.f;
#pragma unroll
    for (int w = 0; w < WN; ++w) sum += s[w].y * __builtin_amdgcn_exp2f((s[w].x - from) * kLog2E);
    ((float2*)p.stats)[(int64_t)(t.n0 / BN) * p.M + t.m0 + row] = make_float2(top, sum);
  }
}

// exp(z - lse), a class's part of its row.  Distance first, as above: z log2 e - lse log2 e in fp32 is off by 8 % at logits of 1e6, by everything at 1e8.  No logit
// is above its row's lse; z, added up here in another order than the one that lse came from, may be, by its rounding (NaN stays NaN).
template <typename T>
__device__ __forceinline__ float probability(float z, float lse) {
  return exp_of<T>(__builtin_elementwise_minimum(z - lse, 0.f));
}

// The gradient of the logits, divided by the scale, in place of the logits; zeros behind the last class.
template <typename T, int FM, int C, int WAVES>
__device__ __forceinline__ void loss_gradient(const ProductParams& p, const Tile& t, f32x4 (&acc)[2 * FM][C]) {
  constexpr int R = 2 * FM, WN = WAVES / 2;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm = wave / WN, wn = wave % WN, fr = lane & 15;
  const int col = t.n0 + wn * C * 16 + 4 * (lane >> 4);
  const float inverse = 1.f / *p.scale;
#pragma unroll
  for (int i = 0; i < R; ++i) {
    int row = wm * R * 16 + 16 * i + fr;
    row = t.m0 + (row < t.m ? row : t.m - 1);
    const int target = p.targets[row] - p.class0 - col;
    const float lse = p.row_lse[row], all = p.row_all[row] * inverse, one = p.row_loss[row] * inverse;
#pragma unroll
    for (int j = 0; j < C; ++j)
#pragma unroll
      for (int v = 0; v < 4; ++v) acc[i][j][v] = probability<T>(acc[i][j][v], lse) * all;
    if (__any((unsigned)target < 16u * C)) {
#pragma unroll
      for (int j = 0; j < C; ++j)
#pragma unroll
        for (int v = 0; v < 4; ++v) acc[i][j][v] -= target == 16 * j + v ? one : 0.f;
    }
  }
  if (t.n0 + 16 * C * WN > p.classes) {
#pragma unroll
    for (int j = 0; j < C; ++j)
#pragma unroll
      for (int v = 0; v < 4; ++v)
        if (col + 16 * j + v >= p.classes) {
#pragma unroll
          for (int i = 0; i < R; ++i) acc[i][j][v] = 0.f;
        }
  }
}

// What becomes of a tile's sums.
template <typename T, int KIND, int FM, int C, int WAVES>
__device__ __forceinline__ void finish_tile(const ProductParams& p, const Tile& t, unsigned char* lds, f32x4 (&acc)[2 * FM][C]) {
  if constexpr (KIND == kGated) {
    store_gated<T, FM, C, WAVES>(p, t, lds, acc);
  } else {
    if constexpr (KIND == kLogSum)
      if (p.splits == 1) return store_log_sums<FM, C, WAVES>(p, t, lds, acc);
    if constexpr (KIND == kLossGrad)
      if (p.splits == 1) loss_gradient<T, FM, C, WAVES>(p, t, acc);
    store_tile<T, KIND, FM, C, WAVES>(p, t, lds, acc);
  }
}

template <typename T, int KIND, typename A, typename B>
__device__ __forceinline__ void init_operands(const ProductParams& p, const Tile& t, A& a, B& b) {
  if constexpr (over_rows(KIND)) {
    a.init((const T*)p.a + (int64_t)t.k0 * p.a_ld + t.m0, p.M - t.m0, t.m0, p.a_ld);
    b.init((const T*)p.b + (int64_t)t.k0 * p.b_ld + t.n0, p.N - t.n0, t.n0, p.b_ld);
  } else {
    const T* w = (const T*)p.b + (int64_t)t.group * p.b_group;
    a.init((const T*)p.a + (int64_t)t.m0 * p.a_ld, t.m, 0, p.a_ld);
    if constexpr (KIND == kGated) b.init_halves(w + (int64_t)t.n0 * p.b_ld, p.N - t.n0, p.half, p.b_ld);
    else b.init(reduces_rows(KIND) ? w + t.n0 : w + (int64_t)t.n0 * p.b_ld, (KIND == kLossGrad ? p.classes : p.N) - t.n0, t.n0, p.b_ld);
  }
}
// This workgroup's K tiles of `all`.
__device__ __forceinline__ void own_k_tiles(const Tile& t, int all, int* kt0, int* kt1) {
  *kt0 = 0;
  *kt1 = all;
  if (t.slices > 1) {
    const int per = (all + t.slices - 1) / t.slices;
    *kt0 = t.slice * per < all ? t.slice * per : all;
    *kt1 = *kt0 + per < all ? *kt0 + per : all;
  }
}

// Operands at any alignment, and fp32 in parts: through registers, two stages, two K tiles ahead.  (Parts from an LDS ring of fp32 tiles, split by every
// wavefront that reads them, are twice the splitting: 4096^3 850 us, 800 here.)
// fp32 sums that do not end finite -- an operand was infinite, NaN or within half a bf16 step of overflow, which leave no finite remainder, or a sum came so
// near to overflow that hi hi went beyond it -- are not what fp32 arithmetic gives; their workgroup computes its tile again with fp32
// instructions.
template <typename T, int KIND, int FM, int FN>
__global__ __launch_bounds__(256, 2) void product_kernel(const ProductParams p) {
  constexpr int BM = 64 * FM, BN = 64 * FN, R = 2 * FM, C = 2 * FN;      // fragments of a wavefront
  using A = Fetch<T, BM, over_rows(KIND)>;
  using B = FetchOf<T, KIND, BN, 16 * C>;
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  unsigned char *const lds_a = lds, *const lds_b = lds + 2 * A::STAGE;
  Tile t;
  if (!place<KIND, BM, BN>(p, &t)) return;
  const int wave = threadIdx.x >> 6, wm = wave >> 1, wn = wave & 1;

  A a;
  B b;
  init_operands<T, KIND>(p, t, a, b);
  int kt0, kt1;
  own_k_tiles(t, (t.k + A::DEPTH - 1) / A::DEPTH, &kt0, &kt1);

  f32x4 acc[R][C];
#pragma unroll
  for (int i = 0; i < R; ++i)
#pragma unroll
    for (int j = 0; j < C; ++j) acc[i][j] = (f32x4){0.f, 0.f, 0.f, 0.f};

  u32x4 ra[2][A::LOADS], rb[2][B::LOADS];      // of tiles kt0, kt0 + 2 ..., and of the others
  bool native = true;
  if constexpr (sizeof(T) == 4) {
    using SA = Split<BM, over_rows(KIND)>;
    using SB = Split<BN, reduces_rows(KIND)>;
    unsigned char *const split_a = lds, *const split_b = lds + 2 * SA::STAGE;
    const unsigned first_a = SA::first(wm * R * 16), first_b = SB::first(wn * C * 16);
    // tile kt from stage `at`, while tile kt + 1 (in na, nb) is split and goes to the other stage, and tile kt + 3 is asked for
    auto tile = [&](auto all, int kt, u32x4 (&na)[A::LOADS], u32x4 (&nb)[B::LOADS], int at) {
      constexpr bool WHOLE = decltype(all)::value;
      const unsigned char *const stage_a = split_a + at * SA::STAGE, *const stage_b = split_b + at * SB::STAGE;
      __syncthreads();          // the tile is complete, and the other stage was read
      u32x4 fa[3][R], fb[3][C];
#pragma unroll
      for (int part = 0; part < 3; ++part) {
#pragma unroll
        for (int j = 0; j < C; ++j) fb[part][j] = SB::fragment(stage_b + part * SB::PLANE, first_b, j);
#pragma unroll
        for (int i = 0; i < R; ++i) fa[part][i] = SA::fragment(stage_a + part * SA::PLANE, first_a, i);
      }
      u32x2 pa[A::LOADS][3], pb[B::LOADS][3];
      a.shift(na);
      b.shift(nb);
      SA::split(na, pa);
      SB::split(nb, pb);
      constexpr int ORDER[6][2] = {{0, 0}, {0, 1}, {1, 0}, {1, 1}, {0, 2}, {2, 0}};      // as the parts arrive
#pragma unroll
      for (int o = 0; o < 6; ++o)
#pragma unroll
        for (int i = 0; i < R; ++i) mma_row<__bf16, C>(fa[ORDER[o][0]][i], fb[ORDER[o][1]], acc[i]);
      SA::put(split_a + (at ^ 1) * SA::STAGE, pa);
      SB::put(split_b + (at ^ 1) * SB::STAGE, pb);
      // the splitting runs beside the matrix instructions
#pragma unroll
      for (int i = 0; i < 6 * R * C; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x002, 3, 0);
      }
      a.template fetch<WHOLE>(na, kt + 3, t.k);
      b.template fetch<WHOLE>(nb, kt + 3, t.k);
    };
    {
      u32x2 pa[A::LOADS][3], pb[B::LOADS][3];
      if (a.whole(kt0 + 1, t.k) && b.whole(kt0 + 1, t.k)) {
        a.template fetch<true>(ra[0], kt0, t.k);
        b.template fetch<true>(rb[0], kt0, t.k);
        a.template fetch<true>(ra[1], kt0 + 1, t.k);
        b.template fetch<true>(rb[1], kt0 + 1, t.k);
      } else {
        a.template fetch<false>(ra[0], kt0, t.k);
        b.template fetch<false>(rb[0], kt0, t.k);
        a.template fetch<false>(ra[1], kt0 + 1, t.k);
        b.template fetch<false>(rb[1], kt0 + 1, t.k);
      }
      a.shift(ra[0]);
      b.shift(rb[0]);
      SA::split(ra[0], pa);
      SB::split(rb[0], pb);
      SA::put(split_a, pa);
      SB::put(split_b, pb);
      a.template fetch<false>(ra[0], kt0 + 2, t.k);
      b.template fetch<false>(rb[0], kt0 + 2, t.k);
    }
    int kt = kt0;
    for (; kt + 1 < kt1 && a.whole(kt + 4, t.k) && b.whole(kt + 4, t.k); kt += 2) {
      tile(std::true_type{}, kt, ra[1], rb[1], 0);
      tile(std::true_type{}, kt + 1, ra[0], rb[0], 1);
    }
    for (; kt < kt1; kt += 2) {
      tile(std::false_type{}, kt, ra[1], rb[1], 0);
      if (kt + 1 < kt1) tile(std::false_type{}, kt + 1, ra[0], rb[0], 1);
    }
    native = false;
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
      for (int j = 0; j < C; ++j)
#pragma unroll
        for (int v = 0; v < 4; ++v) native = native || !(__builtin_fabsf(acc[i][j][v]) < __builtin_inff());
    native = __syncthreads_or(native);
    if (native) {
#pragma unroll
      for (int i = 0; i < R; ++i)
#pragma unroll
        for (int j = 0; j < C; ++j) acc[i][j] = (f32x4){0.f, 0.f, 0.f, 0.f};
    }
  }
  if (native) {
    const unsigned first_a = A::first(wm * R * 16), first_b = B::first(wn * C * 16);
    auto tile = [&](auto all, int kt, u32x4 (&na)[A::LOADS], u32x4 (&nb)[B::LOADS], int stage) {
      constexpr bool WHOLE = decltype(all)::value;
      a.shift(na);
      b.shift(nb);
      A::put(lds_a + stage * A::STAGE, na);
      B::put(lds_b + stage * B::STAGE, nb);
      __syncthreads();
      a.template fetch<WHOLE>(na, kt + 2, t.k);
      b.template fetch<WHOLE>(nb, kt + 2, t.k);
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        u32x4 fa[R], fb[C];
#pragma unroll
        for (int i = 0; i < R; ++i) fa[i] = A::fragment(lds_a + stage * A::STAGE, first_a, i, s);
#pragma unroll
        for (int j = 0; j < C; ++j) fb[j] = B::fragment(lds_b + stage * B::STAGE, first_b, j, s);
#pragma unroll
        for (int i = 0; i < R; ++i) mma_row<T, C>(fa[i], fb, acc[i]);
      }
    };
    if (sizeof(T) == 4) __syncthreads();      // the parts' stages were read
    a.template fetch<false>(ra[0], kt0, t.k);
    b.template fetch<false>(rb[0], kt0, t.k);
    a.template fetch<false>(ra[1], kt0 + 1, t.k);
    b.template fetch<false>(rb[1], kt0 + 1, t.k);
    int kt = kt0;
    for (; kt + 1 < kt1 && a.whole(kt + 3, t.k) && b.whole(kt + 3, t.k); kt += 2) {
      tile(std::true_type{}, kt, ra[0], rb[0], 0);
      tile(std::true_type{}, kt + 1, ra[1], rb[1], 1);
    }
    for (; kt < kt1; kt += 2) {
      tile(std::false_type{}, kt, ra[0], rb[0], 0);
      if (kt + 1 < kt1) tile(std::false_type{}, kt + 1, ra[1], rb[1], 1);
    }
  }
  finish_tile<T, KIND, FM, C, 4>(p, t, lds, acc);
}

// Operands in whole 16-byte pieces: LDS-direct loads into a ring of S stages, one barrier for each K tile.  A K tile is two matrix-instruction steps of R
// fragment rows each, and beside the rows' matrix instructions go
//   rows 0 .. R - 1             the fragment reads of step 1,
//   rows 0 .. R/2 - 1           the second half of tile kt + S - 1's loads,
//   behind row R + R/2 - 1      wait, barrier: tile kt + 1 is complete in LDS, and everybody has read the whole of tile kt,
//   rows R + R/2 .. 2 R - 1     the fragment reads of tile kt + 1's step 0, and the first half of tile kt + S's loads, into tile kt's stage.
// (All of a tile's loads behind the barrier: 4096^3 on zeros 94 us instead of 87; over three quarters of a tile: 90.)
// Behind the last tile the loop loads zeros and reads fragments that nobody uses: the counts then never change.
// Tiles of 256 x 256, whose two stages leave 32 KB of LDS: a third stage of B (SB = S + 1), the operand that more often comes from memory (weights; A's
// panels are shared by more tiles).  Both loads of a tile are then for K tile kt + 2, B's with 1 3/4 tiles of time to arrive instead of 3/4
// (inputs from memory, bf16: a gated unit of 4096 rows, 4096 -> 8192 432 -> 405 us; 8192 rows in 16 groups, 1024 -> 2048 with gradients 347 -> 321; the cross
// entropy of 8192 rows, 2048 -> 65536 with gradients 6.45 -> 6.30 ms).
#define PRODUCT_FENCE() __builtin_amdgcn_sched_barrier(0)

template <typename T, int KIND, int FM, int FN, int S, int SB, int WAVES, int PIECE>
__global__ __launch_bounds__(64 * WAVES, S * 64 * (FM + FN) * kDepthBytes > 80 * 1024 ? 1 : 2) void product_stream_kernel(const ProductParams p) {
  constexpr int BM = 64 * FM, BN = 64 * FN, R = 2 * FM, C = 8 * FN / WAVES;      // fragments of a wavefront
  using A = Stream<T, BM, over_rows(KIND), WAVES, PIECE>;
  using B = StreamOf<T, KIND, BN, 16 * C, WAVES, PIECE>;
  constexpr int LOADS = A::LOADS + B::LOADS, HALF = R / 2;
  constexpr bool MORE = SB == S + 1;
  static_assert(MORE ? S == 2 && A::LOADS == B::LOADS : SB == S, "the first half of a tile's loads is A's, the second B's");
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  unsigned char *const lds_a = lds, *const lds_b = lds + S * A::STAGE;
  Tile t;
  if (!place<KIND, BM, BN>(p, &t)) return;
  const int wave = threadIdx.x >> 6, wm = wave / (WAVES / 2), wn = wave % (WAVES / 2);
  A a;
  B b;
  init_operands<T, KIND>(p, t, a, b);
  int kt0, kt1;
  own_k_tiles(t, (t.k + A::DEPTH - 1) / A::DEPTH, &kt0, &kt1);

  f32x4 acc[R][C];
#pragma unroll
  for (int i = 0; i < R; ++i)
#pragma unroll
    for (int j = 0; j < C; ++j) acc[i][j] = (f32x4){0.f, 0.f, 0.f, 0.f};

  if (kt0 < kt1) {
    int left = (kt1 * A::DEPTH < t.k ? kt1 * A::DEPTH : t.k) - kt0 * A::DEPTH;      // of this workgroup's part of the reduction, from the next tile on
    a.base += (uint64_t)kt0 * a.step;
    b.base += (uint64_t)kt0 * b.step;
    const unsigned own = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)) * A::BLOCK;
    auto load = [&](int first, int last, int stage) {
#pragma unroll
      for (int u = 0; u < LOADS; ++u)
        if (u >= first && u < last) {
          if (u < A::LOADS) a.load(u, own + stage * A::STAGE);
          else b.load(u - A::LOADS, own + S * A::STAGE + stage * B::STAGE);
        }
    };
    // pieces first .. last - 1 of a tile are about to be loaded, `depth` of whose k exist (the last one, or none behind it)
    auto cut = [&](int first, int last, int depth) {
      if (depth >= A::DEPTH) return;
#pragma unroll
      for (int u = 0; u < LOADS; ++u)
        if (u >= first && u < last) {
          if (u < A::LOADS) a.cut(u, depth);
          else b.cut(u - A::LOADS, depth);
        }
    };
    auto next = [&] {
      left -= A::DEPTH;
      a.base += a.step;
      b.base += b.step;
    };
#pragma unroll
    for (int i = 0; i < S - !MORE; ++i) {
      cut(0, LOADS, left);
      load(0, LOADS, i);
      next();
    }
    if constexpr (MORE) {
      wait_loads<LOADS>();
    } else {
      cut(0, LOADS / 2, left);
      load(0, LOADS / 2, S - 1);
      wait_loads<LOADS / 2 + (S - 2) * LOADS>();
    }
    asm volatile("s_barrier" ::: "memory");
    const unsigned first_a = A::first(wm * R * 16), first_b = B::first(wn * C * 16);
    u32x4 fa[R], fb[2][C];
#pragma unroll
    for (int j = 0; j < C; ++j) fb[0][j] = B::fragment(lds_b, first_b, j, 0);
#pragma unroll
    for (int i = 0; i < R; ++i) fa[i] = A::fragment(lds_a, first_a, i, 0);

    const int tiles = kt1 - kt0;
    int cur = 0, before = SB - 1;              // stages of tile kt and, of B, of tile kt - 1
    int at_b = 0;                              // B's stage of tile kt
    for (int kt = 0; kt < tiles; ++kt) {
      const int nxt = cur + 1 == S ? 0 : cur + 1, next_b = at_b + 1 == SB ? 0 : at_b + 1;
      if (left < (MORE ? 1 : 2) * A::DEPTH) {      // (here and not beside the loads: the rest of the loop is one block)
        cut(LOADS / 2, LOADS, left);
        cut(0, LOADS / 2, MORE ? left : left - A::DEPTH);
      }
      unsigned cur_a = first_a + cur * A::STAGE, cur_b = first_b + at_b * B::STAGE, nxt_a = first_a + nxt * A::STAGE, nxt_b = first_b + next_b * B::STAGE;
      // (opaque: else every fragment's address would be kept in a register of its own over the whole loop)
      asm volatile("" : "+v"(cur_a), "+v"(cur_b), "+v"(nxt_a), "+v"(nxt_b));
      auto read_b = [&](int st, unsigned at, int first, int last) {
#pragma unroll
        for (int j = 0; j < C; ++j)
          if (j >= first && j < last) fb[st][j] = B::fragment(lds_b, at, j, st);
      };
      auto read_a = [&](int st, unsigned at, int first, int last) {
#pragma unroll
        for (int i = 0; i < R; ++i)
          if (i >= first && i < last) fa[i] = A::fragment(lds_a, at, i, st);
      };
#pragma unroll
      for (int row = 0; row < 2 * R; ++row) {
        const int st = row / R, i = row % R;
        if (row == R + HALF) {
          asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((S - 2) * LOADS + (MORE ? LOADS / 2 : 0)) : "memory");
          asm volatile("s_barrier" ::: "memory");
          PRODUCT_FENCE();
        }
        mma_row<T, C>(fa[i], fb[st], acc[i]);
        if (row < R) {
          read_a(1, cur_a, row, row + 1);
          read_b(1, cur_b, row * C / R, (row + 1) * C / R);
        }
        if (row < HALF) load(LOADS / 2 + row * (LOADS / 2) / HALF, LOADS / 2 + (row + 1) * (LOADS / 2) / HALF, before);
        if (row >= R + HALF) {
          // B's fragments and A's first ones, which were used before the barrier, in the first half of these rows; the others behind their use
          const int at = row - R - HALF, early = HALF > 1 ? HALF / 2 : 1;
          if (at < early) read_b(0, nxt_b, at * C / early, (at + 1) * C / early);
          if (at < early) read_a(0, nxt_a, at * HALF / early, (at + 1) * HALF / early);
          read_a(0, nxt_a, HALF + at, HALF + at + 1);
          load(at * (LOADS / 2) / HALF, (at + 1) * (LOADS / 2) / HALF, cur);
        }
        PRODUCT_FENCE();
        if (row == (MORE ? 2 * R - 1 : HALF - 1)) next();
      }
      before = at_b;
      at_b = next_b;
      cur = nxt;
    }
    wait_loads<0>();
  }
  finish_tile<T, KIND, FM, C, WAVES>(p, t, lds, acc);
}

// The slices of a split reduction, added in their order, and the epilogue: one row (blockIdx.x / strips), 2048 columns.
template <typename T, int KIND>
__global__ __launch_bounds__(256) void product_join_kernel(const ProductParams p, int strips) {
  const int row = (int)(blockIdx.x / (unsigned)strips), col = ((int)(blockIdx.x % (unsigned)strips) * 256 + (int)threadIdx.x) * 8, n = p.N - col;
  int64_t images = over_rows(KIND) && p.groups ? (int64_t)p.groups * p.M : p.M;
  int group = 0, slices = p.splits;
  int64_t at = (int64_t)row * p.c_ld + col;
  if (over_rows(KIND)) {
    group = row / p.M;
    at = group * p.c_group + (int64_t)(row % p.M) * p.c_ld + col;
  } else if (p.groups) {
    group = group_of_row(p.offsets, p.groups, p.rows, row);
    if (group < 0) return;
    if (KIND == kSumGrad) {
      images = limited(p.offsets[1], p.rows);
      slices = sum_slices(p, (int)images);
    }
  }
  if (n <= 0) return;
  float v[8], bias[8];
  auto total = [&](float (&v)[8], int64_t image, const float* from) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = 0.f;
#pragma unroll 4
    for (int s = 0; s < slices; ++s) {
      Eight<float> part;
      part.load(from + (int64_t)s * image, n, false);
      float f[8];
      part.get(f);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += f[e];
    }
  };
  if constexpr (KIND == kGated) {
    float u[8];
    const float* from = p.partial + (int64_t)row * 2 * p.N + col;
    total(v, images * 2 * p.N, from);
    total(u, images * 2 * p.N, from + p.N);
    finish_gated<T>(p, row, col, n, v, u);
    return;
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) bias[e] = 0.f;
  total(v, images * p.N, p.partial + (int64_t)row * p.N + col);
  if constexpr (KIND == kLossGrad) {
    const float inverse = 1.f / *p.scale, lse = p.row_lse[row], all = p.row_all[row] * inverse, one = p.row_loss[row] * inverse;
    const int target = p.targets[row] - p.class0 - col;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = col + e < p.classes ? probability<T>(v[e], lse) * all - (target == e ? one : 0.f) : 0.f;
  }
  Eight<T> r;
  if constexpr (KIND == kForward) {
    if (p.bias) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < n) bias[e] = p.bias[(int64_t)group * p.N + col + e];
    }
    if (p.residual) r.load((const T*)p.residual + at, n, p.vec && n >= 8);
  }
  finish<T, KIND>(p, scaled(KIND) ? *p.scale : 1.f, row, col, at, n, v, bias, r);
}

// ---- host ---------------------------------------------------------------------
struct TileShape {
  int fm, fn, stages, stages_b, resident, waves;      // resident: workgroups that fit a CU
};
// What each is for, bf16: 0 many outputs (4096^3: 101 us, 105 and 146 on the next two); 1 half as many, or groups of a few hundred rows (8192 rows of
// 32 groups, 2048 -> 4096: 216, 199, 274; 2048 x 4096 x 4096: 73, 54, 73); 2 few of them, and fp32, whose matrix instructions take so long that
// nothing else matters; 3 so few that tile 2's would leave CUs idle (1024^3: 8.5 us on tile 2, 6.9; fp32 1000^3: 27.3 and 21.5; 777 rows of 5
// groups, 200 -> 328, fp32: 12.0 and 8.2).  Operands that are no whole 16-byte pieces: fp32 loads words into LDS instead (1000 x 777 x 1283: 31 us
// and 32 through the registers; 333 x 555 x 777: 12.7 and 15.0), bf16 runs on product_kernel in tile 2's shape.
constexpr TileShape kTiles[] = {{4, 4, 2, 3, 1, 8}, {2, 4, 3, 3, 1, 8}, {1, 2, 3, 3, 2, 4}, {1, 1, 4, 4, 2, 4}};
constexpr int kTileCount = 4, kSmallTile = 2, kLeastTile = 3;

// A kernel's LDS beyond 64 KB has to be allowed once on each device.
template <typename K>
hipError_t allow_lds(K kernel, int bytes, std::atomic<uint64_t>& done) {
  int dev = 0;
  if (const hipError_t e = hipGetDevice(&dev); e != hipSuccess) return e;
  const uint64_t bit = dev < 64 ? (uint64_t)1 << dev : 0;
  if (done.load(std::memory_order_relaxed) & bit) return hipSuccess;
  const hipError_t e = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == hipSuccess) done.fetch_or(bit, std::memory_order_relaxed);
  return e;
}

template <typename T, int KIND, int TILE, int PIECE = 16>
hipError_t launch_stream(const ProductParams& p, dim3 grid, hipStream_t stream) {
  constexpr TileShape s = kTiles[TILE];
  constexpr int bytes = 64 * (s.stages * s.fm + s.stages_b * s.fn) * kDepthBytes;
  if constexpr (bytes > 65536) {
    static std::atomic<uint64_t> done{0};
    if (const hipError_t e = allow_lds(product_stream_kernel<T, KIND, s.fm, s.fn, s.stages, s.stages_b, s.waves, PIECE>, bytes, done); e != hipSuccess) return e;
  }
  product_stream_kernel<T, KIND, s.fm, s.fn, s.stages, s.stages_b, s.waves, PIECE><<<grid, dim3(64 * s.waves), bytes, stream>>>(p);
  return hipGetLastError();
}

template <typename T, int KIND>
hipError_t launch_kind(const ProductPlan& plan, Access access, ProductParams& p, hipStream_t stream) {
  const TileShape s = kTiles[plan.tile];
  const int bm = 64 * s.fm, bn = KIND == kGated ? 32 * s.fn : 64 * s.fn;      // (outputs)
  p.tiles_n = (p.N + bn - 1) / bn;
  p.tiles_m = (p.M + bm - 1) / bm;
  p.splits = plan.splits;
  int64_t total = (int64_t)p.tiles_m * p.tiles_n;
  if (p.groups) {
    // every group's last tile may be part of one
    if (over_rows(KIND)) total = (spread((uint64_t)total, (uint64_t)p.groups) ? (total + 7) / 8 * 8 : total) * p.groups;
    else total = ((int64_t)p.M / bm + std::min<int64_t>(p.groups, p.M)) * p.tiles_n;
  }
  dim3 grid((unsigned)((total + 7) / 8 * 8), (unsigned)plan.splits);
  if (KIND == kSumGrad) {
    const int depth = kDepthBytes / (int)sizeof(T);
    p.tile_rows = bm;
    p.most_slices = std::max(plan.splits, (p.K + depth - 1) / depth / 2);
    grid = dim3((unsigned)(((int64_t)p.tiles_m * p.tiles_n + 7) / 8 * 8 * plan.splits));
  }
  hipError_t e = hipSuccess;
  if (access == kWords && !plan.parts) {
    if constexpr (sizeof(T) == 4) e = plan.tile == kLeastTile ? launch_stream<T, KIND, kLeastTile, 4>(p, grid, stream) : launch_stream<T, KIND, kSmallTile, 4>(p, grid, stream);
  } else if (access == kPieces && !plan.parts) {
    if (plan.tile == kLeastTile) e = launch_stream<T, KIND, kLeastTile>(p, grid, stream);
    else if (sizeof(T) == 4 || plan.tile == kSmallTile) e = launch_stream<T, KIND, kSmallTile>(p, grid, stream);
    else if constexpr (sizeof(T) == 2) e = plan.tile == 0 ? launch_stream<T, KIND, 0>(p, grid, stream) : launch_stream<T, KIND, 1>(p, grid, stream);
  } else {
    constexpr TileShape s = kTiles[kSmallTile];
    constexpr int bytes = 2 * 64 * (s.fm + s.fn) * (sizeof(T) == 4 ? 3 * 64 : kDepthBytes);
    if constexpr (bytes > 65536) {
      static std::atomic<uint64_t> done{0};
      if (e = allow_lds(product_kernel<T, KIND, s.fm, s.fn>, bytes, done); e != hipSuccess) return e;
    }
    product_kernel<T, KIND, s.fm, s.fn><<<grid, dim3(256), bytes, stream>>>(p);
    e = hipGetLastError();
  }
  if (e != hipSuccess || plan.splits == 1 || KIND == kLogSum) return e;      // (its join is xent.hip's)
  const int strips = (p.N + 2047) / 2048;
  const int64_t rows = over_rows(KIND) ? (int64_t)std::max(1, p.groups) * p.M : p.M;
  product_join_kernel<T, KIND><<<dim3((unsigned)(rows * strips)), dim3(256), 0, stream>>>(p, strips);
  return hipGetLastError();
}
}  // namespace
}  // namespace stripe
