// Products of the linear layer on the gfx950 matrix cores, dense or with rows sorted by group (see ProductKind for the three
// layouts).
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
#include <algorithm>
#include <atomic>
#include <cmath>

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
  GroupChunk chunk;      // of up to 64 groups: all of them
  if (KIND != kWeightGrad && p.groups) {
    if (p.groups <= 64) {
      chunk = group_chunk(p.offsets, p.groups, p.rows, 0, limited(p.offsets[0], p.rows), 0, BM);
      row_tiles = (unsigned)lane_value(chunk.through, 63);
    } else {
      row_tiles = (unsigned)count_row_tiles(p.offsets, p.groups, p.rows, BM);
    }
  }
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
    RowTile r = {0, 0, 0};
    if (p.groups <= 64) tile_in_chunk(chunk, 0, BM, tm, &r);
    else r = find_row_tile(p.offsets, p.groups, p.rows, BM, tm);
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
  __device__ __forceinline__ void store(T* q, int n, bool whole) const {
    if (whole) {
#pragma unroll
      for (int i = 0; i < (int)sizeof(T) / 2; ++i) *(u32x4*)(q + i * kVec<T>) = v[i];
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

template <typename T, int KIND>
__device__ __forceinline__ void finish(const ProductParams& p, int64_t at, int n, float (&v)[8], const float (&bias)[8], const Eight<T>& r) {
  const bool whole = p.vec && n >= 8;
  Eight<T> out;
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
  out.store((T*)p.c + at, n, whole);
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
  const int64_t image = KIND == kWeightGrad ? (int64_t)t.group * p.M : 0;
  const int64_t images = KIND == kWeightGrad && p.groups ? (int64_t)p.groups * p.M : p.M;
  const int64_t base = (KIND == kWeightGrad ? t.group * p.c_group : 0) + (int64_t)t.m0 * p.c_ld;
  auto key = [](int row) { return COLS == 64 ? row & 15 : (row >> 1) & 7; };
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
              out.store(p.partial + ((int64_t)blockIdx.y * images + image + t.m0 + row) * p.N + col, n, false);
            } else {
              finish<T, KIND>(p, base + (int64_t)row * p.c_ld + col, n, v, bias, now[q]);
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

template <typename T, int KIND, typename A, typename B>
__device__ __forceinline__ void init_operands(const ProductParams& p, const Tile& t, A& a, B& b) {
  if constexpr (KIND == kWeightGrad) {
    a.init((const T*)p.a + (int64_t)t.k0 * p.a_ld + t.m0, p.M - t.m0, t.m0, p.a_ld);
    b.init((const T*)p.b + (int64_t)t.k0 * p.b_ld + t.n0, p.N - t.n0, t.n0, p.b_ld);
  } else {
    const T* w = (const T*)p.b + (int64_t)t.group * p.b_group;
    a.init((const T*)p.a + (int64_t)t.m0 * p.a_ld, t.m, 0, p.a_ld);
    b.init(KIND == kForward ? w + (int64_t)t.n0 * p.b_ld : w + t.n0, p.N - t.n0, t.n0, p.b_ld);
  }
}
// This workgroup's K tiles of `all`.
__device__ __forceinline__ void own_k_tiles(const ProductParams& p, int all, int* kt0, int* kt1) {
  *kt0 = 0;
  *kt1 = all;
  if (p.splits > 1) {
    const int per = (all + p.splits - 1) / p.splits;
    *kt0 = (int)blockIdx.y * per < all ? (int)blockIdx.y * per : all;
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
  using A = Fetch<T, BM, KIND == kWeightGrad>;
  using B = Fetch<T, BN, KIND != kForward>;
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  unsigned char *const lds_a = lds, *const lds_b = lds + 2 * A::STAGE;
  Tile t;
  if (!place<KIND, BM, BN>(p, &t)) return;
  const int wave = threadIdx.x >> 6, wm = wave >> 1, wn = wave & 1;

  A a;
  B b;
  init_operands<T, KIND>(p, t, a, b);
  int kt0, kt1;
  own_k_tiles(p, (t.k + A::DEPTH - 1) / A::DEPTH, &kt0, &kt1);

  f32x4 acc[R][C];
#pragma unroll
  for (int i = 0; i < R; ++i)
#pragma unroll
    for (int j = 0; j < C; ++j) acc[i][j] = (f32x4){0.f, 0.f, 0.f, 0.f};

  u32x4 ra[2][A::LOADS], rb[2][B::LOADS];      // of tiles kt0, kt0 + 2 ..., and of the others
  bool native = true;
  if constexpr (sizeof(T) == 4) {
    using SA = Split<BM, KIND == kWeightGrad>;
    using SB = Split<BN, KIND != kForward>;
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
  store_tile<T, KIND, FM, C, 4>(p, t, lds, acc);
}

// Operands in whole 16-byte pieces: LDS-direct loads into a ring of S stages, one barrier for each K tile.  A K tile is two matrix-instruction steps of R
// fragment rows each, and beside the rows' matrix instructions go
//   rows 0 .. R - 1             the fragment reads of step 1,
//   rows 0 .. R/2 - 1           the second half of tile kt + S - 1's loads,
//   behind row R + R/2 - 1      wait, barrier: tile kt + 1 is complete in LDS, and everybody has read the whole of tile kt,
//   rows R + R/2 .. 2 R - 1     the fragment reads of tile kt + 1's step 0, and the first half of tile kt + S's loads, into tile kt's stage.
// (All of a tile's loads behind the barrier: 4096^3 on zeros 94 us instead of 87; over three quarters of a tile: 90.)
// Behind the last tile the loop loads zeros and reads fragments that nobody uses: the counts then never change.
#define PRODUCT_FENCE() __builtin_amdgcn_sched_barrier(0)

template <typename T, int KIND, int FM, int FN, int S, int WAVES, int PIECE>
__global__ __launch_bounds__(64 * WAVES, S * 64 * (FM + FN) * kDepthBytes > 80 * 1024 ? 1 : 2) void product_stream_kernel(const ProductParams p) {
  constexpr int BM = 64 * FM, BN = 64 * FN, R = 2 * FM, C = 8 * FN / WAVES;      // fragments of a wavefront
  using A = Stream<T, BM, KIND == kWeightGrad, WAVES, PIECE>;
  using B = Stream<T, BN, KIND != kForward, WAVES, PIECE>;
  constexpr int LOADS = A::LOADS + B::LOADS, HALF = R / 2;
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  unsigned char *const lds_a = lds, *const lds_b = lds + S * A::STAGE;
  Tile t;
  if (!place<KIND, BM, BN>(p, &t)) return;
  const int wave = threadIdx.x >> 6, wm = wave / (WAVES / 2), wn = wave % (WAVES / 2);
  A a;
  B b;
  init_operands<T, KIND>(p, t, a, b);
  int kt0, kt1;
  own_k_tiles(p, (t.k + A::DEPTH - 1) / A::DEPTH, &kt0, &kt1);

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
    for (int i = 0; i < S - 1; ++i) {
      cut(0, LOADS, left);
      load(0, LOADS, i);
      next();
    }
    cut(0, LOADS / 2, left);
    load(0, LOADS / 2, S - 1);
    wait_loads<LOADS / 2 + (S - 2) * LOADS>();
    asm volatile("s_barrier" ::: "memory");
    const unsigned first_a = A::first(wm * R * 16), first_b = B::first(wn * C * 16);
    u32x4 fa[R], fb[2][C];
#pragma unroll
    for (int j = 0; j < C; ++j) fb[0][j] = B::fragment(lds_b, first_b, j, 0);
#pragma unroll
    for (int i = 0; i < R; ++i) fa[i] = A::fragment(lds_a, first_a, i, 0);

    const int tiles = kt1 - kt0;
    int cur = 0, before = S - 1;      // stages of tile kt and of tile kt - 1
    for (int kt = 0; kt < tiles; ++kt) {
      const int nxt = cur + 1 == S ? 0 : cur + 1;
      if (left < 2 * A::DEPTH) {      // (here and not beside the loads: the rest of the loop is one block)
        cut(LOADS / 2, LOADS, left);
        cut(0, LOADS / 2, left - A::DEPTH);
      }
      unsigned cur_a = first_a + cur * A::STAGE, cur_b = first_b + cur * B::STAGE, nxt_a = first_a + nxt * A::STAGE, nxt_b = first_b + nxt * B::STAGE;
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
          asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((S - 2) * LOADS) : "memory");
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
        if (row == HALF - 1) next();
      }
      before = cur;
      cur = nxt;
    }
    wait_loads<0>();
  }
  store_tile<T, KIND, FM, C, WAVES>(p, t, lds, acc);
}

// The slices of a split reduction, added in their order, and the epilogue: one row (blockIdx.x / strips), 2048 columns.
template <typename T, int KIND>
__global__ __launch_bounds__(256) void product_join_kernel(const ProductParams p, int strips) {
  const int row = (int)(blockIdx.x / (unsigned)strips), col = ((int)(blockIdx.x % (unsigned)strips) * 256 + (int)threadIdx.x) * 8, n = p.N - col;
  const int64_t images = KIND == kWeightGrad && p.groups ? (int64_t)p.groups * p.M : p.M;
  int group = 0;
  int64_t at = (int64_t)row * p.c_ld + col;
  if (KIND == kWeightGrad) {
    group = row / p.M;
    at = group * p.c_group + (int64_t)(row % p.M) * p.c_ld + col;
  } else if (p.groups) {
    group = group_of_row(p.offsets, p.groups, p.rows, row);
    if (group < 0) return;
  }
  if (n <= 0) return;
  float v[8], bias[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = bias[e] = 0.f;
  const float* from = p.partial + (int64_t)row * p.N + col;
#pragma unroll 4
  for (int s = 0; s < p.splits; ++s) {
    Eight<float> part;
    part.load(from + (int64_t)s * images * p.N, n, false);
    float f[8];
    part.get(f);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] += f[e];
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
  finish<T, KIND>(p, at, n, v, bias, r);
}

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
struct TileShape {
  int fm, fn, stages, resident, waves;      // resident: workgroups that fit a CU
};
// What each is for, bf16: 0 many outputs (4096^3: 100 us, 112 and 150 on the next two); 1 half as many, or groups of a few hundred rows (8192 rows of
// 32 groups, 2048 -> 4096: 216, 199, 274; 2048 x 4096 x 4096: 83, 57, 76); 2 few of them, and fp32, whose matrix instructions take so long that
// nothing else matters; 3 so few that tile 2's would leave CUs idle (1024^3: 8.5 us on tile 2, 6.9; fp32 1000^3: 27.3 and 21.5; 777 rows of 5
// groups, 200 -> 328, fp32: 12.0 and 8.2).  Operands that are no whole 16-byte pieces: fp32 loads words into LDS instead (1000 x 777 x 1283: 31 us
// and 32 through the registers; 333 x 555 x 777: 12.7 and 15.0), bf16 runs on product_kernel in tile 2's shape.
constexpr TileShape kTiles[] = {{4, 4, 2, 1, 8}, {2, 4, 3, 1, 8}, {1, 2, 3, 2, 4}, {1, 1, 4, 2, 4}};
constexpr int kTileCount = 4, kSmallTile = 2, kLeastTile = 3;

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
  constexpr TileTime t[] = {{1.1, 1.45, 6, 9}, {0.56, 0.76, 4, 5}, {0.28, 0.5, 3, 5}, {0.22, 0.35, 2, 4}};
  return t[tile];
}

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
  constexpr int bytes = s.stages * 64 * (s.fm + s.fn) * kDepthBytes;
  if constexpr (bytes > 65536) {
    static std::atomic<uint64_t> done{0};
    if (const hipError_t e = allow_lds(product_stream_kernel<T, KIND, s.fm, s.fn, s.stages, s.waves, PIECE>, bytes, done); e != hipSuccess) return e;
  }
  product_stream_kernel<T, KIND, s.fm, s.fn, s.stages, s.waves, PIECE><<<grid, dim3(64 * s.waves), bytes, stream>>>(p);
  return hipGetLastError();
}

template <typename T, int KIND>
hipError_t launch_kind(const ProductPlan& plan, Access access, ProductParams& p, hipStream_t stream) {
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
  if (e != hipSuccess || plan.splits == 1) return e;
  const int strips = (p.N + 2047) / 2048;
  const int64_t rows = KIND == kWeightGrad ? (int64_t)std::max(1, p.groups) * p.M : p.M;
  product_join_kernel<T, KIND><<<dim3((unsigned)(rows * strips)), dim3(256), 0, stream>>>(p, strips);
  return hipGetLastError();
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

// The tile and the slices of the reduction with the smallest estimated time: the workgroups of the CU that has most of them one after the other,
// or in pairs where two fit.
ProductPlan plan_product(ProductKind kind, int dtype, int64_t rows, int64_t in, int64_t out, int groups, Access access, bool odd_rows) {
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
  for (int variant = 0; variant < kTileCount; ++variant) {
    // loads into LDS: bf16 any tile, fp32 the small ones; the kernel for any alignment has the small one's shape, for fp32 in parts (variant 1)
    const bool parts = f32 && variant == 1;
    const int tile = parts ? kSmallTile : variant;
    if (access == kAny ? (f32 ? !parts : tile != kSmallTile) : (f32 && variant == 0) || (forced_tile >= 0 && forced_tile != variant)) continue;
    const TileShape s = kTiles[tile];
    const TileTime t = tile_time(tile, dtype, access, parts);
    const int64_t bm = 64 * s.fm, bn = 64 * s.fn;
    const double row_tiles = kind == kWeightGrad ? (double)((m + bm - 1) / bm * images)
                             : groups            ? (double)m / (double)bm + 0.5 * std::min<double>(groups, (double)m)
                                                 : (double)((m + bm - 1) / bm);
    const double tiles = row_tiles * (double)((n + bn - 1) / bn);
    for (int splits = 1; splits <= 16; ++splits) {
      if (splits > 1 && (k_tiles < 2 * splits || (forced_splits && splits != forced_splits))) continue;
      const int64_t bytes = splits > 1 ? splits * images * m * n * 4 : 0;
      if (bytes > (64 << 20)) continue;
      const double workgroups = std::max(1.0, tiles * splits), most = std::ceil(workgroups / 256), full = std::min(1.0, workgroups / 256);
      const double kt = std::ceil((double)k_tiles / splits);
      double us = 4;
      if (s.resident == 1) us += most * (kt * (t.k_few + (t.k_full - t.k_few) * full) + t.store_few + (t.store_full - t.store_few) * full);
      else us += std::floor(most / 2) * (kt * t.k_full + t.store_full) + std::fmod(most, 2) * (kt * t.k_few + t.store_few);
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
      }
    }
  }
  if (kind == kForward && rows <= (groups ? 8 * (int64_t)groups : 64)) {
    const RowsTime few = rows_time(dtype, rows, in, out, groups, odd_rows);
    if (best_workgroups > 256) best = std::max(best, few.floor);
    plan.few = few.us <= 1.05 * best;
  }
  if (const int forced = tune_int("product_few", -1); forced >= 0 && kind == kForward) plan.few = forced != 0;
  if ((groups ? rows / 16 + std::min<int64_t>(groups, rows) : (rows + 15) / 16) * ((out + 15) / 16) >= 1 << 23) plan.few = false;      // 2^32 lanes
  if (plan.few) plan.splits = 1, plan.ws_bytes = 0;
  return plan;
}

std::string product_name(ProductKind kind, int dtype, const ProductPlan& plan, Access access) {
  if (plan.few) return std::string("product_rows_") + (dtype == STRIPE_F32 ? "f32_" : "bf16_") + "16x16";
  const TileShape s = kTiles[plan.tile];
  return std::string(access != kAny && !plan.parts ? "product_stream_" : "product_") + (kind == kForward ? "nt_" : kind == kInputGrad ? "nn_" : "tn_") + (dtype == STRIPE_F32 ? "f32_" : "bf16_") +
         std::to_string(64 * s.fm) + "x" + std::to_string(64 * s.fn) + (plan.parts ? "_parts" : access != kAny ? "_s" + std::to_string(s.stages) : "") + (access == kWords && !plan.parts ? "_words" : "") +
         (plan.splits > 1 ? "_k" + std::to_string(plan.splits) : "");
}

hipError_t launch_product(ProductKind kind, int dtype, const ProductPlan& plan, Access access, ProductParams p, hipStream_t stream) {
  if (plan.few) return launch_product_rows(dtype, p, stream);
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
