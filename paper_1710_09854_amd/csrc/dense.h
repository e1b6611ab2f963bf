// Tiled matrix products on the matrix cores of gfx950, shared by the orthogonalisation and the gated
// feed-forward kernels: D[i][j] = sum_k A(i, k) B(j, k), 16-bit factors, sums in 32 bits.
//
// Either operand may be stored along K (its row i holds A(i, 0), A(i, 1), ...) or down K (its row k holds
// A(0, k), A(1, k), ...), so that no product needs a transposed copy: what is stored down K is turned by the
// LDS reads that feed the matrix cores (ds_read_b64_tr_b16).
//
// A workgroup's tile of BM x BN results takes its operands through LDS, a slice of 64 of K at a time: slices are
// fetched straight into LDS (no registers), two to four deep, so that the next ones travel while this one is
// multiplied. Rows and columns past an operand's end and chunks past its K read as zero through the buffer's bounds
// check.
// Both sides' 16-byte chunks are kept in an order that puts what 16 lanes read at once into different banks.
// A block of 16 columns of results takes, of 16 G neighbouring columns, a four of each 4 G: a lane then ends with
// 4 G neighbouring results of a row and stores them at once (G blocks of four; G = 4, or 2 for narrow tiles).
//
// What bounds it: the matrix cores and the power they may draw. The three products of 8192 x 4096 x 12288 in bfloat16 by
// tiles of 256 x 256, traced: 1,218 TFLOP/s with both sides along K (and the feed-forward's epilogue), 1,313 with one
// down it, 1,109 with both, where the installed library's product of 8192^3 reaches 1,420. Small
// products take small tiles, for there they have too few to fill 256 compute units, and are bound by the latency of
// a slice.
#ifndef GSPAR_DENSE_H
#define GSPAR_DENSE_H

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>
#include <type_traits>

#include "gspar.h"

namespace gspar {
namespace dense {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef __bf16 bfl8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint16_t u16x4 __attribute__((ext_vector_type(4)));
// The same at any address that the element's type allows, which is all that an access to global memory needs.
typedef f32x4 f32x4_any __attribute__((aligned(4)));
typedef u32x4 u32x4_any __attribute__((aligned(2)));
typedef u16x4 u16x4_any __attribute__((aligned(2)));

struct F16 {};
struct BF16 {};

template <class T>
__device__ __forceinline__ f32x4 mfma(u32x4 a, u32x4 b, f32x4 c) {
  if constexpr (std::is_same_v<T, F16>)
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, a), __builtin_bit_cast(half8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bfl8, a), __builtin_bit_cast(bfl8, b), c, 0, 0, 0);
}

__device__ __forceinline__ float bf16_to_float(uint16_t v) { return __builtin_bit_cast(float, (uint32_t)v << 16); }
__device__ __forceinline__ uint16_t float_to_bf16(float v) { return __builtin_bit_cast(uint16_t, (__bf16)v); }
__device__ __forceinline__ float f16_to_float(uint16_t v) { return (float)__builtin_bit_cast(_Float16, v); }
__device__ __forceinline__ uint16_t float_to_f16(float v) { return __builtin_bit_cast(uint16_t, (_Float16)v); }

template <class T>
__device__ __forceinline__ uint16_t to16(float v) {
  return std::is_same_v<T, F16> ? float_to_f16(v) : float_to_bf16(v);
}
template <class T>
__device__ __forceinline__ float from16(uint16_t v) {
  return std::is_same_v<T, F16> ? f16_to_float(v) : bf16_to_float(v);
}

// An element of a tensor of one of the three types, and back (rounded to nearest even).
__device__ __forceinline__ float load_as(const void* p, int64_t i, int type) {
  if (type == GSPAR_F32) return ((const float*)p)[i];
  const uint16_t v = ((const uint16_t*)p)[i];
  return type == GSPAR_BF16 ? bf16_to_float(v) : f16_to_float(v);
}
__device__ __forceinline__ void store_as(void* p, int64_t i, int type, float v) {
  if (type == GSPAR_F32) ((float*)p)[i] = v;
  else ((uint16_t*)p)[i] = type == GSPAR_BF16 ? float_to_bf16(v) : float_to_f16(v);
}
// Four elements of a row from element i on, of which `n` are there.
__device__ __forceinline__ f32x4 load4(const void* p, int64_t i, int type, int64_t n) {
  f32x4 v;
  if (n >= 4) {
    if (type == GSPAR_F32) return *(const f32x4_any*)((const float*)p + i);
    const u16x4 h = *(const u16x4_any*)((const uint16_t*)p + i);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = type == GSPAR_BF16 ? bf16_to_float(h[e]) : f16_to_float(h[e]);
    return v;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = e < n ? load_as(p, i + e, type) : 0.f;
  return v;
}
__device__ __forceinline__ void store4(void* p, int64_t i, int type, int64_t n, f32x4 v) {
  if (n >= 4) {
    if (type == GSPAR_F32) {
      *(f32x4_any*)((float*)p + i) = v;
    } else {
      u16x4 h;
#pragma unroll
      for (int e = 0; e < 4; ++e) h[e] = type == GSPAR_BF16 ? float_to_bf16(v[e]) : float_to_f16(v[e]);
      *(u16x4_any*)((uint16_t*)p + i) = h;
    }
    return;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (e < n) store_as(p, i + e, type, v[e]);
}

// 4 G elements of a row, of which `n`, 4 G or more or a multiple of eight, are there (G is even).
template <int G>
__device__ __forceinline__ void load_row(const void* p, int64_t i, int type, int64_t n, f32x4 (&v)[G]) {
#pragma unroll
  for (int g = 0; g < G; g += 2) {
    if (4 * g >= n) break;
    if (type == GSPAR_F32) {
      v[g] = *(const f32x4_any*)((const float*)p + i + 4 * g);
      v[g + 1] = *(const f32x4_any*)((const float*)p + i + 4 * g + 4);
    } else {
      const u32x4 h = *(const u32x4_any*)((const uint16_t*)p + i + 4 * g);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint16_t x = (uint16_t)(h[e / 2] >> 16 * (e & 1));
        v[g + e / 4][e % 4] = type == GSPAR_BF16 ? bf16_to_float(x) : f16_to_float(x);
      }
    }
  }
}
template <int G>
__device__ __forceinline__ void store_row(void* p, int64_t i, int type, int64_t n, const f32x4 (&v)[G]) {
#pragma unroll
  for (int g = 0; g < G; g += 2) {
    if (4 * g >= n) break;
    if (type == GSPAR_F32) {
      *(f32x4_any*)((float*)p + i + 4 * g) = v[g];
      *(f32x4_any*)((float*)p + i + 4 * g + 4) = v[g + 1];
    } else {
      u32x4 h;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float a = v[g + e / 2][2 * (e & 1)], b = v[g + e / 2][2 * (e & 1) + 1];
        h[e] = type == GSPAR_BF16 ? float_to_bf16(a) | (uint32_t)float_to_bf16(b) << 16
                                  : float_to_f16(a) | (uint32_t)float_to_f16(b) << 16;
      }
      *(u32x4_any*)((uint16_t*)p + i + 4 * g) = h;
    }
  }
}
inline int64_t type_size(int type) { return type == GSPAR_F32 ? 4 : 2; }
inline bool type_ok(int type) { return type == GSPAR_F32 || type == GSPAR_BF16 || type == GSPAR_F16; }

constexpr int kSlice = 128;  // bytes of K in a slice, for an operand stored along K

// An operand's rows: base of row 0, bytes from one to the next, their number, and the bytes of one. Bases, pitches and
// the bytes of a row are multiples of 16 (a load that the end cuts reads as zero whole), and a tile's rows (256, or a
// slice's 64) span less than 2^31 bytes.
struct Rows {
  const char* base;
  int64_t ld;
  int64_t rows;
  int64_t bytes;
};

// The rows from row0 on, from byte `from` of each, behind a bounds check at the last row's end.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t window(const Rows& r, int64_t row0, int64_t from) {
  const int64_t left = r.rows - row0;
  int64_t bytes = left > 0 ? (left - 1) * r.ld + r.bytes - from : 0;
  if (bytes > 0x7FFFFFFF) bytes = 0x7FFFFFFF;
  const char* p = r.base + (left > 0 ? row0 * r.ld + from : 0);
  return __builtin_amdgcn_make_buffer_rsrc((void*)p, 0, (int)bytes, 0x00027000);
}

// The LDS of a stage. Every stage is an object of its own, so that the compiler knows that reads of one do not
// wait for fetches into another.
template <class C, int kStage>
__device__ __forceinline__ char* stage() {
  __shared__ __align__(1024) char lds[C::kGroups * C::kStage];
  return lds;
}

// A number that is the same in every lane, for the compiler to keep in scalar registers.
__device__ __forceinline__ int64_t uniform(int64_t v) {
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v), hi = __builtin_amdgcn_readfirstlane((uint32_t)((uint64_t)v >> 32));
  return (int64_t)((uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ const char* uniform(const char* p) { return (const char*)uniform((int64_t)p); }

__device__ __forceinline__ void fetch16(__amdgpu_buffer_rsrc_t buf, uint32_t off, char* lds) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(buf, (__attribute__((address_space(3))) void*)lds, 16, off, 0, 0, 0);
}

// BM x BN results by WM x WN waves; a wave has FM x FN blocks of 16 x 16. kPairs: an element is two 16-bit
// numbers, upper and lower, kept as 32 uppers and their 32 lowers in turn; a slice is 32 of K then.
// kStages slices are held at once: one is multiplied while the others travel. kGroups: so many groups of WM x WN
// waves take the slices in turn, each with its own stages, and add their sums at the end: where tiles are too few to
// give a compute unit two workgroups, the groups hide each other's waits.
template <int BM_, int BN_, int WM_, int WN_, int kStages_, bool kPairs_ = false, int kGroups_ = 1>
struct Tile {
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_;
  static constexpr bool kPairs = kPairs_;
  static constexpr int kGroups = kGroups_;
  static constexpr int kWaves = WM * WN, kThreads = 64 * kWaves * kGroups;  // kWaves: of a group
  static constexpr int FM = BM / WM / 16, FN = BN / WN / 16;
  static constexpr int kStage = (BM + BN) * kSlice;
  static constexpr int kStages = kStages_;
  static_assert(kGroups == 1 || (kGroups == 2 && BM * BN * 4 <= kGroups * kStage), "sums that one group leaves for the other");
  static constexpr int kLoads = (BM + BN) / 8 / kWaves;  // of a slice, per wave
  static constexpr int kStep = kPairs ? 32 : 64;  // of K
  static constexpr int G = FN % 4 == 0 ? 4 : FN % 2 == 0 ? 2 : 1;  // blocks whose columns are dealt in fours
  static_assert(BM % (8 * kWaves) == 0 && BN % (8 * kWaves) == 0 && kWaves % 2 == 0, "whole loads, rows of one parity");
};

// The four that block f takes from part q (of 4 G columns) of its 16 G: the f-th, odd parts' neighbours swapped
// (the places in LDS of the two parities then differ by more than multiples of a chunk).
template <int G>
__device__ __forceinline__ int four_of(int f, int q) { return (f % G) ^ (G > 1 ? q & 1 : 0); }

// One side of a tile: N rows of results, of which this wave multiplies F blocks of 16 from row `mine` on. Every wave
// fetches N / 8 / kWaves loads of 1 KiB of a slice.
//
// Along K. Two: rows of two operands in turn, 8 of each.
template <int N, int kWaves, int F, int G, bool kTwo = false>
struct Along {
  static constexpr int kLoads = N / 8 / kWaves;
  static_assert(!kTwo || kWaves % 2 == 0, "a wave's loads are all of one operand");
  __amdgpu_buffer_rsrc_t buf;
  uint32_t off[kLoads];
  static constexpr int kPlaces = G > 1 ? 2 : 1;  // of an even and an odd block; the others are whole rows further
  uint32_t bytes, place[kPlaces];
  int wave;

  // Chunk c of row r is kept at c ^ turn(r). Lanes 0..15 read chunk c of rows 4 G q + i (+ a constant), q and i
  // in 0..3: with the row's parity (two rows fill all banks), they fill 16 places.
  static __device__ __forceinline__ int turn(int r) { return ((r >> 1) & 1) | (((r / (4 * G)) & 3) << 1); }
  __device__ __forceinline__ uint32_t chunk(int load, int lane) const {
    return ((lane & 7) ^ turn(load * 8 + (lane >> 3))) * 16;
  }
  __device__ __forceinline__ Along(const Rows& r0, const Rows& r1, int64_t row0, int mine)
      : bytes((uint32_t)r0.bytes) {
    const int lane = threadIdx.x & 63;
    wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) % kWaves;
    // every load is 8 rows, of one operand; with an even number of waves a wave's are all of the same
    const bool second = kTwo && (wave & 1);
    const Rows mine_of = {uniform(second ? r1.base : r0.base), uniform(second ? r1.ld : r0.ld), r0.rows, r0.bytes};
    buf = window(mine_of, row0, 0);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int load = wave + i * kWaves, row = load * 8 + (lane >> 3);
      off[i] = chunk(load, lane) + (uint32_t)((kTwo ? (row >> 4) * 8 + (row & 7) : row) * mine_of.ld);
    }
    const int q = (lane & 15) >> 2;
#pragma unroll
    for (int f = 0; f < kPlaces; ++f) {
      const int r = mine + q * 4 * G + four_of<G>(f, q) * 4 + (lane & 3);
      place[f] = (uint32_t)(r * kSlice + ((lane >> 4) ^ turn(r)) * 16);
    }
  }
  __device__ __forceinline__ void fetch(int s, char* lds) {
    const bool tail = (uint32_t)(s + 1) * kSlice > bytes;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int q = wave + i * kWaves;
      uint32_t at = off[i] + (uint32_t)s * kSlice;
      if (tail && (uint32_t)s * kSlice + chunk(q, threadIdx.x & 63) >= bytes) at = 0x80000000u;
      fetch16(buf, at, lds + q * 1024);
    }
  }
  // block f's factors of half h of the slice
  __device__ __forceinline__ u32x4 read(const char* lds, int h, int f) const {
    return *(const u32x4*)(lds + (place[f % kPlaces] ^ (h * 64)) + ((f / G) * 16 * G + (f % G - f % kPlaces) * 4) * kSlice);
  }
};

// Down K. Two: the first `cut` slices come from one operand's rows and the others from the second's.
template <int N, int kWaves, int F, int G, bool kPairs, bool kTwo = false>
struct Down {
  static constexpr int kLoads = N / 8 / kWaves;
  static constexpr int kRow = N * (kPairs ? 4 : 2);       // bytes of a slice's row
  static constexpr int kRowsK = kPairs ? 32 : 64;
  // Chunk c of row k is kept at c ^ turn(k). 32 lanes read at once, 8 bytes each: rows k .. k + 3 and k + 8 ..
  // k + 11, and of each row a four of columns at four places 4 G apart: one unit of 32 bytes (G = 1), a half of each
  // half of two units, the parities' halves in turn (G = 2), or half of one half of four units, likewise (G = 4).
  // The turns by k & 1, k & 2 and k & 8 move rows to units or halves that the others do not use; odd multiples of
  // 128 bytes alternate between the halves of all banks by themselves.
  static constexpr bool kAlternate = kRow % 256 == 128;
  static constexpr int k1 = G == 1 ? (kAlternate ? 0 : 2) : G == 2 ? (kAlternate ? 0 : 4) : kPairs ? 4 : 8;
  static constexpr int k2 = G == 1 ? (kAlternate ? 2 : 4) : G == 2 ? (kAlternate ? 4 : 8) : 1;
  static constexpr int k8 = G == 1 ? (kAlternate ? 4 : 8) : G == 2 ? 1 : 2;
  static constexpr int kMost = k1 > k2 ? (k1 > k8 ? k1 : k8) : (k2 > k8 ? k2 : k8);
  static_assert((kRow / 16) % (2 * kMost) == 0, "turns stay in the row");
  // the operand that is being read, from its slice 0 on, and the one that follows
  const char *base, *base2;
  int64_t ld, rows, bytes, from, ld2, rows2;
  int cut, first, wave;
  uint32_t off[kLoads], place[F];

  static __device__ __forceinline__ int turn(int k) { return ((k & 1) ? k1 : 0) ^ ((k & 2) ? k2 : 0) ^ ((k & 8) ? k8 : 0); }
  __device__ __forceinline__ Down(const Rows& a, const Rows& b, int cut_, int64_t col0, int mine)
      : base(a.base), base2(b.base), ld(a.ld), rows(a.rows), bytes(a.bytes), ld2(b.ld), rows2(b.rows), cut(cut_), first(0) {
    const int lane = threadIdx.x & 63;
    wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) % kWaves;
    from = col0 * (kPairs ? 4 : 2);
    offsets();
    const int k = (lane >> 4) * 8 + ((lane & 15) >> 2);
#pragma unroll
    for (int f = 0; f < F; ++f) {
      const int c = mine + (f / G) * 16 * G + (lane & 3) * 4 * G + four_of<G>(f, lane & 3) * 4;
      const int byte = kPairs ? (c >> 5) * 128 + (c & 31) * 2 : c * 2;
      place[f] = (uint32_t)(k * kRow + (byte ^ (turn(k) * 16)));
    }
  }
  __device__ __forceinline__ void offsets() {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int at = (wave + i * kWaves) * 1024 + lane * 16, k = at / kRow;
      off[i] = (uint32_t)(k * ld) + ((at % kRow) ^ (turn(k) * 16));
    }
  }
  __device__ __forceinline__ void fetch(int s, char* lds) {
    if (kTwo && s >= cut && first == 0) {
      base = base2;
      ld = ld2;
      rows = rows2;
      first = cut;
      offsets();
    }
    const __amdgpu_buffer_rsrc_t buf = window({base, ld, rows, bytes}, (int64_t)(s - first) * kRowsK, from);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) fetch16(buf, off[i], lds + (wave + i * kWaves) * 1024);
  }
  // Of rows k .. k + 3, k = 8 (l / 16), lanes 0..15 (16..31, ...) read four columns of a row each, and lane i of
  // them receives the (i % 4)th column that lane i / 4 of a row read, all four of K; a second read brings rows
  // k + 4 .. k + 7.
  __device__ __forceinline__ u32x4 read(const char* lds, int h, int f) const {
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) s16x4 lds4;
    const char* p = lds + (kPairs ? place[f] ^ (h * 64) : place[f] + h * 32 * kRow);
    const u32x2 a = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)p));
    const u32x2 b = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(p + 4 * kRow)));
    return u32x4{a.x, a.y, b.x, b.y};
  }
};

// Place of the workgroup's tile: blocks are dealt to the 8 XCDs in turn, so each XCD is given a run of
// neighbouring tiles, whose operands its L2 then holds for several of them.
__device__ __forceinline__ int xcd_order(int b, int n) {
  const int per = n >> 3, more = n & 7, x = b & 7, i = b >> 3;
  return x < more ? x * (per + 1) + i : more * (per + 1) + (x - more) * per + i;
}

// Tile t of tm x tn in bands of eight rows of tiles, down a band's columns.
__device__ __forceinline__ void banded(int t, int tm, int tn, int& i, int& j) {
  constexpr int kBand = 8;
  const int band = t / (kBand * tn), in = t - band * kBand * tn;
  const int h = min(kBand, tm - band * kBand);
  j = in / h;
  i = band * kBand + in - j * h;
}

// Tile t of the lower triangle (j <= i).
__device__ __forceinline__ void triangle(int t, int& i, int& j) {
  i = (int)((sqrtf(8.0f * t + 1.0f) - 1.0f) * 0.5f);
  while (i * (i + 1) / 2 > t) --i;
  while ((i + 1) * (i + 2) / 2 <= t) ++i;
  j = t - i * (i + 1) / 2;
}

// This wave's first row (of 16-row blocks) on either side of the tile.
template <class C>
__device__ __forceinline__ int mine_m() { return (__builtin_amdgcn_readfirstlane(threadIdx.x >> 6) % C::kWaves / C::WN) * C::FM * 16; }
template <class C>
__device__ __forceinline__ int mine_n() { return (__builtin_amdgcn_readfirstlane(threadIdx.x >> 6) % C::WN) * C::FN * 16; }

template <class C, bool kTwo = false>
using AlongM = Along<C::BM, C::kWaves, C::FM, 1, kTwo>;
template <class C, bool kTwo = false>
using AlongN = Along<C::BN, C::kWaves, C::FN, C::G, kTwo>;
template <class C, bool kTwo = false>
using DownM = Down<C::BM, C::kWaves, C::FM, 1, C::kPairs, kTwo>;
template <class C, bool kTwo = false>
using DownN = Down<C::BN, C::kWaves, C::FN, C::G, C::kPairs, kTwo>;

template <class T, class C>
__device__ __forceinline__ void products(const u32x4 (&a)[C::FM], const u32x4 (&b)[C::FN], f32x4 (&acc)[C::FN][C::FM]) {
#pragma unroll
  for (int i = 0; i < C::FM; ++i)
#pragma unroll
    for (int j = 0; j < C::FN; ++j) acc[j][i] = mfma<T>(b[j], a[i], acc[j][i]);
}
template <class Side, int F>
__device__ __forceinline__ void read(const Side& side, const char* lds, int h, u32x4 (&to)[F]) {
#pragma unroll
  for (int f = 0; f < F; ++f) to[f] = side.read(lds, h, f);
}

// acc[fn][fm] (lane l: columns 4 (l / 16) .. + 3 of block fn as dealt, row l % 16 of block fm) += the tile's sums
// over `steps` slices of K. kPairs: upper * upper + upper * lower + lower * upper.
//
// The reads of LDS run half a slice ahead of the products: while the first half is multiplied the second is
// read, and while that is multiplied the first half of the next slice. One barrier a slice, between the
// halves: it tells that every wave's part of the next slice has arrived, and that every wave has read the whole
// of this one, whose stage the slice after the others is then fetched into. (With both halves read where they
// are used, waves read in step and multiply in step: 4096^3 takes 113 us instead of 101.) In tiles of 64 x 64 a
// half's products are too short to hide a read, and both halves are read at once (1024 x 512 x 4608: 17 us
// against 22).
template <class T, class C, class SideM, class SideN>
struct Pipeline {
  SideM& A;
  SideN& B;
  const int group, start, steps;
  u32x4 a0[C::FM], a1[C::FM], b0[C::FN], b1[C::FN];
  f32x4 (&acc)[C::FN][C::FM];
  static constexpr bool kRunAhead = C::BM > 64;

  // Waits until at most kLoadsLeft loads are under way and no read of LDS, and for the other waves. The empty
  // statements keep the compiler's loads on their sides (the builtins alone say nothing of memory).
  template <int kLoadsLeft>
  static __device__ __forceinline__ void meet() {
    static_assert(kLoadsLeft < 64, "the counter's width");
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt((kLoadsLeft & 15) | ((kLoadsLeft >> 4) << 14) | 0x70);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  }
  template <int I>
  __device__ __forceinline__ char* at() const { return stage<C, I % C::kStages>() + group * C::kStage; }
  // slices past the last one read as zero: the count of loads stays the same
  template <int I>
  __device__ __forceinline__ void fetch(int s) {
    A.fetch(start + s * C::kGroups + group, at<I>());
    B.fetch(start + s * C::kGroups + group, at<I>() + C::BM * kSlice);
  }
  template <int I>
  __device__ __forceinline__ void fill() {
    if constexpr (I < C::kStages - (kRunAhead ? 0 : 1)) {
      fetch<I>(I);
      fill<I + 1>();
    }
  }
  // slices s, s + 1, .. from stage I on; true after the last one
  template <int I>
  __device__ __forceinline__ bool step(int& s) {
    if constexpr (I == C::kStages) {
      return false;
    } else {
      const char *la = at<I>(), *lb = la + C::BM * kSlice;
      const char *na = at<I + 1>(), *nb = na + C::BM * kSlice;
      if constexpr (!kRunAhead) {
        meet<(C::kStages - 2) * C::kLoads>();
        read(B, lb, 0, b0);
        read(A, la, 0, a0);
        fetch<I + C::kStages - 1>(s + C::kStages - 1);  // over the slice before this one
        read(B, lb, 1, b1);
        read(A, la, 1, a1);
        products<T, C>(a0, b0, acc);
        if constexpr (C::kPairs) {
          products<T, C>(a0, b1, acc);
          products<T, C>(a1, b0, acc);
        } else {
          products<T, C>(a1, b1, acc);
        }
      } else {
        read(B, lb, 1, b1);
        read(A, la, 1, a1);
        products<T, C>(a0, b0, acc);
        meet<(C::kStages - 2) * C::kLoads>();
        if constexpr (!C::kPairs) {
          read(B, nb, 0, b0);
          read(A, na, 0, a0);
          fetch<I>(s + C::kStages);
          products<T, C>(a1, b1, acc);
        } else {
          fetch<I>(s + C::kStages);
          products<T, C>(a0, b1, acc);
          read(A, na, 0, a0);
#pragma unroll
          for (int j = 0; j < C::FN; ++j) {
#pragma unroll
            for (int i = 0; i < C::FM; ++i) acc[j][i] = mfma<T>(b0[j], a1[i], acc[j][i]);
            b0[j] = B.read(nb, 0, j);
          }
        }
      }
      if (++s * C::kGroups >= steps) return true;
      return step<I + 1>(s);
    }
  }
  __device__ __forceinline__ void run() {
    fill<0>();
    if constexpr (kRunAhead) {
      meet<(C::kStages - 1) * C::kLoads>();
      read(B, at<0>() + C::BM * kSlice, 0, b0);
      read(A, at<0>(), 0, a0);
    }
    int s = 0;
    while (!step<0>(s)) {
    }
    __builtin_amdgcn_s_waitcnt(0x0F70);  // no fetch is under way when the workgroup gives its LDS back
  }
};

// The product's slices start .. start + steps - 1 (an even number where two groups share them, but for K's end).
template <class T, class C, class SideM, class SideN>
__device__ __forceinline__ void multiply(SideM& A, SideN& B, int steps, f32x4 (&acc)[C::FN][C::FM], int start = 0) {
  const int group = C::kGroups > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) / C::kWaves : 0;
  Pipeline<T, C, SideM, SideN> p{A, B, group, start, steps, {}, {}, {}, {}, acc};
  p.run();
}

// K in parts: workgroups of the same tile take some of its slices each and leave their sums, as their threads hold
// them, for a second launch that adds them in order.
template <class C>
constexpr int64_t kPartFours = (int64_t)C::FN * C::FM * C::kThreads;
template <class C>
__device__ __forceinline__ void leave_part(const f32x4 (&acc)[C::FN][C::FM], f32x4* part) {
#pragma unroll
  for (int j = 0; j < C::FN; ++j)
#pragma unroll
    for (int i = 0; i < C::FM; ++i) part[(j * C::FM + i) * C::kThreads + threadIdx.x] = acc[j][i];
}
// The second launch has C::FM workgroups a tile, each with one block of rows of every wave (15 tiles of 192 x 192 of
// three matrices: 20.4 -> 13.5 us), and reads four parts at once (28 tiles of 128 x 128 in 15 parts: 20.2 -> 10.2 us).
template <class C>
__device__ __forceinline__ void join_parts(f32x4 (&acc)[C::FN][C::FM], const f32x4* part, int parts, int block) {
  f32x4 sum[C::FN] = {};
  const f32x4* from = part + block * C::kThreads + threadIdx.x;
  for (int p = 0; p < parts; p += 4) {
    f32x4 v[4][C::FN];  // four parts under way at once
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (p + q < parts) {
#pragma unroll
        for (int j = 0; j < C::FN; ++j) v[q][j] = from[(p + q) * kPartFours<C> + j * C::FM * C::kThreads];
      }
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (p + q < parts) {
#pragma unroll
        for (int j = 0; j < C::FN; ++j) sum[j] += v[q][j];
      }
  }
#pragma unroll
  for (int i = 0; i < C::FM; ++i)
#pragma unroll
    for (int j = 0; j < C::FN; ++j)
      if (i == block) acc[j][i] = sum[j];
}

template <class C>
__device__ __forceinline__ void clear(f32x4 (&acc)[C::FN][C::FM]) {
#pragma unroll
  for (int j = 0; j < C::FN; ++j)
#pragma unroll
    for (int i = 0; i < C::FM; ++i) acc[j][i] = f32x4{0.f, 0.f, 0.f, 0.f};
}

// f(row, column, the 4 G sums along the row from there) for each of the lane's results. Two groups of waves first
// add their sums, the second's to the first's; each takes half of the results. block: this block of rows alone.
template <class C, class F>
__device__ __forceinline__ void each(const f32x4 (&acc)[C::FN][C::FM], F&& f, int block = -1) {
  const int lane = threadIdx.x & 63, wave = (threadIdx.x >> 6) % C::kWaves, group = (threadIdx.x >> 6) / C::kWaves;
  const int r0 = (wave / C::WN) * C::FM * 16 + (lane & 15), c0 = (wave % C::WN) * C::FN * 16 + (lane >> 4) * 4 * C::G;
  auto owner = [](int i, int j) { return C::kGroups > 1 ? (i * (C::FN / C::G) + j / C::G) % C::kGroups : 0; };
  f32x4* sums = nullptr;
  if constexpr (C::kGroups > 1) {
    sums = (f32x4*)stage<C, 0>() + wave * 64 + lane;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < C::FN; ++j)
#pragma unroll
      for (int i = 0; i < C::FM; ++i)
        if (owner(i, j) != group && (block < 0 || i == block)) sums[(j * C::FM + i) * C::kWaves * 64] = acc[j][i];
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < C::FM; ++i)
#pragma unroll
    for (int j = 0; j < C::FN; j += C::G) {
      if ((C::kGroups > 1 && owner(i, j) != group) || (block >= 0 && i != block)) continue;
      f32x4 v[C::G];
#pragma unroll
      for (int g = 0; g < C::G; ++g) {
        v[g] = acc[j + g][i];
        if constexpr (C::kGroups > 1) {
          const f32x4 other = sums[((j + g) * C::FM + i) * C::kWaves * 64];
          v[g] = group == 0 ? v[g] + other : other + v[g];
        }
      }
      if constexpr (C::G > 1) {
        if (lane & 16) {
#pragma unroll
          for (int g = 0; g < C::G; g += 2) {
            const f32x4 t = v[g];
            v[g] = v[g + 1];
            v[g + 1] = t;
          }
        }
      }
      f(r0 + i * 16, c0 + j * 16, v);
    }
}

// 4 G numbers of 16 bits to consecutive places.
template <int G>
__device__ __forceinline__ void put16(uint16_t* to, const u16x4 (&v)[G]) {
  if constexpr (G == 1) {
    *(u16x4_any*)to = v[0];
  } else {
#pragma unroll
    for (int g = 0; g < G; g += 2) {
      const u32x2 a = __builtin_bit_cast(u32x2, v[g]), b = __builtin_bit_cast(u32x2, v[g + 1]);
      *(u32x4_any*)(to + 4 * g) = u32x4{a.x, a.y, b.x, b.y};
    }
  }
}
template <int G>
__device__ __forceinline__ void get16(const uint16_t* from, u16x4 (&v)[G]) {
  if constexpr (G == 1) {
    v[0] = *(const u16x4*)from;
  } else {
#pragma unroll
    for (int g = 0; g < G; g += 2) {
      const u32x4 a = *(const u32x4*)(from + 4 * g);
      v[g] = __builtin_bit_cast(u16x4, u32x2{a.x, a.y});
      v[g + 1] = __builtin_bit_cast(u16x4, u32x2{a.z, a.w});
    }
  }
}

// How a product is taken: which tile, and in how many parts of K.
struct Way {
  int tile, parts, per;  // per: slices of a part
  int64_t fours;         // of 16 bytes, that the parts leave
};

// The way that takes least time: rounds of workgroups times the slices of each and the time of a slice, and the time
// that a round's first fetches and its results take, `tiles(side)` being the number of tiles of that side, plus the
// second launch and the parts' bytes. us a slice, 16-bit numbers (a slice is 64 of K) and pairs of them (32 of K): the
// figures that choose best among the products of whole calls, and in brackets what one round of full tiles takes, 16
// slices and 64 (along K and with one side down it). Small tiles take as long for either, for they are bound by a slice's
// bytes on their way into LDS, which are the same:
//   256 x 256                                       1.5 and 1.97  [1.5 to 1.85 and 1.95]
//   192 x 192                                       0.95 and 1.2  [0.92 and 1.14]
//   128 x 128, two on a compute unit                1.0 and 1.16  [0.88 to 0.91 and 1.10]
//   128 x 128 by two groups of waves, one on a unit 0.6 for both  [0.50 to 0.53 and 0.55 to 0.57]
//   64 x 64 by two groups                           0.26 for both [0.21 and 0.20 to 0.22]
//   64 x 64 by one, two on a compute unit           0.5 for both  [0.36 to 0.43 and 0.37 to 0.45]
// 1024 x 512 x 4608 takes 43 us by 128 x 128 and 17 to 21 by 64 x 64, which has 128 tiles where the other has 32; 512
// tiles of 64 x 64 of 1000 in pairs at once 21.7 us and in two rounds of 256 by two groups 23.8; 136 tiles of 2048 in pairs
// 23.3 and 17.6; not for parts of K: 128 tiles of 5632 in four take 17.2 us and by two groups 15.8. Parts, 5 us and their bytes at 8 TB/s (they stay in the caches): the
// 512 x 512 of a 512 x 4608 matrix in pairs takes 32 us whole and 16.5 in parts. The rounds' ends count where K is
// short: six products 1024 x 4096 x 1024 take 94 us by 256 x 256 (two rounds of 16 slices) and 88 by 128 x 128.
template <class Tiles>
Way way_of(bool pairs, bool k192, int64_t slices, bool may_split, Tiles&& tiles) {
  const int side[6] = {256, 192, 128, 128, 64, 64}, at_once[6] = {256, 256, 512, 256, 256, 512}, groups[6] = {1, 1, 1, 2, 2, 1};
  const double slice[2][6] = {{1.5, 0.95, 1.0, 0.6, 0.26, 0.5}, {1.97, 1.2, 1.16, 0.6, 0.26, 0.5}};
  const double ends[6] = {4.0, 3.0, 1.0, 1.0, 0.5, 0.5};
  Way best{};
  double least = 0.0;
  for (int i = 0; i < 6; ++i) {
    if (i == 1 && !k192) continue;
    const int64_t n = tiles(side[i]), fours = (int64_t)side[i] * side[i] / 4 * groups[i];
    for (int p = 1; p <= (may_split && i < 5 ? 16 : 1); ++p) {
      int64_t per = (slices + p - 1) / p;
      per += per & 1;
      const int64_t parts = p == 1 ? 1 : (slices + per - 1) / per;
      if (p > 1 && (parts < 2 || per < 4 || n * parts * fours > (1 << 22))) continue;
      const double rounds = (double)((n * parts + at_once[i] - 1) / at_once[i]);
      double t = rounds * ((double)(p == 1 ? slices : per) * slice[pairs][i] + ends[i]);
      if (parts > 1) t += 5.0 + (double)(n * parts * fours) * 32 / 8e6;
      if (best.parts == 0 || t < least) {
        least = t;
        best = {i, (int)parts, (int)(p == 1 ? slices : per), parts > 1 ? n * parts * fours : 0};
      }
    }
  }
  return best;
}

// f of a way's tile.
template <bool kPairs, bool k192 = true, class F>
void with_tile(const Way& way, F&& f) {
  switch (way.tile) {
    case 0: return f(Tile<256, 256, kPairs ? 2 : 4, kPairs ? 4 : 2, 2, kPairs>{});
    case 1:
      if constexpr (k192) return f(Tile<192, 192, 4, 2, 3, kPairs>{});
      [[fallthrough]];
    case 2: return f(Tile<128, 128, 2, 2, 2, kPairs>{});
    case 3: return f(Tile<128, 128, 2, 2, 2, kPairs, 2>{});
    case 4: return f(Tile<64, 64, 2, 2, 4, kPairs, 2>{});
    default: return f(Tile<64, 64, 2, 2, 4, kPairs>{});
  }
}

inline int64_t up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }
inline int64_t ceil_div(int64_t v, int64_t by) { return (v + by - 1) / by; }

// Whether every kernel launched since the last check was accepted.
inline int launched() { return hipGetLastError() == hipSuccess ? GSPAR_OK : GSPAR_ERR_HIP; }

}  // namespace dense
}  // namespace gspar

#endif
