// Orthogonalised updates: Newton-Schulz steps on matrix cores, and the momentum / weight step around them.
//
// X_0 = U / (|U|_F + eps) for a matrix U of R x C, taken by its shorter side (R <= C), then
//   A = X X^T,   B = b A + c A^2,   X <- a X + B X
// drives the singular values of X towards one and leaves its singular vectors. A and B are symmetric:
// only the lower triangle of their tiles is computed, and each tile is written twice.
//
// Precision. Rounding X to 16 bits between steps would lose the directions of small singular values
// (a matrix of falling strengths comes out 1 to 10 per cent off), because a X lifts them together with
// their rounding. So X is kept as a sum of two fp16 numbers (22 bits), scaled by 2^12 so that both parts
// of every entry that matters are normal numbers. With bfloat16 results the products take the upper parts
// alone: their rounding turns a large direction a little, which the next step keeps orthogonal, but does
// not enter the small ones. The diagonals of A and B are carried in 32 bits beside the products, for near
// the end a + b + c is 0.7 while its terms are 3.4, 4.8 and 2.0. That leaves errors of 3e-4 to 9e-4 (2-norm)
// where rounding to bfloat16 makes 1.7e-3; rounding to float16 makes 2.1e-4, so float16 results take the other
// way. With float32 and float16 results each product is upper * upper + upper * lower + lower * upper in 32-bit
// sums, as exact as 32-bit arithmetic. The parts are fp16 and not bf16: after the normalisation nothing exceeds the
// bound that the host derives from the coefficients, so the range is known and the three more bits are free.
#include "dense.h"

#include <algorithm>

namespace gspar {
namespace dense {
namespace {

constexpr float kUnit = 4096.f;              // a stored number is 2^12 times its value
constexpr float kPerSum = 1.f / (4096.f * 4096.f);
constexpr double kMostStored = 15.0;         // 65504 / 4096, with room for rounding

// Storage of a matrix by rows. kPairs: 32 upper halves and their 32 lower halves in turn. Else the
// upper halves, and the lower ones, where kept, in a buffer of the same layout.
template <bool kPairs>
__device__ __forceinline__ int64_t place(int64_t row, int64_t ld, int64_t k) {
  return kPairs ? row * ld + (k >> 5) * 128 + (k & 31) * 2 : row * ld + k * 2;
}

struct Parts {
  uint16_t hi, lo;
};
__device__ __forceinline__ Parts split(float v) {
  const _Float16 h = (_Float16)v;
  const _Float16 l = (_Float16)(v - (float)h);
  return {__builtin_bit_cast(uint16_t, h), __builtin_bit_cast(uint16_t, l)};
}

// 4 G numbers along a row, from element k on (a multiple of 4 G).
template <bool kPairs, int G>
__device__ __forceinline__ void put(char* hi, char* lo, int64_t row, int64_t ld, int64_t k, const f32x4 (&v)[G]) {
  u16x4 h[G], l[G];
#pragma unroll
  for (int g = 0; g < G; ++g)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const Parts p = split(v[g][e]);
      h[g][e] = p.hi;
      l[g][e] = p.lo;
    }
  const int64_t at = place<kPairs>(row, ld, k);
  put16((uint16_t*)(hi + at), h);
  if (kPairs) put16((uint16_t*)(hi + at + 64), l);
  else if (lo) put16((uint16_t*)(lo + at), l);
}
template <bool kPairs, int G>
__device__ __forceinline__ void get(const char* hi, const char* lo, int64_t row, int64_t ld, int64_t k, f32x4 (&v)[G]) {
  const int64_t at = place<kPairs>(row, ld, k);
  u16x4 h[G], l[G] = {};
  get16((const uint16_t*)(hi + at), h);
  if (kPairs) get16((const uint16_t*)(hi + at + 64), l);
  else if (lo) get16((const uint16_t*)(lo + at), l);
#pragma unroll
  for (int g = 0; g < G; ++g)
#pragma unroll
    for (int e = 0; e < 4; ++e) v[g][e] = f16_to_float(h[g][e]) + f16_to_float(l[g][e]);
}

// The matrices of a call and the step around them. Element (i, j) of matrix t is at t * stride + i * ld + j.
struct Tensor {
  void* p;
  int64_t ld, stride;
  int type;
};

struct Job {
  int64_t batch, m, n;       // as the caller has them
  int64_t R, C, Rp, Cp;      // shorter and longer side, and both rounded up to 64
  bool tall;                 // m > n: R are columns
  int steps;
  float a, b, c;
  double eps;
  Tensor g, mom, w, half, out;  // mom: momentum (null: none); w: weights; half: a 16-bit copy of them; out: result alone
  float beta;
  bool nesterov;
  float decay, rate;         // w <- decay w - rate o; out <- rate o
  uint32_t* flags;
  // workspace, per matrix
  char *x[2], *lo[2], *A, *B;  // X (R rows) and its lower parts, before and after a step; A and B (R rows)
  float *da, *db;              // their diagonals
  double *part, *norm2;        // partial sums of squares, and their sums
  f32x4* parted;               // what parts of K leave
  Way gram, square, apply;     // how the three products of a step are taken
  int parts;
  int64_t xrow, arow;          // bytes from row to row of X (and lo), and of A and B
  // the same for panels (sides up to 128): X by panels, and two buffers of the workgroups' parts of A
  int panels, per_group, groups;  // panels of 128 columns; those of a workgroup; workgroups of a matrix
  float* px;                   // X, 32 bits: prows (64 or 128) rows of panels * 128
  int64_t prows;
  f32x4* pa[2];
  bool direct;                 // the panels read and write the caller's rows themselves
};

// ------------------------------------------------------------------------------------------
// U, its norm, and X_0.
// ------------------------------------------------------------------------------------------
constexpr int kNormThreads = 256;

// From this magnitude on a number is an infinity in a tensor of the type: half a place past its largest number.
__device__ __forceinline__ float past_range(int type) {
  return type == GSPAR_F16 ? 65520.f : type == GSPAR_BF16 ? 0x1.FFp127f : INFINITY;
}

// Four entries of U from (i, j) on, of which n are there; the new momentum in mnew. A momentum that its type cannot hold
// makes U infinite, and so its matrix's step one that is skipped.
__device__ __forceinline__ f32x4 update_at(const Job& J, int64_t t, int64_t i, int64_t j, int64_t n, f32x4& mnew) {
  f32x4 g = load4(J.g.p, t * J.g.stride + i * J.g.ld + j, J.g.type, n);
  if (!J.mom.p) return g;
  mnew = load4(J.mom.p, t * J.mom.stride + i * J.mom.ld + j, J.mom.type, n);
  const float past = past_range(J.mom.type);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    mnew[e] = fmaf(J.beta, mnew[e], g[e]);
    g[e] = !(fabsf(mnew[e]) < past) ? INFINITY : J.nesterov ? fmaf(J.beta, mnew[e], g[e]) : mnew[e];
  }
  return g;
}

// The wave's sum, the same in every lane; in a fixed order.
__device__ __forceinline__ double wave_sum(double s) {
#pragma unroll
  for (int h = 32; h > 0; h >>= 1) s += __shfl_xor(s, h);
  return s;
}
// The workgroup's sum, likewise, through an array of a number a wave.
template <int kWaves>
__device__ __forceinline__ double block_sum(double s, double (&sums)[kWaves]) {
  s = wave_sum(s);
  if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = s;
  __syncthreads();
  s = sums[0];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) s += sums[w];
  return s;
}
// |U|^2 from the parts that k_norm left, the same in every lane of a workgroup.
template <int kWaves>
__device__ __forceinline__ double norm2_of(const Job& J, int64_t t, double (&sums)[kWaves]) {
  double s = 0.0;
  for (int i = threadIdx.x; i < J.parts; i += 64 * kWaves) s += J.part[t * J.parts + i];
  return block_sum(s, sums);
}

// What takes U to X_0, from |U|^2: 0 where U is zero, whatever eps is (with eps = 0 the reciprocal would be infinite and X_0
// NaN), and NaN where U is not finite.
__device__ __forceinline__ double inverse_norm(const Job& J, double s2) {
  if (!(s2 < INFINITY)) return (double)NAN;
  return s2 > 0.0 ? 1.0 / (sqrt(s2) + J.eps) : 0.0;
}

// Sums of squares in 64 bits: no overflow or loss whatever the scale of the update. A row is read by 2^k
// threads, four entries each, several rows at once where it is short. Bound by its bytes: 4096^2 in bfloat16 in 15 us,
// six 1024 x 4096 with momentum (151 MB) in 39; small matrices by latency (4 to 5 us).
__global__ void __launch_bounds__(kNormThreads) k_norm(Job J, int per_row) {
  const int64_t t = blockIdx.y;
  const int64_t rows = (J.m + J.parts - 1) / J.parts;
  const int64_t r1 = min(J.m, (blockIdx.x + 1) * rows);
  const int64_t j0 = (threadIdx.x & (per_row - 1)) * 4;
  double s = 0.0;
  f32x4 unused;
  for (int64_t i = blockIdx.x * rows + threadIdx.x / per_row; i < r1; i += kNormThreads / per_row)
    for (int64_t j = j0; j < J.n; j += per_row * 4) {
      const f32x4 u = update_at(J, t, i, j, J.n - j, unused);
#pragma unroll
      for (int e = 0; e < 4; ++e) s = fma((double)u[e], (double)u[e], s);
    }
  __shared__ double sums[kNormThreads / 64];
  s = block_sum(s, sums);
  if (threadIdx.x == 0) J.part[t * J.parts + blockIdx.x] = s;
}

// X_0 by 64 x 64 tiles of (R, C), and the new momentum. Tall matrices are turned in LDS. Bound by its bytes: 4096^2 in
// bfloat16 (101 MB) in 27 us, six 1024 x 4096 with momentum (352 MB) in 60.
template <bool kPairs>
__global__ void __launch_bounds__(kNormThreads) k_first(Job J) {
  const int64_t t = blockIdx.z;
  __shared__ float tile[64][65];
  __shared__ double sums[kNormThreads / 64];
  const double s2 = norm2_of(J, t, sums);
  const bool fine = s2 < INFINITY;  // not where U holds an infinity or NaN
  if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) {
    J.norm2[t] = s2;
    if (J.flags) J.flags[t] = !fine ? GSPAR_FLAG_NONFINITE : s2 == 0.0 ? GSPAR_FLAG_ALLZERO : 0u;
  }
  const double inv = inverse_norm(J, s2);
  const int64_t r0 = (int64_t)blockIdx.y * 64, c0 = (int64_t)blockIdx.x * 64;
  char* hi = J.x[0] + t * J.R * J.xrow;
  char* lo = kPairs ? nullptr : J.lo[0] + t * J.R * J.xrow;
  const int64_t pitch = (int64_t)J.panels * 128;
  auto put_first = [&](int64_t r, int64_t c, const f32x4 (&v)[1]) {
    if (J.px) *(f32x4*)(J.px + (t * J.prows + r) * pitch + c) = v[0];
    else put<kPairs>(hi, lo, r, J.xrow, c, v);
  };
  // read along the caller's rows, four entries a thread
  const int four = (threadIdx.x & 15) * 4, row = threadIdx.x >> 4;
  const int64_t j = (J.tall ? r0 : c0) + four;
#pragma unroll
  for (int k = row; k < 64; k += 16) {
    const int64_t i = (J.tall ? c0 : r0) + k;
    f32x4 x[1] = {{0.f, 0.f, 0.f, 0.f}};
    if (i < J.m && j < J.n) {
      f32x4 mnew;
      const f32x4 u = update_at(J, t, i, j, J.n - j, mnew);
      if (J.mom.p && fine) store4(J.mom.p, t * J.mom.stride + i * J.mom.ld + j, J.mom.type, J.n - j, mnew);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[0][e] = j + e < J.n ? (float)(u[e] * inv) * kUnit : 0.f;
    }
    if (!J.tall) {
      if (i < (J.px ? J.prows : J.R)) put_first(i, j, x);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) tile[four + e][k] = x[0][e];
    }
  }
  if (!J.tall) return;
  __syncthreads();
#pragma unroll
  for (int k = row; k < 64; k += 16)
    if (r0 + k < (J.px ? J.prows : J.R)) {
      const f32x4 x[1] = {{tile[k][four], tile[k][four + 1], tile[k][four + 2], tile[k][four + 3]}};
      put_first(r0 + k, c0 + four, x);
    }
}

// ------------------------------------------------------------------------------------------
// The three products of a step.
// ------------------------------------------------------------------------------------------
__device__ __forceinline__ Rows rows_of(const char* base, int64_t t, int64_t rows, int64_t ld) {
  return {base + t * rows * ld, ld, rows, ld};
}

// The other side of a tile off the diagonal is turned in LDS, in the stages that the product is done with, and leaves by
// 16 bytes (4096^2: 84.8 -> 83.4 us for A, 89.2 -> 87.9 for B). Row jn has the tile's column jn, chunk c of 16 bytes at
// c ^ turn, so that the four rows that a wave writes at once lie in different banks. Pairs of 256 x 256 do not fit: they
// write their elements one by one (in two passes through LDS: 181 us for 172, 7 x 1811^2).
template <class C>
struct Mirror {
  static constexpr bool kFits = !C::kPairs || C::BM < 256;
  static constexpr int kRow = C::BM * 2, kChunks = C::BM / 8;
  static __device__ __forceinline__ char* at(int part, int jn, int im) {
    char* base;
    if constexpr (C::kGroups == 2) base = stage<C, 1>() + part * C::BM * kRow;  // the first holds the groups' sums
    else if constexpr (C::kPairs && C::BM == 192)
      base = (jn < 64 ? stage<C, 0>() : jn < 128 ? stage<C, 1>() - 64 * kRow : stage<C, 2>() - 128 * kRow) + part * 64 * kRow;
    else if constexpr (C::kPairs) base = part ? stage<C, 1>() : stage<C, 0>();
    else base = jn < 128 ? stage<C, 0>() : stage<C, 1>() - 128 * kRow;
    return base + jn * kRow + ((im >> 3) ^ (((jn >> 4) & 3) << 1)) * 16 + (im & 7) * 2;
  }
  static __device__ __forceinline__ void write(char* M, const Job& J, int64_t i0, int64_t j0, int block) {
    __syncthreads();
    for (int n = threadIdx.x; n < C::BN * kChunks; n += C::kThreads) {
      const int jn = n / kChunks, c = n % kChunks * 8;
      if (j0 + jn >= J.R || i0 + c >= J.Rp || (block >= 0 && (c >> 4) % C::FM != block)) continue;
      char* to = M + place<C::kPairs>(j0 + jn, J.arow, i0 + c);
      *(u32x4*)to = *(const u32x4*)at(0, jn, c);
      if constexpr (C::kPairs) *(u32x4*)(to + 64) = *(const u32x4*)at(1, jn, c);
    }
  }
};

// Writes values of a symmetric matrix at (i, j ..) of the tile at (i0, j0) and, off the diagonal tiles, leaves or writes
// them for the other side.
template <class C>
__device__ __forceinline__ void put_symmetric(char* M, float* diag, const Job& J, int64_t i0, int64_t j0, int row, int col,
                                              f32x4 (&v)[C::G]) {
  constexpr bool kPairs = C::kPairs;
  const int64_t i = i0 + row, j = j0 + col;
  if (i >= J.Rp || j >= J.Rp) return;  // rows past R hold zeros: they fill the columns past R of the mirror
#pragma unroll
  for (int g = 0; g < C::G; ++g) {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (i == j + 4 * g + e && i < J.R) {
        diag[i] = v[g][e];
        if (!kPairs) v[g][e] = 0.f;
      }
    v[g] = v[g] * kUnit;
  }
  if (i < J.R) put<kPairs>(M, nullptr, i, J.arow, j, v);
  if (i0 == j0) return;
#pragma unroll
  for (int g = 0; g < C::G; ++g)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int c = 4 * g + e;
      const Parts p = split(v[g][e]);
      if constexpr (Mirror<C>::kFits) {
        *(uint16_t*)Mirror<C>::at(0, col + c, row) = p.hi;
        if (kPairs) *(uint16_t*)Mirror<C>::at(1, col + c, row) = p.lo;
      } else if (j + c < J.R) {
        const int64_t at = place<kPairs>(j + c, J.arow, i);
        *(uint16_t*)(M + at) = p.hi;
        if (kPairs) *(uint16_t*)(M + at + 64) = p.lo;
      }
    }
}

// A = X X^T (kSquare: B = b A + c A^2). Step: the whole product, a part of K, or what the parts left. Only tiles of the
// lower triangle are computed. Large ones are bound by the matrix cores (4096^2: A 80 us and B 85, 860 and 810 TFLOP/s of
// what is needed; 253 tiles of 192 x 192 fill the compute units), small ones by a unit's path into LDS and latency
// (R = 1000, C = 2048 in pairs: 18 and 11 us).
enum { kWhole, kPart, kJoin };
template <class C, bool kSquare, int kDo>
__global__ void __launch_bounds__(C::kThreads, C::kThreads / 256) k_symmetric(Job J, int which, int tiles, int per) {
  constexpr bool kPairs = C::kPairs;
  const int64_t t = blockIdx.y;
  int ti, tj;
  const int tile = xcd_order(blockIdx.x, tiles);
  triangle(tile, ti, tj);
  f32x4 acc[C::FN][C::FM];
  clear<C>(acc);
  if constexpr (kDo != kJoin) {
    const Rows X = kSquare ? rows_of(J.A, t, J.R, J.arow) : rows_of(J.x[which], t, J.R, J.xrow);
    const int all = (int)((kSquare ? J.Rp : J.Cp) / C::kStep), start = kDo == kPart ? (int)blockIdx.z * per : 0;
    AlongM<C> left(X, X, (int64_t)ti * C::BM, mine_m<C>());
    AlongN<C> right(X, X, (int64_t)tj * C::BN, mine_n<C>());
    multiply<F16, C>(left, right, kDo == kPart ? min(per, all - start) : all, acc, start);
  }
  if constexpr (kDo == kPart) {
    leave_part<C>(acc, J.parted + ((t * tiles + tile) * gridDim.z + blockIdx.z) * kPartFours<C>);
    return;
  }
  const int block = kDo == kJoin ? (int)blockIdx.z : -1;
  if constexpr (kDo == kJoin) join_parts<C>(acc, J.parted + (t * tiles + tile) * per * kPartFours<C>, per, block);
  char* M = (kSquare ? J.B : J.A) + t * J.R * J.arow;
  float* da = J.da + t * J.Rp;
  float* db = J.db + t * J.Rp;
  const char* A = J.A + t * J.R * J.arow;
  __syncthreads();  // the stages are read
  each<C>(acc, [&](int row, int col, f32x4 (&v)[C::G]) {
    const int64_t i = (int64_t)ti * C::BM + row, j = (int64_t)tj * C::BN + col;
#pragma unroll
    for (int g = 0; g < C::G; ++g) v[g] = v[g] * kPerSum;
    if (kSquare && i < J.R && j < J.Rp) {
      f32x4 o[C::G];
      get<kPairs>(A, nullptr, i, J.arow, j, o);
      const float di = da[i];
#pragma unroll
      for (int g = 0; g < C::G; ++g) {
        o[g] = o[g] * (1.f / kUnit);
        if (kPairs) {
          v[g] = J.b * o[g] + J.c * v[g];
        } else {
          // A = O + D: A^2 = O^2 + D O + O D + D^2
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int64_t c = j + 4 * g + e;
            const float dj = c < J.R ? da[c] : 0.f;
            v[g][e] = i == c ? J.b * di + J.c * fmaf(di, di, v[g][e]) : J.b * o[g][e] + J.c * fmaf(di + dj, o[g][e], v[g][e]);
          }
        }
      }
    }
    put_symmetric<C>(M, kSquare ? db : da, J, (int64_t)ti * C::BM, (int64_t)tj * C::BN, row, col, v);
  }, block);
  if constexpr (Mirror<C>::kFits) {
    if (ti != tj) Mirror<C>::write(M, J, (int64_t)ti * C::BM, (int64_t)tj * C::BN, block);
  }
}

// X <- a X + B X, by tiles of (R, C), or of (C, R) when kAcross (the last step of a tall matrix, whose
// results then lie along the caller's rows). X lies down K, B (symmetric) along it. The last step writes the
// result. whole: X has its lower parts; keep: the new X gets them. 4096^2: 133 us, 100 of them the product's; the rest are
// X and its lower parts, read for a X and written, which no other tile's product hides in the last round. 6 x 1024 x 4096:
// 86 us, bound by those bytes.
template <class C, bool kLast, bool kAcross>
__global__ void __launch_bounds__(C::kThreads, C::kThreads / 256) k_apply(Job J, int which, int tm, int tn, bool whole, bool keep) {
  constexpr bool kPairs = C::kPairs;
  const int64_t t = blockIdx.y;
  int ti, tj;
  banded(xcd_order(blockIdx.x, tm * tn), tm, tn, ti, tj);
  const Rows B = rows_of(J.B, t, J.R, J.arow), X = rows_of(J.x[which], t, J.R, J.xrow);
  const int steps = (int)(J.Rp / C::kStep);
  f32x4 acc[C::FN][C::FM];
  clear<C>(acc);
  if constexpr (kAcross) {
    DownM<C> left(X, X, 0, (int64_t)ti * C::BM, mine_m<C>());
    AlongN<C> right(B, B, (int64_t)tj * C::BN, mine_n<C>());
    multiply<F16, C>(left, right, steps, acc);
  } else {
    AlongM<C> left(B, B, (int64_t)ti * C::BM, mine_m<C>());
    DownN<C> right(X, X, 0, (int64_t)tj * C::BN, mine_n<C>());
    multiply<F16, C>(left, right, steps, acc);
  }
  const char* x = J.x[which] + t * J.R * J.xrow;
  const char* lo = kPairs || !whole ? nullptr : J.lo[which] + t * J.R * J.xrow;
  const float* db = J.db + t * J.Rp;
  char* nx = J.x[which ^ 1] + t * J.R * J.xrow;
  char* nlo = kPairs || !keep ? nullptr : J.lo[which ^ 1] + t * J.R * J.xrow;
  each<C>(acc, [&](int row, int col, f32x4 (&v)[C::G]) {
    const int64_t p = (int64_t)ti * C::BM + row, q = (int64_t)tj * C::BN + col;
    f32x4 old[C::G], d[C::G];
#pragma unroll
    for (int g = 0; g < C::G; ++g) d[g] = f32x4{J.a, J.a, J.a, J.a};
    if (kAcross) {
      // p along C, q along R
      if (p >= J.C || q >= J.R) return;
#pragma unroll
      for (int g = 0; g < C::G; ++g)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int64_t r = q + 4 * g + e;
          old[g][e] = 0.f;
          if (r < J.R) {
            const char* at = x + place<kPairs>(r, J.xrow, p);
            old[g][e] = f16_to_float(*(const uint16_t*)at);
            if (kPairs) old[g][e] += f16_to_float(*(const uint16_t*)(at + 64));
            else if (whole) old[g][e] += f16_to_float(*(const uint16_t*)(lo + place<false>(r, J.xrow, p)));
            if (!kPairs) d[g][e] += db[r];
          }
        }
    } else {
      if (p >= J.R || q >= (kLast ? J.C : J.Cp)) return;
      get<kPairs>(x, lo, p, J.xrow, q, old);
      if (!kPairs) {
#pragma unroll
        for (int g = 0; g < C::G; ++g) d[g] = d[g] + db[p];
      }
    }
#pragma unroll
    for (int g = 0; g < C::G; ++g)
#pragma unroll
      for (int e = 0; e < 4; ++e) v[g][e] = fmaf(d[g][e], old[g][e], v[g][e] * (1.f / kUnit));
    if (!kLast) {
      put<kPairs>(nx, nlo, p, J.xrow, q, v);
      return;
    }
    const int64_t n = J.n - q;
#pragma unroll
    for (int g = 0; g < C::G; ++g) v[g] = v[g] * (1.f / kUnit) * J.rate;
    if (!J.w.p) {
      store_row(J.out.p, t * J.out.stride + p * J.out.ld + q, J.out.type, n, v);
      return;
    }
    if (!(J.norm2[t] < INFINITY)) return;  // a non-finite update leaves the weights as they were
    f32x4 w[C::G];
    const int64_t at = t * J.w.stride + p * J.w.ld + q;
    load_row(J.w.p, at, J.w.type, n, w);
#pragma unroll
    for (int g = 0; g < C::G; ++g)
#pragma unroll
      for (int e = 0; e < 4; ++e) w[g][e] = fmaf(J.decay, w[g][e], -v[g][e]);
    store_row(J.w.p, at, J.w.type, n, w);
    if (J.half.p) store_row(J.half.p, t * J.half.stride + p * J.half.ld + q, J.half.type, n, w);
  });
}

// The result from the last step's X, where the caller's rows are no multiple of eight long: by 64 x 64 tiles of (m, n).
// Bound by its bytes: 16 x 256 x 2756 in 32 bits (135 MB) in 30 us.
template <bool kPairs>
__global__ void __launch_bounds__(kNormThreads) k_result(Job J, int which) {
  const int64_t t = blockIdx.z;
  __shared__ float tile[64][65];
  const char* x = J.x[which] + t * J.R * J.xrow;
  const char* lo = kPairs ? nullptr : J.lo[which] + t * J.R * J.xrow;
  const int64_t i0 = (int64_t)blockIdx.y * 64, j0 = (int64_t)blockIdx.x * 64;
  const int four = (threadIdx.x & 15) * 4, row = threadIdx.x >> 4;
#pragma unroll
  for (int k = row; k < 64; k += 16) {
    // along X's rows
    const int64_t r = (J.tall ? j0 : i0) + k, c = (J.tall ? i0 : j0) + four;
    f32x4 v[1] = {{0.f, 0.f, 0.f, 0.f}};
    if (r < J.R && c < J.Cp) {
      if (J.px) v[0] = *(const f32x4*)(J.px + (t * J.prows + r) * J.panels * 128 + c);
      else get<kPairs>(x, lo, r, J.xrow, c, v);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) (J.tall ? tile[four + e][k] : tile[k][four + e]) = v[0][e];
  }
  __syncthreads();
  if (J.w.p && !(J.norm2[t] < INFINITY)) return;  // a non-finite update leaves the weights as they were
#pragma unroll
  for (int k = row; k < 64; k += 16) {
    const int64_t i = i0 + k, j = j0 + four, n = J.n - j;
    if (i >= J.m || n <= 0) continue;
    f32x4 v;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = J.rate * (tile[k][four + e] * (1.f / kUnit));
    if (!J.w.p) {
      store4(J.out.p, t * J.out.stride + i * J.out.ld + j, J.out.type, n, v);
      continue;
    }
    const int64_t at = t * J.w.stride + i * J.w.ld + j;
    f32x4 w = load4(J.w.p, at, J.w.type, n);
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = fmaf(J.decay, w[e], -v[e]);
    store4(J.w.p, at, J.w.type, n, w);
    if (J.half.p) store4(J.half.p, t * J.half.stride + i * J.half.ld + j, J.half.type, n, w);
  }
}

// ------------------------------------------------------------------------------------------
// Sides up to 128: panels.
//
// All of A and B fit into LDS, so a workgroup takes a panel of 128 columns of X (or a few of them), forms B for
// itself, applies it to its panel, and leaves its part of the next A: one launch a step instead of three, and one
// launch in all where the matrix is a single panel. A launch's end is what tells the workgroups that the others'
// parts are there. X stays in 32 bits, in the registers' own order in the workspace between launches; the parts of
// A are summed in the order of the panels.
//
// What bounds it: latency. One panel of 128 x 128 is 32 matrix-core instructions of a wave and product (96 for
// pairs), between barriers: 9 us a launch for 64 x 576 in pairs, 20 for 32 matrices of 128 x 1024 (the first kernels,
// three products a step: 90 and 132 us a call; by panels 57 and 116).
// ------------------------------------------------------------------------------------------
constexpr int kPanel = 128, kPanelThreads = 512;
constexpr int64_t kPanelSide = 128;  // sides up to this go by panels

// A plane of numbers in LDS, rows of 128: chunk c of 16 bytes of row r is kept at c ^ turn, so that 16 rows' chunks,
// and the rows that a transposing read takes, lie in different banks (all but two of those).
__device__ __forceinline__ uint32_t plane_at(int row, int col) {
  const int turn = ((row & 7) << 1) | ((row >> 3) & 1);
  return (uint32_t)(row * 256 + (((col >> 3) ^ turn) << 4) + (col & 7) * 2);
}
__device__ __forceinline__ u32x4 plane_along(const char* p, int row, int col) { return *(const u32x4*)(p + plane_at(row, col)); }
__device__ __forceinline__ u32x4 plane_down(const char* p, int k, int col) {
  typedef short s16x4 __attribute__((ext_vector_type(4)));
  typedef __attribute__((address_space(3))) s16x4 lds4;
  const int lane = threadIdx.x & 63;
  const int row = k + (lane >> 4) * 8 + ((lane & 15) >> 2), c = col + (lane & 3) * 4;
  const u32x2 a = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(p + plane_at(row, c))));
  const u32x2 b = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(p + plane_at(row + 4, c))));
  return u32x4{a.x, a.y, b.x, b.y};
}

// A lane's RB fours of a tensor whose rows' length C is a multiple of eight: of
// rows b * 16 + lr, columns c .. c + 3; zeros outside R x C. Every load is issued before the first is waited for:
// places outside repeat one inside.
template <int RB>
__device__ __forceinline__ void load_fours(const Job& J, const Tensor& T, int64_t t, int lr, int64_t c, f32x4 (&v)[RB]) {
  const int64_t first = t * T.stride + min(c, J.C - 4);
  if (T.type == GSPAR_F32) {
#pragma unroll
    for (int b = 0; b < RB; ++b) v[b] = *(const f32x4_any*)((const float*)T.p + first + min((int64_t)(b * 16 + lr), J.R - 1) * T.ld);
  } else {
    u16x4 h[RB];
#pragma unroll
    for (int b = 0; b < RB; ++b) h[b] = *(const u16x4_any*)((const uint16_t*)T.p + first + min((int64_t)(b * 16 + lr), J.R - 1) * T.ld);
#pragma unroll
    for (int b = 0; b < RB; ++b)
#pragma unroll
      for (int e = 0; e < 4; ++e) v[b][e] = T.type == GSPAR_BF16 ? bf16_to_float(h[b][e]) : f16_to_float(h[b][e]);
  }
#pragma unroll
  for (int b = 0; b < RB; ++b)
    if (c >= J.C || b * 16 + lr >= J.R) v[b] = f32x4{0.f, 0.f, 0.f, 0.f};
}
template <int RB>
__device__ __forceinline__ void store_fours(const Job& J, const Tensor& T, int64_t t, int lr, int64_t c, const f32x4 (&v)[RB]) {
  if (c >= J.C) return;
#pragma unroll
  for (int b = 0; b < RB; ++b) {
    const int64_t r = b * 16 + lr, at = t * T.stride + r * T.ld + c;
    if (r >= J.R) return;
    if (T.type == GSPAR_F32) {
      *(f32x4_any*)((float*)T.p + at) = v[b];
    } else {
      u16x4 h;
#pragma unroll
      for (int e = 0; e < 4; ++e) h[e] = T.type == GSPAR_BF16 ? float_to_bf16(v[b][e]) : float_to_f16(v[b][e]);
      *(u16x4_any*)((uint16_t*)T.p + at) = h;
    }
  }
}

// Stages from .. to: 0 makes X_0 and its part of A, k makes the k-th step. A launch has one of them, or all where
// the matrix is one panel.
template <int RP, bool kPairs>
__global__ void __launch_bounds__(kPanelThreads) k_panel(Job J, int from, int to) {
  constexpr int RB = RP / 16, NB = RB * (RB + 1) / 2, NQ = (NB + 7) / 8, kParts = kPairs ? 2 : 1;
  __shared__ __align__(1024) char xs[kParts][RP * 256];
  __shared__ __align__(1024) char as[kParts][RP * 256];  // A, then B
  __shared__ float diag[2][RP];
  __shared__ double sums[kPanelThreads / 64];
  int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t t = blockIdx.x;
  const bool alone = J.groups == 1 && J.panels == 1;
  int lr, lc;  // a lane's row and first column of a block of results
  // Makes the lane's number new to the compiler: it then forms the hundreds of places in LDS where they are used
  // instead of keeping them all in registers from one stage to the next.
  auto fresh = [&] {
    asm volatile("" : "+v"(lane));
    lr = lane & 15;
    lc = (lane >> 4) * 4;
  };
  // Blocks of a symmetric matrix: the q-th is row q % RB and, d = q / RB further, column (row + d) % RB; they
  // meet every pair of rows once. Wave w has those with q % 8 = w.
  auto row_of = [&](int q) { return q % RB; };
  auto col_of = [&](int q) { return (q % RB + q / RB) % RB; };
  auto put_block = [&](int q, f32x4 v) {  // v, times 2^12, into the planes, on both sides of the diagonal
    const int i = row_of(q) * 16 + lr, j = col_of(q) * 16 + lc;
    u16x4 h, l;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const Parts p = split(v[e] * kUnit);
      h[e] = p.hi;
      l[e] = p.lo;
    }
    *(u16x4*)(as[0] + plane_at(i, j)) = h;
    if (kPairs) *(u16x4*)(as[kParts - 1] + plane_at(i, j)) = l;
    if (row_of(q) != col_of(q)) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        *(uint16_t*)(as[0] + plane_at(j + e, i)) = h[e];
        if (kPairs) *(uint16_t*)(as[kParts - 1] + plane_at(j + e, i)) = l[e];
      }
    }
  };
  // a block's sum over K = 32 steps of two planes' rows
  auto symmetric = [&](const char (*p)[RP * 256], int q, int steps, f32x4 acc) {
    const int i = row_of(q) * 16 + lr, j = col_of(q) * 16 + lr;
    for (int k = 0; k < steps; ++k) {
      const int c = k * 32 + (lane >> 4) * 8;
      const u32x4 a = plane_along(p[0], i, c), b = plane_along(p[0], j, c);
      acc = mfma<F16>(b, a, acc);
      if constexpr (kPairs) {
        acc = mfma<F16>(plane_along(p[1], j, c), a, acc);
        acc = mfma<F16>(b, plane_along(p[1], i, c), acc);
      }
    }
    return acc;
  };

  f32x4 aq[NQ], x[RB];
  for (int k = from; k <= to; ++k) {
    const bool last = k == J.steps;
    fresh();
    double inv = 0.0;
    bool fine = true;
    if (k == 0 && J.direct && !alone) {
      const double s2 = norm2_of(J, t, sums);
      fine = s2 < INFINITY;
      inv = inverse_norm(J, s2);
      if (blockIdx.y == 0 && threadIdx.x == 0) {
        J.norm2[t] = s2;
        if (J.flags) J.flags[t] = !fine ? GSPAR_FLAG_NONFINITE : s2 == 0.0 ? GSPAR_FLAG_ALLZERO : 0u;
      }
    }
    // the first panel's X travels while A and B are made
    const int64_t pitch = (int64_t)J.panels * kPanel;
    auto row_at = [&](int panel) { return J.px + (t * RP + lr) * pitch + (int64_t)panel * kPanel + wave * 16 + lc; };
    auto load_x = [&](int panel) {
      const float* from = row_at(panel);
#pragma unroll
      for (int b = 0; b < RB; ++b) x[b] = *(const f32x4*)(from + b * 16 * pitch);
    };
    const bool by_rows = k == 0 ? !J.direct : !alone;
    if (by_rows && k > 0) load_x((int)blockIdx.y * J.per_group);
    if (k > 0) {
      // A: the sum of the parts, four groups' at a time; B in its place
      if (!alone) {
        const f32x4* p = J.pa[(k - 1) & 1] + (t * J.groups * NB + wave) * 64 + lane;
#pragma unroll
        for (int n = 0; n < NQ; ++n) aq[n] = f32x4{0.f, 0.f, 0.f, 0.f};
        for (int g0 = 0; g0 < J.groups; g0 += 4) {
          f32x4 v[4][NQ];
#pragma unroll
          for (int g = 0; g < 4; ++g)
#pragma unroll
            for (int n = 0; n < NQ; ++n) v[g][n] = p[((int64_t)min(g0 + g, J.groups - 1) * NB + min(n * 8, NB - 1 - wave)) * 64];
#pragma unroll
          for (int g = 0; g < 4; ++g)
            if (g0 + g < J.groups) {
#pragma unroll
              for (int n = 0; n < NQ; ++n) aq[n] += v[g][n];
            }
        }
      }
#pragma unroll
      for (int n = 0; n < NQ; ++n) {
        const int q = n * 8 + wave;
        if (q >= NB) continue;
        aq[n] = aq[n] * kPerSum;
        f32x4 o = aq[n];
        if (row_of(q) == col_of(q)) {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (lr == lc + e) {
              diag[0][row_of(q) * 16 + lr] = o[e];
              if (!kPairs) o[e] = 0.f;
            }
        }
        put_block(q, o);
      }
      __syncthreads();
      f32x4 bq[NQ];
#pragma unroll
      for (int n = 0; n < NQ; ++n) {
        const int q = n * 8 + wave;
        if (q >= NB) continue;
        const f32x4 s = symmetric(as, q, RP / 32, f32x4{0.f, 0.f, 0.f, 0.f}) * kPerSum;
        const bool on = row_of(q) == col_of(q);
        const float di = diag[0][row_of(q) * 16 + lr];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float dj = diag[0][col_of(q) * 16 + lc + e], o = aq[n][e];
          // A = O + D where the diagonal is carried apart: A^2 = O^2 + D O + O D + D^2
          if (kPairs) bq[n][e] = J.b * o + J.c * s[e];
          else if (on && lr == lc + e) bq[n][e] = J.b * di + J.c * fmaf(di, di, s[e]);
          else bq[n][e] = J.b * o + J.c * fmaf(di + dj, o, s[e]);
        }
      }
      __syncthreads();
#pragma unroll
      for (int n = 0; n < NQ; ++n) {
        const int q = n * 8 + wave;
        if (q >= NB) continue;
        if (row_of(q) == col_of(q)) {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (lr == lc + e) {
              diag[1][row_of(q) * 16 + lr] = bq[n][e];
              if (!kPairs) bq[n][e] = 0.f;
            }
        }
        put_block(q, bq[n]);
      }
    }
#pragma unroll
    for (int n = 0; n < NQ; ++n) aq[n] = f32x4{0.f, 0.f, 0.f, 0.f};

    for (int pn = 0; pn < J.per_group; ++pn) {
      const int panel = (int)blockIdx.y * J.per_group + pn;
      if (panel >= J.panels) break;
      fresh();
      // this wave's 16 columns of the panel, all rows: row b * 16 + lr, columns c .. c + 3
      const int64_t c = (int64_t)panel * kPanel + wave * 16 + lc;
      float* kept = row_at(panel);
      if (k == 0 && J.direct) {
        // U, and the new momentum
        f32x4 m[RB];
        load_fours<RB>(J, J.g, t, lr, c, x);
        if (J.mom.p) {
          load_fours<RB>(J, J.mom, t, lr, c, m);
          const float past = past_range(J.mom.type);
#pragma unroll
          for (int b = 0; b < RB; ++b)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              m[b][e] = fmaf(J.beta, m[b][e], x[b][e]);
              x[b][e] = !(fabsf(m[b][e]) < past) ? INFINITY : J.nesterov ? fmaf(J.beta, m[b][e], x[b][e]) : m[b][e];
            }
        }
        if (alone) {
          double s2 = 0.0;
#pragma unroll
          for (int b = 0; b < RB; ++b)
#pragma unroll
            for (int e = 0; e < 4; ++e) s2 = fma((double)x[b][e], (double)x[b][e], s2);
          s2 = block_sum(s2, sums);
          fine = s2 < INFINITY;
          inv = inverse_norm(J, s2);
          if (threadIdx.x == 0) {
            J.norm2[t] = s2;
            if (J.flags) J.flags[t] = !fine ? GSPAR_FLAG_NONFINITE : s2 == 0.0 ? GSPAR_FLAG_ALLZERO : 0u;
          }
        }
        if (J.mom.p && fine) store_fours<RB>(J, J.mom, t, lr, c, m);
#pragma unroll
        for (int b = 0; b < RB; ++b)
#pragma unroll
          for (int e = 0; e < 4; ++e) x[b][e] = b * 16 + lr < J.R ? (float)(x[b][e] * inv) * kUnit : 0.f;
      } else if (by_rows && (k == 0 || pn > 0)) {
        load_x(panel);
      }
      auto put_x = [&]() {
#pragma unroll
        for (int b = 0; b < RB; ++b) {
          u16x4 h, l;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const Parts p = split(x[b][e]);
            h[e] = p.hi;
            l[e] = p.lo;
          }
          const uint32_t at = plane_at(b * 16 + lr, wave * 16 + lc);
          *(u16x4*)(xs[0] + at) = h;
          if (kPairs) *(u16x4*)(xs[kParts - 1] + at) = l;
        }
      };
      if (k > 0) {
        // a wave's columns are its own: what it reads of X it wrote itself
        put_x();
        __syncthreads();
        f32x4 y[RB];
#pragma unroll
        for (int b = 0; b < RB; ++b) y[b] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < RP / 32; ++s) {
          const u32x4 xh = plane_down(xs[0], s * 32, wave * 16);
          u32x4 xl;
          if (kPairs) xl = plane_down(xs[kParts - 1], s * 32, wave * 16);
#pragma unroll
          for (int b = 0; b < RB; ++b) {
            const u32x4 bh = plane_along(as[0], b * 16 + lr, s * 32 + (lane >> 4) * 8);
            y[b] = mfma<F16>(xh, bh, y[b]);
            if constexpr (kPairs) {
              y[b] = mfma<F16>(xl, bh, y[b]);
              y[b] = mfma<F16>(xh, plane_along(as[1], b * 16 + lr, s * 32 + (lane >> 4) * 8), y[b]);
            }
          }
        }
#pragma unroll
        for (int b = 0; b < RB; ++b) {
          const float d = kPairs ? J.a : J.a + diag[1][b * 16 + lr];
#pragma unroll
          for (int e = 0; e < 4; ++e) x[b][e] = fmaf(d, x[b][e], y[b][e] * (1.f / kUnit));
        }
      }
      if (last) {
        if (!J.direct) {
#pragma unroll
          for (int b = 0; b < RB; ++b) *(f32x4*)(kept + b * 16 * pitch) = x[b];
          continue;
        }
#pragma unroll
        for (int b = 0; b < RB; ++b) x[b] = x[b] * (1.f / kUnit) * J.rate;
        if (!J.w.p) {
          store_fours<RB>(J, J.out, t, lr, c, x);
        } else if (J.norm2[t] < INFINITY) {  // a non-finite update leaves the weights as they were
          f32x4 w[RB];
          load_fours<RB>(J, J.w, t, lr, c, w);
#pragma unroll
          for (int b = 0; b < RB; ++b)
#pragma unroll
            for (int e = 0; e < 4; ++e) w[b][e] = fmaf(J.decay, w[b][e], -x[b][e]);
          store_fours<RB>(J, J.w, t, lr, c, w);
          if (J.half.p) store_fours<RB>(J, J.half, t, lr, c, w);
        }
        continue;
      }
      if (!alone) {
#pragma unroll
        for (int b = 0; b < RB; ++b) *(f32x4*)(kept + b * 16 * pitch) = x[b];
      }
      // this panel's part of the next A
      fresh();
      put_x();
      __syncthreads();
#pragma unroll
      for (int n = 0; n < NQ; ++n) {
        const int q = n * 8 + wave;
        if (q < NB) aq[n] = symmetric(xs, q, kPanel / 32, aq[n]);
      }
      __syncthreads();
    }
    if (!last && !alone) {
#pragma unroll
      for (int n = 0; n < NQ; ++n) {
        const int q = n * 8 + wave;
        if (q < NB) J.pa[k & 1][((t * J.groups + blockIdx.y) * NB + q) * 64 + lane] = aq[n];
      }
    }
  }
}

// ------------------------------------------------------------------------------------------
// Launches.
// ------------------------------------------------------------------------------------------
template <int RP, bool kPairs>
void run_panels(const Job& J, hipStream_t s) {
  const dim3 grid((unsigned)J.batch, (unsigned)J.groups), block(kPanelThreads);
  if (J.groups == 1 && J.panels == 1) {
    hipLaunchKernelGGL((k_panel<RP, kPairs>), grid, block, 0, s, J, 0, J.steps);
    return;
  }
  for (int k = 0; k <= J.steps; ++k) hipLaunchKernelGGL((k_panel<RP, kPairs>), grid, block, 0, s, J, k, k);
}

template <bool kPairs>
int run_job(Job& J, hipStream_t s) {
  int per_row = 8;
  while (per_row < kNormThreads && per_row * 4 < J.n) per_row *= 2;
  const unsigned batch = (unsigned)J.batch;
  const bool panels = J.R <= kPanelSide;
  // rows of eights are read and written by vectors, where they start does not matter; others' ends need single elements
  const bool vec = J.n % 8 == 0;
  J.direct = panels && vec && !J.tall;  // panels read and write the caller's rows themselves
  if (!J.direct || J.panels > 1) hipLaunchKernelGGL(k_norm, dim3(J.parts, batch), dim3(kNormThreads), 0, s, J, per_row);
  if (!J.direct)
    hipLaunchKernelGGL((k_first<kPairs>), dim3((unsigned)((panels ? J.panels * 128 : J.Cp) / 64), (unsigned)(J.Rp / 64), batch),
                       dim3(kNormThreads), 0, s, J);
  int w = 0;
  auto result = [&] {
    hipLaunchKernelGGL((k_result<kPairs>), dim3((unsigned)ceil_div(J.n, 64), (unsigned)ceil_div(J.m, 64), batch),
                       dim3(kNormThreads), 0, s, J, w);
    return launched();
  };
  if (panels) {
    if (J.R <= 64) run_panels<64, kPairs>(J, s);
    else run_panels<128, kPairs>(J, s);
    return J.direct ? launched() : result();
  }
  for (int k = 0; k < J.steps; ++k) {
    auto symmetric = [&](const Way& way, auto square) {
      constexpr bool kSquare = decltype(square)::value;
      with_tile<kPairs>(way, [&](auto tile) {
        typedef decltype(tile) C;
        const int side = (int)ceil_div(J.R, C::BM), tiles = side * (side + 1) / 2;
        const dim3 block(C::kThreads);
        if (way.parts > 1) {
          hipLaunchKernelGGL((k_symmetric<C, kSquare, kPart>), dim3(tiles, batch, way.parts), block, 0, s, J, w, tiles, way.per);
          hipLaunchKernelGGL((k_symmetric<C, kSquare, kJoin>), dim3(tiles, batch, C::FM), block, 0, s, J, w, tiles, way.parts);
        } else {
          hipLaunchKernelGGL((k_symmetric<C, kSquare, kWhole>), dim3(tiles, batch), block, 0, s, J, w, tiles, 0);
        }
      });
    };
    symmetric(J.gram, std::false_type{});
    symmetric(J.square, std::true_type{});
    with_tile<kPairs>(J.apply, [&](auto tile) {
      typedef decltype(tile) C;
      const int tr = (int)ceil_div(J.R, C::BM), tc = (int)ceil_div(J.C, C::BN);
      const dim3 grid(tr * tc, batch), block(C::kThreads);
      // A step lifts the rounding of its X by |a| at most. The last one's, 2^-12 |a| for the usual a of 3.4, is below what
      // the products' roundings leave: its X goes without lower parts (6 x 1024 x 4096, the last product: 115 -> 110 us).
      // A larger |a| keeps them. (Pairs have both parts in one place, and keep them.)
      const bool light = std::fabs(J.a) <= 4.f, whole = !light || k == 0 || k + 1 < J.steps, keep = !light || k + 2 != J.steps;
      if (k + 1 < J.steps || !vec) hipLaunchKernelGGL((k_apply<C, false, false>), grid, block, 0, s, J, w, tr, tc, whole, keep);
      else if (!J.tall) hipLaunchKernelGGL((k_apply<C, true, false>), grid, block, 0, s, J, w, tr, tc, whole, keep);
      else hipLaunchKernelGGL((k_apply<C, true, true>), grid, block, 0, s, J, w, tc, tr, whole, keep);
    });
    w ^= 1;
  }
  return vec ? launched() : result();
}

// Sides, pitches and places in the workspace; returns the workspace's size.
size_t lay_out(Job& J, int64_t batch, int64_t m, int64_t n, bool pairs, char* ws) {
  J.batch = batch;
  J.m = m;
  J.n = n;
  J.tall = m > n;
  J.R = std::min(m, n);
  J.C = std::max(m, n);
  J.Rp = up(J.R, 64);
  J.Cp = up(J.C, 64);
  const int64_t e = pairs ? 4 : 2;
  J.xrow = J.Cp * e;
  J.arow = J.Rp * e;
  // four entries a thread at least, and workgroups enough to fill the device a few times
  J.parts = (int)std::max<int64_t>(1, std::min(std::min<int64_t>(1024, 2048 / batch), std::min(m, ceil_div(m * n, 1024))));
  size_t at = 0;
  auto take = [&](int64_t bytes) {
    char* p = ws ? ws + at : nullptr;
    at += (size_t)up(bytes, 256);
    return p;
  };
  J.part = (double*)take(batch * J.parts * 8);
  J.norm2 = (double*)take(batch * 8);
  if (J.R <= kPanelSide) {
    // A workgroup sums the parts of all of them, so a matrix has 32 at most, and no more than fill the device.
    J.panels = (int)ceil_div(J.C, kPanel);
    const int64_t most = std::max<int64_t>(1, std::min<int64_t>(32, 512 / batch));
    J.per_group = (int)ceil_div(J.panels, most);
    J.groups = (int)ceil_div(J.panels, J.per_group);
    const int64_t rb = J.R <= 64 ? 4 : 8;
    J.prows = rb * 16;
    J.px = (float*)take(batch * J.prows * J.panels * kPanel * 4);
    for (int k = 0; k < 2; ++k) J.pa[k] = (f32x4*)take(batch * J.groups * rb * (rb + 1) / 2 * 1024);
    return at;
  }
  auto triangles = [&](int64_t side) {
    const int64_t k = ceil_div(J.R, side);
    return k * (k + 1) / 2 * batch;
  };
  const int64_t step = pairs ? 32 : 64;
  J.gram = way_of(pairs, true, J.Cp / step, true, triangles);
  J.square = way_of(pairs, true, J.Rp / step, true, triangles);
  J.apply = way_of(pairs, true, J.Rp / step, false, [&](int64_t side) { return ceil_div(J.R, side) * ceil_div(J.C, side) * batch; });
  if (const int64_t fours = std::max(J.gram.fours, J.square.fours)) J.parted = (f32x4*)take(fours * 16);
  for (int k = 0; k < 2; ++k) {
    J.x[k] = take(batch * J.R * J.xrow);
    J.lo[k] = pairs ? nullptr : take(batch * J.R * J.xrow);
  }
  J.A = take(batch * J.R * J.arow);
  J.B = take(batch * J.R * J.arow);
  J.da = (float*)take(batch * J.Rp * 4);
  J.db = (float*)take(batch * J.Rp * 4);
  return at;
}

// Whether the products take both parts of X, by the type of the result.
bool in_pairs(int type) { return type != GSPAR_BF16; }

bool sides_ok(int64_t batch, int64_t m, int64_t n) {
  return batch >= 1 && batch <= 65535 && m >= 1 && n >= 1 && m <= (1 << 20) && n <= (1 << 20);
}

bool tensor_ok(Tensor& t, int64_t batch, int64_t m, int64_t n) {
  if (!t.p || !type_ok(t.type) || ((uintptr_t)t.p & (type_size(t.type) - 1))) return false;
  if (m > 1 && t.ld < n) return false;
  if (m == 1) t.ld = n;
  if (batch > 1 && t.stride < (m - 1) * t.ld + n) return false;
  return true;
}

// The coefficients have to keep every singular value, and every entry of A and B, within what is stored:
// from [0, 1] the largest value that each step can reach is followed on a grid.
bool coefficients_ok(const double* coef, int steps) {
  if (!coef) return false;
  for (int i = 0; i < 3; ++i)
    if (!(std::fabs(coef[i]) <= 1e3)) return false;
  double top = 1.001;
  for (int k = 0; k < steps; ++k) {
    double next = 0.0;
    for (int i = 0; i <= 4096; ++i) {
      const double x = top * i / 4096, y = x * x, q = coef[1] * y + coef[2] * y * y;
      if (std::fabs(q) > kMostStored || y > kMostStored) return false;
      next = std::max(next, std::fabs(x * (coef[0] + q)));
    }
    top = next * 1.01;
  }
  return top <= 4.0;
}

int common(Job& J, int64_t batch, int64_t m, int64_t n, bool pairs, int steps, const double* coef, double eps, void* ws,
           size_t ws_bytes) {
  if (steps < 1 || steps > 32 || !coefficients_ok(coef, steps) || !(eps >= 0.0 && eps < INFINITY)) return GSPAR_ERR_ARG;
  if (!ws || ((uintptr_t)ws & 255) || ws_bytes < lay_out(J, batch, m, n, pairs, nullptr)) return GSPAR_ERR_WORKSPACE;
  lay_out(J, batch, m, n, pairs, (char*)ws);
  J.steps = steps;
  J.a = (float)coef[0];
  J.b = (float)coef[1];
  J.c = (float)coef[2];
  J.eps = eps;
  return GSPAR_OK;
}

}  // namespace
}  // namespace dense
}  // namespace gspar

using namespace gspar::dense;

extern "C" {

size_t gspar_orthogonalize_workspace_bytes(int64_t batch, int64_t m, int64_t n, int out_type) {
  if (!sides_ok(batch, m, n) || !type_ok(out_type)) return 0;
  Job J;
  return lay_out(J, batch, m, n, in_pairs(out_type), nullptr);
}

int gspar_orthogonalize(const void* g, int g_type, int64_t batch, int64_t m, int64_t n, int64_t ldg, int64_t stride_g,
                        int steps, const double* coefficients, double eps, double scale, void* out, int out_type,
                        int64_t ldo, int64_t stride_o, uint32_t* flags, void* ws, size_t ws_bytes, void* stream) {
  if (!sides_ok(batch, m, n) || !(std::fabs(scale) < INFINITY)) return GSPAR_ERR_ARG;
  Job J{};
  J.g = {(void*)g, ldg, stride_g, g_type};
  J.out = {out, ldo, stride_o, out_type};
  if (!tensor_ok(J.g, batch, m, n) || !tensor_ok(J.out, batch, m, n)) return GSPAR_ERR_ARG;
  const bool pairs = in_pairs(out_type);
  if (const int rc = common(J, batch, m, n, pairs, steps, coefficients, eps, ws, ws_bytes)) return rc;
  J.rate = (float)scale;
  J.flags = flags;
  return pairs ? run_job<true>(J, (hipStream_t)stream) : run_job<false>(J, (hipStream_t)stream);
}

int gspar_muon_step(void* w, int w_type, int64_t ldw, int64_t stride_w, void* momentum, int momentum_type, int64_t ldm,
                    int64_t stride_m, const void* g, int g_type, int64_t ldg, int64_t stride_g, int64_t batch, int64_t m,
                    int64_t n, double lr, double beta, int nesterov, double weight_decay, double scale, int steps,
                    const double* coefficients, double eps, void* w_copy, int copy_type, int64_t ldc, int64_t stride_c,
                    uint32_t* flags, void* ws, size_t ws_bytes, void* stream) {
  if (!sides_ok(batch, m, n)) return GSPAR_ERR_ARG;
  if (!(std::fabs(lr) < INFINITY) || !(beta >= 0.0 && beta < INFINITY) || !(std::fabs(weight_decay) < INFINITY) ||
      !(std::fabs(scale) < INFINITY) || !(std::fabs(lr * scale) < INFINITY) || !(std::fabs(lr * weight_decay) < INFINITY))
    return GSPAR_ERR_ARG;
  Job J{};
  J.w = {w, ldw, stride_w, w_type};
  J.mom = {momentum, ldm, stride_m, momentum_type};
  J.g = {(void*)g, ldg, stride_g, g_type};
  if (!tensor_ok(J.w, batch, m, n) || !tensor_ok(J.mom, batch, m, n) || !tensor_ok(J.g, batch, m, n)) return GSPAR_ERR_ARG;
  if (w_copy) {
    J.half = {w_copy, ldc, stride_c, copy_type};
    if (!tensor_ok(J.half, batch, m, n)) return GSPAR_ERR_ARG;
  }
  const bool pairs = in_pairs(w_type);
  if (const int rc = common(J, batch, m, n, pairs, steps, coefficients, eps, ws, ws_bytes)) return rc;
  J.beta = (float)beta;
  J.nesterov = nesterov != 0;
  J.decay = (float)(1.0 - lr * weight_decay);
  J.rate = (float)(lr * scale);
  J.flags = flags;
  return pairs ? run_job<true>(J, (hipStream_t)stream) : run_job<false>(J, (hipStream_t)stream);
}

}  // extern "C"
