// A gated feed-forward block, h = act(x Wg^T) * (x Wu^T), and its backward pass, on matrix cores.
//
// Forward: one product whose right operand takes 8 rows of Wg and 8 of Wu in turn, so that the lane that
// holds a gate's sums holds the up projection's of the same units, and the activation and the product are
// its epilogue. For a later backward pass it keeps both sums, rounded to 24 bits (a float without its last
// eight): rounding them to the tensors' 16 would add errors of the size of the gradients' own rounding.
//
// Backward: dG = dh u act'(g) and dU = dh act(g) from the kept sums in one pass, then
// dx = [dG dU] [Wg; Wu] and [dWg; dWu] = [dG dU]^T x as one product each. dG and dU are rounded to the
// tensors' type once: a product of matrix cores takes 16-bit factors; its sums are of 32 bits. A gradient's error (2-norm)
// so is sqrt(2) times its own rounding: 2.35e-3 for bfloat16, whose rounding makes 1.66e-3.
#include "dense.h"

#include <algorithm>

namespace gspar {
namespace dense {
namespace {

// act(g) and its derivative. Each act is g times a probability p, which is formed without a difference of near numbers,
// so that its tail keeps its digits. So is 1 - p in the tanh form (r), whose slope multiplies it by terms in g^3. SiLU's
// 1 - p is a difference, off by 2^-25 at most: it is added to one, times g, which is 17 or less where p is not one
// itself, so the slope is off by 2^-20 at most there. Reciprocals are the hardware's, within one unit of the last place
// of 32 bits. What all of these go into is rounded to 16.
template <int kAct>
__device__ __forceinline__ void activate(float g, float& a, float& da) {
  if constexpr (kAct == GSPAR_SILU) {
    const float p = __builtin_amdgcn_rcpf(1.f + __expf(-g));
    a = g * p;
    da = p * fmaf(g, 1.f - p, 1.f);
  } else if constexpr (kAct == GSPAR_GELU) {
    const float p = 0.5f * erfcf(g * -0.70710678118654752f);
    a = g * p;
    da = fmaf(g * 0.39894228040143268f, __expf(-0.5f * g * g), p);
  } else {
    // 0.5 (1 + tanh(y)) = 1 / (1 + exp(-2y)) with y = k (g + q g^3)
    const float k2 = 1.59576912160573072f, q = 0.044715f;
    const float gg = fminf(g * g, 1e4f);  // p is 0 or 1 beyond
    const float y2 = k2 * g * fmaf(q, gg, 1.f);
    const float p = __builtin_amdgcn_rcpf(1.f + __expf(-y2)), r = __builtin_amdgcn_rcpf(1.f + __expf(y2));
    a = g * p;
    // from the small factor on: p r is 0 where the others' product would pass the range of 32 bits
    da = fmaf(g * (p * r) * k2, fmaf(3.f * q, gg, 1.f), p);
  }
}

// f of the activation's number as a constant.
template <class F>
void with_act(int act, F&& f) {
  if (act == GSPAR_SILU) f(std::integral_constant<int, GSPAR_SILU>{});
  else if (act == GSPAR_GELU) f(std::integral_constant<int, GSPAR_GELU>{});
  else f(std::integral_constant<int, GSPAR_GELU_TANH>{});
}

// A float rounded to its upper 24 bits; a NaN stays one.
__device__ __forceinline__ uint32_t to24(float v) {
  const uint32_t b = __builtin_bit_cast(uint32_t, v);
  return (b & 0x7FFFFFFFu) > 0x7F800000u ? 0x7FC000u : (b + 0x80u) >> 8;
}
__device__ __forceinline__ float from24(uint32_t hi, uint32_t lo) {
  return __builtin_bit_cast(float, (hi << 16) | (lo << 8));
}

// The kept sums: three planes of 16-bit words, [tokens][ld]: the gate's upper halves, the up projection's,
// and the low bytes of both.
struct Saved {
  uint16_t* p;
  int64_t ld, plane;
};

struct FF {
  int64_t T, D, F;
  Rows x, wg, wu;
  int act;
  uint16_t* h;
  int64_t ldh;
  Saved kept;
};

// Bound by the matrix cores where tokens are many: 8192 x 4096 x 12288 in bfloat16 in 1,354 us (1,218 TFLOP/s, traced) with
// the sums kept (604 MB of its writes) and 1,198 without; 1003 x 2048 x 5461 in float16 in 52, a call (172 tiles of
// 256 x 256 on 256 compute units).
template <class T, class C, bool kKeep, int kAct>
__global__ void __launch_bounds__(C::kThreads, C::kThreads / 256) k_ff_forward(FF J, int tm, int tn) {
  int ti, tj;
  banded(xcd_order(blockIdx.x, tm * tn), tm, tn, ti, tj);
  f32x4 acc[C::FN][C::FM];
  clear<C>(acc);
  {
    AlongM<C> left(J.x, J.x, (int64_t)ti * C::BM, mine_m<C>());
    AlongN<C, true> right(J.wg, J.wu, (int64_t)tj * (C::BN / 2), mine_n<C>());
    multiply<T, C>(left, right, (int)((J.x.bytes + kSlice - 1) / kSlice), acc);
  }
  static_assert(C::G == 4, "a lane's 16 columns are 8 of the gate's and the same 8 of the up projection's");
  each<C>(acc, [&](int row, int col, const f32x4 (&v)[4]) {
    const int64_t t = (int64_t)ti * C::BM + row, f = (int64_t)tj * (C::BN / 2) + col / 2;
    if (t >= J.T || f >= J.F) return;
    u16x4 h[2], k0[2], k1[2], k2[2];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float g = v[e / 4][e % 4], u = v[2 + e / 4][e % 4];
      float a, da;
      activate<kAct>(g, a, da);
      h[e / 4][e % 4] = to16<T>(a * u);
      if constexpr (kKeep) {
        const uint32_t kg = to24(g), ku = to24(u);
        k0[e / 4][e % 4] = (uint16_t)(kg >> 8);
        k1[e / 4][e % 4] = (uint16_t)(ku >> 8);
        k2[e / 4][e % 4] = (uint16_t)((kg & 0xFF) | ((ku & 0xFF) << 8));
      }
    }
    if constexpr (kKeep) {  // rows of the kept planes are padded to a multiple of eight
      uint16_t* k = J.kept.p + t * J.kept.ld + f;
      put16(k, k0);
      put16(k + J.kept.plane, k1);
      put16(k + 2 * J.kept.plane, k2);
    }
    uint16_t* to = J.h + t * J.ldh + f;
    if (f + 8 <= J.F) {
      put16(to, h);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (f + e < J.F) to[e] = h[e / 4][e % 4];
    }
  });
}

// Few tokens: the weights' bytes bound the pass, so it reads them once, straight into registers. A workgroup has
// 16 UB units of both projections and up to 16 TT tokens; its eight waves share out D, and add their sums in LDS.
// The products are D[unit][token] with the weights' rows on the left. A lane reads 8 elements of a row at once, at any
// alignment that the type allows, so no operand is copied; rows past F or T repeat the last one (a row of results
// depends on its own operand's row alone) and are not stored. 24 x 4096 x 12288: 48 us, 4.2 TB/s (41 where a
// cache still holds some of the last call's weights); one token of 1024 x 2816: 5.2 us, latency. (By tiles, the weights
// through LDS: 56 and 16 us a call; so 47 and 10.)
struct Few {
  const uint16_t *x, *wg, *wu;
  int64_t ldx, ldg, ldu;
};

// Elements d .. d + 7 of a row of D, zeros past its end.
__device__ __forceinline__ u32x4 eight(const uint16_t* row, int64_t d, int64_t D) {
  if (d + 8 <= D) return *(const u32x4_any*)(row + d);
  uint16_t v[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = d + e < D ? row[d + e] : (uint16_t)0;
  return __builtin_bit_cast(u32x4, v);
}

template <class T, int UB, int TT, bool kKeep, int kAct>
__global__ void __launch_bounds__(512) k_ff_few(FF J, Few P) {
  constexpr int kWaves = 8;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t f0 = (int64_t)blockIdx.x * 16 * UB;
  const uint16_t *g[UB], *u[UB], *x[TT];
#pragma unroll
  for (int b = 0; b < UB; ++b) {
    const int64_t f = min(f0 + 16 * b + (lane & 15), J.F - 1);
    g[b] = P.wg + f * P.ldg;
    u[b] = P.wu + f * P.ldu;
  }
#pragma unroll
  for (int t = 0; t < TT; ++t) x[t] = P.x + min((int64_t)(16 * t + (lane & 15)), J.T - 1) * P.ldx;
  f32x4 ag[UB][TT], au[UB][TT];
#pragma unroll
  for (int b = 0; b < UB; ++b)
#pragma unroll
    for (int t = 0; t < TT; ++t) ag[b][t] = au[b][t] = f32x4{0.f, 0.f, 0.f, 0.f};

  // steps of 32 of D; each wave has so many in a row, kBatch of them under way at once
  constexpr int kBatch = UB == 1 ? 4 : 2;
  const int all = (int)((J.D + 31) / 32), whole = (int)(J.D / 32), per = (all + kWaves - 1) / kWaves;
  const int first = wave * per, last = min(first + per, whole);
  const int64_t off = (lane >> 4) * 8;
  auto multiply_step = [&](const u32x4 (&vg)[UB], const u32x4 (&vu)[UB], const u32x4 (&vx)[TT]) {
#pragma unroll
    for (int b = 0; b < UB; ++b)
#pragma unroll
      for (int t = 0; t < TT; ++t) {
        ag[b][t] = mfma<T>(vg[b], vx[t], ag[b][t]);
        au[b][t] = mfma<T>(vu[b], vx[t], au[b][t]);
      }
  };
  u32x4 vg[2][kBatch][UB], vu[2][kBatch][UB], vx[2][kBatch][TT];
  auto fetch = [&](int buf, int k) {
#pragma unroll
    for (int s = 0; s < kBatch; ++s) {
      const int64_t d = (int64_t)min(k + s, last - 1) * 32 + off;
#pragma unroll
      for (int b = 0; b < UB; ++b) {
        vg[buf][s][b] = *(const u32x4_any*)(g[b] + d);
        vu[buf][s][b] = *(const u32x4_any*)(u[b] + d);
      }
#pragma unroll
      for (int t = 0; t < TT; ++t) vx[buf][s][t] = *(const u32x4_any*)(x[t] + d);
    }
  };
  auto use = [&](int buf, int k) {
#pragma unroll
    for (int s = 0; s < kBatch; ++s)
      if (k + s < last) multiply_step(vg[buf][s], vu[buf][s], vx[buf][s]);
  };
  if (first < last) {
    fetch(0, first);
    for (int k = first; k < last; k += 2 * kBatch) {
      if (k + kBatch < last) fetch(1, k + kBatch);
      use(0, k);
      if (k + kBatch >= last) break;
      if (k + 2 * kBatch < last) fetch(0, k + 2 * kBatch);
      use(1, k + kBatch);
    }
  }
  if (whole < all && wave == whole / per) {  // the step that D ends in
    u32x4 tg[UB], tu[UB], tx[TT];
    const int64_t d = (int64_t)whole * 32 + off;
#pragma unroll
    for (int b = 0; b < UB; ++b) {
      tg[b] = eight(g[b], d, J.D);
      tu[b] = eight(u[b], d, J.D);
    }
#pragma unroll
    for (int t = 0; t < TT; ++t) tx[t] = eight(x[t], d, J.D);
    multiply_step(tg, tu, tx);
  }

  __shared__ f32x4 sums[kWaves][UB * TT * 2][64];
#pragma unroll
  for (int b = 0; b < UB; ++b)
#pragma unroll
    for (int t = 0; t < TT; ++t) {
      sums[wave][(b * TT + t) * 2][lane] = ag[b][t];
      sums[wave][(b * TT + t) * 2 + 1][lane] = au[b][t];
    }
  __syncthreads();
  if (wave >= UB * TT) return;
  f32x4 sg = sums[0][wave * 2][lane], su = sums[0][wave * 2 + 1][lane];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) {
    sg += sums[w][wave * 2][lane];
    su += sums[w][wave * 2 + 1][lane];
  }
  const int64_t t = (wave % TT) * 16 + (lane & 15), f = f0 + (wave / TT) * 16 + (lane >> 4) * 4;
  if (t >= J.T || f >= J.F) return;
  u16x4 h, k0, k1, k2;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    float a, da;
    activate<kAct>(sg[e], a, da);
    h[e] = to16<T>(a * su[e]);
    const uint32_t kg = to24(sg[e]), ku = to24(su[e]);
    k0[e] = (uint16_t)(kg >> 8);
    k1[e] = (uint16_t)(ku >> 8);
    k2[e] = (uint16_t)((kg & 0xFF) | ((ku & 0xFF) << 8));
  }
  if constexpr (kKeep) {  // rows of the kept planes are padded to a multiple of eight
    uint16_t* k = J.kept.p + t * J.kept.ld + f;
    *(u16x4*)k = k0;
    *(u16x4*)(k + J.kept.plane) = k1;
    *(u16x4*)(k + 2 * J.kept.plane) = k2;
  }
  uint16_t* to = J.h + t * J.ldh + f;
  if (f + 4 <= J.F) {
    *(u16x4_any*)to = h;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (f + e < J.F) to[e] = h[e];
  }
}

// Copies of the operands whose rows the products cannot read where they are: dst [rows][ld] <- src [rows][cols], zeros
// past cols, in one launch, 16 bytes at a time at any alignment that the type allows (1296 x 3459 and 2 x 1472 x 3459:
// 12 us; 25 in three launches).
struct Copies {
  struct One {
    const uint16_t* src;
    int64_t ld, rows;
    uint16_t* dst;
  } of[3];
  int n = 0;
  int64_t cols, pitch;
};
// A row is copied by 2^k threads, several rows at once where it is short.
__global__ void __launch_bounds__(256) k_pack(Copies J, int per_row) {
  const Copies::One M = J.of[blockIdx.z];
  const int64_t c = ((int64_t)blockIdx.x * 256 + (threadIdx.x & (per_row - 1))) * 8;
  if (c >= J.pitch) return;
  const int at_once = 256 / per_row;
  for (int64_t r = (int64_t)blockIdx.y * at_once + threadIdx.x / per_row; r < M.rows; r += (int64_t)gridDim.y * at_once)
    *(u32x4*)(M.dst + r * J.pitch + c) = eight(M.src + r * M.ld, c, J.cols);
}

// dG and dU, [tokens][2 ld]: dG in the first ld columns and dU in the others, zeros past F. Eight of each a
// thread. Bound by its bytes: 8192 x 12288 in bfloat16 (1.2 GB) in 260 us, 4.6 TB/s.
template <class T, int kAct>
__global__ void __launch_bounds__(256) k_ff_between(FF J, const uint16_t* dh, int64_t lddh, uint16_t* dgu, int64_t ld) {
  const int64_t f = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
  if (f >= ld) return;
  for (int64_t t = blockIdx.y; t < J.T; t += gridDim.y) {
    uint16_t vg[8] = {}, vu[8] = {};
    if (f < J.F) {
      uint16_t k0[8], k1[8], k2[8], d[8];
      const uint16_t* k = J.kept.p + t * J.kept.ld + f;  // planes padded to a multiple of eight
      *(u32x4*)k0 = *(const u32x4*)k;
      *(u32x4*)k1 = *(const u32x4*)(k + J.kept.plane);
      *(u32x4*)k2 = *(const u32x4*)(k + 2 * J.kept.plane);
      *(u32x4*)d = eight(dh + t * lddh, f, J.F);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float g = from24(k0[e], k2[e] & 0xFF), u = from24(k1[e], k2[e] >> 8), v = from16<T>(d[e]);
        float a, da;
        activate<kAct>(g, a, da);
        vg[e] = f + e < J.F ? to16<T>(v * u * da) : (uint16_t)0;
        vu[e] = f + e < J.F ? to16<T>(v * a) : (uint16_t)0;
      }
    }
    uint16_t* to = dgu + t * 2 * ld + f;
    *(u32x4*)to = *(const u32x4*)vg;
    *(u32x4*)(to + ld) = *(const u32x4*)vu;
  }
}

// dx = [dG dU] [Wg; Wu] (kDown = false), or [dWg; dWu] = [dG dU]^T x (kDown): out[i][j] = sum_k A(i, k) B(j, k),
// A along K or down it, B down K. Rows of results in [cut0, cut1) are not there (the padding between dG and
// dU); those from cut1 on go to out1. Bound by the matrix cores where all sides are long: 8192 x 4096 x 12288 in
// bfloat16, dx 1,257 us (1,313 TFLOP/s), dW, both operands of which lie down K, 1,487 (1,109).
struct Product {
  Rows a, b0, b1;
  int steps, cut;  // slices of K; those of b0
  uint16_t *out0, *out1;
  int64_t ld0, ld1, rows, cols, cut0, cut1;
};

enum { kWhole, kPart, kJoin };  // a product, a part of its K, or what the parts left
template <class T, class C, bool kDown, int kDo>
__global__ void __launch_bounds__(C::kThreads, C::kThreads / 256) k_product(Product J, int tm, int tn, f32x4* parts, int per) {
  int ti, tj;
  const int tile = xcd_order(blockIdx.x, tm * tn);
  banded(tile, tm, tn, ti, tj);
  f32x4 acc[C::FN][C::FM];
  clear<C>(acc);
  const int start = kDo == kPart ? (int)blockIdx.y * per : 0, steps = kDo == kPart ? min(per, J.steps - start) : J.steps;
  if constexpr (kDo == kJoin) {
    join_parts<C>(acc, parts + (int64_t)tile * per * kPartFours<C>, per, (int)blockIdx.y);
  } else if constexpr (kDown) {
    DownM<C> left(J.a, J.a, 0, (int64_t)ti * C::BM, mine_m<C>());
    DownN<C> right(J.b0, J.b0, 0, (int64_t)tj * C::BN, mine_n<C>());
    multiply<T, C>(left, right, steps, acc, start);
  } else {
    AlongM<C> left(J.a, J.a, (int64_t)ti * C::BM, mine_m<C>());
    DownN<C, true> right(J.b0, J.b1, J.cut, (int64_t)tj * C::BN, mine_n<C>());
    multiply<T, C>(left, right, steps, acc, start);
  }
  if constexpr (kDo == kPart) {
    leave_part<C>(acc, parts + ((int64_t)tile * gridDim.y + blockIdx.y) * kPartFours<C>);
    return;
  }
  each<C>(acc, [&](int row, int col, const f32x4 (&v)[C::G]) {
    const int64_t i = (int64_t)ti * C::BM + row, j = (int64_t)tj * C::BN + col;
    if (i >= J.rows || j >= J.cols || (i >= J.cut0 && i < J.cut1)) return;
    uint16_t* to = i < J.cut1 ? J.out0 + i * J.ld0 : J.out1 + (i - J.cut1) * J.ld1;
    if (j + 4 * C::G <= J.cols) {
      store_row(to, j, std::is_same_v<T, F16> ? GSPAR_F16 : GSPAR_BF16, J.cols - j, v);
    } else {
#pragma unroll
      for (int e = 0; e < 4 * C::G; ++e)
        if (j + e < J.cols) to[j + e] = to16<T>(v[e / 4][e % 4]);
    }
  }, kDo == kJoin ? (int)blockIdx.y : -1);
}

__global__ void __launch_bounds__(256) k_zero_rows(uint16_t* p, int64_t ld, int64_t rows, int64_t cols) {
  const int64_t total = rows * cols;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) p[i / cols * ld + i % cols] = 0;
}

// ------------------------------------------------------------------------------------------
// Launches.
// ------------------------------------------------------------------------------------------
// Tokens up to which the pass for few of them is taken (it copies no operand).
constexpr int64_t kFew = 32;

constexpr int64_t kMostD = 1 << 20, kMostF = 1 << 20, kMostT = 1 << 21;

bool sizes_ok(int64_t T, int64_t D, int64_t F) {
  return T >= 0 && T <= kMostT && D >= 1 && D <= kMostD && F >= 1 && F <= kMostF;
}
bool rows_ok(const void* p, int64_t ld, int64_t rows, int64_t cols) {
  return p && !((uintptr_t)p & 1) && (rows <= 1 || ld >= cols);
}
bool rows_aligned(const void* p, int64_t ld, int64_t rows, int64_t cols) {
  return !((uintptr_t)p & 15) && !(cols & 7) && (rows <= 1 || !(ld & 7));
}
// 256 rows of an operand stay within a buffer's 31 bits of offset
constexpr int64_t kMostLd = 4000000;

struct Take {
  char* ws;
  size_t at = 0;
  uint16_t* operator()(int64_t words) {
    char* p = ws ? ws + at : nullptr;
    at += (size_t)up(words * 2, 256);
    return (uint16_t*)p;
  }
};

int64_t kept_ld(int64_t F) { return up(F, 8); }

struct ForwardSpace {
  uint16_t *x, *wg, *wu;
};
size_t forward_space(int64_t T, int64_t D, int64_t F, bool aligned, char* ws, ForwardSpace* s) {
  Take take{ws};
  ForwardSpace v{};
  if (!aligned && T > kFew) {
    const int64_t Dp = up(D, 8);
    v.x = take(T * Dp);
    v.wg = take(F * Dp);
    v.wu = take(F * Dp);
  }
  if (s) *s = v;
  return std::max<size_t>(take.at, 256);
}

unsigned blocks_for(int64_t items) { return (unsigned)std::min<int64_t>(std::max<int64_t>(ceil_div(items, 256), 1), 1 << 16); }

template <class T>
int forward(FF& J, bool keep, hipStream_t s) {
  const Way way = way_of(false, false, ceil_div(J.D, 64), false, [&](int64_t side) { return ceil_div(J.T, side) * ceil_div(2 * J.F, side); });
  with_tile<false, false>(way, [&](auto tile) {
    // a wave's columns have to be a multiple of 64, for the gate's and the up projection's to meet in a lane
    typedef decltype(tile) Any;
    typedef std::conditional_t<Any::BN == 64, Tile<64, 64, 4, 1, 4, false, Any::kGroups>, Any> C;
    const int tm = (int)ceil_div(J.T, C::BM), tn = (int)ceil_div(J.F, C::BN / 2);
    const dim3 grid((unsigned)((int64_t)tm * tn));
    with_act(J.act, [&](auto act) {
      constexpr int kAct = decltype(act)::value;
      if (keep) hipLaunchKernelGGL((k_ff_forward<T, C, true, kAct>), grid, dim3(C::kThreads), 0, s, J, tm, tn);
      else hipLaunchKernelGGL((k_ff_forward<T, C, false, kAct>), grid, dim3(C::kThreads), 0, s, J, tm, tn);
    });
  });
  return launched();
}

template <class T>
int forward_few(const FF& J, const Few& P, bool keep, hipStream_t s) {
  // Blocks of 16 units a workgroup: what leaves least to the compute unit with most of them, and of equals the
  // larger (the tokens are read once a workgroup). 24 x 4096 x 12288: 59 us with two (384 workgroups on 256 compute
  // units), 57 with one, 47 with three.
  const int64_t blocks = ceil_div(J.F, 16);
  int best = 1;
  auto most = [&](int ub) { return ceil_div(ceil_div(blocks, ub), 256) * ub; };
  for (int ub = 2; ub <= 4; ++ub)
    if (most(ub) <= most(best)) best = ub;
  const dim3 grid((unsigned)ceil_div(blocks, best)), block(512);
  with_act(J.act, [&](auto act) {
    constexpr int kAct = decltype(act)::value;
    auto go = [&](auto ub, auto tt) {
      constexpr int UB = decltype(ub)::value, TT = decltype(tt)::value;
      if (keep) hipLaunchKernelGGL((k_ff_few<T, UB, TT, true, kAct>), grid, block, 0, s, J, P);
      else hipLaunchKernelGGL((k_ff_few<T, UB, TT, false, kAct>), grid, block, 0, s, J, P);
    };
    auto with = [&](auto ub) { J.T <= 16 ? go(ub, std::integral_constant<int, 1>{}) : go(ub, std::integral_constant<int, 2>{}); };
    switch (best) {
      case 1: return with(std::integral_constant<int, 1>{});
      case 2: return with(std::integral_constant<int, 2>{});
      case 3: return with(std::integral_constant<int, 3>{});
      default: return with(std::integral_constant<int, 4>{});
    }
  });
  return launched();
}

Way product_way(int64_t rows, int64_t cols, int64_t steps) {
  return way_of(false, true, steps, true, [&](int64_t side) { return ceil_div(rows, side) * ceil_div(cols, side); });
}

template <class T, bool kDown>
void product(const Product& P, f32x4* parts, hipStream_t s) {
  const Way way = product_way(P.rows, P.cols, P.steps);
  with_tile<false>(way, [&](auto tile) {
    typedef decltype(tile) C;
    const int tm = (int)ceil_div(P.rows, C::BM), tn = (int)ceil_div(P.cols, C::BN);
    const unsigned n = (unsigned)((int64_t)tm * tn);
    const dim3 block(C::kThreads);
    if (way.parts > 1) {
      hipLaunchKernelGGL((k_product<T, C, kDown, kPart>), dim3(n, way.parts), block, 0, s, P, tm, tn, parts, way.per);
      hipLaunchKernelGGL((k_product<T, C, kDown, kJoin>), dim3(n, C::FM), block, 0, s, P, tm, tn, parts, way.parts);
    } else {
      hipLaunchKernelGGL((k_product<T, C, kDown, kWhole>), dim3(n), block, 0, s, P, tm, tn, parts, 0);
    }
  });
}

struct BackwardSpace {
  uint16_t *dgu, *x, *wg, *wu;
  f32x4* parts;
};
size_t backward_space(int64_t T, int64_t D, int64_t F, bool aligned, char* ws, BackwardSpace* s) {
  Take take{ws};
  BackwardSpace v{};
  const int64_t Fp = up(F, 64);
  v.dgu = take(T * 2 * Fp);
  if (!aligned) {
    const int64_t Dp = up(D, 8);
    v.x = take(T * Dp);
    v.wg = take(F * Dp);
    v.wu = take(F * Dp);
  }
  // one product after the other: dx, then both of the weights' gradients, or one
  int64_t fours = 0;
  if (T > 0)
    for (const Way& way : {product_way(T, D, Fp / 32), product_way(Fp + F, D, ceil_div(T, 64)), product_way(F, D, ceil_div(T, 64))})
      fours = std::max(fours, way.fours);
  if (fours) v.parts = (f32x4*)take(fours * 8);
  if (s) *s = v;
  return std::max<size_t>(take.at, 256);
}

template <class T>
int backward(FF& J, const uint16_t* dh, int64_t lddh, uint16_t* dx, int64_t lddx, uint16_t* dwg, int64_t lddg, uint16_t* dwu,
             int64_t lddu, uint16_t* dgu, f32x4* parts, hipStream_t s) {
  const int64_t Fp = up(J.F, 64);
  with_act(J.act, [&](auto act) {
    hipLaunchKernelGGL((k_ff_between<T, decltype(act)::value>), dim3((unsigned)ceil_div(Fp, 2048), (unsigned)std::min<int64_t>(J.T, 16384)), dim3(256), 0, s,
                       J, dh, lddh, dgu, Fp);
  });
  const Rows all{(const char*)dgu, 4 * Fp, J.T, 4 * Fp};
  if (dx) {
    Product P{all, J.wg, J.wu, (int)(Fp / 32), (int)(Fp / 64), dx, dx, lddx, lddx, J.T, J.D, J.T, J.T};
    product<T, false>(P, parts, s);
  }
  if (dwg || dwu) {
    // both, or the one that is asked for
    Product P{all, J.x, J.x, (int)ceil_div(J.T, 64), 0, dwg, dwu, lddg, lddu, Fp + J.F, J.D, J.F, Fp};
    if (!dwg || !dwu) {
      P.a.base += dwg ? 0 : Fp * 2;
      P.a.bytes = Fp * 2;
      P.out0 = dwg ? dwg : dwu;
      P.ld0 = dwg ? lddg : lddu;
      P.rows = P.cut0 = P.cut1 = J.F;
    }
    product<T, true>(P, parts, s);
  }
  return launched();
}

// x and the weights as the products read them: where they are if their rows start on 16-byte boundaries, else
// copied.
bool operands_aligned(const void* x, int64_t ldx, const void* wg, int64_t ldg, const void* wu, int64_t ldu, int64_t T, int64_t D,
                      int64_t F) {
  return rows_aligned(x, ldx, T, D) && rows_aligned(wg, ldg, F, D) && rows_aligned(wu, ldu, F, D) &&
         std::max(T > 1 ? ldx : 0, F > 1 ? std::max(ldg, ldu) : 0) <= kMostLd;
}
Rows operand(const void* p, int64_t ld, int64_t rows, int64_t cols, uint16_t* copy, Copies& copies) {
  if (rows == 1) ld = cols;
  if (!copy) return {(const char*)p, ld * 2, rows, cols * 2};
  const int64_t pitch = up(cols, 8);
  copies.of[copies.n++] = {(const uint16_t*)p, ld, rows, copy};
  copies.cols = cols;
  copies.pitch = pitch;
  return {(const char*)copy, pitch * 2, rows, pitch * 2};
}
void make(const Copies& c, hipStream_t s) {
  if (!c.n) return;
  int64_t rows = 0;
  for (int k = 0; k < c.n; ++k) rows = std::max(rows, c.of[k].rows);
  int per_row = 8;
  while (per_row < 256 && per_row * 8 < c.pitch) per_row *= 2;
  hipLaunchKernelGGL(k_pack, dim3((unsigned)ceil_div(c.pitch, 2048), (unsigned)std::min<int64_t>(ceil_div(rows, 256 / per_row), 16384), c.n),
                     dim3(256), 0, s, c, per_row);
}

}  // namespace
}  // namespace dense
}  // namespace gspar

using namespace gspar::dense;

extern "C" {

size_t gspar_gated_ff_saved_bytes(int64_t tokens, int64_t d_hidden) {
  if (!sizes_ok(tokens, 1, d_hidden)) return 0;
  return (size_t)std::max<int64_t>(6 * tokens * kept_ld(d_hidden), 16);
}

size_t gspar_gated_ff_workspace_bytes(int64_t tokens, int64_t d_in, int64_t d_hidden, int aligned, int backward_) {
  if (!sizes_ok(tokens, d_in, d_hidden)) return 0;
  if (backward_) return backward_space(tokens, d_in, d_hidden, aligned && !(d_in & 7), nullptr, nullptr);
  return forward_space(tokens, d_in, d_hidden, aligned && !(d_in & 7), nullptr, nullptr);
}

int gspar_gated_ff_forward(const void* x, int64_t ldx, const void* w_gate, int64_t ldg, const void* w_up, int64_t ldu,
                           int type, int64_t tokens, int64_t d_in, int64_t d_hidden, int act, void* h, int64_t ldh,
                           void* saved, void* ws, size_t ws_bytes, void* stream) {
  if (!sizes_ok(tokens, d_in, d_hidden) || (type != GSPAR_BF16 && type != GSPAR_F16) || act < GSPAR_SILU || act > GSPAR_GELU_TANH)
    return GSPAR_ERR_ARG;
  if (tokens == 0) return GSPAR_OK;
  if (!rows_ok(x, ldx, tokens, d_in) || !rows_ok(w_gate, ldg, d_hidden, d_in) || !rows_ok(w_up, ldu, d_hidden, d_in) ||
      !rows_ok(h, ldh, tokens, d_hidden) || ((uintptr_t)saved & 15))
    return GSPAR_ERR_ARG;
  hipStream_t s = (hipStream_t)stream;
  FF J{};
  J.T = tokens;
  J.D = d_in;
  J.F = d_hidden;
  J.act = act;
  J.h = (uint16_t*)h;
  J.ldh = tokens > 1 ? ldh : d_hidden;
  J.kept = {(uint16_t*)saved, kept_ld(d_hidden), tokens * kept_ld(d_hidden)};
  const bool aligned = operands_aligned(x, ldx, w_gate, ldg, w_up, ldu, tokens, d_in, d_hidden);
  if (!ws || ((uintptr_t)ws & 255) || ws_bytes < forward_space(tokens, d_in, d_hidden, aligned, nullptr, nullptr))
    return GSPAR_ERR_WORKSPACE;
  if (tokens <= kFew) {
    const Few P{(const uint16_t*)x, (const uint16_t*)w_gate, (const uint16_t*)w_up, ldx, ldg, ldu};
    return type == GSPAR_F16 ? forward_few<F16>(J, P, saved != nullptr, s) : forward_few<BF16>(J, P, saved != nullptr, s);
  }
  ForwardSpace v;
  forward_space(tokens, d_in, d_hidden, aligned, (char*)ws, &v);
  Copies copies;
  J.x = operand(x, ldx, tokens, d_in, v.x, copies);
  J.wg = operand(w_gate, ldg, d_hidden, d_in, v.wg, copies);
  J.wu = operand(w_up, ldu, d_hidden, d_in, v.wu, copies);
  make(copies, s);
  return type == GSPAR_F16 ? forward<F16>(J, saved != nullptr, s) : forward<BF16>(J, saved != nullptr, s);
}

int gspar_gated_ff_backward(const void* dh, int64_t lddh, const void* x, int64_t ldx, const void* w_gate, int64_t ldg,
                            const void* w_up, int64_t ldu, const void* saved, int type, int64_t tokens, int64_t d_in,
                            int64_t d_hidden, int act, void* dx, int64_t lddx, void* dw_gate, int64_t lddg, void* dw_up,
                            int64_t lddu, void* ws, size_t ws_bytes, void* stream) {
  if (!sizes_ok(tokens, d_in, d_hidden) || (type != GSPAR_BF16 && type != GSPAR_F16) || act < GSPAR_SILU || act > GSPAR_GELU_TANH)
    return GSPAR_ERR_ARG;
  if ((dx && !rows_ok(dx, lddx, tokens, d_in)) || (dw_gate && !rows_ok(dw_gate, lddg, d_hidden, d_in)) ||
      (dw_up && !rows_ok(dw_up, lddu, d_hidden, d_in)))
    return GSPAR_ERR_ARG;
  hipStream_t s = (hipStream_t)stream;
  if (tokens == 0) {  // no token: the weights' gradients are zero
    if (dw_gate) hipLaunchKernelGGL(k_zero_rows, dim3(blocks_for(d_in * d_hidden)), dim3(256), 0, s, (uint16_t*)dw_gate, lddg, d_hidden, d_in);
    if (dw_up) hipLaunchKernelGGL(k_zero_rows, dim3(blocks_for(d_in * d_hidden)), dim3(256), 0, s, (uint16_t*)dw_up, lddu, d_hidden, d_in);
    return dw_gate || dw_up ? launched() : GSPAR_OK;
  }
  if (!rows_ok(dh, lddh, tokens, d_hidden) || !rows_ok(x, ldx, tokens, d_in) || !rows_ok(w_gate, ldg, d_hidden, d_in) ||
      !rows_ok(w_up, ldu, d_hidden, d_in) || !saved || ((uintptr_t)saved & 15))
    return GSPAR_ERR_ARG;
  const bool aligned = operands_aligned(x, ldx, w_gate, ldg, w_up, ldu, tokens, d_in, d_hidden);
  if (!ws || ((uintptr_t)ws & 255) || ws_bytes < backward_space(tokens, d_in, d_hidden, aligned, nullptr, nullptr))
    return GSPAR_ERR_WORKSPACE;
  BackwardSpace v;
  backward_space(tokens, d_in, d_hidden, aligned, (char*)ws, &v);
  FF J{};
  J.T = tokens;
  J.D = d_in;
  J.F = d_hidden;
  J.act = act;
  J.kept = {(uint16_t*)saved, kept_ld(d_hidden), tokens * kept_ld(d_hidden)};
  Copies copies;
  if (dw_gate || dw_up) J.x = operand(x, ldx, tokens, d_in, v.x, copies);
  if (dx) {
    J.wg = operand(w_gate, ldg, d_hidden, d_in, v.wg, copies);
    J.wu = operand(w_up, ldu, d_hidden, d_in, v.wu, copies);
  }
  make(copies, s);
  auto run = [&](auto t) {
    return backward<decltype(t)>(J, (const uint16_t*)dh, lddh, (uint16_t*)dx, lddx, (uint16_t*)dw_gate, lddg, (uint16_t*)dw_up,
                                 lddu, v.dgu, v.parts, s);
  };
  return type == GSPAR_F16 ? run(F16{}) : run(BF16{});
}

}  // extern "C"
