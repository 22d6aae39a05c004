// Layer norm over the last axis, forward and backward, with the reduction of gamma's and beta's gradients over the rows.
//
// Bound: DRAM.  Forward a row is read once, kept in registers for mean, squares and result, and written once; backward the same of x and
// grad_y, while every thread adds up grad_y h and grad_y of its columns over the rows that its block takes.  A block's sums go to the
// workspace, and a second kernel adds the blocks' up, always in the same order: P(sum), the all-reduce and the reduce-scatter of data
// parallelism are which blocks it adds and where it stores.
//
// G threads share a row, each with NV times eight of its elements.  Rows too long for registers (over 16384, backward 8192) are read again for
// each pass, out of L2.
//
// Mean and deviation: a first mean c from the row's sum, then the sum of d^2, d = x - c.  Where c is more than four deviations its own rounding shows beside them:
// one more sum over the row gives f = sum d / n, the mean is c + f, the difference from it d - f and n times the variance sum d^2 - f sum d.  Of equal elements d
// is a few units in the last place, at most 28 for rows in registers (32 additions in a thread, nine levels of a tree), so its sums are whole numbers of those
// units and of their squares, below 28^2 2^14 < 2^24 and exact; f is d then, and the variance zero.
#include <atomic>

#include "blocks8.h"

namespace sbp {

namespace {

struct NormJob {
  const void* x;
  const void* dy;      // backward
  void* out;           // y, or grad_x
  float* mean;
  float* rstd;
  long long rows, ldx, lddy, ldo;
};
struct NormParams {
  NormJob j[SBP_MAX_K];
  const void* gamma;   // null: ones
  const void* beta;    // null: zeros
  int gamma_f32, beta_f32;
  int gamma_whole, beta_whole;      // 16-byte aligned
  long long cols;
  float eps;
  float* parts;        // backward: [job * blocks of a job + block][2][cols]; null: the sums are not wanted
  int first_only;      // the jobs are replicas: the sums of the first one's rows are wanted
};

__device__ __forceinline__ float vector_at(const void* p, int f32, long long c, float none) {
  if (!p) return none;
  if (f32) return SBP_GUARD(static_cast<const float*>(p) + c, 4) ? static_cast<const float*>(p)[c] : 0.f;
  return SBP_GUARD(static_cast<const __nv_bfloat16*>(p) + c, 2) ? __bfloat162float(static_cast<const __nv_bfloat16*>(p)[c]) : 0.f;
}

// Eight elements of gamma or beta; `whole`: they may be loaded as vectors.
template <bool VEC>
__device__ __forceinline__ void vector8(const void* p, int f32, int whole, long long col, int n, int step, float none, float (&v)[8]) {
  if (VEC && whole && n > 0) {
    if (f32) load8<true>(static_cast<const float*>(p) + col, v);
    else load8<true>(static_cast<const __nv_bfloat16*>(p) + col, v);
    return;
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = e < n ? vector_at(p, f32, col + e * step, none) : 0.f;
}

// Where thread t of G finds its elements of chunk i (8 G elements): VEC eight that follow one another, else every G-th.
template <int G, bool VEC>
struct Piece {
  long long col;
  int n;
  static constexpr int step = VEC ? 1 : G;
  __device__ __forceinline__ Piece(int i, int t, long long cols) {
    col = (long long)i * (8 * G) + (VEC ? t * 8 : t);
    if constexpr (VEC) n = col < cols ? 8 : 0;
    else n = col < cols ? (int)min((cols - col + G - 1) / G, 8LL) : 0;
  }
};

// Sums over the G threads of a row; G over 32 is the whole block.  `turn` alternates between two buffers, so one barrier does.  Of two sums each half of a
// warp adds one, and every thread adds the warps' parts itself.
template <int G, int N, typename T>
__device__ __forceinline__ void row_sums(T (&s)[N], T (*buf)[N][32], int& turn) {
  static_assert(N <= 2, "a half of the warp each");
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  T v = s[0];
  if constexpr (N == 2) {
    const T other = lane & 16 ? s[0] : s[1];
    v = lane & 16 ? s[1] : s[0];
    v += __shfl_xor_sync(0xffffffffu, other, 16);
  }
#pragma unroll
  for (int d = N == 2 ? 8 : 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
  if constexpr (G > 32) {
    if ((lane & (N == 2 ? 15 : 31)) == 0) buf[turn][lane >> 4][warp] = v;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < N; ++k) {
      T part[G / 32];
#pragma unroll
      for (int w = 0; w < G / 32; ++w) part[w] = buf[turn][k][w];
#pragma unroll
      for (int d = G / 64; d > 0; d >>= 1)
#pragma unroll
        for (int w = 0; w < d; ++w) part[w] += part[w + d];
      s[k] = part[0];
    }
    turn ^= 1;
  } else {
    s[0] = v;
    if constexpr (N == 2) {
      s[0] = __shfl_sync(0xffffffffu, v, 0);
      s[1] = __shfl_sync(0xffffffffu, v, 16);
    }
  }
}

__device__ __forceinline__ void pairs_of(const float (&u)[8], unsigned long long (&v)[4]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = pair_of(u[2 * e], u[2 * e + 1]);
}

// Is a first mean more than four times the deviation, by the sum of the squares of differences from it?  (NaN: no.  The mean of zeros is none.)
__device__ __forceinline__ bool far_row(float c, float squares, float inv_n) { return squares * inv_n * 16.f <= c * c && c != 0.f; }

// What the first mean is off by, given the sum of the differences: times the reciprocal of n, with one step of correction, right where the
// quotient is a number of fp32.
__device__ __forceinline__ float mean_off(float sum_d, float n, float inv_n) {
  const float q = sum_d * inv_n;
  return fmaf(fmaf(-q, n, sum_d), inv_n, q);
}
// 1 / deviation.  (Squares that overflow leave an infinite variance, as the multiply-add keeps it; NaN stays.)
__device__ __forceinline__ float inverse_deviation(float squares, float f, float sum_d, float inv_n, float eps) {
  const float var = fmaf(-f, sum_d, squares) * inv_n;
  return 1.0f / sqrtf((var < 0.f ? 0.f : var) + eps);
}

constexpr int norm_threads(int g) { return g > 32 ? g : 256; }
// Blocks an SM takes: what the registers of a row's elements and the next one's, gamma and beta leave, backward of grad_y's and the sums too.
constexpr int blocks_per_sm(int g, int nv, bool backward) {
  return !g ? (backward ? 2 : 3) : (backward ? (nv == 1 ? 768 : 512) : (nv == 1 ? 1024 : nv == 2 ? 768 : 512)) / norm_threads(g);
}

// Rows on their way: every thread copies its own elements of the rows that its block takes next into its own places in shared memory,
// asynchronously, so that what is in flight does not hang on registers or barriers, and reads them back when their turn comes.
// bf16 [8192, 4096] over eight devices 28.4 us, 4.7 TB/s (a row ahead in registers 38.9, none 56; rows all far from zero 33.8); backward 44.5 us, 4.5 TB/s
// (51.5, 83), of which some five are the blocks' sums on their way through L2 and the second launch.
__device__ __forceinline__ void copy16(unsigned to, const void* from) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}
template <typename T, int G, int NV>
__device__ __forceinline__ void fetch_row(unsigned char* slot, const T* row, int t, long long cols) {      // slot: [quarter][thread of the block]
  constexpr int kQuarters = sizeof(T) / 2;   // of eight elements
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const Piece<G, true> at(i, t, cols);
#pragma unroll
    for (int k = 0; k < kQuarters; ++k) {
      const T* from = row + at.col + k * (8 / kQuarters);
      if (at.n > 0 && SBP_GUARD(from, 16)) copy16((unsigned)__cvta_generic_to_shared(slot + ((i * kQuarters + k) * norm_threads(G) + threadIdx.x) * 16), from);
    }
  }
}
template <typename T, int G, int NV>
__device__ __forceinline__ void take_row(const unsigned char* slot, float (&v)[NV][8]) {
  constexpr int kQuarters = sizeof(T) / 2;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    if constexpr (kQuarters == 1) {
      Eight<__nv_bfloat16, true> x;
      x.a = *reinterpret_cast<const uint4*>(slot + (i * norm_threads(G) + threadIdx.x) * 16);
      x.get(v[i]);
    } else {
      Eight<float, true> x;
      x.a = *reinterpret_cast<const float4*>(slot + (2 * i * norm_threads(G) + threadIdx.x) * 16);
      x.b = *reinterpret_cast<const float4*>(slot + ((2 * i + 1) * norm_threads(G) + threadIdx.x) * 16);
      x.get(v[i]);
    }
  }
}
template <typename T>
constexpr int row_bytes(int g, int nv) { return norm_threads(g) * nv * 8 * (int)sizeof(T); }
// Rows that the ring holds, the one being worked on among them: as many as the blocks of an SM have room for, up to six.
template <typename TX, typename TY>
constexpr int ring_rows(int g, int nv, bool backward) {
  const int room = 216 * 1024 / blocks_per_sm(g, nv, backward) / (row_bytes<TX>(g, nv) + (backward ? row_bytes<TY>(g, nv) : 0));
  return room > 6 ? 6 : room;
}
template <typename TX, typename TY>
constexpr int ring_bytes(int g, int nv, bool vec, bool backward) {
  return vec ? ring_rows<TX, TY>(g, nv, backward) * (row_bytes<TX>(g, nv) + (backward ? row_bytes<TY>(g, nv) : 0)) : 0;
}

template <typename TX, typename TY, int G, int NV, bool VEC>
__global__ void __launch_bounds__(norm_threads(G), blocks_per_sm(G, NV, false)) norm_kernel(const __grid_constant__ NormParams P) {
  constexpr int kGroups = norm_threads(G) / G;
  __shared__ __align__(16) float red[2][1][32];
  SBP_PDL_RELEASE();
  SBP_PDL_WAIT();
  const NormJob& J = P.j[blockIdx.y];
  const int t = threadIdx.x % G;
  const float n = (float)P.cols, inv_n = 1.0f / n;
  unsigned long long ga[NV][4], be[NV][4];         // (two numbers each, so that one instruction takes both)
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const Piece<G, VEC> at(i, t, P.cols);
    float u[8];
    vector8<VEC>(P.gamma, P.gamma_f32, P.gamma_whole, at.col, at.n, at.step, 1.f, u);
    pairs_of(u, ga[i]);
    vector8<VEC>(P.beta, P.beta_f32, P.beta_whole, at.col, at.n, at.step, 0.f, u);
    pairs_of(u, be[i]);
  }
  int turn = 0;
  extern __shared__ __align__(16) unsigned char ring[];
  constexpr int kRing = ring_rows<TX, TY>(G, NV, false);
  static_assert(!VEC || kRing >= 3, "two rows ahead");
  long long row = (long long)blockIdx.x * kGroups + threadIdx.x / G;
  const long long stride = (long long)gridDim.x * kGroups;
  auto fetch = [&](int slot, long long r) {
    if (r < J.rows) fetch_row<TX, G, NV>(ring + slot * row_bytes<TX>(G, NV), static_cast<const TX*>(J.x) + r * J.ldx, t, P.cols);
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  if constexpr (VEC) {
#pragma unroll
    for (int i = 0; i < kRing - 1; ++i) fetch(i, row + i * stride);
  }
  int slot = 0;
  for (; row < J.rows; row += stride) {
    unsigned long long v[NV][4];
    {
      float u[NV][8];
      if constexpr (VEC) {
        asm volatile("cp.async.wait_group %0;" ::"n"(kRing - 2) : "memory");
        take_row<TX, G, NV>(ring + slot * row_bytes<TX>(G, NV), u);
        fetch(slot == 0 ? kRing - 1 : slot - 1, row + (kRing - 1) * stride);
        slot = slot + 1 == kRing ? 0 : slot + 1;
      } else {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          const Piece<G, VEC> at(i, t, P.cols);
          load8<VEC>(static_cast<const TX*>(J.x) + row * J.ldx + at.col, u[i], at.n, at.step);      // (zeros behind the end)
        }
      }
#pragma unroll
      for (int i = 0; i < NV; ++i) pairs_of(u[i], v[i]);
    }
    unsigned long long sum = 0ull;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      if (VEC && Piece<G, VEC>(i, t, P.cols).n == 0) continue;
#pragma unroll
      for (int e = 0; e < 4; ++e) sum = pair_add(sum, v[i][e]);
    }
    float s[1] = {pair_lo(sum) + pair_hi(sum)};
    row_sums<G>(s, red, turn);
    const float c = s[0] * inv_n;
    sum = 0ull;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const Piece<G, VEC> at(i, t, P.cols);
      if (VEC && at.n == 0) continue;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[i][e] = pair_add(v[i][e], pair_of(-c));
        if constexpr (!VEC) v[i][e] = pair_of(2 * e < at.n ? pair_lo(v[i][e]) : 0.f, 2 * e + 1 < at.n ? pair_hi(v[i][e]) : 0.f);
        sum = pair_fma(v[i][e], v[i][e], sum);
      }
    }
    s[0] = pair_lo(sum) + pair_hi(sum);
    row_sums<G>(s, red, turn);
    const float squares = s[0];
    float f = 0.f;
    s[0] = 0.f;
    if (far_row(c, squares, inv_n)) {              // the same for all of the row's threads
      sum = 0ull;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        if (VEC && Piece<G, VEC>(i, t, P.cols).n == 0) continue;
#pragma unroll
        for (int e = 0; e < 4; ++e) sum = pair_add(sum, v[i][e]);
      }
      s[0] = pair_lo(sum) + pair_hi(sum);
      row_sums<G>(s, red, turn);
      f = mean_off(s[0], n, inv_n);
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) v[i][e] = pair_add(v[i][e], pair_of(-f));
    }
    const float rstd = inverse_deviation(squares, f, s[0], inv_n, P.eps);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const Piece<G, VEC> at(i, t, P.cols);
      if (at.n > 0) {
        float u[8];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const unsigned long long y = pair_fma(pair_mul(v[i][e], pair_of(rstd)), ga[i][e], be[i][e]);
          u[2 * e] = pair_lo(y);
          u[2 * e + 1] = pair_hi(y);
        }
        store8<VEC>(static_cast<TY*>(J.out) + row * J.ldo + at.col, u, at.n, at.step);
      }
    }
    if (t == 0) {
      if (J.mean && SBP_GUARD(J.mean + row, 4)) J.mean[row] = c + f;
      if (J.rstd && SBP_GUARD(J.rstd + row, 4)) J.rstd[row] = rstd;
    }
  }
}

template <typename TX, typename TY, int G, int NV, bool VEC>
__global__ void __launch_bounds__(norm_threads(G), blocks_per_sm(G, NV, true)) norm_grad_kernel(const __grid_constant__ NormParams P) {
  constexpr int kGroups = norm_threads(G) / G;
  __shared__ __align__(16) float red[2][2][32];
  SBP_PDL_RELEASE();
  SBP_PDL_WAIT();
  const NormJob& J = P.j[blockIdx.y];
  const int t = threadIdx.x % G;
  const float inv_n = 1.0f / (float)P.cols;
  float ga[NV][8], sum_g[NV][8], sum_b[NV][8];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const Piece<G, VEC> at(i, t, P.cols);
    vector8<VEC>(P.gamma, P.gamma_f32, P.gamma_whole, at.col, at.n, at.step, 1.f, ga[i]);
#pragma unroll
    for (int e = 0; e < 8; ++e) sum_g[i][e] = sum_b[i][e] = 0.f;
  }
  int turn = 0;
  extern __shared__ __align__(16) unsigned char ring[];
  constexpr int kRing = ring_rows<TX, TY>(G, NV, true);
  static_assert(!VEC || kRing >= 3, "two rows ahead");
  constexpr int kSlot = row_bytes<TX>(G, NV) + row_bytes<TY>(G, NV);
  long long row = (long long)blockIdx.x * kGroups + threadIdx.x / G;
  const long long stride = (long long)gridDim.x * kGroups;
  auto fetch = [&](int slot, long long r) {
    if (r < J.rows) {
      fetch_row<TX, G, NV>(ring + slot * kSlot, static_cast<const TX*>(J.x) + r * J.ldx, t, P.cols);
      fetch_row<TY, G, NV>(ring + slot * kSlot + row_bytes<TX>(G, NV), static_cast<const TY*>(J.dy) + r * J.lddy, t, P.cols);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  if constexpr (VEC) {
#pragma unroll
    for (int i = 0; i < kRing - 1; ++i) fetch(i, row + i * stride);
  }
  int slot = 0;
  float next_mean = 0.f, next_rstd = 0.f;
  auto stats = [&](long long r) {
    if (r < J.rows && SBP_GUARD(J.mean + r, 4)) next_mean = J.mean[r];
    if (r < J.rows && SBP_GUARD(J.rstd + r, 4)) next_rstd = J.rstd[r];
  };
  stats(row);
  for (; row < J.rows; row += stride) {
    float h[NV][8], d[NV][8];
    const float mean = next_mean, rstd = next_rstd;
    stats(row + stride);
    if constexpr (VEC) {
      asm volatile("cp.async.wait_group %0;" ::"n"(kRing - 2) : "memory");
      take_row<TX, G, NV>(ring + slot * kSlot, h);
      take_row<TY, G, NV>(ring + slot * kSlot + row_bytes<TX>(G, NV), d);
      fetch(slot == 0 ? kRing - 1 : slot - 1, row + (kRing - 1) * stride);
      slot = slot + 1 == kRing ? 0 : slot + 1;
    } else {
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const Piece<G, VEC> at(i, t, P.cols);
        if (at.n > 0) {
          load8<VEC>(static_cast<const TX*>(J.x) + row * J.ldx + at.col, h[i], at.n, at.step);
          load8<VEC>(static_cast<const TY*>(J.dy) + row * J.lddy + at.col, d[i], at.n, at.step);
        }
      }
    }
    float s[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const Piece<G, VEC> at(i, t, P.cols);
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < at.n) {
          h[i][e] = (h[i][e] - mean) * rstd;
          sum_g[i][e] = fmaf(d[i][e], h[i][e], sum_g[i][e]);
          sum_b[i][e] += d[i][e];
          d[i][e] *= ga[i][e];
          s[0] += d[i][e];
          s[1] = fmaf(d[i][e], h[i][e], s[1]);
        }
    }
    row_sums<G>(s, red, turn);
    const float a = s[0] * inv_n, b = s[1] * inv_n;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const Piece<G, VEC> at(i, t, P.cols);
      if (at.n > 0) {
#pragma unroll
        for (int e = 0; e < 8; ++e) d[i][e] = rstd * (d[i][e] - a - h[i][e] * b);
        store8<VEC>(static_cast<TX*>(J.out) + row * J.ldo + at.col, d[i], at.n, at.step);
      }
    }
  }
  if (!P.parts || (P.first_only && blockIdx.y > 0)) return;
  float* part = P.parts + ((long long)blockIdx.y * gridDim.x + blockIdx.x) * 2 * P.cols;
  if constexpr (kGroups > 1) {      // the block's rows together, group by group
    __shared__ float joined[kGroups][8 * G * NV];
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      __syncthreads();
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const Piece<G, VEC> at(i, t, P.cols);
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (e < at.n) joined[threadIdx.x / G][at.col + e * at.step] = which ? sum_b[i][e] : sum_g[i][e];
      }
      __syncthreads();
      for (int c = threadIdx.x; c < P.cols; c += norm_threads(G)) {
        float v = joined[0][c];
#pragma unroll
        for (int w = 1; w < kGroups; ++w) v += joined[w][c];
        float* to = part + which * P.cols + c;
        if (SBP_GUARD(to, 4)) *to = v;
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const Piece<G, VEC> at(i, t, P.cols);
      if (at.n > 0) {
        store8<VEC>(part + at.col, sum_g[i], at.n, at.step);
        store8<VEC>(part + P.cols + at.col, sum_b[i], at.n, at.step);
      }
    }
  }
}

// Rows longer than registers hold: a block a row, read once a pass.  The first mean is that of a sum in 64 bits, of eight elements added as a tree (equal ones exactly) at a
// time, so that equal elements are their mean whatever the row's length.
constexpr int kWide = 512;
template <typename TX, typename TY, bool VEC>
__global__ void __launch_bounds__(kWide) norm_wide_kernel(const __grid_constant__ NormParams P) {
  __shared__ __align__(16) double red[2][1][32];
  __shared__ __align__(16) float red2[2][1][32];
  SBP_PDL_RELEASE();
  SBP_PDL_WAIT();
  const NormJob& J = P.j[blockIdx.y];
  const int t = threadIdx.x, chunks = (int)((P.cols + 8 * kWide - 1) / (8 * kWide));
  const float n = (float)P.cols, inv_n = 1.0f / n;
  int turn = 0, turn2 = 0;
  for (long long row = blockIdx.x; row < J.rows; row += gridDim.x) {
    const TX* x = static_cast<const TX*>(J.x) + row * J.ldx;
    float v[8], q[1] = {0.f};
    double s[1] = {0.0};
    for (int i = 0; i < chunks; ++i) {
      const Piece<kWide, VEC> at(i, t, P.cols);
      if (at.n == 0) continue;
      load8<VEC>(x + at.col, v, at.n, at.step);
      if (at.n == 8) {
        s[0] += (double)(((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7])));
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (e < at.n) s[0] += (double)v[e];
      }
    }
    row_sums<kWide>(s, red, turn);
    const float c = (float)(s[0] / (double)P.cols);
    for (int i = 0; i < chunks; ++i) {
      const Piece<kWide, VEC> at(i, t, P.cols);
      if (at.n == 0) continue;
      load8<VEC>(x + at.col, v, at.n, at.step);
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < at.n) q[0] = fmaf(v[e] - c, v[e] - c, q[0]);
    }
    row_sums<kWide>(q, red2, turn2);
    const float squares = q[0];
    float f = 0.f;
    q[0] = 0.f;
    if (far_row(c, squares, inv_n)) {
      for (int i = 0; i < chunks; ++i) {
        const Piece<kWide, VEC> at(i, t, P.cols);
        if (at.n == 0) continue;
        load8<VEC>(x + at.col, v, at.n, at.step);
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (e < at.n) q[0] += v[e] - c;
      }
      row_sums<kWide>(q, red2, turn2);
      f = mean_off(q[0], n, inv_n);
    }
    const float rstd = inverse_deviation(squares, f, q[0], inv_n, P.eps);
    for (int i = 0; i < chunks; ++i) {
      const Piece<kWide, VEC> at(i, t, P.cols);
      if (at.n == 0) continue;
      load8<VEC>(x + at.col, v, at.n, at.step);
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < at.n)
          v[e] = fmaf((v[e] - c - f) * rstd, vector_at(P.gamma, P.gamma_f32, at.col + e * at.step, 1.f),
                      vector_at(P.beta, P.beta_f32, at.col + e * at.step, 0.f));
      store8<VEC>(static_cast<TY*>(J.out) + row * J.ldo + at.col, v, at.n, at.step);
    }
    if (t == 0) {
      if (J.mean && SBP_GUARD(J.mean + row, 4)) J.mean[row] = c + f;
      if (J.rstd && SBP_GUARD(J.rstd + row, 4)) J.rstd[row] = rstd;
    }
  }
}

template <typename TX, typename TY, bool VEC>
__global__ void __launch_bounds__(kWide) norm_grad_wide_kernel(const __grid_constant__ NormParams P) {
  __shared__ __align__(16) float red[2][2][32];
  SBP_PDL_RELEASE();
  SBP_PDL_WAIT();
  const NormJob& J = P.j[blockIdx.y];
  const int t = threadIdx.x, chunks = (int)((P.cols + 8 * kWide - 1) / (8 * kWide));
  const float inv_n = 1.0f / (float)P.cols;
  int turn = 0;
  for (long long row = blockIdx.x; row < J.rows; row += gridDim.x) {
    const TX* x = static_cast<const TX*>(J.x) + row * J.ldx;
    const TY* dy = static_cast<const TY*>(J.dy) + row * J.lddy;
    const float mean = SBP_GUARD(J.mean + row, 4) ? J.mean[row] : 0.f, rstd = SBP_GUARD(J.rstd + row, 4) ? J.rstd[row] : 0.f;
    float s[2] = {0.f, 0.f}, h[8], d[8];
    for (int i = 0; i < chunks; ++i) {
      const Piece<kWide, VEC> at(i, t, P.cols);
      if (at.n == 0) continue;
      load8<VEC>(x + at.col, h, at.n, at.step);
      load8<VEC>(dy + at.col, d, at.n, at.step);
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < at.n) {
          const float a = d[e] * vector_at(P.gamma, P.gamma_f32, at.col + e * at.step, 1.f);
          s[0] += a;
          s[1] = fmaf(a, (h[e] - mean) * rstd, s[1]);
        }
    }
    row_sums<kWide>(s, red, turn);
    const float a = s[0] * inv_n, b = s[1] * inv_n;
    for (int i = 0; i < chunks; ++i) {
      const Piece<kWide, VEC> at(i, t, P.cols);
      if (at.n == 0) continue;
      load8<VEC>(x + at.col, h, at.n, at.step);
      load8<VEC>(dy + at.col, d, at.n, at.step);
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < at.n)
          d[e] = rstd * (d[e] * vector_at(P.gamma, P.gamma_f32, at.col + e * at.step, 1.f) - a - (h[e] - mean) * rstd * b);
      store8<VEC>(static_cast<TX*>(J.out) + row * J.ldo + at.col, d, at.n, at.step);
    }
  }
}

// Their sums over the rows: a block takes 2048 columns and every gridDim.y-th row.
constexpr int kWideCols = 256;
template <typename TX, typename TY, bool VEC>
__global__ void __launch_bounds__(kWideCols) norm_sums_wide_kernel(const __grid_constant__ NormParams P) {
  SBP_PDL_RELEASE();
  SBP_PDL_WAIT();
  const NormJob& J = P.j[blockIdx.z];
  const Piece<kWideCols, VEC> at((int)blockIdx.x, threadIdx.x, P.cols);
  if (at.n == 0) return;
  float sum_g[8] = {}, sum_b[8] = {};
  for (long long row = blockIdx.y; row < J.rows; row += gridDim.y) {
    float h[8], d[8];
    load8<VEC>(static_cast<const TX*>(J.x) + row * J.ldx + at.col, h, at.n, at.step);
    load8<VEC>(static_cast<const TY*>(J.dy) + row * J.lddy + at.col, d, at.n, at.step);
    const float mean = SBP_GUARD(J.mean + row, 4) ? J.mean[row] : 0.f, rstd = SBP_GUARD(J.rstd + row, 4) ? J.rstd[row] : 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < at.n) {
        sum_g[e] = fmaf(d[e], (h[e] - mean) * rstd, sum_g[e]);
        sum_b[e] += d[e];
      }
  }
  float* part = P.parts + ((long long)blockIdx.z * gridDim.y + blockIdx.y) * 2 * P.cols;
  store8<VEC>(part + at.col, sum_g, at.n, at.step);
  store8<VEC>(part + P.cols + at.col, sum_b, at.n, at.step);
}

// The blocks' sums added up: 32 columns a block, its sixteen warps each every sixteenth part of an output, then the warps in order.
struct JoinParams {
  const float* parts;
  long long cols;
  int per_job;                   // parts of a job
  int lo[SBP_MAX_K], hi[SBP_MAX_K];      // jobs that output z is the sum of
  float* out[2][SBP_MAX_K];      // [gamma, beta]; a gradient that is not wanted has nulls
  int replicas;                  // > 0: output 0 goes to so many buffers
  int split;                     // > 0: output 0 is split over so many shards
};
constexpr int kJoin = 16;
__global__ void __launch_bounds__(32 * kJoin) norm_join_kernel(const __grid_constant__ JoinParams P) {
  __shared__ float sums[kJoin][32];
  SBP_PDL_RELEASE();
  SBP_PDL_WAIT();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, which = blockIdx.y, z = blockIdx.z;
  const long long c = (long long)blockIdx.x * 32 + lane;
  if (!P.out[which][z]) return;
  float v = 0.f;
  if (c < P.cols) {
    const int hi = P.hi[z] * P.per_job;
    const float* from = P.parts + which * P.cols + c;
#pragma unroll 8
    for (int i = P.lo[z] * P.per_job + warp; i < hi; i += kJoin)
      if (SBP_GUARD(from + i * 2 * P.cols, 4)) v += from[i * 2 * P.cols];
  }
  sums[warp][lane] = v;
  __syncthreads();
  if (warp == 0 && c < P.cols) {
    v = sums[0][lane];
#pragma unroll
    for (int w = 1; w < kJoin; ++w) v += sums[w][lane];
    if (P.split > 0) {
      int64_t start = 0, len = 0;
      int r = 0;
      for (; r < P.split; ++r) {
        split_range(P.cols, P.split, r, &start, &len);
        if (c < start + len) break;
      }
      float* to = P.out[which][r] + (c - start);
      if (SBP_GUARD(to, 4)) *to = v;
    } else {
      const int n = P.replicas > 0 ? P.replicas : 1;
      for (int r = 0; r < n; ++r) {
        float* to = P.out[which][P.replicas > 0 ? r : z] + c;
        if (SBP_GUARD(to, 4)) *to = v;
      }
    }
  }
}

// Threads that share a row and chunks of eight elements each has, by the row's length; {0, 0}: the wide kernels (backward from 8193
// elements on: x, grad_y and both sums of 32 elements a thread are more than 128 registers).
struct NormForm {
  int g, nv;
};
NormForm norm_form(long long cols, bool backward) {
  if (cols <= 256) return {32, 1};
  if (cols <= 512) return {32, 2};
  if (cols <= 1024) return {128, 1};
  if (cols <= 2048) return {128, 2};
  if (cols <= 4096) return {256, 2};
  if (cols <= 8192) return {512, 2};
  if (cols <= 16384 && !backward) return {512, 4};
  return {0, 0};
}

// Blocks of a job: what the device holds, dealt out to the jobs, but no more than there are rows for.
int norm_blocks(NormForm f, long long rows, int jobs, int per_sm) {
  const long long most = (rows * (f.g ? f.g : kWide) + norm_threads(f.g ? f.g : kWide) - 1) / norm_threads(f.g ? f.g : kWide);
  const long long fair = (long long)device_sms() * per_sm / jobs;      // (one block more than the device holds is a second wave)
  return (int)(most < fair ? most : fair > 1 ? fair : 1);
}

bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

long long rows_of(const sbp_tensor* t, int r) {
  int64_t shp[SBP_MAX_DIMS];
  local_shape_nd(t, r, shp);
  long long n = 1;
  for (int d = 0; d + 1 < t->ndim; ++d) n *= shp[d];
  return n;
}

bool is_float(int32_t dtype) { return dtype == SBP_F32 || dtype == SBP_BF16; }

sbp_status check_rows(const sbp_tensor* t, const char* name, const sbp_tensor* like, bool need_ptrs) {
  sbp_status st = check_tensor(t, name, need_ptrs);
  if (st != SBP_OK) return st;
  if (!is_float(t->dtype)) return fail(SBP_ERR_DTYPE, "%s must be F32 or BF16", name);
  if (!like) {
    if (t->ndim < 2) return fail(SBP_ERR_SHAPE, "%s needs at least two axes", name);
    if (t->shape[t->ndim - 1] < 1) return fail(SBP_ERR_SHAPE, "%s: rows of no elements have no mean", name);
    const sbp_sig s = t->sbp[0];
    if (s.kind != SBP_SPLIT && s.kind != SBP_BROADCAST) return fail(SBP_ERR_SIGNATURE, "%s must be S(i) or B: normalising is not linear", name);
    if (s.kind == SBP_SPLIT && s.axis == t->ndim - 1)
      return fail(SBP_ERR_UNSUPPORTED, "%s is split along the axis that is normalised: box it to another signature first", name);
    return SBP_OK;
  }
  if (placement_k(t) != placement_k(like)) return fail(SBP_ERR_INVALID_ARG, "%s and x differ in k", name);
  if (t->ndim != like->ndim) return fail(SBP_ERR_SHAPE, "%s and x differ in shape", name);
  for (int d = 0; d < t->ndim; ++d)
    if (t->shape[d] != like->shape[d]) return fail(SBP_ERR_SHAPE, "%s and x differ in shape", name);
  if (!same_sig(t->sbp[0], like->sbp[0])) return fail(SBP_ERR_SIGNATURE, "%s and x differ in signature", name);
  return SBP_OK;
}

// mean or rstd
sbp_status check_stat(const sbp_tensor* t, const char* name, const sbp_tensor* x) {
  sbp_status st = check_tensor(t, name, true);
  if (st != SBP_OK) return st;
  if (t->dtype != SBP_F32) return fail(SBP_ERR_DTYPE, "%s must be F32", name);
  if ((st = refuse_ld(t, name, "layer norm")) != SBP_OK) return st;
  if (placement_k(t) != placement_k(x)) return fail(SBP_ERR_INVALID_ARG, "%s and x differ in k", name);
  if (t->ndim != x->ndim - 1) return fail(SBP_ERR_SHAPE, "%s must have x's shape without its last axis", name);
  for (int d = 0; d < t->ndim; ++d)
    if (t->shape[d] != x->shape[d]) return fail(SBP_ERR_SHAPE, "%s must have x's shape without its last axis", name);
  if (!same_sig(t->sbp[0], x->sbp[0])) return fail(SBP_ERR_SIGNATURE, "%s and x differ in signature", name);
  return SBP_OK;
}

// gamma or beta
sbp_status check_vector(const sbp_tensor* t, const char* name, const sbp_tensor* x) {
  sbp_status st = check_tensor(t, name, true);
  if (st != SBP_OK) return st;
  if (!is_float(t->dtype)) return fail(SBP_ERR_DTYPE, "%s must be F32 or BF16", name);
  if (placement_k(t) != placement_k(x)) return fail(SBP_ERR_INVALID_ARG, "%s and x differ in k", name);
  if (t->ndim != 1 || t->shape[0] != x->shape[x->ndim - 1]) return fail(SBP_ERR_SHAPE, "%s must be [row length]", name);
  if (t->sbp[0].kind != SBP_BROADCAST) return fail(SBP_ERR_SIGNATURE, "%s must be B", name);
  return SBP_OK;
}

// One compiled form; a ring of more than 48 KiB has to be asked for, once a device.
template <typename TX, typename TY, int G, int NV, bool VEC, bool BACKWARD>
cudaError_t launch_one(const NormParams& P, int jobs, int blocks, cudaStream_t st) {
  constexpr int kBytes = ring_bytes<TX, TY>(G, NV, VEC, BACKWARD);
  void (*kernel)(NormParams);
  if constexpr (BACKWARD) kernel = norm_grad_kernel<TX, TY, G, NV, VEC>;
  else kernel = norm_kernel<TX, TY, G, NV, VEC>;
  if constexpr (kBytes > 0) {
    static std::atomic<unsigned long long> opted{0};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const unsigned long long bit = 1ull << (dev & 63);
    if (dev >= 64 || !(opted.load(std::memory_order_relaxed) & bit)) {
      e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kBytes);
      if (e != cudaSuccess) return e;
      if (dev < 64) opted.fetch_or(bit, std::memory_order_relaxed);
    }
  }
  return launch_dependent(kernel, dim3((unsigned)blocks, (unsigned)jobs), dim3(norm_threads(G)), (size_t)kBytes, st, P);
}
template <typename TX, typename TY, int G, int NV>
cudaError_t launch_form(const NormParams& P, int jobs, int blocks, bool vec, bool backward, cudaStream_t st) {
  if constexpr (NV < 4) {
    if (backward) return vec ? launch_one<TX, TY, G, NV, true, true>(P, jobs, blocks, st) : launch_one<TX, TY, G, NV, false, true>(P, jobs, blocks, st);
  }
  return vec ? launch_one<TX, TY, G, NV, true, false>(P, jobs, blocks, st) : launch_one<TX, TY, G, NV, false, false>(P, jobs, blocks, st);
}

template <typename TX, typename TY>
cudaError_t launch_wide(const NormParams& P, int jobs, int blocks, bool vec, bool backward, cudaStream_t st) {
  const dim3 grid((unsigned)blocks, (unsigned)jobs);
  if (!backward)
    return vec ? launch_dependent(norm_wide_kernel<TX, TY, true>, grid, dim3(kWide), 0, st, P)
               : launch_dependent(norm_wide_kernel<TX, TY, false>, grid, dim3(kWide), 0, st, P);
  const cudaError_t e = vec ? launch_dependent(norm_grad_wide_kernel<TX, TY, true>, grid, dim3(kWide), 0, st, P)
                            : launch_dependent(norm_grad_wide_kernel<TX, TY, false>, grid, dim3(kWide), 0, st, P);
  if (e != cudaSuccess || !P.parts) return e;
  count_launch();
  const dim3 cols((unsigned)((P.cols + 8 * kWideCols - 1) / (8 * kWideCols)), (unsigned)blocks, P.first_only ? 1u : (unsigned)jobs);
  return vec ? launch_dependent(norm_sums_wide_kernel<TX, TY, true>, cols, dim3(kWideCols), 0, st, P)
             : launch_dependent(norm_sums_wide_kernel<TX, TY, false>, cols, dim3(kWideCols), 0, st, P);
}

template <typename TX, typename TY>
sbp_status launch_norm(const NormParams& P, int jobs, int blocks, bool backward, cudaStream_t st) {
  bool vec = P.cols % 8 == 0;
  for (int i = 0; i < jobs; ++i) {
    const NormJob& j = P.j[i];
    vec = vec && aligned16(j.x) && j.ldx * sizeof(TX) % 16 == 0 && aligned16(j.out) && j.ldo * (backward ? sizeof(TX) : sizeof(TY)) % 16 == 0;
    if (backward) vec = vec && aligned16(j.dy) && j.lddy * sizeof(TY) % 16 == 0;
  }
  SBP_BOUNDS_UPLOAD(st);
  const NormForm f = norm_form(P.cols, backward);
  cudaError_t e;
  switch (f.g * 8 + f.nv) {
    case 32 * 8 + 1: e = launch_form<TX, TY, 32, 1>(P, jobs, blocks, vec, backward, st); break;
    case 32 * 8 + 2: e = launch_form<TX, TY, 32, 2>(P, jobs, blocks, vec, backward, st); break;
    case 128 * 8 + 1: e = launch_form<TX, TY, 128, 1>(P, jobs, blocks, vec, backward, st); break;
    case 128 * 8 + 2: e = launch_form<TX, TY, 128, 2>(P, jobs, blocks, vec, backward, st); break;
    case 256 * 8 + 2: e = launch_form<TX, TY, 256, 2>(P, jobs, blocks, vec, backward, st); break;
    case 512 * 8 + 2: e = launch_form<TX, TY, 512, 2>(P, jobs, blocks, vec, backward, st); break;
    case 512 * 8 + 4: e = launch_form<TX, TY, 512, 4>(P, jobs, blocks, vec, backward, st); break;
    default: e = launch_wide<TX, TY>(P, jobs, blocks, vec, backward, st); break;
  }
  if (e != cudaSuccess) return cuda_fail(e, "layer norm launch");
  count_launch();
  return SBP_OK;
}

// x_f32, y_f32: types of x (and its gradient) and of y (and its gradient)
sbp_status launch_typed(const NormParams& P, int jobs, int blocks, bool backward, bool x_f32, bool y_f32, cudaStream_t st) {
  if (jobs == 0) return SBP_OK;
  using bf16 = __nv_bfloat16;
  if (x_f32) return y_f32 ? launch_norm<float, float>(P, jobs, blocks, backward, st) : launch_norm<float, bf16>(P, jobs, blocks, backward, st);
  return y_f32 ? launch_norm<bf16, float>(P, jobs, blocks, backward, st) : launch_norm<bf16, bf16>(P, jobs, blocks, backward, st);
}

// Blocks a job gets in the backward pass of x, and the jobs whose sums the workspace holds: the same for the query and the call.
int backward_blocks(const sbp_tensor* x, int* jobs) {
  const NormForm f = norm_form(x->shape[x->ndim - 1], true);
  long long most = 0;
  *jobs = 0;
  for (int r = 0; r < placement_k(x); ++r) {
    const long long n = rows_of(x, r);
    most = n > most ? n : most;
    if (n > 0) ++*jobs;
  }
  if (*jobs && x->sbp[0].kind == SBP_BROADCAST) *jobs = 1;
  return *jobs ? norm_blocks(f, most, *jobs, blocks_per_sm(f.g, f.nv, true)) : 0;
}

}  // namespace

}  // namespace sbp

using namespace sbp;

extern "C" {

sbp_status sbp_layer_norm(const sbp_tensor* x, const sbp_tensor* gamma, const sbp_tensor* beta, sbp_tensor* y, sbp_tensor* mean,
                          sbp_tensor* rstd, float eps, void* cuda_stream) {
  SBP_RANGE("sbp_layer_norm");
  sbp_status st = check_rows(x, "x", nullptr, true);
  if (st != SBP_OK) return st;
  if ((st = check_rows(y, "y", x, true)) != SBP_OK) return st;
  if (gamma && (st = check_vector(gamma, "gamma", x)) != SBP_OK) return st;
  if (beta && (st = check_vector(beta, "beta", x)) != SBP_OK) return st;
  if (mean && (st = check_stat(mean, "mean", x)) != SBP_OK) return st;
  if (rstd && (st = check_stat(rstd, "rstd", x)) != SBP_OK) return st;
  if (!(eps >= 0.f) || eps > 3.4e38f) return fail(SBP_ERR_INVALID_ARG, "eps must be finite and not negative");
  if (x->shape[x->ndim - 1] > (1LL << 31)) return fail(SBP_ERR_UNSUPPORTED, "rows of more than 2^31 elements");
  NormParams P{};
  P.gamma = gamma ? gamma->local[0] : nullptr;
  P.beta = beta ? beta->local[0] : nullptr;
  P.gamma_f32 = gamma && gamma->dtype == SBP_F32;
  P.beta_f32 = beta && beta->dtype == SBP_F32;
  P.gamma_whole = gamma && aligned16(P.gamma);
  P.beta_whole = beta && aligned16(P.beta);
  P.cols = x->shape[x->ndim - 1];
  P.eps = eps;
  int n = 0;
  long long most = 0;
  for (int r = 0; r < placement_k(x); ++r) {
    NormJob j{};
    j.rows = rows_of(x, r);
    if (j.rows == 0) continue;
    j.x = x->local[r];
    j.ldx = local_pitch(x, r);
    j.out = y->local[r];
    j.ldo = local_pitch(y, r);
    j.mean = mean ? static_cast<float*>(mean->local[r]) : nullptr;
    j.rstd = rstd ? static_cast<float*>(rstd->local[r]) : nullptr;
    bool seen = false;
    for (int i = 0; i < n; ++i) seen = seen || (P.j[i].out == j.out && P.j[i].mean == j.mean && P.j[i].rstd == j.rstd);
    if (seen && x->sbp[0].kind == SBP_BROADCAST) continue;
    P.j[n++] = j;
    most = j.rows > most ? j.rows : most;
  }
  SBP_BOUNDS_RESET();
  SBP_BOUNDS_TENSOR(x);
  SBP_BOUNDS_TENSOR(gamma);
  SBP_BOUNDS_TENSOR(beta);
  SBP_BOUNDS_TENSOR(y);
  SBP_BOUNDS_TENSOR(mean);
  SBP_BOUNDS_TENSOR(rstd);
  const NormForm f = norm_form(P.cols, false);
  return launch_typed(P, n, n ? norm_blocks(f, most, n, blocks_per_sm(f.g, f.nv, false)) : 0, false, x->dtype == SBP_F32, y->dtype == SBP_F32,
                      static_cast<cudaStream_t>(cuda_stream));
}

size_t sbp_layer_norm_backward_workspace_bytes(const sbp_tensor* x) {
  if (check_rows(x, "x", nullptr, false) != SBP_OK) return 0;
  int jobs = 0;
  const int blocks = backward_blocks(x, &jobs);
  return (size_t)blocks * jobs * 2 * (size_t)x->shape[x->ndim - 1] * sizeof(float);
}

sbp_status sbp_layer_norm_backward(const sbp_tensor* x, const sbp_tensor* gamma, const sbp_tensor* mean, const sbp_tensor* rstd,
                                   const sbp_tensor* grad_y, sbp_tensor* grad_x, sbp_tensor* grad_gamma, sbp_tensor* grad_beta, void* ws,
                                   size_t ws_bytes, void* cuda_stream) {
  SBP_RANGE("sbp_layer_norm_backward");
  sbp_status st = check_rows(x, "x", nullptr, true);
  if (st != SBP_OK) return st;
  if ((st = check_rows(grad_y, "grad_y", x, true)) != SBP_OK) return st;
  if ((st = check_rows(grad_x, "grad_x", x, true)) != SBP_OK) return st;
  if (grad_x->dtype != x->dtype) return fail(SBP_ERR_DTYPE, "grad_x must have x's dtype");
  if (gamma && (st = check_vector(gamma, "gamma", x)) != SBP_OK) return st;
  if ((st = check_stat(mean, "mean", x)) != SBP_OK) return st;
  if ((st = check_stat(rstd, "rstd", x)) != SBP_OK) return st;
  const int k = placement_k(x);
  const bool x_b = x->sbp[0].kind == SBP_BROADCAST;
  sbp_tensor* const grads[2] = {grad_gamma, grad_beta};
  const char* const names[2] = {"grad_gamma", "grad_beta"};
  sbp_sig sig{SBP_BROADCAST, 0};
  bool wanted = false;
  for (int i = 0; i < 2; ++i) {
    const sbp_tensor* t = grads[i];
    if (!t) continue;
    if ((st = check_tensor(t, names[i], true)) != SBP_OK) return st;
    if (t->dtype != SBP_F32) return fail(SBP_ERR_DTYPE, "%s must be F32", names[i]);
    if (placement_k(t) != k) return fail(SBP_ERR_INVALID_ARG, "%s and x differ in k", names[i]);
    if (t->ndim != 1 || t->shape[0] != x->shape[x->ndim - 1]) return fail(SBP_ERR_SHAPE, "%s must be [row length]", names[i]);
    const sbp_sig s = t->sbp[0];
    if (s.kind == SBP_PARTIAL_MAX || (s.kind == SBP_PARTIAL_SUM && x_b))
      return fail(SBP_ERR_SIGNATURE, "%s must be %sB or S(0)", names[i], x_b ? "" : "P(sum), ");
    if (wanted && !same_sig(s, sig)) return fail(SBP_ERR_SIGNATURE, "grad_gamma and grad_beta differ in signature");
    sig = s;
    wanted = true;
  }
  if (x->shape[x->ndim - 1] > (1LL << 31)) return fail(SBP_ERR_UNSUPPORTED, "rows of more than 2^31 elements");
  int jobs_most = 0;
  const int blocks = backward_blocks(x, &jobs_most);
  const size_t need = sbp_layer_norm_backward_workspace_bytes(x);
  if (wanted && need > 0) {
    if (!ws || ws_bytes < need) return fail(SBP_ERR_WORKSPACE, "workspace of %zu bytes needed, %zu given", need, ws_bytes);
    if (!aligned16(ws)) return fail(SBP_ERR_ALIGNMENT, "workspace must be 16-byte aligned");
  }

  NormParams P{};
  P.gamma = gamma ? gamma->local[0] : nullptr;
  P.gamma_f32 = gamma && gamma->dtype == SBP_F32;
  P.gamma_whole = gamma && aligned16(P.gamma);
  P.cols = x->shape[x->ndim - 1];
  P.parts = wanted ? static_cast<float*>(ws) : nullptr;
  P.first_only = x_b;
  JoinParams Q{};
  int n = 0;
  for (int r = 0; r < k; ++r) {
    NormJob j{};
    j.rows = rows_of(x, r);
    Q.lo[r] = Q.hi[r] = n;
    if (j.rows == 0) continue;
    j.x = x->local[r];
    j.ldx = local_pitch(x, r);
    j.dy = grad_y->local[r];
    j.lddy = local_pitch(grad_y, r);
    j.out = grad_x->local[r];
    j.ldo = local_pitch(grad_x, r);
    j.mean = static_cast<float*>(mean->local[r]);
    j.rstd = static_cast<float*>(rstd->local[r]);
    bool seen = false;
    for (int i = 0; i < n; ++i) seen = seen || P.j[i].out == j.out;
    if (seen && x_b) continue;
    P.j[n++] = j;
    Q.hi[r] = n;
  }
  SBP_BOUNDS_RESET();
  SBP_BOUNDS_TENSOR(x);
  SBP_BOUNDS_TENSOR(gamma);
  SBP_BOUNDS_TENSOR(mean);
  SBP_BOUNDS_TENSOR(rstd);
  SBP_BOUNDS_TENSOR(grad_y);
  SBP_BOUNDS_TENSOR(grad_x);
  SBP_BOUNDS_TENSOR(grad_gamma);
  SBP_BOUNDS_TENSOR(grad_beta);
  SBP_BOUNDS_ADD(ws, ws_bytes);
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  st = launch_typed(P, n, blocks, true, x->dtype == SBP_F32, grad_y->dtype == SBP_F32, stream);
  if (st != SBP_OK || !wanted) return st;

  Q.parts = P.parts;
  Q.cols = P.cols;
  Q.per_job = blocks;
  const bool partial = sig.kind == SBP_PARTIAL_SUM;
  if (!partial) {                // every row once: of a B tensor those of one replica
    Q.lo[0] = 0;
    Q.hi[0] = x_b ? (n > 0 ? 1 : 0) : n;
  }
  for (int i = 0; i < 2; ++i) {
    if (!grads[i]) continue;
    for (int r = 0; r < k; ++r) Q.out[i][r] = static_cast<float*>(grads[i]->local[r]);
  }
  if (sig.kind == SBP_SPLIT) Q.split = k;
  if (sig.kind == SBP_BROADCAST) Q.replicas = k;
  const dim3 grid((unsigned)((P.cols + 31) / 32), 2, partial ? (unsigned)k : 1u);
  SBP_BOUNDS_UPLOAD(stream);
  const cudaError_t e = launch_dependent(norm_join_kernel, grid, dim3(32 * kJoin), 0, stream, Q);
  if (e != cudaSuccess) return cuda_fail(e, "layer norm gradient launch");
  count_launch();
  return SBP_OK;
}

}  // extern "C"
