// 8-bit blocks: quantisation (as stored, transposed, a scale a tile) and GeLU that keeps its input in them, with its gradient.
//
// Bound: DRAM.  bf16 in, one byte out (and the four bytes of a scale a block): 3 bytes an element, 5 with GeLU's result or with the
// gradients.  Right behind it the instructions: 8.7 an element to quantise along rows, 22.1 with GeLU, 22.7 for its gradient (62, 69 and 76 % of the
// issue slots).
// Measured: bf16 [8192, 4096] quantised 17 us, 5.9 TB/s; [4096, 16384] by tiles, transposed 38 us, 5.3 TB/s; GeLU of [8192, 16384] 136 us, 5.0 TB/s, and its
// gradient 134 us.  [8192, 8192]: tiles as stored 37 us, transposed with a scale a column 45 us.
#include <type_traits>

#include "blocks8.h"

namespace sbp {

namespace {

// What one local tensor's kernel blocks need; x is the input (z, grad_y), y the other 16- or 32-bit tensor where there is one.
struct Job8 {
  const void* x;
  void* y;
  unsigned char* q;
  float* s;
  long long rows, cols, ldx, ldy, ldq, lds;      // extents of x
};
struct Jobs8 {
  Job8 j[SBP_MAX_K];
  int per_row_log;      // teams of eight lanes side by side along a row, log2 (row kernel)
  int wide;             // 16-byte stores of values
};

enum { kQuantize = 0, kGelu = 1, kGeluGrad = 2 };
constexpr int rows_at_once(bool vec) { return vec ? 2 : 1; }      // rows a team has in flight

// Blocks of 128 along the rows: a team of eight lanes a block, 16 elements a lane, two rows in flight (one where elements are loaded one by one:
// the code of two, fetched for a small tensor once, costs more than it hides: fp32 [1021, 1537] 6.4 and 4.7 us).  Eight elements a lane, 16 lanes a block:
// quantising [8192, 4096] 20.7 us, what is paid by lane and row being most of the instructions.
template <typename TX, typename TY, int OP, bool VEC>
__global__ void __launch_bounds__(256, VEC && sizeof(TX) == 2 ? 4 : 3) blocks8_row_kernel(const __grid_constant__ Jobs8 P) {
  SBP_PDL_RELEASE();
  SBP_PDL_WAIT();
  constexpr int kRowsAtOnce = rows_at_once(VEC);
  const Job8& J = P.j[blockIdx.z];
  const int team = threadIdx.x >> 3, l = threadIdx.x & 7;
  const long long block = ((long long)blockIdx.y << P.per_row_log) + (team & ((1 << P.per_row_log) - 1));
  const int rows_cta = 32 >> P.per_row_log;      // rows a pass of the CTA covers
  const long long row0 = (long long)blockIdx.x * (rows_cta * kRowsAtOnce) + (team >> P.per_row_log);
  const long long first = block * kBlock8;
  const int have = first < J.cols ? (int)min((long long)kBlock8, J.cols - first) : 0;
  const int rows = (int)min((long long)(rows_cta * kRowsAtOnce), max(0LL, J.rows - row0));      // from this lane's first one on
  // VEC: a lane's 16 elements follow one another, eight are all inside or all outside; else lanes take every eighth
  constexpr int kStep = VEC ? 1 : 8, kNext = VEC ? 8 : 64;      // from one element to the next, from the first eight to the others
  const int at = VEC ? l * 16 : l;
  int n[2];
#pragma unroll
  for (int k = 0; k < 2; ++k) n[k] = VEC ? (at + 8 * k < have ? 8 : 0) : min(8, max(0, (have - at - 64 * k + 7) >> 3));
  const long long col = first + at;
  const TX* px = static_cast<const TX*>(J.x) + row0 * J.ldx + col;
  unsigned char* pq = J.q + row0 * J.ldq + col;
  TY* py = static_cast<TY*>(J.y) + (OP == kQuantize ? 0 : row0 * J.ldy + col);
  float* ps = J.s + row0 * J.lds + block;
  const long long hop_x = rows_cta * J.ldx, hop_q = rows_cta * J.ldq, hop_y = rows_cta * J.ldy, hop_s = rows_cta * J.lds;
  Eight<TX, VEC> x[kRowsAtOnce][2];
#pragma unroll
  for (int i = 0; i < kRowsAtOnce; ++i)
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      x[i][k].clear();
      if (i * rows_cta < rows && n[k] > 0) x[i][k].load(px + i * hop_x + k * kNext, n[k], kStep);
    }
  if constexpr (OP == kGeluGrad) {
    uint2 q[kRowsAtOnce][2];
    float s[kRowsAtOnce];
#pragma unroll
    for (int i = 0; i < kRowsAtOnce; ++i) {
      const bool in = i * rows_cta < rows && n[0] > 0;
      const unsigned char* src = pq + i * hop_q;
      s[i] = in && SBP_GUARD(ps + i * hop_s, 4) ? ps[i * hop_s] : 0.f;
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        q[i][k] = make_uint2(0u, 0u);
        if constexpr (VEC) {
          if (in && n[k] > 0 && SBP_GUARD(src + 8 * k, 8)) q[i][k] = *reinterpret_cast<const uint2*>(src + 8 * k);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (in && e < n[k] && SBP_GUARD(src + k * kNext + e * kStep, 1)) (e < 4 ? q[i][k].x : q[i][k].y) |= (unsigned)src[k * kNext + e * kStep] << (8 * (e & 3));
        }
      }
    }
#pragma unroll
    for (int i = 0; i < kRowsAtOnce; ++i)
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        if (i * rows_cta >= rows || n[k] == 0) continue;
        float v[8];
        x[i][k].get(v);
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
          float a, b;
          two_of_e4m3((e < 4 ? q[i][k].x : q[i][k].y) >> (8 * (e & 3)) & 0xffffu, a, b);
          const unsigned long long z = pair_mul(pair_of(a, b), pair_of(s[i]));
          a = pair_lo(z);
          b = pair_hi(z);
          gelu_slope_two(a, b);
          const unsigned long long w = pair_mul(pair_of(v[e], v[e + 1]), pair_of(a, b));
          v[e] = pair_lo(w);
          v[e + 1] = pair_hi(w);
        }
        store8<VEC>(py + i * hop_y + k * kNext, v, n[k], kStep);
      }
  } else {
#pragma unroll
    for (int i = 0; i < kRowsAtOnce; ++i) {
      unsigned m = max(largest_bits(x[i][0]), largest_bits(x[i][1]));
#pragma unroll
      for (int d = 1; d < 8; d <<= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, d));
      const bool fix = __any_sync(0xffffffffu, m >= 0x7f800000u);      // something is not finite: the maximum of the others
      if (fix) {
        m = 0;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          float c[8];
          x[i][k].get(c);
#pragma unroll
          for (int e = 0; e < 8; ++e) m = max(m, finite_bits(c[e]));
        }
#pragma unroll
        for (int d = 1; d < 8; d <<= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, d));
      }
      if (i * rows_cta >= rows || n[0] == 0) continue;
      const unsigned sb = scale_bits(m);
      const float inv = __uint_as_float(kInvBits - sb);
      uint2 out[2];
      auto convert = [&](auto fix_tag) {
        constexpr bool FIX = decltype(fix_tag)::value;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          float c[8], w[8];
          x[i][k].get(c);
#pragma unroll
          for (int e = 0; e < 8; e += 2) {
            const unsigned long long v = pair_mul(FIX ? pair_of(inf_to_nan(c[e]), inf_to_nan(c[e + 1])) : pair_of(c[e], c[e + 1]), pair_of(inv));
            w[e] = pair_lo(v);
            w[e + 1] = pair_hi(v);
          }
          out[k] = make_uint2(e4m3_four(w), e4m3_four(w + 4));
          if constexpr (OP == kGelu) {
            if (n[k] == 0) continue;
#pragma unroll
            for (int e = 0; e < 8; e += 2) gelu_two<sizeof(TX) == 4, !FIX && sizeof(TX) == 2>(c[e], c[e + 1]);
            store8<VEC>(py + i * hop_y + k * kNext, c, n[k], kStep);
          }
        }
      };
      if (fix) convert(std::true_type{});
      else convert(std::false_type{});
      unsigned char* dst = pq + i * hop_q;
      if constexpr (VEC) {
        if (P.wide) {
          if (SBP_GUARD(dst, 16)) *reinterpret_cast<uint4*>(dst) = make_uint4(out[0].x, out[0].y, out[1].x, out[1].y);
        } else {
#pragma unroll
          for (int k = 0; k < 2; ++k)
            if (n[k] > 0 && SBP_GUARD(dst + 8 * k, 8)) *reinterpret_cast<uint2*>(dst + 8 * k) = out[k];
        }
      } else {
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (e < n[k] && SBP_GUARD(dst + k * kNext + e * kStep, 1)) dst[k * kNext + e * kStep] = (unsigned char)((e < 4 ? out[k].x : out[k].y) >> (8 * (e & 3)));
      }
      if (l == 0 && SBP_GUARD(ps + i * hop_s, 4)) ps[i * hop_s] = __uint_as_float(sb);
    }
  }
}

// Tiles of 128 x 128, and what is written transposed: a CTA a tile of x, in registers.  A thread holds four consecutive rows of
// two groups of eight columns, so that a transposed row's four values are one word of shared memory.
// TRANS without TILES: a scale for each column of the tile.
constexpr int kPitch8 = 33;                  // words of a transposed row in shared memory
template <typename TX, bool TILES, bool TRANS, bool VEC>
__global__ void __launch_bounds__(256, VEC && sizeof(TX) == 2 ? 3 : 2) blocks8_tile_kernel(const __grid_constant__ Jobs8 P) {
  __shared__ unsigned words[TRANS ? kBlock8 * kPitch8 : 1];
  constexpr bool kPacked = VEC && sizeof(TX) == 2;      // magnitudes of bf16 numbers, two to a word
  __shared__ __align__(16) unsigned amax[8][TILES ? 1 : kPacked ? kBlock8 / 2 : kBlock8];      // by warp (and column)
  __shared__ __align__(16) float inv_of[TILES ? 4 : kBlock8];
  SBP_PDL_RELEASE();
  SBP_PDL_WAIT();
  const Job8& J = P.j[blockIdx.z];
  const long long r0 = (long long)blockIdx.x * kBlock8, c0 = (long long)blockIdx.y * kBlock8;
  if (r0 >= J.rows || c0 >= J.cols) return;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int cg = lane & 7, rq = warp * 4 + (lane >> 3);
  const int rows = (int)min((long long)kBlock8, J.rows - r0), cols = (int)min((long long)kBlock8, J.cols - c0);
  Eight<TX, VEC> x[2][4];
#pragma unroll
  for (int g = 0; g < 2; ++g)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = rq * 4 + i, c = g * 64 + cg * 8, n = r < rows ? min(8, cols - c) : 0;
      x[g][i].clear();
      if (n > 0) x[g][i].load(static_cast<const TX*>(J.x) + (r0 + r) * J.ldx + c0 + c, n, 1);
    }
  // The scale of the tile (of every column).  First the largest magnitude of all; where that is not finite, of what is.
  float inv = 0.f;
  bool fix = false;
  if constexpr (TILES) {
    unsigned m = 0;
#pragma unroll
    for (int g = 0; g < 2; ++g)
#pragma unroll
      for (int i = 0; i < 4; ++i) m = max(m, largest_bits(x[g][i]));
    fix = __syncthreads_or(m >= 0x7f800000u);
    if (fix) {
      m = 0;
#pragma unroll
      for (int g = 0; g < 2; ++g)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float v[8];
          x[g][i].get(v);
#pragma unroll
          for (int e = 0; e < 8; ++e) m = max(m, finite_bits(v[e]));
        }
    }
    m = __reduce_max_sync(0xffffffffu, m);
    if (lane == 0) amax[warp][0] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 8; ++w) m = max(m, amax[w][0]);
    const unsigned sb = scale_bits(m);
    inv = __uint_as_float(kInvBits - sb);
    if (threadIdx.x == 0) {
      float* sp = J.s + (TRANS ? (long long)blockIdx.y * J.lds + blockIdx.x : (long long)blockIdx.x * J.lds + blockIdx.y);
      if (SBP_GUARD(sp, 4)) *sp = __uint_as_float(sb);
    }
  } else {
    auto columns = [&](bool finite_only) {
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        constexpr int kWords = kPacked ? 4 : 8;
        unsigned m[kWords] = {};
        if constexpr (kPacked) {
          auto pairs = [&](int i, int w) {       // magnitudes of two columns
            const uint4& a = x[g][i].a;
            unsigned v = (w == 0 ? a.x : w == 1 ? a.y : w == 2 ? a.z : a.w) & 0x7fff7fffu;
            if (finite_only) {
              if ((v & 0x7f80u) == 0x7f80u) v &= 0xffff0000u;
              if ((v & 0x7f800000u) == 0x7f800000u) v &= 0xffffu;
            }
            return v;
          };
#pragma unroll
          for (int w = 0; w < 4; ++w) m[w] = __vmaxs2(__vimax3_s16x2(pairs(0, w), pairs(1, w), pairs(2, w)), pairs(3, w));
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            m[w] = __vmaxs2(m[w], __shfl_xor_sync(0xffffffffu, m[w], 8));
            m[w] = __vmaxs2(m[w], __shfl_xor_sync(0xffffffffu, m[w], 16));
          }
          if (lane < 8) *reinterpret_cast<uint4*>(&amax[warp][g * 32 + cg * 4]) = make_uint4(m[0], m[1], m[2], m[3]);
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float v[8];
            x[g][i].get(v);
#pragma unroll
            for (int e = 0; e < 8; ++e) m[e] = max(m[e], finite_only ? finite_bits(v[e]) : __float_as_uint(v[e]) & 0x7fffffffu);
          }
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            m[e] = max(m[e], __shfl_xor_sync(0xffffffffu, m[e], 8));
            m[e] = max(m[e], __shfl_xor_sync(0xffffffffu, m[e], 16));
          }
          if (lane < 8) {
            *reinterpret_cast<uint4*>(&amax[warp][g * 64 + cg * 8]) = make_uint4(m[0], m[1], m[2], m[3]);
            *reinterpret_cast<uint4*>(&amax[warp][g * 64 + cg * 8 + 4]) = make_uint4(m[4], m[5], m[6], m[7]);
          }
        }
      }
      __syncthreads();
      unsigned m = 0;
      if (threadIdx.x < kBlock8) {
#pragma unroll
        for (int w = 0; w < 8; ++w) {
          if constexpr (kPacked) m = max(m, (amax[w][threadIdx.x >> 1] >> (16 * (threadIdx.x & 1)) & 0xffffu) << 16);
          else m = max(m, amax[w][threadIdx.x]);
        }
        const unsigned sb = scale_bits(m);
        inv_of[threadIdx.x] = __uint_as_float(kInvBits - sb);
        float* sp = J.s + (c0 + threadIdx.x) * J.lds + blockIdx.x;
        if (threadIdx.x < cols && m < 0x7f800000u && SBP_GUARD(sp, 4)) *sp = __uint_as_float(sb);
      }
      return m >= 0x7f800000u;
    };
    fix = __syncthreads_or(columns(false));
    if (fix) {
      columns(true);
      __syncthreads();
    }
  }
  // element e of rows 0..3 of a group of columns, scaled
  auto scaled = [&](int g, float (&v)[4][8]) {
    float s[8];
    if constexpr (!TILES) {
      *reinterpret_cast<float4*>(s) = *reinterpret_cast<const float4*>(&inv_of[g * 64 + cg * 8]);
      *reinterpret_cast<float4*>(s + 4) = *reinterpret_cast<const float4*>(&inv_of[g * 64 + cg * 8 + 4]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[g][i].get(v[i]);
      if (fix) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[i][e] = inf_to_nan(v[i][e]);
      }
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        const unsigned long long w = pair_mul(pair_of(v[i][e], v[i][e + 1]), TILES ? pair_of(inv) : pair_of(s[e], s[e + 1]));
        v[i][e] = pair_lo(w);
        v[i][e + 1] = pair_hi(w);
      }
    }
  };
  if constexpr (!TRANS) {
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      float v[4][8];
      scaled(g, v);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int r = rq * 4 + i, c = g * 64 + cg * 8, n = r < rows ? min(8, cols - c) : 0;
        if (n <= 0) continue;
        unsigned char* dst = J.q + (r0 + r) * J.ldq + c0 + c;
        const unsigned lo = e4m3_four(v[i]), hi = e4m3_four(v[i] + 4);
        if constexpr (VEC) {
          if (SBP_GUARD(dst, 8)) *reinterpret_cast<uint2*>(dst) = make_uint2(lo, hi);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (e < n && SBP_GUARD(dst + e, 1)) dst[e] = (unsigned char)((e < 4 ? lo : hi) >> (8 * (e & 3)));
        }
      }
    }
  } else {
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      float v[4][8];
      scaled(g, v);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float f[4] = {v[0][e], v[1][e], v[2][e], v[3][e]};
        words[(g * 64 + cg * 8 + e) * kPitch8 + rq] = e4m3_four(f);
      }
    }
    __syncthreads();
    // a warp a row of the result at a time, four values a lane
    const bool whole = (reinterpret_cast<unsigned long long>(J.q) & 3) == 0 && (J.ldq & 3) == 0;
    for (int c = warp; c < cols; c += 8) {
      const unsigned w = words[c * kPitch8 + lane];
      unsigned char* dst = J.q + (c0 + c) * J.ldq + r0 + lane * 4;
      const int n = min(4, rows - lane * 4);
      if (whole && n == 4) {
        if (SBP_GUARD(dst, 4)) *reinterpret_cast<unsigned*>(dst) = w;
      } else {
        for (int e = 0; e < n; ++e)
          if (SBP_GUARD(dst + e, 1)) dst[e] = (unsigned char)(w >> (8 * e));
      }
    }
  }
}

bool aligned(const void* p, int bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }

// Rows and columns of shard r's local tensor seen as a matrix.
void matrix_of(const sbp_tensor* t, int r, long long* rows, long long* cols) {
  int64_t shp[SBP_MAX_DIMS];
  local_shape_nd(t, r, shp);
  *rows = 1;
  for (int d = 0; d + 1 < t->ndim; ++d) *rows *= shp[d];
  *cols = shp[t->ndim - 1];
}

// The jobs of a call: one a shard, but replicas written to the same buffers once, and none where nothing is held.
// x, y, q, s in the order of Job8; y may be null.  backward: only y is written.
int make_jobs(const sbp_tensor* x, const sbp_tensor* y, const sbp_tensor* q, const sbp_tensor* s, bool backward, Jobs8* P) {
  int n = 0;
  for (int r = 0; r < placement_k(x); ++r) {
    Job8 j{};
    matrix_of(x, r, &j.rows, &j.cols);
    if (j.rows == 0 || j.cols == 0) continue;
    j.x = x->local[r];
    j.ldx = local_pitch(x, r);
    if (y) {
      j.y = y->local[r];
      j.ldy = local_pitch(y, r);
    }
    j.q = static_cast<unsigned char*>(q->local[r]);
    j.ldq = local_pitch(q, r);
    j.s = static_cast<float*>(s->local[r]);
    j.lds = local_pitch(s, r);
    bool seen = false;
    for (int i = 0; i < n; ++i) seen = seen || (P->j[i].y == j.y && (backward || (P->j[i].q == j.q && P->j[i].s == j.s)));
    if (!seen || x->sbp[0].kind != SBP_BROADCAST) P->j[n++] = j;
  }
  return n;
}

template <typename TX, typename TY, int OP>
sbp_status launch_rows(Jobs8& P, int n, cudaStream_t st) {
  if (n == 0) return SBP_OK;
  bool vec = true, wide = true;
  long long rows = 0, blocks = 0;
  for (int i = 0; i < n; ++i) {
    const Job8& j = P.j[i];
    vec = vec && aligned(j.x, 16) && j.ldx * sizeof(TX) % 16 == 0 && aligned(j.q, 8) && j.ldq % 8 == 0 && j.cols % 8 == 0;
    wide = wide && aligned(j.q, 16) && j.ldq % 16 == 0 && j.cols % 16 == 0;
    if (OP != kQuantize) vec = vec && aligned(j.y, 16) && j.ldy * sizeof(TY) % 16 == 0;
    rows = j.rows > rows ? j.rows : rows;
    blocks = blocks8(j.cols) > blocks ? blocks8(j.cols) : blocks;
  }
  P.wide = wide;
  P.per_row_log = 0;
  while (P.per_row_log < 5 && (1 << P.per_row_log) < blocks) ++P.per_row_log;
  const long long rows_cta = (32 >> P.per_row_log) * rows_at_once(vec);
  const long long gx = (rows + rows_cta - 1) / rows_cta, gy = (blocks + (1 << P.per_row_log) - 1) >> P.per_row_log;
  if (gx > 0x7fffffffLL || gy > 65535) return fail(SBP_ERR_UNSUPPORTED, "tensor too large for one launch");
  const dim3 grid((unsigned)gx, (unsigned)gy, (unsigned)n);
  SBP_BOUNDS_UPLOAD(st);
  const cudaError_t e = vec ? launch_dependent(blocks8_row_kernel<TX, TY, OP, true>, grid, dim3(256), 0, st, P)
                            : launch_dependent(blocks8_row_kernel<TX, TY, OP, false>, grid, dim3(256), 0, st, P);
  if (e != cudaSuccess) return cuda_fail(e, "8-bit block launch");
  count_launch();
  return SBP_OK;
}

template <typename TX>
sbp_status launch_tiles(Jobs8& P, int n, bool tiles, bool trans, cudaStream_t st) {
  if (n == 0) return SBP_OK;
  bool vec = true;
  long long rows = 0, cols = 0;
  for (int i = 0; i < n; ++i) {
    const Job8& j = P.j[i];
    vec = vec && aligned(j.x, 16) && j.ldx * sizeof(TX) % 16 == 0 && j.cols % 8 == 0;
    if (!trans) vec = vec && aligned(j.q, 8) && j.ldq % 8 == 0;
    rows = j.rows > rows ? j.rows : rows;
    cols = j.cols > cols ? j.cols : cols;
  }
  if (blocks8(rows) > 0x7fffffffLL || blocks8(cols) > 65535) return fail(SBP_ERR_UNSUPPORTED, "matrix too large for one launch");
  const dim3 grid((unsigned)blocks8(rows), (unsigned)blocks8(cols), (unsigned)n);
  SBP_BOUNDS_UPLOAD(st);
  cudaError_t e;
  switch ((tiles ? 4 : 0) | (trans ? 2 : 0) | (vec ? 1 : 0)) {
    case 2: e = launch_dependent(blocks8_tile_kernel<TX, false, true, false>, grid, dim3(256), 0, st, P); break;
    case 3: e = launch_dependent(blocks8_tile_kernel<TX, false, true, true>, grid, dim3(256), 0, st, P); break;
    case 4: e = launch_dependent(blocks8_tile_kernel<TX, true, false, false>, grid, dim3(256), 0, st, P); break;
    case 5: e = launch_dependent(blocks8_tile_kernel<TX, true, false, true>, grid, dim3(256), 0, st, P); break;
    case 6: e = launch_dependent(blocks8_tile_kernel<TX, true, true, false>, grid, dim3(256), 0, st, P); break;
    default: e = launch_dependent(blocks8_tile_kernel<TX, true, true, true>, grid, dim3(256), 0, st, P); break;
  }
  if (e != cudaSuccess) return cuda_fail(e, "8-bit tile launch");
  count_launch();
  return SBP_OK;
}

bool is_float(int32_t dtype) { return dtype == SBP_F32 || dtype == SBP_BF16; }

// Shape, signature and placement of two tensors that have been checked.
sbp_status check_same(const sbp_tensor* t, const char* name, const sbp_tensor* like, const char* like_name) {
  if (placement_k(t) != placement_k(like)) return fail(SBP_ERR_INVALID_ARG, "%s and %s differ in k", name, like_name);
  if (t->ndim != like->ndim) return fail(SBP_ERR_SHAPE, "%s and %s differ in shape", name, like_name);
  for (int d = 0; d < t->ndim; ++d)
    if (t->shape[d] != like->shape[d]) return fail(SBP_ERR_SHAPE, "%s and %s differ in shape", name, like_name);
  if (!same_sig(t->sbp[0], like->sbp[0])) return fail(SBP_ERR_SIGNATURE, "%s and %s differ in signature", name, like_name);
  return SBP_OK;
}

// A floating tensor, like another one where that is given.
sbp_status check_like(const sbp_tensor* t, const char* name, const sbp_tensor* like, const char* like_name) {
  sbp_status st = check_tensor(t, name, true);
  if (st != SBP_OK) return st;
  if (!is_float(t->dtype)) return fail(SBP_ERR_DTYPE, "%s must be F32 or BF16", name);
  return like ? check_same(t, name, like, like_name) : SBP_OK;
}

sbp_status check_split_or_b(const sbp_tensor* t, const char* name) {
  if (t->sbp[0].kind != SBP_SPLIT && t->sbp[0].kind != SBP_BROADCAST)
    return fail(SBP_ERR_SIGNATURE, "%s must be S(i) or B: the operation is not linear", name);
  return SBP_OK;
}

}  // namespace

}  // namespace sbp

using namespace sbp;

extern "C" {

sbp_status sbp_quantize8(const sbp_tensor* x, sbp_tensor* values, sbp_tensor* scales, uint32_t flags, void* cuda_stream) {
  SBP_RANGE("sbp_quantize8");
  if (flags & ~(SBP_QUANT_TILES | SBP_TRANS_X)) return fail(SBP_ERR_INVALID_ARG, "unknown flags 0x%x", flags);
  const bool tiles = (flags & SBP_QUANT_TILES) != 0, trans = (flags & SBP_TRANS_X) != 0;
  sbp_status st = check_like(x, "x", nullptr, nullptr);
  if (st != SBP_OK) return st;
  if ((st = check_split_or_b(x, "x")) != SBP_OK) return st;
  if ((st = check_blocks8(values, scales, "values", tiles ? 1 : 0, true, nullptr)) != SBP_OK) return st;
  if (x->ndim != values->ndim) return fail(SBP_ERR_SHAPE, "x and values differ in shape");
  if ((tiles || trans) && x->ndim != 2) return fail(SBP_ERR_SHAPE, "tiles and transposes need a 2-D tensor");
  for (int d = 0; d < x->ndim; ++d)
    if (values->shape[d] != x->shape[trans ? 1 - d : d])
      return fail(SBP_ERR_SHAPE, trans ? "values must have the transposed shape of x" : "x and values differ in shape");
  if (placement_k(x) != placement_k(values)) return fail(SBP_ERR_INVALID_ARG, "x and values differ in k");
  sbp_sig want = x->sbp[0];
  if (trans && want.kind == SBP_SPLIT) want.axis = 1 - want.axis;
  if (!same_sig(values->sbp[0], want)) return fail(SBP_ERR_SIGNATURE, "values must have x's signature%s", trans ? ", its axis exchanged" : "");
  SBP_BOUNDS_RESET();
  SBP_BOUNDS_TENSOR(x);
  SBP_BOUNDS_TENSOR(values);
  SBP_BOUNDS_TENSOR(scales);
  Jobs8 P{};
  const int n = make_jobs(x, nullptr, values, scales, false, &P);
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  if (tiles || trans)
    return x->dtype == SBP_F32 ? launch_tiles<float>(P, n, tiles, trans, stream) : launch_tiles<__nv_bfloat16>(P, n, tiles, trans, stream);
  return x->dtype == SBP_F32 ? launch_rows<float, float, kQuantize>(P, n, stream) : launch_rows<__nv_bfloat16, __nv_bfloat16, kQuantize>(P, n, stream);
}

sbp_status sbp_gelu_save8(const sbp_tensor* z, sbp_tensor* y, sbp_tensor* values, sbp_tensor* scales, void* cuda_stream) {
  SBP_RANGE("sbp_gelu_save8");
  sbp_status st = check_like(z, "z", nullptr, nullptr);
  if (st != SBP_OK) return st;
  if ((st = check_split_or_b(z, "z")) != SBP_OK) return st;
  if ((st = check_like(y, "y", z, "z")) != SBP_OK) return st;
  if ((st = check_blocks8(values, scales, "values", 0, true, nullptr)) != SBP_OK) return st;
  if ((st = check_same(values, "values", z, "z")) != SBP_OK) return st;
  SBP_BOUNDS_RESET();
  SBP_BOUNDS_TENSOR(z);
  SBP_BOUNDS_TENSOR(y);
  SBP_BOUNDS_TENSOR(values);
  SBP_BOUNDS_TENSOR(scales);
  Jobs8 P{};
  const int n = make_jobs(z, y, values, scales, false, &P);
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  using bf16 = __nv_bfloat16;
  switch ((z->dtype == SBP_F32 ? 2 : 0) | (y->dtype == SBP_F32 ? 1 : 0)) {
    case 0: return launch_rows<bf16, bf16, kGelu>(P, n, stream);
    case 1: return launch_rows<bf16, float, kGelu>(P, n, stream);
    case 2: return launch_rows<float, bf16, kGelu>(P, n, stream);
    default: return launch_rows<float, float, kGelu>(P, n, stream);
  }
}

sbp_status sbp_gelu_save8_backward(const sbp_tensor* values, const sbp_tensor* scales, const sbp_tensor* grad_y, sbp_tensor* grad_z,
                                   void* cuda_stream) {
  SBP_RANGE("sbp_gelu_save8_backward");
  sbp_status st = check_blocks8(values, scales, "values", 0, true, nullptr);
  if (st != SBP_OK) return st;
  if ((st = check_split_or_b(values, "values")) != SBP_OK) return st;
  if ((st = check_like(grad_y, "grad_y", values, "values")) != SBP_OK) return st;
  if ((st = check_like(grad_z, "grad_z", values, "values")) != SBP_OK) return st;
  SBP_BOUNDS_RESET();
  SBP_BOUNDS_TENSOR(values);
  SBP_BOUNDS_TENSOR(scales);
  SBP_BOUNDS_TENSOR(grad_y);
  SBP_BOUNDS_TENSOR(grad_z);
  Jobs8 P{};
  const int n = make_jobs(grad_y, grad_z, values, scales, true, &P);
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  using bf16 = __nv_bfloat16;
  switch ((grad_y->dtype == SBP_F32 ? 2 : 0) | (grad_z->dtype == SBP_F32 ? 1 : 0)) {
    case 0: return launch_rows<bf16, bf16, kGeluGrad>(P, n, stream);
    case 1: return launch_rows<bf16, float, kGeluGrad>(P, n, stream);
    case 2: return launch_rows<float, bf16, kGeluGrad>(P, n, stream);
    default: return launch_rows<float, float, kGeluGrad>(P, n, stream);
  }
}

}  // extern "C"
