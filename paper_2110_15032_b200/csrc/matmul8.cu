// MatMul of 8-bit blocks: executes a grouped-GEMM plan (matmul_plan.h) whose operands are e4m3 values with a scale for each block of
// 128 along the contraction, both stored with the contraction last.
//
// A ring slot is one block: rows of 128 bytes are exactly what the 128-byte swizzle holds.  Four tcgen05.mma of K = 32 make the
// block's sum in tensor memory; the accumulating warps multiply it by the block's two scales and add it to fp32 registers while
// the next block's products go to another part of tensor memory.  So any fp32 scale is taken, and what the tensor cores add up
// unscaled is never more than 128 products.
//
//   8 warps (a pair's CTAs: 16)  the accumulators: 32 rows x 64 or fewer of the tile's columns each, a row a thread
//   1 warp    operands by bulk tensor copies (TMA form)
//   1 warp    one elected lane issues the MMAs
//   2 warps   the scales of a block into a ring of their own, asynchronously
//   4 warps   operands by plain loads, where base or pitch is not a multiple of 16 bytes (the other form)
//
// Forms: a CTA pair with 256 x 256 tiles, persistent; single CTAs with 128 x NB tiles, cut along the contraction over a cluster where
// there are few of them.  Few rows (columns): the 128 rows of the tile are the other operand's.
//
// Measured: 8192 x 4096 x 4096 (one scale for 128 columns) 132 us, 2.09 PFLOP/s, 1.25 times the bf16 GEMM rate; 2048^3 15.8 us; a weight of 16384 x 4096
// under 16 rows 15.7 us in one piece, 18.4 us over eight shards.  Bound of the pair form: not the MMAs (512 of 1060 clocks a block) but the round from one block to the one that takes its
// accumulator: products done, the warps woken, 128 columns read and added, the hand-back across the pair, the next products issued.  A first form at 139 us
// took 111 without the additions and 104 without the reads of tensor memory too.  Tried on it: accumulators of 128 and 160 columns, three and four of them (187 and
// 191 us: what a warp pays a block, 400 clocks of waits, is paid more often), 16 accumulating warps (210), two loads of columns under way (142), additions one
// by one instead of in pairs (136), waits that sleep (197).  With a scale for each column 222 us (300 with a row a lane, whose 32 broadcast loads a block take
// shared memory's bandwidth).
#include <cuda_bf16.h>

#include <algorithm>
#include <atomic>
#include <type_traits>

#include "blocks8.h"
#include "bounds_check.h"
#include "matmul_plan.h"
#include "sbp_internal.h"
#include "tc_ptx.h"

namespace sbp {

// Defined in matmul.cu and matmul_tc.cu.
sbp_status build_matmul_plan(const sbp_tensor* x, const sbp_tensor* w, const sbp_tensor* y, uint32_t flags, bool need_ptrs, bool eight,
                             MatmulPlan* plan);
bool tensor_map8(CUtensorMap* map, const void* base, long long rows, long long cols, long long ld, int box_rows);
bool tensor_map8_out(CUtensorMap* map, const void* base, int esz, long long rows, long long cols, long long ld);

namespace {

constexpr int kRows = 128;                   // rows of the A operand a CTA holds
constexpr int kScaleSlots = 3, kGroup = 4;   // slots of the scales' ring, blocks whose scales share one
constexpr int kLoad8 = 32;                   // accumulator columns loaded at a time
constexpr int kPanel = 8;                    // row tiles walked together

struct Params8 {
  CUtensorMap map_a[SBP_MAX_K], map_b[SBP_MAX_K];
  CUtensorMap map_y[SBP_MAX_K], map_rep[SBP_MAX_K];      // where y_tma is set: the result and its replicas
  // as stored, for the loading form: bases, pitches and K of every segment
  const unsigned char* a[SBP_MAX_K];
  const unsigned char* b[SBP_MAX_K];
  long long lda[SBP_MAX_K], ldb[SBP_MAX_K], kseg[SBP_MAX_K];
  const float* sa[SBP_MAX_K];
  const float* sb[SBP_MAX_K];
  int kblocks[SBP_MAX_K];                    // per segment; also the pitch of its scales
  long long m[SBP_MAX_K], n[SBP_MAX_K], row_off[SBP_MAX_K], col_off[SBP_MAX_K], ldy[SBP_MAX_K];
  void* y[SBP_MAX_K];
  void* y_rep[SBP_MAX_K];
  int tile_begin[SBP_MAX_K + 1], tiles_m[SBP_MAX_K], tiles_n[SBP_MAX_K];
  int n_rep, ngroups, nseg, chain, total_tiles;
  int a_tiles, b_tiles;                      // the scales are one for 128 rows (columns)
  int y_tma;                                 // the copy engine can address the result
  int y_align;                               // bytes that every row of the result (and of its replicas) is aligned to, 16 at most
  int out_f32, swap;                         // swap: rows of the tile are columns of the result
  int splits;                                // CTAs of a cluster that share a tile's contraction
  int give_up;                               // self-test: this accumulating warp (1 to 8) acts as if its last wait had run out; 0: none
};

constexpr unsigned idesc8(int rows, int cols) { return (1u << 4) | ((unsigned)(cols >> 3) << 17) | ((unsigned)(rows >> 4) << 24); }

// A bounded wait of a converged warp.  Without a hint how long to sleep: the wait for an accumulator is on the chain from one block's
// products to those after the next.
__device__ __forceinline__ bool wait_long(unsigned bar, unsigned parity, volatile int* abort_flag) {
  const unsigned long long t0 = now_ns();
  for (;;) {
    for (int i = 0; i < 64; ++i) {
      unsigned done;
      asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                   : "=r"(done) : "r"(bar), "r"(parity) : "memory");
      if (__all_sync(0xffffffffu, done)) return true;
    }
    if (__any_sync(0xffffffffu, *abort_flag)) return false;
    if (__any_sync(0xffffffffu, now_ns() - t0 > kWaitLimitNs)) {
      *abort_flag = 1;
      atomicExch(&g_tc_timeout_flag, 1);
      return false;
    }
  }
}
__device__ __forceinline__ bool wait8(unsigned bar, unsigned parity, volatile int* abort_flag) {
  unsigned done;
  asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
               : "=r"(done) : "r"(bar), "r"(parity) : "memory");
  if (__all_sync(0xffffffffu, done)) return true;
  return wait_long(bar, parity, abort_flag);
}

template <bool PAIR>
__device__ __forceinline__ void umma8(unsigned d, unsigned long long a, unsigned long long b, unsigned idesc, unsigned accumulate) {
  if constexpr (PAIR)
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
  else
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}

__device__ __forceinline__ void tma_load_cta(unsigned dst, const CUtensorMap* map, int x, int y, unsigned bar) {
  asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst), "l"(map),
               "r"(x), "r"(y), "r"(bar)
               : "memory");
}

// N accumulator columns of this warp's 32 rows
template <int N>
__device__ __forceinline__ void tmem_columns(unsigned taddr, float (&v)[N]) {
  if constexpr (N == 64) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x64.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32, %33, %34, %35, %36, %37, %38, %39, %40, %41, %42, %43, %44, %45, %46, %47, %48, %49, %50, %51, %52, %53, %54, %55, %56, %57, %58, %59, %60, %61, %62, %63}, [%64];\n\ttcgen05.wait::ld.sync.aligned;"
                 : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]),
                   "=f"(v[16]), "=f"(v[17]), "=f"(v[18]), "=f"(v[19]), "=f"(v[20]), "=f"(v[21]), "=f"(v[22]), "=f"(v[23]), "=f"(v[24]), "=f"(v[25]), "=f"(v[26]), "=f"(v[27]), "=f"(v[28]), "=f"(v[29]), "=f"(v[30]), "=f"(v[31]),
                   "=f"(v[32]), "=f"(v[33]), "=f"(v[34]), "=f"(v[35]), "=f"(v[36]), "=f"(v[37]), "=f"(v[38]), "=f"(v[39]), "=f"(v[40]), "=f"(v[41]), "=f"(v[42]), "=f"(v[43]), "=f"(v[44]), "=f"(v[45]), "=f"(v[46]), "=f"(v[47]),
                   "=f"(v[48]), "=f"(v[49]), "=f"(v[50]), "=f"(v[51]), "=f"(v[52]), "=f"(v[53]), "=f"(v[54]), "=f"(v[55]), "=f"(v[56]), "=f"(v[57]), "=f"(v[58]), "=f"(v[59]), "=f"(v[60]), "=f"(v[61]), "=f"(v[62]), "=f"(v[63])
                 : "r"(taddr)
                 : "memory");
  } else if constexpr (N == 32) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];\n\ttcgen05.wait::ld.sync.aligned;"
                 : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]), "=f"(v[16]), "=f"(v[17]), "=f"(v[18]), "=f"(v[19]), "=f"(v[20]), "=f"(v[21]), "=f"(v[22]), "=f"(v[23]), "=f"(v[24]), "=f"(v[25]), "=f"(v[26]), "=f"(v[27]), "=f"(v[28]), "=f"(v[29]), "=f"(v[30]), "=f"(v[31])
                 : "r"(taddr)
                 : "memory");
  } else if constexpr (N == 16) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n\ttcgen05.wait::ld.sync.aligned;"
                 : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15])
                 : "r"(taddr)
                 : "memory");
  } else {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];\n\ttcgen05.wait::ld.sync.aligned;"
                 : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7])
                 : "r"(taddr)
                 : "memory");
  }
}

// 64 accumulator columns of 16 rows the way the matrix units lay out their results: of every eight columns lane t has 2 (t mod 4) and the next one, in rows t / 4
// (v[4 g], v[4 g + 1]) and t / 4 + 8 (v[4 g + 2], v[4 g + 3]).
__device__ __forceinline__ void tmem_fragments(unsigned taddr, float (&v)[32]) {
    asm volatile("tcgen05.ld.sync.aligned.16x256b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];\n\ttcgen05.wait::ld.sync.aligned;"
                 : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]),
                   "=f"(v[16]), "=f"(v[17]), "=f"(v[18]), "=f"(v[19]), "=f"(v[20]), "=f"(v[21]), "=f"(v[22]), "=f"(v[23]), "=f"(v[24]), "=f"(v[25]), "=f"(v[26]), "=f"(v[27]), "=f"(v[28]), "=f"(v[29]), "=f"(v[30]), "=f"(v[31])
                 : "r"(taddr)
                 : "memory");
}

template <bool PAIR, int NB, bool TMA>
struct Shape8 {
  static constexpr int kColsCta = PAIR ? NB / 2 : NB;            // B rows this CTA loads
  static constexpr int kSlot = (kRows + kColsCta) * 128;
  static constexpr int kCtas = NB <= 32 && TMA ? 2 : 1;          // of an SM: narrow tiles leave room for the next tile's, or the next product's
  static constexpr int kSlots = NB == 16 ? 5 : NB == 32 ? 4 : (168 * 1024) / kSlot;      // 5 (256 and 128 columns), 7, 4, 5
  static constexpr int kAccs = NB == 256 ? 2 : 4;                // accumulators in tensor memory
  static constexpr int kAccCols = NB == 256 ? 256 : NB <= 32 ? 32 : 128;      // columns of one
  static constexpr int kTmem = kAccs * kAccCols;
  static constexpr int kScales = kGroup * (kRows + NB);          // floats of a slot: [row][block], [block][column]
  static constexpr int kAccWarps = 8;
  static constexpr int kCols = NB / (kAccWarps / 4);             // columns of an accumulating warp
  static constexpr int kSlabRow = kCols * 4 < 128 ? kCols * 4 : 128;      // its staging: 32 rows of so many bytes
  static constexpr int kSlab = 32 * kSlabRow;
  static constexpr int kThreads = (kAccWarps + (TMA ? 4 : 8)) * 32;
  static constexpr int kSmem = kSlots * kSlot + kAccWarps * kSlab + kScaleSlots * kScales * 4 + 1024;
};

struct Tile8 {
  int g, m0, n0;
};
__device__ __forceinline__ Tile8 tile_at(const Params8& p, int tile, int tm, int tn) {
  int g = 0;
  while (g + 1 < p.ngroups && tile >= p.tile_begin[g + 1]) ++g;
  const int t = tile - p.tile_begin[g], panel_tiles = kPanel * p.tiles_n[g];
  const int panel = t / panel_tiles, r = t - panel * panel_tiles;
  const int high = min(kPanel, p.tiles_m[g] - panel * kPanel);
  const int n = r / high;
  return {g, (panel * kPanel + (r - n * high)) * tm, n * tn};
}

// The blocks of a tile, or of one CTA's share of it: segment, block inside it, how many.
struct Run8 {
  int s, kb, count;
};
__device__ __forceinline__ Run8 blocks_of(const Params8& p, int g, int slice) {
  const int s_lo = p.chain ? 0 : g, s_hi = p.chain ? p.nseg : g + 1;
  int total = 0;
  for (int s = s_lo; s < s_hi; ++s) total += p.kblocks[s];
  const int first = (int)((long long)total * slice / p.splits);
  Run8 r{s_lo, first, (int)((long long)total * (slice + 1) / p.splits) - first};
  while (r.s + 1 < s_hi && r.kb >= p.kblocks[r.s]) r.kb -= p.kblocks[r.s++];
  return r;
}
__device__ __forceinline__ void next_block(const Params8& p, Run8& r) {
  if (++r.kb < p.kblocks[r.s] || !p.chain) return;
  r.kb = 0;
  do ++r.s;
  while (r.s + 1 < p.nseg && p.kblocks[r.s] == 0);
}

// 16 bytes of a row from byte k on, zeros past `len`; the row may start anywhere.
__device__ __forceinline__ uint4 row_bytes(const unsigned char* row, long long k, long long len) {
  const unsigned char* at = row + k;
  const unsigned off = (unsigned)(reinterpret_cast<unsigned long long>(at) & 3);
  if (k + 20 <= len && (off == 0 || k >= 4)) {      // five aligned words inside the row
    const unsigned* w = reinterpret_cast<const unsigned*>(at - off);
    unsigned v[5];
#pragma unroll
    for (int i = 0; i < 5; ++i) v[i] = SBP_GUARD(w + i, 4) ? w[i] : 0u;
    return make_uint4(__funnelshift_r(v[0], v[1], off * 8), __funnelshift_r(v[1], v[2], off * 8), __funnelshift_r(v[2], v[3], off * 8),
                      __funnelshift_r(v[3], v[4], off * 8));
  }
  unsigned v[4] = {0u, 0u, 0u, 0u};
#pragma unroll
  for (int i = 0; i < 16; ++i)
    if (k + i < len && SBP_GUARD(at + i, 1)) v[i >> 2] |= (unsigned)at[i] << (8 * (i & 3));
  return make_uint4(v[0], v[1], v[2], v[3]);
}

__device__ __forceinline__ void store_one(const Params8& p, void* y, long long at, float v) {
  if (p.out_f32) {
    float* to = static_cast<float*>(y) + at;
    if (SBP_GUARD(to, 4)) *to = v;
  } else {
    __nv_bfloat16* to = static_cast<__nv_bfloat16*>(y) + at;
    if (SBP_GUARD(to, 2)) *to = __float2bfloat16_rn(v);
  }
}

// COLS: a scale a column, else one for 128 columns of the tile.
template <bool PAIR, int NB, bool TMA, bool COLS>
__global__ void __launch_bounds__(Shape8<PAIR, NB, TMA>::kThreads, Shape8<PAIR, NB, TMA>::kCtas) matmul8_kernel(const __grid_constant__ Params8 p) {
  using C = Shape8<PAIR, NB, TMA>;
  constexpr bool kFragments = PAIR && COLS;        // a lane has 32 columns of four rows instead of 128 of one: a fourth of the columns' scales to load
  constexpr int kCols = C::kCols, kAccWarps = C::kAccWarps, kRole = kAccWarps;      // the first warp behind the accumulators
  constexpr int kTileM = PAIR ? 256 : 128;
  extern __shared__ unsigned char smem_raw[];
  __shared__ __align__(8) unsigned long long bar_full[C::kSlots], bar_empty[C::kSlots], bar_acc_full[C::kAccs], bar_acc_empty[C::kAccs],
      bar_sc_full[kScaleSlots], bar_sc_empty[kScaleSlots];
  __shared__ unsigned tmem_base_slot;
  __shared__ int abort_flag_s;
  volatile int* abort_flag = &abort_flag_s;
  unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  unsigned char* staging = smem + C::kSlots * C::kSlot;
  float* scales = reinterpret_cast<float*>(staging + kAccWarps * C::kSlab);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const unsigned rank = PAIR ? cluster_ctarank() : 0u;

  if (tid == 0) {
    abort_flag_s = 0;
    for (int i = 0; i < C::kSlots; ++i) {
      mbar_init(smem_addr(&bar_full[i]), TMA ? 1 : 4);      // PAIR: used in CTA 0, with both CTAs' bytes
      mbar_init(smem_addr(&bar_empty[i]), 1);
    }
    for (int i = 0; i < C::kAccs; ++i) {
      mbar_init(smem_addr(&bar_acc_full[i]), 1);
      mbar_init(smem_addr(&bar_acc_empty[i]), (PAIR ? 2 : 1) * kAccWarps);      // PAIR: used in CTA 0
    }
    for (int i = 0; i < kScaleSlots; ++i) {
      mbar_init(smem_addr(&bar_sc_full[i]), 64);
      mbar_init(smem_addr(&bar_sc_empty[i]), kAccWarps);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == kRole + 1) {
    if constexpr (PAIR) {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&tmem_base_slot)), "r"(C::kTmem) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&tmem_base_slot)), "r"(C::kTmem) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  if constexpr (PAIR) cluster_sync_all();
  else __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const unsigned tmem_base = tmem_base_slot;
  SBP_PDL_RELEASE();
  SBP_PDL_WAIT();

  const int splits = PAIR ? 1 : p.splits, slice = PAIR ? 0 : (int)(blockIdx.x % (unsigned)p.splits);
  const int first = PAIR ? (int)(blockIdx.x >> 1) : (int)(blockIdx.x / (unsigned)p.splits);
  const int stride = PAIR ? (int)(gridDim.x >> 1) : (int)(gridDim.x / (unsigned)p.splits);

  if (warp < kAccWarps) {
    // ------------------------------------------------ accumulators
    if constexpr (PAIR) asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");      // 2 x 216 + 72 = 3 x 168
    const int q = warp & 3, part = warp >> 2;       // lanes and columns
    const int row = q * 32 + lane;                 // of this CTA's 128
    const unsigned acc_empty0 = PAIR ? map_to_cta(smem_addr(&bar_acc_empty[0]), 0) : smem_addr(&bar_acc_empty[0]);
    int a = 0, ss = 0;
    unsigned a_round = 0, s_round = 0;
    float4 rs4 = make_float4(0.f, 0.f, 0.f, 0.f);      // this row's scales of four blocks; times the columns' where those share one
    bool ok = true;
    for (int tile = first; tile < p.total_tiles && ok; tile += stride) {
      const Tile8 tc = tile_at(p, tile, kTileM, NB);
      const int count = blocks_of(p, tc.g, slice).count;
      float acc[kCols];
#pragma unroll
      for (int i = 0; i < kCols; ++i) acc[i] = 0.f;
      for (int c = 0; c < count; ++c) {
        const int j = c % kGroup;
        if (j == 0) {                              // the next blocks' scales
          ok = wait8(smem_addr(&bar_sc_full[ss]), s_round, abort_flag);
          if (!ok) break;
          if constexpr (!kFragments) rs4 = *reinterpret_cast<const float4*>(scales + ss * C::kScales + row * kGroup);
          if constexpr (!COLS) {
            const float4 cs = *reinterpret_cast<const float4*>(scales + ss * C::kScales + (kRows + part * kCols / 128) * kGroup);
            rs4 = make_float4(rs4.x * cs.x, rs4.y * cs.y, rs4.z * cs.z, rs4.w * cs.w);
          }
        }
        const float rs = j == 0 ? rs4.x : j == 1 ? rs4.y : j == 2 ? rs4.z : rs4.w;
        const float* cs = scales + ss * C::kScales + kGroup * kRows + j * NB + part * kCols;
        {
          constexpr int kStep = PAIR ? 64 : kCols < kLoad8 ? kCols : kLoad8;
          ok = wait8(smem_addr(&bar_acc_full[a]), a_round, abort_flag);
          if (!ok) break;
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          const unsigned at = tmem_base + ((unsigned)(q * 32) << 16) + a * C::kAccCols + part * kCols;
          // (the two scales are multiplied by one another first: only their product has to lie in fp32's range)
          auto hand_back = [&]() {                 // the last columns are in registers: the accumulator goes back before they are added
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            __syncwarp();
            if (lane == 0) {
              if constexpr (PAIR) mbar_arrive_cluster(acc_empty0 + a * 8);
              else mbar_arrive(acc_empty0 + a * 8);
            }
          };
          if constexpr (kFragments) {
            const float* rsp = scales + ss * C::kScales + (q * 32 + (lane >> 2)) * kGroup + j;
            const float r[4] = {rsp[0], rsp[8 * kGroup], rsp[16 * kGroup], rsp[24 * kGroup]};
#pragma unroll
            for (int b = 0; b < kCols; b += 64) {
              float2 c[8];
#pragma unroll
              for (int g = 0; g < 8; ++g) c[g] = *reinterpret_cast<const float2*>(cs + b + g * 8 + (lane & 3) * 2);
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                float v[32];
                tmem_fragments(at + b + ((unsigned)(h * 16) << 16), v);
                if (b + 64 == kCols && h == 1) hand_back();
                float* to = acc + (b / 64 * 2 + h) * 32;
#pragma unroll
                for (int g = 0; g < 8; ++g) {
#pragma unroll
                  for (int i = 0; i < 2; ++i) {
                    const unsigned long long w = pair_fma(pair_of(v[4 * g + 2 * i], v[4 * g + 2 * i + 1]), pair_mul(pair_of(c[g].x, c[g].y), pair_of(r[2 * h + i])), pair_of(to[4 * g + 2 * i], to[4 * g + 2 * i + 1]));
                    to[4 * g + 2 * i] = pair_lo(w);
                    to[4 * g + 2 * i + 1] = pair_hi(w);
                  }
                }
              }
            }
          } else
#pragma unroll
          for (int b = 0; b < kCols; b += kStep) {
            float v[kStep];
            tmem_columns(at + b, v);
            if (b + kStep == kCols) hand_back();
            float* to = acc + b;
            if constexpr (!COLS) {
#pragma unroll
              for (int i = 0; i < kStep; i += 2) {
                const unsigned long long w = pair_fma(pair_of(v[i], v[i + 1]), pair_of(rs), pair_of(to[i], to[i + 1]));
                to[i] = pair_lo(w);
                to[i + 1] = pair_hi(w);
              }
            } else {
#pragma unroll
              for (int i = 0; i < kStep; i += 4) {
                const float4 s = *reinterpret_cast<const float4*>(cs + b + i);
                to[i] = fmaf(v[i], s.x * rs, to[i]);
                to[i + 1] = fmaf(v[i + 1], s.y * rs, to[i + 1]);
                to[i + 2] = fmaf(v[i + 2], s.z * rs, to[i + 2]);
                to[i + 3] = fmaf(v[i + 3], s.w * rs, to[i + 3]);
              }
            }
          }
          if (++a == C::kAccs) { a = 0; a_round ^= 1; }
        }
        if (j == kGroup - 1 || c + 1 == count) {
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_addr(&bar_sc_empty[ss]));
          if (++ss == kScaleSlots) { ss = 0; s_round ^= 1; }
        }
      }
      if (splits > 1) {                            // the partial tile, for the cluster to add up; the ring is done with
        if (p.give_up == warp + 1) {
          ok = false;
          *abort_flag = 1;
          atomicExch(&g_tc_timeout_flag, 1);
        }
        float* mine = reinterpret_cast<float*>(smem) + row * (NB + 4) + part * kCols;
        // This barrier has no limit, so a warp whose wait ran out comes here too: others may have seen all their blocks.
        asm volatile("bar.sync 1, 256;" ::: "memory");
        if (!ok) break;
#pragma unroll
        for (int i = 0; i < kCols; i += 4) *reinterpret_cast<float4*>(mine + i) = make_float4(acc[i], acc[i + 1], acc[i + 2], acc[i + 3]);
        break;                                     // (a cluster has one tile)
      }
      if (!ok) break;
      const long long M = p.m[tc.g], N = p.n[tc.g], ldy = p.ldy[tc.g];
      const int n_out = (tc.g == 0 ? p.n_rep : 0) + 1;
      const long long row0 = tc.m0 + (int)rank * kRows, col0 = tc.n0 + part * kCols;
      if (p.swap) {                         // neighbouring lanes are neighbouring columns of the result
        const long long n = row0 + row;
#pragma unroll
        for (int i = 0; i < kCols; ++i) {
          if (n < M && col0 + i < N)
            for (int o = 0; o < n_out; ++o) store_one(p, o == 0 ? p.y[tc.g] : p.y_rep[o - 1], (col0 + i) * ldy + n, acc[i]);
        }
      } else {
        // through a slab of shared memory, so that a warp stores whole pieces of rows
        unsigned char* slab = staging + warp * C::kSlab;
        constexpr int kMask = C::kSlabRow / 16 - 1;
        auto at_chunk = [&](int r, int c) { return slab + r * C::kSlabRow + ((c ^ (r & kMask)) << 4); };      // 16 bytes
        auto rows_out = [&](auto f32_tag) {
          constexpr bool F32 = decltype(f32_tag)::value;
          constexpr int esz = F32 ? 4 : 2, kPiece = kCols < 128 / esz ? kCols : 128 / esz, kChunks = kPiece * esz / 16;
          constexpr int kPer = 16 / esz;           // elements of a 16-byte chunk
          const long long m0 = row0 + q * 32;      // of the warp's 32
#pragma unroll
          for (int s = 0; s < kCols / kPiece; ++s) {
            const long long n0 = col0 + s * kPiece;
            if (m0 >= M || n0 >= N) break;         // the same for the whole warp
            // the store before has been read out of the slab
            if (p.y_tma && lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
            __syncwarp();
            if constexpr (kFragments) {
              constexpr int kGroups = kPiece / 8;  // of eight columns
#pragma unroll
              for (int g = 0; g < kGroups; ++g)
#pragma unroll
                for (int r = 0; r < 4; ++r) {      // rows lane / 4 + 8 r
                  const int line = (lane >> 2) + 8 * r, from = s * kGroups + g;
                  const float* f = acc + (from / 8 * 2 + r / 2) * 32 + from % 8 * 4 + r % 2 * 2;
                  if constexpr (F32) *reinterpret_cast<float2*>(at_chunk(line, g * 2 + (lane >> 1 & 1)) + (lane & 1) * 8) = make_float2(f[0], f[1]);
                  else *reinterpret_cast<unsigned*>(at_chunk(line, g) + (lane & 3) * 4) = bf16_two(f[0], f[1]);
                }
            } else {
#pragma unroll
            for (int c = 0; c < kChunks; ++c) {
              const float* f = acc + s * kPiece + c * kPer;
              uint4 o;
              if constexpr (F32) o = make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
              else o = make_uint4(bf16_two(f[0], f[1]), bf16_two(f[2], f[3]), bf16_two(f[4], f[5]), bf16_two(f[6], f[7]));
              *reinterpret_cast<uint4*>(at_chunk(lane, c)) = o;
            }
            }
            if (kChunks == 8 && p.y_tma) {         // a whole slab
              asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
              __syncwarp();
              if (lane == 0) {
                for (int o = 0; o < n_out; ++o) tma_store_2d(o == 0 ? &p.map_y[tc.g] : &p.map_rep[o - 1], (int)n0, (int)m0, smem_addr(slab));
                asm volatile("cp.async.bulk.commit_group;" ::: "memory");
              }
              continue;
            }
            __syncwarp();
            auto stores = [&](auto unit_tag) {     // pieces of `unit` bytes, neighbouring lanes neighbouring ones
              using Unit = decltype(unit_tag);
              constexpr int unit = sizeof(Unit), kUnits = kPiece * esz / unit, kElems = unit / esz;
              for (int i = lane; i < 32 * kUnits; i += 32) {
                const int r = i / kUnits, u = i % kUnits;
                const long long m = m0 + r, n = n0 + u * kElems;
                if (m >= M || n >= N) continue;
                const unsigned char* from = at_chunk(r, u * unit / 16) + u * unit % 16;
                for (int o = 0; o < n_out; ++o) {
                  unsigned char* to = static_cast<unsigned char*>(o == 0 ? p.y[tc.g] : p.y_rep[o - 1]) + (m * ldy + n) * esz;
                  if (n + kElems <= N) {
                    if (SBP_GUARD(to, unit)) *reinterpret_cast<Unit*>(to) = *reinterpret_cast<const Unit*>(from);
                  } else {
                    for (int e = 0; e < kElems && n + e < N; ++e) {
                      if (!SBP_GUARD(to + e * esz, esz)) continue;
                      if constexpr (F32) *reinterpret_cast<float*>(to + e * 4) = *reinterpret_cast<const float*>(from + e * 4);
                      else *reinterpret_cast<unsigned short*>(to + e * 2) = *reinterpret_cast<const unsigned short*>(from + e * 2);
                    }
                  }
                }
              }
            };
            if (p.y_align == 16) stores(uint4{});
            else if (p.y_align == 8) stores(uint2{});
            else if (F32 || p.y_align == 4) stores(unsigned{});
            else stores((unsigned short)0);
          }
        };
        if (p.out_f32) rows_out(std::true_type{});
        else rows_out(std::false_type{});
      }
    }
    if (p.y_tma && lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
  } else {
    if constexpr (PAIR) asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
    if (warp == kRole && TMA) {
      // ------------------------------------------------ operands, by the copy engine
      const bool leader = elect_one();
      int slot = 0;
      unsigned round = 0;
      long long issued = 0;
      bool ok = true;
      for (int tile = first; tile < p.total_tiles && ok; tile += stride) {
        const Tile8 tc = tile_at(p, tile, kTileM, NB);
        Run8 run = blocks_of(p, tc.g, slice);
        const int arow = (int)p.row_off[tc.g] + tc.m0 + (int)rank * kRows, brow = (int)p.col_off[tc.g] + tc.n0 + (int)rank * C::kColsCta;
        for (int c = 0; c < run.count; ++c) {
          ok = mbar_wait_warp(smem_addr(&bar_empty[slot]), round ^ 1, abort_flag);
          if (!ok) break;
          if (leader) {
            const unsigned sa = smem_addr(smem + slot * C::kSlot), sb = sa + kRows * 128;
            if constexpr (PAIR) {
              const unsigned full0 = map_to_cta(smem_addr(&bar_full[slot]), 0);
              if (rank == 0) mbar_expect_tx(smem_addr(&bar_full[slot]), 2 * C::kSlot);
              tma_load_2d(sa, &p.map_a[run.s], run.kb * 128, arow, full0);
              tma_load_2d(sb, &p.map_b[run.s], run.kb * 128, brow, full0);
            } else {
              mbar_expect_tx(smem_addr(&bar_full[slot]), C::kSlot);
              tma_load_cta(sa, &p.map_a[run.s], run.kb * 128, arow, smem_addr(&bar_full[slot]));
              tma_load_cta(sb, &p.map_b[run.s], run.kb * 128, brow, smem_addr(&bar_full[slot]));
            }
          }
          __syncwarp();
          ++issued;
          if (++slot == C::kSlots) { slot = 0; round ^= 1; }
          next_block(p, run);
        }
      }
      if (*abort_flag && rank == 0 && leader) {    // loads in flight get a bounded chance to land
        for (long long i = issued > C::kSlots ? issued - C::kSlots : 0; i < issued; ++i) {
          const unsigned long long t0 = now_ns();
          while (!mbar_try(smem_addr(&bar_full[i % C::kSlots]), (unsigned)((i / C::kSlots) & 1)) && now_ns() - t0 < 100000000ull) {
          }
        }
      }
    } else if (warp == kRole + 1) {
      // ------------------------------------------------ MMA issuer (PAIR: the first CTA's)
      if (rank == 0) {
        const bool leader = elect_one();
        int slot = 0, a = 0;
        unsigned round = 0, a_round = 0;
        constexpr unsigned idesc = idesc8(kTileM, NB), lo = desc_lo_fixed(16), hi = desc_hi_fixed(1024);
        bool ok = true;
        for (int tile = first; tile < p.total_tiles && ok; tile += stride) {
          const Tile8 tc = tile_at(p, tile, kTileM, NB);
          const int count = blocks_of(p, tc.g, slice).count;
          for (int c = 0; c < count; ++c) {
            // (the operands are there as a rule: their wait comes first, off the chain)
            ok = wait8(smem_addr(&bar_full[slot]), round, abort_flag);
            ok = ok && wait8(smem_addr(&bar_acc_empty[a]), a_round ^ 1, abort_flag);
            if (!ok) break;
            {
              asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
              if (leader) {
                const unsigned sa = smem_addr(smem + slot * C::kSlot), sb = sa + kRows * 128;
#pragma unroll
                for (int kk = 0; kk < 4; ++kk)     // 32 bytes of every row
                  umma8<PAIR>(tmem_base + a * C::kAccCols, desc_pack(lo + (sa >> 4) + kk * 2, hi), desc_pack(lo + (sb >> 4) + kk * 2, hi), idesc,
                              kk == 0 ? 0u : 1u);
                if constexpr (PAIR) {
                  umma_commit_pair(smem_addr(&bar_empty[slot]));
                  umma_commit_pair(smem_addr(&bar_acc_full[a]));
                } else {
                  umma_commit_cta(smem_addr(&bar_empty[slot]));
                  umma_commit_cta(smem_addr(&bar_acc_full[a]));
                }
              }
              __syncwarp();
              if (++a == C::kAccs) { a = 0; a_round ^= 1; }
            }
            if (++slot == C::kSlots) { slot = 0; round ^= 1; }
          }
        }
        if (*abort_flag && leader) {               // products in flight get a bounded chance to finish
          if constexpr (PAIR) umma_commit_pair(smem_addr(&bar_acc_full[a]));
          else umma_commit_cta(smem_addr(&bar_acc_full[a]));
          const unsigned long long t0 = now_ns();
          while (!mbar_try(smem_addr(&bar_acc_full[a]), a_round) && now_ns() - t0 < 100000000ull) {
          }
        }
        __syncwarp();
      }
    } else if (warp == kRole + 2 || warp == kRole + 3) {
      // ------------------------------------------------ scales
      const int t = tid - (kRole + 2) * 32;
      int ss = 0;
      unsigned round = 0;
      bool ok = true;
      for (int tile = first; tile < p.total_tiles && ok; tile += stride) {
        const Tile8 tc = tile_at(p, tile, kTileM, NB);
        Run8 run = blocks_of(p, tc.g, slice);
        const int rows = (int)min((long long)kRows, p.m[tc.g] - tc.m0 - (int)rank * kRows), cols = (int)min((long long)NB, p.n[tc.g] - tc.n0);
        const long long arow = p.row_off[tc.g] + tc.m0 + (int)rank * kRows, bcol = p.col_off[tc.g] + tc.n0;
        for (int c = 0; c < run.count; c += kGroup) {
          ok = mbar_wait_warp(smem_addr(&bar_sc_empty[ss]), round ^ 1, abort_flag);
          if (!ok) break;
          const unsigned to = smem_addr(scales + ss * C::kScales);
          const int n = min(kGroup, run.count - c);
          auto copy = [&](unsigned dst, const float* base, const float* from, bool in) {
            in = in && SBP_GUARD(from, 4);
            asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(in ? from : base), "r"(in ? 4u : 0u) : "memory");
          };
          for (int j = 0; j < n; ++j) {
            const long long pitch = p.kblocks[run.s];
            const float *sa = p.sa[run.s] + run.kb, *sb = p.sb[run.s] + run.kb;
#pragma unroll
            for (int i = 0; i < kRows; i += 64) {
              const long long r = arow + t + i;
              copy(to + ((t + i) * kGroup + j) * 4, sa, sa + (p.a_tiles ? r >> 7 : r) * pitch, t + i < rows);
            }
            if (COLS) {
#pragma unroll
              for (int i = 0; i < NB; i += 64) {
                const long long r = bcol + t + i;
                if (t + i < NB) copy(to + (kGroup * kRows + j * NB + t + i) * 4, sb, sb + (p.b_tiles ? r >> 7 : r) * pitch, t + i < cols);
              }
            } else if (t < (NB + 127) / 128) {
              copy(to + ((kRows + t) * kGroup + j) * 4, sb, sb + ((bcol >> 7) + t) * pitch, t * 128 < cols);
            }
            next_block(p, run);
          }
          asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_addr(&bar_sc_full[ss])) : "memory");
          if (++ss == kScaleSlots) { ss = 0; round ^= 1; }
        }
      }
      asm volatile("cp.async.wait_all;" ::: "memory");
    } else if (warp >= kRole + 4 && !TMA) {
      // ------------------------------------------------ operands, by plain loads: eight threads a row
      const int t = tid - (kRole + 4) * 32, chunk = t & 7;
      int slot = 0;
      unsigned round = 0;
      bool ok = true;
      for (int tile = first; tile < p.total_tiles && ok; tile += stride) {
        const Tile8 tc = tile_at(p, tile, kTileM, NB);
        Run8 run = blocks_of(p, tc.g, slice);
        const int rows = (int)min((long long)kRows, p.m[tc.g] - tc.m0), cols = (int)min((long long)NB, p.n[tc.g] - tc.n0);
        for (int c = 0; c < run.count; ++c) {
          ok = mbar_wait_warp(smem_addr(&bar_empty[slot]), round ^ 1, abort_flag);
          if (!ok) break;
          unsigned char* sa = smem + slot * C::kSlot;
          const long long k = (long long)run.kb * 128 + chunk * 16, len = p.kseg[run.s];
          const unsigned char* A = p.a[run.s] + (p.row_off[tc.g] + tc.m0) * p.lda[run.s];
          const unsigned char* B = p.b[run.s] + (p.col_off[tc.g] + tc.n0) * p.ldb[run.s];
          for (int r = t >> 3; r < kRows; r += 16)
            *reinterpret_cast<uint4*>(sa + r * 128 + ((chunk ^ (r & 7)) << 4)) = r < rows && k < len ? row_bytes(A + r * p.lda[run.s], k, len) : make_uint4(0u, 0u, 0u, 0u);
          for (int r = t >> 3; r < NB; r += 16)
            *reinterpret_cast<uint4*>(sa + kRows * 128 + r * 128 + ((chunk ^ (r & 7)) << 4)) =
                r < cols && k < len ? row_bytes(B + r * p.ldb[run.s], k, len) : make_uint4(0u, 0u, 0u, 0u);
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_addr(&bar_full[slot]));
          if (++slot == C::kSlots) { slot = 0; round ^= 1; }
          next_block(p, run);
        }
      }
    }
    __syncwarp();
  }

  if constexpr (!PAIR) {
    if (splits > 1) {
      // every CTA adds up its share of the tile, slice by slice, and stores it
      cluster_sync_all();
      if (!*abort_flag && warp < kAccWarps) {
        const Tile8 tc = tile_at(p, first, kTileM, NB);
        const long long M = p.m[tc.g], N = p.n[tc.g], ldy = p.ldy[tc.g];
        const int n_out = (tc.g == 0 ? p.n_rep : 0) + 1;
        // four columns at a time: neighbouring threads take neighbouring columns of the result, which are rows of the tile where the
        // operands are exchanged
        constexpr int kQuads = NB / 4;
        const int lo = kRows * kQuads * slice / splits, hi = kRows * kQuads * (slice + 1) / splits;
        for (int e = lo + tid; e < hi; e += kAccWarps * 32) {
          const int r = p.swap ? e & (kRows - 1) : e / kQuads, c = (p.swap ? e / kRows : e % kQuads) * 4;
          const unsigned at = smem_addr(smem) + (unsigned)(r * (NB + 4) + c) * 4;
          float v[4] = {0.f, 0.f, 0.f, 0.f};
          for (int s0 = 0; s0 < splits; s0 += 4) {      // four parts on their way at once, added in order
            float x[4][4];
#pragma unroll
            for (int s = 0; s < 4; ++s)
              if (s0 + s < splits)
                asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                             : "=f"(x[s][0]), "=f"(x[s][1]), "=f"(x[s][2]), "=f"(x[s][3])
                             : "r"(map_to_cta(at, s0 + s))
                             : "memory");
#pragma unroll
            for (int s = 0; s < 4; ++s)
              if (s0 + s < splits) {
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] = s0 + s == 0 ? x[s][i] : v[i] + x[s][i];
              }
          }
          const long long m = tc.m0 + r, n = tc.n0 + c;
          if (m >= M) continue;
          for (int o = 0; o < n_out; ++o) {
            void* y = o == 0 ? p.y[tc.g] : p.y_rep[o - 1];
            if (!p.swap && p.y_align >= 8 && n + 4 <= N) {
              unsigned char* to = static_cast<unsigned char*>(y) + (m * ldy + n) * (p.out_f32 ? 4 : 2);
              if (p.out_f32) {
#pragma unroll
                for (int h = 0; h < 2; ++h)
                  if (SBP_GUARD(to + 8 * h, 8)) *reinterpret_cast<float2*>(to + 8 * h) = make_float2(v[2 * h], v[2 * h + 1]);
              } else if (SBP_GUARD(to, 8)) {
                *reinterpret_cast<uint2*>(to) = make_uint2(bf16_two(v[0], v[1]), bf16_two(v[2], v[3]));
              }
            } else {
#pragma unroll
              for (int i = 0; i < 4; ++i)
                if (n + i < N) store_one(p, y, p.swap ? (n + i) * ldy + m : m * ldy + n + i, v[i]);
            }
          }
        }
      }
    }
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncwarp();
  if (PAIR || splits > 1) cluster_sync_all();      // the partner may still signal this CTA's barriers or read its tile
  else __syncthreads();
  if (warp == kRole + 1) {
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    if constexpr (PAIR) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(C::kTmem) : "memory");
    else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(C::kTmem) : "memory");
  }
}

// Launch of one form, or (p null) the clusters of it that the current device holds at once.
template <bool PAIR, int NB, bool TMA, bool COLS>
sbp_status launch8_form(const Params8* p, int cluster, int ctas, cudaStream_t st, int* capacity) {
  using C = Shape8<PAIR, NB, TMA>;
  static std::atomic<unsigned long long> opted{0};      // one bit per device
  int dev = 0;
  SBP_CUDA_TRY(cudaGetDevice(&dev));
  const unsigned long long bit = 1ull << (dev & 63);
  if (dev >= 64 || !(opted.load(std::memory_order_relaxed) & bit)) {
    SBP_CUDA_TRY(cudaFuncSetAttribute(matmul8_kernel<PAIR, NB, TMA, COLS>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmem));
    if constexpr (PAIR) {      // the accumulators' registers come out of what the block was launched with
      cudaFuncAttributes attr;
      SBP_CUDA_TRY(cudaFuncGetAttributes(&attr, matmul8_kernel<PAIR, NB, TMA, COLS>));
      if (attr.numRegs < 168) return fail(SBP_ERR_UNSUPPORTED, "the 8-bit matmul kernel was built with %d registers a thread", attr.numRegs);
    }
    if (dev < 64) opted.fetch_or(bit, std::memory_order_relaxed);
  }
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)ctas);
  cfg.blockDim = dim3(C::kThreads);
  cfg.dynamicSmemBytes = C::kSmem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)cluster;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = p ? 2 : 1;
  if (!p) {
    cfg.gridDim = dim3((unsigned)(device_sms() / cluster * cluster));
    SBP_CUDA_TRY(cudaOccupancyMaxActiveClusters(capacity, matmul8_kernel<PAIR, NB, TMA, COLS>, &cfg));
    return SBP_OK;
  }
  SBP_BOUNDS_UPLOAD(st);
  const cudaError_t e = cudaLaunchKernelEx(&cfg, matmul8_kernel<PAIR, NB, TMA, COLS>, *p);
  if (e != cudaSuccess) return cuda_fail(e, "8-bit matmul launch");
  count_launch();
  return SBP_OK;
}

int split_index(int splits) { return splits == 1 ? 0 : splits == 2 ? 1 : splits == 4 ? 2 : splits == 8 ? 3 : -1; }

// Never launched: how many clusters the device holds is asked of it, with a form's threads and shared memory.  (Of a kernel that allocates tensor memory
// the runtime says that an SM holds one CTA, also where it runs two.)
__global__ void __launch_bounds__(512) seats_kernel() {}

// Clusters that the device holds at once, asked once a device: of CTA pairs with 256 columns, of `splits` CTAs that take an SM each, or of those of which an
// SM holds two.  148 SMs have room for 37 clusters of four and 18 of eight by their number, for 33 and 15 by where they lie; of two to an SM for 71 and 33.
// Products of 33 and 34, 15 and 16, 71 and 72, 33 and 34 such clusters: 21.6 and 38.9, 19.1 and 34.5, 19.1 and 29.2, 16.3 and 24.4 us.
enum { kPairs = 0, kAlone = 1, kTwo = 2 };
sbp_status ask_clusters(int kind, int splits, int* n) {
  if (kind == kPairs) return launch8_form<true, 256, true, false>(nullptr, 2, 0, nullptr, n);
  constexpr int kStatic = 1024;                    // barriers, and what the launch itself takes
  constexpr int kLarge = Shape8<false, 128, true>::kSmem + kStatic, kSmall = Shape8<false, 32, true>::kSmem + kStatic;
  const int smem = kind == kTwo ? kSmall : kLarge;
  SBP_CUDA_TRY(cudaFuncSetAttribute(seats_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kLarge));      // (whoever asks, so threads may ask at once)
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)(device_sms() / splits * splits));
  cfg.blockDim = dim3(Shape8<false, 32, true>::kThreads);
  cfg.dynamicSmemBytes = smem;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = (unsigned)splits;
  attr.val.clusterDim.y = 1;
  attr.val.clusterDim.z = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  SBP_CUDA_TRY(cudaOccupancyMaxActiveClusters(n, seats_kernel, &cfg));
  return SBP_OK;
}
int cluster_capacity(int kind, int splits) {
  static std::atomic<int> known[64][3][4];
  const int by_number = device_sms() * (kind == kTwo ? 2 : 1) / (kind == kPairs ? 2 : splits);
  if (kind != kPairs && splits == 1) return by_number;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return by_number;
  std::atomic<int>& slot = known[dev][kind][split_index(splits)];
  int n = slot.load(std::memory_order_relaxed);
  if (n == 0) {
    if (ask_clusters(kind, splits, &n) != SBP_OK || n < 1) {
      cudaGetLastError();
      n = by_number;
    }
    slot.store(n, std::memory_order_relaxed);
  }
  return n;
}

struct Form8 {
  bool pair, swap;
  int nb, splits;
};

// Which single forms there are.  Two are no product's choice (choose8): with one scale for 128 columns, 64 columns by the copy engine are dearer a
// block and two to an SM fewer than 32; 16 columns by plain loads dearer a block than 32, more tiles, and 0.26 us less of exchange against
// at least 0.32 us for the two blocks or more of every share.
constexpr bool form_exists(int nb, bool tma, bool cols) { return cols || !(tma ? nb == 64 : nb == 16); }

// What sbp_matmul8_set_form asks for: columns | splits << 16 | swap << 24; 0: the library chooses.
std::atomic<int> g_form8{0};
// Launches by columns (256 >> index), log2 of the CTAs that share a contraction, swap, copy engine, scale for each column.
std::atomic<unsigned long long> g_launches8[5][4][2][2][2];
int form_index(int nb) { return nb == 256 ? 0 : nb == 128 ? 1 : nb == 64 ? 2 : nb == 32 ? 3 : nb == 16 ? 4 : -1; }

long long tiles_of(const MatmulPlan& plan, int tm, int tn, bool swap) {
  long long t = 0;
  for (int g = 0; g < plan.ngroups; ++g)
    if (plan.m[g] > 0 && plan.n[g] > 0)
      t += ((swap ? plan.n[g] : plan.m[g]) + tm - 1) / tm * (((swap ? plan.m[g] : plan.n[g]) + tn - 1) / tn);
  return t;
}

// The form with the least estimated time: 4.5 us, then per wave of clusters (pairs) so many a block and 3 between waves; a contraction shared by a
// cluster costs its exchange.  kBlockUs: with a scale for 128 columns / for each column.
// Of 68 products from 1 x 4096 x 4096 to 4096 x 16384 x 1024, 40 of them drawn, with both kinds of scales the pick is 5 % off the best form on the average; the
// worst are 9 x 4576 x 736 (12.5 for 7.5 us), 28 x 8288 x 592 (10.8 for 7.2) and 4 x 6128 x 224 (8.2 for 5.6), products of a few blocks and many
// CTAs, whose start the estimate does not count; 64 x 4096 x 4096 is 15.0 for 12.2.
Form8 choose8(const MatmulPlan& plan, long long blocks, bool tma, bool x_tiles, bool w_tiles) {
  constexpr double kBlockUs[5][2] = {{0.60, 0.97}, {0.42, 0.90}, {0.39, 0.56}, {0.38, 0.58}, {0.42, 0.46}};
  Form8 best{false, false, 128, 1};
  double least = -1;
  auto scale_each = [&](bool swap) {
    bool cols = !(swap ? x_tiles : w_tiles);
    for (int g = 0; g < plan.ngroups; ++g) cols = cols || (swap ? plan.row_off[g] : plan.col_off[g]) % 128 != 0;
    return cols;
  };
  if (const int want = g_form8.load(std::memory_order_relaxed)) {
    Form8 f{(want & 0xffff) == 256, (want >> 24) != 0, want & 0xffff, (want >> 16) & 0xff};
    while (f.splits > 1 && blocks < 2 * f.splits) f.splits /= 2;
    if (f.pair ? tma : form_exists(f.nb, tma, scale_each(f.swap))) return f;
  }
  auto consider = [&](bool pair, bool swap, int i) {
    const int nb = 256 >> i;
    const bool cols = scale_each(swap);
    if (!form_exists(nb, tma, cols)) return;
    const long long tiles = tiles_of(plan, pair ? 256 : 128, nb, swap);
    const double slow = tma ? 1.0 : 4.0;           // operands by plain loads
    for (int splits = 1; splits <= (pair ? 1 : 8); splits *= 2) {
      if (splits > 1 && blocks < 2 * splits) break;
      const long long held = cluster_capacity(pair ? kPairs : nb <= 32 && tma ? kTwo : kAlone, splits);
      const double waves = (double)((tiles + held - 1) / held);
      const double us = 4.5 + waves * (double)((blocks + splits - 1) / splits) * kBlockUs[i][cols] * slow + 3.0 * (waves - 1.0) +
                        (splits > 1 ? 2.8 + 0.016 * nb + 0.1 * splits : 0.0);
      if (least < 0 || us < least) {
        least = us;
        best = {pair, swap, nb, splits};
      }
    }
  };
  if (tma) consider(true, false, 0);
  for (int i = 1; i < 5; ++i)
    for (bool swap : {false, true}) consider(false, swap, i);
  return best;
}

template <int NB, bool TMA, bool COLS>
sbp_status launch8_single(const Params8& p, int cluster, int ctas, cudaStream_t st) {
  if constexpr (form_exists(NB, TMA, COLS)) return launch8_form<false, NB, TMA, COLS>(&p, cluster, ctas, st, nullptr);
  else return fail(SBP_ERR_UNSUPPORTED, "no 8-bit matmul form of %d columns", NB);
}

template <bool COLS>
sbp_status launch8(const Params8& p, Form8 f, bool tma, cudaStream_t st) {
  const int ctas = p.total_tiles * f.splits;
  sbp_status s;
  switch (f.nb + (tma ? 0 : 1)) {
    case 256: s = launch8_form<true, 256, true, COLS>(&p, 2, 2 * std::min(p.total_tiles, cluster_capacity(kPairs, 1)), st, nullptr); break;
    case 16: s = launch8_single<16, true, COLS>(p, f.splits, ctas, st); break;
    case 17: s = launch8_single<16, false, COLS>(p, f.splits, ctas, st); break;
    case 32: s = launch8_single<32, true, COLS>(p, f.splits, ctas, st); break;
    case 33: s = launch8_single<32, false, COLS>(p, f.splits, ctas, st); break;
    case 64: s = launch8_single<64, true, COLS>(p, f.splits, ctas, st); break;
    case 65: s = launch8_single<64, false, COLS>(p, f.splits, ctas, st); break;
    case 128: s = launch8_single<128, true, COLS>(p, f.splits, ctas, st); break;
    default: s = launch8_single<128, false, COLS>(p, f.splits, ctas, st); break;
  }
  if (s == SBP_OK) g_launches8[form_index(f.nb)][split_index(f.splits)][f.swap][tma][COLS].fetch_add(1, std::memory_order_relaxed);
  return s;
}

sbp_status run_matmul8(const MatmulPlan& plan, const sbp_tensor* x_scales, const sbp_tensor* w_scales, bool x_tiles, bool w_tiles,
                       int give_up, cudaStream_t st) {
  bool tma = true;
  long long blocks = 0;
  int kblocks[SBP_MAX_K];
  for (int s = 0; s < plan.nseg; ++s) {
    if (plan.kseg[s] > (1LL << 31) - 256) return fail(SBP_ERR_UNSUPPORTED, "contraction too long for one launch");
    kblocks[s] = (int)blocks8(plan.kseg[s]);
    if (!plan.chain && s >= plan.ngroups) continue;
    blocks = plan.chain ? blocks + kblocks[s] : std::max<long long>(blocks, kblocks[s]);
    if (plan.kseg[s] == 0) continue;
    for (const void* base : {plan.a[s], plan.b[s]}) tma = tma && reinterpret_cast<uintptr_t>(base) % 16 == 0;
    tma = tma && plan.lda[s] % 16 == 0 && plan.ldb[s] % 16 == 0;
  }
  if (blocks > 0x7fffffffLL) return fail(SBP_ERR_UNSUPPORTED, "contraction too long for one launch");
  const Form8 f = choose8(plan, blocks, tma, x_tiles, w_tiles);
  if (give_up && f.splits == 1) return fail(SBP_ERR_UNSUPPORTED, "no cluster shares this product's contraction");
  Params8 p{};
  p.splits = f.splits;
  p.give_up = give_up;
  p.swap = f.swap;
  p.out_f32 = plan.out_dtype == SBP_F32;
  p.chain = plan.chain;
  p.nseg = plan.nseg;
  p.ngroups = plan.ngroups;
  p.n_rep = plan.n_rep;
  for (int r = 0; r < plan.n_rep; ++r) p.y_rep[r] = plan.y_rep[r];
  p.a_tiles = f.swap ? w_tiles : x_tiles;
  p.b_tiles = f.swap ? x_tiles : w_tiles;
  const int tm = f.pair ? 256 : 128;
  long long rows_all = 0, cols_all = 0, tiles = 0;
  bool whole_blocks = p.b_tiles != 0;              // of columns: 128 of a tile share a scale
  for (int g = 0; g < plan.ngroups; ++g) {
    const bool sw = f.swap;
    p.m[g] = sw ? plan.n[g] : plan.m[g];
    p.n[g] = sw ? plan.m[g] : plan.n[g];
    p.row_off[g] = sw ? plan.col_off[g] : plan.row_off[g];
    p.col_off[g] = sw ? plan.row_off[g] : plan.col_off[g];
    p.ldy[g] = plan.ldy[g];
    p.y[g] = plan.y[g];
    if (p.row_off[g] + p.m[g] > 0x7ffffe00LL || p.col_off[g] + p.n[g] > 0x7ffffe00LL) return fail(SBP_ERR_UNSUPPORTED, "matrix too large for one launch");
    if (p.col_off[g] % 128 != 0) whole_blocks = false;
    rows_all = std::max(rows_all, p.row_off[g] + p.m[g]);
    cols_all = std::max(cols_all, p.col_off[g] + p.n[g]);
    p.tile_begin[g] = (int)tiles;
    p.tiles_m[g] = (int)std::max(1LL, (p.m[g] + tm - 1) / tm);
    p.tiles_n[g] = (int)std::max(1LL, (p.n[g] + f.nb - 1) / f.nb);
    if (p.m[g] > 0 && p.n[g] > 0) tiles += (long long)p.tiles_m[g] * p.tiles_n[g];
    if (tiles > 0x07ffffffLL) return fail(SBP_ERR_UNSUPPORTED, "matrix too large for one launch");
  }
  for (int g = plan.ngroups; g <= SBP_MAX_K; ++g) p.tile_begin[g] = (int)tiles;
  p.total_tiles = (int)tiles;
  if (tiles == 0) return SBP_OK;
  const int esz = p.out_f32 ? 4 : 2;
  bool y_tma = !f.swap && f.splits == 1;
  for (int g = 0; g < plan.ngroups; ++g)
    if (p.m[g] > 0 && p.n[g] > 0) y_tma = y_tma && reinterpret_cast<uintptr_t>(p.y[g]) % 16 == 0 && p.ldy[g] * esz % 16 == 0;
  for (int r = 0; r < p.n_rep; ++r) y_tma = y_tma && reinterpret_cast<uintptr_t>(p.y_rep[r]) % 16 == 0;
  p.y_tma = y_tma;
  uintptr_t bits = 16;                             // the lowest bit set is the alignment
  for (int g = 0; g < plan.ngroups; ++g)
    if (p.m[g] > 0 && p.n[g] > 0) bits |= reinterpret_cast<uintptr_t>(p.y[g]) | (uintptr_t)(p.ldy[g] * esz);
  for (int r = 0; r < p.n_rep; ++r) bits |= reinterpret_cast<uintptr_t>(p.y_rep[r]);
  p.y_align = (int)(bits & (~bits + 1));
  for (int g = 0; y_tma && g < plan.ngroups; ++g)
    if (p.m[g] > 0 && p.n[g] > 0 && !tensor_map8_out(&p.map_y[g], p.y[g], esz, p.m[g], p.n[g], p.ldy[g]))
      return fail(SBP_ERR_CUDA, "cuTensorMapEncodeTiled failed for the result of group %d", g);
  for (int r = 0; y_tma && r < p.n_rep; ++r)
    if (!tensor_map8_out(&p.map_rep[r], p.y_rep[r], esz, p.m[0], p.n[0], p.ldy[0])) return fail(SBP_ERR_CUDA, "cuTensorMapEncodeTiled failed for a result replica");
  for (int s = 0; s < plan.nseg; ++s) {
    p.kblocks[s] = kblocks[s];
    if (!plan.chain && s >= plan.ngroups) continue;
    const sbp_tensor *as = f.swap ? w_scales : x_scales, *bs = f.swap ? x_scales : w_scales;
    p.a[s] = static_cast<const unsigned char*>(f.swap ? plan.b[s] : plan.a[s]);
    p.b[s] = static_cast<const unsigned char*>(f.swap ? plan.a[s] : plan.b[s]);
    p.lda[s] = f.swap ? plan.ldb[s] : plan.lda[s];
    p.ldb[s] = f.swap ? plan.lda[s] : plan.ldb[s];
    p.kseg[s] = plan.kseg[s];
    p.sa[s] = static_cast<const float*>(as->local[s]);
    p.sb[s] = static_cast<const float*>(bs->local[s]);
    const long long rows = plan.chain ? rows_all : p.m[s], cols = plan.chain ? cols_all : p.n[s];
    if (!tma || kblocks[s] == 0 || rows == 0 || cols == 0) continue;
    if (!tensor_map8(&p.map_a[s], p.a[s], rows, p.kseg[s], p.lda[s], kRows) ||
        !tensor_map8(&p.map_b[s], p.b[s], cols, p.kseg[s], p.ldb[s], f.pair ? 128 : f.nb))
      return fail(SBP_ERR_CUDA, "cuTensorMapEncodeTiled failed for an operand of shard %d", s);
  }
  return whole_blocks ? launch8<false>(p, f, tma, st) : launch8<true>(p, f, tma, st);
}

sbp_status matmul8(const sbp_tensor* x, const sbp_tensor* x_scales, const sbp_tensor* w, const sbp_tensor* w_scales, sbp_tensor* y, int give_up,
                   void* cuda_stream) {
  MatmulPlan plan;
  sbp_status st = build_matmul_plan(x, w, y, SBP_TRANS_W, true, true, &plan);
  if (st != SBP_OK) return st;
  bool x_tiles = false, w_tiles = false;
  if ((st = check_blocks8(x, x_scales, "x", -1, true, &x_tiles)) != SBP_OK) return st;
  if ((st = check_blocks8(w, w_scales, "w", -1, true, &w_tiles)) != SBP_OK) return st;
  SBP_BOUNDS_RESET();
  SBP_BOUNDS_TENSOR(x);
  SBP_BOUNDS_TENSOR(x_scales);
  SBP_BOUNDS_TENSOR(w);
  SBP_BOUNDS_TENSOR(w_scales);
  SBP_BOUNDS_TENSOR(y);
  return run_matmul8(plan, x_scales, w_scales, x_tiles, w_tiles, give_up, static_cast<cudaStream_t>(cuda_stream));
}

}  // namespace

sbp_status read_and_clear_matmul8_timeout(bool* timed_out) { return read_and_clear_timeout_flag(timed_out); }

}  // namespace sbp

using namespace sbp;

extern "C" {

sbp_status sbp_matmul8(const sbp_tensor* x, const sbp_tensor* x_scales, const sbp_tensor* w, const sbp_tensor* w_scales, sbp_tensor* y,
                       void* cuda_stream) {
  SBP_RANGE("sbp_matmul8");
  return matmul8(x, x_scales, w, w_scales, y, 0, cuda_stream);
}

sbp_status sbp_matmul8_set_form(int32_t columns, int32_t splits, int32_t exchanged) {
  const bool pair = columns == 256;
  if (columns != 0 && (form_index(columns) < 0 || split_index(splits) < 0 || (pair && (splits != 1 || exchanged))))
    return fail(SBP_ERR_INVALID_ARG, "no form of %d columns with %d splits", columns, splits);
  g_form8.store(columns == 0 ? 0 : columns | splits << 16 | (exchanged ? 1 << 24 : 0), std::memory_order_relaxed);
  return SBP_OK;
}

uint64_t sbp_matmul8_form_launches(int32_t columns, int32_t splits, int32_t exchanged, int32_t copy_engine, int32_t scale_each) {
  const int c = form_index(columns), s = split_index(splits);
  return c < 0 || s < 0 ? 0 : g_launches8[c][s][exchanged != 0][copy_engine != 0][scale_each != 0].load(std::memory_order_relaxed);
}

sbp_status sbp_selftest_matmul8_wait_timeout(const sbp_tensor* x, const sbp_tensor* x_scales, const sbp_tensor* w, const sbp_tensor* w_scales,
                                             sbp_tensor* y, int32_t warp, void* cuda_stream) {
  if (warp < 0 || warp > 7) return fail(SBP_ERR_INVALID_ARG, "warp must be in [0, 7]");
  return matmul8(x, x_scales, w, w_scales, y, warp + 1, cuda_stream);
}

}  // extern "C"
