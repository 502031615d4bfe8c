// Products of linear layers on the 5th-generation tensor cores: D[a][b] = sum_k A[a][k] B[b][k], written through Finish.
//
// A tile of D is 128 kCG rows (a) by kBN columns (b).  One thread per CTA feeds a ring of stages with TMA tile loads (128-byte
// swizzle, zero fill past the ends of a matrix), one issues tcgen05.mma kind::f16 into an FP32 accumulator in tensor memory, eight or
// sixteen warps read it back with tcgen05.ld and finish it, a lane per row: rows are side by side in D's memory, so every warp's
// store is one run of it.  Either operand may have its rows or its k running through memory (the descriptors say which).
// kCG = 2: two CTAs of a cluster share a tile of 256 rows, each holding its 128 rows of A and half of B, which halves what is
// loaded per product; the first one issues the MMAs for both.
//
// binary32 operands come as three bfloat16 planes, x = p0 + p1 + p2 (24 bits).  A stage holds all of them for its 64 k, and of the nine products
// of planes the six largest are formed, the smallest first.  The accumulator is emptied into registers after every block of k and added there with
// rounding to nearest: the tensor cores' additions truncate (emptied so, one-signed sums of 64 to 131,072 terms are 4.5e-8 too small, the worst of 60,000 4.2e-7).
//
// Few tiles: the CTAs of a cluster share a tile's k (splits > 1, kCG = 1), park their sums in shared memory and each finishes a share
// of the columns, adding in the order of the CTAs.
//
// Every wait has an iteration limit; a CTA whose wait runs out raises the status bit, stops issuing, waits for its loads
// under way (again bounded), meets the barriers that others wait at, frees its tensor memory and returns.
#include <cuda.h>

#include <mutex>

#include "linear_tc.cuh"
#include "linear_ptx.cuh"

namespace strads {
namespace {

constexpr int kRows = 128;                 // rows of A that a CTA holds
constexpr int kBlockK = 64;                // 16-bit elements of k per stage = one 128-byte swizzle row
constexpr int kProducts = 6;               // of planes (binary32)
constexpr uint32_t kWaitLimit = kMmaWaitLimit, kStallLimit = kMmaStallLimit;
constexpr size_t kSmemMost = 227 * 1024;

// 16-bit operands with long k (kLong): the accumulator is emptied after runs of kRun blocks, and the runs are added in registers, as binary32's blocks are.
constexpr int kRun = 64;
// Blocks of k up to which one accumulator holds them all.  The tensor cores' additions truncate: a one-signed sum ends 6e-9 of itself too small for every term, so
// that 8,192 (65,536) terms cost a tenth of the half step that binary16's (bfloat16's) result is rounded by.  Kept sums cost little: 2,309 x 2,310 by 16,384
// binary16 175.7 us, with one accumulator 173.5; by 32,768 338 and 338; 40 x 100 by 131,072 81 and 80.
constexpr int kMostHalf = 128, kMostBfloat = 1024;

template <typename T, int kBN, int kCG, bool kLong>
struct Shape {
  static constexpr bool kPlanes = sizeof(T) == 4, kKept = kPlanes || kLong;      // kKept: the sums of a tile are held in registers
  static_assert(!(kPlanes && kLong), "binary32 empties the accumulator every block");
  static constexpr int kCols = kBN / kCG;                                  // rows of B that a CTA holds
  static constexpr int kABytes = kRows * 128;
  static constexpr int kBBytes = (kCols < 64 ? 64 : kCols) * 128;          // (a box along the rows is at least 64 wide)
  static constexpr int kStageBytes = (kPlanes ? 3 : 1) * (kABytes + kBBytes);
  // warps that finish results: sixteen where the epilogue is long for its products (binary32, 4,096^3 with GELU and residual: 815 -> 695 us) or a tile is
  // small; eight, 32 columns at a time, for pairs' tiles of 16 bits, whose products sixteen slow down (8,192^3: 734 against 758 us, with everything in the
  // epilogue 759 against 787; 4,096 x 1,024 x 4,096: 28.5 against 30.3, with everything 43.6 against 42.9)
  static constexpr int kEpiWarps = kBN < 128 || (kBN == 256 && !kPlanes) ? 8 : 16, kTmaWarp = kEpiWarps, kMmaWarp = kEpiWarps + 1, kThreads = 32 * (kEpiWarps + 2);
  static constexpr int kWarpCols = kBN / (kEpiWarps / 4);                 // columns of a tile that each of them reads back
  static constexpr int kChunk = kBN >= 128 && kEpiWarps == 8 && !kLong ? 32 : 16;   // columns of the result that a warp finishes at a time
  static constexpr int kSlotBytes = kChunk * 32 * (int)sizeof(T);         // a chunk: 32 rows of them
  // narrow tiles read far more than they write: no shared memory for results, and two CTAs to an SM, so that up to 2 x 148 tiles
  // are under way at once and share the memory's bandwidth evenly however they divide by 148
  static constexpr bool kNarrow = kBN < 128;
  // per warp two slots for what goes out and two for what comes in (binary32, whose stages need the room: one, and the residual comes straight, 128 bytes
  // an instruction)
  static constexpr int kEpiBytes = kNarrow ? 0 : kEpiWarps * (kPlanes ? 1 : 4) * kSlotBytes;
  static constexpr int kStages = (int)(((kNarrow && !kPlanes ? kSmemMost / 2 - 512 : kSmemMost) - 2048 - kEpiBytes) / kStageBytes);
  static constexpr size_t kSmem = (size_t)kStages * kStageBytes + kEpiBytes + 1024;
  static constexpr uint32_t kTmemCols = 2 * kBN < 32 ? 32 : 2 * kBN;      // two accumulators
  static_assert(kBN * kRows * 4 <= kStages * kStageBytes, "the parked sums take the ring's place");
};

// Where a work item lies: its tile, and how many of the tile's blocks of k are its own.  CTAs that share a tile take its blocks in turn, so that
// what they read at one time lies side by side in memory (32 rows of 8,192 by 28,672 bfloat16: 99 us, 104 with a run of blocks each).
struct Item { int ta, tb, blocks; };
__device__ __forceinline__ Item item_of(const TcArgs& g, int i, int split) {
  // eight tiles along a at a time: what the CTAs work on together reads few different rows and columns
  constexpr int kGroup = 8;
  const int per = kGroup * g.tiles_b, first = i / per * kGroup, high = min(kGroup, g.tiles_a - first), in = i % per;
  return {first + in % high, in / high, (g.blocks - split + g.splits - 1) / g.splits};
}
__device__ __forceinline__ void tma_load_2d(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
               ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}
__device__ __forceinline__ void tma_store_2d(const CUtensorMap* map, uint32_t src, int x, int y) {
  asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%1, %2}], [%3];" ::"l"(map), "r"(x), "r"(y), "r"(src) : "memory");
  asm volatile("cp.async.bulk.commit_group;" ::: "memory");
}
template <int kN>
__device__ __forceinline__ void tma_stores_read() { asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(kN) : "memory"); }
__device__ __forceinline__ void st_shared(uint32_t p, __nv_bfloat16 v) { asm volatile("st.shared.u16 [%0], %1;" ::"r"(p), "h"(__bfloat16_as_ushort(v)) : "memory"); }
__device__ __forceinline__ void st_shared(uint32_t p, __half v) { asm volatile("st.shared.u16 [%0], %1;" ::"r"(p), "h"(__half_as_ushort(v)) : "memory"); }
__device__ __forceinline__ float ld_shared(uint32_t p, float) { float v; asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(p) : "memory"); return v; }
__device__ __forceinline__ float ld_shared(uint32_t p, __nv_bfloat16) {
  unsigned short v;
  asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(p) : "memory");
  return __bfloat162float(__ushort_as_bfloat16(v));
}
__device__ __forceinline__ float ld_shared(uint32_t p, __half) {
  unsigned short v;
  asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(p) : "memory");
  return __half2float(__ushort_as_half(v));
}
template <typename T> __device__ __forceinline__ T as_type(float v) { T t; store_f32(&t, v); return t; }

// What a warp keeps of its way through the results: the slots' use goes on from tile to tile.
struct Epilogue {
  uint32_t in, out, bar;                 // shared memory: two slots each; the two barriers of what comes in
  uint32_t asked, got, put;              // chunks of the residual asked for and used; slots stored from
  bool one;                              // the lane that issues the copies
};

// A chunk of kC columns (b0 ..) of 32 rows (a0 ..; this lane: a0 + lane).  Through shared memory a column is one run of 32 rows,
// which a lane writes and reads without bank conflicts; the copies to and from global memory are TMA's.  (Straight from registers, a
// warp moves 64 bytes an instruction and the memory pipe, which the tensor cores' operands use too, takes about 20 cycles for each:
// 8,192^3 with bias, residual and GELU 1.70 ms.)
template <typename T, int kC>
__device__ __forceinline__ bool finish_chunk(const TcArgs& g, Epilogue& e, const CUtensorMap* map_out, const CUtensorMap* map_pre, float (&v)[kC],
                                             float bias, int a0, int b0, int lane, uint32_t limit) {
  const Finish& f = g.f;
  constexpr int kRow = 32 * (int)sizeof(T), kSlot = kC * kRow, kOut = sizeof(T) == 4 ? 1 : 2;
  const long long a = a0 + lane;
  const bool here = a < g.na;
  const uint32_t mine = (uint32_t)lane * sizeof(T);
  if (!g.out_tma && !g.residual_tma && !g.preact_tma) {
    finish_run<T, kC>(f, v, here ? a : g.na - 1, b0, 1, min(kC, g.nb - b0), here);
    return true;
  }
  float r[kC];
  if (!f.plain) {
    if (g.residual_tma) {
      const uint32_t s = e.got & 1u;
      if (!__all_sync(0xffffffffu, mbar_wait(e.bar + 8 * s, (e.got >> 1) & 1u, limit))) return false;
#pragma unroll
      for (int j = 0; j < kC; ++j) r[j] = ld_shared(e.in + s * kSlot + j * kRow + mine, T());
      ++e.got;
      __syncwarp();
    } else if (f.residual.p) {
      const T* p = static_cast<const T*>(f.residual.p) + (here ? a : g.na - 1) * f.residual.sa + b0 * f.residual.sb;
#pragma unroll
      for (int j = 0; j < kC; ++j) r[j] = load_f32(p + min(j, g.nb - 1 - b0) * f.residual.sb);
    }
    if (f.bias_b == 0) {
#pragma unroll
      for (int j = 0; j < kC; ++j) v[j] += bias;
    } else if (f.bias) {
#pragma unroll
      for (int j = 0; j < kC; ++j) v[j] += load_f32(static_cast<const T*>(f.bias) + min(b0 + j, g.nb - 1));
    }
    if (g.preact_tma) {
      const uint32_t slot = e.out + (e.put++ % kOut) * kSlot;
      if (e.one) tma_stores_read<kOut - 1>();
      __syncwarp();
#pragma unroll
      for (int j = 0; j < kC; ++j) st_shared(slot + j * kRow + mine, as_type<T>(v[j]));
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (e.one) tma_store_2d(map_pre, slot, a0, b0);
    } else if (f.preact.p && here) {
#pragma unroll
      for (int j = 0; j < kC; ++j)
        if (b0 + j < g.nb) store_f32(static_cast<T*>(const_cast<void*>(f.preact.p)) + a * f.preact.sa + (b0 + j) * f.preact.sb, v[j]);
    }
    activate_all<sizeof(T) == 4>(v, f.act);
    if (f.residual.p) {
#pragma unroll
      for (int j = 0; j < kC; ++j) v[j] = fmaf(f.scale, v[j], r[j]);
    } else {
#pragma unroll
      for (int j = 0; j < kC; ++j) v[j] *= f.scale;
    }
  } else {
    if (std::is_same<T, __half>::value && f.factor) {
      const float* p = f.factor + (here ? a : g.na - 1) * f.factor_a;
#pragma unroll
      for (int j = 0; j < kC; ++j) v[j] *= p[min(b0 + j, g.nb - 1) * f.factor_b];
    }
    if (f.scale != 1.f) {
#pragma unroll
      for (int j = 0; j < kC; ++j) v[j] *= f.scale;
    }
  }
  if (g.out_tma) {
    const uint32_t slot = e.out + (e.put++ % kOut) * kSlot;
    if (e.one) tma_stores_read<kOut - 1>();
    __syncwarp();
#pragma unroll
    for (int j = 0; j < kC; ++j) st_shared(slot + j * kRow + mine, as_type<T>(v[j]));
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
    if (e.one) tma_store_2d(map_out, slot, a0, b0);
  } else if (here) {
#pragma unroll
    for (int j = 0; j < kC; ++j)
      if (b0 + j < g.nb) store_f32(static_cast<T*>(const_cast<void*>(f.out.p)) + a * f.out.sa + (b0 + j) * f.out.sb, v[j]);
  }
  return true;
}

template <typename T, int kBN, int kCG, bool kLong>
__global__ void __launch_bounds__(Shape<T, kBN, kCG, kLong>::kThreads, kBN < 128 && sizeof(T) == 2 ? 2 : 1)
k_linear_tc(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ CUtensorMap map_out,
            const __grid_constant__ CUtensorMap map_res, const __grid_constant__ CUtensorMap map_pre, const __grid_constant__ TcArgs g) {
  using S = Shape<T, kBN, kCG, kLong>;
  constexpr bool kPlanes = S::kPlanes, kKept = S::kKept;
  constexpr int kEpiWarps = S::kEpiWarps, kTmaWarp = S::kTmaWarp, kMmaWarp = S::kMmaWarp, kCols = S::kWarpCols;
  extern __shared__ unsigned char dyn[];
  __shared__ __align__(8) uint64_t s_full[S::kStages], s_empty[S::kStages], s_tfull[2], s_tempty[2], s_in[kEpiWarps][2];
  __shared__ uint32_t s_tmem;
  __shared__ volatile int s_abort;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  uint32_t rank = 0;
  if (kCG == 2 || g.splits > 1) asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  const bool leader = kCG == 1 || rank == 0;
  const uint32_t tiles = (smem_u32(dyn) + 1023u) & ~1023u;
  const uint32_t full = smem_u32(s_full), empty = smem_u32(s_empty), tfull = smem_u32(s_tfull), tempty = smem_u32(s_tempty);
  const uint32_t limit = g.stall ? kStallLimit : kWaitLimit;

  if (threadIdx.x == 0) {
    s_abort = 0;
    for (int i = 0; i < S::kStages; ++i) { mbar_init(full + 8 * i, 1); mbar_init(empty + 8 * i, 1); }
    for (int i = 0; i < 2; ++i) { mbar_init(tfull + 8 * i, 1); mbar_init(tempty + 8 * i, kEpiWarps * kCG); }
    for (int i = 0; i < 2 * kEpiWarps; ++i) mbar_init(smem_u32(s_in) + 8 * i, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_a) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_b) : "memory");
  }
  if (warp == kMmaWarp) {
    if (kCG == 2) {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&s_tmem)), "r"(S::kTmemCols) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
    } else {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&s_tmem)), "r"(S::kTmemCols) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  if (kCG == 2 || g.splits > 1) cluster_sync();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem = s_tmem;
  chain_begin();

  // work items of this CTA (pair): tiles in turn, or its share of one tile's k
  const int split = g.splits > 1 ? (int)rank : 0;
  const int first = g.splits > 1 ? (int)blockIdx.x / g.splits : (int)blockIdx.x / kCG;
  const int stride = g.splits > 1 ? 0x40000000 : (int)gridDim.x / kCG;
  const int n_items = g.tiles_a * g.tiles_b;

  if (warp == kTmaWarp) {
    if (elect_one()) {
      uint32_t n = 0;                                    // stages filled so far
      bool ok = true;
      const uint32_t bytes = (kPlanes ? 3u : 1u) * (uint32_t)(S::kABytes + (g.b_rows_inner ? (S::kCols < 64 ? 64 : S::kCols) : S::kCols) * 128);
      for (int i = first; i < n_items && ok; i += stride) {
        const Item w = item_of(g, i, split);
        const int a0 = w.ta * kRows * kCG + (kCG == 2 ? (int)rank * kRows : 0), b0 = w.tb * kBN + (kCG == 2 ? (int)rank * S::kCols : 0);
        for (int k = 0; k < w.blocks; ++k, ++n) {
          const uint32_t s = n % S::kStages;
          ok = !s_abort && mbar_wait(empty + 8 * s, ((n / S::kStages) & 1u) ^ 1u, limit);
          if (!ok) break;
          if (g.stall) continue;                         // (withheld: the consumers' waits run out)
          const int k0 = (k * g.splits + split) * kBlockK;
          const uint32_t bar = kCG == 2 ? mapa(full + 8 * s, 0) : full + 8 * s;
          if (leader) mbar_expect(full + 8 * s, bytes * kCG);
#pragma unroll
          for (int p = 0; p < (kPlanes ? 3 : 1); ++p) {
            const uint32_t sa = tiles + s * S::kStageBytes + p * S::kABytes, sb = tiles + s * S::kStageBytes + (kPlanes ? 3 : 1) * S::kABytes + p * S::kBBytes;
            if (g.a_rows_inner) {
              tma_load<kCG>(sa, &map_a, a0, k0, p, bar);
              tma_load<kCG>(sa + 8192, &map_a, a0 + 64, k0, p, bar);
            } else {
              tma_load<kCG>(sa, &map_a, k0, a0, p, bar);
            }
            if (g.b_rows_inner) {
#pragma unroll
              for (int c = 0; c < (S::kCols < 64 ? 1 : S::kCols / 64); ++c) tma_load<kCG>(sb + c * 8192, &map_b, b0 + c * 64, k0, p, bar);
            } else {
              tma_load<kCG>(sb, &map_b, k0, b0, p, bar);
            }
          }
        }
      }
      // what is still under way lands before the shared memory goes: every stage filled is read by the MMAs, or (having given up) has arrived
      if (!ok) { s_abort = 1; atomicOr(g.status, STRADS_STATUS_WAIT_EXPIRED); }
      if (!g.stall) {
        const uint32_t back = n < (uint32_t)S::kStages ? n : S::kStages;
        for (uint32_t j = n - back; j < n; ++j) {
          const uint32_t bar = ok ? empty : full;
          if (ok || leader) {
            if (!mbar_wait(bar + 8 * (j % S::kStages), (j / S::kStages) & 1u, limit)) {
              if (ok) { s_abort = 1; atomicOr(g.status, STRADS_STATUS_WAIT_EXPIRED); }
              break;
            }
          }
        }
      }
    }
    __syncwarp();
  } else if (warp == kMmaWarp) {
    if (leader) {                                        // (the warp as one; an elected lane issues)
      const bool one = elect_one();
      const uint32_t idesc = (1u << 4) | ((uint32_t)g.bf16 << 7) | ((uint32_t)g.bf16 << 10) | ((uint32_t)g.a_rows_inner << 15) |
                             ((uint32_t)g.b_rows_inner << 16) | ((uint32_t)(kBN >> 3) << 17) | ((uint32_t)(kRows * kCG >> 4) << 24);
      const uint32_t adv_a = g.a_rows_inner ? 128 : 2, adv_b = g.b_rows_inner ? 128 : 2;      // 16 k on, in units of 16 bytes
      uint32_t n = 0, u = 0;                             // stages read; accumulators filled
      bool ok = true;
      for (int i = first; i < n_items && ok; i += stride) {
        const Item w = item_of(g, i, split);
        const int seg = kPlanes ? 1 : kLong ? kRun : w.blocks;      // blocks to an accumulator
        for (int k = 0; k < w.blocks && ok; k += seg, ++u) {
          ok = __all_sync(0xffffffffu, !s_abort && mbar_wait(tempty + 8 * (u & 1u), ((u >> 1) & 1u) ^ 1u, limit));
          if (!ok) break;
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          const uint32_t d = tmem + (u & 1u) * kBN;
          const int len = kLong ? min(seg, w.blocks - k) : seg;
          for (int it = 0; it < len; ++it, ++n) {
            const uint32_t s = n % S::kStages;
            ok = __all_sync(0xffffffffu, !s_abort && mbar_wait(full + 8 * s, (n / S::kStages) & 1u, limit));
            if (!ok) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint32_t sa = tiles + s * S::kStageBytes, sb = sa + (kPlanes ? 3 : 1) * S::kABytes;
            if (one) {
#pragma unroll
              for (int q = 0; q < (kPlanes ? kProducts : 1); ++q) {
                const int pa = kPlanes ? (0x201100 >> (4 * (5 - q))) & 3 : 0, pb = kPlanes ? (0x021010 >> (4 * (5 - q))) & 3 : 0;
                const uint64_t da = umma_desc(sa + pa * S::kABytes, g.a_rows_inner), db = umma_desc(sb + pb * S::kBBytes, g.b_rows_inner);
#pragma unroll
                for (int j = 0; j < kBlockK / 16; ++j)
                  umma<kCG>(d, da + (uint64_t)(j * adv_a), db + (uint64_t)(j * adv_b), idesc, it > 0 || q > 0 || j > 0);
              }
              umma_commit<kCG>(empty + 8 * s);
            }
            __syncwarp();
          }
          if (!ok) break;
          if (one) umma_commit<kCG>(tfull + 8 * (u & 1u));
          __syncwarp();
        }
      }
      if (!ok && lane == 0) { s_abort = 1; atomicOr(g.status, STRADS_STATUS_WAIT_EXPIRED); }
    }
    __syncwarp();
  } else {
    const int quarter = warp & 3, part = warp >> 2;      // tensor memory lanes 32 quarter .. , columns part * kCols ..
    const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
    constexpr int kC = S::kChunk, kChunks = kCols / kC;
    uint32_t u = 0;
    bool ok = true;
    Epilogue e;
    e.out = tiles + S::kStages * S::kStageBytes + warp * (kPlanes ? 1 : 4) * S::kSlotBytes;
    e.in = e.out + 2 * S::kSlotBytes;
    e.bar = smem_u32(s_in) + 16 * warp;
    e.asked = e.got = e.put = 0;
    e.one = elect_one();
    for (int i = first; i < n_items && ok; i += stride) {
      const Item w = item_of(g, i, split);
      const int a0 = w.ta * kRows * kCG + (kCG == 2 ? (int)rank * kRows : 0) + quarter * 32, b0 = w.tb * kBN + part * kCols;
      const int seg = kPlanes ? 1 : kLong ? kRun : w.blocks;
      // chunks that lie in D at all
      const int chunks = a0 < g.na && b0 < g.nb ? min(kChunks, (g.nb - b0 + kC - 1) / kC) : 0;
      // the residual's next chunk is asked for a chunk ahead, a tile's first while its sums are still being formed
      auto ask = [&](int c) {
        if (g.splits == 1 && g.residual_tma && c < chunks) {
          if (e.one) {
            mbar_expect(e.bar + 8 * (e.asked & 1u), 32 * kC * (uint32_t)sizeof(T));
            tma_load_2d(e.in + (e.asked & 1u) * S::kSlotBytes, &map_res, a0, b0 + c * kC, e.bar + 8 * (e.asked & 1u));
          }
          ++e.asked;
        }
      };
      ask(0);
      float bias = 0.f;
      if (g.f.bias && g.f.bias_b == 0 && a0 + lane < g.na) bias = load_f32(static_cast<const T*>(g.f.bias) + (a0 + lane));
      float acc[kKept ? kCols : kC];
      if (kKept)
#pragma unroll
        for (int j = 0; j < kCols; ++j) acc[j] = 0.f;
      for (int k = 0; k < w.blocks && ok; k += seg, ++u) {
        ok = !s_abort && mbar_wait(tfull + 8 * (u & 1u), (u >> 1) & 1u, limit);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const uint32_t d = tmem + (u & 1u) * kBN + lanes + part * kCols;
        if (kKept) {
#pragma unroll
          for (int c = 0; c < kCols / 16; ++c) {
            uint32_t v[16];
            tmem_load16(d + c * 16, v);
            tmem_wait();
#pragma unroll
            for (int j = 0; j < 16; ++j) acc[c * 16 + j] += __uint_as_float(v[j]);
          }
        } else {
#pragma unroll 1
          for (int c = 0; c < kChunks; ++c) {
            if (g.splits == 1 && c >= chunks) break;
            uint32_t v[kC];
            __syncwarp();
#pragma unroll
            for (int q = 0; q < kC / 16; ++q) tmem_load16(d + c * kC + q * 16, v + q * 16);
            tmem_wait();
            float x[kC];
#pragma unroll
            for (int j = 0; j < kC; ++j) x[j] = __uint_as_float(v[j]);
            if (g.splits == 1) {
              ask(c + 1);
              ok = finish_chunk<T, kC>(g, e, &map_out, &map_pre, x, bias, a0, b0 + c * kC, lane, limit);
              if (!ok) break;
            } else {
#pragma unroll
              for (int j = 0; j < kC; ++j)               // (the ring is drained: all of it has been read by the MMAs)
                st_shared(tiles + (uint32_t)(((part * kCols + c * kC + j) * kRows + quarter * 32 + lane) * 4), x[j]);
            }
          }
        }
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster(mapa(tempty + 8 * (u & 1u), kCG == 2 ? 0 : rank));
      }
      if (kKept && ok) {
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
          float x[kC];
#pragma unroll
          for (int j = 0; j < kC; ++j) x[j] = acc[c * kC + j];
          if (g.splits == 1) {
            if (c < chunks && ok) {
              ok = finish_chunk<T, kC>(g, e, &map_out, &map_pre, x, bias, a0, b0 + c * kC, lane, limit);
            }
          } else {
#pragma unroll
            for (int j = 0; j < kC; ++j)
              st_shared(tiles + (uint32_t)(((part * kCols + c * kC + j) * kRows + quarter * 32 + lane) * 4), x[j]);
          }
        }
      }
    }
    if (e.one) {                                         // nothing of this warp's is under way when the shared memory goes
      for (; e.got != e.asked; ++e.got)
        if (!mbar_wait(e.bar + 8 * (e.got & 1u), (e.got >> 1) & 1u, limit)) break;
      asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    }
    if (!ok && lane == 0) { s_abort = 1; atomicOr(g.status, STRADS_STATUS_WAIT_EXPIRED); }
    __syncwarp();
  }

  if (g.splits > 1) {
    // every CTA of the cluster gets here, whatever happened above
    cluster_sync();
    if (!s_abort && warp < kEpiWarps && first < n_items) {
      const Item w = item_of(g, first, split);
      const int row = threadIdx.x & (kRows - 1);
      const long long a = (long long)w.ta * kRows + row;
      // a thread's columns: col, col + step, .., several at a time
      constexpr int kN = 4;
      constexpr int kGroups = kEpiWarps / 4;
      const int step = kGroups * g.splits, end = min(kBN, g.nb - w.tb * kBN);
      for (int col = split * kGroups + (int)(threadIdx.x >> 7); col < end; col += kN * step) {
        const int count = min(kN, (end - col + step - 1) / step);
        float z[kN];
#pragma unroll
        for (int j = 0; j < kN; ++j) z[j] = 0.f;
        for (int sp = 0; sp < g.splits; ++sp) {
          const uint32_t peer = mapa(tiles, (uint32_t)sp);
#pragma unroll
          for (int j = 0; j < kN; ++j) {
            float v;
            asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(peer + (uint32_t)(((col + min(j, count - 1) * step) * kRows + row) * 4)) : "memory");
            z[j] += v;
          }
        }
        finish_run<T, kN>(g.f, z, a < g.na ? a : g.na - 1, (long long)w.tb * kBN + col, step, count, a < g.na);
      }
    }
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  if (kCG == 2 || g.splits > 1) cluster_sync();          // nobody leaves while a neighbour may still reach its barriers or sums
  if (warp == kMmaWarp) {
    __syncwarp();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    if (kCG == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(S::kTmemCols) : "memory");
    else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(S::kTmemCols) : "memory");
  }
}

// What is asked of the driver once per process and device.
struct Device { bool known; int sms; int pairs; int most[9]; };      // most[n]: clusters of n CTAs that fit at once (of bfloat16's 128 columns; every 128-column kernel has an SM to itself)
constexpr int kMaxDevices = 64;
std::mutex g_mutex;
Device g_device[kMaxDevices];

template <typename K>
cudaError_t allow_smem(K kernel, size_t bytes) {
  return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
}
template <typename T, bool kLong>
cudaError_t allow_all() {
  cudaError_t e = allow_smem(k_linear_tc<T, 256, 2, kLong>, Shape<T, 256, 2, kLong>::kSmem);
  if (e == cudaSuccess) e = allow_smem(k_linear_tc<T, 128, 1, kLong>, Shape<T, 128, 1, kLong>::kSmem);
  if (e == cudaSuccess) e = allow_smem(k_linear_tc<T, 64, 1, kLong>, Shape<T, 64, 1, kLong>::kSmem);
  if (e == cudaSuccess) e = allow_smem(k_linear_tc<T, 32, 1, kLong>, Shape<T, 32, 1, kLong>::kSmem);
  return e;
}
template <typename K>
int clusters_that_fit(K kernel, int size, int threads, size_t smem) {
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)size; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)size * 64); cfg.blockDim = dim3((unsigned)threads); cfg.dynamicSmemBytes = smem;
  cfg.attrs = attr; cfg.numAttrs = 1;
  int n = 0;
  const cudaError_t e = cudaOccupancyMaxActiveClusters(&n, kernel, &cfg);
  if (e != cudaSuccess) cudaGetLastError();              // (a size the device refuses is simply not used)
  return e == cudaSuccess ? n : 0;
}

cudaError_t device_of(const Device** out) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= kMaxDevices) return cudaErrorInvalidDevice;
  std::lock_guard<std::mutex> lock(g_mutex);
  Device& d = g_device[dev];
  if (!d.known) {
    if (tensor_map_encoder() == nullptr) return cudaErrorNotSupported;
    if ((e = cudaDeviceGetAttribute(&d.sms, cudaDevAttrMultiProcessorCount, dev)) != cudaSuccess) return e;
    if ((e = allow_all<float, false>()) != cudaSuccess || (e = allow_all<__nv_bfloat16, false>()) != cudaSuccess || (e = allow_all<__half, false>()) != cudaSuccess ||
        (e = allow_all<__nv_bfloat16, true>()) != cudaSuccess || (e = allow_all<__half, true>()) != cudaSuccess)
      return e;
    using Pair = Shape<__nv_bfloat16, 256, 2, false>;
    using One = Shape<__nv_bfloat16, 128, 1, false>;
    d.pairs = clusters_that_fit(k_linear_tc<__nv_bfloat16, 256, 2, false>, 2, Pair::kThreads, Pair::kSmem);
    if (d.pairs < 1) return cudaErrorNotSupported;
    for (int n = 2; n <= 8; ++n) d.most[n] = clusters_that_fit(k_linear_tc<__nv_bfloat16, 128, 1, false>, n, One::kThreads, One::kSmem);
    d.known = true;
  }
  *out = &d;
  return cudaSuccess;
}

// A result, or what is laid out like it, 32 rows by `cols` columns at a time; false where TMA cannot address it.
template <typename T>
bool encode_result(CUtensorMap* map, const Side& m, int na, int nb, int cols) {
  if (m.p == nullptr || (m.sa != 1 && na > 1) || ((uintptr_t)m.p & 15) != 0 || (nb > 1 && ((m.sb * (long long)sizeof(T)) % 16 != 0 || m.sb < na))) return false;
  const cuuint64_t dims[2] = {(cuuint64_t)na, (cuuint64_t)nb};
  const cuuint64_t strides[1] = {nb > 1 ? (cuuint64_t)m.sb * sizeof(T) : ((cuuint64_t)na * sizeof(T) + 15) / 16 * 16};
  const cuuint32_t box[2] = {32, (cuuint32_t)cols}, estr[2] = {1, 1};
  const CUtensorMapDataType type = sizeof(T) == 4 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_UINT16;
  return tensor_map_encoder()(map, type, 2, const_cast<void*>(m.p), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE,
                  CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename T, int kBN, int kCG, bool kLong>
cudaError_t launch_kernel(const Planes& A, const Planes& B, TcArgs g, unsigned ctas, cudaStream_t s) {
  using S = Shape<T, kBN, kCG, kLong>;
  alignas(64) CUtensorMap ma, mb, mo = {}, mr = {}, mp = {};
  if (!encode_operand(&ma, A, g.bf16, kRows) || !encode_operand(&mb, B, g.bf16, S::kCols)) return cudaErrorInvalidValue;
  constexpr int kC = S::kChunk;
  if (g.splits == 1 && !S::kNarrow) {                    // (shared tiles are finished element by element)
    g.out_tma = encode_result<T>(&mo, g.f.out, g.na, g.nb, kC);
    g.residual_tma = !S::kKept && encode_result<T>(&mr, g.f.residual, g.na, g.nb, kC);
    g.preact_tma = encode_result<T>(&mp, g.f.preact, g.na, g.nb, kC);
  }
  return launch_chained_cluster(k_linear_tc<T, kBN, kCG, kLong>, ctas, S::kThreads, S::kSmem, s, kCG == 2 ? 2 : g.splits, ma, mb, mo, mr, mp, g);
}

int ceil_div(long long a, long long b) { return (int)((a + b - 1) / b); }

template <typename T, int kBN, int kCG>
cudaError_t launch(const Planes& A, const Planes& B, const TcArgs& g, unsigned ctas, cudaStream_t s) {
  if constexpr (sizeof(T) == 2)
    if (ceil_div(g.blocks, g.splits) > (std::is_same<T, __half>::value ? kMostHalf : kMostBfloat)) return launch_kernel<T, kBN, kCG, true>(A, B, g, ctas, s);
  return launch_kernel<T, kBN, kCG, false>(A, B, g, ctas, s);
}

template <typename T>
cudaError_t launch_typed(const Device& d, const Planes& A, const Planes& B, TcArgs g, cudaStream_t s) {
  const int wide = ceil_div(g.na, 256), narrow = ceil_div(g.na, kRows);
  // pairs of CTAs on 256 x 256 where they fill the GPU once; else tiles of 128 rows, as wide as b calls for
  if ((long long)wide * ceil_div(g.nb, 256) >= d.pairs) {
    g.tiles_a = wide; g.tiles_b = ceil_div(g.nb, 256); g.splits = 1;
    const long long n = (long long)g.tiles_a * g.tiles_b;
    return launch<T, 256, 2>(A, B, g, 2u * (unsigned)(n < d.pairs ? n : d.pairs), s);
  }
  const int bn = g.nb > 64 ? 128 : g.nb > 32 ? 64 : 32;
  g.tiles_a = narrow; g.tiles_b = ceil_div(g.nb, bn); g.splits = 1;
  const long long n = (long long)g.tiles_a * g.tiles_b;
  // few tiles: as many CTAs to a tile as fit the GPU (narrow tiles: two to an SM), each with four blocks of k at least
  const int slots = bn == 128 ? d.sms : 2 * d.sms;
  for (int size = 8; size >= 2 && g.splits == 1; --size)
    if (n * size <= slots && size * 4 <= g.blocks && (bn < 128 || d.most[size] >= n)) g.splits = size;
  const unsigned ctas = g.splits > 1 ? (unsigned)n * g.splits : (unsigned)(n < slots ? n : slots);
  if (bn == 128) return launch<T, 128, 1>(A, B, g, ctas, s);
  if (bn == 64) return launch<T, 64, 1>(A, B, g, ctas, s);
  return launch<T, 32, 1>(A, B, g, ctas, s);
}

}  // namespace

EncodeFn tensor_map_encoder() {
  static const EncodeFn found = [] {
    void* fn = nullptr;
    cudaDriverEntryPointQueryResult qres;
    const cudaError_t e = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &qres);
    return e == cudaSuccess && qres == cudaDriverEntryPointSuccess ? reinterpret_cast<EncodeFn>(fn) : nullptr;
  }();
  return found;
}

// box: {64, rows} where k runs through memory, {64, 64} where the rows do.
bool encode_operand(CUtensorMap* map, const Planes& m, bool bf16, int box_rows) {
  const cuuint64_t dims[3] = {(cuuint64_t)m.inner, (cuuint64_t)m.outer, (cuuint64_t)m.planes};
  const cuuint64_t pitch = (cuuint64_t)m.ld * 2, plane = m.planes > 1 ? (cuuint64_t)m.plane * 2 : pitch;
  const cuuint64_t strides[2] = {pitch, plane};
  const cuuint32_t box[3] = {64, (cuuint32_t)(m.rows_inner ? 64 : box_rows), 1}, estr[3] = {1, 1, 1};
  return tensor_map_encoder()(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<void*>(m.p), dims, strides,
                              box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

cudaError_t launch_linear_tc(int type, const Planes& A, const Planes& B, long long na, long long nb, long long nk, const Finish& f,
                             unsigned int* status, bool stall, cudaStream_t s) {
  const Device* d = nullptr;
  const cudaError_t e = device_of(&d);
  if (e != cudaSuccess) return e;
  TcArgs g = {};
  g.na = (int)na; g.nb = (int)nb; g.blocks = ceil_div(nk, kBlockK);
  g.a_rows_inner = A.rows_inner; g.b_rows_inner = B.rows_inner; g.bf16 = type != STRADS_F16;
  g.f = f; g.status = status; g.stall = stall;
  return type == STRADS_F32 ? launch_typed<float>(*d, A, B, g, s)
       : type == STRADS_BF16 ? launch_typed<__nv_bfloat16>(*d, A, B, g, s) : launch_typed<__half>(*d, A, B, g, s);
}

}  // namespace strads
