// Products of linear layers on the 5th-generation tensor cores: D[a][b] = sum_k A[a][k] B[b][k], written through Finish.
//
// A tile of D is 128 kCG rows (a) by kBN columns (b).  One thread per CTA feeds a ring of stages with TMA tile loads (128-byte
// swizzle, zero fill past the ends of a matrix), one issues tcgen05.mma kind::f16 into an FP32 accumulator in tensor memory, eight
// warps read it back with tcgen05.ld and finish it, a lane per row: rows are side by side in D's memory, so every warp's
// store is one run of it.  Either operand may have its rows or its k running through memory (the descriptors say which).
// kCG = 2: two CTAs of a cluster share a tile of 256 rows, each holding its 128 rows of A and half of B, which halves what is
// loaded per product; the first one issues the MMAs for both.
//
// binary32 operands come as three bfloat16 planes, x = p0 + p1 + p2 (24 bits).  Of the nine products of planes the six largest are formed,
// the smallest first.  The accumulator is emptied into registers every kSegment blocks of k and added there with rounding to nearest: the
// tensor cores' additions truncate, which over a long k would cost more than the parts left out.
//
// Few tiles: the CTAs of a cluster share a tile's k (splits > 1, kCG = 1), park their sums in shared memory and each finishes a share
// of the columns, adding in the order of the CTAs.
//
// Every wait has an iteration limit; a CTA whose wait runs out raises the status bit, stops issuing, waits for its loads
// under way (again bounded), meets the barriers that others wait at, frees its tensor memory and returns.
#include <cuda.h>

#include <mutex>

#include "linear_tc.cuh"

namespace strads {
namespace {

constexpr int kRows = 128;                 // rows of A that a CTA holds
constexpr int kBlockK = 64;                // 16-bit elements of k per stage = one 128-byte swizzle row
constexpr int kEpiWarps = 8;
constexpr int kTmaWarp = kEpiWarps, kMmaWarp = kEpiWarps + 1;
constexpr int kThreads = 32 * (kEpiWarps + 2);
constexpr int kSegment = 4;                // blocks of k between two emptyings of the accumulator (binary32)
constexpr int kProducts = 6;
constexpr uint32_t kWaitLimit = 1u << 24, kStallLimit = 1u << 14;
constexpr size_t kSmemMost = 227 * 1024;

template <int kBN, int kCG>
struct Shape {
  static constexpr int kCols = kBN / kCG;                                  // rows of B that a CTA holds
  static constexpr int kABytes = kRows * 128;
  static constexpr int kBBytes = (kCols < 64 ? 64 : kCols) * 128;          // (a box along the rows is at least 64 wide)
  static constexpr int kStageBytes = kABytes + kBBytes;
  static constexpr int kStages = (int)((kSmemMost - 2048) / kStageBytes) < 8 ? (int)((kSmemMost - 2048) / kStageBytes) : 8;
  static constexpr size_t kSmem = (size_t)kStages * kStageBytes + 1024;
  static constexpr uint32_t kTmemCols = 2 * kBN < 32 ? 32 : 2 * kBN;      // two accumulators
  static_assert(kBN * kRows * 4 <= kStages * kStageBytes, "the parked sums take the ring's place");
};

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void mbar_expect(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ uint32_t mapa(uint32_t addr, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
  return r;
}
__device__ __forceinline__ void mbar_arrive_cluster(uint32_t bar) {         // bar: a cluster address
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ bool mbar_wait(uint32_t bar, uint32_t parity, uint32_t limit) {
  for (uint32_t it = 0; it < limit; ++it) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    if (ok) return true;
  }
  return false;
}
template <int kCG>
__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
  if (kCG == 2)
    asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
  else
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}
// Shared-memory descriptor, 128-byte swizzle.  k along memory: rows of 128 bytes, groups of 8 rows 1,024 bytes apart.  Rows along
// memory: runs of 64 rows, a k per 128 bytes, groups of 8 k 1,024 bytes apart, the next 64 rows 8,192 bytes on.
__device__ __forceinline__ uint64_t umma_desc(uint32_t saddr, bool rows_inner) {
  return (uint64_t)((saddr & 0x3FFFFu) >> 4) | ((uint64_t)(rows_inner ? 8192 >> 4 : 1) << 16) | ((uint64_t)(1024 >> 4) << 32) |
         ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}
template <int kCG>
__device__ __forceinline__ void umma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  if (kCG == 2)
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
  else
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
template <int kCG>
__device__ __forceinline__ void umma_commit(uint32_t bar) {                  // kCG = 2: on the barrier of both CTAs
  if (kCG == 2)
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                 ::"r"(bar), "h"((uint16_t)3) : "memory");
  else
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tmem_load16(uint32_t taddr, uint32_t* v) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]),
        "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
      : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
}

// Where a work item lies: its tile, and its share of the tile's blocks of k.
struct Item { int ta, tb, k0, k1; };
__device__ __forceinline__ Item item_of(const TcArgs& g, int i, int split) {
  // eight tiles along a at a time: what the CTAs work on together reads few different rows and columns
  constexpr int kGroup = 8;
  const int per = kGroup * g.tiles_b, first = i / per * kGroup, high = min(kGroup, g.tiles_a - first), in = i % per;
  return {first + in % high, in / high, (int)((long long)g.blocks * split / g.splits), (int)((long long)g.blocks * (split + 1) / g.splits)};
}
// Block of k and planes that come `it`-th in a segment of `len` blocks from k0 on.  Smallest products first.
struct Step { int kb, pa, pb; };
template <bool kPlanes>
__device__ __forceinline__ Step step_of(int k0, int len, int it) {
  if (!kPlanes) return {k0 + it, 0, 0};
  const int q = it / len;
  return {k0 + it % len, (0x201100 >> (4 * (5 - q))) & 3, (0x021010 >> (4 * (5 - q))) & 3};
}

// Sixteen columns of one row.
template <typename T>
__device__ __forceinline__ void finish16(const Finish& f, const float* z, long long a, long long b0, int nb) {
  if (f.plain) {
#pragma unroll
    for (int j = 0; j < 16; ++j)
      if (b0 + j < nb) store_f32(static_cast<T*>(const_cast<void*>(f.out.p)) + a * f.out.sa + (b0 + j) * f.out.sb, f.scale * z[j]);
    return;
  }
  float r[16];
#pragma unroll
  for (int j = 0; j < 16; ++j)                           // (all before the stores: out may be the residual)
    r[j] = f.residual.p && b0 + j < nb ? load_f32(static_cast<const T*>(f.residual.p) + a * f.residual.sa + (b0 + j) * f.residual.sb) : 0.f;
  float v[16];
#pragma unroll
  for (int j = 0; j < 16; ++j) {
    v[j] = z[j];
    if (f.bias && b0 + j < nb) v[j] += load_f32(static_cast<const T*>(f.bias) + a * f.bias_a + (b0 + j) * f.bias_b);
  }
  if (f.preact.p)
#pragma unroll
    for (int j = 0; j < 16; ++j)
      if (b0 + j < nb) store_f32(static_cast<T*>(const_cast<void*>(f.preact.p)) + a * f.preact.sa + (b0 + j) * f.preact.sb, v[j]);
  activate_all<16>(v, f.act);
#pragma unroll
  for (int j = 0; j < 16; ++j)
    if (b0 + j < nb) store_f32(static_cast<T*>(const_cast<void*>(f.out.p)) + a * f.out.sa + (b0 + j) * f.out.sb, f.scale * v[j] + r[j]);
}

template <typename T, int kBN, int kCG>
__global__ void __launch_bounds__(kThreads, 1)
k_linear_tc(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ TcArgs g) {
  using S = Shape<kBN, kCG>;
  constexpr bool kPlanes = sizeof(T) == 4;
  constexpr int kHalf = kBN / 2;                         // columns of a tile that an epilogue warp reads back
  extern __shared__ unsigned char dyn[];
  __shared__ __align__(8) uint64_t s_full[S::kStages], s_empty[S::kStages], s_tfull[2], s_tempty[2];
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
    if (lane == 0) {
      uint32_t n = 0;                                    // stages filled so far
      bool ok = true;
      const uint32_t bytes = (uint32_t)(S::kABytes + (g.b_rows_inner ? (S::kCols < 64 ? 64 : S::kCols) : S::kCols) * 128);
      for (int i = first; i < n_items && ok; i += stride) {
        const Item w = item_of(g, i, split);
        const int a0 = w.ta * kRows * kCG + (kCG == 2 ? (int)rank * kRows : 0), b0 = w.tb * kBN + (kCG == 2 ? (int)rank * S::kCols : 0);
        const int seg = kPlanes ? kSegment : w.k1 - w.k0;
        for (int k = w.k0; k < w.k1 && ok; k += seg) {
          const int len = min(seg, w.k1 - k), steps = len * (kPlanes ? kProducts : 1);
          for (int it = 0; it < steps; ++it, ++n) {
            const uint32_t s = n % S::kStages;
            ok = !s_abort && mbar_wait(empty + 8 * s, ((n / S::kStages) & 1u) ^ 1u, limit);
            if (!ok) break;
            if (g.stall) continue;                       // (withheld: the consumers' waits run out)
            const Step st = step_of<kPlanes>(k, len, it);
            const uint32_t bar = kCG == 2 ? mapa(full + 8 * s, 0) : full + 8 * s;
            if (leader) mbar_expect(full + 8 * s, bytes * kCG);
            const uint32_t sa = tiles + s * S::kStageBytes, sb = sa + S::kABytes;
            if (g.a_rows_inner) {
              tma_load<kCG>(sa, &map_a, a0, st.kb * kBlockK, st.pa, bar);
              tma_load<kCG>(sa + 8192, &map_a, a0 + 64, st.kb * kBlockK, st.pa, bar);
            } else {
              tma_load<kCG>(sa, &map_a, st.kb * kBlockK, a0, st.pa, bar);
            }
            if (g.b_rows_inner) {
#pragma unroll
              for (int c = 0; c < (S::kCols < 64 ? 1 : S::kCols / 64); ++c)
                tma_load<kCG>(sb + c * 8192, &map_b, b0 + c * 64, st.kb * kBlockK, st.pb, bar);
            } else {
              tma_load<kCG>(sb, &map_b, st.kb * kBlockK, b0, st.pb, bar);
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
    if (lane == 0 && leader) {
      const uint32_t idesc = (1u << 4) | ((uint32_t)g.bf16 << 7) | ((uint32_t)g.bf16 << 10) | ((uint32_t)g.a_rows_inner << 15) |
                             ((uint32_t)g.b_rows_inner << 16) | ((uint32_t)(kBN >> 3) << 17) | ((uint32_t)(kRows * kCG >> 4) << 24);
      const uint32_t adv_a = g.a_rows_inner ? 128 : 2, adv_b = g.b_rows_inner ? 128 : 2;      // 16 k on, in units of 16 bytes
      uint32_t n = 0, u = 0;                             // stages read; accumulators filled
      bool ok = true;
      for (int i = first; i < n_items && ok; i += stride) {
        const Item w = item_of(g, i, split);
        const int seg = kPlanes ? kSegment : w.k1 - w.k0;
        for (int k = w.k0; k < w.k1 && ok; k += seg, ++u) {
          const int steps = min(seg, w.k1 - k) * (kPlanes ? kProducts : 1);
          ok = !s_abort && mbar_wait(tempty + 8 * (u & 1u), ((u >> 1) & 1u) ^ 1u, limit);
          if (!ok) break;
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          const uint32_t d = tmem + (u & 1u) * kBN;
          for (int it = 0; it < steps; ++it, ++n) {
            const uint32_t s = n % S::kStages;
            ok = !s_abort && mbar_wait(full + 8 * s, (n / S::kStages) & 1u, limit);
            if (!ok) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint32_t sa = tiles + s * S::kStageBytes;
            const uint64_t da = umma_desc(sa, g.a_rows_inner), db = umma_desc(sa + S::kABytes, g.b_rows_inner);
#pragma unroll
            for (int j = 0; j < kBlockK / 16; ++j)
              umma<kCG>(d, da + (uint64_t)(j * adv_a), db + (uint64_t)(j * adv_b), idesc, it > 0 || j > 0);
            umma_commit<kCG>(empty + 8 * s);
          }
          if (!ok) break;
          umma_commit<kCG>(tfull + 8 * (u & 1u));
        }
      }
      if (!ok) { s_abort = 1; atomicOr(g.status, STRADS_STATUS_WAIT_EXPIRED); }
    }
    __syncwarp();
  } else {
    const int quarter = warp & 3, half = warp >> 2;      // tensor memory lanes 32 quarter .. , columns half * kHalf ..
    const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
    uint32_t u = 0;
    bool ok = true;
    for (int i = first; i < n_items && ok; i += stride) {
      const Item w = item_of(g, i, split);
      const long long a = (long long)w.ta * kRows * kCG + (kCG == 2 ? (int)rank * kRows : 0) + quarter * 32 + lane;
      const long long b0 = (long long)w.tb * kBN + half * kHalf;
      const int seg = kPlanes ? kSegment : w.k1 - w.k0;
      float acc[kPlanes ? kHalf : 16];
      if (kPlanes)
#pragma unroll
        for (int j = 0; j < kHalf; ++j) acc[j] = 0.f;
      for (int k = w.k0; k < w.k1 && ok; k += seg, ++u) {
        ok = !s_abort && mbar_wait(tfull + 8 * (u & 1u), (u >> 1) & 1u, limit);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const uint32_t d = tmem + (u & 1u) * kBN + lanes + half * kHalf;
#pragma unroll
        for (int c = 0; c < kHalf / 16; ++c) {
          uint32_t v[16];
          __syncwarp();
          tmem_load16(d + c * 16, v);
          tmem_wait();
          if (kPlanes) {
#pragma unroll
            for (int j = 0; j < 16; ++j) acc[c * 16 + j] += __uint_as_float(v[j]);
          } else if (g.splits == 1) {
#pragma unroll
            for (int j = 0; j < 16; ++j) acc[j] = __uint_as_float(v[j]);
            if (a < g.na) finish16<T>(g.f, acc, a, b0 + c * 16, g.nb);
          } else {
#pragma unroll
            for (int j = 0; j < 16; ++j)                 // (the ring is drained: all of it has been read by the MMAs)
              asm volatile("st.shared.f32 [%0], %1;" ::"r"(tiles + (uint32_t)(((half * kHalf + c * 16 + j) * kRows + quarter * 32 + lane) * 4)),
                           "f"(__uint_as_float(v[j])) : "memory");
          }
        }
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster(mapa(tempty + 8 * (u & 1u), kCG == 2 ? 0 : rank));
      }
      if (kPlanes && ok) {
#pragma unroll
        for (int c = 0; c < kHalf / 16; ++c) {
          if (g.splits == 1) {
            if (a < g.na) finish16<T>(g.f, acc + c * 16, a, b0 + c * 16, g.nb);
          } else {
#pragma unroll
            for (int j = 0; j < 16; ++j)
              asm volatile("st.shared.f32 [%0], %1;" ::"r"(tiles + (uint32_t)(((half * kHalf + c * 16 + j) * kRows + quarter * 32 + lane) * 4)),
                           "f"(acc[c * 16 + j]) : "memory");
          }
        }
      }
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
      for (int col = split * 2 + (int)(threadIdx.x >> 7); col < kBN; col += 2 * g.splits) {
        const long long b = (long long)w.tb * kBN + col;
        if (a >= g.na || b >= g.nb) continue;
        float z = 0.f;
        for (int sp = 0; sp < g.splits; ++sp) {
          float v;
          asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(mapa(tiles + (uint32_t)((col * kRows + row) * 4), (uint32_t)sp)) : "memory");
          z += v;
        }
        finish<T>(g.f, z, a, b);
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

using EncodeFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                              const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// What is asked of the driver once per process and device.
struct Device { bool known; int sms; int pairs; int most[9]; };      // most[n]: clusters of n CTAs that fit at once
constexpr int kMaxDevices = 64;
std::mutex g_mutex;
EncodeFn g_encode;
Device g_device[kMaxDevices];

template <typename K>
cudaError_t allow_smem(K kernel, size_t bytes) {
  return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
}
template <typename T>
cudaError_t allow_all() {
  cudaError_t e = allow_smem(k_linear_tc<T, 256, 2>, Shape<256, 2>::kSmem);
  if (e == cudaSuccess) e = allow_smem(k_linear_tc<T, 128, 1>, Shape<128, 1>::kSmem);
  if (e == cudaSuccess) e = allow_smem(k_linear_tc<T, 64, 1>, Shape<64, 1>::kSmem);
  if (e == cudaSuccess) e = allow_smem(k_linear_tc<T, 32, 1>, Shape<32, 1>::kSmem);
  return e;
}
template <typename K>
int clusters_that_fit(K kernel, int size, size_t smem) {
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)size; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)size * 64); cfg.blockDim = dim3(kThreads); cfg.dynamicSmemBytes = smem;
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
    if (g_encode == nullptr) {
      void* fn = nullptr;
      cudaDriverEntryPointQueryResult qres;
      if ((e = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &qres)) != cudaSuccess) return e;
      if (fn == nullptr || qres != cudaDriverEntryPointSuccess) return cudaErrorNotSupported;
      g_encode = reinterpret_cast<EncodeFn>(fn);
    }
    if ((e = cudaDeviceGetAttribute(&d.sms, cudaDevAttrMultiProcessorCount, dev)) != cudaSuccess) return e;
    if ((e = allow_all<float>()) != cudaSuccess || (e = allow_all<__nv_bfloat16>()) != cudaSuccess || (e = allow_all<__half>()) != cudaSuccess) return e;
    d.pairs = clusters_that_fit(k_linear_tc<__nv_bfloat16, 256, 2>, 2, Shape<256, 2>::kSmem);
    if (d.pairs < 1) return cudaErrorNotSupported;
    for (int n = 2; n <= 8; ++n) d.most[n] = clusters_that_fit(k_linear_tc<__nv_bfloat16, 128, 1>, n, Shape<128, 1>::kSmem);
    d.known = true;
  }
  *out = &d;
  return cudaSuccess;
}

// box: {64, rows} where k runs through memory, {64, 64} where the rows do.
bool encode(CUtensorMap* map, const Planes& m, bool bf16, int box_rows) {
  const cuuint64_t dims[3] = {(cuuint64_t)m.inner, (cuuint64_t)m.outer, (cuuint64_t)m.planes};
  const cuuint64_t pitch = (cuuint64_t)m.ld * 2, plane = m.planes > 1 ? (cuuint64_t)m.plane * 2 : pitch;
  const cuuint64_t strides[2] = {pitch, plane};
  const cuuint32_t box[3] = {(cuuint32_t)kBlockK, (cuuint32_t)(m.rows_inner ? kBlockK : box_rows), 1};
  const cuuint32_t estr[3] = {1, 1, 1};
  return g_encode(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<void*>(m.p), dims, strides, box,
                  estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename T, int kBN, int kCG>
cudaError_t launch(const Planes& A, const Planes& B, TcArgs g, unsigned ctas, cudaStream_t s) {
  using S = Shape<kBN, kCG>;
  alignas(64) CUtensorMap ma, mb;
  if (!encode(&ma, A, g.bf16, kRows) || !encode(&mb, B, g.bf16, S::kCols)) return cudaErrorInvalidValue;
  return launch_chained_cluster(k_linear_tc<T, kBN, kCG>, ctas, kThreads, S::kSmem, s, kCG == 2 ? 2 : g.splits, ma, mb, g);
}

int ceil_div(long long a, long long b) { return (int)((a + b - 1) / b); }

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
  // few tiles: as many CTAs to a tile as the GPU holds at once, each with two stages' worth of k at least
  if (n * 2 <= d.sms)
    for (int size = 8; size >= 2; --size)
      if (d.most[size] >= n && size * 2 <= g.blocks) { g.splits = size; break; }
  const unsigned ctas = g.splits > 1 ? (unsigned)n * g.splits : (unsigned)(n < d.sms ? n : d.sms);
  if (bn == 128) return launch<T, 128, 1>(A, B, g, ctas, s);
  if (bn == 64) return launch<T, 64, 1>(A, B, g, ctas, s);
  return launch<T, 32, 1>(A, B, g, ctas, s);
}

}  // namespace

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
