// binary32 products with few rows on one side (5 to 128): the margins of a path of fits, a gradient for some responses.  Bound by
// reading the long side once, so it is read where it is, 4 bytes an element, and split into three bfloat16 planes on its way into
// shared memory; the short side comes as planes in memory (a few hundred rows at most, written by the pass before).
//
// A tile is 128 rows of the long side by kBN = 32 or 64 of the short one.  Eight warps load a tile's block of 64 k (two blocks ahead, in
// registers), split it and store it in the layout that the tensor cores read (128-byte swizzle; rows or k along memory, as in global
// memory); one thread brings the short side's block by TMA; one issues the six largest of the nine products of planes, smallest first;
// four warps empty the accumulator into registers every kSegment blocks (the tensor cores' additions truncate) and add there.
//
// The blocks of all tiles, one tile after another, are dealt out evenly: every CTA takes a run of them, so that all SMs finish together
// however the tiles divide.  A tile that falls to more than one CTA is left as partial sums in the workspace and finished by a second kernel, in the
// order of the CTAs.  Waits are bounded as in linear_tc.cu.
#include "linear_tc.cuh"
#include "linear_ptx.cuh"

namespace strads {
namespace {

constexpr int kRows = 128, kBlockK = 64, kPlane = 16384, kShortPlane = 8192, kStageBytes = 3 * (kPlane + kShortPlane), kStages = 3;
constexpr int kEpiWarps = 4, kLoadWarps = 8, kTmaWarp = 12, kMmaWarp = 13, kThreads = 32 * 14;
constexpr int kLoadThreads = 32 * kLoadWarps, kGroups = kRows * kBlockK / 8 / kLoadThreads;      // groups of 8 neighbours per thread and block
constexpr int kSegment = 4;
constexpr int kMostCtas = 148;           // (a GPU with fewer SMs takes them in turn)
constexpr size_t kSmem = (size_t)kStages * kStageBytes + 1024;

struct SplitArgs {
  Operand L;
  long long nk;
  int nl, ns, blocks, tiles_l, tiles_s, ctas;
  int l_rows_inner, s_rows_inner, vec, long_is_b, stall;
  float* partial;                        // [2 ctas][kBN][128]
  unsigned int* status;
  Finish f;
};

// Blocks [first, last) of the whole run of tiles that CTA c takes.
__device__ __forceinline__ long long start_of(const SplitArgs& g, int c) { return (long long)g.tiles_l * g.tiles_s * g.blocks * c / g.ctas; }
// Tiles of one part of the long side follow each other: the second finds it in L2.
__device__ __forceinline__ void tile_of(const SplitArgs& g, int t, int* tl, int* ts) { *tl = t / g.tiles_s; *ts = t % g.tiles_s; }
__device__ __forceinline__ void finish_split(const SplitArgs& g, float v, long long l, long long s) {
  if (g.long_is_b) finish<float>(g.f, v, s, l); else finish<float>(g.f, v, l, s);
}

struct Held { float x[kGroups][8]; };    // what a loading thread holds of a block

template <int kBN>
__global__ void __launch_bounds__(kThreads, 1) k_linear_split(const __grid_constant__ CUtensorMap map_s, const __grid_constant__ SplitArgs g) {
  extern __shared__ unsigned char dyn[];
  __shared__ __align__(8) uint64_t s_full[kStages], s_empty[kStages], s_tfull[2], s_tempty[2];
  __shared__ uint32_t s_tmem;
  __shared__ volatile int s_abort;
  constexpr uint32_t kTmemCols = 2 * kBN;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t tiles = (smem_u32(dyn) + 1023u) & ~1023u;
  const uint32_t full = smem_u32(s_full), empty = smem_u32(s_empty), tfull = smem_u32(s_tfull), tempty = smem_u32(s_tempty);
  const uint32_t limit = g.stall ? kMmaStallLimit : kMmaWaitLimit;
  if (threadIdx.x == 0) {
    s_abort = 0;
    for (int i = 0; i < kStages; ++i) { mbar_init(full + 8 * i, kLoadWarps + 1); mbar_init(empty + 8 * i, 1); }
    for (int i = 0; i < 2; ++i) { mbar_init(tfull + 8 * i, 1); mbar_init(tempty + 8 * i, kEpiWarps); }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_s) : "memory");
  }
  if (warp == kMmaWarp) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&s_tmem)), "r"(kTmemCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem = s_tmem;
  chain_begin();
  const long long u0 = start_of(g, (int)blockIdx.x), u1 = start_of(g, (int)blockIdx.x + 1);

  if (warp >= kEpiWarps && warp < kEpiWarps + kLoadWarps) {
    const int t = (int)threadIdx.x - 32 * kEpiWarps;
    bool ok = true;
    auto load = [&](long long u, Held& h) {
      int tl, ts;
      tile_of(g, (int)(u / g.blocks), &tl, &ts);
      const long long l0 = (long long)tl * kRows, k0 = u % g.blocks * kBlockK;
#pragma unroll
      for (int i = 0; i < kGroups; ++i) {
        const int q = t + i * kLoadThreads;
        // eight neighbours of one row (k along memory: 8 groups a row) or one k (rows along memory: 16 groups)
        const long long l = l0 + (g.l_rows_inner ? q % 16 * 8 : q / 8), k = k0 + (g.l_rows_inner ? q / 16 : q % 8 * 8);
        const long long left = (g.l_rows_inner ? g.nl - l : g.nk - k);
        const float* p = static_cast<const float*>(g.L.p) + l * g.L.rs + k * g.L.ks;
        const bool there = g.l_rows_inner ? k < g.nk : l < g.nl;
        if (g.vec && there && left >= 8) {
#pragma unroll
          for (int j = 0; j < 8; j += 4)
            asm volatile("ld.global.nc.L1::no_allocate.v4.f32 {%0, %1, %2, %3}, [%4];"
                         : "=f"(h.x[i][j]), "=f"(h.x[i][j + 1]), "=f"(h.x[i][j + 2]), "=f"(h.x[i][j + 3]) : "l"(p + j));
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j) h.x[i][j] = there && j < left ? __ldg(p + j) : 0.f;
        }
      }
    };
    auto store = [&](long long n, const Held& h) {
      const uint32_t s = (uint32_t)(n % kStages), at = tiles + s * kStageBytes;
      ok = !s_abort && mbar_wait(empty + 8 * s, ((uint32_t)(n / kStages) & 1u) ^ 1u, limit);
      ok = __all_sync(0xffffffffu, ok) && !g.stall;
      if (!ok) return;
#pragma unroll
      for (int i = 0; i < kGroups; ++i) {
        const int q = t + i * kLoadThreads;
        const uint32_t place = g.l_rows_inner ? (uint32_t)((q % 16 / 8) * 8192 + (q / 16) * 128 + (((q % 8) ^ (q / 16 % 8)) << 4))
                                              : (uint32_t)((q / 8) * 128 + (((q % 8) ^ (q / 8 % 8)) << 4));
        uint32_t w[4][3];
#pragma unroll
        for (int j = 0; j < 4; ++j) split_pair(h.x[i][2 * j], h.x[i][2 * j + 1], w[j]);
#pragma unroll
        for (int p = 0; p < 3; ++p)
          asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at + p * kPlane + place), "r"(w[0][p]), "r"(w[1][p]), "r"(w[2][p]), "r"(w[3][p]) : "memory");
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane == 0) asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(full + 8 * s) : "memory");
    };
    Held a, b;
    if (u0 < u1) load(u0, a);
    if (u0 + 1 < u1) load(u0 + 1, b);
    for (long long u = u0; u < u1 && ok; u += 2) {
      store(u - u0, a);
      if (u + 2 < u1) load(u + 2, a);
      if (ok && u + 1 < u1) {
        store(u + 1 - u0, b);
        if (u + 3 < u1) load(u + 3, b);
      }
    }
    if (!ok && lane == 0) { s_abort = 1; atomicOr(g.status, STRADS_STATUS_WAIT_EXPIRED); }
    __syncwarp();
  } else if (warp == kTmaWarp) {
    if (lane == 0) {
      bool ok = true;
      const uint32_t bytes = 3u * (uint32_t)((g.s_rows_inner ? 64 : kBN) * 128);
      long long n = 0;
      for (long long u = u0; u < u1; ++u, ++n) {
        const uint32_t s = (uint32_t)(n % kStages);
        ok = !s_abort && mbar_wait(empty + 8 * s, ((uint32_t)(n / kStages) & 1u) ^ 1u, limit) && !g.stall;
        if (!ok) break;
        int tl, ts;
        tile_of(g, (int)(u / g.blocks), &tl, &ts);
        const int k0 = (int)(u % g.blocks) * kBlockK, r0 = ts * kBN;
        mbar_expect(full + 8 * s, bytes);
#pragma unroll
        for (int p = 0; p < 3; ++p)
          tma_load<1>(tiles + s * kStageBytes + 3 * kPlane + p * kShortPlane, &map_s, g.s_rows_inner ? r0 : k0, g.s_rows_inner ? k0 : r0, p, full + 8 * s);
      }
      if (!ok) { s_abort = 1; atomicOr(g.status, STRADS_STATUS_WAIT_EXPIRED); }
      // every stage filled is read by the MMAs before the shared memory goes; having given up, what is under way gets its time to land
      for (long long j = n > kStages ? n - kStages : 0; j < n; ++j)
        if (!mbar_wait((ok ? empty : full) + 8 * (uint32_t)(j % kStages), (uint32_t)(j / kStages) & 1u, limit)) {
          if (ok) { s_abort = 1; atomicOr(g.status, STRADS_STATUS_WAIT_EXPIRED); }
          break;
        }
    }
    __syncwarp();
  } else if (warp == kMmaWarp) {
    if (lane == 0) {
      const uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)g.l_rows_inner << 15) | ((uint32_t)g.s_rows_inner << 16) |
                             ((uint32_t)(kBN >> 3) << 17) | ((uint32_t)(kRows >> 4) << 24);
      const uint32_t adv_a = g.l_rows_inner ? 128 : 2, adv_b = g.s_rows_inner ? 128 : 2;
      bool ok = true;
      long long n = 0;
      uint32_t v = 0;
      for (long long u = u0; u < u1 && ok; ++v) {
        // a segment: up to kSegment blocks of one tile
        const int len = (int)min(min((long long)kSegment, u1 - u), g.blocks - u % g.blocks);
        ok = !s_abort && mbar_wait(tempty + 8 * (v & 1u), ((v >> 1) & 1u) ^ 1u, limit);
        if (!ok) break;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const uint32_t d = tmem + (v & 1u) * kBN;
        for (int i = 0; i < len; ++i, ++n) {
          const uint32_t s = (uint32_t)(n % kStages);
          ok = !s_abort && mbar_wait(full + 8 * s, (uint32_t)(n / kStages) & 1u, limit);
          if (!ok) break;
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          const uint32_t at = tiles + s * kStageBytes;
#pragma unroll
          for (int q = 0; q < 6; ++q) {
            const uint64_t da = umma_desc(at + ((0x201100 >> (4 * (5 - q))) & 3) * kPlane, g.l_rows_inner),
                           db = umma_desc(at + 3 * kPlane + ((0x021010 >> (4 * (5 - q))) & 3) * kShortPlane, g.s_rows_inner);
#pragma unroll
            for (int j = 0; j < kBlockK / 16; ++j)
              umma<1>(d, da + (uint64_t)(j * adv_a), db + (uint64_t)(j * adv_b), idesc, i > 0 || q > 0 || j > 0);
          }
          umma_commit<1>(empty + 8 * s);
        }
        if (!ok) break;
        umma_commit<1>(tfull + 8 * (v & 1u));
        u += len;
      }
      if (!ok) { s_abort = 1; atomicOr(g.status, STRADS_STATUS_WAIT_EXPIRED); }
    }
    __syncwarp();
  } else {
    bool ok = true;
    uint32_t v = 0;
    for (long long u = u0; u < u1 && ok;) {
      // a piece: this CTA's blocks of one tile
      const int t = (int)(u / g.blocks);
      const long long end = min(u1, (long long)(t + 1) * g.blocks);
      const bool whole = end - u == g.blocks;
      float acc[kBN];
#pragma unroll
      for (int j = 0; j < kBN; ++j) acc[j] = 0.f;
      for (long long k = u; k < end && ok; k += kSegment, ++v) {
        ok = !s_abort && mbar_wait(tfull + 8 * (v & 1u), (v >> 1) & 1u, limit);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll
        for (int c = 0; c < kBN / 16; ++c) {
          uint32_t r[16];
          tmem_load16(tmem + (v & 1u) * kBN + c * 16 + ((uint32_t)(warp * 32) << 16), r);
          tmem_wait();
#pragma unroll
          for (int j = 0; j < 16; ++j) acc[c * 16 + j] += __uint_as_float(r[j]);
        }
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        __syncwarp();
        if (lane == 0) asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(tempty + 8 * (v & 1u)) : "memory");
      }
      if (!ok) break;
      int tl, ts;
      tile_of(g, t, &tl, &ts);
      const int row = warp * 32 + lane;
      const long long l = (long long)tl * kRows + row;
      if (whole) {
        if (l < g.nl)
#pragma unroll
          for (int j = 0; j < kBN; ++j)
            if (ts * kBN + j < g.ns) finish_split(g, acc[j], l, ts * kBN + j);
      } else {
        float* p = g.partial + ((long long)(2 * blockIdx.x + (u == u0 ? 0 : 1)) * kBN) * kRows + row;
#pragma unroll
        for (int j = 0; j < kBN; ++j) p[j * kRows] = acc[j];
      }
      __syncwarp();
      u = end;
    }
    if (!ok && lane == 0) { s_abort = 1; atomicOr(g.status, STRADS_STATUS_WAIT_EXPIRED); }
    __syncwarp();
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  if (warp == kMmaWarp) {
    __syncwarp();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
  }
}

// Tiles that fell to more than one CTA: a CTA each, adding in the order of the CTAs.
template <int kBN>
__global__ void __launch_bounds__(256) k_linear_split_sum(const __grid_constant__ SplitArgs g) {
  chain_begin();
  const int t = blockIdx.x;
  const long long b0 = (long long)t * g.blocks, b1 = b0 + g.blocks;
  // the CTA that holds the tile's first block: near b0 ctas / (all blocks)
  int c0 = (int)(b0 * g.ctas / ((long long)g.tiles_l * g.tiles_s * g.blocks));
  while (c0 + 1 < g.ctas && start_of(g, c0 + 1) <= b0) ++c0;
  while (c0 > 0 && start_of(g, c0) > b0) --c0;
  if (start_of(g, c0 + 1) >= b1) return;                 // one CTA had all of it and has finished it
  int tl, ts;
  tile_of(g, t, &tl, &ts);
  for (int i = threadIdx.x; i < kBN * kRows; i += 256) {
    const int col = i / kRows, row = i % kRows;
    const long long l = (long long)tl * kRows + row, s = (long long)ts * kBN + col;
    if (l >= g.nl || s >= g.ns) continue;
    float v = 0.f;
    for (int c = c0; c < g.ctas && start_of(g, c) < b1; ++c) {
      const int slot = 2 * c + (start_of(g, c) >= b0 || start_of(g, c) / g.blocks == t ? 0 : 1);
      v += g.partial[((long long)slot * kBN + col) * kRows + row];
    }
    finish_split(g, v, l, s);
  }
}

int width_of(long long ns) { return ns <= 32 ? 32 : 64; }
int ctas_of(long long nl, long long ns, long long nk) {
  const long long units = (nl + kRows - 1) / kRows * ((ns + width_of(ns) - 1) / width_of(ns)) * ((nk + kBlockK - 1) / kBlockK);
  const long long n = (units + 3) / 4;                   // four blocks each at least
  return (int)(n < kMostCtas ? n : kMostCtas);
}

template <int kBN>
cudaError_t launch(const Planes& S, const SplitArgs& g, cudaStream_t s) {
  alignas(64) CUtensorMap map;
  if (tensor_map_encoder() == nullptr) return cudaErrorNotSupported;
  if (!encode_operand(&map, S, true, kBN)) return cudaErrorInvalidValue;
  cudaError_t e = cudaFuncSetAttribute(k_linear_split<kBN>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmem);
  if (e == cudaSuccess) e = launch_chained(k_linear_split<kBN>, dim3((unsigned)g.ctas), kThreads, kSmem, s, map, g);
  if (e == cudaSuccess && g.ctas > 1) e = launch_chained(k_linear_split_sum<kBN>, dim3((unsigned)(g.tiles_l * g.tiles_s)), 256, 0, s, g);
  return e;
}

}  // namespace

size_t linear_split_workspace(long long nl, long long ns, long long nk) {
  return (size_t)2 * ctas_of(nl, ns, nk) * width_of(ns) * kRows * sizeof(float);
}

cudaError_t launch_linear_split(const Operand& L, const Planes& S, long long nl, long long ns, long long nk, bool long_is_b, const Finish& f,
                                void* workspace, unsigned int* status, bool stall, cudaStream_t s) {
  SplitArgs g = {};
  g.L = L; g.nk = nk; g.nl = (int)nl; g.ns = (int)ns;
  g.blocks = (int)((nk + kBlockK - 1) / kBlockK);
  g.tiles_l = (int)((nl + kRows - 1) / kRows);
  g.tiles_s = (int)((ns + width_of(ns) - 1) / width_of(ns));
  g.ctas = ctas_of(nl, ns, nk);
  g.l_rows_inner = L.ks != 1; g.s_rows_inner = S.rows_inner;
  const long long pitch = g.l_rows_inner ? L.ks : L.rs;
  g.vec = ((uintptr_t)L.p & 15) == 0 && pitch % 4 == 0;
  g.long_is_b = long_is_b; g.stall = stall;
  g.partial = static_cast<float*>(workspace);
  g.status = status; g.f = f;
  return width_of(ns) == 32 ? launch<32>(S, g, s) : launch<64>(S, g, s);
}

}  // namespace strads
