// binary32 products with few rows on one side (5 to 128): the margins of a path of fits, a gradient for some responses.  Bound by
// reading the long side once, so it is read where it is, 4 bytes an element, and split into three bfloat16 planes on its way into
// tensor memory; the short side comes as planes in memory (written by the pass before).
//
// A tile is 128 rows of the long side by kBN = 32 or 48 of the short one (48: 128 registers and 188 bytes spilled).  One thread brings blocks of 64 k by TMA, the long side's as it is (the
// ring holds 160 KB of it: what hides the memory's latency); eight warps, a lane per row, split them and put the planes into tensor
// memory, which the tensor cores take their A operand from: shared memory, whose bandwidth would otherwise bound the kernel, is written and
// read once for every element.  One thread issues the products.  The short side's planes lie one behind the other as rows of B, so three
// MMAs form the six largest of the nine products of planes, sorted by size into three accumulators:
//   L0 [S0 S1 S2] -> [c0 c1 c2],   L1 [S0 S1] -> [c1 c2],   L2 [S0] -> [c2],   D = c0 + (c1 + c2).
// Four warps empty them into registers every kSegment blocks (the tensor cores' additions truncate) and add there.
//
// Every CTA has the same number of blocks, however the tiles divide.  With W CTAs, each first takes whole tiles, the CTAs' tiles side by side; of the R
// tiles left, CTAs 0 .. R - 1 take n1 = R B / W of the B blocks of one each, spread evenly over k, and the other W - R what is left of them.  So at any
// time the CTAs read the same few k of neighbouring rows: runs of blocks of one tile after another, each CTA at a k of its own, read a column-major design
// at 5.1 TB/s, where tiles in step reach 5.6.  The tiles shared are left as partial sums in the workspace and finished by a second kernel, in a
// fixed order.  Waits are bounded as in linear_tc.cu.
#include "linear_tc.cuh"
#include "linear_ptx.cuh"

namespace strads {
namespace {

constexpr int kRows = 128, kBlockK = 64, kLongBytes = kRows * kBlockK * 4;
constexpr int kEpiWarps = 4, kSplitWarps = 8, kTmaWarp = 12, kMmaWarp = 13, kThreads = 32 * 14;
constexpr int kSegment = 4;
constexpr int kMostCtas = 148;           // (a GPU with fewer SMs takes them in turn)

template <int kBN>
struct Sizes {
  static constexpr int kShortBytes = 3 * kBN * 128;
  static constexpr int kStageBytes = kLongBytes + kShortBytes;
  static constexpr int kStages = (227 * 1024 - 2048) / kStageBytes;
  static constexpr size_t kSmem = (size_t)kStages * kStageBytes + 1024;
  // tensor memory: two sets of accumulators, then as many of the long side's planes (96 columns each) as fit: with two, splitting waited for the products
  static constexpr uint32_t kD = 3 * kBN, kA = 2 * kD;
  static constexpr int kSets = (512 - (int)kA) / 96;
  static_assert(kSets >= 2 && kShortBytes % 1024 == 0, "");
};

struct SplitArgs {
  int nl, ns, blocks, tiles_l, tiles_s, ctas;
  int rounds, shared, own;               // whole tiles of each CTA; R; n1
  int l_rows_inner, long_is_b, stall;
  float* partial;                        // [ctas + R][kBN][128]
  unsigned int* status;
  Finish f;
};

// Tiles of one part of the long side follow each other: the second finds it in L2.
__device__ __forceinline__ void tile_of(const SplitArgs& g, int t, int* tl, int* ts) { *tl = t / g.tiles_s; *ts = t % g.tiles_s; }
// What the first R CTAs leave of the shared tiles, one tile after another: helper h takes [start, start of h + 1).
__host__ __device__ __forceinline__ long long helper_start(const SplitArgs& g, int h) {
  return (long long)g.shared * (g.blocks - g.own) * h / (g.ctas - g.shared);
}
// Columns s, s + 1, .. of row l (clamped to one that exists; `here`: it does).
template <int kN>
__device__ __forceinline__ void finish_split(const SplitArgs& g, float (&v)[kN], long long l, int s) {
  const bool here = l < g.nl;
  const long long at = here ? l : g.nl - 1;
  const int count = min(kN, g.ns - s);
  if (!g.long_is_b) {
    finish_run<float, kN>(g.f, v, at, s, 1, count, here);
  } else {                                               // (the short side is D's a: its strides change places)
    Finish f = g.f;
    f.out = {g.f.out.p, g.f.out.sb, g.f.out.sa};
    f.residual = {g.f.residual.p, g.f.residual.sb, g.f.residual.sa};
    f.preact = {g.f.preact.p, g.f.preact.sb, g.f.preact.sa};
    f.bias_a = g.f.bias_b; f.bias_b = g.f.bias_a;
    finish_run<float, kN>(f, v, at, s, 1, count, here);
  }
}
// A CTA's blocks, piece by piece: a piece is some or all blocks of one tile.
struct Walk {
  int round, tile, len, at;              // at: blocks of the piece gone through
  int slot;                              // where its sums go (-1: it has the whole tile)
  long long rest, from, end;             // helpers: where they are in what is left of the shared tiles; the piece's first block there; their end
  __device__ __forceinline__ Walk(const SplitArgs& g, int c) : round(-1), rest(0), end(0) {
    if (c >= g.shared) { rest = helper_start(g, c - g.shared); end = helper_start(g, c - g.shared + 1); }
    next_piece(g, c);
  }
  __device__ __forceinline__ void next_piece(const SplitArgs& g, int c) {      // len 0: no more
    ++round;
    at = 0;
    if (round < g.rounds) {
      tile = round * g.ctas + c; len = g.blocks; slot = -1;
    } else if (c < g.shared) {
      len = round == g.rounds ? g.own : 0;
      tile = g.rounds * g.ctas + c; slot = g.own == g.blocks ? -1 : c;
    } else if (rest < end) {
      const int left = g.blocks - g.own, t = (int)(rest / left);
      from = rest - (long long)t * left;
      len = (int)min((long long)left - from, end - rest);
      tile = g.rounds * g.ctas + t; slot = g.shared + t + (c - g.shared);
      rest += len;
    } else {
      len = 0;
    }
  }
};
// Which of a tile's blocks a piece has, one after the other.  k along memory: the first n1 are dealt out first, and what follows is what is left, so that a
// CTA reads on in its rows (10,000 x 100,000 by 20: 675 us, 780 spread).  Rows along memory: the i-th of the n1 is floor(i B / n1); of the others, the one
// that as many of them precede: where a piece begins by division, from there on by counting.
struct Order {
  int k, step, rem, own, next, err;      // the block; floor(B / n1) and what it leaves; the next of the n1, and the remainder there
  bool whole, first;
  __device__ __forceinline__ Order(const SplitArgs& g, const Walk& w, int c) : k(0), step(1), rem(0), own(g.own), next(0), err(0), whole(w.slot < 0 || !g.l_rows_inner), first(c < g.shared) {
    if (w.slot >= 0 && !g.l_rows_inner && !first) k = own + (int)w.from;
    if (whole || w.len == 0) return;
    step = g.blocks / own; rem = g.blocks % own;
    if (first) return;
    const long long B = g.blocks, n1 = own, i = w.from + 1;
    long long m = i * B / (B - n1);                      // m - ceil(m n1 / B) of the first m blocks are among the others: the least m with i of them
    while (m - (m * n1 + B - 1) / B < i) ++m;
    while (m > 1 && m - 1 - ((m - 1) * n1 + B - 1) / B >= i) --m;
    k = (int)(m - 1);
    const long long j = ((long long)k * n1 + B - 1) / B;
    next = (int)(j * B / n1); err = (int)(j * B % n1);
  }
  __device__ __forceinline__ void advance() {
    if (whole) { ++k; return; }
    if (first) { k = hop(k); return; }
    for (++k; k == next; ++k) next = hop(next);
  }
  __device__ __forceinline__ int hop(int p) {
    p += step;
    if ((err += rem) >= own) { err -= own; ++p; }
    return p;
  }
};

__device__ __forceinline__ void tma_load_raw(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
               ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}
// D (+)= A[tensor memory] B[shared memory]^T, K = 16: eight columns of A, two k in each.
__device__ __forceinline__ void umma_a_tmem(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
               ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void tmem_store16(uint32_t taddr, const uint32_t (&v)[16]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
               ::"r"(taddr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]),
                 "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]) : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }

template <int kBN>
__global__ void __launch_bounds__(kThreads, 1)
k_linear_split(const __grid_constant__ CUtensorMap map_l, const __grid_constant__ CUtensorMap map_s, const __grid_constant__ SplitArgs g) {
  using Z = Sizes<kBN>;
  constexpr int kStages = Z::kStages;
  extern __shared__ unsigned char dyn[];
  __shared__ __align__(8) uint64_t s_full[kStages], s_empty[kStages], s_sfull[kStages], s_sempty[kStages], s_afull[Z::kSets], s_aempty[Z::kSets], s_tfull[2], s_tempty[2];
  __shared__ uint32_t s_tmem;
  __shared__ volatile int s_abort;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t ring = (smem_u32(dyn) + 1023u) & ~1023u, shorts = ring + kStages * kLongBytes;
  const uint32_t full = smem_u32(s_full), empty = smem_u32(s_empty), sfull = smem_u32(s_sfull), sempty = smem_u32(s_sempty), afull = smem_u32(s_afull), aempty = smem_u32(s_aempty), tfull = smem_u32(s_tfull),
                 tempty = smem_u32(s_tempty);
  const uint32_t limit = g.stall ? kMmaStallLimit : kMmaWaitLimit;
  if (threadIdx.x == 0) {
    s_abort = 0;
    for (int i = 0; i < kStages; ++i) {
      mbar_init(full + 8 * i, 1); mbar_init(empty + 8 * i, kSplitWarps / 2);
      mbar_init(sfull + 8 * i, 1); mbar_init(sempty + 8 * i, 1);
    }
    for (int i = 0; i < Z::kSets; ++i) { mbar_init(afull + 8 * i, kSplitWarps / 2); mbar_init(aempty + 8 * i, 1); }
    for (int i = 0; i < 2; ++i) { mbar_init(tfull + 8 * i, 1); mbar_init(tempty + 8 * i, kEpiWarps); }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_l) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_s) : "memory");
  }
  if (warp == kMmaWarp) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&s_tmem)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem = s_tmem;
  chain_begin();
  const int cta = (int)blockIdx.x;
  Walk at(g, cta);

  if (warp == kTmaWarp) {
    if (elect_one()) {
      bool ok = true;
      int n = 0;
      Order order(g, at, cta);
      int tl, ts;
      tile_of(g, at.tile, &tl, &ts);
      for (; at.len > 0; ++n) {
        // the long side's ring is free again when a block has been split, the short side's when the products have read it
        const uint32_t s = (uint32_t)(n % kStages), parity = ((uint32_t)(n / kStages) & 1u) ^ 1u, to = ring + s * kLongBytes;
        ok = !s_abort && mbar_wait(empty + 8 * s, parity, limit) && !g.stall;
        if (!ok) break;
        const int k0 = order.k * kBlockK, l0 = tl * kRows;
        mbar_expect(full + 8 * s, (uint32_t)kLongBytes);
        if (g.l_rows_inner) {
          tma_load_raw(to, &map_l, l0, k0, full + 8 * s);
        } else {
          tma_load_raw(to, &map_l, k0, l0, full + 8 * s);
          tma_load_raw(to + kLongBytes / 2, &map_l, k0 + 32, l0, full + 8 * s);
        }
        ok = mbar_wait(sempty + 8 * s, parity, limit);
        if (!ok) { ++n; break; }                         // (the long side's load is under way all the same)
        mbar_expect(sfull + 8 * s, (uint32_t)Z::kShortBytes);
#pragma unroll
        for (int p = 0; p < 3; ++p) tma_load<1>(shorts + s * Z::kShortBytes + p * kBN * 128, &map_s, k0, ts * kBN, p, sfull + 8 * s);
        order.advance();
        if (++at.at == at.len) {
          at.next_piece(g, cta);
          order = Order(g, at, cta);
          tile_of(g, at.tile, &tl, &ts);
        }
      }
      if (!ok) { s_abort = 1; atomicOr(g.status, STRADS_STATUS_WAIT_EXPIRED); }
      // every stage filled is used up before the shared memory goes; having given up, what is under way gets its time to land
      for (int j = n > kStages ? n - kStages : 0; j < n; ++j) {
        const uint32_t at8 = 8 * (uint32_t)(j % kStages), parity = (uint32_t)(j / kStages) & 1u;
        if (!mbar_wait((ok ? empty : full) + at8, parity, limit) || !mbar_wait((ok ? sempty : sfull) + at8, parity, limit)) {
          if (ok) { s_abort = 1; atomicOr(g.status, STRADS_STATUS_WAIT_EXPIRED); }
          break;
        }
      }
    }
    __syncwarp();
  } else if (warp >= kEpiWarps && warp < kEpiWarps + kSplitWarps) {
    const int run = g.rounds * g.blocks + (cta < g.shared ? g.own : g.shared > 0 ? (int)(at.end - helper_start(g, cta - g.shared)) : 0);
    // two groups of four warps, a block each in turn, so that the latencies of one overlap the other's work; a lane per row
    const int row = (warp & 3) * 32 + lane, group = (warp - kEpiWarps) >> 2;
    bool ok = true;
    for (int n = group; n < run; n += 2) {
      const uint32_t s = (uint32_t)(n % kStages), from = ring + s * kLongBytes;
      const uint32_t b = (uint32_t)(n % Z::kSets);
      ok = !s_abort && mbar_wait(full + 8 * s, (uint32_t)(n / kStages) & 1u, limit) &&
           mbar_wait(aempty + 8 * b, ((uint32_t)(n / Z::kSets) & 1u) ^ 1u, limit);
      if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      const uint32_t to = tmem + Z::kA + b * 96 + ((uint32_t)((warp & 3) * 32) << 16);
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        uint32_t p0[16], p1[16], p2[16];
        if (g.l_rows_inner) {
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            float x, y;
            const uint32_t q = from + (uint32_t)((half * 32 + 2 * j) * kRows + row) * 4;
            asm volatile("ld.shared.f32 %0, [%1];" : "=f"(x) : "r"(q) : "memory");
            asm volatile("ld.shared.f32 %0, [%1];" : "=f"(y) : "r"(q + kRows * 4) : "memory");
            uint32_t w[3];
            split_pair(x, y, w);
            p0[j] = w[0]; p1[j] = w[1]; p2[j] = w[2];
          }
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            float4 v;
            const uint32_t q = from + half * (kLongBytes / 2) + row * 128 + ((j ^ (row & 7)) << 4);
            asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(q) : "memory");
            uint32_t w[3];
            split_pair(v.x, v.y, w);
            p0[2 * j] = w[0]; p1[2 * j] = w[1]; p2[2 * j] = w[2];
            split_pair(v.z, v.w, w);
            p0[2 * j + 1] = w[0]; p1[2 * j + 1] = w[1]; p2[2 * j + 1] = w[2];
          }
        }
        __syncwarp();
        tmem_store16(to + half * 16, p0);
        tmem_store16(to + half * 16 + 32, p1);
        tmem_store16(to + half * 16 + 64, p2);
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(empty + 8 * s);         // (all of it has been read into registers)
      asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
      asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
      __syncwarp();
      if (lane == 0) mbar_arrive(afull + 8 * b);
    }
    if (!ok && lane == 0) { s_abort = 1; atomicOr(g.status, STRADS_STATUS_WAIT_EXPIRED); }
    __syncwarp();
  } else if (warp == kMmaWarp) {                         // (the warp as one; an elected lane issues)
    {
      const bool one = elect_one();
      constexpr uint32_t kDesc = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(kRows >> 4) << 24);      // bfloat16, k along memory in B
      bool ok = true;
      uint32_t v = 0;
      int n = 0;
      while (ok && at.len > 0) {
        // a segment: up to kSegment blocks of one piece
        const int len = min(kSegment, at.len - at.at);
        ok = __all_sync(0xffffffffu, !s_abort && mbar_wait(tempty + 8 * (v & 1u), ((v >> 1) & 1u) ^ 1u, limit));
        if (!ok) break;
        const uint32_t d = tmem + (v & 1u) * Z::kD;
        for (int i = 0; i < len; ++i, ++n) {
          const uint32_t s = (uint32_t)(n % kStages), b = (uint32_t)(n % Z::kSets);
          ok = __all_sync(0xffffffffu, !s_abort && mbar_wait(sfull + 8 * s, (uint32_t)(n / kStages) & 1u, limit) &&
                                       mbar_wait(afull + 8 * b, (uint32_t)(n / Z::kSets) & 1u, limit));
          if (!ok) break;
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          const uint64_t db = umma_desc(shorts + s * Z::kShortBytes, false);
          const uint32_t da = tmem + Z::kA + b * 96;
          if (one) {
#pragma unroll
            for (int j = 0; j < kBlockK / 16; ++j) {
              umma_a_tmem(d, da + j * 8, db + (uint64_t)(j * 2), kDesc | ((uint32_t)(3 * kBN >> 3) << 17), i > 0 || j > 0);
              umma_a_tmem(d + kBN, da + 32 + j * 8, db + (uint64_t)(j * 2), kDesc | ((uint32_t)(2 * kBN >> 3) << 17), 1);
              umma_a_tmem(d + 2 * kBN, da + 64 + j * 8, db + (uint64_t)(j * 2), kDesc | ((uint32_t)(kBN >> 3) << 17), 1);
            }
            umma_commit<1>(sempty + 8 * s);
            umma_commit<1>(aempty + 8 * b);
          }
          __syncwarp();
        }
        if (!ok) break;
        if (one) umma_commit<1>(tfull + 8 * (v & 1u));
        __syncwarp();
        ++v;
        if ((at.at += len) == at.len) at.next_piece(g, cta);
      }
      if (!ok && lane == 0) { s_abort = 1; atomicOr(g.status, STRADS_STATUS_WAIT_EXPIRED); }
    }
    __syncwarp();
  } else {
    bool ok = true;
    uint32_t v = 0;
    for (; ok && at.len > 0; at.next_piece(g, cta)) {
      float acc[kBN];
#pragma unroll
      for (int j = 0; j < kBN; ++j) acc[j] = 0.f;
      for (int k = 0; k < at.len && ok; k += kSegment, ++v) {
        ok = !s_abort && mbar_wait(tfull + 8 * (v & 1u), (v >> 1) & 1u, limit);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const uint32_t d = tmem + (v & 1u) * Z::kD + ((uint32_t)(warp * 32) << 16);
#pragma unroll
        for (int c = 0; c < kBN / 16; ++c) {
          uint32_t r0[16], r1[16], r2[16];
          tmem_load16(d + c * 16, r0);
          tmem_load16(d + kBN + c * 16, r1);
          tmem_load16(d + 2 * kBN + c * 16, r2);
          tmem_wait();
#pragma unroll
          for (int j = 0; j < 16; ++j) acc[c * 16 + j] += __uint_as_float(r0[j]) + (__uint_as_float(r1[j]) + __uint_as_float(r2[j]));
        }
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        __syncwarp();
        if (lane == 0) mbar_arrive(tempty + 8 * (v & 1u));
      }
      if (!ok) break;
      int tl, ts;
      tile_of(g, at.tile, &tl, &ts);
      const int row = warp * 32 + lane;
      const long long l = (long long)tl * kRows + row;
      if (at.slot < 0) {
#pragma unroll
        for (int c = 0; c < kBN; c += 16) {
          float z[16];
#pragma unroll
          for (int j = 0; j < 16; ++j) z[j] = acc[c + j];
          if (ts * kBN + c < g.ns) finish_split<16>(g, z, l, ts * kBN + c);
        }
      } else {
        float* p = g.partial + (long long)at.slot * kBN * kRows + row;
#pragma unroll
        for (int j = 0; j < kBN; ++j) p[j * kRows] = acc[j];
      }
      __syncwarp();
    }
    if (!ok && lane == 0) { s_abort = 1; atomicOr(g.status, STRADS_STATUS_WAIT_EXPIRED); }
    __syncwarp();
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  if (warp == kMmaWarp) {
    __syncwarp();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
  }
}

// The shared tiles, eight columns to a CTA: the first CTA's sums, and the helpers' in their order.
template <int kBN>
__global__ void __launch_bounds__(256) k_linear_split_sum(const __grid_constant__ SplitArgs g) {
  chain_begin();
  __shared__ int s_first, s_last;
  __shared__ bool s_any[kMostCtas];                      // (with few blocks left to share, some helpers have none)
  const int t = blockIdx.x;
  if (threadIdx.x == 0) {
    const long long left = g.blocks - g.own, b0 = t * left, b1 = b0 + left;
    // the helper that holds what is left of the tile first: near b0 helpers / (all that is left)
    int h = (int)(b0 * (g.ctas - g.shared) / (left * g.shared));
    while (helper_start(g, h + 1) <= b0) ++h;
    while (h > 0 && helper_start(g, h) > b0) --h;
    s_first = h;
    while (helper_start(g, h + 1) < b1) ++h;
    s_last = h;
  }
  for (int h = threadIdx.x; h < g.ctas - g.shared; h += 256) s_any[h] = helper_start(g, h) < helper_start(g, h + 1);
  __syncthreads();
  int tl, ts;
  tile_of(g, g.rounds * g.ctas + t, &tl, &ts);
  const int row = threadIdx.x & (kRows - 1), col = blockIdx.y * 8 + (threadIdx.x >> 7) * 4;
  if (ts * kBN + col >= g.ns) return;
  float v[4];
  const float* p = g.partial + ((long long)t * kBN + col) * kRows + row;
#pragma unroll
  for (int j = 0; j < 4; ++j) v[j] = p[j * kRows];
  for (int h = s_first; h <= s_last; ++h) {
    if (!s_any[h]) continue;
    p = g.partial + ((long long)(g.shared + t + h) * kBN + col) * kRows + row;
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] += p[j * kRows];
  }
  finish_split<4>(g, v, (long long)tl * kRows + row, ts * kBN + col);
}

// As few tiles along the short side as its width allows (each goes through the long side, the second from L2), the narrower where both make as many.
int width_of(long long ns) { return (ns + 47) / 48 < (ns + 31) / 32 ? 48 : 32; }
int ctas_of(long long nl, long long ns, long long nk) {
  const long long units = (nl + kRows - 1) / kRows * ((ns + width_of(ns) - 1) / width_of(ns)) * ((nk + kBlockK - 1) / kBlockK);
  const long long n = (units + 3) / 4;                   // four blocks each at least
  return (int)(n < kMostCtas ? n : kMostCtas);
}

// The long side as it is: 128 rows of 64 k (rows along memory), or 32 k of 128 rows with the 128-byte swizzle, without which a lane per row would
// meet bank conflicts (k along memory).
bool encode_long(CUtensorMap* map, const Operand& L, long long nl, long long nk) {
  const bool rows_inner = L.ks != 1;
  const cuuint64_t dims[2] = {(cuuint64_t)(rows_inner ? nl : nk), (cuuint64_t)(rows_inner ? nk : nl)};
  const long long pitch = dims[1] > 1 ? (rows_inner ? L.ks : L.rs) : (long long)((dims[0] + 3) / 4 * 4);
  const cuuint64_t strides[1] = {(cuuint64_t)pitch * 4};
  const cuuint32_t box[2] = {rows_inner ? 128u : 32u, rows_inner ? 64u : 128u}, estr[2] = {1, 1};
  return tensor_map_encoder()(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 2, const_cast<void*>(L.p), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                              rows_inner ? CU_TENSOR_MAP_SWIZZLE_NONE : CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int kBN>
cudaError_t launch(const Operand& L, const Planes& S, long long nk, const SplitArgs& g, cudaStream_t s) {
  alignas(64) CUtensorMap ml, ms;
  if (tensor_map_encoder() == nullptr) return cudaErrorNotSupported;
  if (!encode_long(&ml, L, g.nl, nk) || !encode_operand(&ms, S, true, kBN)) return cudaErrorInvalidValue;
  cudaError_t e = cudaFuncSetAttribute(k_linear_split<kBN>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Sizes<kBN>::kSmem);
  if (e == cudaSuccess) e = launch_chained(k_linear_split<kBN>, dim3((unsigned)g.ctas), kThreads, Sizes<kBN>::kSmem, s, ml, ms, g);
  if (e == cudaSuccess && g.shared > 0 && g.own < g.blocks) e = launch_chained(k_linear_split_sum<kBN>, dim3((unsigned)g.shared, kBN / 8), 256, 0, s, g);
  return e;
}

}  // namespace

bool linear_split_takes(const Operand& L, long long nl, long long nk) {
  if (((uintptr_t)L.p & 15) != 0 || (L.rs != 1 && L.ks != 1)) return false;
  const long long pitch = L.ks != 1 ? L.ks : L.rs, inner = L.ks != 1 ? nl : nk, outer = L.ks != 1 ? nk : nl;
  return outer == 1 || (pitch % 4 == 0 && pitch >= inner);
}

size_t linear_split_workspace(long long nl, long long ns, long long nk) {
  return (size_t)2 * ctas_of(nl, ns, nk) * width_of(ns) * kRows * sizeof(float);      // (R < ctas)
}

cudaError_t launch_linear_split(const Operand& L, const Planes& S, long long nl, long long ns, long long nk, bool long_is_b, const Finish& f,
                                void* workspace, unsigned int* status, bool stall, cudaStream_t s) {
  SplitArgs g = {};
  g.nl = (int)nl; g.ns = (int)ns;
  g.blocks = (int)((nk + kBlockK - 1) / kBlockK);
  g.tiles_l = (int)((nl + kRows - 1) / kRows);
  g.tiles_s = (int)((ns + width_of(ns) - 1) / width_of(ns));
  g.ctas = ctas_of(nl, ns, nk);
  const long long tiles = (long long)g.tiles_l * g.tiles_s;
  g.rounds = (int)(tiles / g.ctas);
  g.shared = (int)(tiles % g.ctas);
  g.own = (int)(((long long)g.shared * g.blocks + g.ctas - 1) / g.ctas);
  g.l_rows_inner = L.ks != 1;
  g.long_is_b = long_is_b; g.stall = stall;
  g.partial = static_cast<float*>(workspace);
  g.status = status; g.f = f;
  return width_of(ns) == 32 ? launch<32>(L, S, nk, g, s) : launch<48>(L, S, nk, g, s);
}

}  // namespace strads
