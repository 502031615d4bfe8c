// Products of linear layers with few rows on one side: the margins of one or a few fits, a gradient for one response, a layer
// for single tokens.  Bound by reading the long operand once.  Plain FP32 multiply-adds, no copy of the operand, no tensor
// cores: a tile of theirs would be nearly empty, and binary32 would have to be split first.
//
//   k along memory (k_thin_k): a warp takes rows, a lane every 32nd group of 16 bytes of them; lanes are added by shuffles.
//   rows along memory (k_thin_tiles): tiles of 512 bytes of rows by 32 k come by TMA into a ring, a lane takes the rows of 16 bytes, a warp every
//   eighth k; warps are added through shared memory.  What TMA cannot address goes by k_thin_rows: the same without the ring, a lane the rows of 16
//   bytes (or of 4, where there are few).
//
// What hides the memory's latency is the number of loads under way: four or eight per lane, and as many warps as that leaves registers for (rows along
// memory, 10,000 x 100,000 binary32: 767 us with 4 a lane, 833 with 8, 2,280 with 16 and half the warps); where the rows alone do not
// make enough of them, the warps of a CTA and the CTAs of a cluster share k and add through (distributed) shared memory, in a fixed order.
// The short side is staged in shared memory as binary32, or (k along memory, up to four rows) read through L1 as it is.
#include <mutex>

#include "linear_tc.cuh"
#include "linear_ptx.cuh"

namespace strads {
namespace {

constexpr int kThreads = 256, kWarps = 8;      // k_thin_k
constexpr int kStageFloats = 8192;             // of the short side in shared memory at a time

struct Thin {
  Operand L, S;                                // the long and the short side
  long long nl, nk;
  int ns, splits, swapped, vec, svec;          // swapped: the long side is D's b; vec, svec: 16-byte accesses to the long, the short side
  int wk;                                      // k_thin_k: warps of a CTA that share a row's k (1 or 8)
  int stall;
  unsigned int* status;
  Finish f;
};

__device__ __forceinline__ float load_peer(const float* p, uint32_t rank) {
  uint32_t a;
  float v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_u32(p)), "r"(rank));
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(a) : "memory");
  return v;
}
template <typename T>
__device__ __forceinline__ void finish_thin(const Thin& t, float v, long long l, int s) {
  if (t.swapped) finish<T>(t.f, v, s, l); else finish<T>(t.f, v, l, s);
}

// kBytes of T, as they are and as floats.
template <int kBytes> struct Raw;
template <> struct Raw<16> { uint4 v; };
template <> struct Raw<4> { unsigned int v; };
template <int kBytes>
__device__ __forceinline__ Raw<kBytes> load_raw(const void* p) {
  Raw<kBytes> r;
  r.v = __ldg(static_cast<const decltype(r.v)*>(p));
  return r;
}
// The long side's: read once, so not kept in L1.  (volatile: a batch of them is issued before the first is used, as written)
template <int kBytes>
__device__ __forceinline__ Raw<kBytes> load_once(const void* p) {
  Raw<kBytes> r;
  if constexpr (kBytes == 16)
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(r.v.x), "=r"(r.v.y), "=r"(r.v.z), "=r"(r.v.w) : "l"(p));
  else
    asm volatile("ld.global.nc.L1::no_allocate.u32 %0, [%1];" : "=r"(r.v) : "l"(p));
  return r;
}
template <typename T, int kBytes>
__device__ __forceinline__ void to_floats(const Raw<kBytes>& r, float (&v)[kBytes / sizeof(T)]) {
  const T* x = reinterpret_cast<const T*>(&r);
#pragma unroll
  for (int i = 0; i < (int)(kBytes / sizeof(T)); ++i) v[i] = load_f32(x + i);
}

// The share of k of this CTA.
__device__ __forceinline__ void share(const Thin& t, long long unit, long long* k0, long long* k1) {
  const long long units = (t.nk + unit - 1) / unit, r = t.splits > 1 ? blockIdx.x % t.splits : 0;
  *k0 = units * r / t.splits * unit;
  *k1 = min(t.nk, units * (r + 1) / t.splits * unit);
}

// S[s][k0 .. k0 + n) -> shared memory, [k][kT] or [kT][n], noughts behind the last row.
template <typename T, int kT, bool kByK>
__device__ __forceinline__ void stage_short(const Thin& t, long long k0, int n, float* sh, int pitch) {
  for (int i = threadIdx.x; i < n * kT; i += blockDim.x) {
    const int s = t.S.ks == 1 ? i / n : i % kT, k = t.S.ks == 1 ? i % n : i / kT;
    const float v = s < t.ns ? load_f32(static_cast<const T*>(t.S.p) + s * t.S.rs + (k0 + k) * t.S.ks) : 0.f;
    sh[kByK ? k * kT + s : s * pitch + k] = v;
  }
}

// kDirect: the short side is read as it is (16-byte accesses to both sides).
template <typename T, int kT, int kR, bool kDirect>
__global__ void __launch_bounds__(kThreads) k_thin_k(const __grid_constant__ Thin t) {
  constexpr int kV = 16 / sizeof(T), kStage = kStageFloats / kT, kU = sizeof(T) == 2 && kR * kT <= 2 ? 8 : 4;
  __shared__ __align__(16) float sh[kDirect ? 4 : kStageFloats];
  __shared__ float red[kWarps][kR * kT];
  __shared__ float sum[kWarps][kR * kT];
  chain_begin();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const long long group = (long long)(blockIdx.x / t.splits);
  const long long l0 = t.wk == 1 ? (group * kWarps + warp) * kR : group * kR;
  long long k0, k1;
  share(t, 256, &k0, &k1);
  float acc[kR][kT] = {};
  const T* row[kR];
#pragma unroll
  for (int r = 0; r < kR; ++r) row[r] = static_cast<const T*>(t.L.p) + min(l0 + r, t.nl - 1) * t.L.rs;
  const int at = t.wk == 1 ? lane : warp * 32 + lane, step = t.wk == 1 ? 32 : 256;
  const int stage = kDirect ? 0x40000000 : kStage;
  for (long long kb = k0; kb < k1; kb += stage) {
    const int n = (int)min((long long)stage, k1 - kb);
    if (!kDirect) {
      __syncthreads();
      stage_short<T, kT, false>(t, kb, n, sh, kStage);
      __syncthreads();
    }
    const int groups = t.vec ? n / kV : 0;
    for (int i0 = at; i0 < groups; i0 += step * kU) {
      Raw<16> x[kU][kR], y[kU][kDirect ? kT : 1];
#pragma unroll
      for (int u = 0; u < kU; ++u) {
        const long long i = min(i0 + u * step, groups - 1);      // (one past the end reads the last again, for nothing)
#pragma unroll
        for (int r = 0; r < kR; ++r) x[u][r] = load_once<16>(row[r] + kb + i * kV);
        if (kDirect)
#pragma unroll
          for (int s = 0; s < kT; ++s) y[u][s] = load_raw<16>(static_cast<const T*>(t.S.p) + min(s, t.ns - 1) * t.S.rs + kb + i * kV);
      }
#pragma unroll
      for (int u = 0; u < kU; ++u) {
        const int i = i0 + u * step;
        if (i >= groups) break;
        float xf[kR][kV];
#pragma unroll
        for (int r = 0; r < kR; ++r) to_floats<T, 16>(x[u][r], xf[r]);
#pragma unroll
        for (int s = 0; s < kT; ++s) {
          float yf[kV];
          if (kDirect) {
            to_floats<T, 16>(y[u][kDirect ? s : 0], yf);
          } else {
#pragma unroll
            for (int v = 0; v < kV; v += 4) *reinterpret_cast<float4*>(yf + v) = *reinterpret_cast<const float4*>(sh + s * kStage + i * kV + v);
          }
#pragma unroll
          for (int r = 0; r < kR; ++r)
#pragma unroll
            for (int v = 0; v < kV; ++v) acc[r][s] = fmaf(xf[r][v], yf[v], acc[r][s]);
        }
      }
    }
    for (int k = groups * kV + at; k < n; k += step) {
#pragma unroll
      for (int r = 0; r < kR; ++r) {
        const float x = load_f32(row[r] + (kb + k) * t.L.ks);
#pragma unroll
        for (int s = 0; s < kT; ++s) {
          const float y = !kDirect ? sh[s * kStage + k] : load_f32(static_cast<const T*>(t.S.p) + min(s, t.ns - 1) * t.S.rs + kb + k);
          acc[r][s] = fmaf(x, y, acc[r][s]);
        }
      }
    }
  }
#pragma unroll
  for (int r = 0; r < kR; ++r)
#pragma unroll
    for (int s = 0; s < kT; ++s) {
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) acc[r][s] += __shfl_xor_sync(0xffffffffu, acc[r][s], o);
      if (lane == 0) red[warp][r * kT + s] = acc[r][s];
    }
  if (t.wk == 1 && t.splits == 1) {                      // a warp finishes its own rows
    __syncwarp();
    for (int e = lane; e < kR * kT; e += 32)
      if (l0 + e / kT < t.nl && e % kT < t.ns) finish_thin<T>(t, red[warp][e], l0 + e / kT, e % kT);
    return;
  }
  // sums of the CTA: one set per warp, or one for all of them
  __syncthreads();
  const int sets = t.wk == 1 ? kWarps : 1;
  for (int i = threadIdx.x; i < sets * kR * kT; i += kThreads) {
    const int w = i / (kR * kT), e = i % (kR * kT);
    float v = red[w][e];
    if (t.wk != 1) for (int u = 1; u < kWarps; ++u) v += red[u][e];
    sum[w][e] = v;
  }
  if (t.splits > 1) cluster_sync(); else __syncthreads();
  if (t.splits == 1 || blockIdx.x % t.splits == 0) {
    for (int i = threadIdx.x; i < sets * kR * kT; i += kThreads) {
      const int w = i / (kR * kT), e = i % (kR * kT), s = e % kT;
      const long long l = (t.wk == 1 ? (group * kWarps + w) * kR : group * kR) + e / kT;
      if (l >= t.nl || s >= t.ns) continue;
      float v = sum[w][e];
      for (int p = 1; p < t.splits; ++p) v += load_peer(&sum[w][e], (uint32_t)p);
      finish_thin<T>(t, v, l, s);
    }
  }
  if (t.splits > 1) cluster_sync();                      // nobody leaves while its sums may be read
}

constexpr int kRowWarps = 16, kRowThreads = 32 * kRowWarps;
template <typename T, int kT, int kBytes>
__global__ void __launch_bounds__(kRowThreads) k_thin_rows(const __grid_constant__ Thin t) {
  constexpr int kV = kBytes / sizeof(T), kTile = 32 * kV, kStage = kStageFloats / kT, kU = sizeof(T) == 2 && kT == 1 ? 8 : 4;
  constexpr int kSums = kT * kTile;
  extern __shared__ __align__(16) float sh[];            // the stage; when the last of the short side has been used, [warp][kSums]
  __shared__ float sum[kSums];
  chain_begin();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const long long l0 = (long long)(blockIdx.x / t.splits) * kTile, l = l0 + lane * kV;
  long long k0, k1;
  share(t, 16, &k0, &k1);
  const bool whole = t.vec && l + kV <= t.nl;
  float acc[kT][kV] = {};
  auto add = [&](int k, const float (&x)[kV]) {
#pragma unroll
    for (int s = 0; s < kT; ++s) {
      const float y = sh[k * kT + s];
#pragma unroll
      for (int v = 0; v < kV; ++v) acc[s][v] = fmaf(x[v], y, acc[s][v]);
    }
  };
  for (long long kb = k0; kb < k1; kb += kStage) {
    const int n = (int)min((long long)kStage, k1 - kb);
    __syncthreads();
    stage_short<T, kT, true>(t, kb, n, sh, 0);
    __syncthreads();
    const T* at = static_cast<const T*>(t.L.p) + kb * t.L.ks + l * t.L.rs;
    if (whole) {
      for (int i0 = warp; i0 < n; i0 += kRowWarps * kU) {
        Raw<kBytes> x[kU];
#pragma unroll
        for (int u = 0; u < kU; ++u) x[u] = load_once<kBytes>(at + min(i0 + u * kRowWarps, n - 1) * t.L.ks);
#pragma unroll
        for (int u = 0; u < kU; ++u) {
          if (i0 + u * kRowWarps >= n) break;
          float xf[kV];
          to_floats<T, kBytes>(x[u], xf);
          add(i0 + u * kRowWarps, xf);
        }
      }
    } else if (l < t.nl) {
      for (int k = warp; k < n; k += kRowWarps) {
        float xf[kV];
#pragma unroll
        for (int v = 0; v < kV; ++v) xf[v] = l + v < t.nl ? load_f32(at + k * t.L.ks + v * t.L.rs) : 0.f;
        add(k, xf);
      }
    }
  }
  __syncthreads();
#pragma unroll
  for (int s = 0; s < kT; ++s)
#pragma unroll
    for (int v = 0; v < kV; ++v) sh[warp * kSums + s * kTile + v * 32 + lane] = acc[s][v];      // (a lane's rows 32 apart: no bank conflicts)
  __syncthreads();
  for (int i = threadIdx.x; i < kSums; i += kRowThreads) {
    float a = sh[i];
#pragma unroll
    for (int w = 1; w < kRowWarps; ++w) a += sh[w * kSums + i];
    sum[i] = a;
  }
  if (t.splits > 1) cluster_sync(); else __syncthreads();
  const int rank = t.splits > 1 ? (int)(blockIdx.x % t.splits) : 0;
  for (int i = rank * kRowThreads + threadIdx.x; i < kT * kTile; i += kRowThreads * t.splits) {
    const int s = i / kTile, j = i % kTile;              // row j of the tile is lane j / kV's, its (j % kV)-th
    if (l0 + j >= t.nl || s >= t.ns) continue;
    const float* p = sum + s * kTile + (j % kV) * 32 + j / kV;
    float v = 0.f;
    if (t.splits == 1) v = *p;
    else for (int q = 0; q < t.splits; ++q) v += load_peer(p, (uint32_t)q);
    finish_thin<T>(t, v, l0 + j, s);
  }
  if (t.splits > 1) cluster_sync();
}

// ---- rows along memory, by TMA ----
constexpr int kTileK = 32, kTileBytes = 512 * kTileK, kTileStages = 6, kTileWarps = 8;
constexpr size_t kTileSmem = (size_t)kTileStages * kTileBytes + 1024;
template <typename T, int kT>
__global__ void __launch_bounds__(32 * (kTileWarps + 1), 2) k_thin_tiles(const __grid_constant__ CUtensorMap map, const __grid_constant__ Thin t) {
  constexpr int kV = 16 / sizeof(T), kTile = 32 * kV, kSums = kT * kTile, kRows = kTileK / kTileWarps;
  extern __shared__ unsigned char dyn[];
  __shared__ __align__(8) uint64_t s_full[kTileStages], s_empty[kTileStages];
  __shared__ float sum[kSums];
  __shared__ volatile int s_abort;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint32_t ring = (smem_u32(dyn) + 127u) & ~127u, full = smem_u32(s_full), empty = smem_u32(s_empty);
  const uint32_t limit = t.stall ? kMmaStallLimit : kMmaWaitLimit;
  if (threadIdx.x == 0) {
    s_abort = 0;
    for (int i = 0; i < kTileStages; ++i) { mbar_init(full + 8 * i, 1); mbar_init(empty + 8 * i, kTileWarps); }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map) : "memory");
  }
  __syncthreads();
  chain_begin();
  const long long l0 = (long long)(blockIdx.x / t.splits) * kTile;
  const int rank = t.splits > 1 ? (int)(blockIdx.x % t.splits) : 0;
  // blocks of 32 k of this CTA: rank, rank + splits, ..
  const int blocks = (int)((t.nk + kTileK - 1) / kTileK), mine = (blocks - rank + t.splits - 1) / t.splits;
  bool ok = true;
  float acc[kT][kV] = {};
  if (warp == kTileWarps) {
    if (elect_one()) {
      int n = 0;
      for (; n < mine; ++n) {
        const uint32_t s = (uint32_t)(n % kTileStages);
        ok = !s_abort && mbar_wait(empty + 8 * s, ((uint32_t)(n / kTileStages) & 1u) ^ 1u, limit) && !t.stall;
        if (!ok) break;
        mbar_expect(full + 8 * s, (uint32_t)kTileBytes);
        asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                     ::"r"(ring + s * kTileBytes), "l"(&map), "r"((int)l0), "r"((rank + n * t.splits) * kTileK), "r"(full + 8 * s) : "memory");
      }
      // nothing is under way when the shared memory goes
      for (int j = n > kTileStages ? n - kTileStages : 0; j < n; ++j)
        if (!mbar_wait(full + 8 * (uint32_t)(j % kTileStages), (uint32_t)(j / kTileStages) & 1u, limit)) { ok = false; break; }
      if (!ok) { s_abort = 1; atomicOr(t.status, STRADS_STATUS_WAIT_EXPIRED); }
    }
    __syncwarp();
  } else {
    // the short side's values of this warp's rows of a block: lane r * kT + s holds that of row r; a block ahead
    const int r = lane / kT, sr = lane % kT;
    auto fetch = [&](int n) {
      const long long k = (long long)(rank + n * t.splits) * kTileK + warp * kRows + r;
      return r < kRows && sr < t.ns && n < mine && k < t.nk ? load_f32(static_cast<const T*>(t.S.p) + sr * t.S.rs + k * t.S.ks) : 0.f;
    };
    float held = fetch(0);
    for (int n = 0; n < mine; ++n) {
      const float now = held;
      held = fetch(n + 1);
      const uint32_t s = (uint32_t)(n % kTileStages);
      ok = __all_sync(0xffffffffu, !s_abort && mbar_wait(full + 8 * s, (uint32_t)(n / kTileStages) & 1u, limit));
      if (!ok) break;
#pragma unroll
      for (int i = 0; i < kRows; ++i) {
        uint4 raw;
        asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(raw.x), "=r"(raw.y), "=r"(raw.z), "=r"(raw.w)
                     : "r"(ring + s * kTileBytes + (warp * kRows + i) * 512 + lane * 16) : "memory");
        Raw<16> w;
        w.v = raw;
        float x[kV];
        to_floats<T, 16>(w, x);
#pragma unroll
        for (int q = 0; q < kT; ++q) {
          const float y = __shfl_sync(0xffffffffu, now, i * kT + q);
#pragma unroll
          for (int v = 0; v < kV; ++v) acc[q][v] = fmaf(x[v], y, acc[q][v]);
        }
      }
      __syncwarp();
      if (lane == 0) asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(empty + 8 * s) : "memory");
    }
    if (!ok && lane == 0) { s_abort = 1; atomicOr(t.status, STRADS_STATUS_WAIT_EXPIRED); }
  }
  __syncthreads();                                       // (all of the ring has been read: the warps' sums take its place)
  float* part = reinterpret_cast<float*>(dyn);
  if (warp < kTileWarps)
#pragma unroll
    for (int q = 0; q < kT; ++q)
#pragma unroll
      for (int v = 0; v < kV; ++v) part[warp * kSums + q * kTile + v * 32 + lane] = acc[q][v];
  __syncthreads();
  for (int i = threadIdx.x; i < kSums; i += 32 * (kTileWarps + 1)) {
    float a = part[i];
#pragma unroll
    for (int w = 1; w < kTileWarps; ++w) a += part[w * kSums + i];
    sum[i] = a;
  }
  if (t.splits > 1) cluster_sync(); else __syncthreads();
  if (!s_abort)
    for (int i = rank * 32 * (kTileWarps + 1) + threadIdx.x; i < kSums; i += 32 * (kTileWarps + 1) * t.splits) {
      const int q = i / kTile, j = i % kTile;
      if (l0 + j >= t.nl || q >= t.ns) continue;
      const float* p = sum + q * kTile + (j % kV) * 32 + j / kV;
      float v = 0.f;
      if (t.splits == 1) v = *p;
      else for (int c = 0; c < t.splits; ++c) v += load_peer(p, (uint32_t)c);
      finish_thin<T>(t, v, l0 + j, q);
    }
  if (t.splits > 1) cluster_sync();
}

bool vec_ok(const void* p, long long pitch, long long rows, size_t size) { return ((uintptr_t)p & 15) == 0 && (rows <= 1 || (pitch * (long long)size) % 16 == 0); }

template <typename T, int kT, int kBytes>
cudaError_t launch_rows(const Thin& t, long long tiles, cudaStream_t s) {
  if (t.splits > 8) {                                    // (clusters of more than 8 CTAs: the device takes them on request)
    const cudaError_t e = cudaFuncSetAttribute(k_thin_rows<T, kT, kBytes>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e != cudaSuccess) return e;
  }
  constexpr size_t kSums = sizeof(float) * kRowWarps * kT * 32 * (kBytes / sizeof(T)), kStage = sizeof(float) * kStageFloats, kSmem = kSums > kStage ? kSums : kStage;
  if (kSmem + 8192 > 48 * 1024) {
    const cudaError_t e = cudaFuncSetAttribute(k_thin_rows<T, kT, kBytes>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmem);
    if (e != cudaSuccess) return e;
  }
  return launch_chained_cluster(k_thin_rows<T, kT, kBytes>, dim3((unsigned)(tiles * t.splits)), kRowThreads, kSmem, s, t.splits, t);
}
template <typename T, int kT>
cudaError_t launch_tiles(Thin t, int sms, cudaStream_t s) {
  constexpr int kTile = 512 / (int)sizeof(T);
  const long long tiles = (t.nl + kTile - 1) / kTile, blocks = (t.nk + kTileK - 1) / kTileK;
  // as many CTAs to a tile as leave all of them resident, two to an SM, with four blocks each at least
  t.splits = 1;
  for (int n = 2; n <= 16; ++n)
    if (tiles * n <= 2ll * sms && blocks >= 4ll * n) t.splits = n;
  alignas(64) CUtensorMap map;
  const cuuint64_t dims[2] = {(cuuint64_t)t.nl, (cuuint64_t)t.nk}, strides[1] = {(cuuint64_t)t.L.ks * sizeof(T)};
  const cuuint32_t box[2] = {(cuuint32_t)kTile, (cuuint32_t)kTileK}, estr[2] = {1, 1};
  if (tensor_map_encoder()(&map, sizeof(T) == 4 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_UINT16, 2, const_cast<void*>(t.L.p), dims, strides, box,
                           estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                           CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
    return cudaErrorInvalidValue;
  cudaError_t e = cudaFuncSetAttribute(k_thin_tiles<T, kT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kTileSmem);
  if (e == cudaSuccess && t.splits > 8) e = cudaFuncSetAttribute(k_thin_tiles<T, kT>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  if (e != cudaSuccess) return e;
  return launch_chained_cluster(k_thin_tiles<T, kT>, dim3((unsigned)(tiles * t.splits)), 32 * (kTileWarps + 1), kTileSmem, s, t.splits, map, t);
}
template <typename T, int kT>
cudaError_t launch(Thin t, int sms, cudaStream_t s) {
  const bool along_k = t.L.ks == 1 || t.L.rs != 1;
  t.splits = 1;
  if (along_k) {
    t.vec = t.L.ks == 1 && vec_ok(t.L.p, t.L.rs, t.nl, sizeof(T));
    t.svec = t.S.ks == 1 && vec_ok(t.S.p, t.S.rs, t.ns, sizeof(T));
    constexpr int kR = kT >= 4 ? 2 : 1;
    const long long warps = (t.nl + kR - 1) / kR;
    t.wk = warps >= 8ll * sms ? 1 : kWarps;              // few rows: the warps of a CTA share them
    const long long groups = t.wk == 1 ? (warps + kWarps - 1) / kWarps : warps;
    while (t.splits < 8 && groups * t.splits * 2 <= 2 * sms && t.nk >= 4096ll * t.splits) t.splits *= 2;
    const dim3 grid((unsigned)(groups * t.splits));
    if (t.vec && t.svec) return launch_chained_cluster(k_thin_k<T, kT, kR, true>, grid, kThreads, 0, s, t.splits, t);
    return launch_chained_cluster(k_thin_k<T, kT, kR, false>, grid, kThreads, 0, s, t.splits, t);
  }
  t.vec = vec_ok(t.L.p, t.L.ks, t.nk, sizeof(T));
  if (t.vec && t.nk > 1 && t.L.ks >= t.nl && tensor_map_encoder() != nullptr) return launch_tiles<T, kT>(t, sms, s);
  // 16 bytes of a row per lane where that leaves enough CTAs, 4 otherwise; then as many CTAs to a tile as keep four on every SM
  const long long wide = (t.nl + 512 / (int)sizeof(T) - 1) / (512 / (int)sizeof(T)), narrow = (t.nl + 128 / (int)sizeof(T) - 1) / (128 / (int)sizeof(T));
  const bool few = wide * 32 < sms;
  const long long tiles = few ? narrow : wide;
  while (t.splits < 16 && tiles * t.splits < 4ll * sms && t.nk >= 512ll * t.splits) t.splits *= 2;
  return few ? launch_rows<T, kT, 4>(t, tiles, s) : launch_rows<T, kT, 16>(t, tiles, s);
}
template <typename T>
cudaError_t by_short(const Thin& t, int sms, cudaStream_t s) {
  return t.ns == 1 ? launch<T, 1>(t, sms, s) : t.ns == 2 ? launch<T, 2>(t, sms, s) : launch<T, 4>(t, sms, s);
}

}  // namespace

cudaError_t launch_linear_thin(int type, const Operand& A, const Operand& B, long long na, long long nb, long long nk, const Finish& f, unsigned int* status,
                               bool stall, cudaStream_t s) {
  int dev = 0, sms = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  if (e != cudaSuccess) return e;
  Thin t = {};
  t.f = f; t.nk = nk; t.status = status; t.stall = stall;
  t.swapped = na < nb;
  t.L = t.swapped ? B : A; t.S = t.swapped ? A : B;
  t.nl = t.swapped ? nb : na; t.ns = (int)(t.swapped ? na : nb);
  return type == STRADS_F32 ? by_short<float>(t, sms, s) : type == STRADS_BF16 ? by_short<__nv_bfloat16>(t, sms, s) : by_short<__half>(t, sms, s);
}

}  // namespace strads
