// Linear layers: out = residual + scale act(x w^T + bias) and its gradient.  Argument checks, workspace, the passes that bring
// operands into the form that the products read, and which kernel forms which product.
#include <cmath>

#include "linear_tc.cuh"

namespace strads {
namespace {

__device__ unsigned int g_linear_status;       // STRADS_STATUS_* bits of the layers' bounded waits

constexpr int kThreads = 256;

// ---- lines of binary16 gradients (see k_linear_tops) ----
// 2^-e for the power 2^e that brings a magnitude to 2^14 .. 2^15, and 2^e from that.  (A line of noughts: 2^126.)
__device__ __forceinline__ float line_factor(unsigned int half_bits) {
  const unsigned int b = __float_as_uint(__half2float(__ushort_as_half((unsigned short)half_bits)));
  return __uint_as_float((max(b >> 23, 15u) - 14u) << 23);
}
__device__ __forceinline__ float line_power(float factor) { return __uint_as_float((254u << 23) - __float_as_uint(factor)); }
// The largest magnitudes of the blocks of rows (columns: [blocks][m]) and of the blocks of 256 columns (rows: [columns][n]), and the factors to be formed from them:
// those of columns by the first `column_ctas` CTAs, 32 each, of rows by the others, 256 each.
struct LinesJob {
  const unsigned short *col_tops, *row_tops;
  float *column_factors, *row_factors;
  long long n, m;
  int blocks, columns, column_ctas, ctas;
};
__device__ __forceinline__ void form_factors(const LinesJob& j, int cta, unsigned int (&top)[8][32]) {
  unsigned int t = 0u;
  if (cta >= j.column_ctas) {
    const long long r = (long long)(cta - j.column_ctas) * kThreads + threadIdx.x;
    if (r >= j.n) return;
#pragma unroll 4
    for (int i = 0; i < j.columns; ++i) t = max(t, (unsigned int)j.row_tops[i * j.n + r]);
    j.row_factors[r] = line_factor(t);
    return;
  }
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const long long c = (long long)cta * 32 + lane;
  if (c < j.m)
#pragma unroll 4
    for (int r = j.blocks * warp / 8; r < j.blocks * (warp + 1) / 8; ++r) t = max(t, (unsigned int)j.col_tops[r * j.m + c]);
  top[warp][lane] = t;
  __syncthreads();
  if (warp != 0 || c >= j.m) return;
#pragma unroll
  for (int w = 1; w < 8; ++w) t = max(t, top[w][lane]);
  j.column_factors[c] = line_factor(t);
}

// ---- operands of the tensor-core products that cannot be read in place ----
// dst[plane][outer][ld] from src, eight neighbours per thread; binary32 as three planes of bfloat16 (split_pair).  All operands of a call that
// need it in one launch.
struct Copy {
  const void* src;
  long long outer_stride, inner_stride, outer, inner, ld, plane;
  unsigned short* dst;
  int vec;
};
constexpr int kMostCopies = 3;
struct Copies { Copy c[kMostCopies]; int n, ctas; long long groups; };      // (the first `ctas` CTAs of the launch)
template <typename T>
__device__ __forceinline__ void copy_group(const Copy& c, long long i) {
  const long long per = c.ld / 8, o = i / per, k = i % per * 8;
  const T* at = static_cast<const T*>(c.src) + o * c.outer_stride + k * c.inner_stride;
  __align__(16) T x[8];
  if (c.vec && k + 8 <= c.inner) {
#pragma unroll
    for (int j = 0; j < (int)sizeof(T) / 2; ++j) reinterpret_cast<uint4*>(x)[j] = __ldg(reinterpret_cast<const uint4*>(at) + j);
  } else {
    const long long last = c.inner - 1 - k;              // (clamped, not branched: all loads under way at once)
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = at[(j < last ? j : last) * c.inner_stride];
#pragma unroll
    for (int j = 0; j < 8; ++j) if (j > last) store_f32(&x[j], 0.f);
  }
  unsigned short* to = c.dst + o * c.ld + k;
  if (sizeof(T) == 2) {
    *reinterpret_cast<uint4*>(to) = *reinterpret_cast<const uint4*>(x);
  } else {
    __align__(16) uint32_t p[3][4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      uint32_t w[3];
      split_pair(load_f32(&x[2 * j]), load_f32(&x[2 * j + 1]), w);
      p[0][j] = w[0]; p[1][j] = w[1]; p[2][j] = w[2];
    }
#pragma unroll
    for (int q = 0; q < 3; ++q) *reinterpret_cast<uint4*>(to + q * c.plane) = *reinterpret_cast<const uint4*>(p[q]);
  }
}
template <typename T>
__global__ void __launch_bounds__(kThreads) k_linear_pack(const __grid_constant__ Copies all, const __grid_constant__ LinesJob lines) {
  __shared__ unsigned int top[8][32];
  chain_begin();
  if ((int)blockIdx.x >= all.ctas) {
    form_factors(lines, (int)blockIdx.x - all.ctas, top);
    return;
  }
  // the groups of all matrices as one run, so that a thread's loads do not wait for those of another matrix
  const long long stride = (long long)all.ctas * kThreads;
  for (long long i = (long long)blockIdx.x * kThreads + threadIdx.x; i < all.groups; i += stride) {
    long long at = i;
    int n = 0;
    while (n + 1 < all.n && at >= all.c[n].plane / 8) at -= all.c[n++].plane / 8;
    copy_group<T>(all.c[n], at);
  }
}

// ---- gz = gout act'(preact), and its column sums ----
// (scale stays outside, a factor of the 32-bit sums as it is with the identity: inside, gz of binary16 would leave its range with it.)
// binary16, through an activation: gz may lie above 65,504, or below 2^-14 where the type has fewer digits or none, although the sums over it are numbers of the
// type.  It is held with a power of two that brings the largest finite |gout| of a line to 2^14 .. 2^15 (and so gz below 1.13 times that): of its row in the copy that
// gx is formed from, of its column in gw's; the products' epilogue takes the power back.  What is below 2^-29 of that |gout| is off by up to 2^-39 of it.
// k_linear_tops looks at gout alone: half of what forms gz, and no exponentials (SiLU, all launches of a gradient of 4,096 x 8,192 by 64: 119 us, from gz itself 156, with
// gz rounded as it is 80; 2,048^3: 73, 78, 63; 333 x 1,001 x 517: 31, 31, 26).
struct Lines { const float *row_factors, *column_factors; __half* by_column; };      // 2^-e of every row and column; gz with its column's power (gz: with its row's)
constexpr unsigned int kHalfAbs = 0x7fff7fffu, kHalfInfinity = 0x7c007c00u;
__device__ __forceinline__ unsigned int finite_halves(unsigned int x) {      // magnitudes of two of them, 0 for what is not finite
  x &= kHalfAbs;
  return x & ~__vcmpgeu2(x, kHalfInfinity);
}
// col_tops [gridDim.y][m] of the CTA's rows, row_tops [gridDim.x][n] of its 256 columns (each may be null), as bits of the type.
__global__ void __launch_bounds__(kThreads) k_linear_tops(Operand gout, long long n, long long m, unsigned short* col_tops, unsigned short* row_tops, long long rows, int vec) {
  constexpr int kU = 4;
  __shared__ uint4 top[8][32];
  chain_begin();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const long long c = (long long)blockIdx.x * 256 + lane * 8, r0 = (long long)blockIdx.y * rows, r1 = min(n, r0 + rows);
  const int count = (int)min(8ll, m - c);
  const bool whole = vec && count == 8;
  uint4 most = {0u, 0u, 0u, 0u};
  for (long long r = r0 + warp; r < r1; r += 8 * kU) {
    uint4 x[kU];
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      x[u] = {0u, 0u, 0u, 0u};
      const unsigned short* p = static_cast<const unsigned short*>(gout.p) + min(r + 8 * u, r1 - 1) * gout.rs + c * gout.ks;
      if (whole) {
        x[u] = __ldg(reinterpret_cast<const uint4*>(p));
      } else if (count > 0) {                            // (past the last column: that column again)
        unsigned int w[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = p[min(j, count - 1) * gout.ks];
        x[u] = {w[0] | w[1] << 16, w[2] | w[3] << 16, w[4] | w[5] << 16, w[6] | w[7] << 16};
      }
    }
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      x[u] = {finite_halves(x[u].x), finite_halves(x[u].y), finite_halves(x[u].z), finite_halves(x[u].w)};
      most = {__vmaxu2(most.x, x[u].x), __vmaxu2(most.y, x[u].y), __vmaxu2(most.z, x[u].z), __vmaxu2(most.w, x[u].w)};
      if (row_tops != nullptr) {
        const unsigned int t = __vmaxu2(__vmaxu2(x[u].x, x[u].y), __vmaxu2(x[u].z, x[u].w)), all = __reduce_max_sync(0xffffffffu, max(t >> 16, t & 0xffffu));
        if (lane == 0 && r + 8 * u < r1) row_tops[(long long)blockIdx.x * n + r + 8 * u] = (unsigned short)all;
      }
    }
  }
  if (col_tops == nullptr) return;
  top[warp][lane] = most;
  __syncthreads();
  const long long col = (long long)blockIdx.x * 256 + threadIdx.x;
  if (col >= m) return;
  unsigned int t = 0u;
#pragma unroll
  for (int w = 0; w < 8; ++w) t = max(t, (unsigned int)reinterpret_cast<const unsigned short*>(&top[w][0])[threadIdx.x]);
  col_tops[(long long)blockIdx.y * m + col] = (unsigned short)t;
}

// A CTA takes 256 columns of `rows` rows, a lane eight columns, a warp every eighth row, kU of them at a time so that their loads are under way
// together.  Three CTAs to an SM (80 registers): the pass waits for memory, and warps hide that better than rows of one lane (gradient of 4,096 x 8,192
// bfloat16 by 64, SiLU / GELU: 62 / 69 us; four rows at a time and one CTA 99 / 80, two CTAs 66 / 75; four CTAs 60 / 66, with spills that cost binary32
// and small ones more; at three, instances spill up to 72 bytes, binary16's with lines up to 296, which one row at a time avoids but takes longer: 119 -> 124).
// gz (may be null) [n][ld], rounded to T; partial (may be null) [gridDim.y][m]: the sums of the CTA's rows, of gz before its rounding.
template <typename T, bool kVec>
__device__ __forceinline__ void load8(const T* p, long long stride, int count, T (&x)[8]) {
  if (kVec) {
#pragma unroll
    for (int j = 0; j < (int)sizeof(T) / 2; ++j) reinterpret_cast<uint4*>(x)[j] = __ldg(reinterpret_cast<const uint4*>(p) + j);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = p[min(j, count - 1) * stride];
  }
}
template <typename T, int kAct, bool kVec>
__device__ __forceinline__ void gz_rows(const Operand& gout, const Operand& preact, long long m, T* gz, long long ld, long long c, long long r0,
                                        long long r1, int warp, const Lines& lines, float (&total)[8]) {
  constexpr bool kLines = std::is_same<T, __half>::value && kAct != STRADS_ACT_IDENTITY;
  constexpr int kU = 2;
  const int count = (int)min(8ll, m - c);
  float power[kLines ? 8 : 1] = {};
  if (kLines && lines.by_column != nullptr)
#pragma unroll
    for (int j = 0; j < (kLines ? 8 : 0); ++j) power[j] = line_power(lines.column_factors[c + min(j, count - 1)]);
  for (long long r = r0 + warp; r < r1; r += 8 * kU) {
    __align__(16) T g[kU][8], z[kU][8];
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      const long long row = min(r + 8 * u, r1 - 1);
      load8<T, kVec>(static_cast<const T*>(gout.p) + row * gout.rs + c * gout.ks, gout.ks, count, g[u]);
      if (kAct != STRADS_ACT_IDENTITY) load8<T, kVec>(static_cast<const T*>(preact.p) + row * preact.rs + c * preact.ks, preact.ks, count, z[u]);
    }
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      if (r + 8 * u >= r1) break;
      __align__(16) T out[8];
      __align__(16) T out_c[kLines ? 8 : 1];
      const float row_power = kLines && gz != nullptr ? line_power(lines.row_factors[r + 8 * u]) : 1.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        float v = load_f32(&g[u][j]);
        if (kAct != STRADS_ACT_IDENTITY) v *= slope_as<sizeof(T) == 4, kAct>(load_f32(&z[u][j]));
        if (kVec || j < count) total[j] += v;
        store_f32(&out[j], kLines ? v * row_power : v);
        if (kLines) store_f32(&out_c[kLines ? j : 0], v * power[kLines ? j : 0]);
      }
      if (kLines && lines.by_column != nullptr) *reinterpret_cast<uint4*>(lines.by_column + (r + 8 * u) * ld + c) = *reinterpret_cast<const uint4*>(out_c);
      if (gz != nullptr)                                 // (ld is a multiple of 8: the last group has its place)
#pragma unroll
        for (int j = 0; j < (int)sizeof(T) / 2; ++j) reinterpret_cast<uint4*>(gz + (r + 8 * u) * ld + c)[j] = reinterpret_cast<const uint4*>(out)[j];
    }
  }
}
template <typename T, int kAct>
__global__ void __launch_bounds__(kThreads, 3) k_linear_gz(Operand gout, Operand preact, long long n, long long m, T* gz, long long ld,
                                                        float* partial, long long rows, int vec, Lines lines) {
  __shared__ float sum[8][256 + 8];
  chain_begin();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const long long c = (long long)blockIdx.x * 256 + lane * 8, r0 = (long long)blockIdx.y * rows, r1 = min(n, r0 + rows);
  float total[8] = {};
  if (vec && c + 8 <= m) gz_rows<T, kAct, true>(gout, preact, m, gz, ld, c, r0, r1, warp, lines, total);
  else if (c < m) gz_rows<T, kAct, false>(gout, preact, m, gz, ld, c, r0, r1, warp, lines, total);
  if (partial == nullptr) return;
#pragma unroll
  for (int j = 0; j < 8; ++j) sum[warp][j * 33 + lane] = total[j];
  __syncthreads();
  const long long col = (long long)blockIdx.x * 256 + threadIdx.x;
  if (col < m) {
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < 8; ++w) v += sum[w][(threadIdx.x & 7) * 33 + (threadIdx.x >> 3)];
    partial[(long long)blockIdx.y * m + col] = v;
  }
}
// 32 columns to a CTA, eight warps taking a run of the blocks of rows each.
template <typename T>
__global__ void __launch_bounds__(kThreads) k_linear_bias_grad(const float* partial, int blocks, long long m, float scale, T* gbias) {
  __shared__ float sum[8][32];
  chain_begin();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const long long c = (long long)blockIdx.x * 32 + lane;
  float s = 0.f;
  if (c < m)
#pragma unroll 4
    for (int r = blocks * warp / 8; r < blocks * (warp + 1) / 8; ++r) s += partial[r * m + c];
  sum[warp][lane] = s;
  __syncthreads();
  if (warp == 0 && c < m) {
#pragma unroll
    for (int w = 1; w < 8; ++w) s += sum[w][lane];
    store_f32(gbias + c, scale * s);
  }
}

template <typename T>
__global__ void __launch_bounds__(kThreads) k_linear_zero(T* p, long long rows, long long cols, long long rs, long long cs) {
  chain_begin();
  for (long long i = (long long)blockIdx.x * kThreads + threadIdx.x; i < rows * cols; i += (long long)gridDim.x * kThreads)
    store_f32(p + i / cols * rs + i % cols * cs, 0.f);
}

// ---- the order of kernels ----
// A call is gone through twice by the same code: with `run` false to add up the workspace, then to launch.  `all`: a query for any call of
// this configuration: everything is wanted, and where gout and the results will lie is not known.
struct Call {
  int type;
  size_t size;                           // of an element
  char* ws;
  size_t used;
  bool run, all, stall;
  cudaStream_t stream;
  cudaError_t err;
  unsigned int* status;
  Copies copies;                         // to be made before the next product
  LinesJob lines;                        // likewise, in the same launch
  void* take(size_t bytes) {
    void* p = ws + used;
    used += (bytes + 255) / 256 * 256;
    return p;
  }
};
constexpr int kGrid = 148 * 8;           // CTAs of the passes over an operand: enough to keep the memory busy

unsigned ctas_for(long long groups) {
  const long long n = (groups + kThreads - 1) / kThreads;
  return (unsigned)(n < 1 ? 1 : n > kGrid ? kGrid : n);
}
bool vec_rows(const void* p, long long pitch, long long rows, size_t size) {
  return ((uintptr_t)p & 15) == 0 && (rows == 1 || (pitch * (long long)size) % 16 == 0);
}

// Whether TMA reads a 16-bit operand where it is: one of its strides 1, the other and its start on 16 bytes.
bool in_place(const Operand& m, long long rows, long long nk) {
  const bool rows_inner = m.ks != 1 && (m.rs == 1 || rows == 1) && nk > 1;
  const long long inner = rows_inner ? rows : nk, outer = rows_inner ? nk : rows, outer_stride = rows_inner ? m.ks : m.rs, inner_stride = rows_inner ? m.rs : m.ks;
  return (inner_stride == 1 || inner == 1) && ((uintptr_t)m.p & 15) == 0 && (outer == 1 || (outer_stride % 8 == 0 && outer_stride >= inner));
}

// `unknown`: where the matrix lies is not known yet (a workspace query), so that it has to be taken for one that is copied.
Planes bring(Call& c, const Operand& m, long long rows, long long nk, bool unknown = false, bool k_inner = false) {
  const bool rows_inner = !k_inner && m.ks != 1 && (m.rs == 1 || rows == 1) && nk > 1;
  Planes p = {};
  p.rows_inner = rows_inner;
  p.inner = rows_inner ? rows : nk;
  p.outer = rows_inner ? nk : rows;
  const long long outer_stride = rows_inner ? m.ks : m.rs, inner_stride = rows_inner ? m.rs : m.ks;
  p.planes = c.size == 4 ? 3 : 1;
  if (!unknown && !k_inner && c.size == 2 && in_place(m, rows, nk)) {
    p.p = m.p;
    p.ld = p.outer == 1 ? (p.inner + 7) / 8 * 8 : outer_stride;
    return p;
  }
  p.ld = (p.inner + 7) / 8 * 8;
  p.plane = p.outer * p.ld;
  if (unknown && p.inner * ((p.outer + 7) / 8 * 8) > p.plane) p.plane = p.inner * ((p.outer + 7) / 8 * 8);      // (either order)
  void* dst = c.take((size_t)p.plane * p.planes * 2);
  p.p = dst;
  if (!c.run) return p;
  c.copies.c[c.copies.n++] = {m.p, outer_stride, inner_stride, p.outer, p.inner, p.ld, p.plane, static_cast<unsigned short*>(dst),
                              inner_stride == 1 && vec_rows(m.p, outer_stride, p.outer, c.size)};
  return p;
}
// The copies asked for so far, and the factors of lines, in one launch.
void copy(Call& c) {
  if (!c.run || c.err != cudaSuccess || (c.copies.n == 0 && c.lines.ctas == 0)) return;
  c.copies.groups = 0;
  for (int i = 0; i < c.copies.n; ++i) c.copies.groups += c.copies.c[i].plane / 8;
  c.copies.ctas = c.copies.n > 0 ? (int)ctas_for(c.copies.groups) : 0;
  const unsigned grid = (unsigned)(c.copies.ctas + c.lines.ctas);
  c.err = c.size == 4 ? launch_chained(k_linear_pack<float>, grid, kThreads, 0, c.stream, c.copies, c.lines)
                      : launch_chained(k_linear_pack<__half>, grid, kThreads, 0, c.stream, c.copies, c.lines);
  c.copies.n = 0;
  c.lines.ctas = 0;
}

// A matrix as one side of products, brought into the workspace at most once: the other side of its transpose is the same copy.
struct Matrix {
  Operand m;                             // element (row, column)
  long long rows, cols;
  bool unknown, brought;
  int order;                             // which of two equally long sides counts as the longer: the same whichever way D lies
  Planes p;
};
Operand operand_of(const strads_const_matrix_t& m) { return Operand{m.data, (long long)m.row_stride, (long long)m.col_stride}; }
Matrix matrix_of(const Operand& m, long long rows, long long cols, int order) {
  Matrix x = {};
  x.m = m; x.rows = rows; x.cols = cols; x.order = order;
  return x;
}
Planes side_of(Call& c, Matrix& x, bool columns_as_rows) {
  if (!x.brought) { x.p = bring(c, x.m, x.rows, x.cols, x.unknown); x.brought = true; }
  Planes p = x.p;
  if (columns_as_rows) p.rows_inner = !p.rows_inner;
  return p;
}

// D = A B^T, A and B matrices or (t) their transposes: which kernel forms it, and its operands as that reads them.
struct Product {
  enum Way { kNone, kThin, kSplit, kTensor } way;
  Operand a, b;
  long long na, nb, nk;
  Planes pa, pb;
  void* ws;
  bool b_long;
  Finish f;
};
Product plan(Call& c, Matrix& A, bool ta, Matrix& B, bool tb, const Finish& f) {
  Product d = {};
  d.a = ta ? Operand{A.m.p, A.m.ks, A.m.rs} : A.m;
  d.b = tb ? Operand{B.m.p, B.m.ks, B.m.rs} : B.m;
  d.na = ta ? A.cols : A.rows; d.nb = tb ? B.cols : B.rows; d.nk = ta ? A.rows : A.cols;
  d.f = f;
  d.b_long = d.na < d.nb || (d.na == d.nb && B.order < A.order);
  const Operand &l = d.b_long ? d.b : d.a, &sh = d.b_long ? d.a : d.b;
  const long long nl = d.b_long ? d.nb : d.na, ns = d.b_long ? d.na : d.nb;
  const bool unknown = (d.b_long ? B : A).unknown;       // (a query: room for any way)
  // Few rows on one side: streamed, if the tensor cores would first have to copy the long side or split it; 16-bit ones that they read where they are go
  // there at once (4,096 x 4,096 bfloat16: 11 us whatever the rows, streamed 14 with two, 13 with four), but for one row with k along memory (10.7) and
  // for long sides of so few rows that they make few tiles.  Those, four rows, out of cold L2, streamed / tensor cores: k along memory, 16,384 of it, 64 rows of
  // the long side 10 / 20 us, 512 14 / 23, 1,024 23 / 25, 1,536 31 / 27, 2,048 37 / 29; k = 1,024: 8 / 12, 8 / 12, 10 / 12, 12 / 12, 14 / 14.  (Rows along memory and
  // k = 16,384 the tensor cores are ahead throughout, 39 / 21 at 64 rows; k = 1,024 level.)
  // binary32, streamed / split: 4,096 x 4,096, one row 23 / 31, four 31 / 31; 1,000 x 10,000 21 / 29, 23 / 29; 10,000 x 20,000 by columns 141 / 156, 170 / 158, by rows
  // 162 / 152, 301 / 150.
  d.way = Product::kThin;
  if (ns <= kThinMost && !unknown && (c.size == 4 || !in_place(l, nl, d.nk) || (ns == 1 && l.ks == 1) || nl < 2048)) return d;
  // binary32 with up to kSplitMost rows on one side: the other is read once, where it is, and split on the way (4 bytes an element for every 32 or 48
  // rows, most of them from L2, where planes in memory cost 16).  Split / planes: 10,000 x 20,000 by 8 rows 150 / 643 us, by 128 395 / 864, by 256 760 / 1,333; 4,096 x
  // 4,096 31 / 84, 49 / 78, 82 / 98: the planes' own rule would be later still.
  if (c.size == 4 && ns <= kSplitMost && (unknown || linear_split_takes(l, nl, d.nk))) {
    d.way = Product::kSplit;
    d.pb = bring(c, sh, ns, d.nk, false, true);
    d.ws = c.take(linear_split_workspace(nl, ns, d.nk));
    if (!unknown) return d;
  }
  d.way = Product::kTensor;
  d.pa = side_of(c, A, ta);
  d.pb = side_of(c, B, tb);
  return d;
}
void launch(Call& c, const Product& d) {
  if (!c.run || c.err != cudaSuccess || d.way == Product::kNone) return;
  if (d.way == Product::kThin)
    c.err = launch_linear_thin(c.type, d.a, d.b, d.na, d.nb, d.nk, d.f, c.status, c.stall, c.stream);
  else if (d.way == Product::kSplit)
    c.err = launch_linear_split(d.b_long ? d.b : d.a, d.pb, d.b_long ? d.nb : d.na, d.b_long ? d.na : d.nb, d.nk, d.b_long, d.f, d.ws, c.status, c.stall, c.stream);
  else
    c.err = launch_linear_tc(c.type, d.pa, d.pb, d.na, d.nb, d.nk, d.f, c.status, c.stall, c.stream);
}

Side side(const void* p, long long rs, long long cs, bool a_is_rows) { return a_is_rows ? Side{p, rs, cs} : Side{p, cs, rs}; }
// Which of D's sides runs through memory (the rows only where the columns do not).
bool rows_run(long long rs, long long cs) { return cs != 1 && rs == 1; }

void forward(Call& c, const strads_linear_config_t& g, const void* bias, const strads_const_matrix_t* residual, const strads_matrix_t* out,
             const strads_matrix_t* preact) {
  Matrix x = matrix_of(operand_of(g.x), g.n_rows, g.n_in, 0), w = matrix_of(operand_of(g.w), g.n_out, g.n_in, 1);
  Finish f = {};
  f.act = g.activation; f.scale = g.scale; f.bias = bias;
  bool ar = false;
  if (out != nullptr) {
    ar = rows_run(out->row_stride, out->col_stride);
    f.out = side(out->data, out->row_stride, out->col_stride, ar);
  }
  if (residual) f.residual = side(residual->data, residual->row_stride, residual->col_stride, ar);
  if (preact) f.preact = side(preact->data, preact->row_stride, preact->col_stride, ar);
  f.bias_a = ar ? 0 : 1; f.bias_b = ar ? 1 : 0;
  f.plain = g.activation == STRADS_ACT_IDENTITY && bias == nullptr && residual == nullptr && preact == nullptr;
  const Product d = ar ? plan(c, x, false, w, false, f) : plan(c, w, false, x, false, f);
  copy(c);
  launch(c, d);
}

// gz = gout act'(z) and its column sums: the places of what they need, and their kernels' arguments.  The products read gz from `for_x` and `for_w`; binary16's, through an
// activation, with the factors of the lines that their results keep.
template <typename T>
struct Gz {
  bool formed, by_lines;
  long long columns, rows, ld;           // blocks of 256 columns, and of `rows` rows
  int blocks;
  T *for_x, *for_w;
  unsigned short *row_tops, *col_tops;
  float *row_factors, *column_factors, *partial;
};
template <typename T>
Gz<T> plan_z(Call& c, const strads_linear_config_t& g, bool want_x, bool want_w, bool want_bias) {
  Gz<T> k = {};
  k.formed = g.activation != STRADS_ACT_IDENTITY && (want_x || want_w);
  k.by_lines = k.formed && std::is_same<T, __half>::value;
  // at most 128 blocks of rows; of 64 rows where that leaves four CTAs to an SM, else of as few as 8
  k.columns = (g.n_out + 255) / 256;
  k.rows = (g.n_rows * k.columns + 4 * 148 - 1) / (4 * 148);
  if (k.rows > 64) k.rows = 64;
  if (k.rows * 128 < g.n_rows) k.rows = (g.n_rows + 127) / 128;
  k.rows = (k.rows + 7) / 8 * 8;
  k.blocks = (int)((g.n_rows + k.rows - 1) / k.rows);
  k.ld = (g.n_out + 7) / 8 * 8;
  const size_t n = (size_t)g.n_rows, m = (size_t)g.n_out, bytes = n * (size_t)k.ld * sizeof(T);
  if (k.formed && (want_x || !k.by_lines)) k.for_x = static_cast<T*>(c.take(bytes));
  k.for_w = !k.by_lines ? k.for_x : want_w ? static_cast<T*>(c.take(bytes)) : nullptr;
  if (k.by_lines && want_x) {
    k.row_tops = static_cast<unsigned short*>(c.take(n * (size_t)k.columns * 2));
    k.row_factors = static_cast<float*>(c.take(n * 4));
  }
  if (k.by_lines && want_w) {
    k.col_tops = static_cast<unsigned short*>(c.take(m * (size_t)k.blocks * 2));
    k.column_factors = static_cast<float*>(c.take(m * 4));
  }
  if (want_bias) k.partial = static_cast<float*>(c.take((size_t)k.blocks * m * sizeof(float)));
  return k;
}
// What the factors of lines are formed from; they themselves come with the next copies.
template <typename T>
void tops_of_gout(Call& c, const Gz<T>& k, const strads_linear_config_t& g, const strads_const_matrix_t& gout) {
  if (!c.run || c.err != cudaSuccess) return;
  const Operand o = operand_of(gout);
  const long long n = g.n_rows, m = g.n_out;
  const int vec = o.ks == 1 && vec_rows(o.p, o.rs, n, sizeof(T));
  c.err = launch_chained(k_linear_tops, dim3((unsigned)k.columns, (unsigned)k.blocks), kThreads, 0, c.stream, o, n, m, k.col_tops, k.row_tops, k.rows, vec);
  const int column_ctas = k.col_tops ? (int)((m + 31) / 32) : 0, row_ctas = k.row_tops ? (int)((n + kThreads - 1) / kThreads) : 0;
  c.lines = {k.col_tops, k.row_tops, k.column_factors, k.row_factors, n, m, k.blocks, (int)k.columns, column_ctas, column_ctas + row_ctas};
}
template <typename T>
void gradient_of_z(Call& c, const Gz<T>& k, const strads_linear_config_t& g, const strads_const_matrix_t& gout, const strads_const_matrix_t* preact, T* gbias) {
  if (!c.run || c.err != cudaSuccess || (!k.formed && gbias == nullptr)) return;
  const Operand o = operand_of(gout);
  Operand z = {};
  if (preact) z = operand_of(*preact);
  const int vec = gout.col_stride == 1 && vec_rows(gout.data, gout.row_stride, g.n_rows, sizeof(T)) &&
                  (g.activation == STRADS_ACT_IDENTITY || (z.ks == 1 && vec_rows(z.p, z.rs, g.n_rows, sizeof(T))));
  Lines lines = {};
  if constexpr (std::is_same<T, __half>::value) lines = {k.row_factors, k.column_factors, k.by_lines ? k.for_w : nullptr};
  void (*kernel)(Operand, Operand, long long, long long, T*, long long, float*, long long, int, Lines) = k_linear_gz<T, STRADS_ACT_IDENTITY>;
  switch (g.activation) {
    case STRADS_ACT_RELU: kernel = k_linear_gz<T, STRADS_ACT_RELU>; break;
    case STRADS_ACT_SIGMOID: kernel = k_linear_gz<T, STRADS_ACT_SIGMOID>; break;
    case STRADS_ACT_GELU: kernel = k_linear_gz<T, STRADS_ACT_GELU>; break;
    case STRADS_ACT_GELU_TANH: kernel = k_linear_gz<T, STRADS_ACT_GELU_TANH>; break;
    case STRADS_ACT_SILU: kernel = k_linear_gz<T, STRADS_ACT_SILU>; break;
    default: break;
  }
  c.err = launch_chained(kernel, dim3((unsigned)k.columns, (unsigned)k.blocks), kThreads, 0, c.stream, o, z, (long long)g.n_rows, (long long)g.n_out,
                         k.for_x, k.ld, k.partial, k.rows, vec, lines);
  if (gbias != nullptr && c.err == cudaSuccess)
    c.err = launch_chained(k_linear_bias_grad<T>, dim3((unsigned)((g.n_out + 31) / 32)), kThreads, 0, c.stream, static_cast<const float*>(k.partial), k.blocks, (long long)g.n_out, g.scale, gbias);
}

template <typename T>
void backward(Call& c, const strads_linear_config_t& g, const strads_const_matrix_t& gout, const strads_const_matrix_t* preact, const strads_matrix_t* gx,
              const strads_matrix_t* gw, void* gbias) {
  if (g.n_rows == 0) {
    if (!c.run) return;
    if (gw != nullptr)
      c.err = launch_chained(k_linear_zero<T>, ctas_for(g.n_out * g.n_in), kThreads, 0, c.stream, static_cast<T*>(gw->data), (long long)g.n_out, (long long)g.n_in, (long long)gw->row_stride, (long long)gw->col_stride);
    if (gbias != nullptr && c.err == cudaSuccess)
      c.err = launch_chained(k_linear_zero<T>, ctas_for(g.n_out), kThreads, 0, c.stream, static_cast<T*>(gbias), 1ll, (long long)g.n_out, (long long)g.n_out, 1ll);
    return;
  }
  // the identity's gz is gout itself; otherwise gz is formed, and its column sums on the way; scale is a factor of the results
  const bool want_x = gx != nullptr || c.all, want_w = gw != nullptr || c.all;
  const Gz<T> gz = plan_z<T>(c, g, want_x, want_w, gbias != nullptr || c.all);
  Operand for_x = operand_of(gout), for_w = for_x;
  if (gz.formed) { for_x = {gz.for_x, gz.ld, 1}; for_w = {gz.for_w, gz.ld, 1}; }
  Matrix z = matrix_of(for_x, g.n_rows, g.n_out, 2), z_w = matrix_of(for_w, g.n_rows, g.n_out, 2);
  Matrix x = matrix_of(operand_of(g.x), g.n_rows, g.n_in, 0), w = matrix_of(operand_of(g.w), g.n_out, g.n_in, 1);
  Matrix& zw = gz.by_lines ? z_w : z;      // (else one and the same, brought once)
  z.unknown = !gz.formed && c.all;
  Finish f = {};
  f.plain = 1;
  f.scale = g.scale;
  Product dx = {}, dw = {};
  if (want_x) {
    const bool ar = gx != nullptr && rows_run(gx->row_stride, gx->col_stride);
    if (gx != nullptr) f.out = side(gx->data, gx->row_stride, gx->col_stride, ar);
    f.factor = gz.row_factors; f.factor_a = ar ? 1 : 0; f.factor_b = ar ? 0 : 1;
    dx = ar ? plan(c, z, false, w, true, f) : plan(c, w, true, z, false, f);
  }
  if (want_w) {
    const bool ar = gw != nullptr && rows_run(gw->row_stride, gw->col_stride);
    if (gw != nullptr) f.out = side(gw->data, gw->row_stride, gw->col_stride, ar);
    f.factor = gz.column_factors; f.factor_a = ar ? 1 : 0; f.factor_b = ar ? 0 : 1;
    dw = ar ? plan(c, zw, true, x, true, f) : plan(c, x, true, zw, true, f);
  }
  if (gz.by_lines) {                     // (gz is read where it is: the copies are of others, and go with the factors that it needs)
    tops_of_gout(c, gz, g, gout);
    copy(c);
  }
  gradient_of_z(c, gz, g, gout, preact, static_cast<T*>(gbias));
  copy(c);
  launch(c, dx);
  launch(c, dw);
}
void backward_of(Call& c, const strads_linear_config_t& g, const strads_const_matrix_t& gout, const strads_const_matrix_t* preact, const strads_matrix_t* gx,
                 const strads_matrix_t* gw, void* gbias) {
  if (g.type == STRADS_F32) backward<float>(c, g, gout, preact, gx, gw, gbias);
  else if (g.type == STRADS_BF16) backward<__nv_bfloat16>(c, g, gout, preact, gx, gw, gbias);
  else backward<__half>(c, g, gout, preact, gx, gw, gbias);
}
Call call_of(const strads_linear_config_t& g, bool run, bool all) {
  Call c = {};
  c.type = g.type; c.size = g.type == STRADS_F32 ? 4 : 2;
  c.run = run; c.all = all; c.stall = (g.flags & STRADS_LINEAR_FLAG_STALL) != 0;
  c.ws = run ? static_cast<char*>(g.workspace) : nullptr;
  c.stream = static_cast<cudaStream_t>(g.stream);
  c.err = cudaSuccess;
  if (run) {
    void* p = nullptr;
    c.err = cudaGetSymbolAddress(&p, g_linear_status);
    c.status = static_cast<unsigned int*>(p);
  }
  return c;
}

bool valid_strides(long long rs, long long cs) { return rs >= 0 && cs >= 0; }
bool valid_in(const strads_const_matrix_t& m, int size) {
  return m.data != nullptr && ((uintptr_t)m.data % size) == 0 && valid_strides(m.row_stride, m.col_stride);
}
// What is written: no two elements at one place.  (Two strides with extents: the inner run, (n - 1) strides long, must end before the outer step.)
bool valid_out(const strads_matrix_t& m, int size, long long rows, long long cols) {
  if (m.data == nullptr || ((uintptr_t)m.data % size) != 0 || !valid_strides(m.row_stride, m.col_stride)) return false;
  long long s1 = m.row_stride, n1 = rows, s2 = m.col_stride, n2 = cols;
  if (n1 <= 1) { s1 = 0; n1 = 1; }
  if (n2 <= 1) { s2 = 0; n2 = 1; }
  if ((n1 > 1 && s1 == 0) || (n2 > 1 && s2 == 0)) return false;
  if (n1 == 1 || n2 == 1) return true;
  return s1 <= s2 ? (s2 - 1) / s1 >= n1 - 1 : (s1 - 1) / s2 >= n2 - 1;
}

int check(const strads_linear_config_t& c) {
  if (c.type < STRADS_F32 || c.type > STRADS_F16 || c.activation < STRADS_ACT_IDENTITY || c.activation > STRADS_ACT_SILU) return STRADS_ERR_INVALID_ARG;
  if (c.n_rows < 0 || c.n_in < 1 || c.n_out < 1 || !std::isfinite(c.scale) || (c.flags & ~STRADS_LINEAR_FLAG_STALL) != 0) return STRADS_ERR_INVALID_ARG;
  constexpr long long kMost = 1ll << 30;                 // (places of tiles, and what lies past the last, fit 32 bits)
  if (c.n_rows > kMost || c.n_in > kMost || c.n_out > kMost) return STRADS_ERR_UNSUPPORTED;
  const int size = c.type == STRADS_F32 ? 4 : 2;
  if (!valid_in(c.w, size) || (c.n_rows > 0 && !valid_in(c.x, size))) return STRADS_ERR_INVALID_ARG;
  return STRADS_OK;
}

}  // namespace
}  // namespace strads

using namespace strads;

extern "C" {

int strads_linear_workspace_bytes(const strads_linear_config_t* cfg, size_t* forward_out, size_t* backward_out) {
  if (cfg == nullptr || forward_out == nullptr || backward_out == nullptr) return STRADS_ERR_INVALID_ARG;
  const int rc = check(*cfg);
  if (rc != STRADS_OK) return rc;
  Call f = call_of(*cfg, false, true), b = call_of(*cfg, false, true);
  if (cfg->n_rows > 0) {
    forward(f, *cfg, nullptr, nullptr, nullptr, nullptr);
    backward_of(b, *cfg, strads_const_matrix_t{nullptr, 0, 0}, nullptr, nullptr, nullptr, nullptr);
  }
  *forward_out = f.used;
  *backward_out = b.used;
  return STRADS_OK;
}

static int check_workspace(const strads_linear_config_t& c, size_t need) {
  if (c.workspace_bytes < need) return STRADS_ERR_WORKSPACE_TOO_SMALL;
  return need > 0 && (c.workspace == nullptr || ((uintptr_t)c.workspace & 255) != 0) ? STRADS_ERR_INVALID_ARG : STRADS_OK;
}

int strads_linear_forward(const strads_linear_config_t* cfg, const void* bias, const strads_const_matrix_t* residual,
                          const strads_matrix_t* out, const strads_matrix_t* preact) {
  if (cfg == nullptr) return STRADS_ERR_INVALID_ARG;
  int rc = check(*cfg);
  if (rc != STRADS_OK) return rc;
  const strads_linear_config_t& c = *cfg;
  if (c.n_rows == 0) return STRADS_OK;
  const int size = c.type == STRADS_F32 ? 4 : 2;
  if (out == nullptr || !valid_out(*out, size, c.n_rows, c.n_out) || (preact != nullptr && !valid_out(*preact, size, c.n_rows, c.n_out)) ||
      (residual != nullptr && !valid_in(*residual, size)) || ((uintptr_t)bias % size) != 0)
    return STRADS_ERR_INVALID_ARG;
  Call sizes = call_of(c, false, false);
  forward(sizes, c, bias, residual, out, preact);
  if ((rc = check_workspace(c, sizes.used)) != STRADS_OK) return rc;
  Call call = call_of(c, true, false);
  forward(call, c, bias, residual, out, preact);
  return call.err == cudaSuccess ? STRADS_OK : cuda_failed(call.err, "strads_linear_forward");
}

int strads_linear_backward(const strads_linear_config_t* cfg, const strads_const_matrix_t* gout, const strads_const_matrix_t* preact,
                           const strads_matrix_t* gx, const strads_matrix_t* gw, void* gbias) {
  if (cfg == nullptr) return STRADS_ERR_INVALID_ARG;
  int rc = check(*cfg);
  if (rc != STRADS_OK) return rc;
  const strads_linear_config_t& c = *cfg;
  const int size = c.type == STRADS_F32 ? 4 : 2;
  if (c.n_rows > 0) {
    if (gout == nullptr || !valid_in(*gout, size) || (preact != nullptr && !valid_in(*preact, size)) ||
        (preact == nullptr && c.activation != STRADS_ACT_IDENTITY) || (gx != nullptr && !valid_out(*gx, size, c.n_rows, c.n_in)))
      return STRADS_ERR_INVALID_ARG;
  }
  if ((gw != nullptr && !valid_out(*gw, size, c.n_out, c.n_in)) || ((uintptr_t)gbias % size) != 0) return STRADS_ERR_INVALID_ARG;
  if (gx == nullptr && gw == nullptr && gbias == nullptr) return STRADS_OK;
  const strads_const_matrix_t none = {nullptr, 0, 0};
  const strads_const_matrix_t& g = gout ? *gout : none;
  Call sizes = call_of(c, false, false);
  backward_of(sizes, c, g, preact, gx, gw, gbias);
  if ((rc = check_workspace(c, sizes.used)) != STRADS_OK) return rc;
  Call call = call_of(c, true, false);
  backward_of(call, c, g, preact, gx, gw, gbias);
  return call.err == cudaSuccess ? STRADS_OK : cuda_failed(call.err, "strads_linear_backward");
}

int strads_linear_status(uint32_t* bits_host_out) {
  if (bits_host_out == nullptr) return STRADS_ERR_INVALID_ARG;
  const unsigned int none = 0u;
  unsigned int bits = 0u;
  cudaError_t e = cudaDeviceSynchronize();
  if (e == cudaSuccess) e = cudaMemcpyFromSymbol(&bits, g_linear_status, sizeof(bits));
  if (e == cudaSuccess && bits != 0u) e = cudaMemcpyToSymbol(g_linear_status, &none, sizeof(none));
  if (e != cudaSuccess) return cuda_failed(e, "strads_linear_status");
  *bits_host_out = bits;
  return (bits & STRADS_STATUS_WAIT_EXPIRED) ? STRADS_ERR_TIMEOUT : STRADS_OK;
}

}  // extern "C"
