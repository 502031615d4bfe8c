// A step of AdamW (Adam with decoupled weight decay) over many tensors at once, with an optional L1 threshold, the moments
// held in 32 or in 8 bits; and the reading back of moments held in 8.
//
//   g = grad_scale * grad        m = beta1 m + (1 - beta1) g        v = beta2 v + (1 - beta2) g^2
//   d = sqrt(v) / sqrt(1 - beta2^t) + eps      p = p (1 - lr decay) - lr / (1 - beta1^t) m / d      p = S(p, lr l1 / d)
//
// Every element is a fixed sequence of correctly rounded binary32 operations (explicit _rn intrinsics, never contracted), so
// the result does not depend on how the tensors are cut into CTAs or on their alignment.  The scalars of a step are formed in
// binary64 and rounded once.
//
// 8 bits: a tensor is cut into blocks of 256; a block keeps one binary32 scale for each moment.  m = s q |q| with q in
// -127 .. 127 (-128: not finite), sqrt(v) = s q^2 with q in 0 .. 254 (255: not finite).  Squares of the codes, because
// moments spread over orders of magnitude: the largest of a block are held to 0.8 % (m) and 0.4 % (sqrt v), the smallest that
// is not nought is 1/16,129 and 1/64,516 of the largest.  A root that is not 0 never becomes 0: its coefficient would move by m / eps.
//
// Bound by memory: 28 bytes an element with everything in 32 bits, 16 with 16-bit parameters and gradients, masters and 8-bit
// moments.  A warp takes a block of 256 at a time, a lane two groups of four neighbours 128 apart, so that every
// access of the warp is one run of memory whatever the type; the block's maxima are one warp reduction.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <cmath>
#include <new>

#include "strads_internal.cuh"

namespace strads {
namespace {

constexpr int kBlock = 256;                    // elements that share a scale
constexpr int kThreads = 256;
// Elements that a CTA takes: a block for each of its warps (100 M bfloat16 parameters with masters and 8-bit moments: 341 us; two blocks one after the
// other 438, four 394).
constexpr long long kChunk = (long long)(kThreads / 32) * kBlock;
constexpr float kTiny = 7.888609052210118e-31f;      // 2^-100: a block whose largest magnitude is below is stored as noughts

struct Entry {
  void* param; float* master; const void* grad; void* m; void* v; float* m_scale; float* v_scale;
  long long n_vec;                             // elements, times two, plus one where all pointers allow vector accesses
};
// The tensors of a launch travel as kernel parameters (at most 32,764 bytes): nothing to upload, nothing to keep alive, and a
// captured launch holds its own copy.
template <int kCap>
struct Table {
  int count;
  int first[kCap + 1];                         // CTA at which a tensor starts
  Entry e[kCap];
};
constexpr int kSmall = 16, kLarge = 440;

struct Scalars { float b1, ob1, b2, ob2, move, unbias, keep, eps, threshold, grad_scale; };
struct Step {
  Scalars c;
  double lr, beta1, beta2, weight_decay, l1, grad_scale;
  long long step;
  const float* lr_dev; const float* grad_scale_dev; const long long* step_dev; const int* skip_dev;
};

__host__ __device__ inline double power(double b, long long t) {      // b^t, t >= 0, by squaring
  double r = 1.0;
  for (; t > 0; t >>= 1, b *= b) if (t & 1) r *= b;
  return r;
}
__host__ __device__ inline void form_scalars(const Step& s, double lr, long long t, Scalars* c) {
  c->move = (float)(lr / (1.0 - power(s.beta1, t)));
  c->unbias = (float)(1.0 / sqrt(1.0 - power(s.beta2, t)));
  c->keep = (float)(1.0 - lr * s.weight_decay);
  c->threshold = (float)(lr * s.l1);
}

template <typename T> __device__ __forceinline__ T from_f32(float x);
template <> __device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half from_f32<__half>(float x) { return __float2half_rn(x); }

template <typename T> struct alignas(4 * sizeof(T)) Four { T x[4]; };

// A lane's eight elements of a block of which n are there: two groups of four, at lane * 4 and 128 + lane * 4.
// kFull: all 256 are, and 16 bytes of them may be accessed at once.  Elements that are not there read as 0.
template <typename T, bool kFull>
__device__ __forceinline__ void load8(const T* p, int n, int lane, float (&x)[8]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int i = h * 128 + lane * 4;
    if (kFull) {
      const Four<T> f = *reinterpret_cast<const Four<T>*>(p + i);
#pragma unroll
      for (int j = 0; j < 4; ++j) x[4 * h + j] = (float)f.x[j];
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) x[4 * h + j] = i + j < n ? (float)p[i + j] : 0.f;
    }
  }
}
template <typename T, bool kFull>
__device__ __forceinline__ void store8(T* p, int n, int lane, const float (&x)[8]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int i = h * 128 + lane * 4;
    if (kFull) {
      Four<T> f;
#pragma unroll
      for (int j = 0; j < 4; ++j) f.x[j] = from_f32<T>(x[4 * h + j]);
      *reinterpret_cast<Four<T>*>(p + i) = f;
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) if (i + j < n) p[i + j] = from_f32<T>(x[4 * h + j]);
    }
  }
}
// The same for codes, four in a word.
template <bool kFull>
__device__ __forceinline__ void load_codes(const void* codes, int n, int lane, unsigned int (&w)[2]) {
  const unsigned char* p = static_cast<const unsigned char*>(codes);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int i = h * 128 + lane * 4;
    if (kFull) {
      w[h] = *reinterpret_cast<const unsigned int*>(p + i);
    } else {
      w[h] = 0u;
#pragma unroll
      for (int j = 0; j < 4; ++j) if (i + j < n) w[h] |= (unsigned int)p[i + j] << (8 * j);
    }
  }
}
template <bool kFull>
__device__ __forceinline__ void store_codes(void* codes, int n, int lane, const unsigned int (&w)[2]) {
  unsigned char* p = static_cast<unsigned char*>(codes);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int i = h * 128 + lane * 4;
    if (kFull) {
      *reinterpret_cast<unsigned int*>(p + i) = w[h];
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) if (i + j < n) p[i + j] = (unsigned char)(w[h] >> (8 * j));
    }
  }
}

// Between codes and floats by the sum with 2^23 or 1.5 2^23, whose last bits then are the integer: the conversion instructions go through the
// unit that the roots and quotients need, at a quarter of the rate.
constexpr float kUnsigned = 8388608.f, kRounded = 12582912.f;
constexpr unsigned int kInfinity = 0x7f800000u;
__device__ __forceinline__ unsigned int zero_bytes(unsigned int x) { return (x - 0x01010101u) & ~x & 0x80808080u; }      // not 0: there is one
__device__ __forceinline__ float byte_as_float(unsigned int word, int j) {      // of byte j, plus kUnsigned
  return __uint_as_float(__byte_perm(word, 0x4b000000u, 0x7440u | (unsigned int)j));
}
// First moments, and roots of second ones, of eight codes.  The codes for what is not finite are looked for four at a time.
__device__ __forceinline__ void decode_m(const unsigned int (&w)[2], float s, float (&m)[8]) {
  const unsigned int x[2] = {w[0] ^ 0x80808080u, w[1] ^ 0x80808080u};      // the code plus 128: 0 stands for NaN
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float q = __fsub_rn(byte_as_float(x[j >> 2], j & 3), kUnsigned + 128.f);
    m[j] = __fmul_rn(__fmul_rn(q, fabsf(q)), s);
  }
  if (zero_bytes(x[0]) | zero_bytes(x[1])) {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (((x[j >> 2] >> (8 * (j & 3))) & 0xffu) == 0u) m[j] = __uint_as_float(0x7fc00000u);
  }
}
__device__ __forceinline__ void decode_root(const unsigned int (&w)[2], float s, float (&root)[8]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float q = __fsub_rn(byte_as_float(w[j >> 2], j & 3), kUnsigned);
    root[j] = __fmul_rn(__fmul_rn(q, q), s);
  }
  if (zero_bytes(~w[0]) | zero_bytes(~w[1])) {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (((w[j >> 2] >> (8 * (j & 3))) & 0xffu) == 255u) root[j] = __uint_as_float(0x7fc00000u);
  }
}
// Magnitudes order like their bits; what is not finite comes last.  The largest finite one of the block's x (this lane's eight, and the other lanes').
__device__ __forceinline__ float largest(const float (&x)[8], bool* all_finite) {
  unsigned int top = 0u;
#pragma unroll
  for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(fabsf(x[j])));
  top = __reduce_max_sync(0xffffffffu, top);
  *all_finite = top < kInfinity;
  if (top >= kInfinity) {
    top = 0u;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const unsigned int b = __float_as_uint(fabsf(x[j]));
      if (b < kInfinity) top = max(top, b);
    }
    top = __reduce_max_sync(0xffffffffu, top);
  }
  return __uint_as_float(top);
}
// Codes of eight values: the integer nearest to the correctly rounded root of |x| r (ties to even), with the value's sign.  The approximate root is
// good to 2^-14 where it matters (up to 254); only where one lies within 2^-12 of the middle between two integers are the exact ones needed.
// Without a sign, what is not 0 gets at least 1.
template <bool kSigned>
__device__ __forceinline__ void encode(const float (&x)[8], float r, bool all_finite, unsigned int (&w)[2]) {
  float t[8];
  bool near = false;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    float root;
    asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(root) : "f"(__fmul_rn(fabsf(x[j]), r)));
    if (kSigned) root = copysignf(root, x[j]);
    t[j] = __fadd_rn(root, kRounded);
    near = near || fabsf(__fsub_rn(root, __fsub_rn(t[j], kRounded))) > 0.499755859375f;
  }
  if (near) {
#pragma unroll 1
    for (int j = 0; j < 8; ++j) {
      float root = __fsqrt_rn(__fmul_rn(fabsf(x[j]), r));
      if (kSigned) root = copysignf(root, x[j]);
      const float v = __fadd_rn(root, kRounded);
#pragma unroll
      for (int i = 0; i < 8; ++i) if (i == j) t[i] = v;
    }
  }
  if (!kSigned)
#pragma unroll
    for (int j = 0; j < 8; ++j) t[j] = fmaxf(t[j], x[j] > 0.f ? kRounded + 1.f : kRounded);
#pragma unroll
  for (int h = 0; h < 2; ++h)
    w[h] = __byte_perm(__byte_perm(__float_as_uint(t[4 * h]), __float_as_uint(t[4 * h + 1]), 0x0040u),
                       __byte_perm(__float_as_uint(t[4 * h + 2]), __float_as_uint(t[4 * h + 3]), 0x0040u), 0x5410u);
  if (!all_finite) {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (__float_as_uint(fabsf(x[j])) >= kInfinity) {
        const unsigned int at = 8u * (j & 3);
        w[j >> 2] = (w[j >> 2] & ~(0xffu << at)) | ((kSigned ? 0x80u : 0xffu) << at);
      }
  }
}

// The scale of a block whose largest finite magnitude is `top`, and its inverse (both 0 where the block is stored as noughts).
__device__ __forceinline__ float scale_of(float top, float inverse_of_largest_code_squared, float* inverse) {
  const float s = top >= kTiny ? __fmul_rn(top, inverse_of_largest_code_squared) : 0.f;
  *inverse = s > 0.f ? __frcp_rn(s) : 0.f;
  return s;
}

// CTA -> tensor: the last entry that starts at or before it.
template <int kCap>
__device__ __forceinline__ int find_tensor(const Table<kCap>& t) {
  int lo = 0, hi = t.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (t.first[mid] <= (int)blockIdx.x) lo = mid; else hi = mid - 1;
  }
  return lo;
}

// One block of n elements from `at` on, by a warp.
template <typename P, typename G, bool kMaster, int kBits, bool kFull>
__device__ __forceinline__ void step_block(const Entry& e, const Scalars& c, long long at, int n, int lane) {
  P* param = static_cast<P*>(e.param) + at;
  float p[8], g[8], m[8], v[8];
  if (kMaster) load8<float, kFull>(e.master + at, n, lane, p); else load8<P, kFull>(param, n, lane, p);
  load8<G, kFull>(static_cast<const G*>(e.grad) + at, n, lane, g);
  if (kBits == 32) {
    load8<float, kFull>(static_cast<const float*>(e.m) + at, n, lane, m);
    load8<float, kFull>(static_cast<const float*>(e.v) + at, n, lane, v);
  } else {
    unsigned int w1[2], w2[2];
    load_codes<kFull>(static_cast<const unsigned char*>(e.m) + at, n, lane, w1);
    load_codes<kFull>(static_cast<const unsigned char*>(e.v) + at, n, lane, w2);
    const float s1 = e.m_scale[at / kBlock], s2 = e.v_scale[at / kBlock];
    decode_m(w1, s1, m);
    decode_root(w2, s2, v);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = __fmul_rn(v[j], v[j]);
  }
  float root[8], inv[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float gj = __fmul_rn(g[j], c.grad_scale);
    m[j] = __fadd_rn(__fmul_rn(m[j], c.b1), __fmul_rn(gj, c.ob1));
    v[j] = __fadd_rn(__fmul_rn(v[j], c.b2), __fmul_rn(__fmul_rn(gj, gj), c.ob2));
    root[j] = __fsqrt_rn(v[j]);
    inv[j] = __frcp_rn(__fadd_rn(__fmul_rn(root[j], c.unbias), c.eps));
    p[j] = __fsub_rn(__fmul_rn(p[j], c.keep), __fmul_rn(__fmul_rn(m[j], c.move), inv[j]));
  }
  if (c.threshold > 0.f) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float size = __fsub_rn(fabsf(p[j]), __fmul_rn(c.threshold, inv[j]));
      p[j] = size < 0.f ? 0.f : copysignf(size, p[j]);      // (a NaN stays one)
    }
  }
  store8<P, kFull>(param, n, lane, p);
  if (kMaster) store8<float, kFull>(e.master + at, n, lane, p);
  if (kBits == 32) {
    store8<float, kFull>(static_cast<float*>(e.m) + at, n, lane, m);
    store8<float, kFull>(static_cast<float*>(e.v) + at, n, lane, v);
  } else {
    unsigned int w[2];
    float r;
    bool all_finite;
    const float s1 = scale_of(largest(m, &all_finite), 1.f / 16129.f, &r);
    encode<true>(m, r, all_finite, w);
    store_codes<kFull>(static_cast<unsigned char*>(e.m) + at, n, lane, w);
    const float s2 = scale_of(largest(root, &all_finite), 1.f / 64516.f, &r);
    encode<false>(root, r, all_finite, w);
    store_codes<kFull>(static_cast<unsigned char*>(e.v) + at, n, lane, w);
    if (lane == 0) { e.m_scale[at / kBlock] = s1; e.v_scale[at / kBlock] = s2; }
  }
}

// 8 bits: five CTAs to an SM (48 registers, 4 to 8 bytes spilled, and a frame of 80 for the rare exact roots): bound by issuing some 85 instructions an
// element, it wants the warps (341 -> 320 us at 100 M parameters; six CTAs, with more spills, 352).
template <typename P, typename G, bool kMaster, int kBits, int kCap>
__global__ void __launch_bounds__(kThreads, kBits == 8 ? 5 : 1) k_adamw(const __grid_constant__ Table<kCap> t, const __grid_constant__ Step s) {
  if (s.skip_dev != nullptr && *s.skip_dev != 0) return;
  __shared__ Scalars sc;
  Scalars c = s.c;
  if (s.lr_dev != nullptr || s.step_dev != nullptr || s.grad_scale_dev != nullptr) {
    if (threadIdx.x == 0) {
      sc = c;
      form_scalars(s, s.lr_dev ? (double)*s.lr_dev : s.lr, s.step_dev ? *s.step_dev : s.step, &sc);
      if (s.grad_scale_dev) sc.grad_scale = *s.grad_scale_dev;
    }
    __syncthreads();
    c = sc;
  }
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int ti = find_tensor(t);
  const Entry& e = t.e[ti];
  const long long n_all = e.n_vec >> 1, at = (long long)((int)blockIdx.x - t.first[ti]) * kChunk + warp * kBlock;
  if (at >= n_all) return;
  if ((e.n_vec & 1) && at + kBlock <= n_all) step_block<P, G, kMaster, kBits, true>(e, c, at, kBlock, lane);
  else step_block<P, G, kMaster, kBits, false>(e, c, at, (int)min((long long)kBlock, n_all - at), lane);
}

// Moments held in 8 bits as the values that they stand for: entry.param receives m, entry.master v.
template <bool kFull>
__device__ __forceinline__ void unpack_block(const Entry& e, long long at, int n, int lane) {
  const float s1 = e.m_scale[at / kBlock], s2 = e.v_scale[at / kBlock];
  unsigned int w1[2], w2[2];
  load_codes<kFull>(static_cast<const unsigned char*>(e.m) + at, n, lane, w1);
  load_codes<kFull>(static_cast<const unsigned char*>(e.v) + at, n, lane, w2);
  float m[8], v[8];
  decode_m(w1, s1, m);
  decode_root(w2, s2, v);
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = __fmul_rn(v[j], v[j]);
  store8<float, kFull>(static_cast<float*>(e.param) + at, n, lane, m);
  store8<float, kFull>(e.master + at, n, lane, v);
}
template <int kCap>
__global__ void __launch_bounds__(kThreads) k_adamw_unpack(const __grid_constant__ Table<kCap> t) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int ti = find_tensor(t);
  const Entry& e = t.e[ti];
  const long long n_all = e.n_vec >> 1, at = (long long)((int)blockIdx.x - t.first[ti]) * kChunk + warp * kBlock;
  if (at >= n_all) return;
  if ((e.n_vec & 1) && at + kBlock <= n_all) unpack_block<true>(e, at, kBlock, lane);
  else unpack_block<false>(e, at, (int)min((long long)kBlock, n_all - at), lane);
}

bool aligned(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }
size_t size_of(int type) { return type == STRADS_F32 ? 4 : 2; }

// Cuts the list into launches of at most kLarge tensors; `launch(table, ctas)` enqueues one.
template <int kCap, typename F>
int fill_and_launch(const Entry* list, int count, F&& launch) {
  Table<kCap>* t = new (std::nothrow) Table<kCap>;      // (30 KB: not on the caller's stack)
  if (t == nullptr) return STRADS_ERR_CUDA;
  int rc = STRADS_OK;
  for (int i = 0; i < count && rc == STRADS_OK;) {
    t->count = 0;
    long long ctas = 0;
    while (i < count && t->count < kCap) {
      const long long more = ((list[i].n_vec >> 1) + kChunk - 1) / kChunk;
      if (ctas + more > 0x7fffffffll) break;             // (never on the first: sizes are checked)
      t->e[t->count] = list[i];
      t->first[t->count++] = (int)ctas;
      ctas += more;
      ++i;
    }
    t->first[t->count] = (int)ctas;
    rc = launch(*t, (unsigned)ctas);
  }
  delete t;
  return rc;
}
template <typename F>
int each_launch(const Entry* list, int count, F&& launch) {
  return count <= kSmall ? fill_and_launch<kSmall>(list, count, launch) : fill_and_launch<kLarge>(list, count, launch);
}

template <typename P, typename G, bool kMaster, int kBits>
int launch_step(const Entry* list, int count, const Step& s, cudaStream_t stream) {
  return each_launch(list, count, [&](const auto& table, unsigned ctas) {
    constexpr int kCap = sizeof(table.e) / sizeof(Entry);
    k_adamw<P, G, kMaster, kBits, kCap><<<ctas, kThreads, 0, stream>>>(table, s);
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? STRADS_OK : cuda_failed(e, "adamw step");
  });
}
template <typename P, typename G, bool kMaster>
int by_bits(int bits, const Entry* list, int count, const Step& s, cudaStream_t stream) {
  return bits == 8 ? launch_step<P, G, kMaster, 8>(list, count, s, stream) : launch_step<P, G, kMaster, 32>(list, count, s, stream);
}
template <typename P>
int by_grad(int grad_type, bool master, int bits, const Entry* list, int count, const Step& s, cudaStream_t stream) {
  if (grad_type == STRADS_F32)
    return master ? by_bits<P, float, true>(bits, list, count, s, stream) : by_bits<P, float, false>(bits, list, count, s, stream);
  return master ? by_bits<P, P, true>(bits, list, count, s, stream) : by_bits<P, P, false>(bits, list, count, s, stream);
}

constexpr long long kMaxElements = 1ll << 40;
constexpr float kLeastEps = 1.17549435e-38f;      // 2^-126: a smaller one's inverse may be infinite, and 0 times that (both moments 0) no step

// No two tensors may share parameters: the order in which they would be written is open.  Lists in the order of their
// addresses, as views of one flat buffer are, are checked on the way through.
bool distinct(const strads_adamw_tensor_t* t, int count, size_t size) {
  bool ascending = true;
  uintptr_t end = 0;
  for (int i = 0; i < count && ascending; ++i) {
    if (t[i].n == 0) continue;
    const uintptr_t b = (uintptr_t)t[i].param;
    ascending = b >= end;
    end = b + (size_t)t[i].n * size;
  }
  if (ascending) return true;
  struct Range { uintptr_t b, e; };
  Range* r = new (std::nothrow) Range[count];
  if (r == nullptr) return false;
  int k = 0;
  for (int i = 0; i < count; ++i)
    if (t[i].n > 0) r[k++] = {(uintptr_t)t[i].param, (uintptr_t)t[i].param + (size_t)t[i].n * size};
  std::sort(r, r + k, [](const Range& a, const Range& b) { return a.b < b.b; });
  bool ok = true;
  for (int i = 1; i < k; ++i) ok = ok && r[i].b >= r[i - 1].e;
  delete[] r;
  return ok;
}

}  // namespace
}  // namespace strads

using namespace strads;

extern "C" {

int strads_adamw_step(const strads_adamw_config_t* cfg, const strads_adamw_tensor_t* tensors, int32_t count) {
  if (cfg == nullptr || count < 0 || (count > 0 && tensors == nullptr)) return STRADS_ERR_INVALID_ARG;
  const strads_adamw_config_t& c = *cfg;
  if (c.state_bits != 32 && c.state_bits != 8) return STRADS_ERR_INVALID_ARG;
  if (c.param_type < STRADS_F32 || c.param_type > STRADS_F16) return STRADS_ERR_INVALID_ARG;
  if (c.grad_type != STRADS_F32 && c.grad_type != c.param_type) return STRADS_ERR_INVALID_ARG;
  if (!(c.lr >= 0.0 && c.lr <= 1e30) || !(c.beta1 >= 0.0 && c.beta1 < 1.0) || !(c.beta2 >= 0.0 && c.beta2 < 1.0) ||
      !((float)c.eps >= kLeastEps && c.eps <= 1e30) || !(c.weight_decay >= 0.0 && c.weight_decay <= 1e30) || !(c.l1 >= 0.0 && c.l1 <= 1e30) ||
      !(std::fabs(c.grad_scale) <= 1e30) || (c.step < 1 && c.step_dev == nullptr))
    return STRADS_ERR_INVALID_ARG;
  const size_t ps = size_of(c.param_type), gs = size_of(c.grad_type), ss = c.state_bits == 32 ? 4 : 1;
  bool masters = false, any = false;
  int live = 0;
  for (int i = 0; i < count; ++i) {
    const strads_adamw_tensor_t& t = tensors[i];
    if (t.n < 0) return STRADS_ERR_INVALID_ARG;
    if (t.n > kMaxElements) return STRADS_ERR_UNSUPPORTED;
    if (t.n == 0) continue;
    if (t.param == nullptr || t.grad == nullptr || t.m == nullptr || t.v == nullptr) return STRADS_ERR_INVALID_ARG;
    if (!aligned(t.param, ps) || !aligned(t.grad, gs) || !aligned(t.m, ss) || !aligned(t.v, ss) || !aligned(t.master, 4))
      return STRADS_ERR_INVALID_ARG;
    if (c.state_bits == 8 && (t.m_scale == nullptr || t.v_scale == nullptr || !aligned(t.m_scale, 4) || !aligned(t.v_scale, 4)))
      return STRADS_ERR_INVALID_ARG;
    if (t.master != nullptr && c.param_type == STRADS_F32) return STRADS_ERR_INVALID_ARG;
    if (any && masters != (t.master != nullptr)) return STRADS_ERR_INVALID_ARG;
    masters = t.master != nullptr;
    any = true;
    ++live;
  }
  if (live == 0) return STRADS_OK;
  if (!distinct(tensors, count, ps)) return STRADS_ERR_INVALID_ARG;
  Entry* list = new (std::nothrow) Entry[live];
  if (list == nullptr) return STRADS_ERR_INVALID_ARG;
  int k = 0;
  for (int i = 0; i < count; ++i) {
    const strads_adamw_tensor_t& t = tensors[i];
    if (t.n == 0) continue;
    const bool vec = aligned(t.param, 4 * ps) && aligned(t.grad, 4 * gs) && aligned(t.m, 4 * ss) && aligned(t.v, 4 * ss) &&
                     aligned(t.master, 16);
    list[k++] = Entry{t.param, t.master, t.grad, t.m, t.v, t.m_scale, t.v_scale, 2 * (long long)t.n + (vec ? 1 : 0)};
  }
  Step s;
  s.lr = c.lr; s.beta1 = c.beta1; s.beta2 = c.beta2; s.weight_decay = c.weight_decay; s.l1 = c.l1; s.grad_scale = c.grad_scale;
  s.step = c.step;
  s.lr_dev = c.lr_dev; s.grad_scale_dev = c.grad_scale_dev;
  s.step_dev = reinterpret_cast<const long long*>(c.step_dev); s.skip_dev = c.skip_dev;
  s.c.b1 = (float)c.beta1; s.c.ob1 = (float)(1.0 - c.beta1); s.c.b2 = (float)c.beta2; s.c.ob2 = (float)(1.0 - c.beta2);
  s.c.eps = (float)c.eps; s.c.grad_scale = (float)c.grad_scale;
  form_scalars(s, s.lr, s.step < 1 ? 1 : s.step, &s.c);
  const cudaStream_t stream = static_cast<cudaStream_t>(c.stream);
  int rc;
  if (c.param_type == STRADS_F32) rc = by_bits<float, float, false>(c.state_bits, list, live, s, stream);
  else if (c.param_type == STRADS_BF16) rc = by_grad<__nv_bfloat16>(c.grad_type, masters, c.state_bits, list, live, s, stream);
  else rc = by_grad<__half>(c.grad_type, masters, c.state_bits, list, live, s, stream);
  delete[] list;
  return rc;
}

int strads_adamw_unpack(const strads_adamw_tensor_t* tensors, float* const* m_out, float* const* v_out, int32_t count, void* stream) {
  if (count < 0 || (count > 0 && (tensors == nullptr || m_out == nullptr || v_out == nullptr))) return STRADS_ERR_INVALID_ARG;
  Entry* list = new (std::nothrow) Entry[count > 0 ? count : 1];
  if (list == nullptr) return STRADS_ERR_INVALID_ARG;
  int k = 0;
  for (int i = 0; i < count; ++i) {
    const strads_adamw_tensor_t& t = tensors[i];
    int bad = t.n < 0 ? STRADS_ERR_INVALID_ARG : (t.n > kMaxElements ? STRADS_ERR_UNSUPPORTED : STRADS_OK);
    if (bad == STRADS_OK && t.n > 0 &&
        (t.m == nullptr || t.v == nullptr || t.m_scale == nullptr || t.v_scale == nullptr || m_out[i] == nullptr || v_out[i] == nullptr ||
         !aligned(t.m_scale, 4) || !aligned(t.v_scale, 4) || !aligned(m_out[i], 4) || !aligned(v_out[i], 4)))
      bad = STRADS_ERR_INVALID_ARG;
    if (bad != STRADS_OK) { delete[] list; return bad; }
    if (t.n == 0) continue;
    const bool vec = aligned(t.m, 4) && aligned(t.v, 4) && aligned(m_out[i], 16) && aligned(v_out[i], 16);
    list[k++] = Entry{m_out[i], v_out[i], nullptr, t.m, t.v, t.m_scale, t.v_scale, 2 * (long long)t.n + (vec ? 1 : 0)};
  }
  const int rc = each_launch(list, k, [&](const auto& table, unsigned ctas) {
    constexpr int kCap = sizeof(table.e) / sizeof(Entry);
    k_adamw_unpack<kCap><<<ctas, kThreads, 0, static_cast<cudaStream_t>(stream)>>>(table);
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? STRADS_OK : cuda_failed(e, "adamw unpack");
  });
  delete[] list;
  return rc;
}

}  // extern "C"
