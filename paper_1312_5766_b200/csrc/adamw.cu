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
constexpr long long kChunk = 2048;             // elements a CTA takes: a block for each of its warps
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
// Elements that are not there read as 0.
template <typename T, typename U>
__device__ __forceinline__ void load8(const T* p, int n, bool vec, int lane, U (&x)[8]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int i = h * 128 + lane * 4;
    if (vec && i + 4 <= n) {
      const Four<T> f = *reinterpret_cast<const Four<T>*>(p + i);
#pragma unroll
      for (int j = 0; j < 4; ++j) x[4 * h + j] = (U)f.x[j];
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) x[4 * h + j] = i + j < n ? (U)p[i + j] : (U)0.f;
    }
  }
}
template <typename T>
__device__ __forceinline__ void store8(T* p, int n, bool vec, int lane, const T (&x)[8]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int i = h * 128 + lane * 4;
    if (vec && i + 4 <= n) {
      Four<T> f;
#pragma unroll
      for (int j = 0; j < 4; ++j) f.x[j] = x[4 * h + j];
      *reinterpret_cast<Four<T>*>(p + i) = f;
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) if (i + j < n) p[i + j] = x[4 * h + j];
    }
  }
}

__device__ __forceinline__ bool finite(float mag) { return mag <= 3.402823466e38f; }      // (of a magnitude; false for NaN)
__device__ __forceinline__ float warp_max(float mag) {                                      // magnitudes order like their bits
  return __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(mag)));
}
// Between codes and floats by the sum with 2^23 or 1.5 2^23, whose last bits then are the integer: the conversion instructions go through the
// unit that the roots and quotients need, at a quarter of the rate.
constexpr float kUnsigned = 8388608.f, kRounded = 12582912.f;
__device__ __forceinline__ float decode_m(unsigned int byte, float s) {      // byte: the code as stored, -128 .. 127
  const float q = __fsub_rn(__uint_as_float(0x4b000000u | (byte ^ 0x80u)), kUnsigned + 128.f);
  return byte == 0x80u ? __uint_as_float(0x7fc00000u) : __fmul_rn(__fmul_rn(q, fabsf(q)), s);
}
__device__ __forceinline__ float decode_root(unsigned int byte, float s) {
  const float q = __fsub_rn(__uint_as_float(0x4b000000u | byte), kUnsigned);
  return byte == 255u ? __uint_as_float(0x7fc00000u) : __fmul_rn(__fmul_rn(q, q), s);
}
// The integer nearest to the correctly rounded root of x (ties to even), x <= 2^16, in the last bits.  The approximate root is good to 2^-14
// there; only where it lies within 2^-12 of the middle between two integers is the exact one needed.
__device__ __forceinline__ unsigned int nearest_root(float x) {
  float r;
  asm("sqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(x));
  float t = __fadd_rn(r, kRounded);
  if (fabsf(fabsf(r - (t - kRounded)) - 0.5f) < 0.000244140625f) t = __fadd_rn(__fsqrt_rn(x), kRounded);
  return __float_as_uint(t);
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

template <typename P, typename G, bool kMaster, int kBits, int kCap>
__global__ void __launch_bounds__(kThreads) k_adamw(const __grid_constant__ Table<kCap> t, const __grid_constant__ Step s) {
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
  const bool vec = e.n_vec & 1;
  const long long n_all = e.n_vec >> 1, at = (long long)((int)blockIdx.x - t.first[ti]) * kChunk + warp * kBlock;
  if (at >= n_all) return;
  const int n = (int)min((long long)kBlock, n_all - at);
  P* param = static_cast<P*>(e.param) + at;
  float p[8], g[8], m[8], v[8];
  if (kMaster) load8(e.master + at, n, vec, lane, p); else load8(param, n, vec, lane, p);
  load8(static_cast<const G*>(e.grad) + at, n, vec, lane, g);
  if (kBits == 32) {
    load8(static_cast<const float*>(e.m) + at, n, vec, lane, m);
    load8(static_cast<const float*>(e.v) + at, n, vec, lane, v);
  } else {
    unsigned int q[8];
    const float s1 = e.m_scale[at / kBlock], s2 = e.v_scale[at / kBlock];
    load8(static_cast<const unsigned char*>(e.m) + at, n, vec, lane, q);
#pragma unroll
    for (int j = 0; j < 8; ++j) m[j] = decode_m(q[j], s1);
    load8(static_cast<const unsigned char*>(e.v) + at, n, vec, lane, q);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float root = decode_root(q[j], s2);
      v[j] = __fmul_rn(root, root);
    }
  }
  float root[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float gj = __fmul_rn(g[j], c.grad_scale);
    m[j] = __fadd_rn(__fmul_rn(m[j], c.b1), __fmul_rn(gj, c.ob1));
    v[j] = __fadd_rn(__fmul_rn(v[j], c.b2), __fmul_rn(__fmul_rn(gj, gj), c.ob2));
    root[j] = __fsqrt_rn(v[j]);
    const float inv = __frcp_rn(__fadd_rn(__fmul_rn(root[j], c.unbias), c.eps));
    p[j] = __fsub_rn(__fmul_rn(p[j], c.keep), __fmul_rn(__fmul_rn(m[j], c.move), inv));
    if (c.threshold > 0.f) {
      const float size = __fsub_rn(fabsf(p[j]), __fmul_rn(c.threshold, inv));
      p[j] = size < 0.f ? 0.f : copysignf(size, p[j]);      // (a NaN stays one)
    }
  }
  P out[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) out[j] = from_f32<P>(p[j]);
  store8(param, n, vec, lane, out);
  if (kMaster) store8(e.master + at, n, vec, lane, p);
  if (kBits == 32) {
    store8(static_cast<float*>(e.m) + at, n, vec, lane, m);
    store8(static_cast<float*>(e.v) + at, n, vec, lane, v);
    return;
  }
  float top1 = 0.f, top2 = 0.f;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float a = fabsf(m[j]);
    if (finite(a)) top1 = fmaxf(top1, a);
    if (finite(root[j])) top2 = fmaxf(top2, root[j]);
  }
  float r1, r2;
  const float s1 = scale_of(warp_max(top1), 1.f / 16129.f, &r1), s2 = scale_of(warp_max(top2), 1.f / 64516.f, &r2);
  unsigned char q1[8], q2[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float a = fabsf(m[j]);
    const unsigned int q = nearest_root(__fmul_rn(a, r1)), w = nearest_root(__fmul_rn(root[j], r2));
    q1[j] = (unsigned char)(finite(a) ? (m[j] < 0.f ? 0u - q : q) : 0x80u);
    q2[j] = (unsigned char)(finite(root[j]) ? (root[j] > 0.f && (w & 0xffu) == 0u ? 1u : w) : 255u);
  }
  store8(static_cast<unsigned char*>(e.m) + at, n, vec, lane, q1);
  store8(static_cast<unsigned char*>(e.v) + at, n, vec, lane, q2);
  if (lane == 0) { e.m_scale[at / kBlock] = s1; e.v_scale[at / kBlock] = s2; }
}

// Moments held in 8 bits as the values that they stand for: entry.param receives m, entry.master v.
template <int kCap>
__global__ void __launch_bounds__(kThreads) k_adamw_unpack(const __grid_constant__ Table<kCap> t) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int ti = find_tensor(t);
  const Entry& e = t.e[ti];
  const bool vec = e.n_vec & 1;
  const long long n_all = e.n_vec >> 1, at = (long long)((int)blockIdx.x - t.first[ti]) * kChunk + warp * kBlock;
  if (at >= n_all) return;
  const int n = (int)min((long long)kBlock, n_all - at);
  const float s1 = e.m_scale[at / kBlock], s2 = e.v_scale[at / kBlock];
  unsigned int q1[8], q2[8];
  load8(static_cast<const unsigned char*>(e.m) + at, n, vec, lane, q1);
  load8(static_cast<const unsigned char*>(e.v) + at, n, vec, lane, q2);
  float m[8], v[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float root = decode_root(q2[j], s2);
    m[j] = decode_m(q1[j], s1);
    v[j] = __fmul_rn(root, root);
  }
  store8(static_cast<float*>(e.param) + at, n, vec, lane, m);
  store8(e.master + at, n, vec, lane, v);
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
      !((float)c.eps > 0.f && c.eps <= 1e30) || !(c.weight_decay >= 0.0 && c.weight_decay <= 1e30) || !(c.l1 >= 0.0 && c.l1 <= 1e30) ||
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
