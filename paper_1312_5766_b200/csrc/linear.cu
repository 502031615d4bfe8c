// Linear layers: out = residual + scale act(x w^T + bias) and its gradient.  Argument checks, workspace, and which kernel
// forms which product.
#include <cmath>

#include "linear.cuh"

namespace strads {
namespace {

__device__ unsigned int g_linear_status;       // STRADS_STATUS_* bits of the layers' bounded waits

// ---- products, one 64 x 64 tile of D per CTA, any strides ----
constexpr int kTile = 64, kDepth = 16;
template <typename TA, typename TB, typename T>
__global__ void __launch_bounds__(256) k_linear_simple(Operand A, Operand B, long long na, long long nb, long long nk, Finish f) {
  __shared__ float sa[kDepth][kTile + 1], sb[kDepth][kTile + 1];
  const int t = threadIdx.x, ta = t % 16, tb = t / 16;
  const long long a0 = (long long)blockIdx.x * kTile, b0 = (long long)blockIdx.y * kTile;
  float acc[4][4] = {};
  for (long long k0 = 0; k0 < nk; k0 += kDepth) {
    for (int i = t; i < kTile * kDepth; i += 256) {
      const int ra = A.ks == 1 ? i / kDepth : i % kTile, ka = A.ks == 1 ? i % kDepth : i / kTile;
      const int rb = B.ks == 1 ? i / kDepth : i % kTile, kb = B.ks == 1 ? i % kDepth : i / kTile;
      sa[ka][ra] = a0 + ra < na && k0 + ka < nk ? load_f32(static_cast<const TA*>(A.p) + (a0 + ra) * A.rs + (k0 + ka) * A.ks) : 0.f;
      sb[kb][rb] = b0 + rb < nb && k0 + kb < nk ? load_f32(static_cast<const TB*>(B.p) + (b0 + rb) * B.rs + (k0 + kb) * B.ks) : 0.f;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kDepth; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(sa[k][ta + 16 * i], sb[k][tb + 16 * j], acc[i][j]);
    __syncthreads();
  }
  for (int i = 0; i < 4; ++i)
    for (int j = 0; j < 4; ++j) {
      const long long a = a0 + ta + 16 * i, b = b0 + tb + 16 * j;
      if (a < na && b < nb) finish<T>(f, acc[i][j], a, b);
    }
}

// gz[n][m] = scale gout act'(preact), binary32.
template <typename T>
__global__ void k_linear_slope(Operand gout, Operand preact, long long n, long long m, int act, float scale, float* gz) {
  for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < n * m; i += (long long)gridDim.x * blockDim.x) {
    const long long r = i / m, c = i % m;
    float g = scale * load_f32(static_cast<const T*>(gout.p) + r * gout.rs + c * gout.ks);
    if (act != STRADS_ACT_IDENTITY) g *= slope(load_f32(static_cast<const T*>(preact.p) + r * preact.rs + c * preact.ks), act);
    gz[i] = g;
  }
}
template <typename T>
__global__ void k_linear_bias_grad(const float* gz, long long n, long long m, T* gbias) {
  const long long c = (long long)blockIdx.x * blockDim.x + threadIdx.x;
  if (c >= m) return;
  float s = 0.f;
  for (long long r = 0; r < n; ++r) s += gz[r * m + c];
  store_f32(gbias + c, s);
}

template <typename TA, typename TB, typename T>
cudaError_t product(const Operand& A, const Operand& B, long long na, long long nb, long long nk, const Finish& f, cudaStream_t s) {
  const dim3 grid((unsigned)((na + kTile - 1) / kTile), (unsigned)((nb + kTile - 1) / kTile));
  k_linear_simple<TA, TB, T><<<grid, 256, 0, s>>>(A, B, na, nb, nk, f);
  return cudaGetLastError();
}

bool valid_strides(long long rs, long long cs) { return rs >= 0 && cs >= 0; }
bool valid_in(const strads_const_matrix_t& m, int size) {
  return m.data != nullptr && ((uintptr_t)m.data % size) == 0 && valid_strides(m.row_stride, m.col_stride);
}
// What is written: no two elements at one place.  (Two strides with extents: the inner run must end before the outer step.)
bool valid_out(const strads_matrix_t& m, int size, long long rows, long long cols) {
  if (m.data == nullptr || ((uintptr_t)m.data % size) != 0 || !valid_strides(m.row_stride, m.col_stride)) return false;
  long long s1 = m.row_stride, n1 = rows, s2 = m.col_stride, n2 = cols;
  if (n1 <= 1) { s1 = 0; n1 = 1; }
  if (n2 <= 1) { s2 = 0; n2 = 1; }
  if ((n1 > 1 && s1 == 0) || (n2 > 1 && s2 == 0)) return false;
  if (n1 == 1 || n2 == 1) return true;
  return s1 <= s2 ? s2 / s1 >= n1 : s1 / s2 >= n2;
}

int check(const strads_linear_config_t& c) {
  if (c.type < STRADS_F32 || c.type > STRADS_F16 || c.activation < STRADS_ACT_IDENTITY || c.activation > STRADS_ACT_SILU) return STRADS_ERR_INVALID_ARG;
  if (c.n_rows < 0 || c.n_in < 1 || c.n_out < 1 || !std::isfinite(c.scale) || (c.flags & ~STRADS_LINEAR_FLAG_STALL) != 0) return STRADS_ERR_INVALID_ARG;
  if (c.n_rows > 0x7fffffffll || c.n_in > 0x7fffffffll || c.n_out > 0x7fffffffll) return STRADS_ERR_UNSUPPORTED;
  const int size = c.type == STRADS_F32 ? 4 : 2;
  if (!valid_in(c.w, size) || (c.n_rows > 0 && !valid_in(c.x, size))) return STRADS_ERR_INVALID_ARG;
  return STRADS_OK;
}

template <typename T>
cudaError_t forward(const strads_linear_config_t& c, const void* bias, const strads_const_matrix_t* residual, const strads_matrix_t& out,
                    const strads_matrix_t* preact, cudaStream_t s) {
  Finish f = {};
  f.act = c.activation; f.scale = c.scale;
  f.plain = 0;
  f.bias = bias;
  f.bias_a = 1;
  f.out = {out.data, out.col_stride, out.row_stride};
  if (residual) f.residual = {residual->data, residual->col_stride, residual->row_stride};
  if (preact) f.preact = {preact->data, preact->col_stride, preact->row_stride};
  return product<T, T, T>({c.w.data, c.w.row_stride, c.w.col_stride}, {c.x.data, c.x.row_stride, c.x.col_stride}, c.n_out, c.n_rows, c.n_in, f, s);
}

template <typename T>
cudaError_t backward(const strads_linear_config_t& c, const strads_const_matrix_t& gout, const strads_const_matrix_t* preact, const strads_matrix_t* gx,
                     const strads_matrix_t* gw, void* gbias, cudaStream_t s) {
  float* gz = static_cast<float*>(c.workspace);
  const Operand z = preact ? Operand{preact->data, preact->row_stride, preact->col_stride} : Operand{};
  cudaError_t e = cudaSuccess;
  if (c.n_rows > 0) {
    k_linear_slope<T><<<1184, 256, 0, s>>>({gout.data, gout.row_stride, gout.col_stride}, z, c.n_rows, c.n_out, c.activation, c.scale, gz);
    if ((e = cudaGetLastError()) != cudaSuccess) return e;
  }
  Finish f = {};
  f.plain = 1;
  if (gx != nullptr && c.n_rows > 0) {
    f.out = {gx->data, gx->col_stride, gx->row_stride};
    if ((e = product<T, float, T>({c.w.data, c.w.col_stride, c.w.row_stride}, {gz, c.n_out, 1}, c.n_in, c.n_rows, c.n_out, f, s)) != cudaSuccess) return e;
  }
  if (gw != nullptr) {
    f.out = {gw->data, gw->col_stride, gw->row_stride};
    if ((e = product<T, float, T>({c.x.data, c.x.col_stride, c.x.row_stride}, {gz, 1, c.n_out}, c.n_in, c.n_out, c.n_rows, f, s)) != cudaSuccess) return e;
  }
  if (gbias != nullptr) {
    k_linear_bias_grad<T><<<(unsigned)((c.n_out + 255) / 256), 256, 0, s>>>(gz, c.n_rows, c.n_out, static_cast<T*>(gbias));
    e = cudaGetLastError();
  }
  return e;
}

}  // namespace
}  // namespace strads

using namespace strads;

extern "C" {

int strads_linear_workspace_bytes(const strads_linear_config_t* cfg, size_t* forward_out, size_t* backward_out) {
  if (cfg == nullptr || forward_out == nullptr || backward_out == nullptr) return STRADS_ERR_INVALID_ARG;
  const int rc = check(*cfg);
  if (rc != STRADS_OK) return rc;
  *forward_out = 0;
  *backward_out = (size_t)cfg->n_rows * (size_t)cfg->n_out * sizeof(float);
  return STRADS_OK;
}

static int check_workspace(const strads_linear_config_t& c, int which) {
  size_t need[2];
  const int rc = strads_linear_workspace_bytes(&c, &need[0], &need[1]);
  if (rc != STRADS_OK) return rc;
  if (need[which] == 0) return STRADS_OK;
  if (c.workspace == nullptr || ((uintptr_t)c.workspace & 255) != 0) return STRADS_ERR_INVALID_ARG;
  return c.workspace_bytes < need[which] ? STRADS_ERR_WORKSPACE_TOO_SMALL : STRADS_OK;
}

int strads_linear_forward(const strads_linear_config_t* cfg, const void* bias, const strads_const_matrix_t* residual,
                          const strads_matrix_t* out, const strads_matrix_t* preact) {
  if (cfg == nullptr) return STRADS_ERR_INVALID_ARG;
  int rc = check_workspace(*cfg, 0);
  if (rc != STRADS_OK) return rc;
  const strads_linear_config_t& c = *cfg;
  if (c.n_rows == 0) return STRADS_OK;
  const int size = c.type == STRADS_F32 ? 4 : 2;
  if (out == nullptr || !valid_out(*out, size, c.n_rows, c.n_out) || (preact != nullptr && !valid_out(*preact, size, c.n_rows, c.n_out)) ||
      (residual != nullptr && !valid_in(*residual, size)) || ((uintptr_t)bias % size) != 0)
    return STRADS_ERR_INVALID_ARG;
  const cudaStream_t s = static_cast<cudaStream_t>(c.stream);
  const cudaError_t e = c.type == STRADS_F32 ? forward<float>(c, bias, residual, *out, preact, s)
                      : c.type == STRADS_BF16 ? forward<__nv_bfloat16>(c, bias, residual, *out, preact, s)
                                              : forward<__half>(c, bias, residual, *out, preact, s);
  return e == cudaSuccess ? STRADS_OK : cuda_failed(e, "strads_linear_forward");
}

int strads_linear_backward(const strads_linear_config_t* cfg, const strads_const_matrix_t* gout, const strads_const_matrix_t* preact,
                           const strads_matrix_t* gx, const strads_matrix_t* gw, void* gbias) {
  if (cfg == nullptr) return STRADS_ERR_INVALID_ARG;
  int rc = check_workspace(*cfg, 1);
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
  const cudaStream_t s = static_cast<cudaStream_t>(c.stream);
  const cudaError_t e = c.type == STRADS_F32 ? backward<float>(c, g, preact, gx, gw, gbias, s)
                      : c.type == STRADS_BF16 ? backward<__nv_bfloat16>(c, g, preact, gx, gw, gbias, s)
                                              : backward<__half>(c, g, preact, gx, gw, gbias, s);
  return e == cudaSuccess ? STRADS_OK : cuda_failed(e, "strads_linear_backward");
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
