// Linear layers: the tensor-core products' interface.
#pragma once
#include <cuda.h>

#include "linear.cuh"

namespace strads {

// A 16-bit matrix as TMA reads it: `outer` runs of `inner` elements, `ld` apart (a multiple of 8; p on 16 bytes), the same again
// for every plane.  rows_inner: the rows of the operand run through memory, else its k does.
struct Planes { const void* p; long long inner, outer, ld, plane; int planes, rows_inner; };

struct TcArgs {
  int na, nb, blocks;                    // rows of A and B; blocks of 64 along k
  int tiles_a, tiles_b, splits;
  int a_rows_inner, b_rows_inner, bf16, stall;
  int out_tma, residual_tma, preact_tma;   // which of D, the residual and z go through shared memory by TMA
  unsigned int* status;
  Finish f;
};

// D = A B^T of 16-bit matrices, or (type STRADS_F32) of binary32 ones as three planes of bfloat16; nk >= 1.
cudaError_t launch_linear_tc(int type, const Planes& A, const Planes& B, long long na, long long nb, long long nk, const Finish& f,
                             unsigned int* status, bool stall, cudaStream_t s);

using EncodeFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                              const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeFn tensor_map_encoder();           // null: the driver has none
bool encode_operand(CUtensorMap* map, const Planes& m, bool bf16, int box_rows);

// ---- binary32 products with up to kSplitMost rows on one side (linear_split.cu) ----
// The long side L is read where it is, if linear_split_takes it, and split into planes on its way; the short one comes as planes, k along memory.
constexpr int kSplitMost = 128;
bool linear_split_takes(const Operand& L, long long nl, long long nk);
size_t linear_split_workspace(long long nl, long long ns, long long nk);      // (the same on every device)
cudaError_t launch_linear_split(const Operand& L, const Planes& S, long long nl, long long ns, long long nk, bool long_is_b, const Finish& f,
                                void* workspace, unsigned int* status, bool stall, cudaStream_t s);

// x = p0 + p1 + p2 (24 bits), two neighbours at a time: p0 cut off (so that it cannot overflow), p1 rounded to nearest, p2 what is left.
// What is not finite becomes NaN in p1 and p2.
__device__ __forceinline__ void split_pair(float x, float y, uint32_t (&p)[3]) {
  const uint32_t xb = __float_as_uint(x), yb = __float_as_uint(y);
  p[0] = __byte_perm(xb, yb, 0x7632);
  const float x1 = x - __uint_as_float(xb & 0xffff0000u), y1 = y - __uint_as_float(yb & 0xffff0000u);
  const __nv_bfloat162 m = __floats2bfloat162_rn(x1, y1);
  p[1] = *reinterpret_cast<const uint32_t*>(&m);
  const __nv_bfloat162 l = __floats2bfloat162_rn(x1 - __uint_as_float(p[1] << 16), y1 - __uint_as_float(p[1] & 0xffff0000u));
  p[2] = *reinterpret_cast<const uint32_t*>(&l);
}

}  // namespace strads
