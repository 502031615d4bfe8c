// Linear layers: the tensor-core products' interface.
#pragma once
#include "linear.cuh"

namespace strads {

// A 16-bit matrix as TMA reads it: `outer` runs of `inner` elements, `ld` apart (a multiple of 8; p on 16 bytes), the same again
// for every plane.  rows_inner: the rows of the operand run through memory, else its k does.
struct Planes { const void* p; long long inner, outer, ld, plane; int planes, rows_inner; };

struct TcArgs {
  int na, nb, blocks;                    // rows of A and B; blocks of 64 along k
  int tiles_a, tiles_b, splits;
  int a_rows_inner, b_rows_inner, bf16, stall;
  unsigned int* status;
  Finish f;
};

// D = A B^T of 16-bit matrices, or (type STRADS_F32) of binary32 ones as three planes of bfloat16; nk >= 1.
cudaError_t launch_linear_tc(int type, const Planes& A, const Planes& B, long long na, long long nb, long long nk, const Finish& f,
                             unsigned int* status, bool stall, cudaStream_t s);

}  // namespace strads
