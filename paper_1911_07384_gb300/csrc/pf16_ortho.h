// Orthogonalised updates (pf16_ortho.cu): what the C-ABI layer hands to the kernels.
#pragma once
#include <cstdint>
#include <cuda_runtime.h>

namespace pf16 {

constexpr int kOrthoMax = 256;       // matrices in one call (PF16_ORTHO_MAX_MATRICES)
constexpr int kOrthoMaxParts = 512;  // partial sums of squares of one matrix
constexpr int kOrthoBlk = 8192;      // bytes of a 64 x 64 binary16 block

// One matrix.  Inside, it is m x n with m <= n (transposed when `tall`), kept as
// a grid of mb x nb blocks of 64 x 64 elements, zero past its edges.
struct OrthoMat {
  const uint16_t* g;
  uint16_t* v;        // momentum (null: plain orthogonalisation)
  uint16_t* w;        // weights updated in place, or the output
  uint8_t* ws;        // x16[2], x32, a16, b16 (ortho_layout)
  int rows, cols;     // as the caller sees it
  int mb, nb;
  int part0, parts;   // its partial sums of squares
  int tall;
  float scale;        // of the orthogonalised update in the weights' step
};

struct OrthoParams {
  int count, steps;
  int max_items;      // most work items of one phase, over all matrices together
  int muon, nesterov;
  float lr, momentum, wd;
  uint32_t* ticket;   // work items handed out
  uint32_t* done;     // [count] items finished of each matrix
  float* parts;       // partial sums of squares
  int total_parts;
  int* status;
  unsigned long long wait_limit_ns;
  // first item of each matrix within each kind of phase (pack, symmetric
  // product, full product); entry `count` is the kind's total
  int pre_pack[kOrthoMax + 1], pre_sym[kOrthoMax + 1], pre_full[kOrthoMax + 1];
  OrthoMat mat[kOrthoMax];
};

struct OrthoLayout {
  size_t x16, x32, a16, b16, bytes;
};
__host__ __device__ inline OrthoLayout ortho_layout(long long mb, long long nb) {
  OrthoLayout l;
  const size_t xb = (size_t)mb * nb * kOrthoBlk, ab = (size_t)mb * mb * kOrthoBlk;
  l.x16 = 0;            // two buffers of xb bytes
  l.x32 = 2 * xb;
  l.a16 = 4 * xb;
  l.b16 = 4 * xb + ab;
  l.bytes = 4 * xb + 2 * ab;
  return l;
}

cudaError_t launch_ortho(const OrthoParams& p, int sms, cudaStream_t s);

}  // namespace pf16
