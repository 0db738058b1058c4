// Linear layers in 8-bit integers: rows quantised with one scale each
// (pf16_quantize_i8) and the product of two such matrices (pf16_linear_i8).
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include "pf16_int8.h"
#include "pf16_internal.h"
#include "pf16_ptx.cuh"

namespace pf16 {

namespace {

__device__ __forceinline__ float h2f(uint16_t h) { return __half2float(__ushort_as_half(h)); }
__device__ __forceinline__ uint16_t f2h(float f) { return __half_as_ushort(__float2half_rn(f)); }
__device__ __forceinline__ uint32_t f2h2(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// ---------------------------------------------------------------------------
// q = rint(127 x / a), a = max |x| of the row, ties to even.
//
// 127 x is exact in FP32 (18 bits).  Two binary16 numbers' quotient 127 x / a
// is either exactly half an integer or at least 2^-19 of its own size away from
// one, so the FP32 quotient decides the rounding as the real one does, provided
// it is exact where that is a tie: r = 1 / a gives p r to within an ulp or two, and one
// Newton correction with the residual p - q a, which an FMA computes exactly, removes that.
// ---------------------------------------------------------------------------
struct RowScale {
  float a, r;
};
__device__ __forceinline__ RowScale row_scale(float a) {
  const bool ok = a > 0.f && a <= 65504.f;
  return RowScale{a, ok ? 1.f / a : 0.f};
}
__device__ __forceinline__ uint32_t quant1(uint16_t h, const RowScale& s) {
  const float p = 127.f * h2f(h);
  float q = p * s.r;
  q = fmaf(fmaf(-q, s.a, p), s.r, q);
  return __float_as_uint(q + 12582912.f);  // 1.5 * 2^23: the integer in the low bits
}
__device__ __forceinline__ uint32_t abs_max2(uint32_t m, uint32_t v) {
  const __half2 r = __hmax2_nan(*reinterpret_cast<const __half2*>(&m), __habs2(*reinterpret_cast<const __half2*>(&v)));
  return *reinterpret_cast<const uint32_t*>(&r);
}
// the row's scale: NaN (and zeros for the integers) where the row holds an infinity or a NaN
__device__ __forceinline__ float stored_scale(float a) {
  return a <= 65504.f ? a / 127.f : __int_as_float(0x7fffffff);
}

}  // namespace

// One row by each group of G threads (G <= 32: part of a warp; 256: the CTA).
// VEC: rows of whole 16-byte vectors, of which a thread keeps its first KEEP in registers between the
// maximum and the rounding and reads the others twice.
template <int G, int KEEP, bool VEC>
__global__ void __launch_bounds__(256) k_quantize_i8(const uint16_t* __restrict__ x, int8_t* __restrict__ q,
                                                     float* __restrict__ scale, long long m, int k) {
  pdl_wait();
  constexpr int ROWS = 256 / G;
  const int g = (int)threadIdx.x % G;
  const long long row = (long long)blockIdx.x * ROWS + threadIdx.x / G;
  const bool live = row < m;
  const uint16_t* xr = x + (live ? row : 0) * k;
  uint4 keep[KEEP > 0 ? KEEP : 1];
  uint32_t mx = 0;
  if (VEC) {
    const int nv = live ? k >> 3 : 0;
    const uint4* xv = reinterpret_cast<const uint4*>(xr);
#pragma unroll
    for (int i = 0; i < KEEP; ++i)
      keep[i] = g + i * G < nv ? __ldcs(xv + g + i * G) : make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int i = 0; i < KEEP; ++i)
      mx = abs_max2(abs_max2(abs_max2(abs_max2(mx, keep[i].x), keep[i].y), keep[i].z), keep[i].w);
    for (int c = g + KEEP * G; c < nv; c += G) {
      const uint4 v = xv[c];
      mx = abs_max2(abs_max2(abs_max2(abs_max2(mx, v.x), v.y), v.z), v.w);
    }
  } else {
    for (int c = g; c < (live ? k : 0); c += G) mx = abs_max2(mx, (uint32_t)xr[c]);
  }
  constexpr int W = G < 32 ? G : 32;
#pragma unroll
  for (int o = W / 2; o > 0; o >>= 1) mx = abs_max2(mx, __shfl_xor_sync(0xffffffffu, mx, o));
  mx = abs_max2(mx, mx >> 16);
  if (G > 32) {
    __shared__ uint32_t red[8];
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = mx;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 8; ++i) mx = abs_max2(mx, red[i]);
  }
  if (!live) return;
  const float a = h2f((uint16_t)mx);
  const RowScale s = row_scale(a);
  if (g == 0) scale[row] = stored_scale(a);
  int8_t* qr = q + row * k;
  // with r = 0 (a zero row, or one that is not finite) the integers are zero
  if (VEC) {
    const int nv = k >> 3;
    const uint4* xv = reinterpret_cast<const uint4*>(xr);
    auto put = [&](int c, const uint4& v) {
      const uint32_t* h = reinterpret_cast<const uint32_t*>(&v);
      uint2 o = make_uint2(0, 0);
      if (s.r != 0.f) {
        uint32_t b[8];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          b[2 * j] = quant1((uint16_t)h[j], s);
          b[2 * j + 1] = quant1((uint16_t)(h[j] >> 16), s);
        }
        o.x = prmt(prmt(b[0], b[1], 0x0040), prmt(b[2], b[3], 0x0040), 0x5410);
        o.y = prmt(prmt(b[4], b[5], 0x0040), prmt(b[6], b[7], 0x0040), 0x5410);
      }
      __stcs(reinterpret_cast<uint2*>(qr) + c, o);
    };
#pragma unroll
    for (int i = 0; i < KEEP; ++i)
      if (g + i * G < nv) put(g + i * G, keep[i]);
    for (int c = g + KEEP * G; c < nv; c += G) put(c, xv[c]);
  } else {
    for (int c = g; c < k; c += G) qr[c] = s.r != 0.f ? (int8_t)quant1(xr[c], s) : (int8_t)0;
  }
}

template <int G, int KEEP>
static cudaError_t quantize_g(const uint16_t* x, int8_t* q, float* scale, long long m, int k, cudaStream_t s) {
  const long long blocks = (m + 256 / G - 1) / (256 / G);
  const dim3 grid((unsigned)blocks), block(256);
  const cudaError_t e = (k & 7) == 0 ? launch_pdl(k_quantize_i8<G, KEEP, true>, grid, block, 0, s, x, q, scale, m, k)
                                     : launch_pdl(k_quantize_i8<G, 0, false>, grid, block, 0, s, x, q, scale, m, k);
  return e == cudaSuccess ? counted_launches(1) : e;
}

cudaError_t launch_quantize_i8(const uint16_t* x, int8_t* q, float* scale, long long m, int k, cudaStream_t s) {
  if (k <= 64) return quantize_g<8, 1>(x, q, scale, m, k, s);
  if (k <= 128) return quantize_g<16, 1>(x, q, scale, m, k, s);
  if (k <= 1024) return quantize_g<32, 4>(x, q, scale, m, k, s);
  return quantize_g<256, 4>(x, q, scale, m, k, s);
}

// ---------------------------------------------------------------------------
// The product for a few rows of x: each warp takes one output channel, its
// lanes 16 bytes of the weight row at a time, and multiplies them with the MT
// rows of x by dp4a (exact 32-bit sums).  Bound by the weight's bytes, read once.
// ---------------------------------------------------------------------------
namespace {

// 16 bytes of a row of k bytes from byte c on, zero past its end; ALIGNED: rows start at multiples
// of 16 and hold whole vectors.
template <bool ALIGNED>
__device__ __forceinline__ uint4 load16(const int8_t* row, int c, int k) {
  if (ALIGNED) return c < k ? __ldg(reinterpret_cast<const uint4*>(row + c)) : make_uint4(0, 0, 0, 0);
  uint32_t v[4] = {0, 0, 0, 0};
#pragma unroll
  for (int j = 0; j < 16; ++j)
    if (c + j < k) v[j >> 2] |= (uint32_t)(uint8_t)row[c + j] << ((j & 3) * 8);
  return make_uint4(v[0], v[1], v[2], v[3]);
}

}  // namespace

template <int MT, bool ALIGNED>
__global__ void __launch_bounds__(256) k_linear_i8_rows(const LinearI8 a) {
  pdl_wait();
  const int lane = (int)threadIdx.x & 31;
  const int j = (int)blockIdx.x * 8 + ((int)threadIdx.x >> 5);
  const int m0 = (int)blockIdx.y * MT;
  if (j >= a.n) return;
  const int8_t* w = a.w + (long long)j * a.k;
  int acc[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) acc[i] = 0;
#pragma unroll 2
  for (int c = lane * 16; c < a.k; c += 512) {
    const uint4 wv = load16<ALIGNED>(w, c, a.k);
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      if (m0 + i < a.m) {
        const uint4 xv = load16<ALIGNED>(a.x + (long long)(m0 + i) * a.k, c, a.k);
        acc[i] = __dp4a((int)wv.x, (int)xv.x, acc[i]);
        acc[i] = __dp4a((int)wv.y, (int)xv.y, acc[i]);
        acc[i] = __dp4a((int)wv.z, (int)xv.z, acc[i]);
        acc[i] = __dp4a((int)wv.w, (int)xv.w, acc[i]);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int s = __reduce_add_sync(0xffffffffu, acc[i]);
    if (lane == 0 && m0 + i < a.m)
      a.y[(long long)(m0 + i) * a.n + j] =
          f2h(fmaf((float)s, a.sx[m0 + i] * a.sw[j], a.bias ? h2f(a.bias[j]) : 0.f));
  }
}

cudaError_t launch_linear_i8(const LinearI8& a, int sms, int* status, cudaStream_t s) {
  (void)sms;
  (void)status;
  const bool al = (a.k & 15) == 0;
  const dim3 grid((unsigned)((a.n + 7) / 8), (unsigned)((a.m + 7) / 8));
  const cudaError_t e = al ? launch_pdl(k_linear_i8_rows<8, true>, grid, dim3(256), 0, s, a)
                           : launch_pdl(k_linear_i8_rows<8, false>, grid, dim3(256), 0, s, a);
  return e == cudaSuccess ? counted_launches(1) : e;
}

}  // namespace pf16
