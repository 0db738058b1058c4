// Orthogonalised updates: Newton-Schulz iterations on a list of matrices, and
// the optimiser step around them (pf16_orthogonalize, pf16_muon_update).
//
// For each matrix U (m <= n inside): X0 = U / |U|_F, then `steps` times
//     A = X X^T,   B = b A + c A A,   X <- a X + B X,
// with the quintic's coefficients (a, b, c), whose map s -> a s + b s^3 + c s^5
// keeps [0, 1.21] in itself and lifts small singular values towards 1.
//
// Precision.  X is held in FP32; the tensor cores multiply binary16 copies and
// accumulate in FP32.  Rounding only the products' operands, and never X
// itself, is what keeps the small singular values: the map multiplies them by
// 3.44 a step, errors among them, and the a X term passes X on unrounded while
// B X is small where they are small.  (A rank-8 matrix with 1% of noise:
// 4e-4 off the exact result in the 2-norm, against 4e-2 with X kept in
// binary16.)  The copies are scaled by powers of two so that no element
// overflows (|X| <= 1.21, |A| <= 1.45, |B| <= 2.81) and small ones stay normal.
//
// Layout.  Every matrix of the iteration is a grid of 64 x 64 binary16 blocks,
// each 8 KB contiguous in the 128-byte-swizzled order that tcgen05.mma reads.
// An operand tile is two blocks, brought in by untiled bulk copies, and the
// same block serves as a K-major operand or, transposed, as an MN-major one:
// X needs no transposed copy, and of the symmetric A and B only the tiles on
// and below the diagonal are computed and stored.  The caller's arrays, of any
// size and alignment of rows, are touched by the first and last phase only.
//
// Schedule.  One persistent kernel runs all phases of all matrices: work items
// (a block to pack, a 128 x 128 tile of a product) are numbered phase by phase
// and handed out by an atomic ticket, and an item starts once the item count of
// its matrix shows the previous phase complete.  An item waits only for items
// with smaller tickets, which running CTAs hold, so the kernel makes progress
// with any number of its CTAs resident.
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include "pf16_internal.h"
#include "pf16_ortho.h"
#include "pf16_ptx.cuh"

namespace pf16 {

namespace {

constexpr float kA = 3.4445f, kB = -4.7750f, kC = 2.0315f;
// powers of two of the binary16 copies
constexpr float kSx = 32768.f, kSa = 32768.f, kSb = 16384.f;

constexpr int kStages = 6;
constexpr int kStageBytes = 4 * kOrthoBlk;  // two blocks of each operand
constexpr int kRing = 4;                    // work items in flight inside a CTA
constexpr int kEpi = 256;                   // epilogue threads: two warps for each quarter of the accumulator's rows
constexpr int kThreads = 64 + kEpi;         // and a warp each for the loads and the MMAs
constexpr int kPackPitch = 65;
constexpr int kOrthoSmem = 1024 + kStages * kStageBytes + kStageBytes + 256;

enum ItemKind : int { kPack = 0, kSym1 = 1, kSym2 = 2, kFull = 3, kStop = 4 };
struct Item {
  int kind, mat, I, J, step;
};

__device__ __forceinline__ void fence_proxy_async_all() { asm volatile("fence.proxy.async;" ::: "memory"); }
__device__ __forceinline__ uint32_t ld_acquire(const uint32_t* p) {
  uint32_t v;
  asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
  return v;
}
__device__ __forceinline__ void red_release_add(uint32_t* p, uint32_t v) {
  asm volatile("red.release.gpu.global.add.u32 [%0], %1;" ::"l"(p), "r"(v) : "memory");
}
__device__ __forceinline__ void bulk_store_1d(void* dst, uint32_t src, uint32_t bytes) {
  asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(
                   reinterpret_cast<uint64_t>(dst)),
               "r"(src), "r"(bytes)
               : "memory");
}
__device__ __forceinline__ void epi_barrier() { asm volatile("bar.sync 1, 256;" ::: "memory"); }

__device__ __forceinline__ float h2f(uint16_t h) { return __half2float(__ushort_as_half(h)); }
__device__ __forceinline__ uint16_t f2h(float f) { return __half_as_ushort(__float2half_rn(f)); }
__device__ __forceinline__ uint32_t f2h2(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ float2 h22f(uint32_t v) {
  return __half22float2(*reinterpret_cast<const __half2*>(&v));
}

// the largest i with pre[i] <= t, pre[0] = 0 and t < pre[n]
__device__ __forceinline__ int find_mat(const int* pre, int n, int t) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (pre[mid] <= t)
      lo = mid;
    else
      hi = mid;
  }
  return lo;
}

__device__ __forceinline__ int sym_tiles(int mt) { return mt * (mt + 1) / 2; }

// Ticket -> work item, and the number of finished items of its matrix that it waits for.
__device__ __forceinline__ Item decode(const OrthoParams& p, uint32_t ticket, uint32_t& need) {
  Item it;
  const int n = p.count;
  const int tp = p.pre_pack[n], ts = p.pre_sym[n], tf = p.pre_full[n];
  need = 0;
  it.step = 0;
  if (ticket < (uint32_t)tp) {
    it.kind = kPack;
    it.mat = find_mat(p.pre_pack, n, (int)ticket);
    const int local = (int)ticket - p.pre_pack[it.mat];
    it.I = local / p.mat[it.mat].nb;
    it.J = local % p.mat[it.mat].nb;
    return it;
  }
  uint32_t t = ticket - (uint32_t)tp;
  const uint32_t per = (uint32_t)(2 * ts + tf);
  it.step = (int)(t / per);
  t -= (uint32_t)it.step * per;
  if (it.step >= p.steps) {
    it.kind = kStop;
    it.mat = it.I = it.J = 0;
    return it;
  }
  if (t < (uint32_t)(2 * ts)) {
    it.kind = t < (uint32_t)ts ? kSym1 : kSym2;
    if (it.kind == kSym2) t -= (uint32_t)ts;
    it.mat = find_mat(p.pre_sym, n, (int)t);
    const int local = (int)t - p.pre_sym[it.mat];
    // row I of the lower triangle holds tiles I(I+1)/2 .. I(I+1)/2 + I
    int I = (int)((sqrtf(8.f * (float)local + 1.f) - 1.f) * 0.5f);
    while (sym_tiles(I) > local) --I;
    while (sym_tiles(I + 1) <= local) ++I;
    it.I = I;
    it.J = local - sym_tiles(I);
  } else {
    t -= (uint32_t)(2 * ts);
    it.kind = kFull;
    it.mat = find_mat(p.pre_full, n, (int)t);
    const int local = (int)t - p.pre_full[it.mat];
    const int mt = (p.mat[it.mat].mb + 1) >> 1;
    it.I = local % mt;  // column by column: neighbours share X's blocks
    it.J = local / mt;
  }
  const OrthoMat& M = p.mat[it.mat];
  const int mt = (M.mb + 1) >> 1, nt = (M.nb + 1) >> 1;
  const uint32_t sym = (uint32_t)sym_tiles(mt);
  need = (uint32_t)(M.mb * M.nb) + (uint32_t)it.step * (2 * sym + (uint32_t)(mt * nt)) +
         (uint32_t)(it.kind - kSym1) * sym;
  return it;
}

}  // namespace

// ---------------------------------------------------------------------------
// Sums of squares (fixed chunks, fixed trees: the same bits every time) and, for
// the optimiser step, the momentum: v <- rn16(momentum * v + g).  Also clears
// the main kernel's counters.
// ---------------------------------------------------------------------------
__device__ __forceinline__ float ortho_u(const OrthoParams& p, float g, float v) {
  return p.nesterov ? fmaf(p.momentum, v, g) : v;
}

__global__ void __launch_bounds__(256) k_ortho_norm(const __grid_constant__ OrthoParams p) {
  pdl_wait();
  const int tid = (int)threadIdx.x;
  if (blockIdx.x == 0) {
    if (tid == 0) *p.ticket = 0;
    for (int i = tid; i < p.count; i += 256) p.done[i] = 0;
  }
  // the matrix whose partial sums hold this block
  int lo = 0, hi = p.count;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (p.mat[mid].part0 <= (int)blockIdx.x)
      lo = mid;
    else
      hi = mid;
  }
  const OrthoMat& M = p.mat[lo];
  const long long n = (long long)M.rows * M.cols, vecs = (n + 7) / 8;
  const long long per = (vecs + M.parts - 1) / M.parts;
  const long long v0 = ((long long)blockIdx.x - M.part0) * per;
  const long long v1 = v0 + per < vecs ? v0 + per : vecs;
  float sum = 0.f;
  for (long long i = v0 + tid; i < v1; i += 256) {
    const bool whole = i * 8 + 8 <= n;
    const int cnt = whole ? 8 : (int)(n - i * 8);
    uint16_t g[8], v[8];
    if (whole) {
      *reinterpret_cast<uint4*>(g) = reinterpret_cast<const uint4*>(M.g)[i];
      if (p.muon) *reinterpret_cast<uint4*>(v) = reinterpret_cast<const uint4*>(M.v)[i];
    } else {
      for (int j = 0; j < 8; ++j) {
        g[j] = j < cnt ? M.g[i * 8 + j] : 0;
        v[j] = p.muon && j < cnt ? M.v[i * 8 + j] : 0;
      }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      float u = h2f(g[j]);
      if (p.muon) {
        v[j] = f2h(fmaf(p.momentum, h2f(v[j]), u));
        u = ortho_u(p, u, h2f(v[j]));
      }
      sum = fmaf(u, u, sum);
    }
    if (p.muon) {
      if (whole)
        reinterpret_cast<uint4*>(M.v)[i] = *reinterpret_cast<uint4*>(v);
      else
        for (int j = 0; j < cnt; ++j) M.v[i * 8 + j] = v[j];
    }
  }
  __shared__ float red[8];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_down_sync(0xffffffffu, sum, o);
  if ((tid & 31) == 0) red[tid >> 5] = sum;
  __syncthreads();
  if (tid == 0) {
    float s = 0.f;
    for (int i = 0; i < 8; ++i) s += red[i];
    p.parts[blockIdx.x] = s;
  }
}

namespace {

// 1 / |U|_F from the matrix's partial sums, the same in all epilogue threads.  A zero
// matrix gives 0 (its result is zero); a norm that is not finite gives NaN, and
// with it a result of NaNs only.
__device__ __forceinline__ float inv_norm(const OrthoParams& p, const OrthoMat& M, float* red, int t) {
  float s = 0.f;
  for (int i = t; i < M.parts; i += kEpi) s += __ldcg(p.parts + M.part0 + i);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_down_sync(0xffffffffu, s, o);
  if ((t & 31) == 0) red[t >> 5] = s;
  epi_barrier();
  s = ((red[0] + red[1]) + (red[2] + red[3])) + ((red[4] + red[5]) + (red[6] + red[7]));
  if (s == 0.f) return 0.f;
  if (!(s <= 3.402823466e38f)) return __int_as_float(0x7fffffff);
  return 1.f / sqrtf(s);
}

// One 64 x 64 block of X0, FP32 and scaled binary16, by the epilogue threads.  The loads are
// in flight while the norm is summed.
__device__ void pack_block(const OrthoParams& p, const OrthoMat& M, int bi, int bj, float* tile, float* red, int t,
                           int& inv_mat, float& inv, int mat) {
  const int r0 = M.tall ? bj * 64 : bi * 64, c0 = M.tall ? bi * 64 : bj * 64;  // in the caller's matrix
  float u[16];
  const bool vec = (M.cols & 7) == 0;
  if (vec) {  // rows of whole vectors: eight elements a load
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int rr = i * 32 + (t >> 3), cc = (t & 7) * 8;
      uint4 g = make_uint4(0, 0, 0, 0), v = g;
      if (r0 + rr < M.rows && c0 + cc < M.cols) {
        const long long at = (long long)(r0 + rr) * M.cols + (c0 + cc);
        g = __ldg(reinterpret_cast<const uint4*>(M.g + at));
        if (p.muon) v = __ldcg(reinterpret_cast<const uint4*>(M.v + at));
      }
      const uint32_t gw[4] = {g.x, g.y, g.z, g.w}, vw[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float2 x = h22f(gw[j]);
        if (p.muon) {
          const float2 y = h22f(vw[j]);
          x.x = ortho_u(p, x.x, y.x);
          x.y = ortho_u(p, x.y, y.y);
        }
        u[i * 8 + 2 * j] = x.x;
        u[i * 8 + 2 * j + 1] = x.y;
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int rr = i * 4 + (t >> 6), cc = t & 63;
      u[i] = 0.f;
      if (r0 + rr < M.rows && c0 + cc < M.cols) {
        const long long at = (long long)(r0 + rr) * M.cols + (c0 + cc);
        u[i] = h2f(__ldg(M.g + at));
        if (p.muon) u[i] = ortho_u(p, u[i], h2f(__ldcg(M.v + at)));
      }
    }
  }
  if (inv_mat != mat) {
    inv = inv_norm(p, M, red, t);
    inv_mat = mat;
  }
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int rr = vec ? (i >> 3) * 32 + (t >> 3) : i * 4 + (t >> 6), cc = vec ? (t & 7) * 8 + (i & 7) : t & 63;
    float x = u[i] * inv;
    if (inv != inv) x = r0 + rr < M.rows && c0 + cc < M.cols ? inv : 0.f;
    tile[M.tall ? cc * kPackPitch + rr : rr * kPackPitch + cc] = x;
  }
  epi_barrier();
  const OrthoLayout L = ortho_layout(M.mb, M.nb);
  const size_t blk = (size_t)bi * M.nb + bj;
  uint8_t* x32 = M.ws + L.x32 + blk * (2 * kOrthoBlk);
  uint8_t* x16 = M.ws + L.x16 + blk * kOrthoBlk;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int row = t & 63, c4 = (t >> 6) + 4 * i;
    const float* s = tile + row * kPackPitch + c4 * 4;
    __stcg(reinterpret_cast<float4*>(x32 + (c4 * 64 + row) * 16), make_float4(s[0], s[1], s[2], s[3]));
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int row = (t >> 3) + 32 * i, ch = t & 7;
    const float* s = tile + row * kPackPitch + ch * 8;
    uint4 v;
    v.x = f2h2(s[0] * kSx, s[1] * kSx);
    v.y = f2h2(s[2] * kSx, s[3] * kSx);
    v.z = f2h2(s[4] * kSx, s[5] * kSx);
    v.w = f2h2(s[6] * kSx, s[7] * kSx);
    __stcg(reinterpret_cast<uint4*>(x16 + row * 128 + ((ch ^ (row & 7)) << 4)), v);
  }
}

__device__ __forceinline__ float muon_w(const OrthoParams& p, const OrthoMat& M, float w, float x) {
  return w - p.lr * fmaf(M.scale, x, p.wd * w);
}

// The final step's 64 columns from c on of inner row r: written to the caller's output, or
// the weights' step taken with them (their loads all issued first).
__device__ __forceinline__ void finish64(const OrthoParams& p, const OrthoMat& M, int r, int c, const float* x) {
  if (M.tall) {  // inner row r is the caller's column: neighbouring lanes write neighbouring elements
    if (r >= M.cols) return;
    uint16_t* o = M.w + (long long)c * M.cols + r;
    const int left = M.rows - c;
#pragma unroll
    for (int h = 0; h < 64; h += 32) {
      float w[32];
      if (p.muon) {
#pragma unroll
        for (int j = 0; j < 32; ++j) w[j] = h + j < left ? h2f(o[(long long)(h + j) * M.cols]) : 0.f;
      }
#pragma unroll
      for (int j = 0; j < 32; ++j)
        if (h + j < left) o[(long long)(h + j) * M.cols] = f2h(p.muon ? muon_w(p, M, w[j], x[h + j]) : x[h + j]);
    }
    return;
  }
  if (r >= M.rows) return;
  uint16_t* o = M.w + (long long)r * M.cols + c;
  const int left = M.cols - c;
  if ((M.cols & 7) == 0) {
    uint4 v[8];
    if (p.muon) {
#pragma unroll
      for (int h = 0; h < 8; ++h)
        v[h] = h * 8 < left ? *reinterpret_cast<const uint4*>(o + 8 * h) : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int h = 0; h < 8; ++h) {
      uint32_t q[4] = {v[h].x, v[h].y, v[h].z, v[h].w};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float2 y = make_float2(x[8 * h + 2 * j], x[8 * h + 2 * j + 1]);
        if (p.muon) {
          const float2 w = h22f(q[j]);
          y.x = muon_w(p, M, w.x, y.x);
          y.y = muon_w(p, M, w.y, y.y);
        }
        q[j] = f2h2(y.x, y.y);
      }
      if (h * 8 < left) *reinterpret_cast<uint4*>(o + 8 * h) = make_uint4(q[0], q[1], q[2], q[3]);
    }
    return;
  }
#pragma unroll
  for (int h = 0; h < 64; h += 32) {
    float w[32];
    if (p.muon) {
#pragma unroll
      for (int j = 0; j < 32; ++j) w[j] = h + j < left ? h2f(o[h + j]) : 0.f;
    }
#pragma unroll
    for (int j = 0; j < 32; ++j)
      if (h + j < left) o[h + j] = f2h(p.muon ? muon_w(p, M, w[j], x[h + j]) : x[h + j]);
  }
}

__device__ __forceinline__ void record_timeout(int* status, volatile int* abort_flag) {
  atomicCAS(status, 0, -7);  // PF16_ERR_TIMEOUT
  *abort_flag = 1;
}

}  // namespace

__global__ void __launch_bounds__(kThreads, 1) k_ortho(const __grid_constant__ OrthoParams p) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                             ~static_cast<uintptr_t>(1023));
  uint8_t* staging = smem + kStages * kStageBytes;
  __shared__ uint64_t full[kStages], empty[kStages], item_full[kRing], item_empty[kRing], acc_full[2], acc_empty[2],
      last;
  __shared__ Item ring[kRing];
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_s, drained;
  __shared__ float red[kEpi / 32];
  volatile int* abort_flag = &abort_s;
  const int warp = (int)threadIdx.x >> 5;
  if (threadIdx.x == 0) {
    for (int i = 0; i < kStages; ++i) {
      mbar_init(smem_u32(&full[i]), 1);
      mbar_init(smem_u32(&empty[i]), 1);
    }
    for (int i = 0; i < kRing; ++i) {
      mbar_init(smem_u32(&item_full[i]), 1);
      mbar_init(smem_u32(&item_empty[i]), 1 + kEpi / 32);  // the MMA thread and the epilogue warps
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(smem_u32(&acc_full[i]), 1);
      mbar_init(smem_u32(&acc_empty[i]), kEpi / 32);
    }
    mbar_init(smem_u32(&last), 1);
    abort_s = 0;
    drained = 1;
    fence_mbar_init();
  }
  if (warp == 1) {
    tmem_alloc(smem_u32(&tmem_slot), 256);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  pdl_wait();
  const uint32_t tmem = tmem_slot;
  const uint64_t lim = p.wait_limit_ns;  // for a dependency; the waits inside a CTA may hold one

  if (warp == 0) {
    if (elect_one()) {
      int stage = 0, slot = 0;
      uint32_t phase = 0, rphase = 0, issued = 0;
      uint32_t ticket = atomicAdd(p.ticket, 1u);
      while (true) {
        uint32_t need;
        Item it = decode(p, ticket, need);
        if (it.kind != kStop) ticket = atomicAdd(p.ticket, 1u);  // (its latency passes behind this item)
        const OrthoMat& M = p.mat[it.mat];
        if (!mbar_wait(smem_u32(&item_empty[slot]), rphase ^ 1, 3 * lim)) {
          record_timeout(p.status, abort_flag);
          break;
        }
        if (it.kind != kStop && it.kind != kPack) {
          const uint32_t* d = p.done + it.mat;
          if (ld_acquire(d) < need) {
            const uint64_t t0 = globaltimer_ns();
            while (ld_acquire(d) < need) {
              if (*abort_flag || globaltimer_ns() - t0 > lim) {
                record_timeout(p.status, abort_flag);
                break;
              }
            }
          }
          if (*abort_flag) it.kind = kStop;
        }
        ring[slot] = it;
        mbar_arrive(smem_u32(&item_full[slot]));
        if (++slot == kRing) {
          slot = 0;
          rphase ^= 1;
        }
        if (it.kind == kStop) break;
        if (it.kind == kPack) continue;
        fence_proxy_async_all();  // the blocks' writers used both proxies
        const OrthoLayout L = ortho_layout(M.mb, M.nb);
        const uint8_t* X = M.ws + L.x16 + (size_t)(it.step & 1) * M.mb * M.nb * kOrthoBlk;
        const uint8_t* S = M.ws + (it.kind == kFull ? L.b16 : L.a16);  // the symmetric operand
        const int nkb = it.kind == kSym1 ? M.nb : M.mb;
        const int ra = it.I * 2 + 1 < M.mb ? 2 : 1;
        const int rb = it.kind == kFull ? (it.J * 2 + 1 < M.nb ? 2 : 1) : (it.J * 2 + 1 < M.mb ? 2 : 1);
        const bool same = it.kind != kFull && it.I == it.J;  // one operand serves as both
        for (int kb = 0; kb < nkb; ++kb) {
          if (!mbar_wait(smem_u32(&empty[stage]), phase ^ 1, 3 * lim)) {
            record_timeout(p.status, abort_flag);
            break;
          }
          const uint32_t bar = smem_u32(&full[stage]);
          const uint32_t sa = smem_u32(smem + stage * kStageBytes), sb = sa + 2 * kOrthoBlk;
          mbar_arrive_expect_tx(bar, (uint32_t)((ra + (same ? 0 : rb)) * kOrthoBlk));
          for (int i = 0; i < ra; ++i) {
            const int r = it.I * 2 + i;
            const size_t blk = it.kind == kSym1 ? (size_t)r * M.nb + kb
                               : (kb >> 1) <= it.I ? (size_t)r * M.mb + kb : (size_t)kb * M.mb + r;
            bulk_load_1d(sa + i * kOrthoBlk, (it.kind == kSym1 ? X : S) + blk * kOrthoBlk, kOrthoBlk, bar);
          }
          if (!same)
            for (int i = 0; i < rb; ++i) {
              const int r = it.J * 2 + i;
              const size_t blk = it.kind == kSym1 ? (size_t)r * M.nb + kb
                                 : it.kind == kFull ? (size_t)kb * M.nb + r
                                 : (kb >> 1) <= it.J ? (size_t)r * M.mb + kb : (size_t)kb * M.mb + r;
              bulk_load_1d(sb + i * kOrthoBlk, (it.kind == kSym2 ? S : X) + blk * kOrthoBlk, kOrthoBlk, bar);
            }
          ++issued;
          if (++stage == kStages) {
            stage = 0;
            phase ^= 1;
          }
        }
        if (*abort_flag) break;
      }
      if (*abort_flag) {  // copies in flight land before the CTA ends
        for (int i = 0; i < kStages && (uint32_t)i < issued; ++i) {
          stage = stage == 0 ? kStages - 1 : stage - 1;
          if (stage == kStages - 1) phase ^= 1;
          mbar_wait(smem_u32(&full[stage]), phase, 1000000000ull);
        }
      }
    }
  } else if (warp == 1) {
    if (elect_one()) {
      int stage = 0, slot = 0, acc = 0;
      uint32_t phase = 0, rphase = 0, aphase = 0;
      const uint64_t kdesc = smem_desc(0, 16, 1024, 2), mndesc = smem_desc(0, 8192, 1024, 2);
      while (!*abort_flag) {
        if (!mbar_wait(smem_u32(&item_full[slot]), rphase, 2 * lim)) {
          record_timeout(p.status, abort_flag);
          break;
        }
        const Item it = ring[slot];
        mbar_arrive(smem_u32(&item_empty[slot]));
        if (++slot == kRing) {
          slot = 0;
          rphase ^= 1;
        }
        if (it.kind == kStop) break;
        if (it.kind == kPack) continue;
        const OrthoMat& M = p.mat[it.mat];
        const int nkb = it.kind == kSym1 ? M.nb : M.mb;
        const bool same = it.kind != kFull && it.I == it.J;
        if (!mbar_wait(smem_u32(&acc_empty[acc]), aphase ^ 1, 2 * lim)) {
          record_timeout(p.status, abort_flag);
          break;
        }
        tc_fence_after();
        const uint32_t d = tmem + (uint32_t)(acc * 128);
        for (int kb = 0; kb < nkb; ++kb) {
          if (!mbar_wait(smem_u32(&full[stage]), phase, 2 * lim)) {
            record_timeout(p.status, abort_flag);
            break;
          }
          tc_fence_after();
          const bool a_mn = it.kind != kSym1 && (kb >> 1) > it.I;
          const bool b_mn = it.kind == kFull || (it.kind == kSym2 && (kb >> 1) > it.J);
          const uint32_t sa = desc_addr16(smem_u32(smem + stage * kStageBytes));
          const uint32_t sb = same ? sa : sa + (2 * kOrthoBlk >> 4);
          const uint64_t ad = (a_mn ? mndesc : kdesc) + sa, bd = (b_mn ? mndesc : kdesc) + sb;
          const uint32_t as = a_mn ? 2048 >> 4 : 32 >> 4, bs = b_mn ? 2048 >> 4 : 32 >> 4;
          const uint32_t idesc = idesc_f16(128, 128, false, false, true) | (a_mn ? 1u << 15 : 0u) |
                                 (b_mn ? 1u << 16 : 0u);
#pragma unroll
          for (int kk = 0; kk < 4; ++kk)
            tc_mma_f16(d, ad + (uint64_t)(kk * as), bd + (uint64_t)(kk * bs), idesc, kb > 0 || kk > 0);
          tc_commit(smem_u32(&empty[stage]));
          if (++stage == kStages) {
            stage = 0;
            phase ^= 1;
          }
        }
        if (*abort_flag) break;
        tc_commit(smem_u32(&acc_full[acc]));
        acc ^= 1;
        if (acc == 0) aphase ^= 1;
      }
      tc_commit(smem_u32(&last));  // nothing runs in TMEM when it is released
      if (!mbar_wait(smem_u32(&last), 0, lim)) {
        record_timeout(p.status, abort_flag);
        drained = 0;
      }
    }
  } else {
    const int t = (int)threadIdx.x - 64;
    const int lane = t & 31, quad = warp & 3;
    const int row = quad * 32 + lane;     // of the tile (TMEM lane)
    const int half = t >> 7;              // its columns, 64 of them
    const int rr = row & 63;
    int slot = 0, acc = 0, inv_mat = -1;
    float inv = 0.f;
    uint32_t rphase = 0, aphase = 0;
    while (true) {
      if (!mbar_wait(smem_u32(&item_full[slot]), rphase, 2 * lim)) {
        record_timeout(p.status, abort_flag);
        break;
      }
      const Item it = ring[slot];
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&item_empty[slot]));
      if (++slot == kRing) {
        slot = 0;
        rphase ^= 1;
      }
      if (it.kind == kStop) break;
      const OrthoMat& M = p.mat[it.mat];
      if (it.kind == kPack) {
        pack_block(p, M, it.I, it.J, reinterpret_cast<float*>(staging), red, t, inv_mat, inv, it.mat);
        fence_proxy_async_all();
        epi_barrier();
        if (t == 0) {
          __threadfence();
          red_release_add(p.done + it.mat, 1u);
        }
        continue;
      }
      const OrthoLayout L = ortho_layout(M.mb, M.nb);
      const bool full_kind = it.kind == kFull;
      const bool final_step = full_kind && it.step == p.steps - 1;
      const int ncb = full_kind ? M.nb : M.mb;  // block columns of the result
      const int bi = it.I * 2 + (row >> 6), bj = it.J * 2 + half;
      const bool in = bi < M.mb && bj < ncb;
      // what the result adds to the product, loaded while the product runs (the
      // item's dependency, which the loading warp has seen, covers it)
      float x[64];
      float4* x32 = reinterpret_cast<float4*>(M.ws + L.x32 + ((size_t)bi * M.nb + bj) * (2 * kOrthoBlk)) + rr;
      if (full_kind) {
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          const float4 o = in ? __ldcg(x32 + j * 64) : make_float4(0.f, 0.f, 0.f, 0.f);
          x[4 * j] = kA * o.x;
          x[4 * j + 1] = kA * o.y;
          x[4 * j + 2] = kA * o.z;
          x[4 * j + 3] = kA * o.w;
        }
      } else if (it.kind == kSym2) {
        const uint8_t* src = M.ws + L.a16 + ((size_t)bi * M.mb + bj) * kOrthoBlk + rr * 128;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const uint4 o = in ? __ldcg(reinterpret_cast<const uint4*>(src + ((j ^ (rr & 7)) << 4)))
                             : make_uint4(0, 0, 0, 0);
          const uint32_t ow[4] = {o.x, o.y, o.z, o.w};
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const float2 f = h22f(ow[q]);
            x[8 * j + 2 * q] = f.x * (kB * kSb / kSa);
            x[8 * j + 2 * q + 1] = f.y * (kB * kSb / kSa);
          }
        }
      } else {
#pragma unroll
        for (int j = 0; j < 64; ++j) x[j] = 0.f;
      }
      if (!mbar_wait(smem_u32(&acc_full[acc]), aphase, 2 * lim)) {
        record_timeout(p.status, abort_flag);
        break;
      }
      tc_fence_after();
      const float mul = it.kind == kSym1   ? kSa / (kSx * kSx)
                        : it.kind == kSym2 ? kC * kSb / (kSa * kSa)
                                           : 1.f / (kSx * kSb);
#pragma unroll
      for (int c = 0; c < 64; c += 32) {
        uint32_t r[32];
        tmem_ld16(tmem + ((uint32_t)(quad * 32) << 16) + (uint32_t)(acc * 128 + half * 64 + c), r);
        tmem_ld16(tmem + ((uint32_t)(quad * 32) << 16) + (uint32_t)(acc * 128 + half * 64 + c + 16), r + 16);
        tmem_ld_wait();
#pragma unroll
        for (int j = 0; j < 32; ++j) x[c + j] = fmaf(__uint_as_float(r[j]), mul, x[c + j]);
      }
      if (final_step) {
        if (in) finish64(p, M, it.I * 128 + row, it.J * 128 + half * 64, x);
      } else {
        if (full_kind) {
          if (in) {
#pragma unroll
            for (int j = 0; j < 16; ++j)
              __stcg(x32 + j * 64, make_float4(x[4 * j], x[4 * j + 1], x[4 * j + 2], x[4 * j + 3]));
          }
#pragma unroll
          for (int j = 0; j < 64; ++j) x[j] *= kSx;
        }
        const uint32_t st = smem_u32(staging) + (uint32_t)(((row >> 6) * 2 + half) * kOrthoBlk + rr * 128);
#pragma unroll
        for (int h = 0; h < 8; ++h)
          st_shared_v4(st + (uint32_t)((h ^ (rr & 7)) << 4),
                       make_uint4(f2h2(x[8 * h], x[8 * h + 1]), f2h2(x[8 * h + 2], x[8 * h + 3]),
                                  f2h2(x[8 * h + 4], x[8 * h + 5]), f2h2(x[8 * h + 6], x[8 * h + 7])));
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&acc_empty[acc]));
      acc ^= 1;
      if (acc == 0) aphase ^= 1;
      fence_proxy_async_all();
      epi_barrier();
      if (t == 0) {
        if (!final_step) {
          uint8_t* out = M.ws + (it.kind == kSym1   ? L.a16
                                 : it.kind == kSym2 ? L.b16
                                                    : L.x16 + (size_t)((it.step + 1) & 1) * M.mb * M.nb * kOrthoBlk);
          for (int q = 0; q < 4; ++q) {
            const int obi = it.I * 2 + (q >> 1), obj = it.J * 2 + (q & 1);
            if (obi < M.mb && obj < ncb)
              bulk_store_1d(out + ((size_t)obi * ncb + obj) * kOrthoBlk, smem_u32(staging) + q * kOrthoBlk, kOrthoBlk);
          }
          bulk_commit();
          bulk_wait0();
          fence_proxy_async_all();
        }
        __threadfence();
        red_release_add(p.done + it.mat, 1u);
      }
      epi_barrier();  // the staging buffer is free again
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1 && drained) {
    tc_fence_after();
    tmem_dealloc(tmem, 256);
  }
}

cudaError_t launch_ortho(const OrthoParams& p, int sms, cudaStream_t s) {
  cudaError_t e = cudaFuncSetAttribute(k_ortho, cudaFuncAttributeMaxDynamicSharedMemorySize, kOrthoSmem);
  if (e != cudaSuccess) return e;
  e = launch_pdl(k_ortho_norm, dim3((unsigned)p.total_parts), dim3(256), 0, s, p);
  if (e != cudaSuccess) return e;
  const int grid = p.max_items < sms ? p.max_items : sms;
  e = launch_pdl(k_ortho, dim3((unsigned)grid), dim3(kThreads), kOrthoSmem, s, p);
  if (e != cudaSuccess) return e;
  return counted_launches(2);
}

}  // namespace pf16
