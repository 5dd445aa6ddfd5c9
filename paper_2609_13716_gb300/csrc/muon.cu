// muon.cu -- orthogonalised updates of weight matrices (include/aht.h states the method):
// momentum, Newton-Schulz orthogonalisation on tensor cores, weight update, for a set of
// matrices at once.
//
// Each matrix is taken with its short side m as rows (a tall one transposed) and padded
// with zeros to whole 128 x 128 blocks.  Of the three products of a step,
//   A = X X^T,   B = a I + b A + c A A,   X' = B X,
// the first two are symmetric: only blocks (I, J) with I <= J are computed and stored, and
// block (J, I) is the same data read with the other operand major.
//
// Precision: products accurate to fp32 on 16-bit tensor cores.  An operand is stored as
// hi + lo, two fp16 of it scaled by a power of two (hi the nearest fp16, lo the nearest fp16
// of the rest: 22 significant bits), and a product is hi hi + hi lo + lo hi, accumulated in
// fp32.  fp16 suits the iteration because its operands are bounded: with ||X||_F <= 1 every
// singular value of X stays in [0, 1.21] (the quintic's maximum over [0, 1.21]), so the
// entries of X, A and B stay below 1.21, 1.47 and 3.45, and with the scales 2^14, 2^14 and
// 2^13 nothing leaves fp16's range while lo's subnormal step is 2^-39 of 1.
//
// Storage: block [128 rows r][128 columns c] as 256 core matrices of 8 x 8, core (c / 8,
// r / 8) at ((c / 8) * 16 + r / 8) * 128, 32 KB contiguous, so a block moves by one bulk
// copy and serves as a K-major operand (rows as M or N, columns as K) or as an MN-major one
// (columns as M or N, rows as K).
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

#include "kernels.h"
#include "tc_common.cuh"

namespace aht {
aht_status set_last_error(aht_status s, const char* msg);  // the message of aht_last_error
}  // namespace aht

using namespace aht;

namespace {

constexpr int kB = 128;                        // block edge
constexpr uint32_t kBlk = kB * kB * 2;         // bytes of one fp16 block
constexpr uint32_t kHalf = kBlk / 2;           // 64 of K of one block
constexpr uint32_t kStage = 4 * kHalf;         // lo of B, hi and lo of A, hi of B
constexpr int kStages = 3;
constexpr int kAcc = 4;                        // accumulators in tensor memory
constexpr int kGemmThreads = 320;              // producer, MMA, 8 epilogue warps
constexpr int kEpiThreads = 256;
constexpr float kA = 3.4445f, kBq = -4.7750f, kC = 2.0315f;  // Jordan et al. 2024
constexpr float kSX = 16384.0f, kSA = 16384.0f, kSB = 8192.0f;
constexpr int kNormBlocks = 256;               // most partial sums of squares per matrix
constexpr int kMaxSteps = 32;

struct Mat {
  int32_t rows, cols, m, n, mb, nb, tall;
  int32_t norm_blocks;                         // partial sums of squares
  int64_t x[2], a, b;                          // byte offsets of the hi blocks
  int64_t x_lo, s_lo;                          // from a hi block to its lo block
};

enum Phase : int { kGram = 0, kPoly = 1, kApply = 2 };

// The caller's arrays of one call, by value (at most AHT_MUON_MAX_MATRICES).
struct Ptrs {
  const void* in[AHT_MUON_MAX_MATRICES];       // gradient or the matrix to orthogonalise
  void* out[AHT_MUON_MAX_MATRICES];            // weights or the orthogonalised matrix
  float* mom[AHT_MUON_MAX_MATRICES];
  int32_t ld_in[AHT_MUON_MAX_MATRICES], ld_out[AHT_MUON_MAX_MATRICES], ld_mom[AHT_MUON_MAX_MATRICES];
};

struct Common {
  const Mat* mats;
  uint8_t* ws;
  double* norm;                                // [n_mats][kNormBlocks]
  uint32_t* done;                              // [n_mats][3 phases][kMaxSteps] finished tiles
  uint32_t* status;
  const int4* items;                           // (matrix, phase, I, J) of one step
  int32_t n_items, steps;
  int32_t bf16_in, bf16_out, update, nesterov;
  float mu, eps, decay, lr;                    // decay = 1 - lr * weight_decay
};

__device__ __forceinline__ float load_in(const Common& c, const Ptrs& p, int k, int64_t r, int64_t col) {
  const int64_t at = r * p.ld_in[k] + col;
  return c.bf16_in ? __bfloat162float(static_cast<const __nv_bfloat16*>(p.in[k])[at])
                   : static_cast<const float*>(p.in[k])[at];
}

// ---- momentum and the sum of squares of U ------------------------------------------------
// Also clears the tile counters of the call.
__global__ void __launch_bounds__(256) momentum_norm(const __grid_constant__ Common c, const __grid_constant__ Ptrs p) {
  const int k = blockIdx.y;
  const Mat m = c.mats[k];
  if ((int)blockIdx.x >= m.norm_blocks) return;
  if (blockIdx.x == 0 && threadIdx.x < 3 * kMaxSteps) c.done[k * 3 * kMaxSteps + threadIdx.x] = 0;
  const uint32_t total = (uint32_t)m.rows * (uint32_t)m.cols;  // at most 2^28
  double sum = 0.0;
  for (uint32_t e = blockIdx.x * 256 + threadIdx.x; e < total; e += m.norm_blocks * 256) {
    const uint32_t r = e / (uint32_t)m.cols, col = e - r * (uint32_t)m.cols;
    float u = load_in(c, p, k, r, col);
    if (c.update) {
      float* mp = p.mom[k] + (int64_t)r * p.ld_mom[k] + col;
      const float mom = fmaf(c.mu, *mp, u);
      *mp = mom;
      u = c.nesterov ? fmaf(c.mu, mom, u) : mom;
    }
    sum += (double)(u * u);
  }
  __shared__ double sh[256];
  sh[threadIdx.x] = sum;
  for (int s = 128; s > 0; s >>= 1) {
    __syncthreads();
    if (threadIdx.x < s) sh[threadIdx.x] += sh[threadIdx.x + s];
  }
  if (threadIdx.x == 0) c.norm[k * kNormBlocks + blockIdx.x] = sh[0];
}

// 8 values (already scaled) -> their hi and lo chunks
__device__ __forceinline__ void split8(const float* v, uint4& hi, uint4& lo) {
  uint32_t h[4], l[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __half2 hh = __floats2half2_rn(v[2 * i], v[2 * i + 1]);
    const float2 f = __half22float2(hh);
    const __half2 ll = __floats2half2_rn(v[2 * i] - f.x, v[2 * i + 1] - f.y);
    h[i] = *reinterpret_cast<const uint32_t*>(&hh);
    l[i] = *reinterpret_cast<const uint32_t*>(&ll);
  }
  hi = make_uint4(h[0], h[1], h[2], h[3]);
  lo = make_uint4(l[0], l[1], l[2], l[3]);
}

// byte offset in a block of the chunk of row r holding columns 8 cb .. 8 cb + 7
__device__ __forceinline__ int64_t chunk_at(int r, int cb) { return ((cb * 16 + (r >> 3)) << 7) + ((r & 7) << 4); }

// ---- X = U / (||U||_F + eps), split into blocks -------------------------------------------
// One thread per 8-column chunk of a row of X; consecutive threads take consecutive rows.
__global__ void __launch_bounds__(256) normalise(const __grid_constant__ Common c, const __grid_constant__ Ptrs p) {
  const int k = blockIdx.y;
  const Mat m = c.mats[k];
  const int64_t chunks = (int64_t)m.mb * m.nb * 2048;
  if ((int64_t)blockIdx.x * 256 >= chunks) return;
  __shared__ double sh[256];
  sh[threadIdx.x] = (int)threadIdx.x < m.norm_blocks ? c.norm[k * kNormBlocks + threadIdx.x] : 0.0;
  for (int s = 128; s > 0; s >>= 1) {
    __syncthreads();
    if (threadIdx.x < s) sh[threadIdx.x] += sh[threadIdx.x + s];
  }
  __syncthreads();
  const float inv = (float)(1.0 / (sqrt(sh[0]) + (double)c.eps));
  uint8_t* x = c.ws + m.x[0];
  for (int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x; q < chunks; q += (int64_t)gridDim.x * 256) {
    const int blk = (int)(q >> 11);
    const int r = (int)(q & 127), cb = (int)(q >> 7) & 15;
    const int bi = blk / m.nb, i = bi * kB + r, j0 = (blk - bi * m.nb) * kB + 8 * cb;
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int j = j0 + e;
      v[e] = 0.0f;
      if (i < m.m && j < m.n) {
        const int64_t row = m.tall ? j : i, col = m.tall ? i : j;
        float u = load_in(c, p, k, row, col);
        if (c.update) {
          const float mom = p.mom[k][row * p.ld_mom[k] + col];
          u = c.nesterov ? fmaf(c.mu, mom, u) : mom;
        }
        v[e] = (u * inv) * kSX;
      }
    }
    uint4 hi, lo;
    split8(v, hi, lo);
    uint8_t* at = x + (int64_t)blk * kBlk + chunk_at(r, cb);
    *reinterpret_cast<uint4*>(at) = hi;
    *reinterpret_cast<uint4*>(at + m.x_lo) = lo;
  }
}

// ---- the products -------------------------------------------------------------------------
// Block (I, k) of a symmetric matrix as an operand with rows I: stored when I <= k, else
// block (k, I) with the other major.
struct Operand {
  int64_t at;          // byte offset of the hi block in the workspace
  int64_t lo;          // offset of its lo block
  bool mn;             // MN-major
};
__device__ __forceinline__ Operand sym(int64_t s, int64_t lo, int mb, int I, int k) {
  const bool up = I <= k;
  return Operand{s + ((int64_t)(up ? I : k) * mb + (up ? k : I)) * kBlk, lo, !up};
}

__device__ __forceinline__ void operands(int phase, const Mat& m, int cur, int I, int J, int k, Operand& A, Operand& B) {
  const int64_t x = cur ? m.x[1] : m.x[0];
  if (phase == kGram) {
    A = Operand{x + ((int64_t)I * m.nb + k) * kBlk, m.x_lo, false};
    B = Operand{x + ((int64_t)J * m.nb + k) * kBlk, m.x_lo, false};
  } else if (phase == kPoly) {
    A = sym(m.a, m.s_lo, m.mb, I, k);
    B = sym(m.a, m.s_lo, m.mb, J, k);
  } else {
    A = sym(m.b, m.s_lo, m.mb, I, k);
    B = Operand{x + ((int64_t)k * m.nb + J) * kBlk, m.x_lo, true};
  }
}

__device__ __forceinline__ uint32_t ld_acquire(const uint32_t* p) {
  uint32_t v;
  asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
  return v;
}
__device__ __forceinline__ void add_release(uint32_t* p) {
  asm volatile("red.release.gpu.global.add.u32 [%0], 1;" ::"l"(p) : "memory");
}
// Orders this thread's ordinary accesses to global memory with bulk copies, both ways.
__device__ __forceinline__ void fence_proxy_global() { asm volatile("fence.proxy.async.global;" ::: "memory"); }

// The 64 rows r0.. of a block (all its columns): core matrices [16 column groups][8 row
// groups], 16 KB.
__device__ __forceinline__ void rows_g2s(void* dst, const CUtensorMap* map, int64_t block, int r0, uint64_t* mbar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(
          tc::smem_u32(dst)),
      "l"(map), "r"(0), "r"(r0 >> 3), "r"((int)(block * 16)), "r"(tc::smem_u32(mbar))
      : "memory");
}

// One persistent cooperative kernel runs every product of the call: the items (step, phase,
// matrix, I, J) in that order, item g on CTA g mod grid.  An item begins when the tiles that
// it reads are complete (counters per matrix, phase and step), so matrices advance
// independently and a CTA without work in one matrix's phase goes on with another's.  An
// item only waits for earlier ones and all CTAs are resident, so the earliest unfinished item
// always runs.
//
// Warp 0 streams stages of 64 of K, the hi and lo halves of a block of A and of B (A alone
// where they are the same block); four lanes issue one copy each, since a lane needs about 240
// clocks per copy and a stage is 768 clocks of products.  A half with K along its columns is
// contiguous; one with K along its rows is a 3-D tensor copy.  Warp 1 (one lane) issues the
// products, the small ones first, 128 of K into one of four accumulators.  Warps 2-9 add each
// accumulator to fp32 registers (the tensor core rounds its running sum towards zero: summed
// over all of K the bias of a 1024-wide product showed as 2e-5 of the result; 128 at a time it
// stays near 1e-6) and run the tile's epilogue.
__global__ void __launch_bounds__(kGemmThreads, 1)
    products(const __grid_constant__ Common c, const __grid_constant__ Ptrs p, const __grid_constant__ CUtensorMap map) {
  extern __shared__ __align__(1024) uint8_t smem[];
  __shared__ __align__(8) uint64_t full_bar[kStages], empty_bar[kStages];
  __shared__ __align__(8) uint64_t accf_bar[kAcc], acce_bar[kAcc], drain_bar;
  __shared__ uint32_t tmem_slot;
  __shared__ volatile int abort_flag;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    for (int s = 0; s < kStages; ++s) {
      tc::mbar_init(&full_bar[s], 1);
      tc::mbar_init(&empty_bar[s], 1);
    }
    for (int i = 0; i < kAcc; ++i) {
      tc::mbar_init(&accf_bar[i], 1);
      tc::mbar_init(&acce_bar[i], kEpiThreads);
    }
    tc::mbar_init(&drain_bar, 1);
    tc::mbar_init_fence();
    abort_flag = 0;
  }
  if (warp == 0) tc::tmem_alloc(&tmem_slot, 512);
  tc::fence_before_sync();
  __syncthreads();
  tc::fence_after_sync();
  const uint32_t tmem = tmem_slot;
  int issued = 0;  // (producer) stages filled
  const int n_all = c.n_items * c.steps;

  auto wait_or_abort = [&](uint64_t* bar, uint32_t parity) {
    bool ok = false;
    for (int tries = 0; tries < 1000 && !ok && !abort_flag; ++tries) ok = tc::mbar_wait(bar, parity, 2000000ull);
    return ok;
  };
  // the tiles an item reads are complete (bounded wait)
  auto ready = [&](const Mat& m, int k, int phase, int it) {
    if (phase == kGram && it == 0) return true;
    const uint32_t tri = (uint32_t)(m.mb * (m.mb + 1) / 2);
    const int from = phase == kGram ? kApply : phase - 1;
    const uint32_t want = from == kApply ? (uint32_t)(m.mb * m.nb) : tri;
    const uint32_t* at = c.done + (k * 3 + from) * kMaxSteps + (phase == kGram ? it - 1 : it);
    if (ld_acquire(at) >= want) return true;
    const uint64_t t0 = tc::globaltimer_ns();
    for (uint32_t i = 0; i < (1u << 30) && !abort_flag; ++i) {
      if (ld_acquire(at) >= want) return true;
      if ((i & 63u) == 63u && tc::globaltimer_ns() - t0 > 2000000000ull) return false;
    }
    return false;
  };
  auto k_blocks = [&](const Mat& m, int phase) { return phase == kGram ? m.nb : m.mb; };

  if (warp == 0) {
    if (lane < 4) {
      const bool of_a = lane == 1 || lane == 2, lo = lane == 0 || lane == 2;
      uint8_t* dst0 = smem + lane * kHalf;
      bool ok = true;
      int s = 0;
      for (int g = blockIdx.x; ok && g < n_all; g += gridDim.x) {
        const int it = g / c.n_items;
        const int4 item = c.items[g - it * c.n_items];
        const Mat m = c.mats[item.x];
        if (!(ok = ready(m, item.x, item.y, it))) break;
        fence_proxy_global();
        const int K = k_blocks(m, item.y);
        for (int k = 0; ok && k < K; ++k) {
          Operand A, B;
          operands(item.y, m, it & 1, item.z, item.w, k, A, B);
          const bool same = A.at == B.at;
          const Operand& o = of_a ? A : B;
          const int64_t off = o.at + (lo ? o.lo : 0);
          for (int h = 0; h < 2; ++h) {
            if (issued >= kStages && !(ok = wait_or_abort(&empty_bar[s], (uint32_t)(issued / kStages - 1) & 1u))) break;
            if (lane == 0) tc::mbar_expect_tx(&full_bar[s], same ? 2 * kHalf : kStage);
            if (of_a || !same) {
              uint8_t* dst = dst0 + (size_t)s * kStage;
              if (o.mn) rows_g2s(dst, &map, off / kBlk, 64 * h, &full_bar[s]);
              else tc::bulk_g2s(dst, c.ws + off + h * kHalf, kHalf, &full_bar[s]);
            }
            ++issued;
            if (++s == kStages) s = 0;
          }
        }
      }
      if (!ok) abort_flag = 1;
    }
  } else if (warp == 1) {
    if (lane == 0) {
      const uint32_t idesc = (1u << 4) | ((uint32_t)(kB >> 3) << 17) | ((uint32_t)(kB >> 4) << 24);  // fp16 -> fp32
      const uint32_t base = tc::smem_u32(smem);
      int j = 0, s = 0;
      uint32_t par = 0;
      bool ok = true;
      for (int g = blockIdx.x; ok && g < n_all; g += gridDim.x) {
        const int it = g / c.n_items;
        const int4 item = c.items[g - it * c.n_items];
        const int K = item.y == kGram ? c.mats[item.x].nb : c.mats[item.x].mb;
        const bool same = item.y != kApply && item.z == item.w;
        for (int k = 0; ok && k < K; ++k, ++j) {
          // the majors of operands(): a symmetric block is stored when row <= column
          const bool a_mn = item.y != kGram && item.z > k;
          const bool b_mn = item.y == kApply || (item.y == kPoly && item.w > k);
          const uint32_t id = idesc | (a_mn ? 1u << 15 : 0u) | (b_mn ? 1u << 16 : 0u);
          const uint32_t da = a_mn ? 16u : 256u, db = b_mn ? 16u : 256u;  // 16 of K, in 16-byte units
          const int acc = j % kAcc;
          if (j >= kAcc && !(ok = wait_or_abort(&acce_bar[acc], (uint32_t)(j / kAcc - 1) & 1u))) break;
          const uint32_t D = tmem + (uint32_t)(acc * kB);
          auto desc = [&](uint32_t addr, bool mn) {
            return mn ? tc::smem_desc(addr, 128u, 1024u) : tc::smem_desc(addr, 2048u, 128u);
          };
          for (int h = 0; h < 2; ++h) {
            if (!(ok = wait_or_abort(&full_bar[s], par))) break;
            tc::fence_after_sync();
            const uint32_t at = base + (uint32_t)s * kStage;
            const uint64_t a_hi = desc(at + kHalf, a_mn), a_lo = desc(at + 2 * kHalf, a_mn);
            const uint64_t b_hi = same ? a_hi : desc(at + 3 * kHalf, b_mn), b_lo = same ? a_lo : desc(at, b_mn);
            auto mma = [&](uint64_t a, uint64_t b, bool first) {
#pragma unroll
              for (int kk = 0; kk < 4; ++kk)
                tc::mma_ss(D, a + (uint64_t)(da * kk), b + (uint64_t)(db * kk), id, !(first && kk == 0));
            };
            mma(a_hi, b_lo, h == 0);
            mma(a_lo, b_hi, false);
            mma(a_hi, b_hi, false);
            tc::commit(&empty_bar[s]);
            if (++s == kStages) {
              s = 0;
              par ^= 1u;
            }
          }
          if (ok) tc::commit(&accf_bar[acc]);
        }
      }
      if (!ok) abort_flag = 1;
    }
  } else {
    const int q = warp & 3, r = 32 * q + lane;      // row of the tile
    const uint32_t lane_base = (uint32_t)(32 * q) << 16;
    const int c_beg = ((warp - 2) >> 2) * 64;       // this warp's half of the columns
    int j = 0;
    bool ok = true;
    for (int g = blockIdx.x; g < n_all; g += gridDim.x) {
      const int it = g / c.n_items;
      const int4 item = c.items[g - it * c.n_items];
      const Mat& m = c.mats[item.x];
      const int phase = item.y, I = item.z, J = item.w, K = phase == kGram ? m.nb : m.mb;
      float f[64];
#pragma unroll
      for (int e = 0; e < 64; ++e) f[e] = 0.0f;
      for (int k = 0; k < K; ++k, ++j) {
        const int acc = j % kAcc;
        bool got = false;
        if (ok) got = wait_or_abort(&accf_bar[acc], (uint32_t)(j / kAcc) & 1u);
        ok = __all_sync(0xFFFFFFFFu, ok && got);    // warp-uniform: tensor-memory loads are collective
        if (!ok) break;
        tc::fence_after_sync();
#pragma unroll
        for (int c0 = 0; c0 < 64; c0 += 32) {
          uint32_t v[32];
          tc::ld_x32(tmem + (uint32_t)(acc * kB + c_beg + c0) + lane_base, v);
          tc::wait_ld();
#pragma unroll
          for (int e = 0; e < 32; ++e) f[c0 + e] += __uint_as_float(v[e]);
        }
        tc::fence_before_sync();
        tc::mbar_arrive(&acce_bar[acc]);
      }
      const bool last = phase == kApply && it + 1 == c.steps;
      if (ok && last) {
        const int i = I * kB + r, j0 = J * kB + c_beg;
        if (i < m.m) {
          const float lr = c.update ? c.lr * sqrtf(fmaxf(1.0f, (float)m.rows / (float)m.cols)) : 0.0f;
          const int64_t ld = p.ld_out[item.x], step = m.tall ? ld : 1;
          const int64_t at0 = m.tall ? (int64_t)j0 * ld + i : (int64_t)i * ld + j0;
          void* out = p.out[item.x];
          // rows of whole, aligned groups of four
          const bool four = !m.tall && j0 + 64 <= m.n && !c.bf16_out && ((uintptr_t)out & 15) == 0 && (ld & 3) == 0;
#pragma unroll
          for (int e = 0; e < 64; e += 4) {
            float o[4];
#pragma unroll
            for (int x = 0; x < 4; ++x) o[x] = f[e + x] * (1.0f / (kSB * kSX));
            if (four) {
              float4* w = reinterpret_cast<float4*>(static_cast<float*>(out) + at0 + e);
              if (c.update) {
                const float4 old = *w;
                *w = make_float4(fmaf(-lr, o[0], c.decay * old.x), fmaf(-lr, o[1], c.decay * old.y),
                                 fmaf(-lr, o[2], c.decay * old.z), fmaf(-lr, o[3], c.decay * old.w));
              } else {
                *w = make_float4(o[0], o[1], o[2], o[3]);
              }
              continue;
            }
#pragma unroll
            for (int x = 0; x < 4; ++x) {
              if (j0 + e + x >= m.n) continue;
              const int64_t at = at0 + (e + x) * step;
              if (c.update) {
                float* w = static_cast<float*>(out) + at;
                *w = fmaf(-lr, o[x], c.decay * *w);
              } else if (c.bf16_out) {
                static_cast<__nv_bfloat16*>(out)[at] = __float2bfloat16_rn(o[x]);
              } else {
                static_cast<float*>(out)[at] = o[x];
              }
            }
          }
        }
      } else if (ok) {
        const int64_t blk = (phase == kApply ? (int64_t)I * m.nb : (int64_t)I * m.mb) + J;
        uint8_t* out = c.ws + (phase == kGram ? m.a : phase == kPoly ? m.b : it & 1 ? m.x[0] : m.x[1]) + blk * kBlk;
        const int64_t lo_off = phase == kApply ? m.x_lo : m.s_lo;
        const float scale = phase == kGram ? kSA / (kSX * kSX) : phase == kPoly ? kC * kSB / (kSA * kSA) : 1.0f / kSB;
        const uint8_t* ap = c.ws + m.a + blk * kBlk;
        // complete since before this tile's operands were loaded; acquired by this thread too
        if (phase == kPoly) ld_acquire(c.done + (item.x * 3 + kGram) * kMaxSteps + it);
#pragma unroll
        for (int t = 0; t < 8; ++t) {
          const int cb = (c_beg >> 3) + t;
#pragma unroll
          for (int e = 0; e < 8; ++e) f[8 * t + e] *= scale;
          if (phase == kPoly) {
            const uint4 ah = __ldcg(reinterpret_cast<const uint4*>(ap + chunk_at(r, cb)));
            const uint4 al = __ldcg(reinterpret_cast<const uint4*>(ap + m.s_lo + chunk_at(r, cb)));
            const uint32_t hw[4] = {ah.x, ah.y, ah.z, ah.w}, lw[4] = {al.x, al.y, al.z, al.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float2 h2 = __half22float2(*reinterpret_cast<const __half2*>(&hw[e]));
              const float2 l2 = __half22float2(*reinterpret_cast<const __half2*>(&lw[e]));
              f[8 * t + 2 * e] = fmaf(h2.x + l2.x, kBq * kSB / kSA, f[8 * t + 2 * e]);
              f[8 * t + 2 * e + 1] = fmaf(h2.y + l2.y, kBq * kSB / kSA, f[8 * t + 2 * e + 1]);
            }
#pragma unroll
            for (int e = 0; e < 8; ++e)
              if (I == J && r == 8 * cb + e) f[8 * t + e] += kA * kSB;
          }
          uint4 hi, lo;
          split8(f + 8 * t, hi, lo);
          uint8_t* at = out + chunk_at(r, cb);
          *reinterpret_cast<uint4*>(at) = hi;
          *reinterpret_cast<uint4*>(at + lo_off) = lo;
        }
        fence_proxy_global();
        __threadfence();
      }
      // all eight warps leave together: none is left at the barrier
      ok = !tc::bar_or(1, kEpiThreads, !ok);
      if (!ok) break;
      if (!last && tid == 64) add_release(c.done + (item.x * 3 + phase) * kMaxSteps + it);
    }
    if (!ok) abort_flag = 1;
  }

  // the MMAs and copies this CTA issued complete (bounded), then tensor memory is freed
  tc::fence_before_sync();
  __syncthreads();
  if (tid == 0 && abort_flag) atomicOr(c.status, kStatusTimeout);
  if (warp == 1 && lane == 0) {
    tc::commit(&drain_bar);
    tc::mbar_wait(&drain_bar, 0);
  }
  if (warp == 0 && lane == 0 && abort_flag) {
    for (int d = issued - 1; d >= 0 && d >= issued - kStages; --d)
      tc::mbar_wait(&full_bar[d % kStages], (uint32_t)(d / kStages) & 1u);
  }
  tc::fence_before_sync();
  __syncthreads();
  if (warp == 0) {
    tc::fence_after_sync();
    tc::tmem_dealloc(tmem, 512);
  }
}

struct MuonDeviceGuard {
  int prev = -1;
  explicit MuonDeviceGuard(int dev) {
    if (cudaGetDevice(&prev) == cudaSuccess && prev != dev) cudaSetDevice(dev);
    else prev = -1;
  }
  ~MuonDeviceGuard() {
    if (prev >= 0) cudaSetDevice(prev);
  }
};

}  // namespace

struct aht_muon {
  int device = 0;
  cudaStream_t stream = nullptr;
  aht_muon_config cfg{};
  std::vector<Mat> mats;
  int n_sms = 0, n_items = 0;
  int norm_blocks = 0, norm_chunks = 0;  // CTAs per matrix of momentum_norm and normalise
  Mat* d_mats = nullptr;
  int4* items = nullptr;
  uint32_t* done = nullptr;
  CUtensorMap map{};
  uint8_t* ws = nullptr;
  double* norm = nullptr;
  uint32_t* status = nullptr;
  std::vector<void*> owned;
};

namespace {

#define MUON_CUDA(call)                                                                \
  do {                                                                                 \
    cudaError_t e_ = (call);                                                           \
    if (e_ != cudaSuccess) return set_last_error(AHT_ECUDA, cudaGetErrorString(e_));  \
  } while (0)

aht_status run(aht_muon* s, Common c, const Ptrs& p) {
  MuonDeviceGuard g(s->device);
  c.mats = s->d_mats;
  c.ws = s->ws;
  c.norm = s->norm;
  c.done = s->done;
  c.status = s->status;
  c.items = s->items;
  c.n_items = s->n_items;
  c.steps = s->cfg.steps;
  c.eps = s->cfg.eps;
  c.mu = s->cfg.momentum;
  c.nesterov = s->cfg.nesterov;
  const unsigned n = (unsigned)s->mats.size();
  momentum_norm<<<dim3((unsigned)s->norm_blocks, n), 256, 0, s->stream>>>(c, p);
  MUON_CUDA(cudaGetLastError());
  normalise<<<dim3((unsigned)s->norm_chunks, n), 256, 0, s->stream>>>(c, p);
  MUON_CUDA(cudaGetLastError());
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)std::min(s->n_items, s->n_sms));
  cfg.blockDim = dim3(kGemmThreads);
  cfg.dynamicSmemBytes = kStages * kStage;
  cfg.stream = s->stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeCooperative;  // every CTA resident: they wait for one another's tiles
  attr[0].val.cooperative = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  MUON_CUDA(cudaLaunchKernelEx(&cfg, products, c, p, s->map));
  return AHT_OK;
}

// The workspace as a tensor of core matrices: [blocks * 16 column groups][16 row groups][64
// fp16], copied in boxes of 16 column groups x 8 row groups.
aht_status make_map(aht_muon* s, int64_t bytes) {
  void* fn = nullptr;
  cudaDriverEntryPointQueryResult found;
  MUON_CUDA(cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &found));
  if (found != cudaDriverEntryPointSuccess || !fn)
    return set_last_error(AHT_ECUDA, "the driver has no cuTensorMapEncodeTiled");
  const cuuint64_t dims[3] = {64, 16, (cuuint64_t)(bytes / 2048)}, strides[2] = {128, 2048};
  const cuuint32_t box[3] = {64, 8, 16}, one[3] = {1, 1, 1};
  const CUresult e = reinterpret_cast<decltype(&cuTensorMapEncodeTiled)>(fn)(
      &s->map, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, s->ws, dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
      CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return e == CUDA_SUCCESS ? AHT_OK : set_last_error(AHT_ECUDA, "cuTensorMapEncodeTiled failed");
}

aht_status create(int32_t n, const int32_t* rows, const int32_t* cols, const aht_muon_config* cfg, cudaStream_t stream,
                  aht_muon* s) {
  s->stream = stream;
  s->cfg = *cfg;
  MUON_CUDA(cudaGetDevice(&s->device));
  MUON_CUDA(cudaDeviceGetAttribute(&s->n_sms, cudaDevAttrMultiProcessorCount, s->device));
  int64_t at = 0, most = 0;
  auto region = [&](int64_t blocks) {
    const int64_t o = at;
    at += 2 * blocks * kBlk;      // hi, then lo
    return o;
  };
  std::vector<int4> items[3];
  for (int k = 0; k < n; ++k) {
    Mat m{};
    m.rows = rows[k];
    m.cols = cols[k];
    m.tall = rows[k] > cols[k];
    m.m = std::min(rows[k], cols[k]);
    m.n = std::max(rows[k], cols[k]);
    m.mb = (m.m + kB - 1) / kB;
    m.nb = (m.n + kB - 1) / kB;
    m.x[0] = region((int64_t)m.mb * m.nb);
    m.x[1] = region((int64_t)m.mb * m.nb);
    m.a = region((int64_t)m.mb * m.mb);
    m.b = region((int64_t)m.mb * m.mb);
    m.x_lo = (int64_t)m.mb * m.nb * kBlk;
    m.s_lo = (int64_t)m.mb * m.mb * kBlk;
    m.norm_blocks = (int)std::min<int64_t>(((int64_t)m.rows * m.cols + 2047) / 2048, kNormBlocks);
    most = std::max(most, (int64_t)m.mb * m.nb);
    s->norm_blocks = std::max(s->norm_blocks, m.norm_blocks);
    s->mats.push_back(m);
    for (int I = 0; I < m.mb; ++I) {
      for (int J = I; J < m.mb; ++J) {
        items[kGram].push_back(make_int4(k, kGram, I, J));
        items[kPoly].push_back(make_int4(k, kPoly, I, J));
      }
      for (int J = 0; J < m.nb; ++J) items[kApply].push_back(make_int4(k, kApply, I, J));
    }
  }
  // the longest tiles of a phase first
  std::vector<int4> all;
  for (int ph = 0; ph < 3; ++ph) {
    std::stable_sort(items[ph].begin(), items[ph].end(), [&](const int4& x, const int4& y) {
      const Mat &a = s->mats[x.x], &b = s->mats[y.x];
      return (ph == kGram ? a.nb : a.mb) > (ph == kGram ? b.nb : b.mb);
    });
    all.insert(all.end(), items[ph].begin(), items[ph].end());
  }
  if (all.size() > (1u << 31) / (size_t)cfg->steps / 2) return set_last_error(AHT_EINVAL, "too many tiles in one call");
  s->n_items = (int)all.size();
  s->norm_chunks = (int)std::min<int64_t>(most * 8, 1024);
  auto alloc = [&](void** ptr, size_t bytes) {
    if (cudaMalloc(ptr, bytes) != cudaSuccess) {
      cudaGetLastError();
      return false;
    }
    s->owned.push_back(*ptr);
    return true;
  };
  auto up = [&](void** dst, const void* h, size_t bytes) {
    return alloc(dst, bytes) && cudaMemcpy(*dst, h, bytes, cudaMemcpyHostToDevice) == cudaSuccess;
  };
  if (!up((void**)&s->d_mats, s->mats.data(), s->mats.size() * sizeof(Mat)) ||
      !up((void**)&s->items, all.data(), all.size() * sizeof(int4)) || !alloc((void**)&s->ws, (size_t)at) ||
      !alloc((void**)&s->norm, (size_t)n * kNormBlocks * sizeof(double)) ||
      !alloc((void**)&s->done, (size_t)n * 3 * kMaxSteps * 4) || !alloc((void**)&s->status, 4) ||
      cudaMemset(s->status, 0, 4) != cudaSuccess)
    return set_last_error(AHT_ENOMEM, "workspace allocation failed");
  MUON_CUDA(cudaFuncSetAttribute(products, cudaFuncAttributeMaxDynamicSharedMemorySize, kStages * (int)kStage));
  return make_map(s, at);
}

}  // namespace

extern "C" {

aht_status aht_muon_create(int32_t n, const int32_t* rows, const int32_t* cols, const aht_muon_config* cfg,
                           void* cuda_stream, aht_muon** out) {
  if (!out) return set_last_error(AHT_EINVAL, "out is NULL");
  *out = nullptr;
  if (!rows || !cols || !cfg) return set_last_error(AHT_EINVAL, "NULL sizes or config");
  if (n < 1 || n > AHT_MUON_MAX_MATRICES) return set_last_error(AHT_EINVAL, "1 to AHT_MUON_MAX_MATRICES matrices");
  for (int k = 0; k < n; ++k)
    if (rows[k] < 1 || cols[k] < 1 || rows[k] > AHT_MUON_MAX_DIM || cols[k] > AHT_MUON_MAX_DIM)
      return set_last_error(AHT_EINVAL, "rows and cols must be in 1..AHT_MUON_MAX_DIM");
  if (!(cfg->momentum >= 0.0f && cfg->momentum < 1.0f))
    return set_last_error(AHT_EINVAL, "momentum must be in [0, 1)");
  if (!(cfg->weight_decay >= 0.0f) || !std::isfinite(cfg->weight_decay) || !(cfg->eps > 0.0f) ||
      !std::isfinite(cfg->eps))
    return set_last_error(AHT_EINVAL, "weight_decay must be >= 0 and eps > 0, both finite");
  if (cfg->steps < 1 || cfg->steps > 32) return set_last_error(AHT_EINVAL, "steps must be in 1..32");
  aht_muon* s = new (std::nothrow) aht_muon();
  if (!s) return set_last_error(AHT_ENOMEM, "host allocation failed");
  aht_status e;
  try {
    e = create(n, rows, cols, cfg, static_cast<cudaStream_t>(cuda_stream), s);
  } catch (const std::bad_alloc&) {
    e = set_last_error(AHT_ENOMEM, "host allocation failed");
  }
  if (e != AHT_OK) {
    aht_muon_destroy(s);
    return e;
  }
  *out = s;
  return AHT_OK;
}

void aht_muon_destroy(aht_muon* s) {
  if (!s) return;
  MuonDeviceGuard g(s->device);
  for (void* q : s->owned) cudaFree(q);
  delete s;
}

aht_status aht_muon_step(aht_muon* s, const aht_muon_matrix* mats, int32_t grad_dtype, float lr) {
  if (!s || !mats) return set_last_error(AHT_EINVAL, "NULL argument");
  if (grad_dtype != AHT_FP32 && grad_dtype != AHT_BF16)
    return set_last_error(AHT_EINVAL, "grad_dtype must be AHT_FP32 or AHT_BF16");
  if (!std::isfinite(lr)) return set_last_error(AHT_EINVAL, "lr must be finite");
  Ptrs p{};
  for (size_t k = 0; k < s->mats.size(); ++k) {
    const aht_muon_matrix& q = mats[k];
    if (!q.W || !q.M || !q.G) return set_last_error(AHT_EINVAL, "NULL weights, momentum or gradient");
    if (q.ldw < s->mats[k].cols || q.ldm < s->mats[k].cols || q.ldg < s->mats[k].cols)
      return set_last_error(AHT_EINVAL, "a row stride is below the matrix's columns");
    p.in[k] = q.G;
    p.out[k] = q.W;
    p.mom[k] = q.M;
    p.ld_in[k] = q.ldg;
    p.ld_out[k] = q.ldw;
    p.ld_mom[k] = q.ldm;
  }
  Common c{};
  c.bf16_in = grad_dtype == AHT_BF16;
  c.update = 1;
  c.decay = 1.0f - lr * s->cfg.weight_decay;
  c.lr = lr;
  return run(s, c, p);
}

aht_status aht_muon_orthogonalize(aht_muon* s, const void* const* in, const int32_t* ld_in, void* const* out,
                                  const int32_t* ld_out, int32_t dtype) {
  if (!s || !in || !out || !ld_in || !ld_out) return set_last_error(AHT_EINVAL, "NULL argument");
  if (dtype != AHT_FP32 && dtype != AHT_BF16) return set_last_error(AHT_EINVAL, "dtype must be AHT_FP32 or AHT_BF16");
  Ptrs p{};
  for (size_t k = 0; k < s->mats.size(); ++k) {
    if (!in[k] || !out[k]) return set_last_error(AHT_EINVAL, "NULL matrix");
    if (ld_in[k] < s->mats[k].cols || ld_out[k] < s->mats[k].cols)
      return set_last_error(AHT_EINVAL, "a row stride is below the matrix's columns");
    p.in[k] = in[k];
    p.out[k] = out[k];
    p.ld_in[k] = ld_in[k];
    p.ld_out[k] = ld_out[k];
  }
  Common c{};
  c.bf16_in = c.bf16_out = dtype == AHT_BF16;
  return run(s, c, p);
}

aht_status aht_muon_sync(aht_muon* s) {
  if (!s) return set_last_error(AHT_EINVAL, "NULL argument");
  MuonDeviceGuard g(s->device);
  MUON_CUDA(cudaStreamSynchronize(s->stream));
  uint32_t st = 0;
  MUON_CUDA(cudaMemcpy(&st, s->status, 4, cudaMemcpyDeviceToHost));
  if (st) {
    cudaMemset(s->status, 0, 4);
    return set_last_error(AHT_ETIMEOUT, "a bounded wait of an orthogonalisation product expired");
  }
  return AHT_OK;
}

}  // extern "C"
