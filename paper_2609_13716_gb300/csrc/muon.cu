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
constexpr int kSlots = 6;                      // blocks in flight per CTA
constexpr int kGemmThreads = 320;              // producer, MMA, 8 epilogue warps
constexpr int kEpiThreads = 256;
constexpr float kA = 3.4445f, kBq = -4.7750f, kC = 2.0315f;  // Jordan et al. 2024
constexpr float kSX = 16384.0f, kSA = 16384.0f, kSB = 8192.0f;
constexpr int kNormBlocks = 64;                // partial sums of squares per matrix

struct Mat {
  int32_t rows, cols, m, n, mb, nb, tall;
  int64_t x[2], a, b;                          // byte offsets of the hi blocks
  int64_t x_lo, s_lo;                          // from a hi block to its lo block
};

enum Phase : int { kGram = 0, kPoly = 1, kApply = 2, kLast = 3 };

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
  uint32_t* status;
  int32_t bf16_in, bf16_out, update, nesterov;
  float mu, eps, decay, lr;                    // decay = 1 - lr * weight_decay
};

__device__ __forceinline__ float load_in(const Common& c, const Ptrs& p, int k, int64_t r, int64_t col) {
  const int64_t at = r * p.ld_in[k] + col;
  return c.bf16_in ? __bfloat162float(static_cast<const __nv_bfloat16*>(p.in[k])[at])
                   : static_cast<const float*>(p.in[k])[at];
}

// ---- momentum and the sum of squares of U ------------------------------------------------
__global__ void __launch_bounds__(256) momentum_norm(const __grid_constant__ Common c, const __grid_constant__ Ptrs p) {
  const int k = blockIdx.y;
  const Mat m = c.mats[k];
  const int64_t total = (int64_t)m.rows * m.cols;
  double sum = 0.0;
  for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < total; e += (int64_t)kNormBlocks * 256) {
    const int64_t r = e / m.cols, col = e - r * m.cols;
    float u = load_in(c, p, k, r, col);
    if (c.update) {
      float* mp = p.mom[k] + r * p.ld_mom[k] + col;
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
  __shared__ double sh[kNormBlocks];
  __shared__ float inv_s;
  if (threadIdx.x < kNormBlocks) sh[threadIdx.x] = c.norm[k * kNormBlocks + threadIdx.x];
  __syncthreads();
  if (threadIdx.x == 0) {
    double s = 0.0;
    for (int i = 0; i < kNormBlocks; ++i) s += sh[i];
    inv_s = (float)(1.0 / (sqrt(s) + (double)c.eps));
  }
  __syncthreads();
  const float inv = inv_s;
  uint8_t* x = c.ws + m.x[0];
  for (int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x; q < chunks; q += (int64_t)gridDim.x * 256) {
    const int64_t blk = q >> 11;
    const int r = (int)(q & 127), cb = (int)(q >> 7) & 15;
    const int64_t i = (blk / m.nb) * kB + r, j0 = (blk % m.nb) * kB + 8 * cb;
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int64_t j = j0 + e;
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
    uint8_t* at = x + blk * kBlk + chunk_at(r, cb);
    *reinterpret_cast<uint4*>(at) = hi;
    *reinterpret_cast<uint4*>(at + m.x_lo) = lo;
  }
}

// ---- the products -------------------------------------------------------------------------
// Block (I, k) of a symmetric matrix as an operand with rows I: stored when I <= k, else
// block (k, I) with the other major.
struct Operand {
  const uint8_t* p;    // hi block
  int64_t lo;          // offset of its lo block
  bool mn;             // MN-major
};
__device__ __forceinline__ Operand sym(const uint8_t* s, int64_t lo, int mb, int I, int k) {
  const bool up = I <= k;
  return Operand{s + ((int64_t)(up ? I : k) * mb + (up ? k : I)) * kBlk, lo, !up};
}

template <int kPhase>
__device__ __forceinline__ void operands(const Common& c, const Mat& m, int cur, int I, int J, int k, Operand& A,
                                         Operand& B) {
  const uint8_t* x = c.ws + m.x[cur];
  if (kPhase == kGram) {
    A = Operand{x + ((int64_t)I * m.nb + k) * kBlk, m.x_lo, false};
    B = Operand{x + ((int64_t)J * m.nb + k) * kBlk, m.x_lo, false};
  } else if (kPhase == kPoly) {
    A = sym(c.ws + m.a, m.s_lo, m.mb, I, k);
    B = sym(c.ws + m.a, m.s_lo, m.mb, J, k);
  } else {
    A = sym(c.ws + m.b, m.s_lo, m.mb, I, k);
    B = Operand{x + ((int64_t)k * m.nb + J) * kBlk, m.x_lo, true};
  }
}

__device__ __forceinline__ uint64_t block_desc(uint32_t addr, bool mn) {
  return mn ? tc::smem_desc(addr, 128u, 2048u) : tc::smem_desc(addr, 2048u, 128u);
}

// A persistent kernel over the tiles (matrix, I, J) of a phase.  Warp 0 streams blocks into
// the slots (per k: hi of A, hi of B, lo of B, lo of A; a tile whose operands are the same
// block loads it once), warp 1 issues the MMAs into one of two accumulators, warps 2-9 run
// the epilogue of the other.
template <int kPhase>
__global__ void __launch_bounds__(kGemmThreads, 1)
    product(const __grid_constant__ Common c, const __grid_constant__ Ptrs p, const int4* __restrict__ tiles,
            int n_tiles, int cur) {
  extern __shared__ __align__(1024) uint8_t smem[];
  __shared__ __align__(8) uint64_t full_bar[kSlots], empty_bar[kSlots];
  __shared__ __align__(8) uint64_t accf_bar[2], acce_bar[2], drain_bar;
  __shared__ uint32_t tmem_slot;
  __shared__ volatile int abort_flag;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    for (int s = 0; s < kSlots; ++s) {
      tc::mbar_init(&full_bar[s], 1);
      tc::mbar_init(&empty_bar[s], 1);
    }
    for (int i = 0; i < 2; ++i) {
      tc::mbar_init(&accf_bar[i], 1);
      tc::mbar_init(&acce_bar[i], kEpiThreads);
    }
    tc::mbar_init(&drain_bar, 1);
    tc::mbar_init_fence();
    abort_flag = 0;
  }
  if (warp == 0) tc::tmem_alloc(&tmem_slot, 256);
  tc::fence_before_sync();
  __syncthreads();
  tc::fence_after_sync();
  const uint32_t tmem = tmem_slot;
  int issued = 0;  // (producer) slots filled

  auto wait_or_abort = [&](uint64_t* bar, uint32_t parity) {
    bool ok = false;
    for (int tries = 0; tries < 1000 && !ok && !abort_flag; ++tries) ok = tc::mbar_wait(bar, parity, 2000000ull);
    return ok;
  };
  auto steps = [&](const Mat& m) { return kPhase == kGram ? m.nb : m.mb; };

  if (warp == 0) {
    if (lane == 0) {
      bool ok = true;
      auto fill = [&](const uint8_t* src) {
        const int s = issued % kSlots, use = issued / kSlots;
        if (use > 0 && !(ok = wait_or_abort(&empty_bar[s], (uint32_t)(use - 1) & 1u))) return;
        tc::mbar_expect_tx(&full_bar[s], kBlk);
        tc::bulk_g2s(smem + (size_t)s * kBlk, src, kBlk, &full_bar[s]);
        ++issued;
      };
      for (int t = blockIdx.x; ok && t < n_tiles; t += gridDim.x) {
        const int4 tile = tiles[t];
        const Mat m = c.mats[tile.x];
        const int K = steps(m);
        for (int k = 0; ok && k < K; ++k) {
          Operand A, B;
          operands<kPhase>(c, m, cur, tile.y, tile.z, k, A, B);
          fill(A.p);
          if (A.p == B.p) {
            if (ok) fill(A.p + A.lo);
            continue;
          }
          if (ok) fill(B.p);
          if (ok) fill(B.p + B.lo);
          if (ok) fill(A.p + A.lo);
        }
      }
      if (!ok) abort_flag = 1;
    }
  } else if (warp == 1) {
    if (lane == 0) {
      const uint32_t idesc = (1u << 4) | ((uint32_t)(kB >> 3) << 17) | ((uint32_t)(kB >> 4) << 24);  // fp16 -> fp32
      const uint32_t base = tc::smem_u32(smem);
      int j = 0, taken = 0;
      bool ok = true;
      auto take = [&](uint32_t& addr) {
        const int s = taken % kSlots;
        ok = ok && wait_or_abort(&full_bar[s], (uint32_t)(taken / kSlots) & 1u);
        tc::fence_after_sync();
        addr = base + (uint32_t)s * kBlk;
        ++taken;
        return s;
      };
      for (int t = blockIdx.x; ok && t < n_tiles; t += gridDim.x, ++j) {
        const int4 tile = tiles[t];
        const Mat m = c.mats[tile.x];
        const int K = steps(m), acc = j & 1;
        if (j >= 2 && !(ok = wait_or_abort(&acce_bar[acc], (uint32_t)((j >> 1) - 1) & 1u))) break;
        tc::fence_after_sync();
        const uint32_t D = tmem + (uint32_t)(acc * kB);
        for (int k = 0; ok && k < K; ++k) {
          Operand A, B;
          operands<kPhase>(c, m, cur, tile.y, tile.z, k, A, B);
          const uint32_t id = idesc | (A.mn ? 1u << 15 : 0u) | (B.mn ? 1u << 16 : 0u);
          const uint32_t da = A.mn ? 16u : 256u, db = B.mn ? 16u : 256u;  // 16 of K, in 16-byte units
          auto mma = [&](uint32_t a, uint32_t b, bool first) {
            const uint64_t ad = block_desc(a, A.mn), bd = block_desc(b, B.mn);
#pragma unroll
            for (int kk = 0; kk < kB / 16; ++kk)
              tc::mma_ss(D, ad + (uint64_t)(da * kk), bd + (uint64_t)(db * kk), id, !(first && kk == 0));
          };
          uint32_t a_hi, a_lo, b_hi, b_lo;
          const int s0 = take(a_hi);
          if (A.p == B.p) {
            if (!ok) break;
            mma(a_hi, a_hi, k == 0);
            const int s1 = take(a_lo);
            if (!ok) break;
            mma(a_hi, a_lo, false);
            mma(a_lo, a_hi, false);
            tc::commit(&empty_bar[s0]);
            tc::commit(&empty_bar[s1]);
            continue;
          }
          const int s1 = take(b_hi);
          if (!ok) break;
          mma(a_hi, b_hi, k == 0);
          const int s2 = take(b_lo);
          if (!ok) break;
          mma(a_hi, b_lo, false);
          tc::commit(&empty_bar[s0]);
          tc::commit(&empty_bar[s2]);
          const int s3 = take(a_lo);
          if (!ok) break;
          mma(a_lo, b_hi, false);
          tc::commit(&empty_bar[s1]);
          tc::commit(&empty_bar[s3]);
        }
        if (ok) tc::commit(&accf_bar[acc]);
      }
      if (!ok) abort_flag = 1;
    }
  } else {
    const int q = warp & 3, r = 32 * q + lane;      // row of the tile
    const uint32_t lane_base = (uint32_t)(32 * q) << 16;
    const int c_beg = ((warp - 2) >> 2) * 64;       // this warp's half of the columns
    int j = 0;
    bool ok = true;
    for (int t = blockIdx.x; t < n_tiles; t += gridDim.x, ++j) {
      const int4 tile = tiles[t];
      const Mat m = c.mats[tile.x];
      const int I = tile.y, J = tile.z, acc = j & 1;
      bool got = false;
      if (ok) got = wait_or_abort(&accf_bar[acc], (uint32_t)(j >> 1) & 1u);
      ok = __all_sync(0xFFFFFFFFu, ok && got);      // warp-uniform: tensor-memory loads are collective
      if (!ok) break;
      tc::fence_after_sync();
      for (int c0 = c_beg; c0 < c_beg + 64; c0 += 32) {
        uint32_t v[32];
        tc::ld_x32(tmem + (uint32_t)(acc * kB + c0) + lane_base, v);
        tc::wait_ld();
        if (kPhase == kLast) {
          const int64_t i = (int64_t)I * kB + r, j0 = (int64_t)J * kB + c0;
          if (i >= m.m) continue;
          const float lr = c.update ? c.lr * sqrtf(fmaxf(1.0f, (float)m.rows / (float)m.cols)) : 0.0f;
#pragma unroll
          for (int e = 0; e < 32; ++e) {
            if (j0 + e >= m.n) break;
            const float o = __uint_as_float(v[e]) * (1.0f / (kSB * kSX));
            const int64_t row = m.tall ? j0 + e : i, col = m.tall ? i : j0 + e;
            const int64_t at = row * p.ld_out[tile.x] + col;
            if (c.update) {
              float* w = static_cast<float*>(p.out[tile.x]) + at;
              *w = fmaf(-lr, o, c.decay * *w);
            } else if (c.bf16_out) {
              static_cast<__nv_bfloat16*>(p.out[tile.x])[at] = __float2bfloat16_rn(o);
            } else {
              static_cast<float*>(p.out[tile.x])[at] = o;
            }
          }
          continue;
        }
        const int64_t blk = (kPhase == kApply ? (int64_t)I * m.nb : (int64_t)I * m.mb) + J;
        uint8_t* out = c.ws + (kPhase == kGram ? m.a : kPhase == kPoly ? m.b : m.x[cur ^ 1]) + blk * kBlk;
        const int64_t lo_off = kPhase == kApply ? m.x_lo : m.s_lo;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const int cb = (c0 >> 3) + g;
          float f[8];
          if (kPhase == kPoly) {
            const uint8_t* ap = c.ws + m.a + blk * kBlk + chunk_at(r, cb);
            const uint4 ah = *reinterpret_cast<const uint4*>(ap), al = *reinterpret_cast<const uint4*>(ap + m.s_lo);
            const uint32_t hw[4] = {ah.x, ah.y, ah.z, ah.w}, lw[4] = {al.x, al.y, al.z, al.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float2 h2 = __half22float2(*reinterpret_cast<const __half2*>(&hw[e]));
              const float2 l2 = __half22float2(*reinterpret_cast<const __half2*>(&lw[e]));
              f[2 * e] = h2.x + l2.x;
              f[2 * e + 1] = h2.y + l2.y;
            }
          }
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float d = __uint_as_float(v[8 * g + e]);
            if (kPhase == kGram) f[e] = d * (kSA / (kSX * kSX));
            if (kPhase == kPoly) {
              f[e] = fmaf(d, kC * kSB / (kSA * kSA), f[e] * (kBq * kSB / kSA));
              if (I == J && r == 8 * cb + e) f[e] += kA * kSB;
            }
            if (kPhase == kApply) f[e] = d * (1.0f / kSB);
          }
          uint4 hi, lo;
          split8(f, hi, lo);
          uint8_t* at = out + chunk_at(r, cb);
          *reinterpret_cast<uint4*>(at) = hi;
          *reinterpret_cast<uint4*>(at + lo_off) = lo;
        }
      }
      tc::fence_before_sync();
      tc::mbar_arrive(&acce_bar[acc]);
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
    for (int d = issued - 1; d >= 0 && d >= issued - kSlots; --d)
      tc::mbar_wait(&full_bar[d % kSlots], (uint32_t)(d / kSlots) & 1u);
  }
  tc::fence_before_sync();
  __syncthreads();
  if (warp == 0) {
    tc::fence_after_sync();
    tc::tmem_dealloc(tmem, 256);
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
  int n_sms = 0, n_sym = 0, n_full = 0;
  int norm_chunks = 0;           // CTAs per matrix of normalise
  Mat* d_mats = nullptr;
  int4 *sym_tiles_gram = nullptr, *sym_tiles = nullptr, *full_tiles = nullptr;
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

template <int kPhase>
aht_status run_product(aht_muon* s, const Common& c, const Ptrs& p, const int4* tiles, int n, int cur) {
  product<kPhase><<<std::min(n, s->n_sms), kGemmThreads, kSlots * kBlk, s->stream>>>(c, p, tiles, n, cur);
  MUON_CUDA(cudaGetLastError());
  return AHT_OK;
}

aht_status run(aht_muon* s, Common c, const Ptrs& p) {
  MuonDeviceGuard g(s->device);
  c.mats = s->d_mats;
  c.ws = s->ws;
  c.norm = s->norm;
  c.status = s->status;
  c.eps = s->cfg.eps;
  c.mu = s->cfg.momentum;
  c.nesterov = s->cfg.nesterov;
  const unsigned n = (unsigned)s->mats.size();
  momentum_norm<<<dim3(kNormBlocks, n), 256, 0, s->stream>>>(c, p);
  MUON_CUDA(cudaGetLastError());
  normalise<<<dim3((unsigned)s->norm_chunks, n), 256, 0, s->stream>>>(c, p);
  MUON_CUDA(cudaGetLastError());
  for (int it = 0; it < s->cfg.steps; ++it) {
    const int cur = it & 1;
    if (aht_status e = run_product<kGram>(s, c, p, s->sym_tiles_gram, s->n_sym, cur)) return e;
    if (aht_status e = run_product<kPoly>(s, c, p, s->sym_tiles, s->n_sym, cur)) return e;
    if (it + 1 < s->cfg.steps) {
      if (aht_status e = run_product<kApply>(s, c, p, s->full_tiles, s->n_full, cur)) return e;
    } else {
      if (aht_status e = run_product<kLast>(s, c, p, s->full_tiles, s->n_full, cur)) return e;
    }
  }
  return AHT_OK;
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
  std::vector<int4> sym, full;
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
    most = std::max(most, (int64_t)m.mb * m.nb);
    s->mats.push_back(m);
    for (int I = 0; I < m.mb; ++I) {
      for (int J = I; J < m.mb; ++J) sym.push_back(make_int4(k, I, J, 0));
      for (int J = 0; J < m.nb; ++J) full.push_back(make_int4(k, I, J, 0));
    }
  }
  // the longest tiles first
  std::vector<int4> gram = sym;
  auto by = [&](bool n_side) {
    return [s, n_side](const int4& x, const int4& y) {
      const Mat &a = s->mats[x.x], &b = s->mats[y.x];
      return (n_side ? a.nb : a.mb) > (n_side ? b.nb : b.mb);
    };
  };
  std::stable_sort(gram.begin(), gram.end(), by(true));
  std::stable_sort(sym.begin(), sym.end(), by(false));
  std::stable_sort(full.begin(), full.end(), by(false));
  s->n_sym = (int)sym.size();
  s->n_full = (int)full.size();
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
      !up((void**)&s->sym_tiles_gram, gram.data(), gram.size() * sizeof(int4)) ||
      !up((void**)&s->sym_tiles, sym.data(), sym.size() * sizeof(int4)) ||
      !up((void**)&s->full_tiles, full.data(), full.size() * sizeof(int4)) || !alloc((void**)&s->ws, (size_t)at) ||
      !alloc((void**)&s->norm, (size_t)n * kNormBlocks * sizeof(double)) || !alloc((void**)&s->status, 4) ||
      cudaMemset(s->status, 0, 4) != cudaSuccess)
    return set_last_error(AHT_ENOMEM, "workspace allocation failed");
  const int smem = kSlots * (int)kBlk;
  MUON_CUDA(cudaFuncSetAttribute(product<kGram>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
  MUON_CUDA(cudaFuncSetAttribute(product<kPoly>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
  MUON_CUDA(cudaFuncSetAttribute(product<kApply>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
  MUON_CUDA(cudaFuncSetAttribute(product<kLast>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
  return AHT_OK;
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
