// muon.cu -- orthogonalised updates of weight matrices (include/aht.h states the method):
// momentum, Newton-Schulz orthogonalisation on tensor cores, weight update, for a set of
// matrices at once.
//
// Each matrix is taken with its short side m as rows (a tall one transposed) and padded
// with zeros to whole 128 x 128 blocks.  Of the three products of a step,
//   A = X X^T,   B = a I + b A + c A A,   X' = B X,
// the first two are symmetric: blocks (I, J) with floor(I / 2) <= floor(J / 2) (row pairs on
// or above the diagonal) are computed and stored, and block (J, I) is the same data read with
// the other operand major.
//
// Precision: products accurate to fp32 on 16-bit tensor cores.  An operand is stored as
// hi + lo, two fp16 of it scaled by a power of two (hi the nearest fp16, lo the nearest fp16
// of the rest: 22 significant bits), and a product is hi hi + hi lo + lo hi, accumulated in
// fp32.  fp16 suits the iteration because its operands are bounded: with ||X||_F <= 1 every
// singular value of X stays in [0, 1.21] (the quintic's maximum over [0, 1.21]), so the
// entries of X, S and B stay below 1.21, 1.47 and 3.45 in size, and with the scales 2^14, 2^14 and
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
#include <array>
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
constexpr uint32_t kHalf = kBlk / 2;           // 64 of K of a block
constexpr uint32_t kStage = 3 * kHalf;         // of A: hi, lo; of B: half of hi, half of lo
constexpr int kStages = 4;                     // two units of 128 of K
constexpr int kAcc = 4;                        // accumulators in tensor memory
constexpr int kGemmThreads = 352;              // copies, 8 epilogue warps, 2 that issue products
constexpr int kEpiThreads = 256;
constexpr float kA = 3.4445f, kBq = -4.7750f, kC = 2.0315f;  // Jordan et al. 2024
constexpr float kSX = 16384.0f, kSA = 16384.0f, kSB = 8192.0f;
// The tensor cores round the running sum of a product towards zero.  Over the 12 additions of
// 64 of K, the small products first, that takes about 2e-7 off a result (a step's two last
// products together 3e-7 to 5e-7), always downwards, and five steps multiply a common factor by 7 to
// 11; every product is scaled back by 2 * 2^-23.  Where the short side, which two of the three
// products sum over, ends early, there are fewer additions and half of it is right.  Error of the
// result in 1e-6, Gaussian matrices, scaled by one and by two 2^-23: 8 x 8 0.8 and 1.3, 16 x 16 0.7
// and 1.3, 24 x 96 0.7 and 1.5, 32 x 32 0.8 and 1.1, 40 x 40 1.1 and 1.1, 64 x 256 3.2 and 2.0,
// 128 x 128 3.0 and 1.9, 1024 x 1024 2.7 and 2.0; fp32 products 0.7, 0.8, 1.2, 0.9, 1.0, 1.4, 1.4, 3.1.
constexpr float up(int short_side) { return short_side <= 32 ? 1.0f + 0x1p-23f : 1.0f + 0x1p-22f; }
constexpr float kShift = kBq / (2.0f * kC), kDiag = kA - kBq * kBq / (4.0f * kC);
constexpr int kNormBlocks = 608;               // most partial sums of squares per matrix (one wave)
constexpr int kMaxSteps = 32;
constexpr int kShareK = 4;                     // least blocks of K of an item that two pairs share
constexpr uint32_t kParcel = 32 * kEpiThreads * 4;  // bytes of half a tile in fp32

struct Mat {
  int32_t rows, cols, m, n, mb, nb, tall;
  int32_t norm_blocks;                         // partial sums of squares
  float scale[3];                              // of a phase's accumulated products, up() among it
  int32_t stores[3];                           // a phase's stores of tiles or, where shared, halves of them
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
  float2* inv;                                 // [n_mats] of inverse_norm
  uint32_t* summed;                            // [n_mats] blocks of momentum_norm that are through, 0 between calls
  uint32_t* done;                              // [n_mats][3 phases][kMaxSteps] finished tiles
  uint32_t* status;
  const int4* items;                           // of one step, see Item
  int32_t n_items, steps;
  int32_t paired;                              // clusters are of two pairs, else of one
  int32_t bf16_in, bf16_out, update, nesterov;
  float mu, eps, decay, lr;                    // decay = 1 - lr * weight_decay
  uint64_t wait_ns;                            // limit of a wait
  int32_t expire_mat, expire_step;             // failure hook: this Gram product is awaited in vain (-1: none)
};

__device__ __forceinline__ float load_in(const Common& c, const Ptrs& p, int k, int64_t r, int64_t col) {
  const int64_t at = r * p.ld_in[k] + col;
  return c.bf16_in ? __bfloat162float(static_cast<const __nv_bfloat16*>(p.in[k])[at])
                   : static_cast<const float*>(p.in[k])[at];
}
// Whether groups of four columns of every row of the inputs are aligned loads.
__device__ __forceinline__ bool fours(const Common& c, const Ptrs& p, int k, int cols) {
  uintptr_t low = (uintptr_t)p.in[k] & (c.bf16_in ? 7 : 15);
  int ld = cols | p.ld_in[k];
  if (c.update) {
    low |= (uintptr_t)p.mom[k] & 15;
    ld |= p.ld_mom[k];
  }
  return low == 0 && (ld & 3) == 0;
}
// (An ordinary load: the kernel before may still be writing the input when this one starts, see
// tc::after_previous(), and the read-only path is for data that nobody writes meanwhile.)
__device__ __forceinline__ float4 load_in4(const Common& c, const Ptrs& p, int k, int64_t r, int64_t col) {
  const int64_t at = r * p.ld_in[k] + col;
  if (!c.bf16_in) return *reinterpret_cast<const float4*>(static_cast<const float*>(p.in[k]) + at);
  const uint2 w = *reinterpret_cast<const uint2*>(static_cast<const __nv_bfloat16*>(p.in[k]) + at);
  return make_float4(__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xFFFF0000u), __uint_as_float(w.y << 16),
                     __uint_as_float(w.y & 0xFFFF0000u));
}
// U of an element from the gradient (or matrix) g and the new momentum
__device__ __forceinline__ float u_of(const Common& c, float g, float mom) {
  return !c.update ? g : c.nesterov ? fmaf(c.mu, mom, g) : mom;
}

// Squares of a few values (at most 64) are summed in fp32 and added up in fp64.  Outside of 2^-60 to
// 2^60 their squares would leave fp32's range, or lose bits below it; a group whose largest is there
// is squared in fp64 (slow, so only there).
__device__ __forceinline__ bool fp32_squares(float largest) {
  return largest == 0.0f || (largest >= 0x1p-60f && largest <= 0x1p60f);
}
__device__ __forceinline__ float largest4(float m, float4 v) {
  return fmaxf(fmaxf(m, fmaxf(fabsf(v.x), fabsf(v.y))), fmaxf(fabsf(v.z), fabsf(v.w)));
}
__device__ __forceinline__ double square64(float v) { return (double)v * (double)v; }
__device__ __forceinline__ double squares64(float4 v) {
  return (square64(v.x) + square64(v.y)) + (square64(v.z) + square64(v.w));
}
// kSX / (||U||_F + eps) as a power of two and the rest, x and y with u * x * y in range for every u of
// U: the norm may lie beyond fp32's largest value, and its inverse too.
__device__ __forceinline__ float2 inverse_norm(double sum_sq, float eps) {
  const double d = sqrt(sum_sq) + (double)eps;
  const int e = min(126, max(-126, (__double2hiint(d) >> 20 & 0x7FF) - 1023));
  const float x = __int_as_float((127 - e) << 23);
  return make_float2(x, (float)(1.0 / (d * (double)x)) * kSX);
}

// ---- momentum and the sum of squares of U ------------------------------------------------
// Also clears the tile counters of the call.  A thread takes four groups of four columns at a
// time (their loads in flight together) where the rows allow it, else single elements.  Bound by
// memory latency: 2048 x 4096, bf16 gradient, 20 us from a cold cache, 84 MB.
__global__ void __launch_bounds__(256) momentum_norm(const __grid_constant__ Common c, const __grid_constant__ Ptrs p) {
  tc::after_previous();
  const int k = blockIdx.y;
  const Mat& m = c.mats[k];
  const int blocks = m.norm_blocks;
  if ((int)blockIdx.x >= blocks) return;
  if (blockIdx.x == 0 && threadIdx.x < 3 * kMaxSteps) c.done[k * 3 * kMaxSteps + threadIdx.x] = 0;
  const uint32_t rows = m.rows, cols = m.cols;  // rows * cols is at most 2^28
  double sum = 0.0;
  if (fours(c, p, k, cols)) {
    const uint32_t c4 = cols / 4, total = rows * c4;
    for (uint32_t e0 = blockIdx.x * 1024 + threadIdx.x; e0 < total; e0 += blocks * 1024) {
      float4 g[4], o[4];
      float* mp[4];
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const uint32_t e = e0 + 256 * x;
        g[x] = o[x] = make_float4(0.f, 0.f, 0.f, 0.f);
        mp[x] = nullptr;
        if (e < total) {
          const uint32_t r = e / c4, col = 4 * (e - r * c4);
          g[x] = load_in4(c, p, k, r, col);
          if (c.update) {
            mp[x] = p.mom[k] + (int64_t)r * p.ld_mom[k] + col;
            o[x] = *reinterpret_cast<const float4*>(mp[x]);
          }
        }
      }
      float part = 0.0f, largest = 0.0f;       // 16 squares in fp32, the rest in fp64
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        if (mp[x]) {
          o[x] = make_float4(fmaf(c.mu, o[x].x, g[x].x), fmaf(c.mu, o[x].y, g[x].y), fmaf(c.mu, o[x].z, g[x].z),
                             fmaf(c.mu, o[x].w, g[x].w));
          *reinterpret_cast<float4*>(mp[x]) = o[x];
        }
        g[x] = make_float4(u_of(c, g[x].x, o[x].x), u_of(c, g[x].y, o[x].y), u_of(c, g[x].z, o[x].z),
                           u_of(c, g[x].w, o[x].w));
        part += (g[x].x * g[x].x + g[x].y * g[x].y) + (g[x].z * g[x].z + g[x].w * g[x].w);
        largest = largest4(largest, g[x]);
      }
      if (fp32_squares(largest)) {
        sum += part;
      } else {
#pragma unroll
        for (int x = 0; x < 4; ++x) sum += squares64(g[x]);
      }
    }
  } else {
    const uint32_t total = rows * cols;
    float part = 0.0f;
    int held = 0;
    for (uint32_t e = blockIdx.x * 256 + threadIdx.x; e < total; e += blocks * 256) {
      const uint32_t r = e / cols, col = e - r * cols;
      const float g = load_in(c, p, k, r, col);
      float mom = 0.0f;
      if (c.update) {
        float* mp = p.mom[k] + (int64_t)r * p.ld_mom[k] + col;
        mom = fmaf(c.mu, *mp, g);
        *mp = mom;
      }
      const float u = u_of(c, g, mom);
      if (fp32_squares(fabsf(u))) part += u * u;
      else sum += square64(u);
      if (++held == 16) {
        sum += part;
        part = 0.0f;
        held = 0;
      }
    }
    sum += part;
  }
  __shared__ double sh[256];
  __shared__ bool last;
  auto block_sum = [&](double v) {             // at thread 0
    sh[threadIdx.x] = v;
    for (int s = 128; s > 0; s >>= 1) {
      __syncthreads();
      if (threadIdx.x < s) sh[threadIdx.x] += sh[threadIdx.x + s];
    }
    return sh[0];
  };
  sum = block_sum(sum);
  if (threadIdx.x == 0) {
    c.norm[k * kNormBlocks + blockIdx.x] = sum;
    __threadfence();
    last = atomicAdd(&c.summed[k], 1u) == (uint32_t)blocks - 1;
  }
  __syncthreads();
  if (!last) return;
  // the last block adds the sums, in their order, and divides once (64-bit additions and divisions
  // are slow: with them in every block of normalise it took 30 us for 2048 x 4096, now 18)
  __threadfence();
  double all = 0.0;
  for (int i = threadIdx.x; i < blocks; i += 256) all += __ldcg(&c.norm[k * kNormBlocks + i]);
  all = block_sum(all);
  if (threadIdx.x == 0) {
    c.inv[k] = inverse_norm(all, c.eps);
    c.summed[k] = 0;
  }
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
// One thread per 8-column chunk of a row of X.  A warp takes 8 rows x 4 chunks of a wide matrix, so
// that it reads and writes runs of 128 bytes (an update of the two S5 heads 263 us; 32 rows of a
// chunk each 275), and 32 rows of a tall one, whose rows are the caller's columns.
__global__ void __launch_bounds__(256) normalise(const __grid_constant__ Common c, const __grid_constant__ Ptrs p) {
  tc::after_previous();
  const int k = blockIdx.y;
  const Mat m = c.mats[k];
  const int64_t chunks = (int64_t)m.mb * m.nb * 2048;
  if ((int64_t)blockIdx.x * 256 >= chunks) return;
  const float2 inv = c.inv[k];
  uint8_t* x = c.ws + m.x[0];
  const bool four = !m.tall && fours(c, p, k, m.cols);
  for (int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x; q < chunks; q += (int64_t)gridDim.x * 256) {
    const int blk = (int)(q >> 11);
    const int z = (int)q & 2047;
    const int r = m.tall ? z & 127 : (z & 7) | (z >> 2 & 0x78);
    const int cb = m.tall ? z >> 7 : (z >> 3 & 3) | (z >> 7 & 12);
    const int bi = blk / m.nb, i = bi * kB + r, j0 = (blk - bi * m.nb) * kB + 8 * cb;
    float v[8];
    if (four && i < m.m && j0 + 8 <= m.n) {
      const float4 g0 = load_in4(c, p, k, i, j0), g1 = load_in4(c, p, k, i, j0 + 4);
      float4 o0 = g0, o1 = g1;
      if (c.update) {
        const float4* mp = reinterpret_cast<const float4*>(p.mom[k] + (int64_t)i * p.ld_mom[k] + j0);
        o0 = mp[0];
        o1 = mp[1];
      }
      const float g[8] = {g0.x, g0.y, g0.z, g0.w, g1.x, g1.y, g1.z, g1.w};
      const float o[8] = {o0.x, o0.y, o0.z, o0.w, o1.x, o1.y, o1.z, o1.w};
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = (u_of(c, g[e], o[e]) * inv.x) * inv.y;
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int j = j0 + e;
        v[e] = 0.0f;
        if (i < m.m && j < m.n) {
          const int64_t row = m.tall ? j : i, col = m.tall ? i : j;
          const float mom = c.update ? p.mom[k][row * p.ld_mom[k] + col] : 0.0f;
          v[e] = (u_of(c, load_in(c, p, k, row, col), mom) * inv.x) * inv.y;
        }
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
// Boxes of the workspace seen as [blocks * 16 column groups][16 row groups][64 fp16]: 64
// columns of 128 rows, 64 rows of 128 columns, 64 columns of 64 rows.
struct Maps {
  CUtensorMap cols, rows, quarter;
};

// Where a lane finds its operand's block for k: from k = turn on it is K-major, blocks in a
// row (first + k); before, it is MN-major, blocks in a column (column + k * stride).  Block
// (I, k) of a symmetric matrix is stored when floor(I / 2) <= floor(k / 2), else it is block
// (k, I) with the other major; the halves make both rows of a pair take the same major, which
// one product instruction needs.
struct Operand {
  int32_t first, column, stride, turn;
  __device__ __forceinline__ bool mn(int k) const { return k < turn; }
  __device__ __forceinline__ int block(int k) const { return mn(k) ? column + k * stride : first + k; }
};
__device__ __forceinline__ Operand operand(int phase, const Mat& m, int cur, bool of_a, bool lo, int I, int J) {
  const int row = of_a ? I : J;
  if (phase == kGram || (phase == kApply && !of_a)) {
    const int x = (int)(((cur ? m.x[1] : m.x[0]) + (lo ? m.x_lo : 0)) / kBlk);
    return Operand{x + row * m.nb, x + J, m.nb, phase == kGram ? 0 : 0x7FFFFFFF};
  }
  const int s = (int)(((phase == kPoly ? m.a : m.b) + (lo ? m.s_lo : 0)) / kBlk);
  return Operand{s + row * m.mb, s + row, m.mb, row & ~1};
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

// An entry of the list of a step's work: (matrix or -1, phase | 4 * part, row pair, J).  Part 0 is all
// of K, 1 and 2 its halves, the parts of the two pairs of a cluster.
struct Item {
  int mat, phase, part, I2, J, it;
};
__device__ __forceinline__ Item item_at(const Common& c, int g) {
  const int it = g / c.n_items;
  const int4 v = c.items[g - it * c.n_items];
  return Item{v.x, v.y & 3, v.y >> 2, v.z, v.w, it};
}
__device__ __forceinline__ int first_k(int part, int K) { return part == 2 ? (K + 1) / 2 : 0; }
__device__ __forceinline__ int end_k(int part, int K) { return part == 1 ? (K + 1) / 2 : K; }

// ---- pairs of CTAs, two in a cluster ----
__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release;\nbarrier.cluster.wait.acquire;" ::: "memory");
}
// The address of a shared object of this CTA in another of the cluster.
__device__ __forceinline__ uint32_t peer_addr(const void* p, int rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(tc::smem_u32(p)), "r"(rank));
  return r;
}
// (cta-scope release: what is handed over is tensor memory, ordered by the tcgen05 fence before
// it; a cluster-scope release waits for the thread's stores, 600 clocks an arrival.)
__device__ __forceinline__ void arrive_at(uint32_t mbar) {
  asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(mbar) : "memory");
}
// The same where reads of shared memory have to be complete before the other side writes there.
__device__ __forceinline__ void arrive_cluster(uint32_t mbar) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(mbar) : "memory");
}
// Sixteen bytes into another CTA of the cluster, counted on a barrier there.
__device__ __forceinline__ void send16(uint32_t to, float4 v, uint32_t mbar) {
  asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v4.b32 [%0], {%1, %2, %3, %4}, [%5];" ::"r"(to),
               "r"(__float_as_uint(v.x)), "r"(__float_as_uint(v.y)), "r"(__float_as_uint(v.z)), "r"(__float_as_uint(v.w)),
               "r"(mbar)
               : "memory");
}
// A box of the workspace into this CTA's shared memory, counted on a barrier of either CTA.
__device__ __forceinline__ void box_g2s(void* dst, const CUtensorMap* map, int row_group, int col_group, uint32_t mbar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], "
      "[%5];" ::"r"(tc::smem_u32(dst)),
      "l"(map), "r"(0), "r"(row_group), "r"(col_group), "r"(mbar)
      : "memory");
}
// D[both CTAs] (+)= A B^T, M = 256 (128 rows of each CTA), N = 128 (64 columns of each CTA).
__device__ __forceinline__ void mma_pair(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\n"
      "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}\n" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(accumulate));
}
// The products issued so far arrive on a barrier of the CTAs of a mask (a pair) when they are complete.
__device__ __forceinline__ void commit_pair(uint64_t* mbar, uint16_t ctas) {
  asm volatile(
      "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(
          tc::smem_u32(mbar)),
      "h"(ctas)
      : "memory");
}

// A 32 x 32 block held as a row a lane (v[e]: column e) becomes a column a lane (v[e]: row e).
__device__ __forceinline__ void transpose32(float* v, int lane) {
#pragma unroll
  for (int s = 16; s > 0; s >>= 1)
#pragma unroll
    for (int e = 0; e < 32; ++e) {
      if (e & s) continue;
      const bool up = lane & s;
      const float got = __shfl_xor_sync(0xFFFFFFFFu, up ? v[e] : v[e + s], s);
      if (up) v[e] = got;
      else v[e + s] = got;
    }
}

// W columns j0.. of 32 rows i0.. of the orthogonal factor, a row a lane (the accumulated
// product f, unscaled), into the caller's matrix: the weight update, or the factor itself.  A wide
// fp32 matrix whose rows allow it takes groups of four columns; a tall one is stored transposed,
// so its lanes write neighbours; any other wide one is turned first (a block of 130 x 777 bf16
// 3 us, a lane writing its row 9; turned fp32 rows 1 us a tile more than groups of four).
// Sixteen elements at a time: their loads are in flight together.
template <int W>
__device__ __forceinline__ void store_result(const Common& c, const Ptrs& p, int k, const Mat& m, int i0, int lane, int j0,
                                             float (&f)[W]) {
  const float lr = c.update ? c.lr * sqrtf(fmaxf(1.0f, (float)m.rows / (float)m.cols)) : 0.0f;
  const int64_t ld = p.ld_out[k];
  void* out = p.out[k];
  if (!m.tall && j0 + W <= m.n && !c.bf16_out && ((uintptr_t)out & 15) == 0 && (ld & 3) == 0) {
    if (i0 + lane >= m.m) return;
    float4* w = reinterpret_cast<float4*>(static_cast<float*>(out) + (int64_t)(i0 + lane) * ld + j0);
#pragma unroll
    for (int b = 0; b < W / 4; b += 4) {
      float4 o[4], old[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float* v = f + 4 * (b + e);
        const float s = m.scale[kApply] / kSX;
        o[e] = make_float4(v[0] * s, v[1] * s, v[2] * s, v[3] * s);
        if (c.update) old[e] = w[b + e];
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (c.update)
          o[e] = make_float4(fmaf(-lr, o[e].x, c.decay * old[e].x), fmaf(-lr, o[e].y, c.decay * old[e].y),
                             fmaf(-lr, o[e].z, c.decay * old[e].z), fmaf(-lr, o[e].w, c.decay * old[e].w));
        w[b + e] = o[e];
      }
    }
    return;
  }
#pragma unroll
  for (int b = 0; b < W; b += 32) {
    if (!m.tall) transpose32(f + b, lane);
    // element e of this lane: row i0 + e, column j0 + b + lane; tall: row i0 + lane, column j0 + b + e
    const int lane_at = m.tall ? i0 + lane : j0 + b + lane, lane_end = m.tall ? m.m : m.n;
    const int e_at = m.tall ? j0 + b : i0, e_end = m.tall ? m.n : m.m;
    if (lane_at >= lane_end) continue;
    // X (i, j) is element (j, i) of a tall matrix, (i, j) of a wide one: e runs over rows of the matrix
    const int64_t at0 = (int64_t)e_at * ld + lane_at;
#pragma unroll
    for (int h = 0; h < 32; h += 16) {
      const int left = e_end - e_at - h;
      const int64_t at = at0 + h * ld;
      float o[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) o[e] = f[b + h + e] * (m.scale[kApply] / kSX);
      if (c.update) {
        float* w = static_cast<float*>(out) + at;
        float old[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) old[e] = e < left ? w[e * ld] : 0.0f;
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (e < left) w[e * ld] = fmaf(-lr, o[e], c.decay * old[e]);
      } else if (c.bf16_out) {
        __nv_bfloat16* w = static_cast<__nv_bfloat16*>(out) + at;
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (e < left) w[e * ld] = __float2bfloat16_rn(o[e]);
      } else {
        float* w = static_cast<float*>(out) + at;
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (e < left) w[e * ld] = o[e];
      }
    }
  }
}

// One persistent cooperative kernel of CTA pairs runs every product of the call: the items
// (step, phase, matrix, row pair, J) in that order, item g on pair g mod pairs; an item is the
// 128 x 128 tiles (I, J) and (I + 1, J), one per CTA.  An item begins when the tiles that it
// reads are complete (counters per matrix, phase and step), so matrices advance independently
// and a pair without work in one matrix's phase goes on with another's.  An item only waits
// for earlier ones and all CTAs are resident, so the earliest unfinished item always runs.
//
// Why pairs: a 128 x 128 product of one CTA reads its operands from shared memory at 128 B
// per clock, all there is, and the copies that refill it (85 B per clock) took 40 % of the
// tensor cores' time.  A pair's product reads the A rows of each CTA and half of B from each,
// 96 B per clock, and refills 64.
//
// Warp 0 streams stages of 64 of K; four lanes issue a copy each, since a lane needs about
// 240 clocks per copy and a stage is 768 clocks of products.  Both CTAs' copies count on
// CTA 0's barrier.  Warps 1 and 10 of CTA 0 issue the products of units of 128 of K in turn,
// the small ones first, 64 of K into one of four accumulators.  Warps 2-9 add each accumulator
// to fp32 registers (the tensor core rounds its running sum towards zero: summed over all of K
// the bias of a 1024-wide product showed as 2e-5 of the result, 128 at a time as 6e-6, 64 at a
// time as 3e-6, fp32 products have 2.6e-6) and run the tile's epilogue.
//
// A phase of few items leaves pairs idle while each item's sum over K runs (1 us per 128).  Where
// no phase has more items than pairs, clusters are of two pairs and share the items with long
// sums: each sums half of K, then sends half of its columns to the other, adds what it receives
// and finishes its half (the exchange costs 1.1 us: 1024 x 1024, 8 blocks of K, 31 us of 183 less; three
// of 130 x 777, where one product of three is shared, 8 of 125).
__global__ void __launch_bounds__(kGemmThreads, 1)
    products(const __grid_constant__ Common c, const __grid_constant__ Ptrs p, const __grid_constant__ Maps maps) {
  extern __shared__ __align__(1024) uint8_t smem[];
  __shared__ __align__(8) uint64_t full_bar[kStages], empty_bar[kStages];
  __shared__ __align__(8) uint64_t accf_bar[kAcc], acce_bar[kAcc], drain_bar, parcel_bar, read_bar, never_bar;
  __shared__ uint32_t tmem_slot;
  __shared__ volatile int abort_flag;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int in_cluster = (int)cluster_rank(), rank = in_cluster & 1, leader = in_cluster & ~1;
  const int pair = (int)blockIdx.x >> 1, pairs = (int)gridDim.x >> 1;
  if (tid == 0) {
    for (int s = 0; s < kStages; ++s) {
      tc::mbar_init(&empty_bar[s], 1);
      tc::mbar_init(&full_bar[s], 1);
    }
    for (int i = 0; i < kAcc; ++i) {
      tc::mbar_init(&accf_bar[i], 1);
      tc::mbar_init(&acce_bar[i], 2 * kEpiThreads / 32);  // a lane of every epilogue warp of the pair
    }
    tc::mbar_init(&drain_bar, 2);
    tc::mbar_init(&parcel_bar, 1);
    tc::mbar_init(&read_bar, 1);
    tc::mbar_init(&never_bar, 1);
    tc::mbar_init_fence();
    abort_flag = 0;
  }
  if (warp == 0) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(tc::smem_u32(&tmem_slot)));
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
  }
  tc::fence_before_sync();
  __syncthreads();
  cluster_sync();
  tc::fence_after_sync();
  const uint32_t tmem = tmem_slot;
  int issued = 0;  // (producer) stages filled
  uint32_t sent = 0;  // (epilogue) halves of tiles exchanged
  const int n_all = c.n_items * c.steps;

  auto wait_or_abort = [&](uint64_t* bar, uint32_t parity) {
    if (tc::mbar_try_wait(bar, parity)) return true;
    const uint64_t t0 = tc::globaltimer_ns();
    for (int tries = 0; tries < 1000 && !abort_flag; ++tries) {
      if (tc::mbar_wait(bar, parity, min((uint64_t)2000000, c.wait_ns))) return true;
      if (tc::globaltimer_ns() - t0 > c.wait_ns) break;
    }
    return false;
  };
  auto wait_warp = [&](uint64_t* bar, uint32_t parity) {  // by a whole warp, which goes on or gives up together
    return (bool)__all_sync(0xFFFFFFFFu, wait_or_abort(bar, parity));
  };
  // the tiles an item reads are complete (bounded wait)
  auto ready = [&](const Mat& m, int k, int phase, int it) {
    if (phase == kGram && it == 0) return true;
    const int from = phase == kGram ? kApply : phase - 1;
    const uint32_t want = (uint32_t)(from == kGram ? m.stores[kGram] : from == kPoly ? m.stores[kPoly] : m.stores[kApply]);
    const uint32_t* at = c.done + (k * 3 + from) * kMaxSteps + (phase == kGram ? it - 1 : it);
    if (ld_acquire(at) >= want) return true;
    const uint64_t t0 = tc::globaltimer_ns();
    for (uint32_t i = 0; i < (1u << 30) && !abort_flag; ++i) {
      if (ld_acquire(at) >= want) return true;
      if ((i & 63u) == 63u && tc::globaltimer_ns() - t0 > c.wait_ns) return false;
    }
    return false;
  };

  if (warp == 0) {
    if (lane < 4) {
      // lane 0: hi of A, 1: lo of A, 2: this CTA's half of B's hi, 3: of its lo
      const bool of_a = lane < 2, lo = lane & 1;
      uint8_t* dst0 = smem + (of_a ? lane * kHalf : 2 * kHalf + (lane - 2) * (kHalf / 2));
      if (lane < 3)
        asm volatile("prefetch.tensormap [%0];" ::"l"(lane == 0 ? &maps.cols : lane == 1 ? &maps.rows : &maps.quarter)
                     : "memory");
      const uint32_t full0 = peer_addr(&full_bar[0], leader);
      const int half0 = of_a ? 0 : 8 * rank;      // this CTA's half of B's rows
      bool ok = true;
      int s = 0;
      uint32_t par = 1;                           // of the release awaited (the first pass waits for none)
      for (int g = pair; ok && g < n_all; g += pairs) {
        const Item t = item_at(c, g);
        if (t.mat < 0) continue;
        const Mat m = c.mats[t.mat];
        const int I = min(2 * t.I2 + rank, m.mb - 1);  // (an odd last row is computed twice, stored once)
        const int K = t.phase == kGram ? m.nb : m.mb;
        const Operand o = operand(t.phase, m, t.it & 1, of_a, lo, I, t.J);
        if (!(ok = ready(m, t.mat, t.phase, t.it))) break;
        fence_proxy_global();
        for (int k = first_k(t.part, K), k_end = end_k(t.part, K); ok && k < k_end; ++k) {
          const bool mn = o.mn(k);
          const int col0 = o.block(k) * 16 + (mn ? half0 : 0);
          const CUtensorMap* map = !of_a ? &maps.quarter : mn ? &maps.rows : &maps.cols;
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            if (issued >= kStages && !(ok = wait_or_abort(&empty_bar[s + h], par))) break;
            if (lane == 0 && rank == 0) tc::mbar_expect_tx(&full_bar[s + h], 2 * kStage);
            box_g2s(dst0 + (s + h) * kStage, map, mn ? 8 * h : half0, mn ? col0 : col0 + 8 * h, full0 + (s + h) * 8);
            ++issued;
          }
          if ((s ^= 2) == 0) par ^= 1u;
        }
      }
      // the last stages' releases have landed before this CTA can leave
      for (int d = max(0, issued - kStages); ok && d < issued; ++d)
        ok = wait_or_abort(&empty_bar[d % kStages], (uint32_t)(d / kStages) & 1u);
      if (!ok) abort_flag = 1;
    }
  } else if (warp == 1 || warp == 10) {
    // The tensor cores queue few products, so whatever a warp does between two of them shows
    // (a satisfied wait costs 185 clocks, a unit of 128 of K is 1536 clocks of products): two
    // warps take the units in turn, one waiting while the other's products run, in
    // warp-uniform loops with one elected lane.
    if (rank == 0) {
      const uint32_t idesc = (1u << 4) | ((uint32_t)(kB >> 3) << 17) | ((uint32_t)(2 * kB >> 4) << 24);  // fp16 -> fp32
      const uint32_t base = tc::smem_u32(smem);
      const bool one = tc::elect_one();
      const uint16_t both = (uint16_t)(3u << leader);
      int j = 0;
      bool ok = true;
      for (int g = pair; ok && g < n_all; g += pairs) {
        const Item t = item_at(c, g);
        if (t.mat < 0) continue;
        const int K = t.phase == kGram ? c.mats[t.mat].nb : c.mats[t.mat].mb;
        for (int k = first_k(t.part, K), k_end = end_k(t.part, K); ok && k < k_end; ++k, ++j) {
          if ((j & 1) != (warp == 10)) continue;
          // the majors of operand()
          const bool a_mn = t.phase != kGram && k < 2 * t.I2;
          const bool b_mn = t.phase == kApply || (t.phase == kPoly && k < (t.J & ~1));
          const uint32_t id = idesc | (a_mn ? 1u << 15 : 0u) | (b_mn ? 1u << 16 : 0u);
          const uint32_t da = a_mn ? 16u : 256u, db = b_mn ? 16u : 128u;  // 16 of K, in 16-byte units
          const int s = 2 * (j & 1);                // stages and accumulators s and s + 1
          const uint32_t par = (uint32_t)(j >> 1) & 1u;
          auto a_desc = [&](uint32_t x) { return a_mn ? tc::smem_desc(x, 128u, 1024u) : tc::smem_desc(x, 2048u, 128u); };
          auto b_desc = [&](uint32_t x) { return b_mn ? tc::smem_desc(x, 128u, 1024u) : tc::smem_desc(x, 1024u, 128u); };
          const uint64_t a0 = a_desc(base + (uint32_t)s * kStage), b0 = b_desc(base + (uint32_t)s * kStage + 2 * kHalf);
          constexpr uint64_t kLoA = kHalf / 16, kLoB = kHalf / 32, kNext = kStage / 16;
          // An item's first products start on half a unit; later units are waited for whole,
          // under the other warp's products.
          const bool first = k == first_k(t.part, K);
          if (!(ok = wait_warp(&full_bar[s], par))) break;
          if (!first && !(ok = wait_warp(&full_bar[s + 1], par))) break;
#pragma unroll
          for (int h = 0; ok && h < 2; ++h) {
            if (first && h == 1 && !(ok = wait_warp(&full_bar[s + 1], par))) break;
            if (j >= 2 && !(ok = wait_warp(&acce_bar[s + h], par ^ 1u))) break;
            tc::fence_after_sync();
            if (one) {
              const uint32_t D = tmem + (uint32_t)((s + h) * kB);
              const uint64_t a = a0 + h * kNext, b = b0 + h * kNext;
              auto mma = [&](uint64_t x, uint64_t y, bool first) {
#pragma unroll
                for (int kk = 0; kk < 4; ++kk)
                  mma_pair(D, x + (uint64_t)(da * kk), y + (uint64_t)(db * kk), id, !(first && kk == 0));
              };
              mma(a, b + kLoB, true);
              mma(a + kLoA, b, false);
              mma(a, b, false);
              commit_pair(&empty_bar[s + h], both);
              commit_pair(&accf_bar[s + h], both);
            }
            __syncwarp();
          }
        }
      }
      if (!ok) abort_flag = 1;
    }
  } else {
    const int q = warp & 3, r = 32 * q + lane;      // row of the tile
    const uint32_t lane_base = (uint32_t)(32 * q) << 16;
    const int c_beg = ((warp - 2) >> 2) * 64;       // this warp's half of the columns
    const uint32_t acce0 = peer_addr(&acce_bar[0], leader);
    // shared items: the halves of a tile that the CTAs of the same rank of the two pairs exchange
    const int other = c.paired ? in_cluster ^ 2 : in_cluster, side = in_cluster >> 1;
    const uint8_t* parcel = smem + kStages * kStage + (tid - 64) * 16;
    const uint32_t to = peer_addr(parcel, other), to_bar = peer_addr(&parcel_bar, other), read = peer_addr(&read_bar, other);
    int j = 0;
    bool ok = true;
    for (int g = pair; g < n_all; g += pairs) {
      const Item t = item_at(c, g);
      if (t.mat < 0) continue;
      const Mat& m = c.mats[t.mat];
      const int phase = t.phase, I = 2 * t.I2 + rank, J = t.J, K = phase == kGram ? m.nb : m.mb;
      const bool mine = I < m.mb;                   // (of an odd last row: nothing to store)
      const int64_t blk = (phase == kApply ? (int64_t)I * m.nb : (int64_t)I * m.mb) + J;
      uint8_t* out = c.ws + (phase == kGram ? m.a : phase == kPoly ? m.b : t.it & 1 ? m.x[0] : m.x[1]) + blk * kBlk;
      const int64_t lo_off = phase == kApply ? m.x_lo : m.s_lo;
      const float scale = m.scale[phase];
      const float diag = phase == kApply || I != J ? 0.0f : phase == kGram ? kShift * kSA : kDiag * kSB;
      const bool last = phase == kApply && t.it + 1 == c.steps;
      // the columns c_at.. of row r, complete: to the workspace or, after the last step, the caller
      auto finish = [&](auto& v, int c_at) {
        constexpr int W = sizeof(v) / sizeof(float);
        if (last) {
          store_result<W>(c, p, t.mat, m, I * kB + 32 * q, lane, J * kB + c_at, v);
          return;
        }
        uint8_t* hi_at = out + chunk_at(r, c_at >> 3);
#pragma unroll
        for (int x = 0; x < W / 8; ++x) {
#pragma unroll
          for (int e = 0; e < 8; ++e) v[8 * x + e] *= scale;
          if (diag != 0.0f) {  // (the tile's row r is its column r)
#pragma unroll
            for (int e = 0; e < 8; ++e) v[8 * x + e] += r == c_at + 8 * x + e ? diag : 0.0f;
          }
          uint4 hi, lo;
          split8(v + 8 * x, hi, lo);
          uint8_t* at = hi_at + x * 2048;  // the next group of 8 columns
          *reinterpret_cast<uint4*>(at) = hi;
          *reinterpret_cast<uint4*>(at + lo_off) = lo;
        }
      };
      float f[64];
#pragma unroll
      for (int e = 0; e < 64; ++e) f[e] = 0.0f;
      if (t.mat == c.expire_mat && phase == kGram && t.it == c.expire_step) ok = wait_warp(&never_bar, 0);
      for (int k = 2 * first_k(t.part, K), k_end = 2 * end_k(t.part, K); ok && k < k_end; ++k, ++j) {
        const int acc = j % kAcc;
        // warp-uniform: tensor-memory loads are collective
        if (!(ok = wait_warp(&accf_bar[acc], (uint32_t)(j / kAcc) & 1u))) break;
        tc::fence_after_sync();
        if (mine) {
#pragma unroll
          for (int c0 = 0; c0 < 64; c0 += 32) {
            uint32_t v[32];
            tc::ld_x32(tmem + (uint32_t)(acc * kB + c_beg + c0) + lane_base, v);
            tc::wait_ld();
#pragma unroll
            for (int e = 0; e < 32; ++e) f[c0 + e] += __uint_as_float(v[e]);
          }
        }
        tc::fence_before_sync();
        __syncwarp();
        if (lane == 0) arrive_at(acce0 + (uint32_t)acc * 8u);
      }
      if (mine && t.part == 0) {
        if (ok) finish(f, c_beg);
      } else if (mine) {
        // Each CTA keeps 32 of the thread's columns and sends the others.
        if (tid == 64) tc::mbar_expect_tx(&parcel_bar, kParcel);
        if (ok && sent > 0) ok = wait_warp(&read_bar, (sent - 1) & 1u);
        float own[32];
        if (ok) {
#pragma unroll
          for (int x = 0; x < 8; ++x) {
            float4 o;
            o.x = side ? f[4 * x] : f[32 + 4 * x];
            o.y = side ? f[4 * x + 1] : f[33 + 4 * x];
            o.z = side ? f[4 * x + 2] : f[34 + 4 * x];
            o.w = side ? f[4 * x + 3] : f[35 + 4 * x];
            send16(to + (uint32_t)x * kEpiThreads * 16u, o, to_bar);
          }
#pragma unroll
          for (int e = 0; e < 32; ++e) own[e] = side ? f[32 + e] : f[e];
          ok = wait_warp(&parcel_bar, sent & 1u);
        }
        ++sent;
        if (ok) {
#pragma unroll
          for (int x = 0; x < 8; ++x) {
            const float4 o = *reinterpret_cast<const float4*>(parcel + x * kEpiThreads * 16);
            own[4 * x] += o.x;
            own[4 * x + 1] += o.y;
            own[4 * x + 2] += o.z;
            own[4 * x + 3] += o.w;
          }
          finish(own, c_beg + 32 * side);
        }
      }
      // all eight warps leave together: none is left at the barrier
      ok = !tc::bar_or(1, kEpiThreads, !ok);
      if (!ok) break;
      if (!last && mine && tid == 64) {  // the barrier ordered the tile's stores before these
        fence_proxy_global();
        add_release(c.done + (t.mat * 3 + phase) * kMaxSteps + t.it);
      }
      if (t.part != 0 && mine && tid == 96) arrive_cluster(read);  // (all eight warps have read theirs)
    }
    if (!ok) abort_flag = 1;
  }

  // the products and copies of the pair complete (bounded), then tensor memory is freed
  tc::fence_before_sync();
  __syncthreads();
  if (tid == 0 && abort_flag) atomicOr(c.status, kStatusTimeout);
  if ((warp == 1 || warp == 10) && rank == 0) {
    if (tc::elect_one())  // the lane that issued this warp's products
      asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(
                       tc::smem_u32(&drain_bar))
                   : "memory");
    __syncwarp();
    tc::mbar_wait(&drain_bar, 0);
  }
  if (warp == 0 && lane == 0 && rank == 0 && abort_flag) {
    for (int d = max(0, issued - kStages); d < issued; ++d)  // (a stage that was not filled never completes)
      tc::mbar_wait(&full_bar[d % kStages], (uint32_t)(d / kStages) & 1u, 10000000ull);
  }
  tc::fence_before_sync();
  __syncthreads();
  cluster_sync();
  if (warp == 2 && abort_flag) {  // what the other pair sent lands before this CTA leaves (bounded)
    tc::mbar_wait(&parcel_bar, (sent - 1) & 1u, 1000000ull);
    tc::mbar_wait(&parcel_bar, sent & 1u, 1000000ull);
  }
  if (warp == 0) {
    tc::fence_after_sync();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem));
  }
}

// ---- matrices of at most 128 rows (short side), whole on chip -----------------------------
// Between the phases of such a matrix products() spends 5 us on counters, fences and copies
// through L2 for 0.8 us of products.  Here a cluster of up to 8 CTAs takes a matrix from the
// gradient to the updated weights in one launch: a CTA holds 128 columns of X and all of S (or
// B) in shared memory.  The CTAs' partial Gram matrices meet in distributed shared memory: each
// CTA receives everyone's part of its share of the rows, sums them in the order of the CTAs and
// sends the sum to all (stores only: a remote load waits 0.3 us).  The other two products need no
// exchange.  Bound by the chain of a step: Gram product 1.7 us, exchange 2.5, the other two 1.9 each
// (128 x 196 and 128 x 128, five steps and the update: 57 us; products() takes 82).
constexpr int kSmallCluster = 8;
constexpr int kSmallThreads = 256;
constexpr uint32_t kStaged = 32 * (kB + 1) * 16;  // 128 x 128 fp32, four columns of a row together, padded
constexpr uint32_t kParts = 7 * 32 * 19 * 16;  // the CTAs' partial sums of one CTA's rows (most: 7 of 19 rows)
constexpr uint32_t kSmallSmem = 2 * kBlk + kStaged + kParts;  // X hi, lo; S hi, lo or staged; partial sums
static_assert(2 * kBlk <= kStaged && kStaged <= kParts, "S hi, lo and a staged matrix fit");

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire;" ::: "memory"); }
__device__ __forceinline__ void peer_store(uint32_t a, float4 v) {
  asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(a), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w) : "memory");
}
__device__ __forceinline__ void peer_store_u32(uint32_t a, uint32_t v) {
  asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(a), "r"(v) : "memory");
}
__device__ __forceinline__ double peer_load_f64(uint32_t a) {
  double v;
  asm volatile("ld.shared::cluster.f64 %0, [%1];" : "=d"(v) : "r"(a) : "memory");
  return v;
}

__global__ void __launch_bounds__(kSmallThreads, 1)
    small_updates(const __grid_constant__ Common c, const __grid_constant__ Ptrs p, int cluster) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  extern __shared__ __align__(1024) uint8_t smem[];
  __shared__ __align__(8) uint64_t done_bar, never_bar;
  __shared__ uint32_t tmem_slot;
  __shared__ uint32_t failed_s;                // a CTA of the cluster gave up
  __shared__ double norm_s[kSmallThreads / 32];
  __shared__ float2 inv_s;
  uint8_t *xs = smem, *ss = smem + 2 * kBlk, *parts = ss + kStaged;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int k = (int)blockIdx.x / cluster, rank = (int)blockIdx.x % cluster;
  const Mat& m = c.mats[k];
  const int nb = m.nb, rows = m.m, cols = m.n, tall = m.tall;
  const float gram_scale = m.scale[kGram], poly_scale = m.scale[kPoly], apply_scale = m.scale[kApply];
  const bool on = rank < nb;                   // (the cluster is as wide as the widest matrix needs)
  const int r = 32 * (warp & 3) + lane, c_beg = 64 * (warp >> 2);  // this thread's row and 64 columns
  const int j0 = rank * kB + c_beg;
  if (tid == 0) {
    tc::mbar_init(&done_bar, 1);
    tc::mbar_init(&never_bar, 1);
    tc::mbar_init_fence();
    failed_s = 0;
  }
  if (warp == 0) tc::tmem_alloc(&tmem_slot, 256);
  tc::fence_before_sync();
  __syncthreads();
  tc::fence_after_sync();
  const uint32_t tmem = tmem_slot, lane_base = (uint32_t)(32 * (warp & 3)) << 16;
  const bool one = warp == 0 && tc::elect_one();
  uint32_t parity = 0, drain = 2;              // drain: parity of the products that were given up
  bool ok = true;

  float f[64];
  auto split_to = [&](uint8_t* hi_block) {     // f -> the hi and lo blocks
#pragma unroll
    for (int t = 0; t < 8; ++t) {
      uint4 hi, lo;
      split8(f + 8 * t, hi, lo);
      uint8_t* at = hi_block + chunk_at(r, (c_beg >> 3) + t);
      *reinterpret_cast<uint4*>(at) = hi;
      *reinterpret_cast<uint4*>(at + kBlk) = lo;
    }
    tc::fence_proxy_async();                   // the products read through the async proxy
  };
  // f = a 128 x 128 x 128 product of hi + lo blocks, 64 of K in each of two accumulators (see
  // products()); b_mn: B's block has K along its rows
  auto product = [&](const uint8_t* a, const uint8_t* b, bool b_mn, bool hook) {
    tc::fence_before_sync();
    __syncthreads();
    tc::fence_after_sync();
    if (ok && one) {
      const uint32_t id = (1u << 4) | ((uint32_t)(kB >> 3) << 17) | ((uint32_t)(kB >> 4) << 24) | (b_mn ? 1u << 16 : 0u);
      const uint64_t ad = tc::smem_desc(tc::smem_u32(a), 2048u, 128u);
      const uint64_t bd = b_mn ? tc::smem_desc(tc::smem_u32(b), 128u, 2048u) : tc::smem_desc(tc::smem_u32(b), 2048u, 128u);
      const uint32_t db = b_mn ? 16u : 256u;
      constexpr uint64_t kLo = kBlk / 16;
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int part = 0; part < 3; ++part)   // hi lo, lo hi, hi hi
#pragma unroll
          for (int kk = 4 * h; kk < 4 * h + 4; ++kk)
            tc::mma_ss(tmem + (uint32_t)(h * kB), ad + 256u * kk + (part == 1 ? kLo : 0),
                       bd + (uint64_t)(db * kk) + (part == 0 ? kLo : 0), id, part > 0 || kk > 4 * h);
      tc::commit(&done_bar);
    }
    bool got = true;
    if (ok) {
      got = tc::mbar_wait(hook ? &never_bar : &done_bar, hook ? 0u : parity, c.wait_ns);
    }
    if (__syncthreads_or(!got)) {              // all threads of the CTA go on alike
      ok = false;
      drain = parity;
    }
    parity ^= 1u;
    tc::fence_after_sync();
#pragma unroll
    for (int e = 0; e < 64; ++e) f[e] = 0.0f;
    if (!ok) return;
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int c0 = 0; c0 < 64; c0 += 32) {
        uint32_t v[32];
        tc::ld_x32(tmem + (uint32_t)(h * kB + c_beg + c0) + lane_base, v);
        tc::wait_ld();
#pragma unroll
        for (int e = 0; e < 32; ++e) f[c0 + e] += __uint_as_float(v[e]);
      }
  };
  auto scale = [&](float s) {
#pragma unroll
    for (int e = 0; e < 64; ++e) f[e] *= s;
  };
  auto add_diag = [&](float d) {               // column c_beg + e of S is row r
    if ((r >> 6) != (c_beg >> 6)) return;      // (warp-uniform)
#pragma unroll
    for (int e = 0; e < 64; ++e) f[e] += r == c_beg + e ? d : 0.0f;
  };
  // four columns 4 c4.. of a row of a staged matrix
  auto at4 = [&](uint8_t* base, int row, int c4) { return base + (c4 * (kB + 1) + row) * 16; };
  auto stage = [&](uint8_t* base) {
#pragma unroll
    for (int q = 0; q < 16; ++q)
      *reinterpret_cast<float4*>(at4(base, r, (c_beg >> 2) + q)) =
          make_float4(f[4 * q], f[4 * q + 1], f[4 * q + 2], f[4 * q + 3]);
  };
  auto unstage = [&](uint8_t* base) {
#pragma unroll
    for (int q = 0; q < 16; ++q) {
      const float4 v = *reinterpret_cast<const float4*>(at4(base, r, (c_beg >> 2) + q));
      f[4 * q] = v.x;
      f[4 * q + 1] = v.y;
      f[4 * q + 2] = v.z;
      f[4 * q + 3] = v.w;
    }
  };

  // Momentum, U and its norm; X = U / (||U||_F + eps).  A wide matrix is read along its rows (a
  // warp 16 rows, a lane 4 columns of each) through a staged copy; a tall one's rows are columns
  // of X, and neighbouring threads, rows of X, read neighbouring elements.
  float sq = 0.0f, largest = 0.0f;             // 64 squares a thread, the rest in fp64
  if (!tall) {
    const bool four = fours(c, p, k, cols);
    const int c0 = rank * kB + 4 * lane;       // first column of this lane
    const int left = on ? min(4, max(0, cols - c0)) : 0;
#pragma unroll
    for (int b = 0; b < 16; b += 8) {          // eight rows' loads in flight together
      float4 g[8], o[8];
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        const int row = 16 * warp + b + x;
        g[x] = o[x] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (row >= rows || left == 0) continue;
        const float* mp = c.update ? p.mom[k] + (int64_t)row * p.ld_mom[k] + c0 : nullptr;
        if (four) {                            // (cols is a multiple of four: left is 4)
          g[x] = load_in4(c, p, k, row, c0);
          if (mp) o[x] = *reinterpret_cast<const float4*>(mp);
        } else {
          float* gs = &g[x].x;
          float* os = &o[x].x;
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (e < left) {
              gs[e] = load_in(c, p, k, row, c0 + e);
              if (mp) os[e] = mp[e];
            }
        }
      }
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        const int row = 16 * warp + b + x;
        o[x] = make_float4(fmaf(c.mu, o[x].x, g[x].x), fmaf(c.mu, o[x].y, g[x].y), fmaf(c.mu, o[x].z, g[x].z),
                           fmaf(c.mu, o[x].w, g[x].w));
        if (c.update && row < rows && left) {
          float* mp = p.mom[k] + (int64_t)row * p.ld_mom[k] + c0;
          if (four) *reinterpret_cast<float4*>(mp) = o[x];
          else {
            const float os[4] = {o[x].x, o[x].y, o[x].z, o[x].w};
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (e < left) mp[e] = os[e];
          }
        }
        const float4 u = make_float4(u_of(c, g[x].x, o[x].x), u_of(c, g[x].y, o[x].y), u_of(c, g[x].z, o[x].z),
                                     u_of(c, g[x].w, o[x].w));
        sq += (u.x * u.x + u.y * u.y) + (u.z * u.z + u.w * u.w);
        largest = largest4(largest, u);
        *reinterpret_cast<float4*>(at4(ss, row, lane)) = u;
      }
    }
  } else {
#pragma unroll
    for (int b = 0; b < 64; b += 16) {         // sixteen columns' loads in flight together
      const int left = on && r < rows ? min(16, max(0, cols - j0 - b)) : 0;
      const int64_t step_m = p.ld_mom[k];
      float* mp = c.update ? p.mom[k] + (int64_t)(j0 + b) * step_m + r : nullptr;
      float mom[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        f[b + e] = e < left ? load_in(c, p, k, j0 + b + e, r) : 0.0f;
        mom[e] = mp && e < left ? mp[e * step_m] : 0.0f;
      }
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        mom[e] = fmaf(c.mu, mom[e], f[b + e]);
        if (mp && e < left) mp[e * step_m] = mom[e];
        f[b + e] = u_of(c, f[b + e], mom[e]);
        sq += f[b + e] * f[b + e];
        largest = fmaxf(largest, fabsf(f[b + e]));
      }
    }
  }
  double warp_sq = sq;
  if (!fp32_squares(largest)) {
    warp_sq = 0.0;
    if (!tall) {                               // this thread's own values of the staged copy
      for (int row = 16 * warp; row < 16 * warp + 16; ++row)
        warp_sq += squares64(*reinterpret_cast<const float4*>(at4(ss, row, lane)));
    } else {
#pragma unroll
      for (int e = 0; e < 64; ++e) warp_sq += square64(f[e]);
    }
  }
#pragma unroll
  for (int x = 16; x > 0; x >>= 1) warp_sq += __shfl_xor_sync(0xFFFFFFFFu, warp_sq, x);
  if (lane == 0) norm_s[warp] = warp_sq;
  __syncthreads();
  if (tid == 0) {
    double t = 0.0;
    for (int w = 0; w < kSmallThreads / 32; ++w) t += norm_s[w];
    norm_s[0] = t;
  }
  cluster_sync();
  if (warp == 0) {
    const double mine = lane < nb ? peer_load_f64(peer_addr(&norm_s[0], lane)) : 0.0;
    double t = 0.0;
    for (int q = 0; q < nb; ++q) t += __shfl_sync(0xFFFFFFFFu, mine, q);
    if (lane == 0) inv_s = inverse_norm(t, c.eps);  // (once: 64-bit arithmetic is slow)
  }
  __syncthreads();
  if (!tall) unstage(ss);
  const float2 inv = inv_s;
#pragma unroll
  for (int e = 0; e < 64; ++e) f[e] = (f[e] * inv.x) * inv.y;
  if (on) split_to(xs);

  // rows of the Gram matrix this CTA sums for all
  const int r_beg = on ? kB * rank / nb : 0, r_cnt = on ? kB * (rank + 1) / nb - r_beg : 0;
  for (int it = 0; it < c.steps; ++it) {
    if (on) product(xs, xs, false, rank == 0 && k == c.expire_mat && it == c.expire_step);
    if (nb == 2) {                             // each takes the other's part whole: one wait
      if (it > 0) cluster_wait();              // the other has read what it received last
      if (on) {
        const uint32_t at = peer_addr(parts, rank ^ 1) + (uint32_t)((c_beg >> 2) * (kB + 1) + r) * 16u;
#pragma unroll
        for (int q = 0; q < 16; ++q)
          peer_store(at + (uint32_t)(q * (kB + 1)) * 16u, make_float4(f[4 * q], f[4 * q + 1], f[4 * q + 2], f[4 * q + 3]));
      }
      cluster_sync();
      if (on) {
#pragma unroll
        for (int q = 0; q < 16; ++q) {         // (a sum of two: the same bits in either order)
          const float4 v = *reinterpret_cast<const float4*>(at4(parts, r, (c_beg >> 2) + q));
          f[4 * q] += v.x;
          f[4 * q + 1] += v.y;
          f[4 * q + 2] += v.z;
          f[4 * q + 3] += v.w;
        }
      }
      cluster_arrive();
    } else if (nb > 2) {
      if (on) {                                // this CTA's part of row r, to the CTA that sums it
        const int owner = min(nb - 1, (r * nb + nb - 1) / kB), first = kB * owner / nb;
        const int to = r < first ? owner - 1 : owner, beg = kB * to / nb, cnt = kB * (to + 1) / nb - beg;
        const uint32_t at = peer_addr(parts, to) + (uint32_t)((rank * 32 + (c_beg >> 2)) * cnt + r - beg) * 16u;
#pragma unroll
        for (int q = 0; q < 16; ++q)
          peer_store(at + (uint32_t)(q * cnt) * 16u, make_float4(f[4 * q], f[4 * q + 1], f[4 * q + 2], f[4 * q + 3]));
      }
      cluster_sync();
      for (int e = tid; e < 32 * r_cnt; e += kSmallThreads) {
        const int c4 = e / r_cnt, row = e - c4 * r_cnt;
        float4 t = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int q = 0; q < nb; ++q) {
          const float4 v = *reinterpret_cast<const float4*>(parts + ((q * 32 + c4) * r_cnt + row) * 16);
          t = make_float4(t.x + v.x, t.y + v.y, t.z + v.z, t.w + v.w);
        }
        const uint32_t off = (uint32_t)(c4 * (kB + 1) + r_beg + row) * 16u;
        for (int q = 0; q < nb; ++q) peer_store(peer_addr(ss, q) + off, t);
      }
      cluster_sync();
      if (on) unstage(ss);
      __syncthreads();                         // (ss is written next)
    }
    if (!on) continue;
    scale(gram_scale);
    add_diag(kShift * kSA);
    split_to(ss);
    product(ss, ss, false, false);
    scale(poly_scale);
    add_diag(kDiag * kSB);
    split_to(ss);
    product(ss, xs, true, false);
    if (it + 1 < c.steps) {
      scale(apply_scale);
      split_to(xs);
    }
  }
  // (the next call's CTAs from here on: from the start on they cost 2 us of 57 instead of saving 1)
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if (nb == 2) cluster_wait();
  // Nothing is stored of a matrix of which a CTA gave up: the others have summed what it did not send.
  if (!ok && tid == 0)
    for (int q = 0; q < cluster; ++q) peer_store_u32(peer_addr(&failed_s, q), 1u);
  cluster_sync();                              // (no CTA reaches into another from here on)
  ok = failed_s == 0;
  // the weights, along their rows like the gradient
  if (on && tall && ok) store_result(c, p, k, m, 32 * (warp & 3), lane, j0, f);
  if (on && !tall) {
    scale(apply_scale / kSX);
    stage(parts);
    __syncthreads();
    const float lr = c.update ? c.lr * sqrtf(fmaxf(1.0f, (float)m.rows / (float)m.cols)) : 0.0f;
    const int c0 = rank * kB + 4 * lane, left = min(4, max(0, cols - c0));
    const bool four = left == 4 && !c.bf16_out && ((uintptr_t)p.out[k] & 15) == 0 && (p.ld_out[k] & 3) == 0;
#pragma unroll
    for (int b = 0; b < 16; b += 8) {
      float4 o[8], old[8];
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        const int row = 16 * warp + b + x;
        o[x] = *reinterpret_cast<const float4*>(at4(parts, row, lane));
        old[x] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (!c.update || !ok || row >= rows) continue;
        const float* w = static_cast<const float*>(p.out[k]) + (int64_t)row * p.ld_out[k] + c0;
        if (four) old[x] = *reinterpret_cast<const float4*>(w);
        else {
          float* os = &old[x].x;
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (e < left) os[e] = w[e];
        }
      }
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        const int row = 16 * warp + b + x;
        if (!ok || row >= rows) continue;
        const int64_t at = (int64_t)row * p.ld_out[k] + c0;
        float v[4] = {o[x].x, o[x].y, o[x].z, o[x].w};
        if (c.update) {
          v[0] = fmaf(-lr, v[0], c.decay * old[x].x);
          v[1] = fmaf(-lr, v[1], c.decay * old[x].y);
          v[2] = fmaf(-lr, v[2], c.decay * old[x].z);
          v[3] = fmaf(-lr, v[3], c.decay * old[x].w);
        }
        if (four) *reinterpret_cast<float4*>(static_cast<float*>(p.out[k]) + at) = make_float4(v[0], v[1], v[2], v[3]);
        else {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if (e >= left) continue;
            if (c.bf16_out) static_cast<__nv_bfloat16*>(p.out[k])[at + e] = __float2bfloat16_rn(v[e]);
            else static_cast<float*>(p.out[k])[at + e] = v[e];
          }
        }
      }
    }
  }

  if (tid == 0 && !ok) atomicOr(c.status, kStatusTimeout);
  if (drain < 2) tc::mbar_wait(&done_bar, drain, 10000000ull);  // before tensor memory goes (bounded)
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
  int n_sms = 0, n_items = 0;
  int norm_blocks = 0, norm_chunks = 0;  // CTAs per matrix of momentum_norm and normalise
  Mat* d_mats = nullptr;
  int4* items = nullptr;
  uint32_t* done = nullptr;
  int cluster = 0;               // CTAs per matrix of small_updates; 0: the set needs products
  Maps maps{};
  int pairs = 0;                 // CTA pairs resident at once
  int paired = 0;                // two of them in a cluster, to share items
  uint8_t* ws = nullptr;
  double* norm = nullptr;
  float2* inv = nullptr;
  uint32_t* summed = nullptr;
  uint32_t* status = nullptr;
  std::vector<void*> owned;
  int32_t expire_mat = -1, expire_step = 0;  // failure hook (aht_debug_muon_expire) of the next call
  uint64_t expire_ns = 0;
};

namespace {

#define MUON_CUDA(call)                                                                \
  do {                                                                                 \
    cudaError_t e_ = (call);                                                           \
    if (e_ != cudaSuccess) return set_last_error(AHT_ECUDA, cudaGetErrorString(e_));  \
  } while (0)

void products_config(cudaLaunchConfig_t& cfg, cudaLaunchAttribute (&attr)[2], int pairs, int paired,
                     cudaStream_t stream) {
  cfg.gridDim = dim3(2u * (unsigned)pairs);
  cfg.blockDim = dim3(kGemmThreads);
  cfg.dynamicSmemBytes = kStages * kStage + (paired ? kParcel : 0);
  cfg.stream = stream;
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim = {paired ? 4u : 2u, 1, 1};
  attr[1].id = cudaLaunchAttributeCooperative;  // every CTA resident: they wait for one another's tiles
  attr[1].val.cooperative = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
}

aht_status run(aht_muon* s, Common c, const Ptrs& p) {
  MuonDeviceGuard g(s->device);
  c.mats = s->d_mats;
  c.ws = s->ws;
  c.norm = s->norm;
  c.inv = s->inv;
  c.summed = s->summed;
  c.done = s->done;
  c.status = s->status;
  c.items = s->items;
  c.n_items = s->n_items;
  c.paired = s->paired;
  c.steps = s->cfg.steps;
  c.eps = s->cfg.eps;
  c.mu = s->cfg.momentum;
  c.nesterov = s->cfg.nesterov;
  c.wait_ns = s->expire_mat < 0 ? 2000000000ull : s->expire_ns;
  c.expire_mat = s->expire_mat;
  c.expire_step = s->expire_step;
  s->expire_mat = -1;
  const unsigned n = (unsigned)s->mats.size();
  cudaLaunchConfig_t cfg{};
  cudaLaunchAttribute attr[2], overlap;        // see tc::after_previous()
  overlap.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  overlap.val.programmaticStreamSerializationAllowed = 1;
  if (s->cluster) {
    cfg.gridDim = dim3(n * (unsigned)s->cluster);
    cfg.blockDim = dim3(kSmallThreads);
    cfg.dynamicSmemBytes = kSmallSmem;
    cfg.stream = s->stream;
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim = {(unsigned)s->cluster, 1, 1};
    attr[1] = overlap;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    MUON_CUDA(cudaLaunchKernelEx(&cfg, small_updates, c, p, s->cluster));
    return AHT_OK;
  }
  cfg.blockDim = dim3(256);
  cfg.stream = s->stream;
  cfg.attrs = &overlap;
  cfg.numAttrs = 1;
  cfg.gridDim = dim3((unsigned)s->norm_blocks, n);
  MUON_CUDA(cudaLaunchKernelEx(&cfg, momentum_norm, c, p));
  cfg.gridDim = dim3((unsigned)s->norm_chunks, n);
  MUON_CUDA(cudaLaunchKernelEx(&cfg, normalise, c, p));
  products_config(cfg, attr, std::min(s->n_items, s->pairs), s->paired, s->stream);
  MUON_CUDA(cudaLaunchKernelEx(&cfg, products, c, p, s->maps));
  return AHT_OK;
}

constexpr char kMisaligned[] = "an address is not a multiple of its elements' size";

// The boxes that the products copy (see Maps).
aht_status make_maps(aht_muon* s, int64_t bytes) {
  void* fn = nullptr;
  cudaDriverEntryPointQueryResult found;
  MUON_CUDA(cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &found));
  if (found != cudaDriverEntryPointSuccess || !fn)
    return set_last_error(AHT_ECUDA, "the driver has no cuTensorMapEncodeTiled");
  const cuuint64_t dims[3] = {64, 16, (cuuint64_t)(bytes / 2048)}, strides[2] = {128, 2048};
  const cuuint32_t one[3] = {1, 1, 1};
  struct Box { CUtensorMap* map; cuuint32_t rows, cols; };
  for (const Box& b : {Box{&s->maps.cols, 16, 8}, Box{&s->maps.rows, 8, 16}, Box{&s->maps.quarter, 8, 8}}) {
    const cuuint32_t box[3] = {64, b.rows, b.cols};
    const CUresult e = reinterpret_cast<decltype(&cuTensorMapEncodeTiled)>(fn)(
        b.map, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, s->ws, dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
        CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (e != CUDA_SUCCESS) return set_last_error(AHT_ECUDA, "cuTensorMapEncodeTiled failed");
  }
  return AHT_OK;
}

// The work of one step (see Item): the phases in order, in each the longest items first.  Where
// clusters are of two pairs and a phase leaves half of the pairs idle, its items with a sum over K
// long enough to pay for the exchange are shared.
struct Work {
  std::vector<int4> items;
  std::vector<std::array<int32_t, 3>> stores;  // see Mat
  size_t most = 0, shared = 0;                 // entries of a phase, items shared
};
Work work_list(const std::vector<Mat>& mats, int pairs, bool paired) {
  Work w;
  w.stores.resize(mats.size());
  for (int ph = kGram; ph <= kApply; ++ph) {
    auto blocks_of_k = [&](const int4& v) { return ph == kGram ? mats[v.x].nb : mats[v.x].mb; };
    std::vector<int4> list;
    for (int k = 0; k < (int)mats.size(); ++k) {
      const Mat& m = mats[k];
      for (int I = 0; 2 * I < m.mb; ++I)
        for (int J = ph == kApply ? 0 : 2 * I; J < (ph == kApply ? m.nb : m.mb); ++J) list.push_back(make_int4(k, ph, I, J));
    }
    std::stable_sort(list.begin(), list.end(),
                     [&](const int4& x, const int4& y) { return blocks_of_k(x) > blocks_of_k(y); });
    size_t shared = 0;
    if (paired)
      while (shared < list.size() && blocks_of_k(list[shared]) >= kShareK) ++shared;
    if (list.size() + shared > (size_t)pairs) shared = 0;
    for (size_t x = 0; x < list.size(); ++x) {
      const int4 v = list[x];
      w.stores[v.x][ph] += (x < shared ? 2 : 1) * std::min(2, mats[v.x].mb - 2 * v.z);
      if (x < shared) {
        w.items.push_back(make_int4(v.x, ph | 4, v.z, v.w));
        w.items.push_back(make_int4(v.x, ph | 8, v.z, v.w));
      } else {
        w.items.push_back(v);
      }
    }
    w.most = std::max(w.most, list.size() + shared);
    w.shared += shared;
    if (paired && (w.items.size() & 1)) w.items.push_back(make_int4(-1, 0, 0, 0));  // (shared ones start at even places)
  }
  return w;
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
    m.scale[kGram] = up(m.m) * kSA / (kSX * kSX);
    m.scale[kPoly] = up(m.m) * kC * kSB / (kSA * kSA);
    m.scale[kApply] = up(m.m) / kSB;
    m.x_lo = (int64_t)m.mb * m.nb * kBlk;
    m.s_lo = (int64_t)m.mb * m.mb * kBlk;
    m.norm_blocks = (int)std::min<int64_t>(((int64_t)m.rows * m.cols + 4095) / 4096, kNormBlocks);
    most = std::max(most, (int64_t)m.mb * m.nb);
    s->norm_blocks = std::max(s->norm_blocks, m.norm_blocks);
    s->mats.push_back(m);
  }
  s->norm_chunks = (int)std::min<int64_t>(most * 8, 4096);
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
  // A set of matrices that each fit a cluster of small_updates runs there; beside a larger one
  // they cost nothing in products(), whose other tiles fill their waits.
  int wide = 0;
  for (const Mat& m : s->mats) wide = std::max(wide, m.mb == 1 ? m.nb : kSmallCluster + 1);
  std::vector<int4> items;
  if (wide <= kSmallCluster) {
    for (s->cluster = 1; s->cluster < wide;) s->cluster *= 2;
    MUON_CUDA(cudaFuncSetAttribute(small_updates, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmallSmem));
  } else {
    MUON_CUDA(cudaFuncSetAttribute(products, cudaFuncAttributeMaxDynamicSharedMemorySize, kStages * (int)kStage + (int)kParcel));
    // Clusters of two pairs where no phase has more items than pairs and some are shared: 1024 x 1024
    // 31 us of 183 less; with more items the matrices' phases overlap, and 72 pairs (clusters of
    // four CTAs leave some SMs empty) are fewer than 76: the set of two S5 heads 288 us instead of 275.
    for (int paired = 1; paired >= 0 && items.empty(); --paired) {
      cudaLaunchConfig_t query{};
      cudaLaunchAttribute attr[2];
      products_config(query, attr, s->n_sms / 4 * 2, paired, s->stream);
      int clusters = 0;
      MUON_CUDA(cudaOccupancyMaxActiveClusters(&clusters, products, &query));
      s->pairs = clusters * (paired + 1);
      s->paired = paired;
      Work w = work_list(s->mats, s->pairs, paired);
      if (clusters < 1 || (paired && (w.most > (size_t)s->pairs || w.shared == 0))) continue;
      items.swap(w.items);
      for (size_t k = 0; k < s->mats.size(); ++k) std::copy(w.stores[k].begin(), w.stores[k].end(), s->mats[k].stores);
    }
    if (!s->pairs) return set_last_error(AHT_ECUDA, "no room for a CTA pair of the products");
  }
  if (items.size() > (1u << 31) / (size_t)cfg->steps / 2) return set_last_error(AHT_EINVAL, "too many tiles in one call");
  s->n_items = (int)items.size();
  if (!up((void**)&s->d_mats, s->mats.data(), s->mats.size() * sizeof(Mat)) || !alloc((void**)&s->ws, (size_t)at) ||
      (s->n_items && !up((void**)&s->items, items.data(), items.size() * sizeof(int4))) ||
      !alloc((void**)&s->norm, (size_t)n * kNormBlocks * sizeof(double)) || !alloc((void**)&s->inv, (size_t)n * sizeof(float2)) ||
      !alloc((void**)&s->summed, (size_t)n * 4) || cudaMemset(s->summed, 0, (size_t)n * 4) != cudaSuccess ||
      !alloc((void**)&s->done, (size_t)n * 3 * kMaxSteps * 4) || !alloc((void**)&s->status, 4) ||
      cudaMemset(s->status, 0, 4) != cudaSuccess)
    return set_last_error(AHT_ENOMEM, "workspace allocation failed");
  MUON_CUDA(cudaStreamSynchronize(cudaStreamLegacy));  // the tables are there, whatever kind of stream s->stream is
  if (s->cluster) return AHT_OK;
  return make_maps(s, at);
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
    if ((((uintptr_t)q.W | (uintptr_t)q.M) & 3) || ((uintptr_t)q.G & (grad_dtype == AHT_FP32 ? 3 : 1)))
      return set_last_error(AHT_EINVAL, kMisaligned);
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
    if (((uintptr_t)in[k] | (uintptr_t)out[k]) & (dtype == AHT_FP32 ? 3 : 1)) return set_last_error(AHT_EINVAL, kMisaligned);
    p.in[k] = in[k];
    p.out[k] = out[k];
    p.ld_in[k] = ld_in[k];
    p.ld_out[k] = ld_out[k];
  }
  Common c{};
  c.bf16_in = c.bf16_out = dtype == AHT_BF16;
  return run(s, c, p);
}

aht_status aht_debug_muon_expire(aht_muon* s, int32_t matrix, int32_t step, int64_t limit_ns) {
  if (!s) return set_last_error(AHT_EINVAL, "NULL argument");
  if (matrix >= 0 && (matrix >= (int64_t)s->mats.size() || step < 0 || step >= s->cfg.steps))
    return set_last_error(AHT_EINVAL, "no such matrix or step");
  if (matrix >= 0 && (limit_ns < 1 || limit_ns > 1000000000))
    return set_last_error(AHT_EINVAL, "limit_ns must be in 1..1e9");
  s->expire_mat = matrix < 0 ? -1 : matrix;
  s->expire_step = step;
  s->expire_ns = (uint64_t)limit_ns;
  return AHT_OK;
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
