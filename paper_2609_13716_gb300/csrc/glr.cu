// glr.cu -- the gated linear recurrence over a collected trajectory (include/aht.h states
// the model): forward over T steps, one serving step (T = 1), and the backward pass.
//
// A lane is one channel d of one env n; its T steps are a chain, lanes are independent.  A
// thread owns V neighbouring channels of one env and a segment of S consecutive steps; a
// warp's row is contiguous.  The next segments are copied while the present one is computed:
// through a ring in shared memory where rows are aligned, else one ahead in registers.
//   - Many lanes: a warp walks its lanes' whole chain, segment after segment.
//   - Few lanes: WT warps of a CTA, and up to 16 CTAs of a cluster, take consecutive segments of
//     the same lanes.  A segment is an affine map of the state it receives, h -> A h + H;
//     the maps are composed over the warps in shared memory and over the CTAs in distributed
//     shared memory, then every thread applies its own from the state that reaches it.  All
//     inputs are read once, and no CTA waits for one outside its cluster.
// The backward pass is the same scan from the end for p = dL/dh of the state a step
// receives, p -> A p + P with the same A.
//
// State, gates and sums are fp32 whatever the tensors' type; each output is rounded once.
// A = 0 stands for a reset in the segment and for nothing else: it drops what it receives, NaN and
// infinity included.  A decay, or a product of them, that underflows stays at 2^-149 instead, so
// that what is not finite comes through whether the steps are split or not.
//
// The backward pass needs the state before every step.  The forward pass leaves it as fp32
// checkpoints every kSeg = 8 steps (0.5 B per element; the rounded h would cost 2-4 B and
// carry bf16 rounding into every gradient), and the backward pass rebuilds the seven states
// between two checkpoints in registers.
#include <cooperative_groups.h>
#include <cuda_bf16.h>

#include <algorithm>
#include <atomic>
#include <type_traits>

#include "kernels.h"
#include "tc_common.cuh"

namespace aht {
aht_status set_last_error(aht_status s, const char* msg);  // the message of aht_last_error
}  // namespace aht

using namespace aht;
namespace cg = cooperative_groups;

namespace {

constexpr int kSeg = AHT_GLR_SEGMENT;  // steps between two checkpoints
constexpr float kGateScale = 8.0f;     // s = 8 softplus(lam)
constexpr int kMaxCluster = 16;

// Limit of a wait for a window's maps, and the window at which the failure hook has CTA 0 of every
// cluster wait for nothing (none: ~0).
struct Waits {
  uint64_t limit_ns;
  uint32_t expire_at;
};
__device__ uint32_t glr_status;        // kStatus* bits since the last aht_glr_sync

struct Seq {
  void* p;
  int64_t st, sn;
};

struct GlrDev {
  int32_t D;
  int64_t T, N;
  Seq x, r, i;
  const float* lam;
  const uint8_t* reset;
  const int32_t* lengths;
};

// ---- V neighbouring channels as one load or store -----------------------------------------
template <int kBytes> struct Word;
template <> struct Word<2> { using T = uint16_t; };
template <> struct Word<4> { using T = uint32_t; };
template <> struct Word<8> { using T = uint2; };
template <> struct Word<16> { using T = uint4; };

template <typename E, int V>
struct Vec {
  using W = typename Word<(int)sizeof(E) * V>::T;
  union {
    W w;
    E e[V];
  };
  __device__ __forceinline__ Vec() {}
  __device__ __forceinline__ void load(const void* p) { w = __ldcs(static_cast<const W*>(p)); }
  __device__ __forceinline__ void store(void* p) const { __stcs(static_cast<W*>(p), w); }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int v = 0; v < V; ++v) e[v] = E(0.0f);
  }
  __device__ __forceinline__ float get(int v) const { return (float)e[v]; }
  __device__ __forceinline__ void set(int v, float f) { e[v] = (E)f; }
  __device__ __forceinline__ void set2(int v, float f0, float f1) {  // v even
    if constexpr (sizeof(E) == 2) {
      const uint32_t both = tc::pack_bf16(f0, f1);
      if constexpr (V == 2) w = both;
      else if constexpr (V == 4) (v ? w.y : w.x) = both;
    } else {
      e[v] = f0;
      e[v + 1] = f1;
    }
  }
};

__device__ __forceinline__ float softplus_f(float x) { return fmaxf(x, 0.0f) + log1pf(expf(-fabsf(x))); }
__device__ __forceinline__ float sigmoid_f(float x) { return 1.0f / (1.0f + expf(-x)); }

// ---- gates, two elements at a time (packed fp32 pairs) -------------------------------------
constexpr float kLog2e = 1.4426950408889634f;
__device__ __forceinline__ uint64_t both(float c) { return tc::f2_pack(c, c); }

// 1 / (1 + 2^(-x log2 e)): the hardware exp2 and reciprocal, 2^-22 relative each; 0 and 1 at
// the infinities.
__device__ __forceinline__ uint64_t sigmoid2(uint64_t x) {
  float a, b;
  tc::f2_unpack(tc::f2_mul(x, both(-kLog2e)), a, b);
  tc::f2_unpack(tc::f2_add(tc::f2_pack(tc::ex2_approx(a), tc::ex2_approx(b)), both(1.0f)), a, b);
  return tc::f2_pack(tc::rcp_approx(a), tc::rcp_approx(b));
}
// A decay or a product of them, which is not to become 0.  (Of 0 and positive numbers the integers are
// in the same order; NaN is above all.)
__device__ __forceinline__ float not_zero(float a) { return __int_as_float(max(__float_as_int(a), 1)); }
// The decay a = exp(z) for z <= 0, and a - 1.  Down to z = -1/4 a - 1 is its series
// z (1 + z/2 + z^2/6 + ... + z^6/5040) (the next term is below 2^-26 there) and a the sum; beyond
// it a is 2^(z log2 e) and a - 1 the difference: rounded the other way round, 1 + (a - 1) would hold
// a small a to 3e-8 of 1 instead of itself (with lam = 4 dr was off by 2e-6 of its norm).
// kSmall: no z of the warp lies beyond.
struct Decay {
  uint64_t a, em;   // a, a - 1
  uint64_t kept;    // both in one: a - 1 (0 or negative) down to z = -1/4, a (positive) beyond
};
template <bool kSmall>
__device__ __forceinline__ Decay decay(uint64_t z) {
  uint64_t s = tc::f2_fma(z, both(1.0f / 5040.0f), both(1.0f / 720.0f));
  s = tc::f2_fma(z, s, both(1.0f / 120.0f));
  s = tc::f2_fma(z, s, both(1.0f / 24.0f));
  s = tc::f2_fma(z, s, both(1.0f / 6.0f));
  s = tc::f2_fma(z, s, both(0.5f));
  s = tc::f2_mul(z, tc::f2_fma(z, s, both(1.0f)));
  const uint64_t near = tc::f2_add(s, both(1.0f));
  if (kSmall) return Decay{near, s, s};
  float z0, z1, s0, s1, n0, n1, a, b, am, bm;
  tc::f2_unpack(z, z0, z1);
  tc::f2_unpack(s, s0, s1);
  tc::f2_unpack(near, n0, n1);
  tc::f2_unpack(tc::f2_mul(z, both(kLog2e)), a, b);
  a = not_zero(tc::ex2_approx(a));
  b = not_zero(tc::ex2_approx(b));
  tc::f2_unpack(tc::f2_add(tc::f2_pack(a, b), both(-1.0f)), am, bm);
  const bool c0 = z0 > -0.25f, c1 = z1 > -0.25f;
  return Decay{tc::f2_pack(c0 ? n0 : a, c1 ? n1 : b), tc::f2_pack(c0 ? s0 : am, c1 ? s1 : bm),
               tc::f2_pack(c0 ? s0 : a, c1 ? s1 : b)};
}
// a and a - 1 of what was kept.
template <bool kSmall>
__device__ __forceinline__ float kept_a(float k) {
  return !kSmall && k > 0.0f ? k : k + 1.0f;
}
template <bool kSmall>
__device__ __forceinline__ uint64_t kept_m1(uint64_t k) {
  if (kSmall) return k;
  float k0, k1, m0, m1;
  tc::f2_unpack(k, k0, k1);
  tc::f2_unpack(tc::f2_add(k, both(-1.0f)), m0, m1);
  return tc::f2_pack(k0 > 0.0f ? m0 : k0, k1 > 0.0f ? m1 : k1);
}
// beta^2 = 1 - a^2 = em (-2 - em)
__device__ __forceinline__ uint64_t beta_sq(uint64_t em) { return tc::f2_mul(em, tc::f2_fma(em, both(-1.0f), both(-2.0f))); }
__device__ __forceinline__ float sqrt_q(float x) {
  float y;
  asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float rsqrt_q(float x) {
  float y;
  asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// A y + b, or b alone where A is 0: after a reset.
__device__ __forceinline__ float apply(float A, float y, float b) { return A == 0.0f ? b : fmaf(A, y, b); }

// Where a warp works: its env, its channels, its segment of a window of steps.
struct Place {
  int64_t n, d;     // env, first channel of this thread
  bool on;          // the thread has channels
  int64_t len;      // steps of env n
  __device__ __forceinline__ Place(const GlrDev& a, int64_t unit, int tiles, int lane, int V, bool any) {
    n = unit / tiles;
    d = ((unit - n * tiles) * 32 + lane) * V;
    on = any && d < a.D;
    len = any && a.lengths ? max((int64_t)0, min(a.T, (int64_t)a.lengths[n])) : any ? a.T : 0;
  }
};

// The rows of a segment, one after another.  The asm keeps the compiler from carrying a
// pointer per row and tensor through the loop over windows (over 100 registers).
struct Walk {
  char* p;
  int64_t step;
  __device__ __forceinline__ Walk(const Seq& s, const void* lane0, int esz, int64_t t) {
    step = s.st * esz;
    p = static_cast<char*>(const_cast<void*>(lane0)) + t * step;
    asm volatile("" : "+l"(p), "+l"(step));
  }
  __device__ __forceinline__ char* next() {
    char* q = p;
    p += step;
    return q;
  }
  __device__ __forceinline__ char* next_back() {
    char* q = p;
    p -= step;
    return q;
  }
};

// A warp's ring of segments in shared memory, filled by asynchronous copies: a row is 32 lanes of
// kLane bytes (2 or 4), copied 16 bytes a lane; what lies past the env's steps or its channels is
// zero.  Rows start on 16-byte boundaries (checked by the host).
template <int kTensors, int S, int kLane, int kExtra>
struct Ring {
  static constexpr int kRow = 32 * kLane, kChunks = kRow / 16, kPer = 32 / kChunks;  // rows an instruction copies
  static constexpr int kStage = kTensors * S * kRow + kExtra;  // bytes of a segment
  static_assert(S % kPer == 0, "whole instructions a segment");
  __device__ __forceinline__ static void copy16(void* dst, const void* src, bool on) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(tc::smem_u32(dst)), "l"(src), "r"(on ? 16 : 0)
                 : "memory");
  }
  __device__ __forceinline__ static void rows(uint8_t* slot, int tensor, const Seq& s, const void* lane0, int esz,
                                              int64_t t0, int64_t left, int lane, bool chunk) {
    const int64_t step = s.st * esz;
    const char* src = static_cast<const char*>(lane0) + (t0 + lane / kChunks) * step + (lane % kChunks) * 16;
    uint8_t* dst = slot + tensor * S * kRow + lane * 16;
#pragma unroll
    for (int k = 0; k < S; k += kPer) {
      const bool on = chunk && k + lane / kChunks < left;
      copy16(dst + k * kRow, on ? src : static_cast<const char*>(s.p), on);
      src += kPer * step;
    }
  }
  __device__ __forceinline__ static void commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
  template <int kLeft>
  __device__ __forceinline__ static void wait() {
    asm volatile("cp.async.wait_group %0;" ::"n"(kLeft) : "memory");
    __syncwarp();
  }
};

// Whether step t0 + lane begins an episode (t0 + lane < len); a ballot of it gives a segment's
// resets.  Loaded with a segment's rows, a window before the ballot waits for it.
template <int S>
__device__ __forceinline__ uint8_t reset_byte(const GlrDev& a, const Place& at, int64_t t0, int lane) {
  return a.reset && lane < S && t0 + lane < at.len ? a.reset[(t0 + lane) * a.N + at.n] : (uint8_t)0;
}

// The map that reaches segment (rank, wt) of a window, from the maps (A, H) that every
// segment publishes, and the composition of the whole window.  Segments run in the order of
// the scan (for the backward pass the caller numbers them from the end).
//
// Between CTAs the maps travel as asynchronous remote stores that count on the receiver's
// mbarrier: a cluster barrier would have to release, that is wait for, every global store the
// threads have in flight (a sixth of the stalls).  Two buffers suffice: a CTA sends for window
// w + 2 after it has everyone's maps of w + 1, which each CTA sends after all its warps have
// read w.
//
// A wait that runs out is for good: from that window on the thread takes NaN for the state it would
// receive, sends nothing (its buffers may still be unread elsewhere) and waits for nothing, so the
// other CTAs' waits run out in turn and the whole pass ends.  What it computes from its own steps
// alone (after a reset among them) stays right.
template <int V, int WT, bool kCluster>
struct Exchange {
  struct Shared {
    float a[2][WT][32][V], h[2][WT][32][V];   // maps of the CTA's warps
    alignas(16) float c[2][kMaxCluster][32][2 * V];  // maps of the cluster's CTAs: A, then H
    alignas(8) uint64_t bar[2];
    uint64_t never;
  };
  __device__ __forceinline__ static void init(Shared& sh) {
    if (!kCluster) return;
    if (threadIdx.x == 0) {
      tc::mbar_init(&sh.bar[0], 1);
      tc::mbar_init(&sh.bar[1], 1);
      tc::mbar_init(&sh.never, 1);
      tc::mbar_init_fence();
    }
    cg::this_cluster().sync();
  }
  // No CTA leaves while another may send to it, or while what was sent is on its way: a thread that
  // gave up at window `lost` has not waited for the maps of that window and the next (bounded).
  __device__ __forceinline__ static void finish(Shared& sh, uint32_t lost) {
    if (!kCluster) return;
    cg::this_cluster().sync();
    if (lost == ~0u) return;
    atomicOr(&glr_status, kStatusTimeout);
    for (uint32_t w = lost; w < lost + 2; ++w) tc::mbar_wait(&sh.bar[w & 1u], (w >> 1) & 1u, 1000000ull);
  }
  __device__ __forceinline__ static void send(const float* to, const float* v, const uint64_t* bar, int dst) {
    uint32_t at, mb;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(tc::smem_u32(to)), "r"(dst));
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(mb) : "r"(tc::smem_u32(bar)), "r"(dst));
    if (V == 1)
      asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v2.b32 [%0], {%1, %2}, [%3];" ::"r"(at),
                   "r"(__float_as_uint(v[0])), "r"(__float_as_uint(v[1])), "r"(mb)
                   : "memory");
    else
      asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v4.b32 [%0], {%1, %2, %3, %4}, [%5];" ::"r"(
                       at),
                   "r"(__float_as_uint(v[0])), "r"(__float_as_uint(v[1])), "r"(__float_as_uint(v[V])),
                   "r"(__float_as_uint(v[2 * V - 1])), "r"(mb)
                   : "memory");
  }
  // carry: the state before the window, in; after the window, out.  in: the state before
  // this segment.  n: windows before this one.  lost: the window at which this thread gave up.
  __device__ __forceinline__ static void run(Shared& sh, const Waits& waits, uint32_t& lost, uint32_t n, int rank,
                                             int n_rank, int wt, int lane, const float (&A)[V], const float (&H)[V],
                                             float (&carry)[V],
                                             float (&in)[V]) {
    const int buf = (int)(n & 1u);
#pragma unroll
    for (int v = 0; v < V; ++v) {
      sh.a[buf][wt][lane][v] = A[v];
      sh.h[buf][wt][lane][v] = H[v];
    }
    __syncthreads();
    float pa[V], ph[V], wa[WT][V], wh[WT][V];  // pa, ph: composition before this warp
#pragma unroll
    for (int w = 0; w < WT; ++w)
#pragma unroll
      for (int v = 0; v < V; ++v) {
        wa[w][v] = sh.a[buf][w][lane][v];
        wh[w][v] = sh.h[buf][w][lane][v];
      }
#pragma unroll
    for (int v = 0; v < V; ++v) {
      pa[v] = 1.0f;
      ph[v] = 0.0f;
    }
    auto then = [&](float* ca, float* ch, int w) {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        ch[v] = apply(wa[w][v], ch[v], wh[w][v]);
        ca[v] *= wa[w][v];
      }
    };
    // (the product may underflow on its way, or pass NaN on to a reset: 0 where a map has one, not 0 else)
    auto end = [&](float* ca, int n_w) {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        bool cut = false;
#pragma unroll
        for (int w = 0; w < WT; ++w) cut = cut || (w < n_w && wa[w][v] == 0.0f);
        ca[v] = cut ? 0.0f : not_zero(ca[v]);
      }
    };
#pragma unroll
    for (int w = 0; w < WT; ++w)
      if (w < wt) then(pa, ph, w);
    end(pa, wt);
    if (kCluster) {
      if (wt == WT - 1 && lost == ~0u) {  // the last warp has the CTA's map: to every CTA of the cluster
        float t[2 * V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
          t[v] = pa[v];
          t[V + v] = ph[v];
        }
        then(t, t + V, WT - 1);
        end(t, WT);
        if (lane == 0) tc::mbar_expect_tx(&sh.bar[buf], (uint32_t)n_rank * 32u * 2u * V * 4u);
        for (int dst = 0; dst < n_rank; ++dst) send(&sh.c[buf][rank][lane][0], t, &sh.bar[buf], dst);
      }
      if (lost == ~0u) {
        const bool hook = n == waits.expire_at && rank == 0;
        if (!tc::mbar_wait(hook ? &sh.never : &sh.bar[buf], hook ? 0u : (n >> 1) & 1u, waits.limit_ns)) lost = n;
      }
#pragma unroll
      for (int v = 0; v < V; ++v) in[v] = carry[v];
      for (int c = 0; c < n_rank; ++c)
#pragma unroll
        for (int v = 0; v < V; ++v) {
          if (c == rank) in[v] = carry[v];
          carry[v] = apply(sh.c[buf][c][lane][v], carry[v], sh.c[buf][c][lane][V + v]);
        }
      if (lost != ~0u) {
#pragma unroll
        for (int v = 0; v < V; ++v) in[v] = carry[v] = __int_as_float(0x7FC00000);
      }
    } else {
#pragma unroll
      for (int v = 0; v < V; ++v) in[v] = carry[v];
#pragma unroll
      for (int w = 0; w < WT; ++w)
#pragma unroll
        for (int v = 0; v < V; ++v) carry[v] = apply(wa[w][v], carry[v], wh[w][v]);
    }
#pragma unroll
    for (int v = 0; v < V; ++v) in[v] = apply(pa[v], in[v], ph[v]);
  }
};

// CTAs of kWarps warps: WT of them share lanes, kWarps / WT lane groups.  kRing > 0: the rows
// come through a ring of that many segments (rows of 4-byte lanes, aligned); 0: the next
// segment waits in registers.
//
// Whole chains are bound by memory (128 x 8192 x 128 fp32 304 us, the rate of a copy; 128 x 16384 x
// 128 bf16 356 us, 6.1 TB/s, and 61 % of the issue slots); split ones by the hand-over of a window
// between a cluster's CTAs (65537 x 1 x 896 fp32 172 us, 5.5 TB/s); one step by its launch.  With
// decay exponents beyond 1/4 (see Decay) the same three take 307, 392 and 187 us.
template <typename E, int V, int S, int WT, int kWarps, bool kCluster, int kRing>
__global__ void __launch_bounds__(32 * kWarps, kRing && WT == 1 && sizeof(E) == 2 ? 5 : 16 / kWarps)
    glr_fwd(const __grid_constant__ GlrDev a, const float* h0, const __grid_constant__ Seq h, float* h_last,
            float* ckpt, int n_rank, Waits waits) {
  tc::after_previous();
  using X = Exchange<V, WT, kCluster>;
  __shared__ typename X::Shared sh;
  constexpr int kE = S * V;
  static_assert(kE % 2 == 0 && (S % kSeg == 0 || kSeg % S == 0), "pairs of elements; segments and checkpoints nest");
  constexpr int WL = kWarps / WT;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, wt = warp % WT;
  const int rank = kCluster ? (int)(blockIdx.x % n_rank) : 0;
  const int tiles = (a.D + 32 * V - 1) / (32 * V);
  const int64_t unit = (int64_t)(kCluster ? blockIdx.x / n_rank : blockIdx.x) * WL + warp / WT;
  const Place at(a, unit, tiles, lane, V, unit < a.N * tiles);
  const int64_t lanes = a.N * a.D, me = at.n * a.D + at.d;
  const int seg = rank * WT + wt;
  const int64_t window = (int64_t)(kCluster ? n_rank : 1) * WT * S;
  X::init(sh);

  float m[V], carry[V];  // m = -s
  bool small = true;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    m[v] = at.on ? -kGateScale * softplus_f(a.lam[at.d + v]) : 0.0f;
    small = small && m[v] > -0.25f;
    carry[v] = at.on && h0 ? h0[me + v] : 0.0f;
  }
  small = __all_sync(0xFFFFFFFFu, small);
  Vec<E, V> nx[S], nr[S], ni[S];
  uint8_t nrs = 0;
  using R = Ring<3, kRing ? S : 8, kRing ? V * (int)sizeof(E) : 4, 0>;
  extern __shared__ __align__(128) uint8_t ring_smem[];
  uint8_t* ring = ring_smem + (kRing ? warp * kRing * R::kStage : 0);
  const bool any = unit < a.N * tiles, chunk = any && at.d - lane * V + lane % R::kChunks * (16 / (int)sizeof(E)) < a.D;
  int slot = 0;
  const E* px = static_cast<const E*>(a.x.p) + at.n * a.x.sn + at.d;
  const E* pr = static_cast<const E*>(a.r.p) + at.n * a.r.sn + at.d;
  const E* pi = static_cast<const E*>(a.i.p) + at.n * a.i.sn + at.d;
  const E* ph = static_cast<const E*>(h.p) + at.n * h.sn + at.d;
  auto fetch_ring = [&](int64_t t0, int to) {
    uint8_t* dst = ring + to * R::kStage;
    const int64_t left = at.len - t0;
    R::rows(dst, 0, a.r, pr - lane * V, sizeof(E), t0, left, lane, chunk);
    R::rows(dst, 1, a.i, pi - lane * V, sizeof(E), t0, left, lane, chunk);
    R::rows(dst, 2, a.x, px - lane * V, sizeof(E), t0, left, lane, chunk);
    R::commit();
  };
  auto fetch = [&](int64_t t0) {
    Walk wr(a.r, pr, sizeof(E), t0), wi(a.i, pi, sizeof(E), t0), wx(a.x, px, sizeof(E), t0);
#pragma unroll
    for (int k = 0; k < S; ++k) {
      nx[k].zero();
      nr[k].zero();
      ni[k].zero();
      const char *qr = wr.next(), *qi = wi.next(), *qx = wx.next();
      if (at.on && t0 + k < at.len) {
        nr[k].load(qr);
        ni[k].load(qi);
        nx[k].load(qx);
      }
    }
    nrs = reset_byte<S>(a, at, t0, lane);
  };
  if (kRing) {
#pragma unroll
    for (int w = 0; w < kRing; ++w) fetch_ring((int64_t)seg * S + w * window, w);
    nrs = reset_byte<S>(a, at, (int64_t)seg * S, lane);
  } else {
    fetch((int64_t)seg * S);
  }
  uint32_t n = 0, lost = ~0u;  // windows so far, see Exchange
  for (int64_t w0 = 0; w0 < a.T; w0 += window, ++n) {
    const int64_t t0 = w0 + (int64_t)seg * S;
    const uint32_t rs = __ballot_sync(0xFFFFFFFFu, nrs != 0);
    // a full segment without a reset needs no masks
    const bool plain = rs == 0 && t0 + S <= at.len;
    float da[kE], b[kE];  // decay and input of element k V + v
    float y[V];
    if (kRing) {
      R::template wait<(kRing > 0 ? kRing - 1 : 0)>();
      const uint8_t* src = ring + slot * R::kStage + lane * V * (int)sizeof(E);
#pragma unroll
      for (int k = 0; k < S; ++k) {
        nr[k].w = *reinterpret_cast<const typename Vec<E, V>::W*>(src + k * R::kRow);
        ni[k].w = *reinterpret_cast<const typename Vec<E, V>::W*>(src + (S + k) * R::kRow);
        nx[k].w = *reinterpret_cast<const typename Vec<E, V>::W*>(src + (2 * S + k) * R::kRow);
      }
    }
    auto gate = [&](auto small_c) {
#pragma unroll
      for (int e = 0; e < kE; e += 2) {
        const int k0 = e / V, v0 = e % V, k1 = (e + 1) / V, v1 = (e + 1) % V;
        const uint64_t rho = sigmoid2(tc::f2_pack(nr[k0].get(v0), nr[k1].get(v1)));
        const Decay q = decay<decltype(small_c)::value>(tc::f2_mul(tc::f2_pack(m[v0], m[v1]), rho));
        const uint64_t iota = sigmoid2(tc::f2_pack(ni[k0].get(v0), ni[k1].get(v1)));
        float b0, b1;
        tc::f2_unpack(beta_sq(q.em), b0, b1);
        const uint64_t ix = tc::f2_mul(iota, tc::f2_pack(nx[k0].get(v0), nx[k1].get(v1)));
        tc::f2_unpack(tc::f2_mul(tc::f2_pack(sqrt_q(b0), sqrt_q(b1)), ix), b[e], b[e + 1]);
        tc::f2_unpack(q.a, da[e], da[e + 1]);
      }
    };
    if (small) gate(std::true_type());
    else gate(std::false_type());
    if (kRing) {
      __syncwarp();                       // every lane has read the slot
      fetch_ring(t0 + kRing * window, slot);
      slot = slot + 1 == kRing ? 0 : slot + 1;
      nrs = reset_byte<S>(a, at, t0 + window, lane);
    } else if (w0 + window < a.T) {
      fetch(t0 + window);
    }
    if (!plain) {
#pragma unroll
      for (int e = 0; e < kE; ++e) {
        const int k = e / V;
        const bool live = t0 + k < at.len;
        da[e] = live ? ((rs >> k) & 1u ? 0.0f : da[e]) : 1.0f;
        b[e] = live ? b[e] : 0.0f;
      }
    }
    if (WT > 1 || kCluster) {
      float A[V], H[V];
#pragma unroll
      for (int v = 0; v < V; ++v) {
        A[v] = da[v];
        H[v] = b[v];
      }
      if (plain) {
#pragma unroll
        for (int e = V; e < kE; ++e) {
          H[e % V] = fmaf(da[e], H[e % V], b[e]);
          A[e % V] *= da[e];
        }
      } else {
#pragma unroll
        for (int e = V; e < kE; ++e) {
          H[e % V] = apply(da[e], H[e % V], b[e]);
          A[e % V] *= da[e];
        }
      }
#pragma unroll
      for (int v = 0; v < V; ++v) A[v] = rs ? 0.0f : not_zero(A[v]);
      X::run(sh, waits, lost, n, rank, n_rank, wt, lane, A, H, carry, y);
    } else {
#pragma unroll
      for (int v = 0; v < V; ++v) y[v] = carry[v];
    }
    auto save = [&](int k) {  // the state before step t0 + k
      if (ckpt && at.on && t0 + k < a.T && (S >= kSeg ? k % kSeg == 0 : k == 0 && t0 % kSeg == 0)) {
        float* c = ckpt + ((t0 + k) / kSeg) * lanes + me;
#pragma unroll
        for (int v = 0; v < V; ++v) c[v] = y[v];
      }
    };
    Walk wh(h, ph, sizeof(E), t0);
    if (plain) {
#pragma unroll
      for (int k = 0; k < S; ++k) {
        if (k % kSeg == 0) save(k);
        Vec<E, V> o;
#pragma unroll
        for (int v = 0; v < V; ++v) y[v] = fmaf(da[k * V + v], y[v], b[k * V + v]);
        if constexpr (V == 1) {
          o.set(0, y[0]);
        } else {
#pragma unroll
          for (int v = 0; v < V; v += 2) o.set2(v, y[v], y[v + 1]);
        }
        char* q = wh.next();
        if (h.p && at.on) o.store(q);
      }
    } else {
#pragma unroll
      for (int k = 0; k < S; ++k) {
        if (k % kSeg == 0) save(k);
        Vec<E, V> o;
#pragma unroll
        for (int v = 0; v < V; ++v) {
          y[v] = apply(da[k * V + v], y[v], b[k * V + v]);
          o.set(v, t0 + k < at.len ? y[v] : 0.0f);
        }
        char* q = wh.next();
        if (h.p && at.on && t0 + k < a.T) o.store(q);
      }
    }
    if (WT == 1 && !kCluster) {
#pragma unroll
      for (int v = 0; v < V; ++v) carry[v] = y[v];
    }
  }
  if (kRing) R::template wait<0>();
  X::finish(sh, lost);
  if (h_last && at.on && seg == 0) {
#pragma unroll
    for (int v = 0; v < V; ++v) h_last[me + v] = carry[v];
  }
}

struct GlrGrad {
  const float* ckpt;
  Seq dh;
  const float* dh_last;
  Seq dx, dr, di;
  float* dh0;
  float* part;  // [segments of a window][N][D] sums of w over a thread's steps
};

// kRing as in glr_fwd; 0: loaded when needed, which other warps cover.
// Reads x, r, i, dh and a checkpoint, writes dx, dr, di: 14.5 bytes an element in bf16 at about 67
// instructions, so issue slots (70 %) and memory bound it together (128 x 4096 x 128 bf16 170 us,
// 5.5 TB/s); split fp32 passes wait for their windows too (4096 x 8 x 512 100 us, 4.2 TB/s).  With
// decay exponents beyond 1/4 194 and 106 us.
template <typename E, int V, int WT, int kWarps, bool kCluster, int kRing>
__global__ void __launch_bounds__(32 * kWarps, 16 / kWarps)
    glr_bwd(const __grid_constant__ GlrDev a, const __grid_constant__ GlrGrad b, int n_rank, Waits waits) {
  tc::after_previous();
  using X = Exchange<V, WT, kCluster>;
  __shared__ typename X::Shared sh;
  constexpr int S = kSeg, WL = kWarps / WT, kE = S * V;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, wt = warp % WT;
  const int rank = kCluster ? (int)(blockIdx.x % n_rank) : 0;
  const int tiles = (a.D + 32 * V - 1) / (32 * V);
  const int64_t unit = (int64_t)(kCluster ? blockIdx.x / n_rank : blockIdx.x) * WL + warp / WT;
  const Place at(a, unit, tiles, lane, V, unit < a.N * tiles);
  const int64_t lanes = a.N * a.D, me = at.n * a.D + at.d;
  const int n_seg = (kCluster ? n_rank : 1) * WT, seg = rank * WT + wt;  // seg 0: the latest steps
  const int64_t window = (int64_t)n_seg * S;
  X::init(sh);
  const int64_t last = (a.T + window - 1) / window * window - (int64_t)(seg + 1) * S;  // its first t0

  float m[V], carry[V], sum[V], comp[V];
  bool small = true;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    m[v] = at.on ? -kGateScale * softplus_f(a.lam[at.d + v]) : 0.0f;
    small = small && m[v] > -0.25f;
    carry[v] = at.on && b.dh_last ? b.dh_last[me + v] : 0.0f;
    sum[v] = comp[v] = 0.0f;
  }
  small = __all_sync(0xFFFFFFFFu, small);
  Vec<E, V> nx[S], nr[S], ni[S], ng[S];
  float nc[V];
  uint8_t nrs = 0;
  using R = Ring<4, S, V * (int)sizeof(E), 128 * V>;  // and the checkpoint
  extern __shared__ __align__(128) uint8_t ring_smem[];
  uint8_t* ring = ring_smem + (kRing ? warp * kRing * R::kStage : 0);
  const bool any = unit < a.N * tiles, chunk = any && at.d - lane * V + lane % R::kChunks * (16 / (int)sizeof(E)) < a.D;
  int slot = 0;
  const E* px = static_cast<const E*>(a.x.p) + at.n * a.x.sn + at.d;
  const E* pr = static_cast<const E*>(a.r.p) + at.n * a.r.sn + at.d;
  const E* pi = static_cast<const E*>(a.i.p) + at.n * a.i.sn + at.d;
  const E* pg = static_cast<const E*>(b.dh.p) + at.n * b.dh.sn + at.d;
  const E* pdx = static_cast<const E*>(b.dx.p) + at.n * b.dx.sn + at.d;
  const E* pdr = static_cast<const E*>(b.dr.p) + at.n * b.dr.sn + at.d;
  const E* pdi = static_cast<const E*>(b.di.p) + at.n * b.di.sn + at.d;
  auto fetch_ring = [&](int64_t t0, int to) {  // (t0 < 0: before the first step, nothing is copied)
    uint8_t* dst = ring + to * R::kStage;
    const int64_t left = t0 < 0 ? 0 : at.len - t0;
    R::rows(dst, 0, a.r, pr - lane * V, sizeof(E), t0, left, lane, chunk);
    R::rows(dst, 1, a.i, pi - lane * V, sizeof(E), t0, left, lane, chunk);
    R::rows(dst, 2, a.x, px - lane * V, sizeof(E), t0, left, lane, chunk);
    if (b.dh.p) R::rows(dst, 3, b.dh, pg - lane * V, sizeof(E), t0, left, lane, chunk);
    // 32 V floats, 4 a lane (V = 1: lanes 0..7)
    const int64_t d4 = at.d - lane * V + 4 * lane;
    const bool on = any && lane < 8 * V && d4 < a.D && left > 0;
    if (lane < 8 * V)
      R::copy16(dst + 4 * S * R::kRow + lane * 16, on ? b.ckpt + (t0 / kSeg) * lanes + at.n * a.D + d4 : b.ckpt, on);
    R::commit();
  };
  auto fetch = [&](int64_t t0) {
    Walk wr(a.r, pr, sizeof(E), t0), wi(a.i, pi, sizeof(E), t0), wx(a.x, px, sizeof(E), t0), wg(b.dh, pg, sizeof(E), t0);
#pragma unroll
    for (int v = 0; v < V; ++v) nc[v] = at.on && t0 < at.len ? __ldcs(b.ckpt + (t0 / kSeg) * lanes + me + v) : 0.0f;
#pragma unroll
    for (int k = 0; k < S; ++k) {
      nx[k].zero();
      nr[k].zero();
      ni[k].zero();
      ng[k].zero();
      const char *qr = wr.next(), *qi = wi.next(), *qx = wx.next(), *qg = wg.next();
      if (at.on && t0 + k < at.len) {
        nr[k].load(qr);
        ni[k].load(qi);
        nx[k].load(qx);
        if (b.dh.p) ng[k].load(qg);
      }
    }
    nrs = reset_byte<S>(a, at, t0, lane);
  };
  if (kRing && a.T > 0) {
#pragma unroll
    for (int w = 0; w < kRing; ++w) fetch_ring(last - w * window, w);
    nrs = reset_byte<S>(a, at, last, lane);
  }
  uint32_t n = 0, lost = ~0u;  // windows so far, see Exchange
  for (int64_t t0 = last, w = (a.T + window - 1) / window; w > 0; --w, t0 -= window, ++n) {
    // Ring: one channel a thread has room for the whole segment, and the slot is refilled as soon
    // as it is read; two read x and dh from the slot where they are used, and refill it last.
    const uint8_t* src = ring + slot * R::kStage + lane * V * (int)sizeof(E);
    using W = typename Vec<E, V>::W;
    if (kRing) {
      R::template wait<(kRing > 0 ? kRing - 1 : 0)>();
#pragma unroll
      for (int k = 0; k < S; ++k) {
        nr[k].w = *reinterpret_cast<const W*>(src + k * R::kRow);
        ni[k].w = *reinterpret_cast<const W*>(src + (S + k) * R::kRow);
        if (V == 1) {
          nx[k].w = *reinterpret_cast<const W*>(src + (2 * S + k) * R::kRow);
          ng[k].w = *reinterpret_cast<const W*>(src + (3 * S + k) * R::kRow);
          if (!b.dh.p) ng[k].zero();
        }
      }
#pragma unroll
      for (int v = 0; v < V; ++v) nc[v] = reinterpret_cast<const float*>(ring + slot * R::kStage + 4 * S * R::kRow)[lane * V + v];
    } else {
      fetch(t0);
    }
    auto x_of = [&](int k) {
      if (!kRing || V == 1) return nx[k];
      Vec<E, V> q;
      q.w = *reinterpret_cast<const W*>(src + (2 * S + k) * R::kRow);
      return q;
    };
    auto g_of = [&](int k) {
      if (!kRing || V == 1) return ng[k];
      Vec<E, V> q;
      q.w = *reinterpret_cast<const W*>(src + (3 * S + k) * R::kRow);
      if (!b.dh.p) q.zero();
      return q;
    };
    float kept[kE], rho[kE], iota[kE], prev[kE], p[V];  // kept: of the decay, see Decay
    float A[V], P[V];
    const uint32_t rs = __ballot_sync(0xFFFFFFFFu, nrs != 0);
    const bool plain = rs == 0 && t0 + S <= at.len;  // no masks needed
#pragma unroll
    for (int v = 0; v < V; ++v) p[v] = nc[v];
    auto refill = [&]() {
      __syncwarp();                       // every lane has read the slot
      fetch_ring(t0 - kRing * window, slot);
      slot = slot + 1 == kRing ? 0 : slot + 1;
    };
    // gates (prev holds beta iota x until the states are rebuilt), the states, the segment's map
    auto rebuild = [&](auto small_c) {
      constexpr bool kSmall = decltype(small_c)::value;
#pragma unroll
      for (int e = 0; e < kE; e += 2) {
        const int k0 = e / V, v0 = e % V, k1 = (e + 1) / V, v1 = (e + 1) % V;
        const uint64_t rh = sigmoid2(tc::f2_pack(nr[k0].get(v0), nr[k1].get(v1)));
        const Decay q = decay<kSmall>(tc::f2_mul(tc::f2_pack(m[v0], m[v1]), rh));
        const uint64_t io = sigmoid2(tc::f2_pack(ni[k0].get(v0), ni[k1].get(v1)));
        float b0, b1;
        tc::f2_unpack(beta_sq(q.em), b0, b1);
        const uint64_t ix = tc::f2_mul(io, tc::f2_pack(x_of(k0).get(v0), x_of(k1).get(v1)));
        tc::f2_unpack(tc::f2_mul(tc::f2_pack(sqrt_q(b0), sqrt_q(b1)), ix), prev[e], prev[e + 1]);
        tc::f2_unpack(rh, rho[e], rho[e + 1]);
        tc::f2_unpack(io, iota[e], iota[e + 1]);
        tc::f2_unpack(q.kept, kept[e], kept[e + 1]);
      }
      if (kRing) {
        nrs = w > 1 ? reset_byte<S>(a, at, t0 - window, lane) : (uint8_t)0;
        if (V == 1) refill();
      }
#pragma unroll
      for (int e = 0; e < kE; ++e) {
        const int k = e / V, v = e % V;
        const float in = prev[e];
        if (!plain && ((rs >> k) & 1u)) p[v] = 0.0f;
        prev[e] = p[v];
        p[v] = fmaf(p[v], kept_a<kSmall>(kept[e]), in);  // (the forward pass's own bits)
      }
      if (WT == 1 && !kCluster) return;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        A[v] = 1.0f;
        P[v] = 0.0f;
      }
#pragma unroll
      for (int e = kE - 1; e >= 0; --e) {
        const int k = e / V, v = e % V;
        const float d = kept_a<kSmall>(kept[e]);
        if (plain) {
          P[v] = d * (g_of(k).get(v) + P[v]);
          A[v] *= d;
        } else if (t0 + k < at.len) {
          const bool cut = (rs >> k) & 1u;
          P[v] = cut ? 0.0f : d * (g_of(k).get(v) + P[v]);
          A[v] *= d;
        }
      }
#pragma unroll
      for (int v = 0; v < V; ++v) A[v] = rs ? 0.0f : not_zero(A[v]);
    };
    if (small) rebuild(std::true_type());
    else rebuild(std::false_type());
    if (WT > 1 || kCluster) {
      X::run(sh, waits, lost, n, rank, n_rank, wt, lane, A, P, carry, p);
    } else {
#pragma unroll
      for (int v = 0; v < V; ++v) p[v] = carry[v];
    }
    float part[V];
#pragma unroll
    for (int v = 0; v < V; ++v) part[v] = 0.0f;
    Walk wdx(b.dx, pdx, sizeof(E), t0 + S - 1), wdr(b.dr, pdr, sizeof(E), t0 + S - 1), wdi(b.di, pdi, sizeof(E), t0 + S - 1);
    auto grads = [&](auto plain_c, auto small_c) {
      constexpr bool kPlain = decltype(plain_c)::value, kSmall = decltype(small_c)::value;
#pragma unroll
      for (int e = kE - 2; e >= 0; e -= 2) {
        const int k0 = e / V, v0 = e % V, k1 = (e + 1) / V, v1 = (e + 1) % V;
        // With G = dL/dh: dx = c1 G, di = c2 dx, w = -q a dL/da = c3 G, dr = c4 w, all but G
        // known before the scan.  1 / beta stays finite where beta = 0 (dx is 0 there, and
        // q / beta -> 0 with q).
        const float d0 = kept_a<kSmall>(kept[e]), d1 = kept_a<kSmall>(kept[e + 1]);
        const uint64_t z = kept_m1<kSmall>(tc::f2_pack(kept[e], kept[e + 1])), rh = tc::f2_pack(rho[e], rho[e + 1]);
        const uint64_t io = tc::f2_pack(iota[e], iota[e + 1]), xx = tc::f2_pack(x_of(k0).get(v0), x_of(k1).get(v1));
        const uint64_t d = tc::f2_pack(d0, d1), b2 = beta_sq(z);
        float s0, s1;
        tc::f2_unpack(b2, s0, s1);
        const uint64_t inv = tc::f2_pack(rsqrt_q(fmaxf(s0, 1e-37f)), rsqrt_q(fmaxf(s1, 1e-37f)));
        const uint64_t c1 = tc::f2_mul(io, tc::f2_mul(b2, inv)), c2 = tc::f2_mul(xx, tc::f2_fma(io, both(-1.0f), both(1.0f)));
        const uint64_t nq = tc::f2_mul(tc::f2_pack(m[v0], m[v1]), rh);  // -q
        const uint64_t c3 = tc::f2_mul(tc::f2_mul(d, nq),
                                       tc::f2_sub(tc::f2_pack(prev[e], prev[e + 1]), tc::f2_mul(tc::f2_mul(inv, d), tc::f2_mul(io, xx))));
        const uint64_t c4 = tc::f2_fma(rh, both(-1.0f), both(1.0f));
        const bool live0 = kPlain || t0 + k0 < at.len, live1 = kPlain || t0 + k1 < at.len;
        const bool cut0 = !kPlain && ((rs >> k0) & 1u), cut1 = !kPlain && ((rs >> k1) & 1u);
        // the scan: element e + 1 is a later step (V = 1) or another channel
        const float G1 = g_of(k1).get(v1) + p[v1];
        p[v1] = live1 ? (cut1 ? 0.0f : d1 * G1) : p[v1];
        const float G0 = g_of(k0).get(v0) + p[v0];
        p[v0] = live0 ? (cut0 ? 0.0f : d0 * G0) : p[v0];
        const uint64_t G = tc::f2_pack(G0, G1), dx = tc::f2_mul(G, c1), w = tc::f2_mul(G, c3);
        float a0, a1, b0, b1, e0, e1, w0, w1;
        tc::f2_unpack(dx, a0, a1);
        tc::f2_unpack(tc::f2_mul(w, c4), b0, b1);
        tc::f2_unpack(tc::f2_mul(dx, c2), e0, e1);
        tc::f2_unpack(w, w0, w1);
        if (!kPlain) {
          if (!live0) a0 = b0 = e0 = w0 = 0.0f;
          if (!live1) a1 = b1 = e1 = w1 = 0.0f;
        }
        part[v1] += w1;
        part[v0] += w0;
        Vec<E, V> ox, orr, oi;
        if constexpr (V == 1) {
          Vec<E, V> px1, pr1, pi1;
          px1.set(0, a1);
          pr1.set(0, b1);
          pi1.set(0, e1);
          char *qx = wdx.next_back(), *qr = wdr.next_back(), *qi = wdi.next_back();
          if (at.on && (kPlain || t0 + k1 < a.T)) {
            px1.store(qx);
            pr1.store(qr);
            pi1.store(qi);
          }
          ox.set(0, a0);
          orr.set(0, b0);
          oi.set(0, e0);
        } else {
          static_assert(V <= 2, "a pair is a row");
          ox.set2(v0, a0, a1);
          orr.set2(v0, b0, b1);
          oi.set2(v0, e0, e1);
        }
        char *qx = wdx.next_back(), *qr = wdr.next_back(), *qi = wdi.next_back();
        if (at.on && (kPlain || t0 + k0 < a.T)) {
          ox.store(qx);
          orr.store(qr);
          oi.store(qi);
        }
      }
    };
    if (small) {
      if (plain) grads(std::true_type(), std::true_type());
      else grads(std::false_type(), std::true_type());
    } else {
      if (plain) grads(std::true_type(), std::false_type());
      else grads(std::false_type(), std::false_type());
    }
    if (kRing && V > 1) refill();
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const float yk = part[v] - comp[v], sk = sum[v] + yk;  // compensated over the segments
      comp[v] = (sk - sum[v]) - yk;
      sum[v] = sk;
      if (WT == 1 && !kCluster) carry[v] = p[v];
    }
  }
  if (kRing) R::template wait<0>();
  X::finish(sh, lost);
  if (!at.on) return;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    if (b.part) b.part[seg * lanes + me + v] = -sum[v];
    if (b.dh0 && seg == 0) b.dh0[me + v] = carry[v];
  }
}

// Sums over rows of part[rows][D] in a fixed order: CTA (x, y) takes 32 channels and the
// rows y, y + gridDim.y, ... ; 32 row-threads per channel, then a tree.  kLast also applies
// dlam[d] = -sum sigmoid(lam) / softplus(lam) (the ratio tends to 1 as lam -> -inf).  part is
// written while CTAs of this kernel already wait in after_previous(), so it is read by ordinary
// loads: no __restrict__, which would let them go through the read-only path.
// Latency: 6 + 5 us for 4096 rows of 128 in two passes, one alone 24.
template <bool kLast>
__global__ void glr_dlam(const float* part, int64_t rows, int32_t D, const float* lam, float* out) {
  tc::after_previous();
  __shared__ float sh[32][33];
  const int d = blockIdx.x * 32 + threadIdx.x;
  float sum = 0.0f, comp = 0.0f;
  if (d < D)
    for (int64_t r = blockIdx.y * 32 + threadIdx.y; r < rows; r += 32 * gridDim.y) {
      const float yk = part[r * D + d] - comp, sk = sum + yk;
      comp = (sk - sum) - yk;
      sum = sk;
    }
  sh[threadIdx.y][threadIdx.x] = sum;
  for (int k = 16; k > 0; k >>= 1) {
    __syncthreads();
    if (threadIdx.y < k) sh[threadIdx.y][threadIdx.x] += sh[threadIdx.y + k][threadIdx.x];
  }
  if (threadIdx.y == 0 && d < D) {
    float v = sh[0][threadIdx.x];
    if (kLast) {
      const float l = lam[d], sp = softplus_f(l);
      v = -v * (sp > 0.0f ? sigmoid_f(l) / sp : 1.0f);
    }
    out[(int64_t)blockIdx.y * D + d] = v;
  }
}

// Whether every one of these addresses is a multiple of its elements' size (a kernel's access to another
// faults).
template <typename... P>
bool elements_of(uintptr_t size, const P*... p) {
  return ((reinterpret_cast<uintptr_t>(p) | ... | uintptr_t(0)) & (size - 1)) == 0;
}
constexpr char kMisaligned[] = "an address is not a multiple of its elements' size";

aht_status check(const aht_glr_args* a) {
  if (!a) return set_last_error(AHT_EINVAL, "args is NULL");
  if (a->dtype != AHT_FP32 && a->dtype != AHT_BF16)
    return set_last_error(AHT_EINVAL, "dtype must be AHT_FP32 or AHT_BF16");
  if (a->T < 0 || a->N < 1 || a->D < 1 || a->D > AHT_GLR_MAX_D)
    return set_last_error(AHT_EINVAL, "sizes: T >= 0, N >= 1, 1 <= D <= AHT_GLR_MAX_D");
  if (a->N > (int64_t(1) << 37) / a->D || (a->T > 0 && a->N > (int64_t(1) << 46) / a->D / a->T))
    return set_last_error(AHT_EINVAL, "N * D must be at most 2^37 and T * N * D at most 2^46");
  if (a->N > (int64_t(1) << 32) / ((a->D + 31) / 32))  // CTAs of a launch
    return set_last_error(AHT_EINVAL, "N * ceil(D / 32) must be at most 2^32");
  if (!a->lam) return set_last_error(AHT_EINVAL, "lam is NULL");
  if (a->T > 0 && (!a->x.data || !a->r.data || !a->i.data)) return set_last_error(AHT_EINVAL, "NULL input sequence");
  if (!elements_of(a->dtype == AHT_FP32 ? 4 : 2, a->x.data, a->r.data, a->i.data) || !elements_of(4, a->lam, a->lengths))
    return set_last_error(AHT_EINVAL, kMisaligned);
  return AHT_OK;
}

Seq seq(const aht_seq& s) { return Seq{s.data, s.st, s.sn}; }
GlrDev dev(const aht_glr_args* a) {
  return GlrDev{a->D, a->T, a->N, seq(a->x), seq(a->r), seq(a->i), a->lam, a->reset, a->lengths};
}

aht_status launched(cudaError_t e) {
  return e == cudaSuccess ? AHT_OK : set_last_error(AHT_ECUDA, cudaGetErrorString(e));
}

// Whether V channels of every row of a sequence start on a boundary of their size.
bool aligned(const Seq& s, int esz, int V, int64_t T, int64_t N) {
  const uintptr_t bytes = (uintptr_t)esz * V;
  return !s.p || ((uintptr_t)s.p % bytes == 0 && (T <= 1 || s.st % V == 0) && (N <= 1 || s.sn % V == 0));
}

// How the lanes and steps of a call are split.
struct Split {
  int wt, cl;      // warps of a CTA and CTAs of a cluster along time
  int64_t units;   // groups of 32 V lanes of one env
  int segs() const { return wt * cl; }
};

// Warps that keep every SM's loads in flight.  A pass with fewer groups than a share of them has its
// steps split, unless it is so short that the windows' hand-overs cost more than the loads gain.
constexpr int kFill = 152 * 12;
// Clusters of n CTAs of a split pass that a GB300 holds at once, two CTAs an SM (as the occupancy
// query answers for the forward kernel; only speed depends on it, so other split kernels, and later
// ones with other registers or shared memory, go by the same numbers).  The largest cluster at which
// every group's is resident is the quickest (65537 x 1 x 896 fp32, 28 groups, forward: 8 CTAs 206 us,
// 9 183, 10 172; 20000 x 2 x 256, 16 groups: 8 66 us, 12 53, 16 in two waves 65).
constexpr int kResident[kMaxCluster + 1] = {0, 304, 152, 97, 74, 58, 46, 38, 36, 30, 28, 23, 23, 19, 14, 14, 14};

Split split_of(int64_t T, int64_t N, int32_t D, int V, int fill) {
  Split p{1, 1, N * ((D + 32 * V - 1) / (32 * V))};
  if (p.units >= fill || T <= 2 * kSeg) return p;
  p.wt = 8;
  for (int cl = 2; cl <= kMaxCluster; ++cl)
    if (p.units <= kResident[cl] && (int64_t)p.wt * cl * kSeg <= T) p.cl = cl;
  return p;
}

// Split / whole, us, by groups.  fp32 (groups of two channels; where these are too few, whole passes
// take one): 100 steps 300 groups 12 / 14, 456 15 / 16, 900 28 / 23; 400 steps 600 62 / 70, 1200 110 / 92;
// 1000 steps 900 166 / 216, 1824 322 / 298.  bf16, two channels: 100 steps 600 14 / 14, 1200 26 / 25; 400
// steps 900 58 / 88, 1600 98 / 100; 1000 steps 1200 149 / 227, 2400 289 / 264.  The rule is off by a
// quarter to a third between its points at 200 to 400 steps of bf16 (200 steps, 900 groups: 33 / 44,
// whole) and for 1000 steps of fp32 with 1200 to 1824 groups of two (1600: 288 split, 272 whole; its one
// channel takes 370).
Split split_fwd(int64_t T, int64_t N, int32_t D, int V) {
  return split_of(T, N, D, V, (int)std::min<int64_t>(std::max<int64_t>(3 * T, kFill / 3), kFill));
}
// One channel a thread, split / whole, us without dlam: 100 x 57 x 256 (456 groups) fp32 14 / 13, bf16
// 14 / 15; 400 x 76 x 256 46 / 44, 41 / 43; 1000 x 76 x 256 100 / 102, 85 / 102; 1000 x 150 x 256 184 / 185,
// 163 / 185.  Two channels are for whole passes that one would not fill (see the dispatch).
Split split_bwd(int64_t T, int64_t N, int32_t D, int V) {
  return split_of(T, N, D, V, V > 1 ? kFill : (int)std::min<int64_t>(std::max<int64_t>(T, kFill / 4), kFill / 2));
}

template <typename K, typename... Args>
aht_status launch(K kernel, dim3 grid, dim3 block, int cl, int smem, cudaStream_t s, Args... args) {
  if (smem > 16 * 1024)  // (with the static part it may pass 48 KB)
    if (aht_status e = launched(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem))) return e;
  if (cl > 8)  // beyond what every device runs
    if (aht_status e = launched(cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1))) return e;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(grid.x * (unsigned)cl, grid.y);
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = (size_t)smem;
  cfg.stream = s;
  // (128 x 4096 x 128 bf16 forward + backward 281 us, 288 without; 4096 x 8 x 512 152, 157)
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;  // see tc::after_previous()
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim = {(unsigned)cl, 1, 1};
  cfg.attrs = attr;
  cfg.numAttrs = cl > 1 ? 2 : 1;
  return launched(cudaLaunchKernelEx(&cfg, kernel, args...));
}

// The failure hook (aht_debug_glr_expire): taken by the next pass that is split over a cluster.
constexpr uint64_t kWaitNs = 2000000000ull;
std::atomic<uint64_t> g_expire{0};     // 0: off, else window << 32 | limit_ns
Waits clustered_waits() {
  const uint64_t hook = g_expire.exchange(0);
  return hook ? Waits{hook & 0xFFFFFFFFu, (uint32_t)(hook >> 32)} : Waits{kWaitNs, ~0u};
}
constexpr Waits kNoWaits{kWaitNs, ~0u};

// Many lanes (or T = 1): a warp per group of 32 V lanes.
template <typename E, int V, int S, int kRing>
aht_status forward_wide(const aht_glr_args* a, const float* h0, const Seq& h, float* h_last, float* ckpt, cudaStream_t s) {
  const int64_t four = (split_fwd(a->T, a->N, a->D, V).units + 3) / 4;
  constexpr int kSmem = 4 * kRing * Ring<3, 8, V * (int)sizeof(E), 0>::kStage;
  static_assert(kRing == 0 || S == 8, "");
  return launch(glr_fwd<E, V, S, 1, 4, false, kRing>, dim3((unsigned)four), dim3(128), 1, kSmem, s, dev(a), h0, h, h_last, ckpt, 1,
                kNoWaits);
}
// Few lanes: 8 warps and p.cl CTAs along time.
template <typename E, int V, int S, int kRing>
aht_status forward_long(const aht_glr_args* a, const Split& p, const float* h0, const Seq& h, float* h_last, float* ckpt,
                        cudaStream_t s) {
  constexpr int kSmem = 8 * kRing * Ring<3, S, V * (int)sizeof(E), 0>::kStage;
  if (p.cl == 1)
    return launch(glr_fwd<E, V, S, 8, 8, false, kRing>, dim3((unsigned)p.units), dim3(256), 1, kSmem, s, dev(a), h0, h, h_last,
                  ckpt, 1, kNoWaits);
  return launch(glr_fwd<E, V, S, 8, 8, true, kRing>, dim3((unsigned)p.units), dim3(256), p.cl, kSmem, s, dev(a), h0, h, h_last,
                ckpt, p.cl, clustered_waits());
}

template <typename E, int V, bool kRows>  // kRows: rows aligned for the ring
aht_status backward(const aht_glr_args* a, const GlrGrad& g, int* rows, cudaStream_t s) {
  const Split p = split_bwd(a->T, a->N, a->D, V);
  const GlrDev d = dev(a);
  *rows = p.segs();
  constexpr int kStage = Ring<4, kSeg, V * (int)sizeof(E), 128 * V>::kStage, kWide = kRows ? 2 : 0, kLong = kRows ? 3 : 0;
  if (V > 1 || p.wt == 1)
    return launch(glr_bwd<E, V, 1, 4, false, kWide>, dim3((unsigned)((p.units + 3) / 4)), dim3(128), 1, 4 * kWide * kStage, s,
                  d, g, 1, kNoWaits);
  if constexpr (V == 1) {
    if (p.cl == 1)
      return launch(glr_bwd<E, V, 8, 8, false, kLong>, dim3((unsigned)p.units), dim3(256), 1, 8 * kLong * kStage, s, d, g, 1,
                    kNoWaits);
    return launch(glr_bwd<E, V, 8, 8, true, kLong>, dim3((unsigned)p.units), dim3(256), p.cl, 8 * kLong * kStage, s, d, g, p.cl,
                  clustered_waits());
  }
  return AHT_EINVAL;  // (V > 1 is wide)
}

constexpr int kSumRows = 64;  // row groups of the first pass of dlam's sum

int64_t part_floats(int64_t T, int64_t N, int32_t D) {
  return (int64_t)std::max(split_bwd(T, N, D, 1).segs(), split_bwd(T, N, D, 2).segs()) * N * D;
}

}  // namespace

extern "C" {

int64_t aht_glr_ckpt_elems(int64_t T, int64_t N, int32_t D) {
  return T < 0 || N < 0 || D < 0 ? 0 : (T + kSeg - 1) / kSeg * N * D;
}

int64_t aht_glr_workspace(int64_t T, int64_t N, int32_t D) {
  return T < 0 || N < 1 || D < 1 ? 0 : (part_floats(T, N, D) + (int64_t)kSumRows * D) * (int64_t)sizeof(float);
}

aht_status aht_glr_forward(const aht_glr_args* a, const float* h0, const aht_seq* h, float* h_last, float* ckpt,
                           void* cuda_stream) {
  if (aht_status e = check(a)) return e;
  const Seq out = h ? seq(*h) : Seq{nullptr, 0, 0};
  if (!out.p && !h_last) return set_last_error(AHT_EINVAL, "neither h nor h_last is asked for");
  const cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  const int esz = a->dtype == AHT_FP32 ? 4 : 2;
  if (!elements_of(esz, out.p) || !elements_of(4, h0, h_last, ckpt)) return set_last_error(AHT_EINVAL, kMisaligned);
  auto fits = [&](int V) {
    return a->D % V == 0 && aligned(seq(a->x), esz, V, a->T, a->N) && aligned(seq(a->r), esz, V, a->T, a->N) &&
           aligned(seq(a->i), esz, V, a->T, a->N) && aligned(out, esz, V, a->T, a->N);
  };
  // groups of 32 V channels that leave at most one thread in `of` without channels
  auto fills = [&](int V, int of) { return (a->D + 32 * V - 1) / (32 * V) * 32 * V <= a->D + a->D / of; };
  const bool rows = fits(16 / esz);      // every row a whole number of aligned 16-byte chunks
  auto wide = [&](int V) { return split_fwd(a->T, a->N, a->D, V).wt == 1; };
  // Wide passes, us for 128 steps (fp32 8192 x 128, bf16 16384 x 128; copies alone take 317): two
  // channels a thread through the ring 305 / 358, two in registers 312 / 420 (four in registers, of an
  // earlier form, 333 / 394).  The ring wants aligned rows, two channels a well-filled warp.
  if (a->dtype == AHT_FP32) {
    if (a->T <= 1)
      return fits(4) ? forward_wide<float, 4, 1, 0>(a, h0, out, h_last, ckpt, s)
                     : forward_wide<float, 1, 2, 0>(a, h0, out, h_last, ckpt, s);
    if (fits(2) && fills(2, 3) && wide(2))
      return rows ? forward_wide<float, 2, kSeg, 2>(a, h0, out, h_last, ckpt, s)
                  : forward_wide<float, 2, kSeg, 0>(a, h0, out, h_last, ckpt, s);
    if (wide(1)) return forward_wide<float, 1, kSeg, 0>(a, h0, out, h_last, ckpt, s);
    const Split p = split_fwd(a->T, a->N, a->D, 1);
    return rows ? forward_long<float, 1, 2 * kSeg, 2>(a, p, h0, out, h_last, ckpt, s)
                : forward_long<float, 1, 2 * kSeg, 0>(a, p, h0, out, h_last, ckpt, s);
  }
  if (a->T <= 1)
    return fits(4)   ? forward_wide<__nv_bfloat16, 4, 1, 0>(a, h0, out, h_last, ckpt, s)
           : fits(2) ? forward_wide<__nv_bfloat16, 2, 1, 0>(a, h0, out, h_last, ckpt, s)
                     : forward_wide<__nv_bfloat16, 1, 2, 0>(a, h0, out, h_last, ckpt, s);
  if (fits(2)) {
    if (wide(2))
      return rows ? forward_wide<__nv_bfloat16, 2, kSeg, 2>(a, h0, out, h_last, ckpt, s)
                  : forward_wide<__nv_bfloat16, 2, kSeg, 0>(a, h0, out, h_last, ckpt, s);
    // One channel a thread while that leaves every CTA resident (65537 x 1 x 896: 173 us against 220
    // with two), two beyond (1000 x 150 x 256: 78 against 88).
    const Split one = split_fwd(a->T, a->N, a->D, 1);
    if (rows && one.units <= kResident[1])
      return forward_long<__nv_bfloat16, 1, 2 * kSeg, 2>(a, one, h0, out, h_last, ckpt, s);
    const Split p = split_fwd(a->T, a->N, a->D, 2);
    return rows ? forward_long<__nv_bfloat16, 2, kSeg, 3>(a, p, h0, out, h_last, ckpt, s)
                : forward_long<__nv_bfloat16, 2, kSeg, 0>(a, p, h0, out, h_last, ckpt, s);
  }
  if (wide(1)) return forward_wide<__nv_bfloat16, 1, kSeg, 0>(a, h0, out, h_last, ckpt, s);
  return forward_long<__nv_bfloat16, 1, 2 * kSeg, 0>(a, split_fwd(a->T, a->N, a->D, 1), h0, out, h_last, ckpt, s);
}

aht_status aht_glr_backward(const aht_glr_args* a, const float* ckpt, const aht_seq* dh, const float* dh_last,
                            const aht_seq* dx, const aht_seq* dr, const aht_seq* di, float* dlam, float* dh0,
                            void* workspace, int64_t workspace_bytes, void* cuda_stream) {
  if (aht_status e = check(a)) return e;
  if (a->T > 0 && !ckpt) return set_last_error(AHT_EINVAL, "ckpt is NULL");
  if (a->T > 0 && (!dx || !dr || !di || !dx->data || !dr->data || !di->data))
    return set_last_error(AHT_EINVAL, "NULL gradient sequence");
  if (dlam && (!workspace || workspace_bytes < aht_glr_workspace(a->T, a->N, a->D)))
    return set_last_error(AHT_EINVAL, "workspace is NULL or smaller than aht_glr_workspace");
  const Seq none{nullptr, 0, 0};
  float* part = dlam ? static_cast<float*>(workspace) : nullptr;
  const GlrGrad g{ckpt,    dh ? seq(*dh) : none, dh_last, dx ? seq(*dx) : none, dr ? seq(*dr) : none,
                  di ? seq(*di) : none, dh0, part};
  const cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  const int esz = a->dtype == AHT_FP32 ? 4 : 2;
  if (!elements_of(esz, g.dh.p, g.dx.p, g.dr.p, g.di.p) || !elements_of(4, ckpt, dh_last, dlam, dh0, part))
    return set_last_error(AHT_EINVAL, kMisaligned);
  auto fits = [&](int V) {
    bool ok = a->D % V == 0;
    for (const Seq& q : {seq(a->x), seq(a->r), seq(a->i), g.dh, g.dx, g.dr, g.di}) ok = ok && aligned(q, esz, V, a->T, a->N);
    return ok;
  };
  // every row a whole number of aligned 16-byte chunks (and the checkpoints' rows)
  const bool rows_16 = fits(16 / esz) && (uintptr_t)ckpt % 16 == 0;
  int segs = 1;
  aht_status e;
  if (a->dtype == AHT_FP32)
    e = rows_16 ? backward<float, 1, true>(a, g, &segs, s) : backward<float, 1, false>(a, g, &segs, s);
  // Two channels a thread while whole groups of them fill the SMs (128 x 16384 x 128: 631 us, one
  // channel 899), one below (1000 x 300 x 256, 1200 groups of two: 232 against 292).
  else if (fits(2) && split_bwd(a->T, a->N, a->D, 2).wt == 1)
    e = rows_16 ? backward<__nv_bfloat16, 2, true>(a, g, &segs, s) : backward<__nv_bfloat16, 2, false>(a, g, &segs, s);
  else
    e = rows_16 ? backward<__nv_bfloat16, 1, true>(a, g, &segs, s) : backward<__nv_bfloat16, 1, false>(a, g, &segs, s);
  if (e != AHT_OK || !dlam) return e;
  const int64_t rows = (int64_t)segs * a->N;
  const dim3 grid((a->D + 31) / 32), block(32, 32);
  if (rows <= 512) return launch(glr_dlam<true>, grid, block, 1, 0, s, part, rows, a->D, a->lam, dlam);
  float* first = part + part_floats(a->T, a->N, a->D);
  if ((e = launch(glr_dlam<false>, dim3(grid.x, kSumRows), block, 1, 0, s, part, rows, a->D, a->lam, first))) return e;
  return launch(glr_dlam<true>, grid, block, 1, 0, s, first, (int64_t)kSumRows, a->D, a->lam, dlam);
}

aht_status aht_glr_sync(void* cuda_stream) {
  if (aht_status e = launched(cudaStreamSynchronize(static_cast<cudaStream_t>(cuda_stream)))) return e;
  uint32_t st = 0;
  if (aht_status e = launched(cudaMemcpyFromSymbol(&st, glr_status, sizeof st))) return e;
  if (!st) return AHT_OK;
  const uint32_t none = 0;
  if (aht_status e = launched(cudaMemcpyToSymbol(glr_status, &none, sizeof none))) return e;
  return set_last_error(AHT_ETIMEOUT, "a bounded wait of a split recurrence expired");
}

aht_status aht_debug_glr_expire(int32_t window, int64_t limit_ns) {
  if (window >= 0 && (limit_ns < 1 || limit_ns > 1000000000))
    return set_last_error(AHT_EINVAL, "limit_ns must be in 1..1e9");
  g_expire = window < 0 ? 0 : (uint64_t)window << 32 | (uint64_t)limit_ns;
  return AHT_OK;
}

}  // extern "C"
