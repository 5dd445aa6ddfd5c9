// linattn.cu -- linear attention with a decay for each head over a collected trajectory
// (include/aht.h states the model): the pass over T steps, one serving step (T = 1) and the gradients.
//
// A chain is one head h of one env n with its state S [K][V]:
//   S <- g S (nothing of it where an episode begins) + k_t v_t^T,   o_t = scale S^T q_t.
// The gradients are chains of the same form.  With G the gradient of the state,
//   dq_t = scale S do_t            the same states, transposed:    (q, k, v) -> (do, v, k),
//   dv_t = G^T k_t,  dk_t = G v_t  from the last step to the first: (k, q, do) and (v, do, q),
// so every pass is one or three "walks" of one kernel, told apart by their operands and direction.
//
// walk: a warp owns up to 128 columns of a state, a thread one to four of them over KT of the K rows, in fp32
// registers, and goes through the steps one at a time: the products have no masked operand, so what is not finite
// reaches exactly the steps that the formulas give it to.  Rows of q, k and v come through a ring of asynchronous
// copies, eight steps a stage.  Per step and column 2 K multiply-adds (in pairs, an operand of which comes from shared
// memory once for a thread's columns); at 64x64 they are 128 of a warp's 318 instructions a step, and the issue of all
// of them bounds it.  Decays cost no instruction: within a window of W steps the state is kept times g^(W - 1 - j), never
// above its own size, so that it overflows where the result itself does.
//
// One step, the serving form, is a kernel of its own (`one_step`).
//
// Few chains: the steps are split into segments.  Each is an affine map of the state it receives,
// S -> A S + U: `walk` computes U from k and v alone, `hand_over` the state each segment receives,
// and `walk` runs every segment from there.
#include <cuda_bf16.h>

#include <algorithm>

#include "op_launch.cuh"

using namespace aht;

namespace {

constexpr int kWindow = 8;      // steps of a ring stage
constexpr int kStages = 2;
constexpr int kWarps = 4;       // of a CTA, each with a chain's columns of its own

struct Rows {                   // element (t, n, h, c) at p[t * st + n * sn + h * sh + c]
  void* p;
  int64_t st, sn, sh;
};

// One walk over the steps of every chain.
struct Walk {
  Rows q, k, v, o;              // o.p NULL: states alone
  int32_t K, V;                 // columns of q and k; of v and o
  int32_t back;                 // 1: from the last step to the first
  float in, out;                // factors of v and of o
  // states [N][H][K * V], element (i, j) at i * si + j * sj (NULL: zeros / not written)
  const float* s_in;
  float* s_out;
  int64_t si_in, sj_in;
  float* seg;                   // split: [segments][N][H][K][V], received states (and U before hand_over)
};

struct Chains {
  int64_t T, N;
  int32_t H, walks;
  const float* log_decay;
  const uint8_t* reset;
  const int32_t* lengths;
  int64_t seg_len;              // steps of a segment
  int32_t segs;
  int32_t* seg_live;            // split: [segs][N] live steps of a segment, -1 where an episode begins in it
  Walk w[3];
  // `chunks`: the walks' blocks of columns, by number
  int32_t parts;
  uint8_t part_walk[6], part_block[6];
};

template <typename E> __device__ __forceinline__ float as_f32(E v);
template <> __device__ __forceinline__ float as_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ float as_f32<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename E> __device__ __forceinline__ E rounded(float v);
template <> __device__ __forceinline__ float rounded<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 rounded<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

__device__ __forceinline__ void copy_16(void* dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(tc::smem_u32(dst)), "l"(src) : "memory");
}
__device__ __forceinline__ void copy_4(void* dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(tc::smem_u32(dst)), "l"(src) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kLeft> __device__ __forceinline__ void copies_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(kLeft) : "memory");
}

// log2 of a head's decay.  Below exp(-10^4) a decay is 0 in fp32 either way, and 0 * steps stays a number
// (log_decay = -inf).
__device__ __forceinline__ float log2_decay(const float* log_decay, int h) {
  const float l = log_decay[h];
  return (l < -1e4f ? -1e4f : l) * 1.4426950408889634f;
}

// KS threads share the K rows of COLS columns, KT each.  Shared memory of a warp: kStages of kWindow rows of q, k and v
// as they are in memory, and, where they are not fp32, one of q and k as fp32.  A thread's KT elements of a row are 16
// bytes apart from the next one's, so that the KS read different banks.
template <typename E, int KT, int KS, int COLS>
struct Plan {
  static constexpr int kKP = KT * KS, kRow = KS > 1 ? KS * (KT + 4) : KT, kVB = 32 / KS * COLS;
  static constexpr bool kRaw = sizeof(E) == 4;
  static constexpr int kRawRow = kRaw ? kRow : kKP;                       // elements of a staged row
  static constexpr int kStage = kWindow * (2 * kRawRow + kVB) * (int)sizeof(E);
  static constexpr int kConv = kRaw ? 0 : 2 * kWindow * kRow * 4, kTable = 2 * (kWindow + 4) * 4;
  static constexpr int kBytes = kStages * kStage + kConv + kTable;
};

// Rows of a walk in its order: row i at p + i * st (st < 0 from the last step to the first).
template <typename E> struct Line {
  const E* p;
  int64_t st;
  bool wide;                    // rows of whole 16-byte chunks
};
template <typename E>
__device__ __forceinline__ Line<E> line_of(const Rows& r, int64_t n, int h, int64_t t0, bool back, int c0, int width) {
  constexpr int kPer = 16 / (int)sizeof(E);
  const E* p = static_cast<const E*>(r.p) + n * r.sn + h * r.sh + t0 * r.st + c0;
  return {p, back ? -r.st : r.st, (uintptr_t)p % 16 == 0 && r.st % kPer == 0 && width % kPer == 0};
}
// Element k's place in a row that is staged with gaps of four elements every kGap (0: none).
template <int kGap> __device__ __forceinline__ int place(int k) { return kGap > 0 ? k + k / (kGap > 0 ? kGap : 1) * 4 : k; }
// Copies `count` rows from row i0 on into a stage.
template <typename E, int kGap>
__device__ __forceinline__ void fetch_rows(E* dst, int row, const Line<E>& l, int width, int i0, int count, int lane) {
  constexpr int kPer = 16 / (int)sizeof(E);
  if (l.wide) {
    const int per = width / kPer;
    int j = lane / per, k = (lane - j * per) * kPer;
    const int dj = 32 / per, dk = (32 - dj * per) * kPer;
    while (j < count) {
      copy_16(dst + j * row + place<kGap>(k), l.p + (i0 + j) * l.st + k);
      j += dj, k += dk;
      if (k >= width) ++j, k -= width;
    }
  } else {
    // Elements one by one: as asynchronous copies where they have four bytes, else a column of the window at a time
    // through registers, so that its loads are in flight together.  (A load, a store, a load and so on: 400x61x3 K 50
    // V 33 fp32 with its gradients 767 us, this way 400.)
    for (int k = lane; k < width; k += 32) {
      const E* r = l.p + i0 * l.st + k;
      E* d = dst + place<kGap>(k);
      if constexpr (sizeof(E) == 4) {
#pragma unroll
        for (int j = 0; j < kWindow; ++j)
          if (j < count) copy_4(d + j * row, r + j * l.st);
      } else {
        E x[kWindow];
#pragma unroll
        for (int j = 0; j < kWindow; ++j)
          if (j < count) x[j] = r[j * l.st];
#pragma unroll
        for (int j = 0; j < kWindow; ++j)
          if (j < count) d[j * row] = x[j];
      }
    }
  }
}

// kStates: a segment's U alone.  Four CTAs an SM where a thread has 64 elements of the state (with three, at 156
// registers, forward + backward of 400x61x3 50x33 fp32 took 372 us, so 330), two where it has 128.
template <typename E, int KT, int KS, int COLS, bool kStates>
__global__ void __launch_bounds__(32 * kWarps, KT * COLS > 64 ? 2 : 4) walk(const __grid_constant__ Chains c, int64_t units) {
  using P = Plan<E, KT, KS, COLS>;
  tc::after_previous();
  extern __shared__ __align__(16) unsigned char smem[];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int64_t u = (int64_t)blockIdx.x * kWarps + warp;
  if (u >= units) return;
  // unit -> segment, env, head, walk, block of columns (neighbours share rows)
  int blocks = (c.w[0].V + P::kVB - 1) / P::kVB;   // (walks of one call may have K and V exchanged)
  for (int i = 1; i < c.walks; ++i) blocks = max(blocks, (c.w[i].V + P::kVB - 1) / P::kVB);
  const int vb = (int)(u % blocks);
  u /= blocks;
  const int wi = (int)(u % c.walks);
  u /= c.walks;
  const int h = (int)(u % c.H);
  u /= c.H;
  const int64_t n = u % c.N;
  const int seg = (int)(u / c.N);
  const Walk& w = c.w[wi];
  if (vb * P::kVB >= w.V) return;

  unsigned char* mine = smem + (size_t)warp * P::kBytes;
  float* conv = reinterpret_cast<float*>(mine + kStages * P::kStage);     // fp32 rows of the present window
  const int part = lane % KS, col = lane / KS * COLS;
  const int c0 = vb * P::kVB + col, k0 = part * KT;                       // the thread's first column and row
  const int K = w.K, VB = min(P::kVB, w.V - vb * P::kVB);
  const bool back = w.back != 0;
  const int64_t len = c.lengths ? min((int64_t)max(c.lengths[n], 0), c.T) : c.T;
  const int64_t t_lo = min(len, (int64_t)seg * c.seg_len);
  const int steps = (int)(min(len, t_lo + c.seg_len) - t_lo);
  const int64_t t0 = back ? t_lo + steps - 1 : t_lo;                      // the walk's first step
  const int64_t chain = n * c.H + h, KV = (int64_t)w.K * w.V;
  const uint8_t* reset = c.reset ? c.reset + t0 * c.N + n : nullptr;      // of step i at i * rst
  const int64_t rst = back ? -c.N : c.N;

  const float l2 = log2_decay(c.log_decay, h);
  // Behind the j-th step of `win` steps the state is kept times g^(win - 1 - j), at most 2^-8 times itself: below 2^-118,
  // where fp32 has bits for no more than that, it loses some of its own.
  const int win = l2 < -4.f ? 1 : l2 < -2.f ? 2 : l2 < -1.f ? 4 : kWindow;

  // ---- the state received
  uint64_t S[COLS][KT / 2];
  const int64_t at_seg = ((int64_t)seg * c.N * c.H + chain) * KV;
  const float* s_in = kStates ? nullptr : c.segs > 1 ? w.seg + at_seg : w.s_in ? w.s_in + chain * KV : nullptr;
  if (kStates || !s_in) {
#pragma unroll
    for (int j = 0; j < COLS; ++j)
#pragma unroll
      for (int i = 0; i < KT / 2; ++i) S[j][i] = 0;
  } else {
    const int64_t si = c.segs > 1 ? w.V : w.si_in, sj = c.segs > 1 ? 1 : w.sj_in;
    s_in += k0 * si + c0 * sj;
    if (COLS == 4 && sj == 1 && si % 4 == 0 && (uintptr_t)s_in % 16 == 0 && c0 + 4 <= w.V) {
#pragma unroll
      for (int i = 0; i < KT / 2; ++i) {
        const int k = k0 + 2 * i;
        const float4 z = {0.f, 0.f, 0.f, 0.f};
        const float4 a = k < K ? *reinterpret_cast<const float4*>(s_in + 2 * i * si) : z;
        const float4 b = k + 1 < K ? *reinterpret_cast<const float4*>(s_in + (2 * i + 1) * si) : z;
        S[0][i] = tc::f2_pack(a.x, b.x);
        S[COLS > 1 ? 1 : 0][i] = tc::f2_pack(a.y, b.y);
        S[COLS > 2 ? 2 : 0][i] = tc::f2_pack(a.z, b.z);
        S[COLS > 2 ? 3 : 0][i] = tc::f2_pack(a.w, b.w);
      }
    } else if (COLS == 2 && sj == 1 && si % 2 == 0 && (uintptr_t)s_in % 8 == 0 && c0 + 2 <= w.V) {
#pragma unroll
      for (int i = 0; i < KT / 2; ++i) {
        const int k = k0 + 2 * i;
        const float2 z = {0.f, 0.f};
        const float2 a = k < K ? *reinterpret_cast<const float2*>(s_in + 2 * i * si) : z;
        const float2 b = k + 1 < K ? *reinterpret_cast<const float2*>(s_in + (2 * i + 1) * si) : z;
        S[0][i] = tc::f2_pack(a.x, b.x);
        S[COLS > 1 ? 1 : 0][i] = tc::f2_pack(a.y, b.y);
      }
    } else if (si == 1 && sj % 4 == 0 && (uintptr_t)s_in % 16 == 0 && K % 4 == 0) {
      // transposed (k0 is a multiple of 4): four rows a load, or a warp reads each sector of its columns eight times
#pragma unroll
      for (int j = 0; j < COLS; ++j)
#pragma unroll
        for (int i = 0; i < KT / 4; ++i) {
          float4 f = {0.f, 0.f, 0.f, 0.f};
          if (c0 + j < w.V && k0 + 4 * i < K) f = *reinterpret_cast<const float4*>(s_in + 4 * i + j * sj);
          S[j][2 * i] = tc::f2_pack(f.x, f.y);
          S[j][2 * i + 1] = tc::f2_pack(f.z, f.w);
        }
    } else {
#pragma unroll
      for (int j = 0; j < COLS; ++j)
#pragma unroll
        for (int i = 0; i < KT / 2; ++i) {
          const int k = k0 + 2 * i;
          const bool in = c0 + j < w.V;
          const float a = in && k < K ? s_in[2 * i * si + j * sj] : 0.f;
          const float b = in && k + 1 < K ? s_in[(2 * i + 1) * si + j * sj] : 0.f;
          S[j][i] = tc::f2_pack(a, b);
        }
    }
  }

  // What the first steps leave behind is dropped at the last reset: of U's segment only the rest counts.
  int first = 0;
  bool any_reset = false;
  if (kStates && reset) {
    for (int e = (steps - 1) / 32 * 32; e >= 0 && steps > 0; e -= 32) {
      const uint32_t m = __ballot_sync(~0u, e + lane < steps && reset[(e + lane) * rst] != 0);
      if (m) {
        first = e + 31 - __clz(m) + (back ? 1 : 0);
        any_reset = true;
        break;
      }
    }
  }

  const Line<E> ql = line_of<E>(w.q, n, h, t0, back, 0, K), kl = line_of<E>(w.k, n, h, t0, back, 0, K);
  const Line<E> vl = line_of<E>(w.v, n, h, t0, back, vb * P::kVB, VB);
  constexpr int kGap = P::kRaw && KS > 1 ? KT : 0;   // (KT is a multiple of a 16-byte copy)
  // (padding between K and kKP is never written by the copies)
  for (int i = lane; i < min(kStages, (steps + kWindow - 1) / kWindow) * P::kStage / 16; i += 32)
    reinterpret_cast<uint4*>(mine)[i] = uint4{0, 0, 0, 0};
  __syncwarp();
  auto fetch = [&](int i0, int stage) {
    const int count = min(kWindow, steps - i0);
    E* q = reinterpret_cast<E*>(mine + stage * P::kStage);
    if (count > 0) {
      if (!kStates) fetch_rows<E, kGap>(q, P::kRawRow, ql, K, i0, count, lane);
      fetch_rows<E, kGap>(q + kWindow * P::kRawRow, P::kRawRow, kl, K, i0, count, lane);
      fetch_rows<E, 0>(q + 2 * kWindow * P::kRawRow, P::kVB, vl, VB, i0, count, lane);
    }
    copies_commit();
  };
#pragma unroll
  for (int x = 0; x < kStages - 1; ++x) fetch(first + x * kWindow, x);

  // g^j and its inverse
  float* pos = reinterpret_cast<float*>(mine + kStages * P::kStage + P::kConv);
  float* neg = pos + kWindow + 4;
  if (lane <= kWindow) pos[lane] = exp2f(l2 * lane), neg[lane] = exp2f(-l2 * lane);
  __syncwarp();

  auto scale_by = [&](float g) {
    const uint64_t g2 = tc::f2_pack(g, g);
#pragma unroll
    for (int y = 0; y < COLS; ++y)
#pragma unroll
      for (int i = 0; i < KT / 2; ++i) S[y][i] = tc::f2_mul(S[y][i], g2);
  };
  auto drop_all = [&]() {
#pragma unroll
    for (int y = 0; y < COLS; ++y)
#pragma unroll
      for (int i = 0; i < KT / 2; ++i) S[y][i] = 0;
  };
  // A step decays what it receives (forward), or passes it on decayed (back).
  if (steps > 0 && !kStates) scale_by(pos[back ? win - 1 : win]);

  // After the KS threads' sums are joined a thread has kOwn columns of the output, from `oc` on.
  constexpr int kOwn = COLS > KS ? COLS / KS : 1;
  int oc = c0;
  bool writes = !kStates && w.o.p;
#pragma unroll
  for (int o = 1, n = COLS; o < KS; o <<= 1) {
    if (n > 1) n /= 2, oc += part & o ? n : 0;
    else writes = writes && !(part & o);
  }
  writes = writes && oc < w.V;
  E* op = nullptr;
  int64_t ost = 0;
  bool wide = false;            // all of them in one store
  if (writes) {
    op = static_cast<E*>(w.o.p) + n * w.o.sn + h * w.o.sh + t0 * w.o.st + oc;
    ost = back ? -w.o.st : w.o.st;
    wide = oc + kOwn <= w.V && (uintptr_t)op % (kOwn * sizeof(E)) == 0 && w.o.st % kOwn == 0;
  }
  auto store = [&](const float (&y)[COLS]) {
    if (!writes) return;
    if (wide && kOwn == 4) {
      if constexpr (sizeof(E) == 4) *reinterpret_cast<float4*>(op) = float4{y[0], y[COLS > 1 ? 1 : 0], y[COLS > 2 ? 2 : 0], y[COLS > 2 ? 3 : 0]};
      else *reinterpret_cast<uint2*>(op) = uint2{tc::pack_bf16(y[0], y[COLS > 1 ? 1 : 0]), tc::pack_bf16(y[COLS > 2 ? 2 : 0], y[COLS > 2 ? 3 : 0])};
    } else if (wide && kOwn == 2) {
      if constexpr (sizeof(E) == 4) *reinterpret_cast<float2*>(op) = float2{y[0], y[COLS > 1 ? 1 : 0]};
      else *reinterpret_cast<uint32_t*>(op) = tc::pack_bf16(y[0], y[COLS > 1 ? 1 : 0]);
    } else {
#pragma unroll
      for (int j = 0; j < kOwn; ++j)
        if (oc + j < w.V) op[j] = rounded<E>(y[j]);
    }
  };

  int stage = 0;
  uint32_t carry = 0;           // back: the step before this window is a reset
  auto reset_at = [&](int i) { return reset && lane < kWindow && i + lane < steps && reset[(i + lane) * rst] != 0; };
  bool next_reset = reset_at(first);
  for (int i0 = first; i0 < steps; i0 += kWindow) {
    copies_wait<kStages - 2>();
    __syncwarp();
    fetch(i0 + (kStages - 1) * kWindow, stage == 0 ? kStages - 1 : stage - 1);
    const int count = min(kWindow, steps - i0);
    uint32_t drops = __ballot_sync(~0u, next_reset);
    next_reset = reset_at(i0 + kWindow);
    if (back) {
      const uint32_t d = drops;
      drops = drops << 1 | carry;
      carry = d >> (count - 1) & 1u;
    }
    const E* raw = reinterpret_cast<const E*>(mine + stage * P::kStage);
    const float *qf, *kf;
    if constexpr (P::kRaw) {
      qf = reinterpret_cast<const float*>(raw);
      kf = qf + kWindow * P::kRow;
    } else {
      qf = conv;
      kf = conv + kWindow * P::kRow;
      for (int i = lane; i < 2 * kWindow * P::kKP / 2; i += 32) {
        const int r = i / (P::kKP / 2), k = i % (P::kKP / 2) * 2;
        if (kStates && r < kWindow) continue;
        const uint32_t p = *reinterpret_cast<const uint32_t*>(raw + r * P::kKP + k);
        *reinterpret_cast<float2*>(conv + r * P::kRow + place<(KS > 1 ? KT : 0)>(k)) =
            float2{__uint_as_float(p << 16), __uint_as_float(p & 0xFFFF0000u)};
      }
      __syncwarp();
    }
    const E* vf = raw + 2 * kWindow * P::kRawRow + col;
    kf += part * (KT + 4);
    qf += part * (KT + 4);
    // one step, the e-th of its window
    auto step = [&](int j, int e) {
      uint64_t vv[COLS];
      {
        const float down = w.in * pos[win - 1 - e];
        float a[COLS];
        if constexpr (COLS == 4 && sizeof(E) == 4) {
          const float4 f = *reinterpret_cast<const float4*>(vf + j * P::kVB);
          a[0] = f.x, a[1] = f.y, a[2] = f.z, a[3] = f.w;
        } else if constexpr (COLS == 4) {
          const uint2 f = *reinterpret_cast<const uint2*>(vf + j * P::kVB);
          a[0] = __uint_as_float(f.x << 16), a[1] = __uint_as_float(f.x & 0xFFFF0000u);
          a[2] = __uint_as_float(f.y << 16), a[3] = __uint_as_float(f.y & 0xFFFF0000u);
        } else {
#pragma unroll
          for (int y = 0; y < COLS; ++y) a[y] = as_f32<E>(vf[j * P::kVB + y]);
        }
#pragma unroll
        for (int y = 0; y < COLS; ++y) vv[y] = tc::f2_pack(a[y] * down, a[y] * down);
      }
      const ulonglong2* k2 = reinterpret_cast<const ulonglong2*>(kf + j * P::kRow);
      if constexpr (kStates) {
#pragma unroll
        for (int i = 0; i < KT / 4; ++i) {
          const ulonglong2 kk = k2[i];
#pragma unroll
          for (int y = 0; y < COLS; ++y) {
            S[y][2 * i] = tc::f2_fma(kk.x, vv[y], S[y][2 * i]);
            S[y][2 * i + 1] = tc::f2_fma(kk.y, vv[y], S[y][2 * i + 1]);
          }
        }
      } else {
        const ulonglong2* q2 = reinterpret_cast<const ulonglong2*>(qf + j * P::kRow);
        uint64_t acc[COLS][2];
#pragma unroll
        for (int i = 0; i < KT / 4; ++i) {
          const ulonglong2 kk = k2[i], qq = q2[i];
#pragma unroll
          for (int y = 0; y < COLS; ++y) {
            S[y][2 * i] = tc::f2_fma(kk.x, vv[y], S[y][2 * i]);
            S[y][2 * i + 1] = tc::f2_fma(kk.y, vv[y], S[y][2 * i + 1]);
            acc[y][0] = i == 0 ? tc::f2_mul(qq.x, S[y][0]) : tc::f2_fma(qq.x, S[y][2 * i], acc[y][0]);
            acc[y][1] = i == 0 ? tc::f2_mul(qq.y, S[y][1]) : tc::f2_fma(qq.y, S[y][2 * i + 1], acc[y][1]);
          }
        }
        float y[COLS];
        const float up = w.out * neg[win - 1 - e];
#pragma unroll
        for (int z = 0; z < COLS; ++z) {
          float a, b;
          tc::f2_unpack(tc::f2_add(acc[z][0], acc[z][1]), a, b);
          y[z] = (a + b) * up;
        }
        // the KS threads' sums: each keeps half of the columns it had
#pragma unroll
        for (int o = 1, n = COLS; o < KS; o <<= 1) {
          if (n > 1) {
            n /= 2;
#pragma unroll
            for (int z = 0; z < COLS; ++z)
              if (z < n) {
                const float give = part & o ? y[z] : y[z + n < COLS ? z + n : z], keep = part & o ? y[z + n < COLS ? z + n : z] : y[z];
                y[z] = keep + __shfl_xor_sync(~0u, give, o);
              }
          } else {
            y[0] += __shfl_xor_sync(~0u, y[0], o);
          }
        }
        store(y);
        op += ost;
      }
    };
    int e = 0;
#pragma unroll 1
    for (int j = 0; j < count; ++j) {
      if (drops >> j & 1u) drop_all();
      step(j, e);
      if (++e == win) {
        // (the last step of a forward walk hands its state on as it is, that of the other decayed)
        if (i0 + j + 1 < steps) scale_by(pos[win]);
        else if (back) scale_by(pos[1]);
        e = 0;
      }
    }
    if (e > 0) scale_by(neg[win - e] * (back ? pos[1] : 1.f));   // (the last window of all: `win` divides a stage)
    __syncwarp();
    stage = stage == kStages - 1 ? 0 : stage + 1;
  }
  copies_wait<0>();
  if (back && carry) drop_all();

  if (writes) {                 // steps behind the end
    op = static_cast<E*>(w.o.p) + n * w.o.sn + h * w.o.sh + oc;
    for (int64_t t = max(len, (int64_t)seg * c.seg_len); t < min(c.T, ((int64_t)seg + 1) * c.seg_len); ++t)
#pragma unroll
      for (int j = 0; j < kOwn; ++j)
        if (oc + j < w.V) op[t * w.o.st + j] = rounded<E>(0.f);
  }
  // ---- the state left behind
  float* s_out = nullptr;
  if (kStates) {
    s_out = w.seg + at_seg;
    if (lane == 0 && h == 0 && vb == 0 && wi == 0) c.seg_live[(int64_t)seg * c.N + n] = any_reset ? -1 : steps;
  } else if (seg == (back ? 0 : c.segs - 1) && w.s_out) {
    s_out = w.s_out + chain * KV;
  }
  if (!s_out) return;
  s_out += (int64_t)k0 * w.V + c0;
  const bool four = COLS == 4 && w.V % 4 == 0 && (uintptr_t)s_out % 16 == 0 && c0 + 4 <= w.V;
  const bool two = COLS == 2 && w.V % 2 == 0 && (uintptr_t)s_out % 8 == 0 && c0 + 2 <= w.V;
#pragma unroll
  for (int i = 0; i < KT / 2; ++i) {
    const int k = k0 + 2 * i;
    float a[COLS], b[COLS];
#pragma unroll
    for (int j = 0; j < COLS; ++j) tc::f2_unpack(S[j][i], a[j], b[j]);
    float* r = s_out + 2 * i * w.V;
    if (four) {
      constexpr int k1 = COLS > 1 ? 1 : 0, k2 = COLS > 2 ? 2 : 0, k3 = COLS > 2 ? 3 : 0;
      if (k < K) *reinterpret_cast<float4*>(r) = float4{a[0], a[k1], a[k2], a[k3]};
      if (k + 1 < K) *reinterpret_cast<float4*>(r + w.V) = float4{b[0], b[k1], b[k2], b[k3]};
    } else if (two) {
      constexpr int k1 = COLS > 1 ? 1 : 0;
      if (k < K) *reinterpret_cast<float2*>(r) = float2{a[0], a[k1]};
      if (k + 1 < K) *reinterpret_cast<float2*>(r + w.V) = float2{b[0], b[k1]};
    } else {
#pragma unroll
      for (int j = 0; j < COLS; ++j)
        if (c0 + j < w.V) {
          if (k < K) r[j] = a[j];
          if (k + 1 < K) r[w.V + j] = b[j];
        }
    }
  }
}

// ---- bf16: chunks of 64 steps on the tensor cores -------------------------------------------
// Rows in a walk's order (i, j), whatever its direction.  Over a chunk, with rows of q, k, v as matrices and S the
// state it receives:
//   O = ((Q K^T) o D) V + diag(enter) Q S,   S <- g^L S + (diag(leave) K)^T V,
// with D_ij = g^(i - j) where row j reaches row i (j <= i, the same episode), `enter` the decay from the chunk's
// beginning to a row and `leave` from a row to its end, each 0 across an episode's beginning.
//   Operands of bf16: P = (Q K^T) o D and S are hi + lo, off by at most 2^-17 of each element, and so is decayed k
// (hi + mid) where the state only feeds bf16 outputs; with one more part, 2^-25, where it is an output itself.  (One part,
// 2^-8, is as much as an output's own rounding, and more where its terms nearly cancel: errors 1.4 times as large for
// 408 us instead of 472, 128 x 4096 x 4 x 64.)  The state stays in fp32 registers, and a chunk's K^T V is summed from 0
// before it is added: sums that grow in the tensor cores' accumulators are truncated at every product.
//   A CTA of D / 16 warps goes from chunk to chunk and chain to chain, the next chunk's rows on their way while
// this one is computed.  A warp has 16 rows of O (and 64 of its columns) and 16 rows of S.  P goes from the
// accumulators of Q K^T to the operand of P V in registers, as does decayed k from its rows; a block of v is
// loaded once for P V and K^T V.  These are warp-wide products (mma.sync): a chunk is a chain of small products
// with work on registers between them, and what bounds it is that work and its latency, not the products: 1775
// instructions a warp and chunk, 48 % of the issue slots, 35 % of the products' pipe; 128 x 4096 x 4 x 64 with both states
// 472 us, 50 % of the measured copy rate.  (A form on tcgen05, chunks of 128 with P and results through tensor memory,
// took 1035 us for that pass as it was first built, and this one 1045 as it was: the steps from there were taken for this
// one alone, so which of the two ends faster is not known.)
//   Masked products are products with 0.  Where anything of a warp's result is not finite, they may have spread it:
// those elements are then computed again from the rows that reach them.
constexpr int kC = 64;                     // steps of a chunk

// D: K padded.  A CTA has kVB columns of v and of the state, its warps 16 rows of O and kVB / kSplit of its columns.
constexpr int kVB = 64;
template <int D> struct TcPlan {
  static constexpr int kThreads = 2 * D, kSplit = D / 64;
  static constexpr int kPitch = 2 * D + 16, kPitchV = 2 * kVB + 16;   // bytes of a staged row: 8 rows in 8 bank groups
  static constexpr int kTile = kC * kPitch, kTileV = kC * kPitchV;
  // One tile of q, two of k and v, S as two operands.  The second one of D = 64 is in v's tile of the next chunk until the
  // outputs are done: with a plane of its own three CTAs share an SM (128x1024x4x64 with gradients 404 us, this way 374).
  static constexpr int kPlane = D * kPitchV;
  static constexpr bool kInV = kPlane == kTileV;
  static constexpr int kQ = 0, kK = kTile, kV = 3 * kTile, kS = 3 * kTile + 2 * kTileV, kSmall = kS + (kInV ? 1 : 2) * kPlane;
  __device__ __forceinline__ static int low(int stage) { return kInV ? kV + (stage ^ 1) * kTileV : kS + kPlane; }
  static constexpr int kZeros = 16;        // before the decays of P: rows that do not reach a row
  static constexpr int kDecays = kZeros + 2 * (kC + 4), kBytes = kSmall + 2 * (kDecays + kC) * 4;   // (two sets, by turn)
  static constexpr int kCtas = D == 64 ? 4 : 2;   // an SM
};

__device__ __forceinline__ void ldsm(uint32_t at, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void ldsm_t(uint32_t at, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint64_t pair_of(uint32_t bf16x2) {
  return tc::f2_pack(__uint_as_float(bf16x2 << 16), __uint_as_float(bf16x2 & 0xFFFF0000u));
}
__device__ __forceinline__ uint32_t bf16_of(uint64_t pair) {
  float a, b;
  tc::f2_unpack(pair, a, b);
  return tc::pack_bf16(a, b);
}
__device__ __forceinline__ uint64_t twice(float v) { return tc::f2_pack(v, v); }
__device__ __forceinline__ bool finite(float v) { return fabsf(v) <= 3.4028234e38f; }

// A chain's share of a CTA's work, by its number.
struct Unit {
  int wi, v0, h, seg, live;     // walk, first column of v, head, segment and its steps
  int64_t n, t0;                // env, first step in the walk's order
};
__device__ __forceinline__ Unit unit_of(const Chains& c, uint32_t u) {
  Unit x;
  const int part = (int)(u % (uint32_t)c.parts);
  x.wi = c.part_walk[part], x.v0 = c.part_block[part] * kVB;
  u /= (uint32_t)c.parts;
  x.h = (int)(u % (uint32_t)c.H);
  u /= (uint32_t)c.H;
  x.n = u % (uint32_t)c.N;
  x.seg = (int)(u / (uint32_t)c.N);
  const int64_t len = c.lengths ? min((int64_t)max(c.lengths[x.n], 0), c.T) : c.T;
  const int64_t t_lo = min(len, (int64_t)x.seg * c.seg_len);
  x.live = (int)(min(len, t_lo + c.seg_len) - t_lo);
  x.t0 = c.w[x.wi].back && x.live > 0 ? t_lo + x.live - 1 : t_lo;
  return x;
}

// A thread's place in the rows of a sequence that it copies: its 16-byte block of row `row0`, then of every kStep-th.
template <int kW> struct From {
  const __nv_bfloat16* p;
  __device__ __forceinline__ void set(const Rows& r, const Unit& x, bool back, int c0, int row0, int block) {
    p = static_cast<const __nv_bfloat16*>(r.p) + x.n * r.sn + x.h * r.sh + x.t0 * r.st + c0;
    p += row0 * (back ? -r.st : r.st) + block * 8;
  }
};
// kCount of the next chunk's rows into a staged tile; rows from `rows` on, and columns from `width` on, are zeros.
template <int kW, int kStep, int kCount>
__device__ __forceinline__ void tile_in(unsigned char* dst, From<kW>& f, int64_t st, int rows, int width, int row0, int block) {
  constexpr int kPitch = 2 * kW + 16;
  unsigned char* d = dst + row0 * kPitch + block * 16;
  const __nv_bfloat16* src = f.p;
  const int64_t step = kStep * st;
  if (((uintptr_t)src % 16 | st % 8 | width % 8) == 0) {   // (the same for all threads of a tile)
    const uint32_t at = tc::smem_u32(d);
    const int left = block * 8 < width ? rows - row0 : 0;
#pragma unroll
    for (int z = 0; z < kCount; ++z, src += step)
      asm volatile("{\n.reg .pred p;\nsetp.gt.s32 p, %2, 0;\n@p cp.async.cg.shared.global [%0], [%1], 16;\n"
                   "@!p st.shared.v4.b32 [%0], {%3, %3, %3, %3};\n}\n" ::"r"(at + z * kStep * kPitch), "l"(src), "r"(left - z * kStep), "r"(0)
                   : "memory");
  } else {
    // Elements one by one, or pairs, the rows' loads in flight together.
    const int e0 = block * 8;
    const bool pairs = ((uintptr_t)src % 4 | st % 2 | width % 2) == 0;
    uint32_t x[kCount][4];
#pragma unroll
    for (int z = 0; z < kCount; ++z) {
      const __nv_bfloat16* r = src + z * step;
      const int left = row0 + z * kStep < rows ? width - e0 : 0;
      if (pairs) {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[z][i] = 2 * i < left ? *reinterpret_cast<const uint32_t*>(r + 2 * i) : 0;
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          x[z][i] = 2 * i < left ? __bfloat16_as_ushort(r[2 * i]) : 0;
          if (2 * i + 1 < left) x[z][i] |= (uint32_t)__bfloat16_as_ushort(r[2 * i + 1]) << 16;
        }
      }
    }
#pragma unroll
    for (int z = 0; z < kCount; ++z) *reinterpret_cast<uint4*>(d + z * kStep * kPitch) = uint4{x[z][0], x[z][1], x[z][2], x[z][3]};
  }
  f.p += kC * st;
}

// What the rows of a chunk receive is dropped before row i where bit i is set, and behind the last one where `end`.
struct Drops {
  uint64_t m;
  bool end;
  __device__ __forceinline__ int last_up_to(int i) const {   // -1: none
    const uint64_t a = m & (~0ull >> (63 - i));
    return a ? 63 - __clzll((long long)a) : -1;
  }
};

// kStates: a segment's U alone.
template <int D, bool kStates>
__global__ void __launch_bounds__(TcPlan<D>::kThreads, TcPlan<D>::kCtas) chunks(const __grid_constant__ Chains c, uint32_t units) {
  using P = TcPlan<D>;
  tc::after_previous();
  extern __shared__ __align__(128) unsigned char sm[];
  __shared__ uint64_t words[2];  // resets of a chunk's rows, by stage
  __shared__ Unit of_turn[2];    // the chain's share that is worked on, and the next one
  constexpr int kNK = D / 16, kNV = kVB / 8, kOV = kNV / P::kSplit, kOB = 16 * kOV;   // (bytes of a warp's columns of O)
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, tr = lane >> 2, tq = lane & 3;
  // Rows 16 rb .. of O, share ch of its columns.  The last rows have four blocks of P, the first ones one: the two warps
  // of a scheduler (every fourth) have different rows (4096x8x4x128 with gradients 636 us before, 605 so).
  const int ch = warp >> 2, rb = ch ? 3 - (warp & 3) : warp & 3;
  const int r0 = 16 * rb + tr, r1 = r0 + 8;          // this thread's rows of O (and, 16 warp for 16 rb, of S)
  // Two sets by turn, since warps may still read the one before: decays by chain, `leave` by chunk.
  float* gz = reinterpret_cast<float*>(sm + P::kSmall) + P::kZeros + P::kDecays;   // in g^0 .. behind zeros
  float* gp = gz + kC + 4;                           // g^0 ..
  int decays = P::kDecays;
  for (int i = threadIdx.x; i < P::kBytes / 16; i += P::kThreads) reinterpret_cast<uint4*>(sm)[i] = uint4{0, 0, 0, 0};
  __syncthreads();

  // ldmatrix addresses within a tile: 16 rows x 16 columns as an A operand (and, transposed, as B of K x N), or as B
  // of N x K (and, transposed, as A)
  const uint32_t base = tc::smem_u32(sm);
  const uint32_t a_at = (uint32_t)((lane & 15) * P::kPitch + (lane >> 4) * 16), v_off = (uint32_t)((lane & 15) * P::kPitchV + (lane >> 4) * 16);
  const uint32_t b_at = (uint32_t)(((lane & 7) + (lane >> 4) * 8) * P::kPitch + (lane >> 3 & 1) * 16);

  float S[kNV][4];
  From<D> fq, fk;
  From<kVB> fv;
  const uint8_t* rp = nullptr;  // warp 0: reset of this lane's first row in the next chunk
  // (q's rows are copied by the warps that use them, which need not wait for the others then)
  const int k_row = threadIdx.x / (D / 8), k_block = threadIdx.x % (D / 8), v_row = threadIdx.x / (kVB / 8), v_block = threadIdx.x % (kVB / 8);
  const int q_row = 16 * rb + (ch * 32 + lane) / (D / 8), q_block = lane % (D / 8);
  auto locate = [&](const Unit& z) {
    const Walk& w = c.w[z.wi];
    const bool back = w.back != 0;
    if (!kStates) fq.set(w.q, z, back, 0, q_row, q_block);
    fk.set(w.k, z, back, 0, k_row, k_block);
    fv.set(w.v, z, back, z.v0, v_row, v_block);
    if (warp == 0) rp = c.reset ? c.reset + (z.t0 + (back ? -lane : lane)) * c.N + z.n : nullptr;
  };
  // The next chunk's rows; warp 0 loads the resets of rows lane and lane + 32.  (Each is a sector of its own: by every
  // warp they would be more requests than the rows.)
  auto fetch_q = [&](const Unit& z, int L) {
    const Walk& w = c.w[z.wi];
    if (!kStates) tile_in<D, P::kThreads / (D / 8) / 4, 4>(sm + P::kQ, fq, w.back ? -w.q.st : w.q.st, L, w.K, q_row, q_block);
  };
  auto fetch_k = [&](const Unit& z, int L, int stage) {
    const Walk& w = c.w[z.wi];
    tile_in<D, P::kThreads / (D / 8), 4>(sm + P::kK + stage * P::kTile, fk, w.back ? -w.k.st : w.k.st, L, w.K, k_row, k_block);
  };
  uint32_t reset0 = 0, reset1 = 0;
  auto fetch_v = [&](const Unit& z, int L, int stage) {
    const Walk& w = c.w[z.wi];
    constexpr int kStep = P::kThreads / (kVB / 8);
    tile_in<kVB, kStep, kC / kStep>(sm + P::kV + stage * P::kTileV, fv, w.back ? -w.v.st : w.v.st, L, w.V - z.v0, v_row, v_block);
    reset0 = reset1 = 0;
    if (warp == 0 && rp) {
      const int64_t rst = w.back ? -c.N : c.N;
      if (lane < L) reset0 = rp[0];
      if (lane + 32 < L) reset1 = rp[32 * rst];
      rp += kC * rst;
    }
  };
  // where a chain's segment receives its state
  auto state_at = [&](const Unit& z) -> const float* {
    const Walk& w = c.w[z.wi];
    const int64_t KV = (int64_t)w.K * w.V, chain = z.n * c.H + z.h;
    return c.segs > 1 ? w.seg + ((int64_t)z.seg * c.N * c.H + chain) * KV : w.s_in ? w.s_in + chain * KV : nullptr;
  };
  auto prefetch_state = [&](const Unit& z) {   // into L2, a chunk ahead
    const Walk& w = c.w[z.wi];
    const float* s_in = state_at(z);
    const int64_t e = (int64_t)threadIdx.x * 32;
    if (s_in && e < w.K * w.V) asm volatile("prefetch.global.L2 [%0];" ::"l"(s_in + e));
    if (s_in && e + P::kThreads * 32 < w.K * w.V) asm volatile("prefetch.global.L2 [%0];" ::"l"(s_in + e + P::kThreads * 32));
  };
  // the state a chain's segment receives
  auto fetch_state = [&](const Unit& z) {
#pragma unroll
    for (int j = 0; j < kNV; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) S[j][e] = 0.f;
    if (kStates) return;
    const Walk& w = c.w[z.wi];
    const float* s_in = state_at(z);
    if (!s_in) return;
    const int64_t si = c.segs > 1 ? w.V : w.si_in, sj = c.segs > 1 ? 1 : w.sj_in;
    const int left = w.V - z.v0;
    s_in += z.v0 * sj;
    const int k0 = 16 * warp + tr;
    const bool two = sj == 1 && si % 2 == 0 && (uintptr_t)s_in % 8 == 0 && w.V % 2 == 0;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if (k0 + 8 * h >= w.K) break;
      const float* r = s_in + (k0 + 8 * h) * si + 2 * tq * sj;
#pragma unroll
      for (int j = 0; j < kNV; ++j) {
        const int v = 8 * j + 2 * tq;
        if (two) {
          if (v < left) {
            const float2 f = *reinterpret_cast<const float2*>(r + 8 * j);
            S[j][2 * h] = f.x, S[j][2 * h + 1] = f.y;
          }
        } else {
          if (v < left) S[j][2 * h] = r[8 * j * sj];
          if (v + 1 < left) S[j][2 * h + 1] = r[(8 * j + 1) * sj];
        }
      }
    }
  };
  auto plane_out = [&](int stage) {      // S as operands of the chunk in a stage
    const int at = (16 * warp + tr) * P::kPitchV + 4 * tq;
#pragma unroll
    for (int j = 0; j < kNV; ++j)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint64_t f = tc::f2_pack(S[j][2 * h], S[j][2 * h + 1]);
        const uint32_t hi = bf16_of(f);
        unsigned char* to = sm + at + 8 * h * P::kPitchV + 16 * j;
        *reinterpret_cast<uint32_t*>(to + P::kS) = hi;
        *reinterpret_cast<uint32_t*>(to + P::low(stage)) = bf16_of(tc::f2_sub(f, pair_of(hi)));
      }
  };

  uint32_t u = blockIdx.x;
  int chunk = 0, stage = 0, turn = 0;
  if (u >= units) return;
  if (threadIdx.x == 0) of_turn[0] = unit_of(c, u);
  __syncthreads();
  bool any_reset = false;
  locate(of_turn[0]);
  fetch_q(of_turn[0], min(kC, of_turn[0].live));
  fetch_k(of_turn[0], min(kC, of_turn[0].live), 0);
  fetch_v(of_turn[0], min(kC, of_turn[0].live), 0);
  copies_commit();
  fetch_state(of_turn[0]);
  auto share_resets = [&](int stage) {
    const uint32_t lo = __ballot_sync(~0u, reset0 != 0), hi = __ballot_sync(~0u, reset1 != 0);
    if (lane == 0) words[stage] = lo | (uint64_t)hi << 32;
  };
  if (warp == 0) share_resets(0);
  __syncthreads();
  while (true) {
    const Unit& x = of_turn[turn];
    const Walk& w = c.w[x.wi];
    const int K = w.K, left = w.V - x.v0, L = min(kC, x.live - kC * chunk);
    const bool last = kC * (chunk + 1) >= x.live;
    const int b = w.back ? 1 : 0;
    const bool received = !kStates && (chunk > 0 || c.segs > 1 || w.s_in);   // (else Q S is 0)
    const bool out = !kStates && last && w.s_out && x.seg == (b ? 0 : c.segs - 1), hands_on = kStates || !last || out;
    const bool three = kStates || w.s_out;
    Drops drops;
    drops.m = words[stage];
    if (chunk == 0) any_reset = false;
    any_reset |= drops.m != 0;
    drops.end = b && L > 0 && (drops.m >> (L - 1) & 1u);
    drops.m <<= b;              // (back, a state is dropped behind the step that begins the episode)
    const int drop_first = drops.m ? __ffsll((long long)drops.m) - 1 : kC, drop_last = drops.end ? kC : drops.last_up_to(kC - 1);
    float* leave = reinterpret_cast<float*>(sm + P::kSmall) + 2 * P::kDecays + stage * kC;   // in g^(to the end), by row
    if (chunk == 0) {
      const float l2 = log2_decay(c.log_decay, x.h);
      gz -= decays, gp -= decays, decays = -decays;
      if (threadIdx.x <= kC) {
        // (one that underflows stays above 0: what is not finite comes through it)
        float g = exp2f(l2 * threadIdx.x);
        g = g < 1.17549435e-38f ? 1.17549435e-38f : g;
        gp[threadIdx.x] = g, gz[threadIdx.x] = g * w.in;
      }
      __syncthreads();          // (`leave` is made from the decays; nobody reads the chain before any more)
      if (threadIdx.x == 0 && u + gridDim.x < units) of_turn[turn ^ 1] = unit_of(c, u + gridDim.x);
      if (received) plane_out(stage);
    }
    if (threadIdx.x < kC) leave[threadIdx.x] = (int)threadIdx.x < L && (int)threadIdx.x >= drop_last ? gz[L - 1 + b - threadIdx.x] : 0.f;
    copies_wait<0>();
    __syncthreads();
    // ---- the next chunk
    const uint32_t u2 = last ? u + gridDim.x : u;
    const Unit& x2 = of_turn[last ? turn ^ 1 : turn];
    if (last && u2 < units) locate(x2);
    const bool more = u2 < units;
    const int chunk2 = last ? 0 : chunk + 1;
    const int L2 = more ? min(kC, x2.live - kC * chunk2) : 0;
    if (more) fetch_k(x2, L2, stage ^ 1);
    if (!kStates && last && more) prefetch_state(x2);

    const uint32_t rows_q = base + P::kQ + (uint32_t)(16 * rb * P::kPitch) + a_at;
    const uint32_t k_at = base + P::kK + stage * P::kTile, v_at = base + P::kV + stage * P::kTileV;
    const unsigned char *k_tile = sm + P::kK + stage * P::kTile, *v_tile = sm + P::kV + stage * P::kTileV;
    auto val = [](const unsigned char* row, int i) { return __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(row)[i]); };

    // ---- O
    if (!kStates && w.o.p && 8 * kOV * ch < left && 16 * rb < L) {
      float acc[kOV][4];
#pragma unroll
      for (int j = 0; j < kOV; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[j][e] = 0.f;
      // Q S, for rows before the first drop
      const bool on0 = received && r0 < drop_first, on1 = received && r1 < drop_first;
      const float e0 = gp[r0 + 1 - b], e1 = gp[r1 + 1 - b];
      if (received && 16 * rb < drop_first) {
#pragma unroll
        for (int i = 0; i < kNK; ++i) {
          uint32_t q[4];
          ldsm(rows_q + 32 * i, q);
#pragma unroll
          for (int g = 0; g < kOV; ++g) {   // (one part of S, then the other: a sum's products far apart)
            uint32_t t[4];
            ldsm_t(base + (g < kOV / 2 ? P::kS : P::low(stage)) + 16 * i * P::kPitchV + kOB * ch + 32 * (g % (kOV / 2)) + v_off, t);
            mma(acc[2 * (g % (kOV / 2))], q, t[0], t[1]);
            mma(acc[2 * (g % (kOV / 2)) + 1], q, t[2], t[3]);
          }
        }
#pragma unroll
        for (int j = 0; j < kOV; ++j) {
          acc[j][0] = on0 ? acc[j][0] * e0 : 0.f, acc[j][1] = on0 ? acc[j][1] * e0 : 0.f;
          acc[j][2] = on1 ? acc[j][2] * e1 : 0.f, acc[j][3] = on1 ? acc[j][3] * e1 : 0.f;
        }
      }
      // the first row that reaches a row
      const int from0 = max(drops.last_up_to(r0), 0), from1 = max(drops.last_up_to(r1), 0);
      const int kb_lo = __shfl_sync(~0u, from0, 0) >> 4;
      uint64_t col[2];          // decay from the columns of a block to its last one
#pragma unroll
      for (int i = 0; i < 2; ++i) col[i] = tc::f2_pack(gp[15 - 8 * i - 2 * tq], gp[14 - 8 * i - 2 * tq]);
#pragma unroll 1
      for (int kb = kb_lo; kb <= rb; ++kb) {
        // P: 16 columns
        float s[2][4] = {};
#pragma unroll
        for (int i = 0; i < kNK; ++i) {
          uint32_t q[4], k[4];
          ldsm(rows_q + 32 * i, q);
          ldsm(k_at + (uint32_t)(16 * kb * P::kPitch) + 32 * i + b_at, k);
          mma(s[0], q, k[0], k[1]);
          mma(s[1], q, k[2], k[3]);
        }
        uint64_t f[4];          // (column block, row)
        if (kb == rb) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float* g = gz + tr + 8 * (i & 1) - 8 * (i >> 1) - 2 * tq;
            f[i] = tc::f2_mul(tc::f2_pack(s[i >> 1][2 * (i & 1)], s[i >> 1][2 * (i & 1) + 1]), tc::f2_pack(g[0], g[-1]));
          }
        } else {
          const float* g = gz + r0 - 16 * kb - 15;
          const uint64_t g0 = twice(g[0]), g1 = twice(g[8]);
#pragma unroll
          for (int i = 0; i < 4; ++i)
            f[i] = tc::f2_mul(tc::f2_mul(tc::f2_pack(s[i >> 1][2 * (i & 1)], s[i >> 1][2 * (i & 1) + 1]), col[i >> 1]), i & 1 ? g1 : g0);
        }
        if (__any_sync(~0u, from1 > 16 * kb)) {   // (rows of an earlier episode)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int d = (i & 1 ? from1 : from0) - 16 * kb - 2 * tq - 8 * (i >> 1);
            float a0, a1;
            tc::f2_unpack(f[i], a0, a1);
            f[i] = tc::f2_pack(d > 0 ? 0.f : a0, d > 1 ? 0.f : a1);
          }
        }
        uint32_t p[4], r[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) p[i] = bf16_of(f[i]), r[i] = bf16_of(tc::f2_sub(f[i], pair_of(p[i])));
#pragma unroll
        for (int g = 0; g < kOV / 2; g += 2) {
          uint32_t v[2][4];
#pragma unroll
          for (int i = 0; i < 2; ++i) ldsm_t(v_at + (uint32_t)(16 * kb * P::kPitchV) + kOB * ch + 32 * (g + i) + v_off, v[i]);
#pragma unroll
          for (int i = 0; i < 8; ++i) mma(acc[2 * g + i % 4], i < 4 ? p : r, v[i / 2 % 2][2 * (i % 2)], v[i / 2 % 2][2 * (i % 2) + 1]);
        }
      }
      // What is not finite: 0 times it is NaN (columns of padding are 0).
      uint64_t zero = 0;
#pragma unroll
      for (int j = 0; j < kOV; ++j)
#pragma unroll
        for (int e = 0; e < 4; e += 2) {
          const uint64_t f = tc::f2_mul(tc::f2_pack(acc[j][e], acc[j][e + 1]), twice(w.out));
          zero = tc::f2_fma(f, 0, zero);
          tc::f2_unpack(f, acc[j][e], acc[j][e + 1]);
        }
      float z0, z1;
      tc::f2_unpack(zero, z0, z1);
      if (__any_sync(~0u, !(z0 + z1 == 0.f))) {
        // It may have come through a product with 0: such elements again, from the rows that reach them alone.
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int r = h ? r1 : r0;
          const unsigned char* q = sm + P::kQ + r * P::kPitch;
          float o[2 * kOV] = {};
          if (h ? on1 : on0)
            for (int k = 0; k < K; ++k) {
              const float qk = val(q, k) * (h ? e1 : e0);
#pragma unroll
              for (int i = 0; i < 2 * kOV; ++i) {
                const unsigned char* s = sm + k * P::kPitchV;
                const int v = 8 * (kOV * ch + i / 2) + 2 * tq + i % 2;
                const float hi = val(s + P::kS, v);
                o[i] += qk * (finite(hi) ? hi + val(s + P::low(stage), v) : hi);
              }
            }
          for (int j = h ? from1 : from0; j <= r; ++j) {
            float qk = 0.f;
            for (int k = 0; k < K; ++k) qk += val(q, k) * val(k_tile + j * P::kPitch, k);
            qk *= gz[r - j];
#pragma unroll
            for (int i = 0; i < 2 * kOV; ++i) o[i] += qk * val(v_tile + j * P::kPitchV, 8 * (kOV * ch + i / 2) + 2 * tq + i % 2);
          }
#pragma unroll
          for (int i = 0; i < 2 * kOV; ++i) {
            float& a = acc[i / 2][2 * h + i % 2];
            if (!finite(a)) a = o[i] * w.out;
          }
        }
        __syncwarp();
      }
      // Outputs, through this warp's rows of q to whole rows.  (With kSplit > 1 two warps
      // read a row of q, where there are columns for both.)
      if (P::kSplit > 1 && left > 8 * kOV) asm volatile("bar.sync %0, 64;" ::"r"(1 + rb) : "memory");
      unsigned char* own = sm + P::kQ + 16 * rb * P::kPitch + kOB * ch;
#pragma unroll
      for (int j = 0; j < kOV; ++j) {
        *reinterpret_cast<uint32_t*>(own + tr * P::kPitch + 16 * j + 4 * tq) = tc::pack_bf16(acc[j][0], acc[j][1]);
        *reinterpret_cast<uint32_t*>(own + (tr + 8) * P::kPitch + 16 * j + 4 * tq) = tc::pack_bf16(acc[j][2], acc[j][3]);
      }
      __syncwarp();
      const int64_t st = b ? -w.o.st : w.o.st;
      __nv_bfloat16* o = static_cast<__nv_bfloat16*>(w.o.p) + x.n * w.o.sn + x.h * w.o.sh + x.t0 * w.o.st + (kC * chunk + 16 * rb) * st + x.v0 + 8 * kOV * ch;
      const int rows = min(16, L - 16 * rb), cols = left - 8 * kOV * ch;
      if (((uintptr_t)o % 16 | w.o.st % 8 | w.V % 8) == 0) {
        const int r = lane / kOV, e = lane % kOV;
        if (8 * e < cols)
#pragma unroll
          for (int z = 0; z < 16; z += 32 / kOV)
            if (r + z < rows) *reinterpret_cast<uint4*>(o + (r + z) * st + 8 * e) = *reinterpret_cast<const uint4*>(own + (r + z) * P::kPitch + 16 * e);
      } else {
        for (int r = 0; r < rows; ++r)
          for (int j = lane; j < min(cols, 8 * kOV); j += 32) o[r * st + j] = reinterpret_cast<const __nv_bfloat16*>(own + r * P::kPitch)[j];
      }
    }
    if (more) {
      if (P::kSplit > 1) asm volatile("bar.sync %0, 64;" ::"r"(1 + rb) : "memory");
      else __syncwarp();        // (the rows of q have been read)
      fetch_q(x2, L2);
      if (P::kInV && received) __syncthreads();  // (and S)
      fetch_v(x2, L2, stage ^ 1);
    }
    copies_commit();

    // ---- the state
    if (hands_on) {
      float U[kNV][4];
#pragma unroll
      for (int j = 0; j < kNV; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) U[j][e] = 0.f;
      const bool keeps = !drops.m && !drops.end;
      if (16 * warp < K) {
#pragma unroll 1
        for (int kb = max(drop_last, 0) >> 4; 16 * kb < L; ++kb) {
          // decayed k: 16 rows, this warp's columns
          uint32_t k[4], hi[4], mid[4], lo[4];
          ldsm_t(k_at + (uint32_t)(16 * kb * P::kPitch) + 32 * warp + b_at, k);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint64_t g = *reinterpret_cast<const uint64_t*>(leave + 16 * kb + 8 * h + 2 * tq);
#pragma unroll
            for (int i = 2 * h; i < 2 * h + 2; ++i) {
              const uint64_t a = tc::f2_mul(pair_of(k[i]), g);
              hi[i] = bf16_of(a);
              const uint64_t r = tc::f2_sub(a, pair_of(hi[i]));
              mid[i] = bf16_of(r);
              if (three) lo[i] = bf16_of(tc::f2_sub(r, pair_of(mid[i])));
            }
          }
#pragma unroll
          for (int g = 0; g < kVB / 16; ++g) {
            uint32_t v[4];
            ldsm_t(v_at + (uint32_t)(16 * kb * P::kPitchV) + 32 * g + v_off, v);
            mma(U[2 * g], hi, v[0], v[1]);
            mma(U[2 * g + 1], hi, v[2], v[3]);
            mma(U[2 * g], mid, v[0], v[1]);
            mma(U[2 * g + 1], mid, v[2], v[3]);
            if (three) {
              mma(U[2 * g], lo, v[0], v[1]);
              mma(U[2 * g + 1], lo, v[2], v[3]);
            }
          }
        }
        // What is not finite: masked rows are 0 times it, and so are parts that are 0.
        uint64_t zero = 0;
#pragma unroll
        for (int j = 0; j < kNV; ++j) zero = tc::f2_fma(tc::f2_pack(U[j][0], U[j][1]), 0, tc::f2_fma(tc::f2_pack(U[j][2], U[j][3]), 0, zero));
        float z0, z1;
        tc::f2_unpack(zero, z0, z1);
        if (__any_sync(~0u, !(z0 + z1 == 0.f))) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            float n[2 * kNV] = {};
            for (int j = max(drop_last, 0); j < L; ++j) {
              const float kw = val(k_tile + j * P::kPitch, 16 * warp + tr + 8 * h) * leave[j];
#pragma unroll
              for (int i = 0; i < 2 * kNV; ++i) n[i] += kw * val(v_tile + j * P::kPitchV, 8 * (i / 2) + 2 * tq + i % 2);
            }
#pragma unroll
            for (int i = 0; i < 2 * kNV; ++i) {
              float& a = U[i / 2][2 * h + i % 2];
              if (!finite(a)) a = n[i];
            }
          }
          __syncwarp();
        }
      }
      const uint64_t g = twice(gp[max(L, 0)]);
#pragma unroll
      for (int j = 0; j < kNV; ++j)
#pragma unroll
        for (int e = 0; e < 4; e += 2) {
          uint64_t f = tc::f2_pack(U[j][e], U[j][e + 1]);
          if (keeps) f = tc::f2_fma(tc::f2_pack(S[j][e], S[j][e + 1]), g, f);
          tc::f2_unpack(f, S[j][e], S[j][e + 1]);
        }
    }

    if (warp == 0 && more) share_resets(stage ^ 1);
    __syncthreads();            // (S has been read)
    // ---- the end of a chain's segment
    if (!last) {
      if (!kStates) plane_out(stage ^ 1);
    } else {
      if (!kStates && w.o.p && c.lengths) {  // steps behind the end
        const int64_t lo = (int64_t)x.seg * c.seg_len, hi = min(c.T, lo + c.seg_len);
        __nv_bfloat16* o = static_cast<__nv_bfloat16*>(w.o.p) + x.n * w.o.sn + x.h * w.o.sh;
        for (int64_t r = lo + x.live + warp; r < hi; r += P::kThreads / 32)
          for (int j = x.v0 + lane; j < min(w.V, x.v0 + kVB); j += 32) o[r * w.o.st + j] = __float2bfloat16_rn(0.f);
      }
      const int64_t KV = (int64_t)K * w.V, chain = x.n * c.H + x.h;
      float* s_out = nullptr;
      if (kStates) {
        s_out = w.seg + ((int64_t)x.seg * c.N * c.H + chain) * KV;
        if (threadIdx.x == 0 && x.h == 0 && x.wi == 0 && x.v0 == 0) c.seg_live[(int64_t)x.seg * c.N + x.n] = any_reset ? -1 : x.live;
      } else if (out) {
        s_out = w.s_out + chain * KV;
      }
      if (s_out) {
        s_out += x.v0;
        const bool two = w.V % 2 == 0 && (uintptr_t)s_out % 8 == 0;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int k = 16 * warp + tr + 8 * h;
          if (k >= K) break;
          float* r = s_out + (int64_t)k * w.V + 2 * tq;
#pragma unroll
          for (int j = 0; j < kNV; ++j) {
            const int v = 8 * j + 2 * tq;
            if (two) {
              if (v < left) *reinterpret_cast<float2*>(r + 8 * j) = float2{S[j][2 * h], S[j][2 * h + 1]};
            } else {
              if (v < left) r[8 * j] = S[j][2 * h];
              if (v + 1 < left) r[8 * j + 1] = S[j][2 * h + 1];
            }
          }
        }
      }
      if (!more) break;
      fetch_state(x2);
    }
    u = u2, chunk = chunk2, turn ^= last ? 1 : 0, stage ^= 1;
  }
  copies_wait<0>();
}

// seg[s] holds segment s's U and becomes the state it receives, in the walk's order.  A thread an element, 256 of one
// chain a CTA (its divisions are 32 bits wide); kHand segments' U at a time, so that their loads are in flight together.
constexpr int kHand = 8;
__global__ void __launch_bounds__(256) hand_over(const __grid_constant__ Chains c) {
  tc::after_previous();
  const Walk& w = c.w[blockIdx.y];
  const uint32_t KV = (uint32_t)(w.K * w.V), parts = (KV + 255) / 256, chain = blockIdx.x / parts;
  const uint32_t e = (blockIdx.x - chain * parts) * 256 + threadIdx.x, n = chain / (uint32_t)c.H;
  if (e >= KV) return;
  const int64_t all = c.N * c.H * KV;
  const float l2 = log2_decay(c.log_decay, (int)(chain - n * (uint32_t)c.H));
  float s = w.s_in ? w.s_in[(int64_t)chain * KV + e / (uint32_t)w.V * w.si_in + e % (uint32_t)w.V * w.sj_in] : 0.f;
  const int first = w.back ? c.segs - 1 : 0, by = w.back ? -1 : 1;
  float* at = w.seg + first * all + (int64_t)chain * KV + e;
  const int32_t* live = c.seg_live + first * c.N + n;
  for (int j = 0; j < c.segs; j += kHand, at += by * kHand * all, live += by * kHand * c.N) {
    float u[kHand], g[kHand];
#pragma unroll
    for (int i = 0; i < kHand; ++i)
      if (j + i < c.segs) {
        u[i] = at[by * i * all];
        const int steps = live[by * i * c.N];
        g[i] = steps < 0 ? -1.f : exp2f(l2 * (float)steps);
      }
#pragma unroll
    for (int i = 0; i < kHand; ++i)
      if (j + i < c.segs) {
        at[by * i * all] = s;
        s = g[i] < 0.f ? u[i] : s * g[i] + u[i];   // (an episode begins within the segment)
      }
  }
}

// ---- one step (T = 1): the serving form -------------------------------------------------------
// The state is read and written once and bounds it, or, for few chains, the latency of that one reading: a thread has VC
// neighbouring columns of every R-th row, up to eight rows' loads at once, and the rows' sums are joined in shared memory.
// (By `walk`, which stages its rows first: 64x4 64x64 bf16 7.9 us a launch in a graph, this way 3.8; 256x4 128x128 60,
// 36; 4096x4 32x32 68, 36.)
constexpr int kStepThreads = 256, kStepRows = 8;    // rows of a thread that are loaded at once

struct Step {
  Walk w;
  const float* log_decay;
  const uint8_t* reset;
  const int32_t* lengths;
  int32_t H, cols, rows, per;   // threads along a row of the state, row groups, chains of a CTA
  uint32_t chains;
};

template <typename E, int VC>
__global__ void __launch_bounds__(kStepThreads) one_step(const __grid_constant__ Step c) {
  tc::after_previous();
  __shared__ float red[kStepThreads * VC];
  const Walk& w = c.w;
  const int K = w.K, V = w.V, of_chain = c.cols * c.rows;
  const int inst = threadIdx.x / of_chain, i = threadIdx.x - inst * of_chain, r = i / c.cols, col = (i - r * c.cols) * VC;
  const uint32_t chain = blockIdx.x * c.per + inst;
  if (inst < c.per && chain < c.chains) {
    const uint32_t n = chain / (uint32_t)c.H, h = chain - n * (uint32_t)c.H;
    const bool live = !c.lengths || c.lengths[n] > 0, fresh = c.reset && c.reset[n];
    const float g = exp2f(log2_decay(c.log_decay, (int)h));
    const E* qs = static_cast<const E*>(w.q.p) + n * w.q.sn + h * w.q.sh;
    const E* ks = static_cast<const E*>(w.k.p) + n * w.k.sn + h * w.k.sh;
    const E* v = static_cast<const E*>(w.v.p) + n * w.v.sn + h * w.v.sh + col;
    const int64_t at = (int64_t)chain * K * V + col;
    float x[VC], sum[VC];
#pragma unroll
    for (int j = 0; j < VC; ++j) x[j] = as_f32<E>(v[j]), sum[j] = 0.f;
    for (int k0 = r; k0 < K; k0 += kStepRows * c.rows) {
      float S[kStepRows][VC], q[kStepRows], k[kStepRows];
#pragma unroll
      for (int z = 0; z < kStepRows; ++z) {
        const int row = k0 + z * c.rows;
#pragma unroll
        for (int j = 0; j < VC; ++j) S[z][j] = 0.f;
        if (row < K) {
          q[z] = as_f32<E>(qs[row]), k[z] = as_f32<E>(ks[row]);
          if (w.s_in) {
            const float* s = w.s_in + at + row * V;
            if constexpr (VC == 4) {
              const float4 f = *reinterpret_cast<const float4*>(s);
              S[z][0] = f.x, S[z][1] = f.y, S[z][2] = f.z, S[z][3] = f.w;
            } else {
              S[z][0] = *s;
            }
          }
        }
      }
#pragma unroll
      for (int z = 0; z < kStepRows; ++z) {
        const int row = k0 + z * c.rows;
        if (row >= K) break;
        if (live) {             // (a reset drops the state whatever it holds)
#pragma unroll
          for (int j = 0; j < VC; ++j) {
            S[z][j] = fmaf(k[z], x[j], fresh ? 0.f : g * S[z][j]);
            sum[j] = fmaf(q[z], S[z][j], sum[j]);
          }
        }
        if (w.s_out) {
          float* s = w.s_out + at + row * V;
          if constexpr (VC == 4) *reinterpret_cast<float4*>(s) = float4{S[z][0], S[z][1], S[z][2], S[z][3]};
          else *s = S[z][0];
        }
      }
    }
#pragma unroll
    for (int j = 0; j < VC; ++j) red[threadIdx.x * VC + j] = sum[j];
  }
  __syncthreads();
  if (!w.o.p) return;
  for (int t = threadIdx.x; t < c.per * V; t += kStepThreads) {
    const int of = t / V, column = t - of * V;
    const uint32_t ch = blockIdx.x * c.per + of;
    if (ch >= c.chains) break;
    float y = 0.f;
    const float* p = red + of * of_chain * VC + column;   // (a row group's columns lie in order)
    for (int z = 0; z < c.rows; ++z) y += p[z * c.cols * VC];
    const uint32_t n = ch / (uint32_t)c.H, h = ch - n * (uint32_t)c.H;
    static_cast<E*>(w.o.p)[n * w.o.sn + h * w.o.sh + column] = rounded<E>(y * w.out);
  }
}

// ---- host ---------------------------------------------------------------------------------
// How a call runs.
struct How {
  bool tc;                      // `chunks`, else `walk`
  int D;                        // chunks: heads' widths padded
  int KT, KS, COLS;             // walk: how a state's columns lie in warps
  int64_t units;                // CTAs (chunks) or warps (walk) without a split
  int segs;
  int64_t seg_len;
};

constexpr int kFill = 152 * 16;  // warps of `walk` that keep every SM busy
// From how many steps of a chunk on a bf16 pass goes by chunks: one costs the same whatever it holds, a step of `walk` by the
// size of its state, and few chains wait for steps (`few`: their chunks run at one time).  Forward passes of 4 heads,
// chunks against `walk` (us): 256 envs 128x128 T = 2 55, 61; 512 envs 96x96 T = 4 98, 86; 4096 envs 64x64 T = 8 205, 164,
// T = 10 203, 197, T = 12 205, 209; 64 envs 64x64 T = 6 12, 14; 4096 envs 32x32 T = 16 162, 143, T = 20 178, 170, T = 24 180,
// 184; 150 envs 32x32 T = 12 12, 16; 4096 envs 16x16 T = 64 217, 195, T = 80 328, 238, T = 128 391, 367 (backward, a third of
// the envs, T = 64 231, 256, T = 128 466, 487); 150 envs 16x16 T = 24 12, 14; 300 envs T = 24 18, 16, T = 48 21, 23.
int chunk_steps(int deep, int64_t chains) {
  const bool few = chains <= 152 * 4;
  return deep > 64 ? 2 : deep > 32 ? (few ? 6 : 10) : deep > 16 ? (few ? 12 : 20) : few ? 24 : chains <= 2 * 152 * 4 ? 32 : 60;
}

How how(int64_t T, int64_t N, int H, int K, int V, int walks, bool bf16) {
  How p{};
  const int wide = walks > 1 ? std::max(K, V) : V, deep = walks > 1 ? wide : K;   // (walks may have them exchanged)
  p.tc = bf16 && T >= chunk_steps(deep, N * H * walks) * ((T + kC - 1) / kC);
  int64_t want, len = std::max<int64_t>(T, 1);
  int step;
  if (p.tc) {
    p.D = deep <= 64 ? 64 : 128;
    const auto blocks = [](int v) { return (v + kVB - 1) / kVB; };
    p.units = N * H * (walks > 1 ? 2 * blocks(K) + blocks(V) : blocks(V));   // (dq and dk have K columns, dv has V)
    step = kC;
    want = std::min<int64_t>(152 * (p.D == 64 ? TcPlan<64>::kCtas : TcPlan<128>::kCtas) / p.units, T / kC);
  } else {
    // 33 to 64 rows and columns, two layouts: a warp a head (half the operands from shared memory, 318 instructions a
    // step for 418) or two warps with half the registers, for so few heads that their steps, 32 at least to a segment,
    // do not make 304 warps.  fp32 forward 64x64, first against second (us): T = 128, heads 8 48, 38; 64 52, 44; 152 54,
    // 56; 549 114, 130; 1100 96, 125; 2432 184, 236; T = 1000, 8 58, 48; 64 89, 101; 549 503, 611; T = 61, 152 39, 39;
    // 549 41, 47.  50x33 backward: T = 61, 150 39, 37; 600 39, 45; T = 400, 402 175, 192; 900 291, 289.
    const int64_t heads = N * H * walks;
    if (deep > 32 && deep <= 64 && wide > 32 && wide <= 64 && heads * std::max<int64_t>(1, T / 32) >= 304)
      p.KT = 64, p.KS = 1, p.COLS = 2;
    else
      p.KT = deep > 64 ? 32 : 16, p.KS = deep > 32 ? 4 : deep > 16 ? 2 : 1, p.COLS = deep > 64 ? 2 : deep <= 16 && wide <= 32 ? 1 : 4;
    p.units = heads * ((wide + 32 / p.KS * p.COLS - 1) / (32 / p.KS * p.COLS));
    step = kWindow;
    want = bf16 ? 1 : std::min<int64_t>((p.KT == 64 ? 152 * 8 : kFill) / p.units, T / 32);   // (few bf16 chains go by chunks)
  }
  if (want >= 2) {
    len = (T + want - 1) / want;
    len = (len + step - 1) / step * step;
  }
  p.segs = (int)std::max<int64_t>(1, (T + len - 1) / len);
  p.seg_len = len;
  return p;
}

int64_t workspace_of(int64_t T, int64_t N, int H, int K, int V, int walks, bool bf16) {
  const How p = how(T, N, H, K, V, walks, bf16);
  return p.segs < 2 ? 0 : ((int64_t)walks * p.segs * N * H * K * V + (p.segs * N + 3) / 4 * 4) * 4;
}

template <typename E, int KT, int KS, int COLS>
aht_status run(const Chains& c, int64_t units, bool states, cudaStream_t s) {
  const Shape sh{dim3((unsigned)((units + kWarps - 1) / kWarps)), dim3(32 * kWarps), kWarps * Plan<E, KT, KS, COLS>::kBytes};
  if constexpr (sizeof(E) == 4)   // (a bf16 pass of steps is not split)
    if (states) return launch_op(walk<E, KT, KS, COLS, true>, sh, s, c, units);
  return launch_op(walk<E, KT, KS, COLS, false>, sh, s, c, units);
}
template <typename E>
aht_status run(const How& p, const Chains& c, bool states, cudaStream_t s) {
  const int64_t units = p.units * p.segs;
  if (p.KT == 64) return run<E, 64, 1, 2>(c, units, states, s);
  if (p.KT == 32) return run<E, 32, 4, 2>(c, units, states, s);
  if (p.KS == 4) return run<E, 16, 4, 4>(c, units, states, s);
  if (p.KS == 2) return run<E, 16, 2, 4>(c, units, states, s);
  return p.COLS == 4 ? run<E, 16, 1, 4>(c, units, states, s) : run<E, 16, 1, 1>(c, units, states, s);
}
template <int D>
aht_status run_chunks(const How& p, const Chains& c, bool states, cudaStream_t s) {
  const int64_t units = p.units * p.segs;
  const Shape sh{dim3((unsigned)std::min<int64_t>(units, 152 * TcPlan<D>::kCtas)), dim3(TcPlan<D>::kThreads), TcPlan<D>::kBytes};
  return states ? launch_op(chunks<D, true>, sh, s, c, (uint32_t)units) : launch_op(chunks<D, false>, sh, s, c, (uint32_t)units);
}

template <typename E>
aht_status run_step(const Chains& c, cudaStream_t s) {
  Step p{c.w[0], c.log_decay, c.reset, c.lengths, c.H, 0, 0, 0, (uint32_t)(c.N * c.H)};
  const bool fours = p.w.V % 4 == 0 && on_boundary(16, p.w.s_in, p.w.s_out);
  p.cols = fours ? p.w.V / 4 : p.w.V;
  // rows of a thread: more in flight (4096x4 64x64 bf16 117 us, with half of them 158), or more threads for few chains
  const int each = p.chains > 512 ? kStepRows : kStepRows / 2;
  p.rows = std::max(1, std::min(kStepThreads / p.cols, (p.w.K + each - 1) / each));
  p.per = kStepThreads / (p.cols * p.rows);
  const Shape sh{dim3((p.chains + p.per - 1) / p.per), dim3(kStepThreads)};
  return fours ? launch_op(one_step<E, 4>, sh, s, p) : launch_op(one_step<E, 1>, sh, s, p);
}

aht_status walks(const aht_linattn_args* a, Chains& c, void* workspace, cudaStream_t s) {
  const bool bf16 = a->dtype == AHT_BF16;
  const How p = how(a->T, a->N, a->H, a->K, a->V, c.walks, bf16);
  c.segs = p.segs;
  c.seg_len = p.seg_len;
  for (int i = 0; i < c.walks; ++i)
    for (int b = 0; b * kVB < c.w[i].V; ++b, ++c.parts) c.part_walk[c.parts] = (uint8_t)i, c.part_block[c.parts] = (uint8_t)b;
  float* at = static_cast<float*>(workspace);
  for (int i = 0; i < c.walks && p.segs > 1; ++i, at += (int64_t)p.segs * a->N * a->H * a->K * a->V) c.w[i].seg = at;
  c.seg_live = reinterpret_cast<int32_t*>(at);
  auto go = [&](bool states) {
    if (p.tc) return p.D == 64 ? run_chunks<64>(p, c, states, s) : run_chunks<128>(p, c, states, s);
    return bf16 ? run<__nv_bfloat16>(p, c, states, s) : run<float>(p, c, states, s);
  };
  if (p.segs > 1) {
    if (aht_status e = go(true)) return e;
    const int64_t ctas = a->N * a->H * (((int64_t)a->K * a->V + 255) / 256);
    if (aht_status e = launch_op(hand_over, Shape{dim3((unsigned)ctas, (unsigned)c.walks), dim3(256), 0}, s, c)) return e;
  }
  return go(false);
}

Rows rows(const aht_heads& h) { return Rows{h.data, h.st, h.sn, h.sh}; }

aht_status check(const aht_linattn_args* a) {
  if (!a) return set_last_error(AHT_EINVAL, "args is NULL");
  if (a->dtype != AHT_FP32 && a->dtype != AHT_BF16) return set_last_error(AHT_EINVAL, "dtype must be AHT_FP32 or AHT_BF16");
  if (a->T < 0 || a->N < 1 || a->H < 1 || a->H > AHT_LINATTN_MAX_HEADS || a->K < 1 || a->K > AHT_LINATTN_MAX_DIM || a->V < 1 ||
      a->V > AHT_LINATTN_MAX_DIM)
    return set_last_error(AHT_EINVAL, "sizes: T >= 0, N >= 1, H in 1..AHT_LINATTN_MAX_HEADS, K and V in 1..AHT_LINATTN_MAX_DIM");
  if (a->N > (int64_t(1) << 24) / a->H || a->T > (int64_t(1) << 30) || (a->T > 0 && a->N > (int64_t(1) << 40) / a->H / a->T))
    return set_last_error(AHT_EINVAL, "N * H must be at most 2^24, T at most 2^30 and T * N * H at most 2^40");
  if (!a->log_decay) return set_last_error(AHT_EINVAL, "log_decay is NULL");
  if (a->T > 0 && (!a->q.data || !a->k.data || !a->v.data)) return set_last_error(AHT_EINVAL, "NULL input sequence");
  if (!on_boundary(a->dtype == AHT_FP32 ? 4 : 2, a->q.data, a->k.data, a->v.data) || !on_boundary(4, a->log_decay, a->lengths))
    return set_last_error(AHT_EINVAL, kMisalignedArray);
  return AHT_OK;
}

aht_status check_workspace(const aht_linattn_args* a, int walks, const void* ws, int64_t bytes) {
  const int64_t need = workspace_of(a->T, a->N, a->H, a->K, a->V, walks, a->dtype == AHT_BF16);
  if (need > 0 && (!ws || bytes < need))
    return set_last_error(AHT_EINVAL, "workspace is NULL or smaller than aht_linattn_workspace");
  return on_boundary(16, ws) ? AHT_OK : set_last_error(AHT_EINVAL, "workspace must be on a boundary of 16 bytes");
}

Chains chains_of(const aht_linattn_args* a) {
  Chains c{};
  c.T = a->T, c.N = a->N, c.H = a->H;
  c.log_decay = a->log_decay, c.reset = a->reset, c.lengths = a->lengths;
  return c;
}

}  // namespace

extern "C" {

int64_t aht_linattn_workspace(int64_t T, int64_t N, int32_t H, int32_t K, int32_t V, int32_t dtype) {
  const bool bf16 = dtype == AHT_BF16;
  if (T < 0 || N < 1 || H < 1 || K < 1 || V < 1 || K > AHT_LINATTN_MAX_DIM || V > AHT_LINATTN_MAX_DIM) return 0;
  return std::max(workspace_of(T, N, H, K, V, 1, bf16), workspace_of(T, N, H, K, V, 3, bf16));
}

aht_status aht_linattn_forward(const aht_linattn_args* a, const float* s0, const aht_heads* o, float* s_last, void* workspace,
                               int64_t workspace_bytes, void* cuda_stream) {
  if (aht_status e = check(a)) return e;
  if (!s_last && (!o || !o->data)) return set_last_error(AHT_EINVAL, "neither o nor s_last is asked for");
  if (!on_boundary(a->dtype == AHT_FP32 ? 4 : 2, o ? o->data : nullptr) || !on_boundary(4, s0, s_last))
    return set_last_error(AHT_EINVAL, kMisalignedArray);
  if (aht_status e = check_workspace(a, 1, workspace, workspace_bytes)) return e;
  Chains c = chains_of(a);
  c.walks = 1;
  c.w[0] = Walk{rows(a->q), rows(a->k), rows(a->v), o ? rows(*o) : Rows{}, a->K, a->V, 0, 1.f, a->scale, s0, s_last, a->V, 1, nullptr};
  if (a->T == 1) return a->dtype == AHT_BF16 ? run_step<__nv_bfloat16>(c, static_cast<cudaStream_t>(cuda_stream))
                                             : run_step<float>(c, static_cast<cudaStream_t>(cuda_stream));
  return walks(a, c, workspace, static_cast<cudaStream_t>(cuda_stream));
}

aht_status aht_linattn_backward(const aht_linattn_args* a, const float* s0, const aht_heads* d_o, const float* ds_last,
                                const aht_heads* dq, const aht_heads* dk, const aht_heads* dv, float* ds0, void* workspace,
                                int64_t workspace_bytes, void* cuda_stream) {
  if (aht_status e = check(a)) return e;
  if (!d_o || !dq || !dk || !dv || (a->T > 0 && (!d_o->data || !dq->data || !dk->data || !dv->data)))
    return set_last_error(AHT_EINVAL, "NULL gradient sequence");
  if (!on_boundary(a->dtype == AHT_FP32 ? 4 : 2, d_o->data, dq->data, dk->data, dv->data) || !on_boundary(4, s0, ds_last, ds0))
    return set_last_error(AHT_EINVAL, kMisalignedArray);
  if (aht_status e = check_workspace(a, 3, workspace, workspace_bytes)) return e;
  Chains c = chains_of(a);
  c.walks = 3;
  const Rows q = rows(a->q), k = rows(a->k), v = rows(a->v), g = rows(*d_o);
  const int32_t K = a->K, V = a->V;
  c.w[0] = Walk{g, v, k, rows(*dq), V, K, 0, 1.f, a->scale, s0, nullptr, 1, V, nullptr};          // state S^T
  c.w[1] = Walk{v, g, q, rows(*dk), V, K, 1, a->scale, 1.f, ds_last, nullptr, 1, V, nullptr};     // G^T
  c.w[2] = Walk{k, q, g, rows(*dv), K, V, 1, a->scale, 1.f, ds_last, ds0, V, 1, nullptr};         // G
  return walks(a, c, workspace, static_cast<cudaStream_t>(cuda_stream));
}

}  // extern "C"
