// policy_loss.cu -- the clipped policy loss with a KL term and its gradient (include/aht.h states it).
//
// A row's sums over the actions, with xm = x - max x and ym = y - max y of the reference's logits y:
//   s = sum e^xm, u = sum e^xm xm, t = sum e^xm (xm - ym), sy = sum e^ym;
//   logp = xm_action - log s,  H = log s - u / s,  KL = t / s - log s + log sy,
// and the gradient from them and the row's own numbers c:
//   e^xm_j (c + cx xm_j - cy ym_j),  + w at where j is the action.
// So a row is gone through twice.  What bounds it is memory: each logit is read from it once and its
// gradient written once; long rows execute about 41 instructions an element over both readings.
//   tiles: up to 64 actions.  Rows lie densely, so a tile of them is copied to shared memory as one span; a
//     thread takes a row (up to 32 actions in registers), beginning at an element of its own so that a warp's
//     reads fall into all banks.
//   rows: more.  A warp, or a CTA, takes a row, and reads it a second time from L1 or L2.  What a CTA reads first stays
//     in L2 until then (evict_last), what it reads again and writes goes first: without that, 304 rows of 256 KB at a
//     time found 14 % of themselves there (4096 x 65536 bf16: 484 us, 440 with it, every logit from memory once; a
//     cluster of CTAs a row that keeps it in shared memory 1144, the clusters' barriers).
// Sums over rows: two fp32 a thread (value and rounding error), fp64 from there, in a fixed order.
#include <cuda_bf16.h>

#include <algorithm>
#include <limits>

#include "op_launch.cuh"

using namespace aht;

namespace {

constexpr int kSums = 5;         // of w times: the clipped term, KL, H, 1 where clipped, 1
constexpr int kMaxCtas = 152 * 16;
constexpr float kInf = std::numeric_limits<float>::infinity();

struct Loss {
  int64_t M, A;
  const void *x, *y, *actions;   // y: the reference's logits or NULL
  void* d;
  int64_t ldx, ldy, ldd;
  const float *old_logp, *adv, *weight, *ref_logp;
  const uint8_t* legal;
  float *logp, *stats;
  double* part;                  // [kSums][kMaxCtas]
  float lo, hi, kl, ent;         // clip borders, coefficients
  float w;                       // without weights
  int action_bytes;
};

constexpr float kLog2e = 1.4426950408889634f;

// e^x for x <= 0: 2 ulp of the hardware exp2, and 2^-24 |x| from its argument (where e^x is small).
__device__ __forceinline__ float exp_of(float x) { return tc::ex2_approx(x * kLog2e); }

// What a row's second pass needs; `on`: it takes part.
struct Row {
  float max_x, max_y, c, cx, cy, at;
  bool on;
};

__device__ __forceinline__ int64_t action_of(const Loss& l, int64_t m) {
  if (l.action_bytes == 1) return static_cast<const uint8_t*>(l.actions)[m];
  if (l.action_bytes == 4) return static_cast<const int32_t*>(l.actions)[m];
  return static_cast<const int64_t*>(l.actions)[m];
}

__device__ __forceinline__ float f32(float v) { return v; }
__device__ __forceinline__ float f32(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename E> __device__ __forceinline__ E rounded(float v);
template <> __device__ __forceinline__ float rounded<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 rounded<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// A row's sums in progress, about the maxima so far.
struct Sums {
  float mx = -kInf, s = 0.f, u = 0.f, t = 0.f, my = -kInf, sy = 0.f;
};

// Moves a row's sums to the maximum `to` of x, and by shift_y in y.  Empty ones, and ones that vanish, become 0; s that is
// not a number stays so, whatever the factor.
__device__ __forceinline__ void move_x(Sums& a, float to, float shift_y) {
  const float d = a.mx - to, r = a.mx == -kInf ? 0.f : exp_of(d);
  a.t = r > 0.f ? r * (a.t + a.s * (d - shift_y)) : 0.f;
  a.u = r > 0.f ? r * (a.u + a.s * d) : 0.f;
  a.s = r * a.s;
  a.mx = to;
}
template <bool kRef>
__device__ __forceinline__ void move_to(Sums& a, float mx, float my) {
  const float dy = kRef && a.my != -kInf ? a.my - my : 0.f;
  move_x(a, mx, dy);
  if (kRef) {
    a.sy *= a.my == -kInf ? 0.f : exp_of(dy);
    a.my = my;
  }
}
template <bool kRef> __device__ __forceinline__ void join(Sums& a, Sums b) {
  const float mx = fmaxf(a.mx, b.mx), my = kRef ? fmaxf(a.my, b.my) : 0.f;
  move_to<kRef>(a, mx, my);
  move_to<kRef>(b, mx, my);
  a.s += b.s, a.u += b.u, a.t += b.t, a.sy += b.sy;
}

// Compensated running sum.
struct Acc {
  float hi = 0.f, lo = 0.f;
  __device__ __forceinline__ void add(float v) {
    const float s = hi + v, b = s - hi;
    lo += (hi - (s - b)) + (v - b);
    hi = s;
  }
  // (of an infinite sum the error is not a number, and the sum says all)
  __device__ __forceinline__ double sum() const { return fabsf(hi) < kInf ? (double)hi + (double)lo : (double)hi; }
};

// e^d - 1 - d.  Near 0, where the difference cancels, its series (to 2^-26.3 of it for |d| < 1/4).
__device__ __forceinline__ float excess(float d) {
  if (fabsf(d) < 0.25f)
    return d * d * (0.5f + d * (1.f / 6 + d * (1.f / 24 + d * (1.f / 120 + d * (1.f / 720 + d * (1.f / 5040))))));
  return expm1f(d) - d;
}

// From the sums over a row to what its gradient needs; the first thread of the row's writes logp and
// adds to the totals.
template <bool kRef>
__device__ __forceinline__ Row finish(const Loss& l, int64_t m, bool on, float xa, const Sums& s, bool first, Acc (&acc)[kSums]) {
  Row r{};
  r.on = on && !(s.mx == -kInf && s.s == 0.f);   // (not a number: the row says so)
  if (!r.on) {
    if (first && l.logp) l.logp[m] = 0.f;
    return r;
  }
  const float w = l.weight ? l.weight[m] : l.w, adv = l.adv[m];
  const float ls = logf(s.s), logp = (xa - s.mx) - ls, inv = 1.f / s.s, H = ls - s.u * inv;
  const float moved = logp - l.old_logp[m], ratio = expf(moved);
  const bool clipped = adv > 0.f ? ratio > l.hi : adv < 0.f && ratio < l.lo;
  const float inside = ratio < l.lo ? l.lo : ratio > l.hi ? l.hi : ratio;  // (NaN stays)
  // (a ratio beyond fp32's range is a number all the same)
  const float a = adv == 0.f && moved < kInf && ratio == kInf ? 0.f : ratio * adv, b = inside * adv;
  const float pg = -(b < a ? b : a);
  float kl = 0.f, at = clipped ? 0.f : -a, lsy = 0.f;
  if (kRef) {
    lsy = logf(s.sy);
    kl = s.t * inv - (ls - lsy);
  } else if (l.ref_logp) {
    const float d = l.ref_logp[m] - logp;
    kl = excess(d);
    if (l.kl > 0.f) at -= l.kl * expm1f(d);
  }
  if (first) {
    if (l.logp) l.logp[m] = logp;
    acc[0].add(w * pg);
    acc[1].add(w * kl);
    acc[2].add(w * H);
    acc[3].add(clipped ? w : 0.f);
    acc[4].add(w);
  }
  // (formed in any case and selected: a branch around it made 2097152 x 20 fp32 148 us of 134)
  const float ws = w * inv, past = kRef ? ls - lsy + kl : 0.f;
  r.max_x = s.mx;
  r.max_y = s.my;
  r.c = ws * (l.ent * (H - ls) - l.kl * (l.kl > 0.f ? past : 0.f) - at);
  r.cx = ws * (l.ent + (kRef ? l.kl : 0.f));
  r.cy = kRef ? ws * l.kl : 0.f;
  r.at = w * at;
  return r;
}

// The gradient of one logit.
template <bool kRef>
__device__ __forceinline__ float slope(const Row& r, float x, float y, bool is_action) {
  const float xm = x - r.max_x, e = exp_of(xm);
  float g = r.c + r.cx * xm;
  if (kRef && r.cy != 0.f) g -= r.cy * (y - r.max_y);   // (without a KL term y may be infinite)
  g = e == 0.f ? 0.f : e * g;   // (0 * inf)
  return is_action ? g + r.at : g;
}

// kl_coef KL; without a coefficient nothing, whatever KL is.
__device__ __forceinline__ double kl_term(const Loss& l, double kl) { return l.kl > 0.f ? (double)l.kl * kl : 0.; }

// The CTA's totals: threads in order through shared memory.
__device__ void totals(const Loss& l, const Acc (&acc)[kSums], double* tmp) {
  __syncthreads();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
#pragma unroll
  for (int i = 0; i < kSums; ++i) {
    double v = acc[i].sum();
    for (int o = 16; o > 0; o >>= 1) v += __shfl_down_sync(~0u, v, o);
    if (lane == 0) tmp[warp * kSums + i] = v;
  }
  __syncthreads();
  if (threadIdx.x < kSums) {
    double v = 0.;
    for (int k = 0; k < warps; ++k) v += tmp[k * kSums + threadIdx.x];
    tmp[threadIdx.x] = v;  // (row 0 was read by this thread first)
    l.part[(int64_t)threadIdx.x * kMaxCtas + blockIdx.x] = v;
  }
  if (gridDim.x == 1) {
    __syncthreads();
    if (threadIdx.x == 0) {
      l.stats[0] = (float)(tmp[0] + kl_term(l, tmp[1]) - (double)l.ent * tmp[2]);
      for (int i = 0; i < kSums; ++i) l.stats[i + 1] = (float)tmp[i];
    }
  }
}

constexpr int kSumWarps = 4;     // of each sum
__global__ void __launch_bounds__(32 * kSums * kSumWarps) sum_parts(const __grid_constant__ Loss l, int parts) {
  tc::after_previous();
  __shared__ double tmp[kSumWarps][kSums];
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, i = w % kSums, q = w / kSums;
  const double* p = l.part + (int64_t)i * kMaxCtas;
  double v[4] = {};                                         // (four loads on their way at a time)
  for (int k = 32 * q + lane; k < parts; k += 128 * kSumWarps)
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (k + 32 * kSumWarps * j < parts) v[j] += p[k + 32 * kSumWarps * j];
  double t = (v[0] + v[1]) + (v[2] + v[3]);
  for (int o = 16; o > 0; o >>= 1) t += __shfl_down_sync(~0u, t, o);
  if (lane == 0) tmp[q][i] = t;
  __syncthreads();
  if (threadIdx.x != 0) return;
  double sum[kSums];
#pragma unroll
  for (int j = 0; j < kSums; ++j) {
    sum[j] = (tmp[0][j] + tmp[1][j]) + (tmp[2][j] + tmp[3][j]);
    l.stats[j + 1] = (float)sum[j];
  }
  l.stats[0] = (float)(sum[0] + kl_term(l, sum[1]) - (double)l.ent * sum[2]);
}

// ---- few actions: dense tiles of rows -------------------------------------------------------
constexpr int kTileRows = 128, kTileA = 64;  // (a thread a row)
constexpr int kTileCtas = 6;                 // an SM

__device__ __forceinline__ void copies_done() { asm volatile("cp.async.wait_all;" ::: "memory"); }

// Copies `rows` rows of A elements to a dense tile; `dense`: they are one 16-byte aligned span.
template <typename T>
__device__ __forceinline__ void tile_in(T* dst, const T* src, int64_t ld, int rows, int A, uint32_t inv, bool dense) {
  const int n = rows * A;
  constexpr int kPer = 16 / (int)sizeof(T);
  if (dense) {
    for (int i = threadIdx.x; i < n / kPer; i += kTileRows)
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(tc::smem_u32(dst + i * kPer)), "l"(src + i * kPer) : "memory");
    for (int i = n / kPer * kPer + threadIdx.x; i < n; i += kTileRows) dst[i] = src[i];
  } else {
    for (int i = threadIdx.x; i < n; i += kTileRows) {
      const int r = (int)((uint32_t)i * inv >> 20);
      dst[i] = src[r * ld + (i - r * A)];
    }
  }
}

// What stands for a logit that has no part, and the lowest one that is taken as it is: its distance to any other logit is
// finite, and 2^-100 of it above 0.  A power of two, so that its product with log2 e is exact but for that factor.
constexpr float kFar = -1.2676506002282294e30f;   // -2^100
constexpr uint32_t kFarBf16 = 0xF180F180u;        // a pair of them

// Four elements of a row.
__device__ __forceinline__ void load_4(const float* p, bool whole, int left, float (&v)[4]) {
  if (whole) {
    const float4 f = *reinterpret_cast<const float4*>(p);
    v[0] = f.x, v[1] = f.y, v[2] = f.z, v[3] = f.w;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = i < left ? p[i] : 0.f;
  }
}
__device__ __forceinline__ void load_4(const __nv_bfloat16* p, bool whole, int left, float (&v)[4]) {
  if (whole) {
    const uint2 f = *reinterpret_cast<const uint2*>(p);
    v[0] = __uint_as_float(f.x << 16), v[1] = __uint_as_float(f.x & 0xFFFF0000u);
    v[2] = __uint_as_float(f.y << 16), v[3] = __uint_as_float(f.y & 0xFFFF0000u);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = i < left ? f32(p[i]) : 0.f;
  }
}
__device__ __forceinline__ void store_4(float* p, bool whole, int left, const float (&v)[4]) {
  if (whole) {
    *reinterpret_cast<float4*>(p) = float4{v[0], v[1], v[2], v[3]};
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < left) p[i] = v[i];
  }
}
__device__ __forceinline__ void store_4(__nv_bfloat16* p, bool whole, int left, const float (&v)[4]) {
  if (whole) {
    *reinterpret_cast<uint2*>(p) = uint2{tc::pack_bf16(v[0], v[1]), tc::pack_bf16(v[2], v[3])};
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < left) p[i] = __float2bfloat16_rn(v[i]);
  }
}

// A row four actions at a time from group `turn` on, up to 4 kG actions in a thread's registers; with kG = 0 each of the
// three passes takes them from the tile again (295236 x 36 bf16, masked: 57 us, one action at a time 85).  False: a legal
// logit is so low that 0 * inf could arise, and nothing was done.
template <typename E, bool kRef, bool kLegal, int kG>
__device__ __forceinline__ bool row_by_fours(const Loss& l, int64_t m, int A, int act, E* xr, const E* yr, const uint8_t* lr, bool grad,
                                             Acc (&acc)[kSums]) {
  const int groups = (A + 3) / 4, turn = (int)threadIdx.x % groups;
  const bool whole = A % 4 == 0;
  auto group = [&](int g) { return 4 * (g + turn >= groups ? g + turn - groups : g + turn); };
  float lx = kInf, ly = kInf;
  auto take = [&](int g, float (&x)[4], float (&y)[4]) {
    const int j = group(g), left = A - j;
    load_4(xr + j, whole, left, x);
    if (kRef) load_4(yr + j, whole, left, y);
    uint32_t legal = 0xFFFFFFFFu;
    if (kLegal) {
      if (whole) {
        legal = *reinterpret_cast<const uint32_t*>(lr + j);
      } else {
        legal = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (i < left && lr[j + i]) legal |= 1u << (8 * i);
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const bool ok = (whole || i < left) && (!kLegal || (legal >> (8 * i) & 0xFFu));
      lx = ok ? fminf(lx, x[i]) : lx;
      x[i] = ok ? x[i] : kFar;  // (e^x of it is 0, and times it as well)
      if (kRef) {
        ly = ok ? fminf(ly, y[i]) : ly;
        y[i] = ok ? y[i] : kFar;
      }
    }
  };
  // f(group, its values) of every group: from registers, or from the tile again
  constexpr int kHeld = kG > 0 ? kG : 1;
  float hx[kHeld][4], hy[kHeld][4];
  auto each = [&](auto&& f) {
    if constexpr (kG > 0) {
#pragma unroll
      for (int g = 0; g < kG; ++g)
        if (g < groups) f(g, hx[g], hy[g]);
    } else {
#pragma unroll 2
      for (int g = 0; g < groups; ++g) {
        float x[4], y[4];
        take(g, x, y);
        f(g, x, y);
      }
    }
  };
  if constexpr (kG > 0) {
#pragma unroll
    for (int g = 0; g < kG; ++g)
      if (g < groups) take(g, hx[g], hy[g]);
  }
  Sums s;
  each([&](int, const float (&x)[4], const float (&y)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      s.mx = fmaxf(s.mx, x[i]);
      if (kRef) s.my = fmaxf(s.my, y[i]);
    }
  });
  if (!(lx > kFar) || (kRef && !(ly > kFar))) return false;
  const uint64_t l2 = tc::f2_pack(kLog2e, kLog2e), mx = tc::f2_pack(-s.mx, -s.mx), my = tc::f2_pack(-s.my, -s.my);
  uint64_t ps = 0, pu = 0, pt = 0, py = 0;
  auto exp_2 = [&](uint64_t v) {
    float a, b;
    tc::f2_unpack(tc::f2_mul(v, l2), a, b);
    return tc::f2_pack(tc::ex2_approx(a), tc::ex2_approx(b));
  };
  each([&](int, const float (&x)[4], const float (&y)[4]) {
#pragma unroll
    for (int i = 0; i < 4; i += 2) {
      const uint64_t xm = tc::f2_add(tc::f2_pack(x[i], x[i + 1]), mx), e = exp_2(xm);
      ps = tc::f2_add(ps, e);
      pu = tc::f2_fma(e, xm, pu);
      if (kRef) {
        const uint64_t ym = tc::f2_add(tc::f2_pack(y[i], y[i + 1]), my);
        pt = tc::f2_fma(e, tc::f2_sub(xm, ym), pt);
        py = tc::f2_add(py, exp_2(ym));
      }
    }
  });
  float a, b;
  tc::f2_unpack(ps, a, b), s.s = a + b;
  tc::f2_unpack(pu, a, b), s.u = a + b;
  tc::f2_unpack(pt, a, b), s.t = a + b;
  tc::f2_unpack(py, a, b), s.sy = a + b;
  const float xa = f32(xr[act]), ya = kRef ? f32(yr[act]) : 0.f;
  const Row row = finish<kRef>(l, m, true, xa, s, true, acc);
  if (!grad) return true;
  const uint64_t cc = tc::f2_pack(row.c, row.c), cx = tc::f2_pack(row.cx, row.cx), cy = tc::f2_pack(-row.cy, -row.cy);
  each([&](int g, const float (&x)[4], const float (&y)[4]) {
    float v[4];
#pragma unroll
    for (int i = 0; i < 4; i += 2) {
      const uint64_t xm = tc::f2_add(tc::f2_pack(x[i], x[i + 1]), mx);
      uint64_t f = tc::f2_fma(cx, xm, cc);
      if (kRef) f = tc::f2_fma(cy, tc::f2_add(tc::f2_pack(y[i], y[i + 1]), my), f);
      tc::f2_unpack(tc::f2_mul(f, exp_2(xm)), v[i], v[i + 1]);
    }
    const int j = group(g);
    store_4(xr + j, whole, A - j, v);
  });
  xr[act] = rounded<E>(slope<kRef>(row, xa, ya, true));
  return true;
}

template <typename E, bool kRef, bool kLegal, int kG>  // kG: groups of four actions in registers; 0: none
__global__ void __launch_bounds__(kTileRows, kG > 5 ? 4 : kTileCtas) tiles(const __grid_constant__ Loss l, int64_t n_tiles) {
  tc::after_previous();
  extern __shared__ __align__(16) unsigned char smem[];
  __shared__ double tmp[kTileRows / 32 * kSums];
  const int A = (int)l.A;
  const uint32_t inv = ((1u << 20) + A - 1) / A;  // i / A for i < 128 * 64: the error i (inv A - 2^20) / 2^20 A is below 1 / A
  const int bytes = (kTileRows * A * (int)sizeof(E) + 15) / 16 * 16;
  E *xs = reinterpret_cast<E*>(smem), *ys = reinterpret_cast<E*>(smem + bytes);
  uint8_t* ls = smem + (kRef ? 2 : 1) * bytes;
  const E *x = static_cast<const E*>(l.x), *y = static_cast<const E*>(l.y);
  E* d = static_cast<E*>(l.d);
  const bool dense_x = l.ldx == A && (uintptr_t)x % 16 == 0, dense_y = kRef && l.ldy == A && (uintptr_t)y % 16 == 0;
  const bool dense_d = l.ldd == A && (uintptr_t)d % 16 == 0, dense_l = (uintptr_t)l.legal % 16 == 0;
  Acc acc[kSums];
  const int r = threadIdx.x, begin = r % A;
  E *xr = xs + r * A, *yr = ys + r * A;
  const uint8_t* lr = ls + r * A;
  for (int64_t t = blockIdx.x; t < n_tiles; t += gridDim.x) {
    const int64_t r0 = t * kTileRows, m = r0 + r;
    const int rows = (int)min((int64_t)kTileRows, l.M - r0);
    const bool in = r < rows;
    tile_in(xs, x + r0 * l.ldx, l.ldx, rows, A, inv, dense_x);
    if (kRef) tile_in(ys, y + r0 * l.ldy, l.ldy, rows, A, inv, dense_y);
    if (kLegal) tile_in(ls, l.legal + r0 * A, (int64_t)A, rows, A, inv, dense_l);
    const int64_t act64 = in ? action_of(l, m) : -1;
    copies_done();
    __syncthreads();
    const int act = act64 >= 0 && act64 < A ? (int)act64 : -1;
    const bool on = act >= 0 && (!kLegal || lr[act]);
    bool done = false;
    if (on) done = row_by_fours<E, kRef, kLegal, kG>(l, m, A, act, xr, yr, lr, d != nullptr, acc);
    if (done) {
    } else if (on) {
      // (elements in turn from `begin`)
      auto each = [&](auto&& f) {
        int j = begin;
#pragma unroll 4
        for (int i = 0; i < A; ++i) {
          f(j);
          j = j + 1 == A ? 0 : j + 1;
        }
      };
      Sums s;
      each([&](int j) {
        if (kLegal && !lr[j]) return;
        s.mx = fmaxf(s.mx, f32(xr[j]));
        if (kRef) s.my = fmaxf(s.my, f32(yr[j]));
      });
      const float ex = s.mx == -kInf ? 0.f : s.mx, ey = s.my == -kInf ? 0.f : s.my;
      each([&](int j) {
        const bool ok = !kLegal || lr[j];
        const float xm = f32(xr[j]) - ex, e = ok ? exp_of(xm) : 0.f;
        s.s += e;
        s.u += e == 0.f ? 0.f : e * xm;
        if (kRef) {
          const float ym = f32(yr[j]) - ey;
          s.t += e == 0.f ? 0.f : e * (xm - ym);
          s.sy += ok ? exp_of(ym) : 0.f;
        }
      });
      s.my = ey;
      const Row row = finish<kRef>(l, m, true, f32(xr[act]), s, true, acc);
      if (d)
        each([&](int j) {
          const float g = row.on && (!kLegal || lr[j]) ? slope<kRef>(row, f32(xr[j]), kRef ? f32(yr[j]) : 0.f, j == act) : 0.f;
          xr[j] = rounded<E>(g);
        });
    } else if (in) {
      Sums none;
      finish<kRef>(l, m, false, 0.f, none, true, acc);
      if (d)
        for (int j = 0; j < A; ++j) xr[j] = rounded<E>(0.f);
    }
    __syncthreads();
    if (d) {
      E* out = d + r0 * l.ldd;
      const int n = rows * A;
      constexpr int kPer = 16 / (int)sizeof(E);
      if (dense_d) {
        for (int i = threadIdx.x; i < n / kPer; i += kTileRows) reinterpret_cast<uint4*>(out)[i] = reinterpret_cast<const uint4*>(xs)[i];
        for (int i = n / kPer * kPer + threadIdx.x; i < n; i += kTileRows) out[i] = xs[i];
      } else {
        for (int i = threadIdx.x; i < n; i += kTileRows) {
          const int k = (int)((uint32_t)i * inv >> 20);
          out[k * l.ldd + (i - k * A)] = xs[i];
        }
      }
      __syncthreads();
    }
  }
  totals(l, acc, tmp);
}

// ---- many actions: a warp or a CTA a row --------------------------------------------------
// V elements of 16 bytes as fp32.
__device__ __forceinline__ void values(const uint4& a, float (&v)[4]) {
  v[0] = __uint_as_float(a.x), v[1] = __uint_as_float(a.y), v[2] = __uint_as_float(a.z), v[3] = __uint_as_float(a.w);
}
__device__ __forceinline__ void values(const uint4& a, float (&v)[8]) {
  const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) v[2 * i] = __uint_as_float(w[i] << 16), v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
}
__device__ __forceinline__ uint4 packed(const float (&v)[4]) {
  return uint4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
}
__device__ __forceinline__ uint4 packed(const float (&v)[8]) {
  return uint4{tc::pack_bf16(v[0], v[1]), tc::pack_bf16(v[2], v[3]), tc::pack_bf16(v[4], v[5]), tc::pack_bf16(v[6], v[7])};
}
template <typename E, int V> __device__ __forceinline__ void store_v(E* p, const float (&v)[V], uint64_t policy) {
  const uint4 w = packed(v);
  asm volatile("st.global.L2::cache_hint.v4.u32 [%0], {%1, %2, %3, %4}, %5;" ::"l"(p), "r"(w.x), "r"(w.y), "r"(w.z), "r"(w.w), "l"(policy)
               : "memory");
}

// Greatest of V elements that were loaded as 16 bytes (not a number: ignored).
__device__ __forceinline__ float greatest(const uint4&, const float (&v)[4]) { return fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3])); }
__device__ __forceinline__ float greatest(const uint4& a, const float (&)[8]) {
  const __nv_bfloat162* p = reinterpret_cast<const __nv_bfloat162*>(&a);
  const __nv_bfloat162 h = __hmax2(__hmax2(p[0], p[1]), __hmax2(p[2], p[3]));
  return fmaxf(__low2float(h), __high2float(h));
}

// Least of V elements (not a number: ignored).
__device__ __forceinline__ float least(const uint4&, const float (&v)[4]) { return fminf(fminf(v[0], v[1]), fminf(v[2], v[3])); }
__device__ __forceinline__ float least(const uint4& a, const float (&)[8]) {
  const __nv_bfloat162* p = reinterpret_cast<const __nv_bfloat162*>(&a);
  const __nv_bfloat162 h = __hmin2(__hmin2(p[0], p[1]), __hmin2(p[2], p[3]));
  return fminf(__low2float(h), __high2float(h));
}
// Logits below kFar (-inf and the type's lowest value among them) become it; what is not a number stays so.
__device__ __forceinline__ void lift(uint4& a, const float (&)[4]) {
  uint32_t* w = reinterpret_cast<uint32_t*>(&a);
#pragma unroll
  for (int i = 0; i < 4; ++i) asm("max.NaN.f32 %0, %0, %1;" : "+r"(w[i]) : "r"(__float_as_uint(kFar)));
}
__device__ __forceinline__ void lift(uint4& a, const float (&)[8]) {
  uint32_t* w = reinterpret_cast<uint32_t*>(&a);
#pragma unroll
  for (int i = 0; i < 4; ++i) asm("max.NaN.bf16x2 %0, %0, %1;" : "+r"(w[i]) : "r"(kFarBf16));
}

// Puts kFar in the place of what is not legal.
template <int V, bool kRef>
__device__ __forceinline__ void hide(const uint8_t* legal, float (&x)[V], float (&y)[V]) {
#pragma unroll
  for (int i = 0; i < V; ++i)
    if (!legal[i]) x[i] = kFar, y[i] = kFar;
}

// Adds V elements, one at a time (`legal`: which of them; NULL: all).
template <int V, bool kRef>
__device__ __forceinline__ void add_each(Sums& s, const float (&x)[V], const float (&y)[V], const uint8_t* legal) {
#pragma unroll
  for (int i = 0; i < V; ++i) {
    if (legal && !legal[i]) continue;
    if (x[i] > s.mx || (kRef && y[i] > s.my)) move_to<kRef>(s, fmaxf(s.mx, x[i]), kRef ? fmaxf(s.my, y[i]) : 0.f);
    const float xm = x[i] - (s.mx == -kInf ? 0.f : s.mx), e = exp_of(xm);
    s.s += e;
    s.u += e == 0.f ? 0.f : e * xm;
    if (kRef) {
      const float ym = y[i] - (s.my == -kInf ? 0.f : s.my);
      s.t += e == 0.f ? 0.f : e * (xm - ym);
      s.sy += exp_of(ym);
    }
  }
}

// The sums of a thread, as pairs and in units of ln 2: with a = x log2 e - cx, b = y log2 e - cy (cx, cy: the maxima times
// log2 e, rounded), s = sum 2^a, u = sum 2^a a, v = sum 2^a b, sy = sum 2^b.  Rounding of cx and cy moves all a and b of a
// row alike and falls out of H, KL and the gradient.  Arithmetic in pairs for an element and its reference, and no element
// is looked at.  That is right where x and y are kFar or more: all a and b are finite then, and what stands at kFar adds 0
// as soon as a maximum lies above it.  x is lifted to that; a lower y, whose KL may be infinite, makes s NaN, as do +inf and
// what is not a number.  Until a maximum lies above kFar the sums hold what stands for nothing: `raise` takes it to 0, and
// `sums_of` leaves it out.
struct Pairs {
  uint64_t s = 0, u = 0, v = 0, sy = 0;
  float mx = kFar, my = kFar, low = 0.f;
};
__device__ __forceinline__ uint64_t both(float v) { return tc::f2_pack(v, v); }
__device__ __forceinline__ uint64_t exp2_of(uint64_t v) {
  float a, b;
  tc::f2_unpack(v, a, b);
  return tc::f2_pack(tc::ex2_approx(a), tc::ex2_approx(b));
}
template <bool kRef> __device__ __forceinline__ void raise(Pairs& p, float hx, float hy) {
  const float mx = fmaxf(p.mx, hx), my = fmaxf(p.my, hy);
  const float dx = p.mx * kLog2e - mx * kLog2e, dy = kRef ? p.my * kLog2e - my * kLog2e : 0.f;
  const uint64_t r = both(tc::ex2_approx(dx));
  p.u = tc::f2_mul(r, tc::f2_fma(p.s, both(dx), p.u));
  if (kRef) {
    p.v = tc::f2_mul(r, tc::f2_fma(p.s, both(dy), p.v));
    p.sy = tc::f2_mul(both(tc::ex2_approx(dy)), p.sy);
  }
  p.s = tc::f2_mul(r, p.s);
  p.mx = mx, p.my = my;
}
template <int V, bool kRef>
__device__ __forceinline__ void add_block(Pairs& p, uint4 xw, const uint4& yw, const uint8_t* legal) {
  float x[V], y[V];
  lift(xw, x);
  values(xw, x);
  if (kRef) values(yw, y);
  float hx, hy = 0.f;
  if (legal) {
    hide<V, kRef>(legal, x, y);
    hx = x[0], hy = y[0];
#pragma unroll
    for (int i = 1; i < V; ++i) hx = fmaxf(hx, x[i]), hy = fmaxf(hy, y[i]);
    if (kRef)
#pragma unroll
      for (int i = 0; i < V; ++i) p.low = fminf(p.low, y[i]);
  } else {
    hx = greatest(xw, x);
    if (kRef) hy = greatest(yw, y), p.low = fminf(p.low, least(yw, y));
  }
  if (hx > p.mx || (kRef && hy > p.my)) raise<kRef>(p, hx, hy);   // (rare after the first blocks)
  const uint64_t l2 = both(kLog2e), cx = both(-p.mx * kLog2e), cy = both(-p.my * kLog2e);
#pragma unroll
  for (int i = 0; i < V; i += 2) {
    const uint64_t a = tc::f2_fma(tc::f2_pack(x[i], x[i + 1]), l2, cx), e = exp2_of(a);
    p.s = tc::f2_add(p.s, e);
    p.u = tc::f2_fma(e, a, p.u);
    if (kRef) {
      const uint64_t b = tc::f2_fma(tc::f2_pack(y[i], y[i + 1]), l2, cy);
      p.v = tc::f2_fma(e, b, p.v);
      p.sy = tc::f2_add(p.sy, exp2_of(b));
    }
  }
}
// As sums about the maxima themselves.
template <bool kRef> __device__ __forceinline__ Sums sums_of(const Pairs& p) {
  Sums m;
  constexpr float kLn2 = 0.6931471805599453f;
  float a, b, v = 0.f;
  m.mx = p.mx, m.my = kRef ? p.my : -kInf;
  tc::f2_unpack(p.s, a, b), m.s = a + b;
  tc::f2_unpack(p.u, a, b), m.u = a + b;
  if (kRef) {
    tc::f2_unpack(p.v, a, b), v = a + b;
    tc::f2_unpack(p.sy, a, b), m.sy = a + b;
    if (p.low < kFar) m.s = kInf - kInf;
  }
  // x log2 e - mx log2 e is a less what cx was rounded by
  const float ox = fmaf(p.mx, kLog2e, -(p.mx * kLog2e)), oy = kRef ? fmaf(p.my, kLog2e, -(p.my * kLog2e)) : 0.f;
  const float rx = tc::ex2_approx(-ox);
  if (kRef) {
    m.t = rx * (m.u - v - m.s * (ox - oy)) * kLn2;
    m.sy = p.my > kFar ? m.sy * tc::ex2_approx(-oy) : 0.f * m.sy;
  }
  m.u = rx * (m.u - m.s * ox) * kLn2;
  m.s *= rx;
  if (!(p.mx > kFar)) m.mx = -kInf, m.s *= 0.f, m.u = 0.f, m.t = 0.f;
  return m;
}

// What becomes of a line in L2: one that is read again stays, another goes first.
__device__ __forceinline__ uint64_t goes_first() {
  uint64_t pol;
  asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(pol));
  return pol;
}
__device__ __forceinline__ uint4 load_16(const uint4* p, uint64_t policy) {
  uint4 v;
  asm volatile("ld.global.L2::cache_hint.v4.u32 {%0, %1, %2, %3}, [%4], %5;" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p), "l"(policy));
  return v;
}

// Adds a row's vectors [0, n) from `lane` on, `step` apart, as pairs, or (`far`) an element at a time.
template <typename E, bool kRef>
__device__ __forceinline__ Sums add_vectors(const uint4* xv, const uint4* yv, const uint8_t* legal, int n, int lane, int step, bool far) {
  const uint64_t stays = tc::l2_evict_last();
  constexpr int V = 16 / (int)sizeof(E);
  if (far) {
    Sums s;
    for (int v = lane; v < n; v += step) {
      float x[V], y[V];
      values(xv[v], x);
      if (kRef) values(yv[v], y);
      add_each<V, kRef>(s, x, y, legal ? legal + v * V : nullptr);
    }
    return s;
  }
  constexpr int kAhead = 2;     // vectors on their way at a time
  Pairs p;
  for (int v0 = lane; v0 < n; v0 += kAhead * step) {
    uint4 xw[kAhead], yw[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
      if (v0 + k * step < n) {
        xw[k] = load_16(xv + v0 + k * step, stays);
        if (kRef) yw[k] = load_16(yv + v0 + k * step, stays);
      }
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
      if (v0 + k * step < n) {
        add_block<V, kRef>(p, xw[k], yw[k], legal ? legal + (v0 + k * step) * V : nullptr);
      }
  }
  return sums_of<kRef>(p);
}
template <typename E, bool kRef> __device__ __forceinline__ void add_one(Sums& s, const E* x, const E* y, const uint8_t* legal, int j) {
  const float xv[1] = {f32(x[j])}, yv[1] = {kRef ? f32(y[j]) : 0.f};
  add_each<1, kRef>(s, xv, yv, legal ? legal + j : nullptr);
}
// The sums of a warp's lanes, for each of them.
template <bool kRef> __device__ __forceinline__ void join_warp(Sums& s) {
  float mx = s.mx, my = s.my;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    mx = fmaxf(mx, __shfl_xor_sync(~0u, mx, o));
    if (kRef) my = fmaxf(my, __shfl_xor_sync(~0u, my, o));
  }
  move_to<kRef>(s, mx, my);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    s.s += __shfl_xor_sync(~0u, s.s, o);
    s.u += __shfl_xor_sync(~0u, s.u, o);
    if (kRef) s.t += __shfl_xor_sync(~0u, s.t, o), s.sy += __shfl_xor_sync(~0u, s.sy, o);
  }
}
__device__ __forceinline__ void put(float* p, const Sums& t) { p[0] = t.mx, p[1] = t.s, p[2] = t.u, p[3] = t.t, p[4] = t.my, p[5] = t.sy; }
__device__ __forceinline__ Sums got(const float* p) { return Sums{p[0], p[1], p[2], p[3], p[4], p[5]}; }
// Whether the pairs' sums of a row that takes part say nothing of it: no number, or no logit, its own or the reference's,
// above kFar.
template <bool kRef> __device__ __forceinline__ bool lost(const Sums& s) {
  return !(fabsf(s.s) + fabsf(s.u) + fabsf(s.t) + fabsf(s.sy) < kInf) || !(s.mx > kFar) || (kRef && !(s.my > kFar));
}

// The gradient of a share of a row.  `act`: the action's place in it.
template <typename E, bool kRef>
__device__ __forceinline__ void grad_vectors(const Row& r, const uint4* xv, const uint4* yv, const uint8_t* legal, E* d, bool d_wide, int n,
                                             int act, int lane, int step, bool far) {
  constexpr int V = 16 / (int)sizeof(E);
  const uint64_t l2 = both(kLog2e), mx = both(-r.max_x), my = both(-r.max_y), cc = both(r.c), cx = both(r.cx), cy = both(-r.cy), first = goes_first();
  for (int v = lane; v < n; v += step) {
    float x[V], y[V], g[V];
    if (r.on) {
      uint4 xw = load_16(xv + v, first);
      if (!far) lift(xw, x);
      values(xw, x);
      if (kRef) values(load_16(yv + v, first), y);
      const int k = act - v * V;
      if (far) {
#pragma unroll
        for (int i = 0; i < V; ++i) g[i] = !legal || legal[v * V + i] ? slope<kRef>(r, x[i], kRef ? y[i] : 0.f, k == i) : 0.f;
      } else {
        if (legal) hide<V, kRef>(legal + v * V, x, y);
#pragma unroll
        for (int i = 0; i < V; i += 2) {
          const uint64_t xm = tc::f2_add(tc::f2_pack(x[i], x[i + 1]), mx);
          uint64_t f = tc::f2_fma(cx, xm, cc);
          if (kRef) f = tc::f2_fma(cy, tc::f2_add(tc::f2_pack(y[i], y[i + 1]), my), f);
          tc::f2_unpack(tc::f2_mul(f, exp2_of(tc::f2_mul(xm, l2))), g[i], g[i + 1]);
        }
        if ((uint32_t)k < V) {
#pragma unroll
          for (int i = 0; i < V; ++i)
            if (k == i) g[i] += r.at;
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) g[i] = 0.f;
    }
    if (d_wide) {
      store_v(d + v * V, g, first);
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) d[v * V + i] = rounded<E>(g[i]);
    }
  }
}
template <typename E, bool kRef>
__device__ __forceinline__ void grad_one(const Row& r, const E* x, const E* y, const uint8_t* legal, E* d, int act, int j) {
  d[j] = rounded<E>(r.on && (!legal || legal[j]) ? slope<kRef>(r, f32(x[j]), kRef ? f32(y[j]) : 0.f, j == act) : 0.f);
}

// A row in memory: elements before the first 16-byte boundary, then vectors where the reference's row is aligned alike.
template <typename E, bool kRef> struct Line {
  const E *x, *y;
  E* d;
  const uint8_t* legal;
  int head, vecs;
  bool d_wide;
  __device__ __forceinline__ Line(const Loss& l, int64_t m) {
    constexpr int V = 16 / (int)sizeof(E);
    const int A = (int)l.A;
    x = static_cast<const E*>(l.x) + m * l.ldx;
    y = kRef ? static_cast<const E*>(l.y) + m * l.ldy : x;
    d = l.d ? static_cast<E*>(l.d) + m * l.ldd : nullptr;
    legal = l.legal ? l.legal + m * A : nullptr;
    head = min(A, (int)((16 - (uintptr_t)x % 16) % 16 / sizeof(E)));
    vecs = (uintptr_t)(y + head) % 16 == 0 ? (A - head) / V : 0;
    d_wide = (uintptr_t)(d + head) % 16 == 0;
  }
  __device__ __forceinline__ const uint4* xv(int v) const { return reinterpret_cast<const uint4*>(x + head) + v; }
  __device__ __forceinline__ const uint4* yv(int v) const { return reinterpret_cast<const uint4*>(y + head) + v; }
  // the elements that are in no vector
  template <typename F> __device__ __forceinline__ void odd(int A, int lane, int step, F&& f) const {
    for (int j = lane; j < (vecs ? head : 0); j += step) f(j);
    for (int j = (vecs ? head + vecs * (16 / (int)sizeof(E)) : 0) + lane; j < A; j += step) f(j);
  }
};

// TPR threads (a warp, or the CTA) a row.
template <typename E, int TPR, int kThreads, bool kRef>
__global__ void __launch_bounds__(kThreads, 1024 / kThreads) rows(const __grid_constant__ Loss l) {
  tc::after_previous();
  constexpr int kGroups = kThreads / TPR, kParts = TPR / 32;
  __shared__ float red[TPR > 32 ? 2 * kParts * 6 : 1];  // (two sets: a row's is read while the next one's is written)
  __shared__ double tmp[kThreads / 32 * kSums];
  const int lane = threadIdx.x % TPR, A = (int)l.A;
  Acc acc[kSums];
  int turn = 0;
  for (int64_t m = (int64_t)blockIdx.x * kGroups + threadIdx.x / TPR; m < l.M; m += (int64_t)gridDim.x * kGroups, turn ^= 1) {
    const Line<E, kRef> row(l, m);
    const int64_t act64 = action_of(l, m);
    const int act = act64 >= 0 && act64 < A ? (int)act64 : -1;
    const bool on = act >= 0 && (!row.legal || row.legal[act]);
    const float xa = on ? f32(row.x[act]) : 0.f;
    const uint8_t* legal = row.legal ? row.legal + row.head : nullptr;
    Sums s;
    bool far = false;           // (an element at a time, where the pairs' sums gave no number)
    while (true) {
      s = Sums{};
      if (on) {
        s = add_vectors<E, kRef>(row.xv(0), row.yv(0), legal, row.vecs, lane, TPR, far);
        row.odd(A, lane, TPR, [&](int j) { add_one<E, kRef>(s, row.x, row.y, row.legal, j); });
      }
      join_warp<kRef>(s);
      __syncwarp();             // (the lanes have read the action's logit, which the gradient may replace)
      if constexpr (TPR > 32) {
        float* set = red + turn * kParts * 6;
        if ((lane & 31) == 0) put(set + lane / 32 * 6, s);
        __syncthreads();
        s = Sums{};
        for (int k = 0; k < kParts; ++k) join<kRef>(s, got(set + k * 6));
      }
      if (far || !on || !lost<kRef>(s)) break;    // (the same for all threads of the row)
      far = true, turn ^= 1;
    }
    const Row r = finish<kRef>(l, m, on, xa, s, lane == 0, acc);
    if (!row.d) continue;
    grad_vectors<E, kRef>(r, row.xv(0), row.yv(0), legal, row.d + row.head, row.d_wide, row.vecs, act - row.head, lane, TPR, far);
    row.odd(A, lane, TPR, [&](int j) { grad_one<E, kRef>(r, row.x, row.y, row.legal, row.d, act, j); });
  }
  totals(l, acc, tmp);
}

// Shared memory of a tile.
template <typename E> int tile_bytes(int A, bool ref, bool legal) {
  return (ref ? 2 : 1) * ((kTileRows * A * (int)sizeof(E) + 15) / 16 * 16) + (legal ? (kTileRows * A + 15) / 16 * 16 : 0);
}

template <typename E, bool kRef, bool kLegal, int kG>
aht_status launch_tiles(Shape sh, const Loss& l, int64_t n_tiles, cudaStream_t s) {
  sh.most = tile_bytes<E>(kG > 0 ? 4 * kG : kTileA, kRef, kLegal);
  return launch_op(tiles<E, kRef, kLegal, kG>, sh, s, l, n_tiles);
}
// Groups of four actions in registers, and CTAs an SM: times (us) of 40 M logits with a reference, fp32 / bf16.  8 actions: 2
// groups 168 / 160, 5 176 / 180.  20: 5 groups 113 / 104, 8 172 / 164; 6 CTAs 111 / 104, 4 135 / 131.  21: 8 groups 147 / 141, none
// 166 / 158; 4 CTAs 145 / 141, 6 182 / 180.  32: 8 groups 113 / 102, none 123 / 115.  64, half legal: tiles 131 / 111, a warp a row
// 612 / 717.
template <typename E, bool kRef, bool kLegal>
aht_status run_tiles(const Shape& sh, const Loss& l, int64_t n_tiles, cudaStream_t s) {
  if (l.A <= 8) return launch_tiles<E, kRef, kLegal, 2>(sh, l, n_tiles, s);
  if (l.A <= 20) return launch_tiles<E, kRef, kLegal, 5>(sh, l, n_tiles, s);
  if (l.A <= 32) return launch_tiles<E, kRef, kLegal, 8>(sh, l, n_tiles, s);
  return launch_tiles<E, kRef, kLegal, 0>(sh, l, n_tiles, s);
}

// Threads of a row of more than kTileA actions, by its bytes and the number of rows: a warp, whose sums are joined without a
// barrier, where there are enough of them, else a CTA.  32, 256 and 512 threads a row, with a reference (us): fp32 1024
// actions x 9728 rows 47, 109, 238, x 64 18, 14, 21; 2048 x 304 23, 21, 27, x 608 23, 27, 33, x 4864 49, 70, 139; 4096 x 1216 41,
// 39, 51, x 2432 53, 53, 86, x 9728 135, 160, 291; 8192 x 4864 152, 127, 193; 16384 x 64 96, 23, 25, x 4864 277, 223, 272; 32768 x
// 64 178, 37, 31, x 2432 354, 254, 236.  bf16 2048 x 4864 37, 66, 135; 8192 x 2432 59, 57, 96, x 4864 84, 100, 172; 32768 x 1216
// 170, 80, 94; 65536 x 64 211, 39, 35, x 1216 334, 141, 145.
int threads_of_row(int64_t A, int64_t M, int bytes) {
  const int64_t row = A * bytes;
  if (A <= 1024 || (row <= 8192 && M >= 608) || (row <= 16384 && M >= 2432)) return 32;
  return row <= 65536 ? 256 : 512;
}

template <typename E, bool kRef>
aht_status go(const Loss& l, cudaStream_t s) {
  int64_t ctas;
  aht_status e;
  if (l.A <= kTileA) {
    const int64_t n_tiles = (l.M + kTileRows - 1) / kTileRows;
    const int smem = tile_bytes<E>((int)l.A, kRef, l.legal != nullptr);
    ctas = std::min<int64_t>(n_tiles, 152 * std::max(1, std::min(l.A > 20 ? 4 : kTileCtas, 226 * 1024 / (smem + 2048))));
    const Shape sh{dim3((unsigned)ctas), dim3(kTileRows), smem};
    e = l.legal ? run_tiles<E, kRef, true>(sh, l, n_tiles, s) : run_tiles<E, kRef, false>(sh, l, n_tiles, s);
  } else if (const int threads = threads_of_row(l.A, l.M, (int)sizeof(E)); threads == 32) {
    ctas = std::min<int64_t>((l.M + 7) / 8, 152 * 4);
    e = launch_op(rows<E, 32, 256, kRef>, Shape{dim3((unsigned)ctas), dim3(256)}, s, l);
  } else if (threads == 256) {
    ctas = std::min<int64_t>(l.M, 152 * 4);
    e = launch_op(rows<E, 256, 256, kRef>, Shape{dim3((unsigned)ctas), dim3(256)}, s, l);
  } else {
    ctas = std::min<int64_t>(l.M, 152 * 2);
    e = launch_op(rows<E, 512, 512, kRef>, Shape{dim3((unsigned)ctas), dim3(512)}, s, l);
  }
  if (e != AHT_OK || ctas == 1) return e;
  return launch_op(sum_parts, Shape{dim3(1), dim3(32 * kSums * kSumWarps)}, s, l, (int)ctas);
}

}  // namespace

extern "C" {

int64_t aht_policy_loss_workspace(int64_t M, int64_t A) {
  return M < 1 || A < 1 ? 0 : (int64_t)kMaxCtas * kSums * (int64_t)sizeof(double);
}

aht_status aht_policy_loss(const aht_policy_loss_args* a, float* stats, float* logp, void* dlogits, int64_t ld_d,
                           void* workspace, int64_t workspace_bytes, void* cuda_stream) {
  if (!a) return set_last_error(AHT_EINVAL, "args is NULL");
  if (a->dtype != AHT_FP32 && a->dtype != AHT_BF16) return set_last_error(AHT_EINVAL, "dtype must be AHT_FP32 or AHT_BF16");
  if (a->action_bytes != 1 && a->action_bytes != 4 && a->action_bytes != 8)
    return set_last_error(AHT_EINVAL, "action_bytes must be 1, 4 or 8");
  if (a->M < 1 || a->A < 1 || a->A > AHT_POLICY_LOSS_MAX_A || a->M > (int64_t(1) << 40))
    return set_last_error(AHT_EINVAL, "sizes: 1 <= M <= 2^40, 1 <= A <= AHT_POLICY_LOSS_MAX_A");
  if (!a->logits || !a->actions || !a->old_logp || !a->advantages || !stats)
    return set_last_error(AHT_EINVAL, "logits, actions, old_logp, advantages or stats is NULL");
  if (a->ref_logits && a->ref_logp) return set_last_error(AHT_EINVAL, "ref_logits and ref_logp exclude one another");
  const int64_t most = int64_t(1) << 46;
  for (int64_t ld : {a->ld, a->ref_logits ? a->ld_ref : a->A, dlogits ? ld_d : a->A})
    if (ld < a->A || ld > most / a->M) return set_last_error(AHT_EINVAL, "rows: ld >= A and M * ld <= 2^46");
  if (!(a->clip_low >= 0.f && a->clip_high >= 0.f && a->kl_coef >= 0.f && a->ent_coef >= 0.f))
    return set_last_error(AHT_EINVAL, "clip_low, clip_high, kl_coef and ent_coef must be 0 or more");
  if (!workspace || workspace_bytes < aht_policy_loss_workspace(a->M, a->A))
    return set_last_error(AHT_EINVAL, "workspace is NULL or smaller than aht_policy_loss_workspace");
  if (!on_boundary(16, workspace)) return set_last_error(AHT_EINVAL, "workspace must be on a boundary of 16 bytes");
  if (!on_boundary(a->dtype == AHT_FP32 ? 4 : 2, a->logits, a->ref_logits, dlogits) || !on_boundary(a->action_bytes, a->actions) ||
      !on_boundary(4, a->old_logp, a->advantages, a->weight, a->ref_logp, stats, logp))
    return set_last_error(AHT_EINVAL, kMisalignedArray);
  Loss l{};
  l.M = a->M, l.A = a->A, l.x = a->logits, l.y = a->ref_logits, l.actions = a->actions, l.d = dlogits;
  l.ldx = a->ld, l.ldy = a->ld_ref, l.ldd = ld_d;
  l.old_logp = a->old_logp, l.adv = a->advantages, l.weight = a->weight, l.ref_logp = a->ref_logp, l.legal = a->legal;
  l.logp = logp, l.stats = stats, l.part = static_cast<double*>(workspace);
  l.lo = 1.f - a->clip_low, l.hi = 1.f + a->clip_high, l.kl = a->kl_coef, l.ent = a->ent_coef;
  l.w = (float)(1.0 / (double)a->M);
  l.action_bytes = a->action_bytes;
  const cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  if (a->dtype == AHT_FP32) return a->ref_logits ? go<float, true>(l, s) : go<float, false>(l, s);
  return a->ref_logits ? go<__nv_bfloat16, true>(l, s) : go<__nv_bfloat16, false>(l, s);
}

}  // extern "C"
