// group_norm.cu -- group norm with an activation over channels-last data, forward and backward
// (include/aht.h states it).
//
// An instance is a group of one sample: L positions of cg neighbouring channels, taken as vectors of V
// channels (16 bytes where rows allow).  A thread keeps to one vector of channels and steps through the
// positions, so that weights, and the gradients' sums over positions and samples, stay in registers.
//   small: up to 8 vectors a thread of up to 32 threads.  The instance stays in registers: each element
//     is read once and written once, the sums are shuffles.  Groups that are neighbours in memory are
//     neighbours in a warp.
//   large: a CTA, or a cluster of up to 8 (16 for few instances), an instance, which stays in shared memory
//     between the passes (it is read again, from L2, where it does not fit).
// The variance is the mean square about the mean, formed after the mean.  Backward, with xh the normalised
// x, z = weight xh + bias, e = dy act'(z) weight, over the m elements of the instance:
//   dx = rstd (e - (sum e + xh sum e xh) / m).
// What bounds both is memory: 2 values an element forward, 3 backward.
// dweight and dbias: a thread's sums go through its CTA into one row a CTA, and `fold` adds the rows, all
// in a fixed order.
#include <cooperative_groups.h>
#include <cuda_bf16.h>

#include <algorithm>
#include <atomic>

#include "op_launch.cuh"

using namespace aht;
namespace cg = cooperative_groups;

namespace {

struct Seq {                    // element (n, l, c) at p[n * sn + l * st + c]
  void* p;
  int64_t st, sn;
};

struct Norm {
  int64_t N, L;
  int32_t C, G, cg, act;
  float eps;
  Seq x, y, dy, dx;
  const float *weight, *bias;
  const int32_t* lengths;
  float *mean, *rstd;           // [N][G] written forward (or NULL), read backward
  float* part;                  // backward: [rows][2][C] sums of dweight and dbias, or NULL
};

// ---- V values at a time, as pairs where V is even --------------------------------------------
template <int V, typename F, typename G>
__device__ __forceinline__ void each_pair(F&& pair, G&& one) {
  if constexpr (V % 2 == 0) {
#pragma unroll
    for (int i = 0; i < V; i += 2) pair(i);
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) one(i);
  }
}
template <int V> __device__ __forceinline__ uint64_t at2(const float (&a)[V], int i) { return tc::f2_pack(a[i], a[i + 1]); }
template <int V> __device__ __forceinline__ void to2(float (&a)[V], int i, uint64_t v) { tc::f2_unpack(v, a[i], a[i + 1]); }
__device__ __forceinline__ uint64_t both(float v) { return tc::f2_pack(v, v); }
// d = a b + c;  d = a - b;  d = a b
template <int V> __device__ __forceinline__ void fma_v(float (&d)[V], const float (&a)[V], const float (&b)[V], const float (&c)[V]) {
  each_pair<V>([&](int i) { to2(d, i, tc::f2_fma(at2(a, i), at2(b, i), at2(c, i))); }, [&](int i) { d[i] = a[i] * b[i] + c[i]; });
}
template <int V> __device__ __forceinline__ void sub_v(float (&d)[V], const float (&a)[V], const float (&b)[V]) {
  each_pair<V>([&](int i) { to2(d, i, tc::f2_sub(at2(a, i), at2(b, i))); }, [&](int i) { d[i] = a[i] - b[i]; });
}
template <int V> __device__ __forceinline__ void mul_v(float (&d)[V], const float (&a)[V], const float (&b)[V]) {
  each_pair<V>([&](int i) { to2(d, i, tc::f2_mul(at2(a, i), at2(b, i))); }, [&](int i) { d[i] = a[i] * b[i]; });
}
template <int V> __device__ __forceinline__ void mul_v(float (&d)[V], const float (&a)[V], float b) {
  each_pair<V>([&](int i) { to2(d, i, tc::f2_mul(at2(a, i), both(b))); }, [&](int i) { d[i] = a[i] * b; });
}
template <int V> __device__ __forceinline__ void add_v(float (&d)[V], const float (&a)[V]) {
  each_pair<V>([&](int i) { to2(d, i, tc::f2_add(at2(d, i), at2(a, i))); }, [&](int i) { d[i] += a[i]; });
}
template <int V> __device__ __forceinline__ void set_v(float (&d)[V], float a) {
#pragma unroll
  for (int i = 0; i < V; ++i) d[i] = a;
}
template <int V> __device__ __forceinline__ float total(const float (&a)[V]) {
  if constexpr (V % 2 == 0) {
    uint64_t s = at2(a, 0);
#pragma unroll
    for (int i = 2; i < V; i += 2) s = tc::f2_add(s, at2(a, i));
    float x, y;
    tc::f2_unpack(s, x, y);
    return x + y;
  }
  return a[0];
}

// ---- activations ----------------------------------------------------------------------------
__device__ __forceinline__ float sigmoid(float z) { return tc::rcp_approx(1.f + tc::ex2_approx(-1.4426950408889634f * z)); }

// Phi(z) and e^(-z^2 / 2).  erf by Abramowitz and Stegun 7.1.26, off by at most 1.5e-7 (a library erfc takes four times
// the instructions: gradients of 4096 x 49 x 64 were bound by them).
struct Normal {
  float cdf, e;
};
__device__ __forceinline__ Normal normal(float z) {
  const float x = fabsf(z) * 0.7071067811865476f, t = tc::rcp_approx(1.f + 0.3275911f * x);
  const float e = tc::ex2_approx(-1.4426950408889634f * x * x);
  const float q = t * (0.254829592f + t * (-0.284496736f + t * (1.421413741f + t * (-1.453152027f + t * 1.061405429f)))) * e;
  return {z < 0.f ? 0.5f * q : 1.f - 0.5f * q, e};   // (erfc(x) = q)
}

// The same of two values, as pairs.
struct Normal2 {
  uint64_t cdf, e;
};
__device__ __forceinline__ uint64_t ex2_pair(uint64_t v) {
  float p, q;
  tc::f2_unpack(v, p, q);
  return tc::f2_pack(tc::ex2_approx(p), tc::ex2_approx(q));
}
__device__ __forceinline__ uint64_t rcp_pair(uint64_t v) {
  float p, q;
  tc::f2_unpack(v, p, q);
  return tc::f2_pack(tc::rcp_approx(p), tc::rcp_approx(q));
}
__device__ __forceinline__ Normal2 normal2(uint64_t z) {
  float a, b, lo0, lo1, hi0, hi1;
  tc::f2_unpack(z, a, b);
  const uint64_t x = tc::f2_pack(fabsf(a) * 0.7071067811865476f, fabsf(b) * 0.7071067811865476f);
  const uint64_t t = rcp_pair(tc::f2_fma(x, both(0.3275911f), both(1.f))), e = ex2_pair(tc::f2_mul(tc::f2_mul(x, both(-1.4426950408889634f)), x));
  uint64_t q = tc::f2_fma(t, both(1.061405429f), both(-1.453152027f));
  q = tc::f2_fma(t, q, both(1.421413741f));
  q = tc::f2_fma(t, q, both(-0.284496736f));
  q = tc::f2_mul(tc::f2_mul(tc::f2_fma(t, q, both(0.254829592f)), t), e);
  tc::f2_unpack(tc::f2_mul(q, both(0.5f)), lo0, lo1);
  tc::f2_unpack(tc::f2_fma(q, both(-0.5f), both(1.f)), hi0, hi1);
  return {tc::f2_pack(a < 0.f ? lo0 : hi0, b < 0.f ? lo1 : hi1), e};
}
__device__ __forceinline__ uint64_t sigmoid2(uint64_t z) {
  return rcp_pair(tc::f2_add(ex2_pair(tc::f2_mul(z, both(-1.4426950408889634f))), both(1.f)));
}

// act(z) of V values; one branch, the same for every thread.
template <int V> __device__ __forceinline__ void activate(int act, float (&z)[V]) {
  if (act == AHT_ACT_SILU) {
    each_pair<V>(
        [&](int i) {
          float p, q;
          const uint64_t x = at2(z, i);
          tc::f2_unpack(tc::f2_mul(x, both(-1.4426950408889634f)), p, q);
          tc::f2_unpack(tc::f2_add(tc::f2_pack(tc::ex2_approx(p), tc::ex2_approx(q)), both(1.f)), p, q);
          to2(z, i, tc::f2_mul(x, tc::f2_pack(tc::rcp_approx(p), tc::rcp_approx(q))));
        },
        [&](int i) { z[i] *= sigmoid(z[i]); });
  } else if (act == AHT_ACT_GELU) {
#pragma unroll
    for (int i = 0; i < V; ++i) z[i] *= normal(z[i]).cdf;
  } else if (act == AHT_ACT_RELU) {
#pragma unroll
    for (int i = 0; i < V; ++i) z[i] = z[i] > 0.f ? z[i] : z[i] == z[i] ? 0.f : z[i];
  }
}
// d[i] <- d[i] act'(z[i]).
template <int V> __device__ __forceinline__ void times_slope(int act, float (&d)[V], const float (&z)[V]) {
  if (act == AHT_ACT_SILU) {
    each_pair<V>(
        [&](int i) {
          const uint64_t x = at2(z, i), s = sigmoid2(x);
          to2(d, i, tc::f2_mul(at2(d, i), tc::f2_mul(s, tc::f2_fma(x, tc::f2_sub(both(1.f), s), both(1.f)))));
        },
        [&](int i) {
          const float s = sigmoid(z[i]);
          d[i] *= s * (1.f + z[i] * (1.f - s));
        });
  } else if (act == AHT_ACT_GELU) {
    each_pair<V>(
        [&](int i) {
          const uint64_t x = at2(z, i);
          const Normal2 n = normal2(x);
          to2(d, i, tc::f2_mul(at2(d, i), tc::f2_fma(tc::f2_mul(x, both(0.3989422804014327f)), n.e, n.cdf)));
        },
        [&](int i) {
          const Normal n = normal(z[i]);
          d[i] *= n.cdf + z[i] * 0.3989422804014327f * n.e;
        });
  } else if (act == AHT_ACT_RELU) {
#pragma unroll
    for (int i = 0; i < V; ++i) d[i] = z[i] > 0.f ? d[i] : z[i] == z[i] ? 0.f : z[i];
  }
}

// ---- V neighbouring channels ----------------------------------------------------------------
template <typename E, int V> struct Raw;
template <> struct Raw<float, 4> { using T = uint4; };
template <> struct Raw<float, 1> { using T = uint32_t; };
template <> struct Raw<__nv_bfloat16, 8> { using T = uint4; };
template <> struct Raw<__nv_bfloat16, 2> { using T = uint32_t; };
template <> struct Raw<__nv_bfloat16, 1> { using T = uint16_t; };

template <typename E, int V> struct Vec {
  typename Raw<E, V>::T w;
  __device__ __forceinline__ void load(const void* p) { w = *static_cast<const typename Raw<E, V>::T*>(p); }
  __device__ __forceinline__ void store(void* p) const { *static_cast<typename Raw<E, V>::T*>(p) = w; }
  __device__ __forceinline__ void get(float (&f)[V]) const {
    if constexpr (sizeof(E) == 4) {
      const float* v = reinterpret_cast<const float*>(&w);
#pragma unroll
      for (int i = 0; i < V; ++i) f[i] = v[i];
    } else if constexpr (V == 1) {
      f[0] = __uint_as_float((uint32_t)w << 16);
    } else {
      const uint32_t* v = reinterpret_cast<const uint32_t*>(&w);
#pragma unroll
      for (int i = 0; i < V / 2; ++i) f[2 * i] = __uint_as_float(v[i] << 16), f[2 * i + 1] = __uint_as_float(v[i] & 0xFFFF0000u);
    }
  }
  __device__ __forceinline__ void set(const float (&f)[V]) {
    if constexpr (sizeof(E) == 4) {
      float* v = reinterpret_cast<float*>(&w);
#pragma unroll
      for (int i = 0; i < V; ++i) v[i] = f[i];
    } else if constexpr (V == 1) {
      w = (uint16_t)(tc::pack_bf16(f[0], 0.f) & 0xFFFFu);
    } else {
      uint32_t* v = reinterpret_cast<uint32_t*>(&w);
#pragma unroll
      for (int i = 0; i < V / 2; ++i) v[i] = tc::pack_bf16(f[2 * i], f[2 * i + 1]);
    }
  }
};

__device__ __forceinline__ int64_t positions(const Norm& a, int64_t n) {
  return a.lengths ? min((int64_t)max(a.lengths[n], 0), a.L) : a.L;
}
template <typename E, int V> __device__ __forceinline__ E* row(const Seq& s, int64_t n, int64_t l, int c) {
  return static_cast<E*>(s.p) + n * s.sn + l * s.st + c;
}

// Weight and bias of V channels from c on (those outside [c0, c1): 0).
template <int V> struct Weights {
  float w[V], b[V];
  __device__ __forceinline__ Weights(const Norm& a, int c, int c0, int c1) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const bool on = c + i >= c0 && c + i < c1;
      w[i] = !on ? 0.f : a.weight ? a.weight[c + i] : 1.f;
      b[i] = on && a.bias ? a.bias[c + i] : 0.f;
    }
  }
};

// ---- small instances ------------------------------------------------------------------------
// Where a thread of `small` is: tpi (a power of two, up to 32) threads an instance, of which `used` (a multiple
// of the vectors of a position) work; the CTA's instances of one step are `gs` groups of `sp` samples.
struct Place {
  int tpi, vpc, used, gs, sp;
};
__device__ __forceinline__ float sum_of(float v, int tpi) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
    if (tpi > o) v += __shfl_xor_sync(~0u, v, o);
  return v;
}

constexpr int kSmallThreads = 256;

template <typename E, int V, int kVecs>
__global__ void __launch_bounds__(kSmallThreads) small_fwd(const __grid_constant__ Norm a, const __grid_constant__ Place p) {
  tc::after_previous();
  const int lane = threadIdx.x % p.tpi, inst = threadIdx.x / p.tpi, gi = inst % p.gs, si = inst / p.gs;
  const int g = blockIdx.y * p.gs + gi;
  const bool mine = si < p.sp && g < a.G && lane < p.used;
  const int c = g * a.cg + lane % p.vpc * V, l0 = lane / p.vpc, dl = p.used / p.vpc, L = (int)a.L;
  const Weights<V> k(a, c, 0, mine ? a.C : 0);
  const int64_t first = (int64_t)blockIdx.x * p.sp + si, step = (int64_t)gridDim.x * p.sp;
  const E* px = row<E, V>(a.x, first, l0, c);
  E* py = row<E, V>(a.y, first, l0, c);
  const int64_t xl = dl * a.x.st, yl = dl * a.y.st, xn = step * a.x.sn, yn = step * a.y.sn;
  const float whole = 1.f / ((float)L * (float)a.cg);
  Vec<E, V> x[kVecs], next[kVecs];
  int len = 0, next_len = 0;
  auto fetch = [&](int64_t n) {  // (the next sample's, while this one is worked on)
    next_len = mine && n < a.N ? (a.lengths ? (int)positions(a, n) : L) : 0;
#pragma unroll
    for (int i = 0; i < kVecs; ++i)
      if (l0 + i * dl < next_len) next[i].load(px + i * xl);
    px += xn;
  };
  fetch(first);
  for (int64_t n = first; n - si < a.N; n += step, py += yn) {
    const bool on = mine && n < a.N;
    len = next_len;
#pragma unroll
    for (int i = 0; i < kVecs; ++i) x[i] = next[i];
    fetch(n + step);
    // (as fp32 from here on, where that fits into registers)
    constexpr bool kOnce = kVecs * V <= 16;
    float s[V], q[V], f[V], m[V], xf[kOnce ? kVecs : 1][V];
    set_v(s, 0.f);
#pragma unroll
    for (int i = 0; i < kVecs; ++i)
      if (l0 + i * dl < len) {
        x[i].get(kOnce ? xf[kOnce ? i : 0] : f);
        add_v(s, kOnce ? xf[kOnce ? i : 0] : f);
      }
    const float im = len == L ? whole : len > 0 ? 1.f / ((float)len * (float)a.cg) : 0.f;
    const float mean = sum_of(total(s), p.tpi) * im;
    set_v(m, mean);
    set_v(q, 0.f);
#pragma unroll
    for (int i = 0; i < kVecs; ++i)
      if (l0 + i * dl < len) {
        if constexpr (kOnce) {
          sub_v(xf[i], xf[i], m);
          fma_v(q, xf[i], xf[i], q);
        } else {
          x[i].get(f);
          sub_v(f, f, m);
          fma_v(q, f, f, q);
        }
      }
    const float var = sum_of(total(q), p.tpi) * im, rstd = len > 0 ? rsqrtf(var + a.eps) : 0.f;
    if (!on) continue;
    if (lane == 0 && a.mean) a.mean[n * a.G + g] = mean, a.rstd[n * a.G + g] = rstd;
    float rw[V];
    mul_v(rw, k.w, rstd);
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
      const int l = l0 + i * dl;
      if (l >= L) break;
      if (l < len) {
        if constexpr (!kOnce) {
          x[i].get(f);
          sub_v(f, f, m);
          fma_v(f, f, rw, k.b);
        } else {
          fma_v(f, xf[i], rw, k.b);
        }
        activate(a.act, f);
      } else {
        set_v(f, 0.f);
      }
      Vec<E, V> y;
      y.set(f);
      y.store(py + i * yl);
    }
  }
}

template <typename E, int V, int kVecs>
__global__ void __launch_bounds__(kSmallThreads) small_bwd(const __grid_constant__ Norm a, const __grid_constant__ Place p) {
  tc::after_previous();
  __shared__ float tmp[kSmallThreads * 2 * V];
  const int lane = threadIdx.x % p.tpi, inst = threadIdx.x / p.tpi, gi = inst % p.gs, si = inst / p.gs;
  const int g = blockIdx.y * p.gs + gi;
  const bool mine = si < p.sp && g < a.G && lane < p.used;
  const int c = g * a.cg + lane % p.vpc * V, l0 = lane / p.vpc, dl = p.used / p.vpc, L = (int)a.L;
  const Weights<V> k(a, c, 0, mine ? a.C : 0);
  const int64_t first = (int64_t)blockIdx.x * p.sp + si, step = (int64_t)gridDim.x * p.sp;
  const E *px = row<E, V>(a.x, first, l0, c), *pd = row<E, V>(a.dy, first, l0, c);
  E* po = row<E, V>(a.dx, first, l0, c);
  const int64_t xl = dl * a.x.st, xn = step * a.x.sn, gl = dl * a.dy.st, gn = step * a.dy.sn, ol = dl * a.dx.st, on_ = step * a.dx.sn;
  const float whole = 1.f / ((float)L * (float)a.cg);
  float dw[V], db[V];
  set_v(dw, 0.f);
  set_v(db, 0.f);
  // (where they fit into registers, the next sample's rows are on their way while this one is worked on)
  constexpr bool kAhead = kVecs <= 2;
  Vec<E, V> x[kVecs], dy[kVecs], nx[kAhead ? kVecs : 1], nd[kAhead ? kVecs : 1];
  float mean = 0.f, rstd = 0.f, next_mean = 0.f, next_rstd = 0.f;
  int len = 0, next_len = 0;
  auto fetch = [&](int64_t n, Vec<E, V>* to_x, Vec<E, V>* to_d) {
    next_len = mine && n < a.N ? (a.lengths ? (int)positions(a, n) : L) : 0;
#pragma unroll
    for (int i = 0; i < kVecs; ++i)
      if (l0 + i * dl < next_len) to_x[i].load(px + i * xl), to_d[i].load(pd + i * gl);
    next_mean = next_len > 0 ? a.mean[n * a.G + g] : 0.f, next_rstd = next_len > 0 ? a.rstd[n * a.G + g] : 0.f;
    px += xn, pd += gn;
  };
  if (kAhead) fetch(first, nx, nd);
  for (int64_t n = first; n - si < a.N; n += step, po += on_) {
    const bool on = mine && n < a.N;
    if constexpr (kAhead) {
#pragma unroll
      for (int i = 0; i < kVecs; ++i) x[i] = nx[i], dy[i] = nd[i];
    } else {
      fetch(n, x, dy);
    }
    len = next_len, mean = next_mean, rstd = next_rstd;
    if (kAhead) fetch(n + step, nx, nd);
    const float im = len == L ? whole : len > 0 ? 1.f / ((float)len * (float)a.cg) : 0.f;
    float s1[V], s2[V], m[V], f[V], e[kVecs][V];
    set_v(s1, 0.f);
    set_v(s2, 0.f);
    set_v(m, mean);
#pragma unroll
    for (int i = 0; i < kVecs; ++i)
      if (l0 + i * dl < len) {
        float z[V];
        x[i].get(f);
        dy[i].get(e[i]);
        sub_v(f, f, m);
        mul_v(f, f, rstd);
        fma_v(z, f, k.w, k.b);
        times_slope(a.act, e[i], z);
        add_v(db, e[i]);
        fma_v(dw, e[i], f, dw);
        mul_v(e[i], e[i], k.w);
        add_v(s1, e[i]);
        fma_v(s2, e[i], f, s2);
      }
    const float t1 = sum_of(total(s1), p.tpi) * im * rstd, t2 = sum_of(total(s2), p.tpi) * im * rstd * rstd;
    if (!on) continue;
    float c1[V], c2[V], r[V];
    set_v(c1, -t1);
    set_v(c2, -t2);
    set_v(r, rstd);
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
      const int l = l0 + i * dl;
      if (l >= L) break;
      if (l < len) {            // rstd e - rstd t1 - (x - mean) rstd^2 t2
        x[i].get(f);
        sub_v(f, f, m);
        fma_v(e[i], e[i], r, c1);
        fma_v(f, f, c2, e[i]);
      } else {
        set_v(f, 0.f);
      }
      Vec<E, V> o;
      o.set(f);
      o.store(po + i * ol);
    }
  }
  if (!a.part) return;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    tmp[threadIdx.x * 2 * V + i] = dw[i];
    tmp[threadIdx.x * 2 * V + V + i] = db[i];
  }
  __syncthreads();
  // channel vector v of group gi: threads (si gs + gi) tpi + v + r vpc
  for (int i = threadIdx.x; i < p.gs * p.vpc * V; i += kSmallThreads) {
    const int v = i / V, j = i % V, gg = v / p.vpc, vv = v % p.vpc, group = blockIdx.y * p.gs + gg;
    if (group >= a.G) continue;
    float w = 0.f, b = 0.f;
    for (int s = 0; s < p.sp; ++s)
      for (int r = vv; r < p.used; r += p.vpc) {
        const float* t = tmp + ((s * p.gs + gg) * p.tpi + r) * 2 * V + j;
        w += t[0];
        b += t[V];
      }
    float* out = a.part + (int64_t)blockIdx.x * 2 * a.C + group * a.cg + vv * V + j;
    out[0] = w;
    out[a.C] = b;
  }
}

// ---- large instances ------------------------------------------------------------------------
// Threads of a CTA (kT): kFew where there are so few instances that each gets whole SMs, else kMany.
constexpr int kMany = 256, kFew = 768;

// Sum of two values over the CTA and its cluster, for every thread.
template <int kT> struct Reduce {
  float cta[kT / 32][2];
  float mine[2][2];             // by turn: this CTA's sums, which the cluster reads
};
template <int kT> __device__ __forceinline__ float2 all_sum(Reduce<kT>& r, float a, float b, int cl, int turn) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) a += __shfl_xor_sync(~0u, a, o), b += __shfl_xor_sync(~0u, b, o);
  __syncthreads();              // (the sums before this one have been read)
  if ((threadIdx.x & 31) == 0) r.cta[threadIdx.x >> 5][0] = a, r.cta[threadIdx.x >> 5][1] = b;
  __syncthreads();
  a = b = 0.f;
  for (int k = 0; k < kT / 32; ++k) a += r.cta[k][0], b += r.cta[k][1];
  if (cl == 1) return {a, b};
  cg::cluster_group c = cg::this_cluster();
  if (threadIdx.x == 0) r.mine[turn][0] = a, r.mine[turn][1] = b;
  c.sync();
  a = b = 0.f;
  for (int k = 0; k < cl; ++k) {
    const float* o = c.map_shared_rank(&r.mine[turn][0], k);
    a += o[0], b += o[1];
  }
  return {a, b};
}

// How an instance's positions lie in a cluster.  A group that does not begin or end on a vector shares its first or
// last one with its neighbours, whose channels are taken as 0 and not written.  `hold`: a CTA's part stays in shared
// memory between the passes, thread by thread.
struct Large {
  int vpc, cl, hold;            // vectors of a position, at most; CTAs
  int64_t part;                 // positions of a CTA
};

// A thread's share of an instance: one vector of channels of every `lanes`-th position, or (many channels) more vectors of
// every position.
template <typename E, int V, int kT> struct Share {
  int c0, c1, vecs, lanes, lane, v;
  bool keeps;                   // to one vector
  static constexpr int kWords = (V * (int)sizeof(E) + 3) / 4;
  uint32_t mask[kWords];        // the group's channels of that vector
  __device__ __forceinline__ Share(const Norm& a, int g) {
    c0 = g * a.cg, c1 = c0 + a.cg;
    const int v0 = c0 / V;
    vecs = (c1 + V - 1) / V - v0;
    keeps = vecs <= kT;
    lanes = keeps ? kT / vecs : 1;
    lane = keeps ? (int)threadIdx.x / vecs : 0;
    v = keeps ? (int)threadIdx.x % vecs : (int)threadIdx.x;
    if (keeps && lane >= lanes) lane = 1 << 30;   // (idle)
    masks(channel(v), mask);
  }
  __device__ __forceinline__ int channel(int vec) const { return c0 / V * V + vec * V; }
  // f(position, vector, its number) for this thread's of [lo, end)
  template <int kAtOnce, typename F> __device__ __forceinline__ void each(int64_t lo, int64_t end, F&& f) const {
    int i = 0;
    if (keeps) {
#pragma unroll kAtOnce
      for (int64_t l = lo + lane; l < end; l += lanes, ++i) f(l, v, i);
    } else {
      for (int64_t l = lo; l < end; ++l)
        for (int u = v; u < vecs; u += kT, ++i) f(l, u, i);
    }
  }
  __device__ __forceinline__ bool in(int c) const { return c >= c0 && c < c1; }
  __device__ __forceinline__ void masks(int c, uint32_t (&m)[kWords]) const {
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
      if constexpr (sizeof(E) == 4) m[i] = in(c + i) ? ~0u : 0u;
      else m[i] = (in(c + 2 * i) ? 0xFFFFu : 0u) | (in(c + 2 * i + 1) ? 0xFFFF0000u : 0u);
    }
  }
  // Neighbours' channels of a vector become 0, whatever they hold.
  __device__ __forceinline__ void cut(int c, Vec<E, V>& x) const {
    if constexpr (V > 1) {
      uint32_t* w = reinterpret_cast<uint32_t*>(&x.w);
      if (keeps) {
#pragma unroll
        for (int i = 0; i < kWords; ++i) w[i] &= mask[i];
      } else if (c < c0 || c + V > c1) {
        uint32_t m[kWords];
        masks(c, m);
#pragma unroll
        for (int i = 0; i < kWords; ++i) w[i] &= m[i];
      }
    }
  }
  __device__ __forceinline__ void store(E* p, int c, const float (&f)[V]) const {
    if (c < c0 || c + V > c1) {
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (c + i >= c0 && c + i < c1) {
          if constexpr (sizeof(E) == 4) p[i] = f[i];
          else p[i] = __float2bfloat16_rn(f[i]);
        }
    } else {
      Vec<E, V> y;
      y.set(f);
      y.store(p);
    }
  }
};

template <typename E, int V, int kT>
__global__ void __launch_bounds__(kT, kMany * 3 / kT) large_fwd(const __grid_constant__ Norm a, const __grid_constant__ Large p) {
  tc::after_previous();
  extern __shared__ __align__(16) unsigned char smem[];
  __shared__ Reduce<kT> red;
  using R = typename Raw<E, V>::T;
  R* held = reinterpret_cast<R*>(smem) + threadIdx.x;
  const int g = blockIdx.y, rank = blockIdx.x % p.cl;
  const Share<E, V, kT> own(a, g);
  const Weights<V> kept(a, own.channel(own.v), own.c0, own.keeps ? own.c1 : own.c0);
  for (int64_t n = blockIdx.x / p.cl; n < a.N; n += gridDim.x / p.cl) {
    const int64_t len = positions(a, n), lo = rank * p.part, hi = min(a.L, lo + p.part), stop = min(len, hi);
    auto get = [&](int64_t l, int vec, int i, float (&f)[V]) {
      Vec<E, V> x;
      if (p.hold) {
        x.w = held[i * kT];
      } else {
        x.load(row<E, V>(a.x, n, l, own.channel(vec)));
        own.cut(own.channel(vec), x);
      }
      x.get(f);
    };
    float s[V], q[V];
    set_v(s, 0.f);
    set_v(q, 0.f);
    own.template each<4>(lo, stop, [&](int64_t l, int vec, int i) {
      Vec<E, V> x;
      x.load(row<E, V>(a.x, n, l, own.channel(vec)));
      own.cut(own.channel(vec), x);
      if (p.hold) held[i * kT] = x.w;
      float f[V];
      x.get(f);
      add_v(s, f);
    });
    const float im = len > 0 ? 1.f / ((float)len * (float)a.cg) : 0.f;
    const float mean = all_sum(red, total(s), 0.f, p.cl, 0).x * im;
    float mean_v[V];            // (of neighbours' channels 0)
#pragma unroll
    for (int i = 0; i < V; ++i) mean_v[i] = own.in(own.channel(own.v) + i) ? mean : 0.f;
    own.template each<4>(lo, stop, [&](int64_t l, int vec, int i) {
      float f[V], m[V];
      get(l, vec, i, f);
#pragma unroll
      for (int z = 0; z < V; ++z) m[z] = own.keeps ? mean_v[z] : own.in(own.channel(vec) + z) ? mean : 0.f;
      sub_v(f, f, m);
      fma_v(q, f, f, q);
    });
    const float var = all_sum(red, total(q), 0.f, p.cl, 1).x * im, rstd = len > 0 ? rsqrtf(var + a.eps) : 0.f;
    if (threadIdx.x == 0 && rank == 0 && a.mean) a.mean[n * a.G + g] = mean, a.rstd[n * a.G + g] = rstd;
    own.template each<4>(lo, hi, [&](int64_t l, int vec, int i) {
      float f[V];
      const int c = own.channel(vec);
      if (l < len) {
        float m[V], rw[V];
        const Weights<V> k = own.keeps ? kept : Weights<V>(a, c, own.c0, own.c1);
        get(l, vec, i, f);
        set_v(m, mean);
        sub_v(f, f, m);
        mul_v(rw, k.w, rstd);
        fma_v(f, f, rw, k.b);
        activate(a.act, f);
      } else {
        set_v(f, 0.f);
      }
      own.store(row<E, V>(a.y, n, l, c), c, f);
    });
  }
  if (p.cl > 1) cg::this_cluster().sync();  // (the others have read this CTA's sums)
}

template <typename E, int V, int kT>
__global__ void __launch_bounds__(kT, kMany * 3 / kT) large_bwd(const __grid_constant__ Norm a, const __grid_constant__ Large p) {
  tc::after_previous();
  extern __shared__ __align__(16) unsigned char smem[];
  __shared__ Reduce<kT> red;
  __shared__ float tmp[kT * V];
  using R = typename Raw<E, V>::T;
  R* held = reinterpret_cast<R*>(smem) + threadIdx.x;
  const int g = blockIdx.y, rank = blockIdx.x % p.cl;
  const Share<E, V, kT> own(a, g);
  const Weights<V> kept(a, own.channel(own.v), own.c0, own.keeps ? own.c1 : own.c0);
  constexpr int kAtOnce = 2;    // positions (their loads are in flight together)
  float dw[V], db[V];
  set_v(dw, 0.f);
  set_v(db, 0.f);
  int turn = 0;
  for (int64_t n = blockIdx.x / p.cl; n < a.N; n += gridDim.x / p.cl, turn ^= 1) {
    const int64_t len = positions(a, n), lo = rank * p.part, hi = min(a.L, lo + p.part), stop = min(len, hi);
    const float mean = a.mean[n * a.G + g], rstd = a.rstd[n * a.G + g];
    // xh, dz and the weights of a vector (neighbours' channels: xh is of no use, dz is 0)
    auto form = [&](const Vec<E, V>& x, const Vec<E, V>& dy, int c, float (&xh)[V], float (&dz)[V], float (&w)[V]) {
      const Weights<V> k = own.keeps ? kept : Weights<V>(a, c, own.c0, own.c1);
      float z[V], m[V];
      x.get(xh);
      dy.get(dz);
      set_v(m, mean);
      sub_v(xh, xh, m);
      mul_v(xh, xh, rstd);
      fma_v(z, xh, k.w, k.b);
      times_slope(a.act, dz, z);
#pragma unroll
      for (int i = 0; i < V; ++i) w[i] = k.w[i];
    };
    // sums of dz and dz xh by channel; the weights come in behind the loop where a thread keeps to one vector
    float d1[V], d2[V];
    set_v(d1, 0.f);
    set_v(d2, 0.f);
    own.template each<kAtOnce>(lo, stop, [&](int64_t l, int vec, int i) {
      Vec<E, V> x, dy;
      const int c = own.channel(vec);
      x.load(row<E, V>(a.x, n, l, c));
      dy.load(row<E, V>(a.dy, n, l, c));
      own.cut(c, x), own.cut(c, dy);
      if (p.hold) held[2 * i * kT] = x.w, held[(2 * i + 1) * kT] = dy.w;
      float xh[V], e[V], w[V];
      form(x, dy, c, xh, e, w);
      if (!own.keeps) mul_v(e, e, w);
      add_v(d1, e);
      fma_v(d2, e, xh, d2);
    });
    if (own.keeps) {
      add_v(db, d1);
      add_v(dw, d2);
      mul_v(d1, d1, kept.w);
      mul_v(d2, d2, kept.w);
    }
    const float im = len > 0 ? 1.f / ((float)len * (float)a.cg) : 0.f;
    const float2 sums = all_sum(red, total(d1), total(d2), p.cl, turn);
    const float t1 = -sums.x * im, t2 = -sums.y * im;
    own.template each<kAtOnce>(lo, hi, [&](int64_t l, int vec, int i) {
      float f[V];
      const int c = own.channel(vec);
      if (l < len) {
        Vec<E, V> x, dy;
        if (p.hold) {
          x.w = held[2 * i * kT], dy.w = held[(2 * i + 1) * kT];
        } else {
          x.load(row<E, V>(a.x, n, l, c));
          dy.load(row<E, V>(a.dy, n, l, c));
          own.cut(c, x), own.cut(c, dy);
        }
        float e[V], c1[V], c2[V], w[V];
        form(x, dy, c, f, e, w);
        set_v(c1, t1);
        set_v(c2, t2);
        fma_v(e, e, w, c1);
        fma_v(f, f, c2, e);
        mul_v(f, f, rstd);
      } else {
        set_v(f, 0.f);
      }
      own.store(row<E, V>(a.dx, n, l, c), c, f);
    });
  }
  if (a.part && own.keeps) {
    for (int half = 0; half < 2; ++half) {
      __syncthreads();
#pragma unroll
      for (int i = 0; i < V; ++i) tmp[threadIdx.x * V + i] = half ? db[i] : dw[i];
      __syncthreads();
      for (int i = threadIdx.x; i < own.vecs * V; i += kT) {
        const int c = own.channel(0) + i;
        if (c < own.c0 || c >= own.c1) continue;
        float v = 0.f;
        for (int r = 0; r < own.lanes; ++r) v += tmp[r * own.vecs * V + i];
        a.part[((int64_t)blockIdx.x * 2 + half) * a.C + c] = v;
      }
    }
  }
  if (p.cl > 1) cg::this_cluster().sync();  // (the others have read this CTA's sums)
}

// dweight and dbias of groups whose positions have more vectors than a CTA has threads: a CTA 32 channels of a
// share of the rows, a row of parts a share.
template <typename E>
__global__ void __launch_bounds__(256) columns(const __grid_constant__ Norm a) {
  tc::after_previous();
  __shared__ float tmp[2][8][32];
  const int lane = threadIdx.x & 31, r = threadIdx.x >> 5, c = blockIdx.y * 32 + lane;
  float dw = 0.f, db = 0.f;
  if (c < a.C) {
    const int g = c / a.cg;
    const Weights<1> k(a, c, 0, a.C);
    const int64_t rows = a.N * a.L;
    for (int64_t i = (int64_t)blockIdx.x * 8 + r; i < rows; i += (int64_t)gridDim.x * 8) {
      const int64_t n = i / a.L, l = i - n * a.L;
      if (l >= positions(a, n)) continue;
      Vec<E, 1> x, dy;
      x.load(row<E, 1>(a.x, n, l, c));
      dy.load(row<E, 1>(a.dy, n, l, c));
      float f[1], d[1];
      x.get(f);
      dy.get(d);
      const float xh = (f[0] - a.mean[n * a.G + g]) * a.rstd[n * a.G + g], z[1] = {xh * k.w[0] + k.b[0]};
      times_slope(a.act, d, z);
      db += d[0];
      dw += d[0] * xh;
    }
  }
  tmp[0][r][lane] = dw, tmp[1][r][lane] = db;
  __syncthreads();
  if (r < 2 && c < a.C) {
    float v = 0.f;
    for (int i = 0; i < 8; ++i) v += tmp[r][i][lane];
    a.part[((int64_t)blockIdx.x * 2 + r) * a.C + c] = v;
  }
}

// Adds the rows of parts: a CTA 8 channels of dweight (y = 0) or dbias (1), 128 threads a channel.
__global__ void __launch_bounds__(1024) fold(const float* part, int rows, int C, float* dweight, float* dbias) {
  tc::after_previous();
  __shared__ float tmp[128][9];
  const int j = threadIdx.x & 7, r = threadIdx.x >> 3, c = blockIdx.x * 8 + j, half = blockIdx.y;
  float* out = half ? dbias : dweight;
  if (!out) return;
  float v = 0.f;
  if (c < C)
#pragma unroll 4
    for (int i = r; i < rows; i += 128) v += part[((int64_t)i * 2 + half) * C + c];
  tmp[r][j] = v;
  for (int o = 64; o > 0; o >>= 1) {
    __syncthreads();
    if (r < o) tmp[r][j] += tmp[r + o][j];
  }
  if (r == 0 && c < C) out[c] = tmp[0][j];
}

// ---- host ---------------------------------------------------------------------------------
constexpr int kCtas = 152 * 4;             // of a pass that keeps sums, and rows of parts
constexpr int kMaxCluster = 8, kWideCluster = 16;   // CTAs of a cluster: of any, of few instances (beyond what every device runs)
constexpr int kHold = 72 * 1024, kHoldFew = 192 * 1024;   // shared memory for an instance's part (else L2 holds it), by threads

// Whether the current device places a cluster of kWideCluster CTAs of kFew threads with all the shared memory that they may
// hold (no GPC of a part of a GPU need have sixteen SMs).  The kernel with the most static memory answers for all; the
// answer is asked for once a device.
std::atomic<int> g_most_ctas{0};           // aht_debug_group_norm_cluster; 0: ask
bool runs_wide() {
  if (const int most = g_most_ctas) return most >= kWideCluster;
  constexpr int kDevices = 64;
  static std::atomic<signed char> known[kDevices];   // 1: it does, -1: it does not
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return false;
  if (dev < kDevices && known[dev]) return known[dev] > 0;
  const auto kernel = large_bwd<__nv_bfloat16, 8, kFew>;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim = {(unsigned)kWideCluster, 1, 1};
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(kWideCluster), cfg.blockDim = dim3(kFew), cfg.dynamicSmemBytes = kHoldFew;
  cfg.attrs = &attr, cfg.numAttrs = 1;
  int n = 0;
  const bool wide = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kHoldFew) == cudaSuccess &&
                    cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) == cudaSuccess &&
                    cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) == cudaSuccess && n > 0;
  if (!wide) cudaGetLastError();             // (nothing of the question stays behind)
  if (dev < kDevices) known[dev] = wide ? 1 : -1;
  return wide;
}

// How a call's instances are laid on threads.
struct How {
  bool small;
  int V, vpc, tpi, vecs;                    // small: threads and vectors a thread
  int cl, threads;                          // large: CTAs and their threads
};

// V: the widest vectors that the rows allow.
How how(const aht_group_norm_args* a, int V) {
  How h{};
  const int cg = a->C / a->G;
  h.V = cg % V == 0 ? V : 1;
  h.vpc = cg / h.V;
  const int64_t vectors = a->L * h.vpc;
  if (h.vpc <= 32 && vectors <= 32 * 8) {
    h.tpi = 1;
    while (h.tpi < 32 && h.tpi < vectors) h.tpi *= 2;
    const int dl = h.tpi / h.vpc;
    const int64_t vecs = (a->L + dl - 1) / dl;
    if (dl > 0 && vecs <= 8) {
      h.small = true;
      h.vecs = vecs <= 1 ? 1 : vecs <= 2 ? 2 : vecs <= 4 ? 4 : 8;
      return h;
    }
  }
  // Groups that straddle vectors are taken as whole vectors of the row where it has them.
  h.V = a->C % V == 0 ? V : 1;
  h.vpc = (cg + h.V - 1) / h.V + (cg % h.V != 0);
  // Enough CTAs for the machine, each with some positions.
  const int64_t insts = a->N * a->G, vecs = a->L * h.vpc;
  h.cl = 1;
  while (h.cl < kMaxCluster && insts * h.cl < 304 && a->L >= 64 * h.cl) h.cl *= 2;
  h.threads = kMany;
  if (h.cl == kMaxCluster) {
    // Few instances get whole SMs, and clusters of 16 where there are no more of them than run at a time (so, and with 8
    // CTAs of 256 threads, us: 4000000 x 16 bf16 896, 4768; 10000 x 64 bf16 21, 44; 19 x 60000 x 32 bf16 115, 152; but
    // 16 x 4000 x 64 bf16 30, 21).  Where the device has no room for such a cluster: 8 CTAs of 256 threads.
    if (insts <= 8 && vecs >= 4 * kMaxCluster * kFew) {
      if (runs_wide()) h.threads = kFew, h.cl = kWideCluster;
    } else if (insts > 8 && insts * kMaxCluster <= 152 && vecs >= 16 * kMaxCluster * kFew) h.threads = kFew;
  }
  return h;
}

bool aligned(const Seq& s, int esz, int V, int64_t N, int64_t L) {
  const uintptr_t bytes = (uintptr_t)esz * V;
  return !s.p || ((uintptr_t)s.p % bytes == 0 && (L <= 1 || s.st % V == 0) && (N <= 1 || s.sn % V == 0));
}

template <typename E, int V, int kVecs>
aht_status run_small(const Norm& a, const Place& p, dim3 grid, bool back, cudaStream_t s) {
  const Shape sh{grid, dim3(kSmallThreads)};
  return back ? launch_op(small_bwd<E, V, kVecs>, sh, s, a, p) : launch_op(small_fwd<E, V, kVecs>, sh, s, a, p);
}

template <typename E, int V>
aht_status run(const Norm& a, const How& h, bool back, int* rows, cudaStream_t s) {
  if (h.small) {
    Place p;
    p.tpi = h.tpi, p.vpc = h.vpc, p.used = h.tpi / h.vpc * h.vpc;
    const int insts = kSmallThreads / h.tpi;
    p.gs = std::min(insts, a.G);
    p.sp = insts / p.gs;
    const int gb = (a.G + p.gs - 1) / p.gs;
    const int64_t most = back ? std::max(1, kCtas / gb) : std::max(1, 152 * 4 / gb);
    const dim3 grid((unsigned)std::min<int64_t>((a.N + p.sp - 1) / p.sp, most), (unsigned)gb);
    *rows = (int)grid.x;
    return h.vecs == 1   ? run_small<E, V, 1>(a, p, grid, back, s)
           : h.vecs == 2 ? run_small<E, V, 2>(a, p, grid, back, s)
           : h.vecs == 4 ? run_small<E, V, 4>(a, p, grid, back, s)
                         : run_small<E, V, 8>(a, p, grid, back, s);
  }
  Large p;
  p.vpc = h.vpc;
  p.cl = h.cl;
  p.part = (a.L + h.cl - 1) / h.cl;
  const int64_t t = h.threads;
  const int64_t slots = h.vpc <= t ? (p.part + t / h.vpc - 1) / (t / h.vpc) : p.part * ((h.vpc + t - 1) / t);
  const int64_t bytes = slots * t * (int)sizeof(typename Raw<E, V>::T) * (back ? 2 : 1);
  const int most = t == kFew ? kHoldFew : kHold;
  p.hold = bytes <= most;
  const int64_t samples = back ? std::max(1, kCtas / (a.G * h.cl)) : 65536;
  const dim3 grid((unsigned)(std::min<int64_t>(a.N, samples) * h.cl), (unsigned)a.G);
  *rows = (int)grid.x;
  const Shape sh{grid, dim3((unsigned)t), p.hold ? (int)bytes : 0, h.cl, most};
  if (t == kFew) return back ? launch_op(large_bwd<E, V, kFew>, sh, s, a, p) : launch_op(large_fwd<E, V, kFew>, sh, s, a, p);
  return back ? launch_op(large_bwd<E, V, kMany>, sh, s, a, p) : launch_op(large_fwd<E, V, kMany>, sh, s, a, p);
}

// The widest vectors that every sequence's rows allow.
int width(const aht_group_norm_args* a, const Norm& d) {
  const int esz = a->dtype == AHT_FP32 ? 4 : 2;
  for (int V : {16 / esz, esz == 2 ? 2 : 1}) {
    bool ok = true;
    for (const Seq& q : {d.x, d.y, d.dy, d.dx}) ok = ok && aligned(q, esz, V, a->N, a->L);
    if (ok) return V;
  }
  return 1;
}

aht_status pass(const aht_group_norm_args* a, const Norm& d, bool back, int* rows, const How& h, cudaStream_t s) {
  if (a->dtype == AHT_FP32) return h.V == 4 ? run<float, 4>(d, h, back, rows, s) : run<float, 1>(d, h, back, rows, s);
  return h.V == 8   ? run<__nv_bfloat16, 8>(d, h, back, rows, s)
         : h.V == 2 ? run<__nv_bfloat16, 2>(d, h, back, rows, s)
                    : run<__nv_bfloat16, 1>(d, h, back, rows, s);
}

aht_status check(const aht_group_norm_args* a) {
  if (!a) return set_last_error(AHT_EINVAL, "args is NULL");
  if (a->dtype != AHT_FP32 && a->dtype != AHT_BF16) return set_last_error(AHT_EINVAL, "dtype must be AHT_FP32 or AHT_BF16");
  if (a->act < AHT_ACT_NONE || a->act > AHT_ACT_GELU) return set_last_error(AHT_EINVAL, "act must be one of AHT_ACT_*");
  if (a->C < 1 || a->C > AHT_GROUP_NORM_MAX_C || a->G < 1 || a->C % a->G)
    return set_last_error(AHT_EINVAL, "channels: C in 1..AHT_GROUP_NORM_MAX_C, a multiple of G");
  if (a->N < 1 || a->L < 1 || a->N > (1 << 30) || a->L > (1 << 30) || a->N > (int64_t(1) << 46) / a->C / a->L)
    return set_last_error(AHT_EINVAL, "sizes: N and L in 1..2^30, N * L * C at most 2^46");
  if (!(a->eps > 0.f)) return set_last_error(AHT_EINVAL, "eps must be above 0");
  if (!a->x.data) return set_last_error(AHT_EINVAL, "x is NULL");
  if (!on_boundary(a->dtype == AHT_FP32 ? 4 : 2, a->x.data) || !on_boundary(4, a->weight, a->bias, a->lengths))
    return set_last_error(AHT_EINVAL, kMisalignedArray);
  return AHT_OK;
}

Seq seq(const aht_seq& s) { return Seq{s.data, s.st, s.sn}; }
Norm norm_of(const aht_group_norm_args* a) {
  Norm d{};
  d.N = a->N, d.L = a->L, d.C = a->C, d.G = a->G, d.cg = a->C / a->G, d.act = a->act, d.eps = a->eps;
  d.x = seq(a->x), d.weight = a->weight, d.bias = a->bias, d.lengths = a->lengths;
  return d;
}

}  // namespace

extern "C" {

aht_status aht_group_norm_forward(const aht_group_norm_args* a, const aht_seq* y, float* mean, float* rstd, void* cuda_stream) {
  if (aht_status e = check(a)) return e;
  if (!y || !y->data) return set_last_error(AHT_EINVAL, "y is NULL");
  if (!mean != !rstd) return set_last_error(AHT_EINVAL, "mean and rstd come together");
  if (!on_boundary(a->dtype == AHT_FP32 ? 4 : 2, y->data) || !on_boundary(4, mean, rstd))
    return set_last_error(AHT_EINVAL, kMisalignedArray);
  Norm d = norm_of(a);
  d.y = seq(*y), d.mean = mean, d.rstd = rstd;
  int rows;
  return pass(a, d, false, &rows, how(a, width(a, d)), static_cast<cudaStream_t>(cuda_stream));
}

int64_t aht_group_norm_workspace(int64_t N, int64_t L, int32_t C, int32_t G, int32_t dtype) {
  (void)dtype;
  if (N < 1 || L < 1 || C < 1 || G < 1 || C > AHT_GROUP_NORM_MAX_C || C % G) return 0;
  return (int64_t)kCtas * 2 * C * (int64_t)sizeof(float);
}

aht_status aht_group_norm_backward(const aht_group_norm_args* a, const float* mean, const float* rstd, const aht_seq* dy,
                                   const aht_seq* dx, float* dweight, float* dbias, void* workspace, int64_t workspace_bytes,
                                   void* cuda_stream) {
  if (aht_status e = check(a)) return e;
  if (!mean || !rstd || !dy || !dy->data || !dx || !dx->data) return set_last_error(AHT_EINVAL, "mean, rstd, dy or dx is NULL");
  const bool sums = dweight || dbias;
  if (sums && (!workspace || workspace_bytes < aht_group_norm_workspace(a->N, a->L, a->C, a->G, a->dtype)))
    return set_last_error(AHT_EINVAL, "workspace is NULL or smaller than aht_group_norm_workspace");
  if (sums && !on_boundary(16, workspace)) return set_last_error(AHT_EINVAL, "workspace must be on a boundary of 16 bytes");
  if (!on_boundary(a->dtype == AHT_FP32 ? 4 : 2, dy->data, dx->data) || !on_boundary(4, mean, rstd, dweight, dbias))
    return set_last_error(AHT_EINVAL, kMisalignedArray);
  Norm d = norm_of(a);
  d.dy = seq(*dy), d.dx = seq(*dx);
  d.mean = const_cast<float*>(mean), d.rstd = const_cast<float*>(rstd);
  d.part = sums ? static_cast<float*>(workspace) : nullptr;
  const cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  const How h = how(a, width(a, d));
  int rows = 0;
  const bool apart = sums && !h.small && h.vpc > h.threads;
  if (apart) {                  // (before dx, which may replace dy)
    rows = (int)std::min<int64_t>((a->N * a->L + 7) / 8, 64);
    const dim3 grid((unsigned)rows, (unsigned)((a->C + 31) / 32));
    if (aht_status e = a->dtype == AHT_FP32 ? launch_op(columns<float>, Shape{grid, dim3(256)}, s, d)
                                                  : launch_op(columns<__nv_bfloat16>, Shape{grid, dim3(256)}, s, d))
      return e;
    if (aht_status e = launch_op(fold, Shape{dim3((unsigned)((a->C + 7) / 8), 2), dim3(1024)}, s, (const float*)d.part, rows, a->C,
                                 dweight, dbias))
      return e;
    d.part = nullptr;
  }
  if (aht_status e = pass(a, d, true, &rows, h, s)) return e;
  if (!sums || apart) return AHT_OK;
  return launch_op(fold, Shape{dim3((unsigned)((a->C + 7) / 8), 2), dim3(1024)}, s, (const float*)d.part, rows, a->C, dweight, dbias);
}

aht_status aht_debug_group_norm_cluster(int32_t most) {
  if (most != 0 && most != kMaxCluster && most != kWideCluster) return set_last_error(AHT_EINVAL, "most must be 0, 8 or 16");
  g_most_ctas = most;
  return AHT_OK;
}

}  // extern "C"
