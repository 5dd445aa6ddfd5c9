// glr.cu -- the gated linear recurrence over a collected trajectory (include/aht.h states
// the model): forward over T steps, one serving step (T = 1), and the backward pass.
//
// A lane is one channel d of one env n; its T steps are a chain, lanes are independent.
// One thread runs one lane here; consecutive threads take consecutive channels, so a warp
// reads contiguous rows.  State, gates and sums are fp32 whatever the tensors' type; each
// output is rounded once.
//
// The backward pass needs the state before every step.  The forward pass leaves it as fp32
// checkpoints every kSeg = 8 steps (0.5 B per element; the rounded h would cost 2-4 B and
// carry bf16 rounding into every gradient), and the backward pass rebuilds the seven states
// between two checkpoints in registers.
#include <cuda_bf16.h>

#include "kernels.h"

namespace aht {
aht_status set_last_error(aht_status s, const char* msg);  // the message of aht_last_error
}  // namespace aht

using namespace aht;

namespace {

constexpr int kSeg = AHT_GLR_SEGMENT;  // steps between two checkpoints
constexpr float kGateScale = 8.0f;     // s = 8 softplus(lam)

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

template <typename E>
__device__ __forceinline__ float ld(const Seq& s, int64_t t, int64_t n, int64_t d) {
  const E* p = static_cast<const E*>(s.p) + t * s.st + n * s.sn + d;
  return (float)__ldg(p);
}
template <typename E>
__device__ __forceinline__ void st(const Seq& s, int64_t t, int64_t n, int64_t d, float v) {
  static_cast<E*>(s.p)[t * s.st + n * s.sn + d] = (E)v;
}

__device__ __forceinline__ float softplus_f(float x) { return fmaxf(x, 0.0f) + log1pf(expf(-fabsf(x))); }
__device__ __forceinline__ float sigmoid_f(float x) { return 1.0f / (1.0f + expf(-x)); }

// The gates of one element: q = s rho, a = exp(-q) = 1 + em, beta^2 = 1 - a^2 = -em (2 + em)
// (no cancellation as a -> 1).
struct Gates {
  float rho, iota, q, a, beta2;
};
__device__ __forceinline__ Gates gates(float s, float r, float i) {
  Gates g;
  g.rho = sigmoid_f(r);
  g.iota = sigmoid_f(i);
  g.q = s * g.rho;
  const float em = expm1f(-g.q);
  g.a = 1.0f + em;
  g.beta2 = -em * (2.0f + em);
  return g;
}

template <typename E>
__global__ void glr_fwd(const GlrDev a, const float* h0, const Seq h, float* h_last, float* ckpt) {
  const int64_t lane = (int64_t)blockIdx.x * blockDim.x + threadIdx.x, lanes = a.N * a.D;
  if (lane >= lanes) return;
  const int64_t n = lane / a.D, d = lane - n * a.D;
  const float s = kGateScale * softplus_f(a.lam[d]);
  const int64_t len = a.lengths ? max((int64_t)0, min(a.T, (int64_t)a.lengths[n])) : a.T;
  float y = h0 ? h0[lane] : 0.0f;
  for (int64_t t = 0; t < a.T; ++t) {
    if (ckpt && t % kSeg == 0) ckpt[(t / kSeg) * lanes + lane] = y;
    if (t < len) {
      const Gates g = gates(s, ld<E>(a.r, t, n, d), ld<E>(a.i, t, n, d));
      const float b = sqrtf(g.beta2) * g.iota * ld<E>(a.x, t, n, d);
      y = a.reset && a.reset[t * a.N + n] ? b : fmaf(g.a, y, b);
    }
    if (h.p) st<E>(h, t, n, d, t < len ? y : 0.0f);
  }
  if (h_last) h_last[lane] = y;
}

struct GlrGrad {
  const float* ckpt;
  Seq dh;
  const float* dh_last;
  Seq dx, dr, di;
  float* dh0;
  float* part;  // [N][D] sums of w over the steps of a lane
};

template <typename E>
__global__ void glr_bwd(const GlrDev a, const GlrGrad b) {
  const int64_t lane = (int64_t)blockIdx.x * blockDim.x + threadIdx.x, lanes = a.N * a.D;
  if (lane >= lanes) return;
  const int64_t n = lane / a.D, d = lane - n * a.D;
  const float s = kGateScale * softplus_f(a.lam[d]);
  const int64_t len = a.lengths ? max((int64_t)0, min(a.T, (int64_t)a.lengths[n])) : a.T;
  float p = b.dh_last ? b.dh_last[lane] : 0.0f;  // gradient of the state a step leaves
  float sum = 0.0f, comp = 0.0f;
  for (int64_t seg = (a.T + kSeg - 1) / kSeg - 1; seg >= 0; --seg) {
    float before[kSeg];
    float y = b.ckpt[seg * lanes + lane];
    const int64_t t0 = seg * kSeg;
#pragma unroll
    for (int k = 0; k < kSeg; ++k) {
      const int64_t t = t0 + k;
      before[k] = 0.0f;
      if (t < len) {
        const bool rs = a.reset && a.reset[t * a.N + n];
        before[k] = rs ? 0.0f : y;
        const Gates g = gates(s, ld<E>(a.r, t, n, d), ld<E>(a.i, t, n, d));
        const float in = sqrtf(g.beta2) * g.iota * ld<E>(a.x, t, n, d);
        y = rs ? in : fmaf(g.a, y, in);
      }
    }
    float part = 0.0f;
#pragma unroll
    for (int k = kSeg - 1; k >= 0; --k) {
      const int64_t t = t0 + k;
      if (t >= a.T) continue;
      float dx = 0.0f, dr = 0.0f, di = 0.0f;
      if (t < len) {
        const bool rs = a.reset && a.reset[t * a.N + n];
        const float x = ld<E>(a.x, t, n, d);
        const Gates g = gates(s, ld<E>(a.r, t, n, d), ld<E>(a.i, t, n, d));
        const float beta = sqrtf(g.beta2);
        const float G = (b.dh.p ? ld<E>(b.dh, t, n, d) : 0.0f) + p;
        dx = G * beta * g.iota;
        di = dx * x * (1.0f - g.iota);
        // w = q a dL/da; q / beta -> 0 with q (beta^2 ~ 2 q)
        const float qb = g.beta2 > 0.0f ? g.q / beta : 0.0f;
        const float w = g.a * G * (g.q * before[k] - qb * g.a * g.iota * x);
        dr = -(1.0f - g.rho) * w;
        part += w;
        p = rs ? 0.0f : g.a * G;
      }
      st<E>(b.dx, t, n, d, dx);
      st<E>(b.dr, t, n, d, dr);
      st<E>(b.di, t, n, d, di);
    }
    const float yk = part - comp, sk = sum + yk;  // compensated over the segments
    comp = (sk - sum) - yk;
    sum = sk;
  }
  if (b.part) b.part[lane] = sum;
  if (b.dh0) b.dh0[lane] = p;
}

// dlam[d] = -(sum over rows of part[row][d]) sigmoid(lam) / softplus(lam), rows in a fixed
// order: 32 row-threads per channel, then a tree.  The ratio tends to 1 as lam -> -inf.
__global__ void glr_dlam(const float* __restrict__ part, int64_t rows, int32_t D, const float* __restrict__ lam,
                         float* __restrict__ dlam) {
  __shared__ float sh[32][33];
  const int d = blockIdx.x * 32 + threadIdx.x;
  float sum = 0.0f, comp = 0.0f;
  if (d < D)
    for (int64_t r = threadIdx.y; r < rows; r += 32) {
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
    const float l = lam[d], sp = softplus_f(l);
    dlam[d] = -sh[0][threadIdx.x] * (sp > 0.0f ? sigmoid_f(l) / sp : 1.0f);
  }
}

aht_status check(const aht_glr_args* a) {
  if (!a) return set_last_error(AHT_EINVAL, "args is NULL");
  if (a->dtype != AHT_FP32 && a->dtype != AHT_BF16)
    return set_last_error(AHT_EINVAL, "dtype must be AHT_FP32 or AHT_BF16");
  if (a->T < 0 || a->N < 1 || a->D < 1 || a->D > AHT_GLR_MAX_D)
    return set_last_error(AHT_EINVAL, "sizes: T >= 0, N >= 1, 1 <= D <= AHT_GLR_MAX_D");
  if (a->N > (int64_t(1) << 37) / a->D || (a->T > 0 && a->N > (int64_t(1) << 46) / a->D / a->T))
    return set_last_error(AHT_EINVAL, "N * D must be at most 2^37 and T * N * D at most 2^46");
  if (!a->lam) return set_last_error(AHT_EINVAL, "lam is NULL");
  if (a->T > 0 && (!a->x.data || !a->r.data || !a->i.data)) return set_last_error(AHT_EINVAL, "NULL input sequence");
  return AHT_OK;
}

Seq seq(const aht_seq& s) { return Seq{s.data, s.st, s.sn}; }
GlrDev dev(const aht_glr_args* a) {
  return GlrDev{a->D, a->T, a->N, seq(a->x), seq(a->r), seq(a->i), a->lam, a->reset, a->lengths};
}

aht_status launched() {
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? AHT_OK : set_last_error(AHT_ECUDA, cudaGetErrorString(e));
}

constexpr int kBlock = 128;
unsigned blocks_of(const aht_glr_args* a) { return (unsigned)((a->N * a->D + kBlock - 1) / kBlock); }

}  // namespace

extern "C" {

int64_t aht_glr_ckpt_elems(int64_t T, int64_t N, int32_t D) {
  return T < 0 || N < 0 || D < 0 ? 0 : (T + kSeg - 1) / kSeg * N * D;
}

int64_t aht_glr_workspace(int64_t T, int64_t N, int32_t D) {
  return T < 0 || N < 0 || D < 0 ? 0 : N * D * (int64_t)sizeof(float);
}

aht_status aht_glr_forward(const aht_glr_args* a, const float* h0, const aht_seq* h, float* h_last, float* ckpt,
                           void* cuda_stream) {
  if (aht_status e = check(a)) return e;
  const Seq out = h ? seq(*h) : Seq{nullptr, 0, 0};
  if (!out.p && !h_last) return set_last_error(AHT_EINVAL, "neither h nor h_last is asked for");
  const cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  if (a->dtype == AHT_FP32)
    glr_fwd<float><<<blocks_of(a), kBlock, 0, s>>>(dev(a), h0, out, h_last, ckpt);
  else
    glr_fwd<__nv_bfloat16><<<blocks_of(a), kBlock, 0, s>>>(dev(a), h0, out, h_last, ckpt);
  return launched();
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
  const GlrGrad g{ckpt,    dh ? seq(*dh) : none, dh_last, dx ? seq(*dx) : none, dr ? seq(*dr) : none,
                  di ? seq(*di) : none, dh0, dlam ? static_cast<float*>(workspace) : nullptr};
  const cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  if (a->dtype == AHT_FP32)
    glr_bwd<float><<<blocks_of(a), kBlock, 0, s>>>(dev(a), g);
  else
    glr_bwd<__nv_bfloat16><<<blocks_of(a), kBlock, 0, s>>>(dev(a), g);
  if (aht_status e = launched()) return e;
  if (!dlam) return AHT_OK;
  glr_dlam<<<(a->D + 31) / 32, dim3(32, 32), 0, s>>>(g.part, a->N, a->D, a->lam, dlam);
  return launched();
}

}  // extern "C"
