// Group norm with an activation over channels-last features, for K workers
// with parameters of their own, and its gradient.
//
// Per sample and group of Cg = C / G channels, m = P Cg values x:
//   mean = sum x / m,  rstd = 1 / sqrt(sum x^2 / m - mean^2 + eps)
//   xhat = (x - mean) rstd,  z = gamma xhat + beta,  y = act(z)
// and with dz = dy act'(z), per channel A_c = sum_p dz xhat, B_c = sum_p dz:
//   s1 = sum_c gamma_c B_c / m,  s2 = sum_c gamma_c A_c / m  (over the group)
//   dx = rstd (gamma dz - s1 - xhat s2)
//   dgamma_c = sum over the worker's samples of A_c, dbeta_c of B_c
//
// Bound by memory.  A workgroup takes a slab of channels of one sample over a
// range of pixels.  Thread t starts at element t vec of the slab and steps by all
// active threads' elements, a multiple of the slab's width, so its channels
// stay the same: sums per channel are kept in registers and parameters are
// loaded once.  With the whole of the channels as the slab a sample is one run
// of memory, and any C does.
//
// The forward sums are taken in binary64 (mean^2 may be far above the
// variance), the backward ones in fp32 over a thread's values and in binary64
// from there on.
#include <hip/hip_ext.h>

#include "saef_device.h"
#include "saef_group_norm.h"

namespace saef {
namespace {

// vec elements of T at an address aligned to T.
template <int kType, int kN>
struct Vals {
  typedef typename Elem<kType>::T T;
  T v[kN];
  __device__ __forceinline__ void load(const T* p) { __builtin_memcpy(v, p, sizeof(v)); }
  __device__ __forceinline__ void load(const T* p, int n) {
#pragma unroll
    for (int j = 0; j < kN; ++j) v[j] = j < n ? p[j] : (T)0.0f;
  }
  __device__ __forceinline__ void store(T* p) const { __builtin_memcpy(p, v, sizeof(v)); }
  __device__ __forceinline__ void store(T* p, int n) const {
#pragma unroll
    for (int j = 0; j < kN; ++j)
      if (j < n) p[j] = v[j];
  }
  __device__ __forceinline__ float operator[](int j) const { return Elem<kType>::to_f32(v[j]); }
  __device__ __forceinline__ void set(int j, float f) { v[j] = Elem<kType>::of_f32(f); }
};

// 1 / (1 + exp(-z)), to 2 or 3 units in the last place: the exponent's product
// with log2 e is carried to twice the precision.
__device__ __forceinline__ float sigmoid(float z) {
  const float l2e = 1.44269502f, l2e_lo = 1.92596303e-8f, ln2 = 0.693147181f;
  const float hi = -z * l2e;
  const float lo = __builtin_fmaf(-z, l2e, -hi) - z * l2e_lo;
  float e = __builtin_amdgcn_exp2f(hi);
  // (an infinite z or exponential stays what it is)
  e = __builtin_fabsf(hi) < 126.0f ? __builtin_fmaf(e, lo * ln2, e) : e;
  return __builtin_amdgcn_rcpf(1.0f + e);
}

template <int kAct>
__device__ __forceinline__ float act_of(float z) {
  if (kAct == kActRelu) return z < 0.0f ? 0.0f : z;
  if (kAct == kActSilu) return z * sigmoid(z);
  return z;
}

// dy act'(z)
template <int kAct>
__device__ __forceinline__ float act_back(float dy, float z) {
  if (kAct == kActRelu) return z > 0.0f ? dy : 0.0f;
  if (kAct == kActSilu) {
    const float s = sigmoid(z);
    return dy * (s * __builtin_fmaf(z, 1.0f - s, 1.0f));
  }
  return dy;
}

// A workgroup's part of a sample: channels [c0, c0 + cw), pixels [p0, p1).
template <int kN>
struct Part {
  int64_t n;       // sample, over all workers
  int64_t first;   // element of the features the thread starts at
  int64_t left;    // elements of the part from there on (0 or less: none)
  int64_t stride;  // elements of the features, and
  int64_t dec;     // of the part, to the thread's next
  int k, s, c0, cw, c, active;

  __device__ __forceinline__ Part(const GroupNormDev& d) {
    int64_t b = blockIdx.x;
    s = (int)(b % d.splits);
    b /= d.splits;
    c0 = (int)(b % d.slabs) * d.slab;
    n = b / d.slabs;
    k = (int)(n / d.N);
    cw = min(d.slab, d.C - c0);
    const int64_t per = (d.P + d.splits - 1) / d.splits;
    const int64_t p0 = min(d.P, s * per), p1 = min(d.P, p0 + per);
    // threads whose elements make up whole pixels of the slab
    const int common = min(kN, cw & -cw);
    const int period = cw / common;
    active = (int)blockDim.x / period * period;
    const int t = (int)threadIdx.x;
    const int f = t * kN;
    const int p = f / cw;
    c = f - p * cw;
    first = (n * d.P + p0 + p) * d.C + c0 + c;
    left = t < active ? (p1 - p0) * cw - f : 0;
    dec = (int64_t)active * kN;
    stride = dec / cw * d.C;
  }
  // channel of the thread's element j
  __device__ __forceinline__ int channel(int j) const {
    int q = c + j;
    while (q >= cw) q -= cw;
    return c0 + q;
  }
};

// Sums over the threads of a workgroup: v[j] of thread t belongs to channel
// (t kN + j) mod cw.  put(c, sum) is called once for each channel c < cw.
template <int kN, typename V, typename F>
__device__ __forceinline__ void channel_sums(const V (&v)[kN], int active, int cw, V* lds, F put) {
  const int t = (int)threadIdx.x;
  if (t < active) {
#pragma unroll
    for (int j = 0; j < kN; ++j) lds[t * kN + j] = v[j];
  }
  __syncthreads();
  for (int c = t; c < cw; c += (int)blockDim.x) {
    double a = 0.0;
    for (int f = c; f < active * kN; f += cw) a += (double)lds[f];
    put(c, a);
  }
  __syncthreads();
}

extern __shared__ __align__(16) unsigned char dyn_lds[];

// Partial sums per channel: forward x and x^2, backward A and B.
// Grid: K N slabs splits workgroups.
template <int kType, int kN, int kAct, bool kBack>
__global__ __launch_bounds__(1024) void k_gn_sums(GroupNormDev d, const void* __restrict__ xv,
                                                  const void* __restrict__ dyv,
                                                  const float* __restrict__ gamma,
                                                  const float* __restrict__ beta, int64_t ld,
                                                  const float* __restrict__ mean,
                                                  const float* __restrict__ rstd) {
  typedef typename Elem<kType>::T T;
  typedef std::conditional_t<kBack, float, double> Sum;
  const Part<kN> w(d);
  const T* x = static_cast<const T*>(xv) + w.first;
  const T* dy = kBack ? static_cast<const T*>(dyv) + w.first : nullptr;
  Sum a0[kN] = {}, a1[kN] = {};
  float mu[kN], rs[kN], ga[kN], be[kN];
  if (kBack && w.left > 0) {
#pragma unroll
    for (int j = 0; j < kN; ++j) {
      const int c = w.channel(j), g = c / d.Cg;
      mu[j] = mean[w.n * d.G + g];
      rs[j] = rstd[w.n * d.G + g];
      ga[j] = gamma[w.k * ld + c];
      be[j] = beta[w.k * ld + c];
    }
  }
  for (int64_t left = w.left; left > 0; left -= w.dec) {
    Vals<kType, kN> xs, ds;
    if (left >= kN) {
      xs.load(x);
      if (kBack) ds.load(dy);
    } else {
      xs.load(x, (int)left);
      if (kBack) ds.load(dy, (int)left);
    }
#pragma unroll
    for (int j = 0; j < kN; ++j) {
      if (kBack) {
        const float h = (xs[j] - mu[j]) * rs[j];
        const float dz = act_back<kAct>(ds[j], __builtin_fmaf(h, ga[j], be[j]));
        if (left > j) {
          a0[j] = __builtin_fmaf(dz, h, (float)a0[j]);
          a1[j] += dz;
        }
      } else {
        const double v = xs[j];
        a0[j] += v;
        a1[j] = __builtin_fma(v, v, (double)a1[j]);
      }
    }
    x += w.stride;
    if (kBack) dy += w.stride;
  }
  Sum* lds = reinterpret_cast<Sum*>(dyn_lds);
  double* part = d.part + ((w.n * d.splits + w.s) * d.C + w.c0) * 2;
  channel_sums(a0, w.active, w.cw, lds, [&](int c, double v) { part[2 * c] = v; });
  channel_sums(a1, w.active, w.cw, lds, [&](int c, double v) { part[2 * c + 1] = v; });
}

struct GroupSums {
  float a, b, c;  // forward: mean, its remainder, rstd; backward: s1, s2
};

// The two sums of each group that the slab meets, over channels and splits
// (backward: weighted by gamma), by `lanes` lanes a group.  put(g, s0, s1).
template <bool kBack, int kN, typename F>
__device__ __forceinline__ void group_sums(const GroupNormDev& d, const Part<kN>& w,
                                           const float* __restrict__ gamma, int64_t ld, F put) {
  const int g0 = w.c0 / d.Cg, g1 = (w.c0 + w.cw - 1) / d.Cg;
  const int64_t terms = (int64_t)d.Cg * d.splits;
  int lanes = 1;
  while (lanes < kWave && lanes < terms) lanes *= 2;
  const int per = (int)blockDim.x / lanes;
  const int at = (int)threadIdx.x / lanes, l = (int)threadIdx.x % lanes;
  // every lane of a wave takes part in each step
  for (int gb = g0; gb <= g1; gb += per) {
    const int g = gb + at;
    double s0 = 0.0, s1 = 0.0;
    if (g <= g1) {
      for (int64_t i = l; i < terms; i += lanes) {
        const int c = g * d.Cg + (int)(i % d.Cg);
        const double* p = d.part + ((w.n * d.splits + i / d.Cg) * d.C + c) * 2;
        const double f = kBack ? (double)gamma[w.k * ld + c] : 1.0;
        s0 += f * p[0];
        s1 += f * p[1];
      }
    }
    for (int o = lanes / 2; o > 0; o >>= 1) {
      s0 += __shfl_xor(s0, o);
      s1 += __shfl_xor(s1, o);
    }
    if (g <= g1 && l == 0) put(g, s0, s1);
  }
}

// The statistics of m values from their sum and sum of squares.
__device__ __forceinline__ GroupSums stats_of(double s0, double s1, double m, float eps) {
  const double mu = s0 / m;
  const double var = s1 / m - mu * mu;
  GroupSums r;
  r.a = (float)mu;
  r.b = (float)(mu - (double)r.a);
  // (a rounding below 0 is 0; what is no number stays none)
  r.c = (float)(1.0 / sqrt((var < 0.0 ? 0.0 : var) + (double)eps));
  return r;
}

template <int kType, int kN, int kAct>
__global__ __launch_bounds__(1024) void k_gn_apply(GroupNormDev d, const void* __restrict__ xv,
                                                   const float* __restrict__ gamma,
                                                   const float* __restrict__ beta, int64_t ld,
                                                   void* __restrict__ yv,
                                                   float* __restrict__ mean,
                                                   float* __restrict__ rstd) {
  typedef typename Elem<kType>::T T;
  const Part<kN> w(d);
  GroupSums* st = reinterpret_cast<GroupSums*>(dyn_lds);
  const int g0 = w.c0 / d.Cg;
  const double m = (double)d.P * d.Cg;
  group_sums<false>(d, w, nullptr, 0, [&](int g, double s0, double s1) {
    const GroupSums r = stats_of(s0, s1, m, d.eps);
    st[g - g0] = r;
    // (a group over several slabs: all write the same)
    if (w.s == 0) {
      mean[w.n * d.G + g] = r.a;
      rstd[w.n * d.G + g] = r.c;
    }
  });
  __syncthreads();
  if (w.left <= 0) return;
  float mu[kN], sc[kN], sh[kN];
#pragma unroll
  for (int j = 0; j < kN; ++j) {
    const int c = w.channel(j);
    const GroupSums r = st[c / d.Cg - g0];
    mu[j] = r.a;
    sc[j] = r.c * gamma[w.k * ld + c];
    sh[j] = __builtin_fmaf(-r.b, sc[j], beta[w.k * ld + c]);
  }
  const T* x = static_cast<const T*>(xv) + w.first;
  T* y = static_cast<T*>(yv) + w.first;
  for (int64_t left = w.left; left > 0; left -= w.dec) {
    Vals<kType, kN> v;
    if (left >= kN) v.load(x); else v.load(x, (int)left);
#pragma unroll
    for (int j = 0; j < kN; ++j)
      v.set(j, act_of<kAct>(__builtin_fmaf(v[j] - mu[j], sc[j], sh[j])));
    if (left >= kN) v.store(y); else v.store(y, (int)left);
    x += w.stride;
    y += w.stride;
  }
}

template <int kType, int kN, int kAct>
__global__ __launch_bounds__(1024) void k_gn_back(GroupNormDev d, const void* __restrict__ dyv,
                                                  const void* __restrict__ xv,
                                                  const float* __restrict__ gamma,
                                                  const float* __restrict__ beta, int64_t ld,
                                                  const float* __restrict__ mean,
                                                  const float* __restrict__ rstd,
                                                  void* __restrict__ dxv) {
  typedef typename Elem<kType>::T T;
  const Part<kN> w(d);
  GroupSums* st = reinterpret_cast<GroupSums*>(dyn_lds);
  const int g0 = w.c0 / d.Cg;
  const double m = (double)d.P * d.Cg;
  group_sums<true>(d, w, gamma, ld, [&](int g, double s0, double s1) {
    st[g - g0] = GroupSums{(float)(s1 / m), (float)(s0 / m), 0.0f};
  });
  __syncthreads();
  if (w.left <= 0) return;
  float mu[kN], rs[kN], ga[kN], be[kN], s1[kN], s2[kN];
#pragma unroll
  for (int j = 0; j < kN; ++j) {
    const int c = w.channel(j), g = c / d.Cg;
    mu[j] = mean[w.n * d.G + g];
    rs[j] = rstd[w.n * d.G + g];
    ga[j] = gamma[w.k * ld + c];
    be[j] = beta[w.k * ld + c];
    s1[j] = st[g - g0].a;
    s2[j] = st[g - g0].b;
  }
  const T* x = static_cast<const T*>(xv) + w.first;
  const T* dy = static_cast<const T*>(dyv) + w.first;
  T* dx = static_cast<T*>(dxv) + w.first;
  for (int64_t left = w.left; left > 0; left -= w.dec) {
    Vals<kType, kN> xs, ds;
    if (left >= kN) {
      xs.load(x);
      ds.load(dy);
    } else {
      xs.load(x, (int)left);
      ds.load(dy, (int)left);
    }
#pragma unroll
    for (int j = 0; j < kN; ++j) {
      const float h = (xs[j] - mu[j]) * rs[j];
      const float dz = act_back<kAct>(ds[j], __builtin_fmaf(h, ga[j], be[j]));
      ds.set(j, rs[j] * (__builtin_fmaf(ga[j], dz, -s1[j]) - h * s2[j]));
    }
    if (left >= kN) ds.store(dx); else ds.store(dx, (int)left);
    x += w.stride;
    dy += w.stride;
    dx += w.stride;
  }
}

// dgamma and dbeta: the channel sums over a worker's samples and splits.
// Grid: K ceil(C / 64) workgroups of 4 waves; wave w adds rows w, w + 4, ...
__global__ __launch_bounds__(kBlock) void k_gn_params(GroupNormDev d, float* __restrict__ dgamma,
                                                      float* __restrict__ dbeta, int64_t ldg) {
  __shared__ double s_a[kWaves][kWave], s_b[kWaves][kWave];
  const unsigned per = (unsigned)((d.C + kWave - 1) / kWave);
  const int k = (int)(blockIdx.x / per);
  const int c = (int)(blockIdx.x % per) * kWave + lane_id();
  const int w = wave_id();
  const int64_t rows = d.N * d.splits;
  double a = 0.0, b = 0.0;
  if (c < d.C) {
    const double* p = d.part + (k * rows * d.C + c) * 2;
    for (int64_t i = w; i < rows; i += kWaves) {
      a += p[i * d.C * 2];
      b += p[i * d.C * 2 + 1];
    }
  }
  s_a[w][lane_id()] = a;
  s_b[w][lane_id()] = b;
  __syncthreads();
  if (w != 0 || c >= d.C) return;
  for (int i = 1; i < kWaves; ++i) {
    a += s_a[i][lane_id()];
    b += s_b[i][lane_id()];
  }
  dgamma[k * ldg + c] = (float)a;
  dbeta[k * ldg + c] = (float)b;
}

// Calls f with the element type, the vector width and the activation as
// constants.
template <typename F>
hipError_t dispatch(int dtype, int vec, int act, F&& f) {
  auto with_act = [&](auto type, auto n) {
    if (act == kActRelu) f(type, n, std::integral_constant<int, kActRelu>());
    else if (act == kActSilu) f(type, n, std::integral_constant<int, kActSilu>());
    else f(type, n, std::integral_constant<int, kActNone>());
  };
  auto with_vec = [&](auto type) {
    constexpr int full = Elem<decltype(type)::value>::kVec;
    if (vec == 1) with_act(type, std::integral_constant<int, 1>());
    else with_act(type, std::integral_constant<int, full>());
  };
  if (dtype == kF32) with_vec(std::integral_constant<int, kF32>());
  else if (dtype == kBF16) with_vec(std::integral_constant<int, kBF16>());
  else with_vec(std::integral_constant<int, kF16>());
  return hipGetLastError();
}

// LDS of a workgroup: a value of each thread's elements, or the group sums.
size_t sums_lds(const GroupNormDev& d, size_t bytes) { return (size_t)d.threads * d.vec * bytes; }
size_t groups_lds(const GroupNormDev& d) { return ((size_t)d.slab / d.Cg + 2) * sizeof(GroupSums); }

}  // namespace

hipError_t launch_group_norm_forward(const GroupNormDev& d, int dtype, int act, const void* x,
                                     const float* gamma, const float* beta, int64_t ld, void* y,
                                     float* mean, float* rstd, hipStream_t s) {
  const LaunchEvents ev;
  const dim3 grid((unsigned)(d.K * d.N * d.slabs * d.splits)), block((unsigned)d.threads);
  return dispatch(dtype, d.vec, act, [&](auto type, auto n, auto a) {
    constexpr int T = decltype(type)::value, V = decltype(n)::value, A = decltype(a)::value;
    SAEF_LAUNCH((k_gn_sums<T, V, kActNone, false>), grid, block, sums_lds(d, sizeof(double)), s, d,
                x, nullptr, nullptr, nullptr, ld, nullptr, nullptr);
    SAEF_LAUNCH((k_gn_apply<T, V, A>), grid, block, groups_lds(d), s, d, x, gamma, beta, ld, y,
                mean, rstd);
  });
}

hipError_t launch_group_norm_backward(const GroupNormDev& d, int dtype, int act, const void* dy,
                                      const void* x, const float* gamma, const float* beta,
                                      int64_t ld, const float* mean, const float* rstd, void* dx,
                                      float* dgamma, float* dbeta, int64_t ldg, hipStream_t s) {
  const LaunchEvents ev;
  const dim3 grid((unsigned)(d.K * d.N * d.slabs * d.splits)), block((unsigned)d.threads);
  const hipError_t err = dispatch(dtype, d.vec, act, [&](auto type, auto n, auto a) {
    constexpr int T = decltype(type)::value, V = decltype(n)::value, A = decltype(a)::value;
    SAEF_LAUNCH((k_gn_sums<T, V, A, true>), grid, block, sums_lds(d, sizeof(float)), s, d, x, dy,
                gamma, beta, ld, mean, rstd);
    SAEF_LAUNCH((k_gn_back<T, V, A>), grid, block, groups_lds(d), s, d, dy, x, gamma, beta, ld,
                mean, rstd, dx);
  });
  if (err != hipSuccess) return err;
  const dim3 pgrid((unsigned)d.K * (unsigned)((d.C + kWave - 1) / kWave));
  SAEF_LAUNCH(k_gn_params, pgrid, dim3(kBlock), 0, s, d, dgamma, dbeta, ldg);
  return hipGetLastError();
}

}  // namespace saef
