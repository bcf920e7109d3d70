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
// variance).  The backward ones are taken in fp32 over a thread's values of a
// channel (at most 64) and, where the channels repeat within a wave, over the lanes
// that share them (a tree of up to 6 levels), in binary64 over a workgroup's; a
// sample's channel sums are kept in fp32 for dgamma, dbeta.
//
// Measured (256 samples, bf16): 196 x 1024 forward 42 us (4.9 TB/s), backward with
// silu 70 us (4.4 TB/s; about 40 us of vector instructions beside it); 12544 x
// 64, read twice, forward 212 us (5.8 TB/s of what it moves), backward 357.
#include <hip/hip_ext.h>

#include <algorithm>

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
  // 16 bytes at the alignment of the smallest element
  typedef unsigned int Raw __attribute__((ext_vector_type(4), aligned(2)));
  __device__ __forceinline__ void load_nt(const T* p) {
    if constexpr (sizeof(v) == 16) {
      const Raw r = __builtin_nontemporal_load(reinterpret_cast<const Raw*>(p));
      __builtin_memcpy(v, &r, 16);
    } else {
      load(p);
    }
  }
  __device__ __forceinline__ void load(const T* p, int n) {
#pragma unroll
    for (int j = 0; j < kN; ++j) v[j] = j < n ? p[j] : (T)0.0f;
  }
  __device__ __forceinline__ void store(T* p) const {
    if constexpr (sizeof(v) == 16) {
      Raw r;
      __builtin_memcpy(&r, v, 16);
      __builtin_nontemporal_store(r, reinterpret_cast<Raw*>(p));
    } else {
      __builtin_memcpy(p, v, sizeof(v));
    }
  }
  __device__ __forceinline__ void store(T* p, int n) const {
#pragma unroll
    for (int j = 0; j < kN; ++j)
      if (j < n) p[j] = v[j];
  }
  __device__ __forceinline__ float operator[](int j) const { return Elem<kType>::to_f32(v[j]); }
  __device__ __forceinline__ void set(int j, float f) { v[j] = Elem<kType>::of_f32(f); }
};

// 1 / (1 + exp(-z)), to about 4 (1 + |z|) 2^-24 relative: four instructions, two of
// them at a quarter of the rate.  An infinite exponential gives 0.
__device__ __forceinline__ float sigmoid(float z) {
  return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.44269504f * z));
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

// The statistics of m values from their sum and sum of squares; inv_m = 1 / m.
struct Stats {
  float mean, rest, rstd;  // mean rounded to fp32, and what that leaves
};
__device__ __forceinline__ Stats stats_of(double s0, double s1, double inv_m, float eps) {
  const double mu = s0 * inv_m;
  const double var = s1 * inv_m - mu * mu;
  Stats r;
  r.mean = (float)mu;
  r.rest = (float)(mu - (double)r.mean);
  // (a rounding below 0 is 0; what is no number stays none)
  r.rstd = (float)rsqrt((var < 0.0 ? 0.0 : var) + (double)eps);
  return r;
}

extern __shared__ __align__(16) unsigned char dyn_lds[];

// Joins pairs of sums: put(i, sum of at(i, 0), at(i, 1), ...) for i < count, of up
// to `terms` terms each.  A power of two of lanes adds up one of them, few enough
// that `most` of them (count, or more) are under way at once: the order of a sum
// depends on `terms` and `most` alone.  All threads of the workgroup call it.
template <typename At, typename Put>
__device__ __forceinline__ void join_sums(int count, int most, int terms, At at, Put put) {
  int lanes = 1;
  while (lanes < kWave && lanes < terms && 2 * lanes * most <= (int)blockDim.x) lanes *= 2;
  const int l = (int)threadIdx.x & (lanes - 1), per = (int)blockDim.x / lanes;
  for (int base = 0; base < count; base += per) {
    const int i = base + (int)threadIdx.x / lanes;
    double2 s = make_double2(0.0, 0.0);
    if (i < count) {
#pragma unroll 4
      for (int q = l; q < terms; q += lanes) {
        const double2 v = at(i, q);
        s.x += v.x;
        s.y += v.y;
      }
    }
    for (int o = lanes / 2; o > 0; o >>= 1) {
      s.x += __shfl_xor(s.x, o);
      s.y += __shfl_xor(s.y, o);
    }
    if (i < count && l == 0) put(i, s);
  }
}
template <typename At, typename Put>
__device__ __forceinline__ void join_sums(int count, int terms, At at, Put put) {
  join_sums(count, count, terms, at, put);
}

// Before a workgroup's threads lay their sums side by side in LDS: where the
// channels repeat every `period` threads, a power of two below a wave, the lanes
// of a wave that share theirs are added first.
__host__ __device__ inline bool folds(int period) {
  return period < kWave && (period & (period - 1)) == 0;
}
template <int kA, typename V>
__device__ __forceinline__ void fold_lanes(V (&v)[kA], V (&w)[kA], int period) {
  if (!folds(period)) return;
  for (int o = kWave / 2; o >= period; o /= 2) {
#pragma unroll
    for (int j = 0; j < kA; ++j) {
      v[j] += __shfl_xor(v[j], o);
      w[j] += __shfl_xor(w[j], o);
    }
  }
}
// This thread's place in the table, or -1; `places`, the threads with sums,
// becomes the number of places.
__device__ __forceinline__ int fold_place(int period, int& places) {
  const int t = (int)threadIdx.x;
  if (!folds(period)) return t < places ? t : -1;
  places = (int)blockDim.x / kWave * period;
  const int l = t % kWave;
  return l < period ? t / kWave * period + l : -1;
}
// Places of a workgroup of `threads` threads, at most.
inline int table_places(int threads, int period) {
  return folds(period) ? threads / kWave * period : threads;
}

// ------------------------------------------------------------------ two passes
// Samples too large for a workgroup are read twice: each workgroup adds up a
// slab of channels over a range of pixels, then a second kernel joins a
// sample's sums and computes the result.  Where the features exceed the last-level
// cache the second goes through the samples backwards, so that what the cache still
// holds is read from there (256 samples of 1.6 MB: 20 us less forward and 18 less
// backward than in the same order; at 103 MB the same order is 1 us ahead).

// Vectors of a thread's in flight.
constexpr int kU = 4;

// A workgroup's part of a sample: channels [c0, c0 + cw), pixels [p0, p1).
template <int kN>
struct Part {
  int64_t n;       // sample, over all workers
  int64_t first;   // element of the features the thread starts at
  int64_t left;    // elements of the part from there on (0 or less: none)
  int64_t stride;  // elements of the features, and
  int64_t dec;     // of the part, to the thread's next vector
  int k, s, b, c0, cw, c, period, active;

  __device__ __forceinline__ Part(const GroupNormDev& d, uint32_t item) {
    s = (int)(item % (uint32_t)d.splits);
    item /= (uint32_t)d.splits;
    b = (int)(item % (uint32_t)d.slabs);
    c0 = b * d.slab;
    n = item / (uint32_t)d.slabs;
    k = (int)((uint32_t)n / (uint32_t)d.N);
    cw = min(d.slab, d.C - c0);
    const int64_t p0 = min(d.P, s * d.split_pixels), p1 = min(d.P, p0 + d.split_pixels);
    // threads whose elements make up whole pixels of the slab
    period = cw / min(kN, cw & -cw);
    active = (int)blockDim.x / period * period;
    const int t = (int)threadIdx.x;
    const int f = t * kN;
    const int p = f / cw;
    c = f - p * cw;
    first = (n * d.P + p0 + p) * d.C + c0 + c;
    left = t < active ? (p1 - p0) * cw - f : 0;
    dec = active * kN;
    stride = (int64_t)(active * kN / cw) * d.C;
  }
  // Calls f(j, channel, group) for the thread's elements j.
  template <typename F>
  __device__ __forceinline__ void channels(const GroupNormDev& d, F f) const {
    int q = c, g = (c0 + c) / d.Cg, in = c0 + c - g * d.Cg;
#pragma unroll
    for (int j = 0; j < kN; ++j) {
      f(j, c0 + q, g);
      ++q;
      if (++in == d.Cg) {
        in = 0;
        ++g;
      }
      if (q == cw) {  // the next pixel (the slab is all channels then)
        q = 0;
        g = 0;
        in = 0;
      }
    }
  }
  // groups that the slab meets, and the channels of the i-th within the slab
  __device__ __forceinline__ int group0(const GroupNormDev& d) const { return c0 / d.Cg; }
  __device__ __forceinline__ int groups(const GroupNormDev& d) const {
    return (c0 + cw - 1) / d.Cg - c0 / d.Cg + 1;
  }
  __device__ __forceinline__ int lo(const GroupNormDev& d, int i) const {
    return max((group0(d) + i) * d.Cg - c0, 0);
  }
  __device__ __forceinline__ int hi(const GroupNormDev& d, int i) const {
    return min((group0(d) + i + 1) * d.Cg - c0, cw);
  }
};

// The vectors of a thread's part, from kS features at once: kU of each are on
// their way while the kU before are used.  kLast: nobody reads them again, so they pass
// the last-level cache by (784 x 512 bf16, 256 samples, backward 190 us, 206 without;
// in the first pass the same costs: 50 MB forward 25 us instead of 20).
template <int kType, int kN, int kS, bool kLast>
struct Stream {
  typedef typename Elem<kType>::T T;
  const T* src[kS];
  int64_t rest, at, dec, stride;
  Vals<kType, kN> v[kU][kS];

  __device__ __forceinline__ Stream(const Part<kN>& w, const void* a, const void* b = nullptr)
      : rest(w.left), at(w.first), dec(w.dec), stride(w.stride) {
    src[0] = static_cast<const T*>(a);
    if (kS > 1) src[kS - 1] = static_cast<const T*>(b);
    if (rest >= kN) fetch(v, rest, at);
  }
  // (vectors past the part's end: the first one again)
  __device__ __forceinline__ void fetch(Vals<kType, kN> (&to)[kU][kS], int64_t left,
                                        int64_t from) const {
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      const int64_t p = left - u * dec >= kN ? from + u * stride : from;
#pragma unroll
      for (int i = 0; i < kS; ++i) {
        if (kLast) to[u][i].load_nt(src[i] + p);
        else to[u][i].load(src[i] + p);
      }
    }
  }
  // Calls f(v, at, n) with the thread's vectors one after another: n elements
  // from element `at` of the features.
  template <typename F>
  __device__ __forceinline__ void each(F f) {
    while (rest >= kN) {
      Vals<kType, kN> next[kU][kS];
      const bool more = rest - kU * dec >= kN;  // (at least one whole vector left)
      if (more) fetch(next, rest - kU * dec, at + kU * stride);
#pragma unroll
      for (int u = 0; u < kU; ++u) {
        if (rest >= kN) {
          f(v[u], at, kN);
          rest -= dec;
          at += stride;
        }
      }
      if (!more) break;
#pragma unroll
      for (int u = 0; u < kU; ++u)
#pragma unroll
        for (int i = 0; i < kS; ++i) v[u][i] = next[u][i];
    }
    // the sample's last elements, fewer than a vector
    if (rest > 0) {
      Vals<kType, kN> last[kS];
#pragma unroll
      for (int i = 0; i < kS; ++i) last[i].load(src[i] + at, (int)rest);
      f(last, at, (int)rest);
    }
  }
};

// The sums of the i-th group of the slab over all pixel ranges and, where
// groups span slabs, all slabs: entry g + b of a row belongs to group g in slab b.
template <int kN, typename Put>
__device__ __forceinline__ void join_groups(const GroupNormDev& d, const Part<kN>& w, Put put) {
  const int Q = d.G + d.slabs - 1;
  // slabs a group may lie in, at most
  const int span = d.slab % d.Cg == 0 ? 1 : min(d.slabs, (d.Cg - 1) / d.slab + 2);
  const double2* pieces = reinterpret_cast<const double2*>(d.pieces) + w.n * d.splits * Q;
  if (span == 1) {  // whole groups: those of this slab
    pieces += w.group0(d) + w.b;
    join_sums(w.groups(d), d.splits, [&](int i, int q) { return pieces[(int64_t)q * Q + i]; }, put);
    return;
  }
  // Every slab of a group joins the same pieces; in one order, that of a slab that meets
  // as many groups as one may, they come to the same statistics.
  const int most = (d.slab + d.Cg - 2) / d.Cg + 1;
  join_sums(w.groups(d), most, d.splits * span, [&](int i, int q) {
    const int g = w.group0(d) + i, b = g * d.Cg / d.slab + q % span;
    if (b > (g * d.Cg + d.Cg - 1) / d.slab) return make_double2(0.0, 0.0);
    return pieces[(int64_t)(q / span) * Q + g + b];
  }, put);
}

// kOne: a vector lies in one group.  Grid: K N slabs splits workgroups.
template <int kType, int kN, bool kOne>
__global__ __launch_bounds__(kBlock) void k_gn_fwd_sums(GroupNormDev d,
                                                        const void* __restrict__ x) {
  constexpr int kA = kOne ? 1 : kN;  // sums of a thread
  const Part<kN> w(d, blockIdx.x);
  double a0[kA] = {}, a1[kA] = {};
  Stream<kType, kN, 1, false>(w, x).each([&](Vals<kType, kN>* v, int64_t, int) {
#pragma unroll
    for (int j = 0; j < kN; ++j) {
      const double f = v[0][j];
      a0[kOne ? 0 : j] += f;
      a1[kOne ? 0 : j] = __builtin_fma(f, f, a1[kOne ? 0 : j]);
    }
  });
  double2* table = reinterpret_cast<double2*>(dyn_lds);
  int places = w.active;
  const int place = fold_place(w.period, places);
  fold_lanes(a0, a1, w.period);
  if (place >= 0) {
#pragma unroll
    for (int j = 0; j < kA; ++j) table[place * kA + j] = make_double2(a0[j], a1[j]);
  }
  __syncthreads();
  // entries of a pixel of the slab, and pixels
  constexpr int kPer = kN / kA;
  const int wide = w.cw / kPer, rows = places * kA / wide, most = min(d.Cg, w.cw) / kPer;
  double2* out = reinterpret_cast<double2*>(d.pieces) +
                 (w.n * d.splits + w.s) * (d.G + d.slabs - 1) + w.group0(d) + w.b;
  join_sums(w.groups(d), rows * most, [&](int i, int q) {
    const int e = w.lo(d, i) / kPer + q % most;
    return e < w.hi(d, i) / kPer ? table[q / most * wide + e] : make_double2(0.0, 0.0);
  }, [&](int i, double2 s) { out[i] = s; });
}

template <int kType, int kN, int kAct>
__global__ __launch_bounds__(kBlock) void k_gn_fwd_apply(GroupNormDev d,
                                                         const void* __restrict__ x,
                                                         const float* __restrict__ gamma,
                                                         const float* __restrict__ beta,
                                                         int64_t ld, void* __restrict__ y,
                                                         float* __restrict__ mean,
                                                         float* __restrict__ rstd) {
  typedef typename Elem<kType>::T T;
  const Part<kN> w(d, d.backwards ? gridDim.x - 1 - blockIdx.x : blockIdx.x);
  Stream<kType, kN, 1, true> in(w, x);
  Stats* st = reinterpret_cast<Stats*>(dyn_lds);
  const int g0 = w.group0(d);
  float mu[kN], sc[kN], sh[kN];
  w.channels(d, [&](int j, int c, int) {
    sc[j] = gamma[w.k * ld + c];
    sh[j] = beta[w.k * ld + c];
  });
  const double inv_m = 1.0 / ((double)d.P * d.Cg);
  join_groups(d, w, [&](int i, double2 s) {
    const Stats r = stats_of(s.x, s.y, inv_m, d.eps);
    st[i] = r;
    // (a group in several slabs: the one of its first channel)
    if (w.s == 0 && (g0 + i) * d.Cg >= w.c0) {
      mean[w.n * d.G + g0 + i] = r.mean;
      rstd[w.n * d.G + g0 + i] = r.rstd;
    }
  });
  __syncthreads();
  if (w.left <= 0) return;
  w.channels(d, [&](int j, int, int g) {
    const Stats r = st[g - g0];
    mu[j] = r.mean;
    sc[j] = r.rstd * sc[j];
    sh[j] = __builtin_fmaf(-r.rest, sc[j], sh[j]);
  });
  in.each([&](Vals<kType, kN>* v, int64_t at, int n) {
#pragma unroll
    for (int j = 0; j < kN; ++j)
      v[0].set(j, act_of<kAct>(__builtin_fmaf(v[0][j] - mu[j], sc[j], sh[j])));
    T* p = static_cast<T*>(y) + at;
    if (n == kN) v[0].store(p); else v[0].store(p, n);
  });
}

// Per channel A and B of the part, and per group their sums weighted by gamma.
template <int kType, int kN, int kAct>
__global__ __launch_bounds__(kBlock) void k_gn_bwd_sums(GroupNormDev d,
                                                        const void* __restrict__ x,
                                                        const void* __restrict__ dy,
                                                        const float* __restrict__ gamma,
                                                        const float* __restrict__ beta,
                                                        int64_t ld,
                                                        const float* __restrict__ mean,
                                                        const float* __restrict__ rstd) {
  const Part<kN> w(d, blockIdx.x);
  Stream<kType, kN, 2, false> in(w, x, dy);
  float a[kN] = {}, b[kN] = {};
  if (w.left > 0) {
    float mu[kN], gs[kN], be[kN];
    w.channels(d, [&](int j, int c, int g) {
      mu[j] = mean[w.n * d.G + g];
      gs[j] = gamma[w.k * ld + c] * rstd[w.n * d.G + g];
      be[j] = beta[w.k * ld + c];
    });
    in.each([&](Vals<kType, kN>* v, int64_t, int n) {
#pragma unroll
      for (int j = 0; j < kN; ++j) {
        const float u = v[0][j] - mu[j];
        const float dz = act_back<kAct>(v[1][j], __builtin_fmaf(u, gs[j], be[j]));
        if (n == kN || j < n) {
          a[j] = __builtin_fmaf(dz, u, a[j]);
          b[j] += dz;
        }
      }
    });
  }
  // element f of the threads' sums side by side belongs to channel f mod cw
  float2* table = reinterpret_cast<float2*>(dyn_lds);
  int places = w.active;
  const int place = fold_place(w.period, places);
  fold_lanes(a, b, w.period);
  const int t = (int)threadIdx.x, elems = places * kN;
  double2* sums = reinterpret_cast<double2*>(table + (elems + 1) / 2 * 2);  // 16-byte aligned
  if (place >= 0) {
#pragma unroll
    for (int j = 0; j < kN; ++j) table[place * kN + j] = make_float2(a[j], b[j]);
  }
  __syncthreads();
  float2* part = reinterpret_cast<float2*>(d.part) + (w.n * d.splits + w.s) * d.C + w.c0;
  for (int c = t; c < w.cw; c += (int)blockDim.x) {
    double2 s = make_double2(0.0, 0.0);
    for (int f = c; f < elems; f += w.cw) {
      s.x += (double)table[f].x;
      s.y += (double)table[f].y;
    }
    s.x *= (double)rstd[w.n * d.G + (w.c0 + c) / d.Cg];
    part[c] = make_float2((float)s.x, (float)s.y);
    const double f = gamma[w.k * ld + w.c0 + c];
    sums[c] = make_double2(f * s.x, f * s.y);
  }
  __syncthreads();
  const int most = min(d.Cg, w.cw);
  double2* out = reinterpret_cast<double2*>(d.pieces) +
                 (w.n * d.splits + w.s) * (d.G + d.slabs - 1) + w.group0(d) + w.b;
  join_sums(w.groups(d), most, [&](int i, int q) {
    const int e = w.lo(d, i) + q;
    return e < w.hi(d, i) ? sums[e] : make_double2(0.0, 0.0);
  }, [&](int i, double2 s) { out[i] = s; });
}

// dgamma and dbeta of 64 channels of a worker: the channel sums over its samples
// and their pixel ranges, which are kept in fp32 (with a pixel or few a sample they are
// as large as the features) and added up in binary64.  The workgroup's waves take
// the rows in turn; block < K ceil(C / 64).
__device__ __forceinline__ void param_sums(const GroupNormDev& d, int splits, unsigned block,
                                           float* __restrict__ dgamma,
                                           float* __restrict__ dbeta, int64_t ldg) {
  double2* table = reinterpret_cast<double2*>(dyn_lds);  // [waves 64]
  const unsigned per = (unsigned)((d.C + kWave - 1) / kWave);
  const int k = (int)(block / per), waves = (int)blockDim.x / kWave;
  const int c = (int)(block % per) * kWave + lane_id();
  const int w = wave_id();
  const int64_t rows = d.N * splits;
  double2 s = make_double2(0.0, 0.0);
  if (c < d.C) {
    const float2* p = reinterpret_cast<const float2*>(d.part) + k * rows * d.C + c;
#pragma unroll 4
    for (int64_t i = w; i < rows; i += waves) {
      const float2 v = p[i * d.C];
      s.x += (double)v.x;
      s.y += (double)v.y;
    }
  }
  table[threadIdx.x] = s;
  __syncthreads();
  if (w != 0 || c >= d.C) return;
  for (int i = 1; i < waves; ++i) {
    s.x += table[i * kWave + lane_id()].x;
    s.y += table[i * kWave + lane_id()].y;
  }
  dgamma[k * ldg + c] = (float)s.x;
  dbeta[k * ldg + c] = (float)s.y;
}

// The first `params` workgroups take dgamma and dbeta along: a launch less.
template <int kType, int kN, int kAct>
__global__ __launch_bounds__(kBlock) void k_gn_bwd_apply(GroupNormDev d,
                                                         const void* __restrict__ dy,
                                                         const void* __restrict__ x,
                                                         const float* __restrict__ gamma,
                                                         const float* __restrict__ beta,
                                                         int64_t ld,
                                                         const float* __restrict__ mean,
                                                         const float* __restrict__ rstd,
                                                         void* __restrict__ dx,
                                                         float* __restrict__ dgamma,
                                                         float* __restrict__ dbeta,
                                                         int64_t ldg, unsigned params) {
  typedef typename Elem<kType>::T T;
  if (blockIdx.x < params) {
    param_sums(d, d.splits, blockIdx.x, dgamma, dbeta, ldg);
    return;
  }
  const Part<kN> w(d, d.backwards ? gridDim.x - 1 - blockIdx.x : blockIdx.x - params);
  Stream<kType, kN, 2, true> in(w, x, dy);
  float2* st = reinterpret_cast<float2*>(dyn_lds);
  const int g0 = w.group0(d);
  float mu[kN], rs[kN], gs[kN], be[kN], k1[kN], k2[kN];
  w.channels(d, [&](int j, int c, int g) {
    mu[j] = mean[w.n * d.G + g];
    rs[j] = rstd[w.n * d.G + g];
    gs[j] = gamma[w.k * ld + c] * rs[j];
    be[j] = beta[w.k * ld + c];
  });
  const double inv_m = 1.0 / ((double)d.P * d.Cg);
  join_groups(d, w, [&](int i, double2 s) {
    st[i] = make_float2((float)(s.y * inv_m), (float)(s.x * inv_m));
  });
  __syncthreads();
  if (w.left <= 0) return;
  // dx = gamma rstd dz - rstd s1 - ((x - mean) rstd) (rstd s2)
  w.channels(d, [&](int j, int, int g) {
    k1[j] = rs[j] * st[g - g0].x;
    k2[j] = rs[j] * st[g - g0].y;
  });
  in.each([&](Vals<kType, kN>* v, int64_t at, int n) {
#pragma unroll
    for (int j = 0; j < kN; ++j) {
      const float u = v[0][j] - mu[j];
      const float dz = act_back<kAct>(v[1][j], __builtin_fmaf(u, gs[j], be[j]));
      v[0].set(j, __builtin_fmaf(gs[j], dz, -__builtin_fmaf(u * rs[j], k2[j], k1[j])));
    }
    T* p = static_cast<T*>(dx) + at;
    if (n == kN) v[0].store(p); else v[0].store(p, n);
  });
}

// ------------------------------------------------------------------ one pass
// Features of a slab small enough for the registers of a workgroup are read once:
// the sums are taken as they arrive, joined over the workgroup in LDS, and the
// result is computed from the registers.  A slab holds whole groups and whole
// 16-byte vectors.
//
// Reads go through a buffer resource over the sample: a vector past its last
// pixel reads 0, which adds nothing to a sum, and is not written.
constexpr int kHeldThreads = 512;  // of a workgroup, at most

template <int kType, int kR>
struct Held {
  static constexpr int kN = Elem<kType>::kVec;
  typedef typename Elem<kType>::T T;
  int64_t n;       // sample, over all workers
  int k, c0, c;    // worker, first channel of the slab and of the thread within it
  int cols;        // columns of vectors in the slab
  int active;      // threads whose vectors make up whole pixels
  uint32_t at;     // byte offset of the thread's first vector in the sample
  uint32_t step;   // and to its next
  uint32_t bytes;  // of the sample

  __device__ __forceinline__ explicit Held(const GroupNormDev& d) {
    c0 = (int)(blockIdx.x % (uint32_t)d.slabs) * d.slab;
    n = blockIdx.x / (uint32_t)d.slabs;
    k = (int)((uint32_t)n / (uint32_t)d.N);
    cols = min(d.slab, d.C - c0) / kN;
    const int t = (int)threadIdx.x;
    const int rows = (int)blockDim.x / cols;
    active = rows * cols;
    const int p = t / cols;
    c = (t - p * cols) * kN;
    bytes = (uint32_t)d.P * (uint32_t)d.C * (uint32_t)sizeof(T);
    step = (uint32_t)rows * (uint32_t)d.C * (uint32_t)sizeof(T);
    at = t < active ? ((uint32_t)p * (uint32_t)d.C + (uint32_t)(c0 + c)) * (uint32_t)sizeof(T)
                    : 0x80000000u;
  }
  // whether any lane of the wave holds a pixel of the sample in vector i
  __device__ __forceinline__ bool any(int i) const { return __ballot(at + i * step < bytes) != 0; }
  __device__ __forceinline__ Buf over(const GroupNormDev& d, const void* p) const {
    return buf_of(static_cast<const T*>(p) + n * d.P * d.C, bytes);
  }
  __device__ __forceinline__ void load(Buf r, u32x4 (&raw)[kR]) const {
#pragma unroll
    for (int i = 0; i < kR; ++i)
      raw[i] = __builtin_amdgcn_raw_buffer_load_b128(r, at + i * step, 0, kAuxNT);
  }
  __device__ __forceinline__ int groups(const GroupNormDev& d) const { return cols * kN / d.Cg; }
};

template <int kType>
__device__ __forceinline__ Vals<kType, Elem<kType>::kVec> vals_of(const u32x4& raw) {
  Vals<kType, Elem<kType>::kVec> v;
  __builtin_memcpy(&v, &raw, 16);
  return v;
}
template <int kType>
__device__ __forceinline__ u32x4 raw_of(const Vals<kType, Elem<kType>::kVec>& v) {
  u32x4 raw;
  __builtin_memcpy(&raw, &v, 16);
  return raw;
}

// Makes the compiler unpack the vectors again where they are used next, instead of
// keeping their values in twice the registers meanwhile (16-bit features, 8
// vectors a thread, forward: 96 registers, 116 otherwise; 99 and 160 where a vector
// meets several groups).
template <int kR>
__device__ __forceinline__ void packed(u32x4 (&raw)[kR]) {
#pragma unroll
  for (int i = 0; i < kR; ++i) {
    uint32_t a = raw[i].x, b = raw[i].y, c = raw[i].z, e = raw[i].w;
    asm volatile("" : "+v"(a), "+v"(b), "+v"(c), "+v"(e));
    raw[i] = u32x4{a, b, c, e};
  }
}

// kOne: a vector lies in one group.  Grid: K N slabs workgroups.
template <int kType, int kAct, int kR, bool kOne>
__global__ __launch_bounds__(kHeldThreads) void k_gn_fwd_held(GroupNormDev d,
                                                              const void* __restrict__ x,
                                                              const float* __restrict__ gamma,
                                                              const float* __restrict__ beta,
                                                              int64_t ld, void* __restrict__ y,
                                                              float* __restrict__ mean,
                                                              float* __restrict__ rstd) {
  constexpr int kN = Elem<kType>::kVec;
  constexpr int kA = kOne ? 1 : kN;  // sums of a thread
  const Held<kType, kR> w(d);
  u32x4 raw[kR];
  w.load(w.over(d, x), raw);
  float ga[kN], be[kN];
#pragma unroll
  for (int j = 0; j < kN; ++j) {
    ga[j] = gamma[w.k * ld + w.c0 + w.c + j];
    be[j] = beta[w.k * ld + w.c0 + w.c + j];
  }
  // entry p kA + j of the table belongs to channel ((p kA + j) mod (cols kA)) kN / kA
  double2* table = reinterpret_cast<double2*>(dyn_lds);
  int places = w.active;
  const int place = fold_place(w.cols, places);
  Stats* st = reinterpret_cast<Stats*>(table + places * kA);
  const int groups = w.groups(d);
  const int wide = d.Cg * kA / kN;           // entries of a group in a pixel
  const int terms = places / w.cols * wide;  // and in all
  const double inv_m = 1.0 / ((double)d.P * d.Cg);
  double a0[kA] = {}, a1[kA] = {};
#pragma unroll
  for (int i = 0; i < kR; ++i) {
    if (!w.any(i)) continue;
    const auto v = vals_of<kType>(raw[i]);
#pragma unroll
    for (int j = 0; j < kN; ++j) {
      const double f = v[j];
      a0[kOne ? 0 : j] += f;
      a1[kOne ? 0 : j] = __builtin_fma(f, f, a1[kOne ? 0 : j]);
    }
  }
  fold_lanes(a0, a1, w.cols);
  if (place >= 0) {
#pragma unroll
    for (int j = 0; j < kA; ++j) table[place * kA + j] = make_double2(a0[j], a1[j]);
  }
  __syncthreads();
  join_sums(groups, terms, [&](int g, int e) {
    return table[e / wide * w.cols * kA + g * wide + e % wide];
  }, [&](int g, double2 s) {
    const Stats r = stats_of(s.x, s.y, inv_m, d.eps);
    st[g] = r;
    const int64_t at = w.n * d.G + w.c0 / d.Cg + g;
    mean[at] = r.mean;
    rstd[at] = r.rstd;
  });
  __syncthreads();
  float mu[kA], sc[kN], sh[kN];
#pragma unroll
  for (int j = 0; j < kN; ++j) {
    const Stats r = st[(w.c + j) / d.Cg];
    if (j < kA) mu[j] = r.mean;
    sc[j] = r.rstd * ga[j];
    sh[j] = __builtin_fmaf(-r.rest, sc[j], be[j]);
  }
  packed(raw);
  const Buf ry = w.over(d, y);
#pragma unroll
  for (int i = 0; i < kR; ++i) {
    if (!w.any(i)) continue;
    auto v = vals_of<kType>(raw[i]);
#pragma unroll
    for (int j = 0; j < kN; ++j)
      v.set(j, act_of<kAct>(__builtin_fmaf(v[j] - mu[kOne ? 0 : j], sc[j], sh[j])));
    __builtin_amdgcn_raw_buffer_store_b128(raw_of<kType>(v), ry, w.at + i * w.step, 0, kAuxNT);
  }
}

// dz is formed once and kept in fp32 beside x.  With one sample a worker its channel
// sums are dgamma and dbeta.  Grid: K N slabs workgroups.
template <int kType, int kAct, int kR, bool kOne>
__global__ __launch_bounds__(kHeldThreads) void k_gn_bwd_held(GroupNormDev d,
                                                              const void* __restrict__ dy,
                                                              const void* __restrict__ x,
                                                              const float* __restrict__ gamma,
                                                              const float* __restrict__ beta,
                                                              int64_t ld,
                                                              const float* __restrict__ mean,
                                                              const float* __restrict__ rstd,
                                                              void* __restrict__ dx,
                                                              float* __restrict__ dgamma,
                                                              float* __restrict__ dbeta,
                                                              int64_t ldg) {
  constexpr int kN = Elem<kType>::kVec;
  constexpr int kA = kOne ? 1 : kN;
  const Held<kType, kR> w(d);
  u32x4 raw[kR], rdy[kR];
  w.load(w.over(d, x), raw);
  w.load(w.over(d, dy), rdy);
  const int t = (int)threadIdx.x;
  float mu[kA], rs[kA], gs[kN], be[kN];
  const int64_t g0 = w.n * d.G + w.c0 / d.Cg;
#pragma unroll
  for (int j = 0; j < kA; ++j) {
    mu[j] = mean[g0 + (w.c + j) / d.Cg];
    rs[j] = rstd[g0 + (w.c + j) / d.Cg];
  }
#pragma unroll
  for (int j = 0; j < kN; ++j) {
    gs[j] = gamma[w.k * ld + w.c0 + w.c + j] * rs[kOne ? 0 : j];
    be[j] = beta[w.k * ld + w.c0 + w.c + j];
  }
  int places = w.active;
  const int place = fold_place(w.cols, places);
  const int cw = w.cols * kN, elems = places * kN, groups = w.groups(d);
  float* ta = reinterpret_cast<float*>(dyn_lds);
  float* tb = ta + elems;
  double* ca = reinterpret_cast<double*>(tb + elems);   // [cw 2] channel sums
  float2* sg = reinterpret_cast<float2*>(ca + 2 * cw);  // [groups] s1, s2
  const double inv_m = 1.0 / ((double)d.P * d.Cg);
  // per channel: sum of dz (x - mean), and of dz
  float a[kN] = {}, b[kN] = {};
  float dz[kR][kN];
#pragma unroll
  for (int i = 0; i < kR; ++i) {
    if (!w.any(i)) continue;
    const auto v = vals_of<kType>(raw[i]), g = vals_of<kType>(rdy[i]);
#pragma unroll
    for (int j = 0; j < kN; ++j) {
      const float u = v[j] - mu[kOne ? 0 : j];
      const float q = act_back<kAct>(g[j], __builtin_fmaf(u, gs[j], be[j]));
      dz[i][j] = q;
      a[j] = __builtin_fmaf(q, u, a[j]);
      b[j] += q;
    }
  }
  // (what this thread's channel sum is scaled by, on its way before the barrier)
  const int c1 = t < cw ? t : t - cw;
  const bool sums = t < 2 * cw;
  const float r1 = sums ? rstd[g0 + c1 / d.Cg] : 0.0f;
  const float ga1 = sums ? gamma[w.k * ld + w.c0 + c1] : 0.0f;
  // element f of the threads' sums side by side belongs to channel f mod cw
  fold_lanes(a, b, w.cols);
  if (place >= 0) {
#pragma unroll
    for (int j = 0; j < kN; ++j) {
      ta[place * kN + j] = a[j];
      tb[place * kN + j] = b[j];
    }
  }
  __syncthreads();
  float* part = d.part + (w.n * d.C + w.c0) * 2;
  for (int e = t; e < 2 * cw; e += (int)blockDim.x) {
    const int c = e >= cw ? e - cw : e;
    const float* p = e >= cw ? tb : ta;
    double s = 0.0;
    for (int f = c; f < elems; f += cw) s += (double)p[f];
    const float r = e == t ? r1 : rstd[g0 + c / d.Cg];
    const float ga = e == t ? ga1 : gamma[w.k * ld + w.c0 + c];
    if (e < cw) s *= (double)r;
    if (d.N > 1) part[2 * c + (e >= cw)] = (float)s;
    else (e < cw ? dgamma : dbeta)[w.k * ldg + w.c0 + c] = (float)s;
    ca[2 * c + (e >= cw)] = s * (double)ga;
  }
  __syncthreads();
  join_sums(groups, d.Cg, [&](int g, int i) {
    return reinterpret_cast<const double2*>(ca)[g * d.Cg + i];
  }, [&](int g, double2 s) { sg[g] = make_float2((float)(s.y * inv_m), (float)(s.x * inv_m)); });
  __syncthreads();
  // dx = gamma rstd dz - rstd s1 - ((x - mean) rstd) (rstd s2)
  float k1[kA], k2[kA];
#pragma unroll
  for (int j = 0; j < kA; ++j) {
    const float2 s = sg[(w.c + j) / d.Cg];
    k1[j] = rs[j] * s.x;
    k2[j] = rs[j] * s.y;
  }
  packed(raw);
  const Buf ro = w.over(d, dx);
#pragma unroll
  for (int i = 0; i < kR; ++i) {
    if (!w.any(i)) continue;
    auto v = vals_of<kType>(raw[i]);
#pragma unroll
    for (int j = 0; j < kN; ++j) {
      const int o = kOne ? 0 : j;
      const float h = (v[j] - mu[o]) * rs[o];
      v.set(j, __builtin_fmaf(gs[j], dz[i][j], -__builtin_fmaf(h, k2[o], k1[o])));
    }
    __builtin_amdgcn_raw_buffer_store_b128(raw_of<kType>(v), ro, w.at + i * w.step, 0, kAuxNT);
  }
}

// ---- channels that vectors do not divide ----------------------------------------
// The same for small samples of any C: the slab is all channels, a sample one run of
// memory, and vectors straddle pixels (Part's layout, without pixel ranges), at any
// alignment.  Thread t's i-th vector: elements left - i dec of the sample from it on.
// Bound by latency (a load, the joins in LDS) up to about a workgroup a CU: 32
// samples of 784 x 6 in bf16 take 9.0 us forward and 12.2 backward, 18 backward with
// a thread to a channel in the join, 11 and 25 read twice; above by memory (2048
// samples of 240 x 30 in f32 22 and 53 us, 5.4 and 3.3 TB/s).
template <int kType, int kR, int kS>
struct Flat {
  static constexpr int kN = Elem<kType>::kVec;
  typedef typename Elem<kType>::T T;
  Vals<kType, kN> v[kR][kS];

  // No load lies under a branch, so that all are on their way together: a vector
  // that passes the sample's end is read where its last whole one is, and the values
  // that are its own are shifted to the front.  (A sample has a vector at least.)
  __device__ __forceinline__ Flat(const GroupNormDev& d, const Part<kN>& w, const void* a,
                                  const void* b = nullptr) {
    const void* src[2] = {a, b};
    typedef unsigned int Raw __attribute__((ext_vector_type(4), aligned(2)));
    Raw raw[kR][kS];
    const int64_t last = (w.n + 1) * d.P * d.C - kN;
#pragma unroll
    for (int i = 0; i < kR; ++i) {
      const int64_t at = min(w.first + i * w.stride, last);
#pragma unroll
      for (int q = 0; q < kS; ++q)
        raw[i][q] = *reinterpret_cast<const Raw*>(static_cast<const T*>(src[q]) + at);
    }
#pragma unroll
    for (int i = 0; i < kR; ++i) {
      const int n = left(w, i);
#pragma unroll
      for (int q = 0; q < kS; ++q) {
        unsigned __int128 bits;
        __builtin_memcpy(&bits, &raw[i][q], 16);
        if (n < kN) bits = n > 0 ? bits >> (kN - n) * 8 * (int)sizeof(T) : 0;
        __builtin_memcpy(v[i][q].v, &bits, 16);
      }
    }
  }
  // elements of the i-th vector that are the sample's
  static __device__ __forceinline__ int left(const Part<kN>& w, int i) {
    return (int)max((int64_t)0, min(w.left - i * w.dec, (int64_t)kN));
  }
};

// Grid: K N workgroups.
template <int kType, int kAct, int kR>
__global__ __launch_bounds__(kHeldThreads) void k_gn_fwd_flat(GroupNormDev d,
                                                              const void* __restrict__ x,
                                                              const float* __restrict__ gamma,
                                                              const float* __restrict__ beta,
                                                              int64_t ld, void* __restrict__ y,
                                                              float* __restrict__ mean,
                                                              float* __restrict__ rstd) {
  constexpr int kN = Elem<kType>::kVec;
  const Part<kN> w(d, blockIdx.x);
  Flat<kType, kR, 1> in(d, w, x);
  float mu[kN], sc[kN], sh[kN];
  w.channels(d, [&](int j, int c, int) {
    sc[j] = gamma[w.k * ld + c];
    sh[j] = beta[w.k * ld + c];
  });
  double a0[kN] = {}, a1[kN] = {};
#pragma unroll
  for (int i = 0; i < kR; ++i) {
#pragma unroll
    for (int j = 0; j < kN; ++j) {  // (past the sample's end: 0)
      const double f = in.v[i][0][j];
      a0[j] += f;
      a1[j] = __builtin_fma(f, f, a1[j]);
    }
  }
  double2* table = reinterpret_cast<double2*>(dyn_lds);
  int places = w.active;
  const int place = fold_place(w.period, places);
  Stats* st = reinterpret_cast<Stats*>(table + places * kN);
  fold_lanes(a0, a1, w.period);
  if (place >= 0) {
#pragma unroll
    for (int j = 0; j < kN; ++j) table[place * kN + j] = make_double2(a0[j], a1[j]);
  }
  __syncthreads();
  const double inv_m = 1.0 / ((double)d.P * d.Cg);
  join_sums(d.G, places * kN / d.C * d.Cg, [&](int g, int q) {
    return table[q / d.Cg * d.C + g * d.Cg + q % d.Cg];
  }, [&](int g, double2 s) {
    const Stats r = stats_of(s.x, s.y, inv_m, d.eps);
    st[g] = r;
    mean[w.n * d.G + g] = r.mean;
    rstd[w.n * d.G + g] = r.rstd;
  });
  __syncthreads();
  w.channels(d, [&](int j, int, int g) {
    const Stats r = st[g];
    mu[j] = r.mean;
    sc[j] = r.rstd * sc[j];
    sh[j] = __builtin_fmaf(-r.rest, sc[j], sh[j]);
  });
  typedef typename Elem<kType>::T T;
#pragma unroll
  for (int i = 0; i < kR; ++i) {
    const int n = Flat<kType, kR, 1>::left(w, i);
    auto v = in.v[i][0];
#pragma unroll
    for (int j = 0; j < kN; ++j)
      v.set(j, act_of<kAct>(__builtin_fmaf(v[j] - mu[j], sc[j], sh[j])));
    T* p = static_cast<T*>(y) + w.first + i * w.stride;
    if (n == kN) v.store(p); else v.store(p, n);
  }
}

// Grid: K N workgroups.
template <int kType, int kAct, int kR>
__global__ __launch_bounds__(kHeldThreads) void k_gn_bwd_flat(GroupNormDev d,
                                                              const void* __restrict__ dy,
                                                              const void* __restrict__ x,
                                                              const float* __restrict__ gamma,
                                                              const float* __restrict__ beta,
                                                              int64_t ld,
                                                              const float* __restrict__ mean,
                                                              const float* __restrict__ rstd,
                                                              void* __restrict__ dx,
                                                              float* __restrict__ dgamma,
                                                              float* __restrict__ dbeta,
                                                              int64_t ldg) {
  constexpr int kN = Elem<kType>::kVec;
  const Part<kN> w(d, blockIdx.x);
  Flat<kType, kR, 2> in(d, w, x, dy);
  float mu[kN], rs[kN], gs[kN], be[kN], k1[kN], k2[kN];
  w.channels(d, [&](int j, int c, int g) {
    mu[j] = mean[w.n * d.G + g];
    rs[j] = rstd[w.n * d.G + g];
    gs[j] = gamma[w.k * ld + c] * rs[j];
    be[j] = beta[w.k * ld + c];
  });
  float a[kN] = {}, b[kN] = {};
  float dz[kR][kN];
#pragma unroll
  for (int i = 0; i < kR; ++i) {
    const int n = Flat<kType, kR, 2>::left(w, i);
#pragma unroll
    for (int j = 0; j < kN; ++j) {
      const float u = in.v[i][0][j] - mu[j];
      const float q = act_back<kAct>(in.v[i][1][j], __builtin_fmaf(u, gs[j], be[j]));
      dz[i][j] = q;
      if (j < n) {
        a[j] = __builtin_fmaf(q, u, a[j]);
        b[j] += q;
      }
    }
  }
  // element f of the threads' sums side by side belongs to channel f mod C
  float2* table = reinterpret_cast<float2*>(dyn_lds);
  int places = w.active;
  const int place = fold_place(w.period, places);
  const int elems = places * kN;
  double2* sums = reinterpret_cast<double2*>(table + elems);
  float2* st = reinterpret_cast<float2*>(sums + d.C);
  fold_lanes(a, b, w.period);
  if (place >= 0) {
#pragma unroll
    for (int j = 0; j < kN; ++j) table[place * kN + j] = make_float2(a[j], b[j]);
  }
  __syncthreads();
  float2* part = reinterpret_cast<float2*>(d.part) + w.n * d.C;
  join_sums(d.C, elems / d.C, [&](int c, int q) {
    const float2 v = table[q * d.C + c];
    return make_double2((double)v.x, (double)v.y);
  }, [&](int c, double2 s) {
    s.x *= (double)rstd[w.n * d.G + c / d.Cg];
    if (d.N > 1) {
      part[c] = make_float2((float)s.x, (float)s.y);
    } else {
      dgamma[w.k * ldg + c] = (float)s.x;
      dbeta[w.k * ldg + c] = (float)s.y;
    }
    const double f = gamma[w.k * ld + c];
    sums[c] = make_double2(f * s.x, f * s.y);
  });
  __syncthreads();
  const double inv_m = 1.0 / ((double)d.P * d.Cg);
  join_sums(d.G, d.Cg, [&](int g, int i) { return sums[g * d.Cg + i]; },
            [&](int g, double2 s) {
    st[g] = make_float2((float)(s.y * inv_m), (float)(s.x * inv_m));
  });
  __syncthreads();
  // dx = gamma rstd dz - rstd s1 - ((x - mean) rstd) (rstd s2)
  w.channels(d, [&](int j, int, int g) {
    k1[j] = rs[j] * st[g].x;
    k2[j] = rs[j] * st[g].y;
  });
  typedef typename Elem<kType>::T T;
#pragma unroll
  for (int i = 0; i < kR; ++i) {
    const int n = Flat<kType, kR, 2>::left(w, i);
    auto v = in.v[i][0];
#pragma unroll
    for (int j = 0; j < kN; ++j) {
      const float h = (v[j] - mu[j]) * rs[j];
      v.set(j, __builtin_fmaf(gs[j], dz[i][j], -__builtin_fmaf(h, k2[j], k1[j])));
    }
    T* p = static_cast<T*>(dx) + w.first + i * w.stride;
    if (n == kN) v.store(p); else v.store(p, n);
  }
}

// Grid: K ceil(C / 64) workgroups of up to kParamWaves waves.
__global__ __launch_bounds__(kParamWaves* kWave) void k_gn_params(GroupNormDev d,
                                                                  float* __restrict__ dgamma,
                                                                  float* __restrict__ dbeta,
                                                                  int64_t ldg) {
  param_sums(d, 1, blockIdx.x, dgamma, dbeta, ldg);
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

// The same for the one-pass kernels: f(type, act, vectors of a thread, one).
template <typename F>
hipError_t dispatch_held(int dtype, int act, int r, bool one, F&& f) {
  auto with_one = [&](auto type, auto a, auto n) {
    if (one) f(type, a, n, std::true_type());
    else f(type, a, n, std::false_type());
  };
  auto with_r = [&](auto type, auto a) {
    if (r == 16) with_one(type, a, std::integral_constant<int, 16>());
    else if (r == 8) with_one(type, a, std::integral_constant<int, 8>());
    else with_one(type, a, std::integral_constant<int, 4>());
  };
  auto with_act = [&](auto type) {
    if (act == kActRelu) with_r(type, std::integral_constant<int, kActRelu>());
    else if (act == kActSilu) with_r(type, std::integral_constant<int, kActSilu>());
    else with_r(type, std::integral_constant<int, kActNone>());
  };
  if (dtype == kF32) with_act(std::integral_constant<int, kF32>());
  else if (dtype == kBF16) with_act(std::integral_constant<int, kBF16>());
  else with_act(std::integral_constant<int, kF16>());
  return hipGetLastError();
}

// f(type, act, vectors of a thread) for the kernels of any C.
template <typename F>
hipError_t dispatch_flat(int dtype, int act, int r, F&& f) {
  auto with_r = [&](auto type, auto a) {
    if (r == 8) f(type, a, std::integral_constant<int, 8>());
    else f(type, a, std::integral_constant<int, 4>());
  };
  auto with_act = [&](auto type) {
    if (act == kActRelu) with_r(type, std::integral_constant<int, kActRelu>());
    else if (act == kActSilu) with_r(type, std::integral_constant<int, kActSilu>());
    else with_r(type, std::integral_constant<int, kActNone>());
  };
  if (dtype == kF32) with_act(std::integral_constant<int, kF32>());
  else if (dtype == kBF16) with_act(std::integral_constant<int, kBF16>());
  else with_act(std::integral_constant<int, kF16>());
  return hipGetLastError();
}

// Places in LDS of the two-pass sums (the last slab may be narrower than the
// others).
int places(const GroupNormDev& d) {
  auto of = [&](int cw) { return table_places(kBlock, cw / std::min(d.vec, cw & -cw)); };
  return std::max(of(d.slab), of(d.C - (d.slabs - 1) * d.slab));
}

bool aligned16(const void* a, const void* b, const void* c) {
  return ((reinterpret_cast<uintptr_t>(a) | reinterpret_cast<uintptr_t>(b) |
           reinterpret_cast<uintptr_t>(c)) & 15u) == 0;
}

// The shape with a workgroup to a sample.
GroupNormDev whole_samples(const GroupNormDev& d) {
  GroupNormDev h = d;
  h.slab = d.C;
  h.slabs = 1;
  h.splits = 1;
  h.split_pixels = d.P;
  return h;
}

}  // namespace

size_t group_norm_held_lds(const GroupNormDev& d, const GroupNormHeld& held, int dtype,
                           bool back) {
  const int vec = 16 / dtype_bytes(dtype), groups = held.slab / d.Cg;
  if (d.C % vec != 0) {
    const int period = d.C / std::min(vec, d.C & -d.C);
    const size_t at = folds(period) ? (size_t)table_places(held.threads, period)
                                    : (size_t)(held.threads / period * period);
    return back ? at * vec * sizeof(float2) + (size_t)d.C * sizeof(double2) +
                      groups * sizeof(float2)
                : at * vec * sizeof(double2) + groups * sizeof(Stats);
  }
  const int last = d.C - (held.slabs - 1) * held.slab;  // channels of the last slab
  const size_t at = (size_t)std::max(table_places(held.threads, held.slab / vec),
                                     table_places(held.threads, last / vec));
  if (back)
    return at * vec * 2 * sizeof(float) + (size_t)held.slab * 2 * sizeof(double) +
           groups * sizeof(float2);
  return at * (d.Cg % vec == 0 ? 1 : vec) * sizeof(double2) + groups * sizeof(Stats);
}

hipError_t launch_group_norm_forward(const GroupNormDev& d, const GroupNormHeld& held, int dtype,
                                     int act, const void* x, const float* gamma,
                                     const float* beta, int64_t ld, void* y, float* mean,
                                     float* rstd, hipStream_t s) {
  const LaunchEvents ev;
  if (held.threads > 0 && d.C % (16 / dtype_bytes(dtype)) != 0) {
    const GroupNormDev h = whole_samples(d);
    const size_t lds = group_norm_held_lds(d, held, dtype, false);
    const dim3 grid((unsigned)(d.K * d.N)), block((unsigned)held.threads);
    return dispatch_flat(dtype, act, held.vectors, [&](auto type, auto a, auto r) {
      constexpr int T = decltype(type)::value, A = decltype(a)::value, R = decltype(r)::value;
      SAEF_LAUNCH((k_gn_fwd_flat<T, A, R>), grid, block, lds, s, h, x, gamma, beta, ld, y, mean,
                  rstd);
    });
  }
  // (16-byte buffer accesses need their alignment; the two passes take any)
  if (held.threads > 0 && aligned16(x, y, nullptr)) {
    GroupNormDev h = d;
    h.slab = held.slab;
    h.slabs = held.slabs;
    const bool one = d.Cg % (16 / dtype_bytes(dtype)) == 0;
    const size_t lds = group_norm_held_lds(d, held, dtype, false);
    const dim3 grid((unsigned)(d.K * d.N * h.slabs)), block((unsigned)held.threads);
    return dispatch_held(dtype, act, held.vectors, one, [&](auto type, auto a, auto r, auto o) {
      constexpr int T = decltype(type)::value, A = decltype(a)::value, R = decltype(r)::value;
      constexpr bool O = decltype(o)::value;
      SAEF_LAUNCH((k_gn_fwd_held<T, A, R, O>), grid, block, lds, s, h, x, gamma, beta, ld, y, mean,
                  rstd);
    });
  }
  const dim3 grid((unsigned)(d.K * d.N * d.slabs * d.splits)), block(kBlock);
  const bool one = d.vec > 1 && d.C % d.vec == 0 && d.Cg % d.vec == 0;
  const size_t lds = (size_t)places(d) * (one ? 1 : d.vec) * sizeof(double2);
  const size_t stats = ((size_t)d.slab / d.Cg + 2) * sizeof(Stats);
  return dispatch(dtype, d.vec, act, [&](auto type, auto n, auto a) {
    constexpr int T = decltype(type)::value, V = decltype(n)::value, A = decltype(a)::value;
    if (one) SAEF_LAUNCH((k_gn_fwd_sums<T, V, true>), grid, block, lds, s, d, x);
    else SAEF_LAUNCH((k_gn_fwd_sums<T, V, false>), grid, block, lds, s, d, x);
    SAEF_LAUNCH((k_gn_fwd_apply<T, V, A>), grid, block, stats, s, d, x, gamma, beta, ld, y, mean,
                rstd);
  });
}

hipError_t launch_group_norm_backward(const GroupNormDev& d, const GroupNormHeld& held, int dtype,
                                      int act, const void* dy, const void* x, const float* gamma,
                                      const float* beta, int64_t ld, const float* mean,
                                      const float* rstd, void* dx, float* dgamma, float* dbeta,
                                      int64_t ldg, hipStream_t s) {
  const LaunchEvents ev;
  const unsigned params = (unsigned)d.K * (unsigned)((d.C + kWave - 1) / kWave);
  const bool flat = d.C % (16 / dtype_bytes(dtype)) != 0;
  if (held.threads > 0 && (flat || aligned16(x, dy, dx))) {
    const size_t lds = group_norm_held_lds(d, held, dtype, true);
    const dim3 block((unsigned)held.threads);
    hipError_t err;
    if (flat) {
      const GroupNormDev h = whole_samples(d);
      err = dispatch_flat(dtype, act, held.vectors, [&](auto type, auto a, auto r) {
        constexpr int T = decltype(type)::value, A = decltype(a)::value, R = decltype(r)::value;
        SAEF_LAUNCH((k_gn_bwd_flat<T, A, R>), dim3((unsigned)(d.K * d.N)), block, lds, s, h, dy, x,
                    gamma, beta, ld, mean, rstd, dx, dgamma, dbeta, ldg);
      });
    } else {
      GroupNormDev h = d;
      h.slab = held.slab;
      h.slabs = held.slabs;
      const bool one = d.Cg % (16 / dtype_bytes(dtype)) == 0;
      const dim3 grid((unsigned)(d.K * d.N * h.slabs));
      err = dispatch_held(dtype, act, held.vectors, one, [&](auto type, auto a, auto r, auto o) {
        constexpr int T = decltype(type)::value, A = decltype(a)::value, R = decltype(r)::value;
        constexpr bool O = decltype(o)::value;
        if constexpr (R <= 8)  // (16 do not fit the registers and are never chosen)
          SAEF_LAUNCH((k_gn_bwd_held<T, A, R, O>), grid, block, lds, s, h, dy, x, gamma, beta, ld,
                      mean, rstd, dx, dgamma, dbeta, ldg);
      });
    }
    if (err != hipSuccess || d.N == 1) return err;
    // four rows a wave, on their way together
    const int waves = (int)std::min<int64_t>(kParamWaves, (d.N + 3) / 4);
    SAEF_LAUNCH(k_gn_params, dim3(params), dim3((unsigned)(waves * kWave)),
                (size_t)(waves * kWave) * sizeof(double2), s, d, dgamma, dbeta, ldg);
    return hipGetLastError();
  }
  const unsigned parts = (unsigned)(d.K * d.N * d.slabs * d.splits);
  const size_t lds = ((size_t)places(d) * d.vec + 1) * sizeof(float2) +
                     (size_t)d.slab * sizeof(double2);
  const size_t apply_lds = std::max(((size_t)d.slab / d.Cg + 2) * sizeof(float2),
                                    (size_t)kBlock * sizeof(double2));
  return dispatch(dtype, d.vec, act, [&](auto type, auto n, auto a) {
    constexpr int T = decltype(type)::value, V = decltype(n)::value, A = decltype(a)::value;
    SAEF_LAUNCH((k_gn_bwd_sums<T, V, A>), dim3(parts), dim3(kBlock), lds, s, d, x, dy, gamma, beta,
                ld, mean, rstd);
    SAEF_LAUNCH((k_gn_bwd_apply<T, V, A>), dim3(params + parts), dim3(kBlock), apply_lds, s, d, dy,
                x, gamma, beta, ld, mean, rstd, dx, dgamma, dbeta, ldg, params);
  });
}

}  // namespace saef
