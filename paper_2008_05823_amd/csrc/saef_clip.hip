// Global gradient norms of K workers over many tensors, and clipping.
//
//   norm_k = sqrt(sum_i g_ki^2)   or   max_i |g_ki|
//   c_k    = min(1, max_norm / (norm_k + 1e-6)),   g_k <- c_k g_k
//
// Both are bound by memory: a gradient is read once for its norm and once
// more to be scaled.  The products of two fp32 (or 16-bit) values are exact
// in binary64 and are summed there, so squares neither overflow nor vanish;
// the sums are taken in one fixed order (lanes, tiles of a run, runs), so results
// are the same from run to run.  A wave takes a run of tiles of one worker: partials need
// no barrier and no atomics.
//
// Measured: norms of 8 rows of 2^28 1.25 ms (6.9 TB/s); bert_base in bf16, 4 workers,
// norms 150 us (5.9 TB/s, left in the last-level cache) and clipping into rows 411 us
// (6.4 TB/s).
#include <hip/hip_ext.h>

#include "saef_clip.h"
#include "saef_device.h"

namespace saef {
namespace {

// A tile of a gradient tensor at any alignment of its elements: `head`
// elements up to the first 16-byte boundary, `nvec` whole 16-byte vectors,
// `tail` elements.
template <int kType>
struct Span {
  typedef typename Elem<kType>::T T;
  T* p;
  int head, nvec, tail;

  __device__ __forceinline__ Span(const DevLayout& lay, const GradsDev& g, int k,
                                  const Tile& tile) {
    p = static_cast<T*>(g.ptr[(int64_t)k * lay.L + tile.l]) +
        (tile.start - lay.tensors[tile.l].off);
    const int mis = (int)(reinterpret_cast<uintptr_t>(p) & 15u);
    head = min(tile.count, ((16 - mis) & 15) / (int)sizeof(T));
    nvec = (tile.count - head) / Elem<kType>::kVec;
    tail = tile.count - head - nvec * Elem<kType>::kVec;
  }
  __device__ __forceinline__ Buf body() const { return buf_of(p + head, (uint32_t)nvec * 16u); }
  __device__ __forceinline__ const T* tail_at() const {
    return p + head + nvec * Elem<kType>::kVec;
  }
};

// Largest magnitude as the bits of |v|: NaN is above every number.
template <bool kInf>
struct Acc {
  double s = 0.0;
  uint32_t m = 0;
  __device__ __forceinline__ void add(float v) {
    if (kInf) {
      m = max(m, __float_as_uint(v) & 0x7fffffffu);
    } else {
      s = __builtin_fma((double)v, (double)v, s);
    }
  }
  __device__ __forceinline__ void join(const Acc& o) {
    s += o.s;
    m = max(m, o.m);
  }
  __device__ __forceinline__ double wave() const { return Acc(*this).fold(); }
  __device__ __forceinline__ double fold() {
    if (kInf) {
#pragma unroll
      for (int o = kWave / 2; o > 0; o >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, o));
      return (double)__uint_as_float(m);
    }
#pragma unroll
    for (int o = kWave / 2; o > 0; o >>= 1) s += __shfl_xor(s, o);
    return s;
  }
};

constexpr int kFinWaves = 4;    // of a workgroup that joins sums
constexpr int kSmallWaves = 16;  // of one that takes a worker's whole gradient

constexpr int kGU = 8;  // 16-byte loads of a wave in flight

// The run of tiles [first, last) and the worker of this wave.  Grid: K times
// ceil(runs / 4) workgroups, worker by worker, a wave per run.
struct Run {
  int k;
  int64_t run, first, last;
  __device__ __forceinline__ Run(const DevLayout& lay, const GradsDev& g, unsigned block) {
    const unsigned per = (unsigned)((g.runs + kWaves - 1) / kWaves);
    k = (int)(block / per);
    run = (int64_t)(block % per) * kWaves + wave_id();
    first = run * g.run_tiles;
    last = min(first + g.run_tiles, lay.n_tiles);
  }
};

// The wave's tile into acc.
template <int kType, bool kInf, int kAux>
__device__ __forceinline__ void add_tile(const Span<kType>& sp, Acc<kInf>& acc) {
  typedef Elem<kType> E;
  const int lane = lane_id();
  const Buf b = sp.body();
  for (int v0 = 0; v0 < sp.nvec; v0 += kGU * kWave) {
    u32x4 raw[kGU];
#pragma unroll
    for (int u = 0; u < kGU; ++u)
      raw[u] = __builtin_amdgcn_raw_buffer_load_b128(b, (v0 + u * kWave + lane) * 16, 0, kAux);
#pragma unroll
    for (int u = 0; u < kGU; ++u) {
      typename E::T v[E::kVec];
      __builtin_memcpy(v, &raw[u], 16);
#pragma unroll
      for (int j = 0; j < E::kVec; ++j) acc.add(E::to_f32(v[j]));
    }
  }
  if (lane < sp.head) acc.add(E::to_f32(sp.p[lane]));
  if (lane < sp.tail) acc.add(E::to_f32(sp.tail_at()[lane]));
}

// A wave adds up its run tile by tile.  The run's sum goes to runs[k][run]; where
// tensor sums are asked for, the part of each tensor in the run goes to the slot
// of its first tile there.
template <int kType, bool kInf, bool kTensors, int kAux>
__global__ __launch_bounds__(kBlock) void k_grad_tiles(DevLayout lay, GradsDev g) {
  const Run r(lay, g, blockIdx.x);
  if (r.first >= lay.n_tiles) return;
  const int lane = lane_id();
  Acc<kInf> all, part;
  Tile tile = lay.tiles[r.first];
  int64_t slot = r.first;
  for (int64_t ti = r.first; ti < r.last; ++ti) {
    const Tile next = lay.tiles[min(ti + 1, lay.n_tiles - 1)];
    add_tile<kType, kInf, kAux>(Span<kType>(lay, g, r.k, tile), part);
    if (kTensors && (next.l != tile.l || ti + 1 == r.last)) {
      all.join(part);
      const double s = part.wave();
      if (lane == 0) g.part[(int64_t)r.k * lay.n_tiles + slot] = s;
      part = Acc<kInf>();
      slot = ti + 1;
    }
    tile = next;
  }
  const double s = kTensors ? all.wave() : part.wave();
  if (lane == 0) g.run_sums[r.k * g.runs + r.run] = s;
}

// A NaN stays: of two values the larger, unless one is no number.
template <bool kInf>
__device__ __forceinline__ double joined(double p, double q) {
  return kInf ? (p >= q || p != p ? p : q) : p + q;
}

// The sum (or the largest) of at(0 .. n-1) over the workgroup, in thread 0.
template <bool kInf, int kW, typename At>
__device__ double block_join(int64_t n, At at) {
  __shared__ double s_v[kW];
  double a = 0.0;
#pragma unroll 4
  for (int64_t i = threadIdx.x; i < n; i += kW * kWave) a = joined<kInf>(a, at(i));
#pragma unroll
  for (int o = kWave / 2; o > 0; o >>= 1) a = joined<kInf>(a, __shfl_xor(a, o));
  if (lane_id() == 0) s_v[wave_id()] = a;
  __syncthreads();
  if (threadIdx.x == 0)
    for (int i = 1; i < kW; ++i) a = joined<kInf>(a, s_v[i]);
  return a;
}

template <bool kInf>
__device__ __forceinline__ float norm_of(double s) {
  return (float)(kInf ? s : sqrt(s));
}

// Grid: K workgroups for the workers' norms, then, if asked for, K L for the
// tensors'.
template <bool kInf>
__global__ __launch_bounds__(kFinWaves* kWave) void k_grad_norms(
    DevLayout lay, GradsDev g, float* __restrict__ norms, float* __restrict__ tensor_norms) {
  if (blockIdx.x < (unsigned)g.K) {
    const double* v = g.run_sums + (int64_t)blockIdx.x * g.runs;
    const double s = block_join<kInf, kFinWaves>(g.runs, [&](int64_t i) { return v[i]; });
    if (threadIdx.x == 0) norms[blockIdx.x] = norm_of<kInf>(s);
    return;
  }
  const unsigned b = blockIdx.x - (unsigned)g.K;
  const TensorInfo t = lay.tensors[b % (unsigned)lay.L];
  const double* v = g.part + (int64_t)(b / (unsigned)lay.L) * lay.n_tiles;
  // the tensor's slots: its first tile, and those where a run begins
  const int64_t first = t.first_tile, run = first / g.run_tiles;
  const int64_t n = (first + t.ntiles - 1) / g.run_tiles - run + 1;
  const double s = block_join<kInf, kFinWaves>(
      n, [&](int64_t i) { return v[i == 0 ? first : (run + i) * g.run_tiles]; });
  if (threadIdx.x == 0) tensor_norms[b] = norm_of<kInf>(s);
}

// Small gradients in one launch: a workgroup takes a worker's, its waves tile by
// tile, and joins the tiles' sums from LDS.  Grid: K.
template <int kType, bool kInf>
__global__ __launch_bounds__(kSmallWaves* kWave) void k_grad_small(
    DevLayout lay, GradsDev g, float* __restrict__ norms, float* __restrict__ tensor_norms) {
  __shared__ double s_tile[kSmallTiles];
  const int k = (int)blockIdx.x;
  for (int ti = wave_id(); ti < (int)lay.n_tiles; ti += kSmallWaves) {
    Acc<kInf> acc;
    add_tile<kType, kInf, 0>(Span<kType>(lay, g, k, lay.tiles[ti]), acc);
    const double s = acc.wave();
    if (lane_id() == 0) s_tile[ti] = s;
  }
  __syncthreads();
  if (tensor_norms != nullptr) {
    for (int l = (int)threadIdx.x; l < lay.L; l += kSmallWaves * kWave) {
      const TensorInfo t = lay.tensors[l];
      double a = 0.0;
      for (int i = 0; i < t.ntiles; ++i) a = joined<kInf>(a, s_tile[t.first_tile + i]);
      tensor_norms[(int64_t)k * lay.L + l] = norm_of<kInf>(a);
    }
  }
  const double s =
      block_join<kInf, kSmallWaves>(lay.n_tiles, [&](int64_t i) { return s_tile[i]; });
  if (threadIdx.x == 0) norms[k] = norm_of<kInf>(s);
}

// c v in the gradient's own type.  The product is rounded to fp32 first, in every
// instruction the compiler may choose (its fused forms for fp16 round once).
template <int kType>
__device__ __forceinline__ typename Elem<kType>::T scaled(typename Elem<kType>::T v, float c) {
  float f = Elem<kType>::to_f32(v) * c;
  if (kType == kF16) asm("" : "+v"(f));
  return Elem<kType>::of_f32(f);
}

// A wave takes a tile.  kRows: into the fp32 rows of the layout; a load is then
// as many elements as a 16-byte store, so that a wave's stores are one run of
// memory (bert_base in bf16, K = 4: 450 us, 662 with 16-byte loads and two stores
// apart).  Grid: K times ceil(n_tiles / 4) workgroups.
template <int kType, bool kRows>
__global__ __launch_bounds__(kBlock) void k_clip(DevLayout lay, GradsDev g, float max_norm,
                                                 const float* __restrict__ norms,
                                                 float* __restrict__ out) {
  const unsigned per = (unsigned)((lay.n_tiles + kWaves - 1) / kWaves);
  const int k = (int)(blockIdx.x / per);
  const int64_t ti = (int64_t)(blockIdx.x % per) * kWaves + wave_id();
  if (ti >= lay.n_tiles) return;
  const float c = clip_factor(max_norm, norms[k]);
  if (!kRows && c == 1.0f) return;  // in place, v * 1 is v
  const int lane = lane_id();
  typedef Elem<kType> E;
  typedef typename E::T T;
  const Tile tile = lay.tiles[ti];
  const Span<kType> sp(lay, g, k, tile);
  const Buf b = sp.body();
  const int tail0 = sp.head + sp.nvec * E::kVec;
  float* row = kRows ? out + (int64_t)k * lay.d_pad + tile.start : nullptr;
  if (kRows) {
    // stores at the alignment of an element
    typedef float f32x4 __attribute__((ext_vector_type(4), aligned(4)));
    constexpr int kLd = 4 * (int)sizeof(T);  // bytes of a load
    const int n4 = sp.nvec * (E::kVec / 4);
    for (int v0 = 0; v0 < n4; v0 += kGU * kWave) {
      T v[kGU][4];
#pragma unroll
      for (int u = 0; u < kGU; ++u) {
        const int at = (v0 + u * kWave + lane) * kLd;
        if (kLd == 16) {
          const u32x4 q = __builtin_amdgcn_raw_buffer_load_b128(b, at, 0, kAuxNT);
          __builtin_memcpy(v[u], &q, kLd);
        } else {
          const u32x2 q = __builtin_amdgcn_raw_buffer_load_b64(b, at, 0, kAuxNT);
          __builtin_memcpy(v[u], &q, kLd);
        }
      }
#pragma unroll
      for (int u = 0; u < kGU; ++u) {
        const int i = v0 + u * kWave + lane;
        const f32x4 q = {E::to_f32(v[u][0]) * c, E::to_f32(v[u][1]) * c, E::to_f32(v[u][2]) * c,
                         E::to_f32(v[u][3]) * c};
        if (i < n4)
          __builtin_nontemporal_store(q, reinterpret_cast<f32x4*>(row + sp.head + 4 * i));
      }
    }
    if (lane < sp.head) row[lane] = E::to_f32(sp.p[lane]) * c;
    if (lane < sp.tail) row[tail0 + lane] = E::to_f32(sp.p[tail0 + lane]) * c;
    return;
  }
  for (int v0 = 0; v0 < sp.nvec; v0 += kGU * kWave) {
    u32x4 raw[kGU];
#pragma unroll
    for (int u = 0; u < kGU; ++u)
      raw[u] = __builtin_amdgcn_raw_buffer_load_b128(b, (v0 + u * kWave + lane) * 16, 0, kAuxNT);
#pragma unroll
    for (int u = 0; u < kGU; ++u) {
      T v[E::kVec];
      __builtin_memcpy(v, &raw[u], 16);
#pragma unroll
      for (int j = 0; j < E::kVec; ++j) v[j] = scaled<kType>(v[j], c);
      __builtin_memcpy(&raw[u], v, 16);
      __builtin_amdgcn_raw_buffer_store_b128(raw[u], b, (v0 + u * kWave + lane) * 16, 0, kAuxNT);
    }
  }
  if (lane < sp.head) sp.p[lane] = scaled<kType>(sp.p[lane], c);
  if (lane < sp.tail) sp.p[tail0 + lane] = scaled<kType>(sp.p[tail0 + lane], c);
}

dim3 run_grid(const GradsDev& g) {
  return dim3((unsigned)(g.K * ((g.runs + kWaves - 1) / kWaves)));
}

}  // namespace

hipError_t launch_grad_norm(const DevLayout& lay, const GradsDev& g, bool inf, float* norms,
                            float* tensor_norms, hipStream_t s) {
  const LaunchEvents ev;
  if (g.runs == 0) {
#define SAEF_GN(T, I)                                                                          \
  SAEF_LAUNCH((k_grad_small<T, I>), dim3((unsigned)g.K), dim3(kSmallWaves * kWave), 0, s, lay, g, \
              norms, tensor_norms)
    if (g.dtype == kF32) { if (inf) SAEF_GN(kF32, true); else SAEF_GN(kF32, false); }
    else if (g.dtype == kBF16) { if (inf) SAEF_GN(kBF16, true); else SAEF_GN(kBF16, false); }
    else { if (inf) SAEF_GN(kF16, true); else SAEF_GN(kF16, false); }
#undef SAEF_GN
    return hipGetLastError();
  }
  const dim3 runs = run_grid(g);
  const dim3 fin((unsigned)g.K * (tensor_norms != nullptr ? 1u + (unsigned)lay.L : 1u));
  const bool tensors = tensor_norms != nullptr;
#define SAEF_GN4(T, I, S, A) \
  SAEF_LAUNCH((k_grad_tiles<T, I, S, A>), runs, dim3(kBlock), 0, s, lay, g)
#define SAEF_GN(T, I)                                                                         \
  do {                                                                                        \
    if (g.cached) { if (tensors) SAEF_GN4(T, I, true, 0); else SAEF_GN4(T, I, false, 0); }    \
    else { if (tensors) SAEF_GN4(T, I, true, kAuxNT); else SAEF_GN4(T, I, false, kAuxNT); }   \
  } while (0)
  if (g.dtype == kF32) { if (inf) SAEF_GN(kF32, true); else SAEF_GN(kF32, false); }
  else if (g.dtype == kBF16) { if (inf) SAEF_GN(kBF16, true); else SAEF_GN(kBF16, false); }
  else { if (inf) SAEF_GN(kF16, true); else SAEF_GN(kF16, false); }
#undef SAEF_GN
#undef SAEF_GN4
  const dim3 fb(kFinWaves * kWave);
  if (inf) SAEF_LAUNCH(k_grad_norms<true>, fin, fb, 0, s, lay, g, norms, tensor_norms);
  else SAEF_LAUNCH(k_grad_norms<false>, fin, fb, 0, s, lay, g, norms, tensor_norms);
  return hipGetLastError();
}

hipError_t launch_clip(const DevLayout& lay, const GradsDev& g, float max_norm,
                       const float* norms, float* out, hipStream_t s) {
  const LaunchEvents ev;
  const dim3 tiles(per_wave_grid(lay) * (unsigned)g.K);
#define SAEF_CL(T, R) \
  SAEF_LAUNCH((k_clip<T, R>), tiles, dim3(kBlock), 0, s, lay, g, max_norm, norms, out)
  const bool rows = out != nullptr;
  if (g.dtype == kF32) { if (rows) SAEF_CL(kF32, true); else SAEF_CL(kF32, false); }
  else if (g.dtype == kBF16) { if (rows) SAEF_CL(kBF16, true); else SAEF_CL(kBF16, false); }
  else { if (rows) SAEF_CL(kF16, true); else SAEF_CL(kF16, false); }
#undef SAEF_CL
  return hipGetLastError();
}

}  // namespace saef
