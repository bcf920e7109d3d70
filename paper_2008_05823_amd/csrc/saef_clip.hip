// Global gradient norms of K workers over many tensors, and clipping.
//
//   norm_k = sqrt(sum_i g_ki^2)   or   max_i |g_ki|
//   c_k    = min(1, max_norm / (norm_k + 1e-6)),   g_k <- c_k g_k
//
// Both are bound by memory: a gradient is read once for its norm and once
// more to be scaled.  The products of two fp32 (or 16-bit) values are exact
// in binary64 and are summed there, so squares neither overflow nor vanish;
// the sums are taken in one fixed order (lanes, tiles of a tensor, tensors),
// so results are the same from run to run.  A wave takes one tile of one
// worker: partials need no barrier and no atomics.
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
  __device__ __forceinline__ double wave() {
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

constexpr int kGU = 8;  // 16-byte loads of a wave in flight

// Grid: K runs of ceil(n_tiles / 4) workgroups, a wave per (worker, tile).
template <int kType, bool kInf>
__global__ __launch_bounds__(kBlock) void k_grad_tiles(DevLayout lay, GradsDev g) {
  const unsigned per = (unsigned)((lay.n_tiles + kWaves - 1) / kWaves);
  const int k = (int)(blockIdx.x / per);
  const int64_t ti = (int64_t)(blockIdx.x % per) * kWaves + wave_id();
  if (ti >= lay.n_tiles) return;
  const int lane = lane_id();
  const Span<kType> sp(lay, g, k, lay.tiles[ti]);
  typedef Elem<kType> E;
  const Buf b = sp.body();
  Acc<kInf> acc;
  for (int v0 = 0; v0 < sp.nvec; v0 += kGU * kWave) {
    u32x4 raw[kGU];
#pragma unroll
    for (int u = 0; u < kGU; ++u)
      raw[u] = __builtin_amdgcn_raw_buffer_load_b128(b, (v0 + u * kWave + lane) * 16, 0, kAuxNT);
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
  const double s = acc.wave();
  if (lane == 0) g.part[(int64_t)k * lay.n_tiles + ti] = s;
}

// The sum (or the largest) of v[0..n) over the workgroup, in thread 0.
template <bool kInf>
__device__ double block_join(const double* __restrict__ v, int64_t n) {
  __shared__ double s_v[kWaves];
  double a = 0.0;
  // a NaN stays: of two values the larger, unless one is no number
  auto join = [](double p, double q) { return kInf ? (p >= q || p != p ? p : q) : p + q; };
  for (int64_t i = threadIdx.x; i < n; i += kBlock) a = join(a, v[i]);
#pragma unroll
  for (int o = kWave / 2; o > 0; o >>= 1) a = join(a, __shfl_xor(a, o));
  if (lane_id() == 0) s_v[wave_id()] = a;
  __syncthreads();
  a = s_v[0];
  for (int i = 1; i < kWaves; ++i) a = join(a, s_v[i]);
  return a;
}

template <bool kInf>
__device__ __forceinline__ float norm_of(double s) {
  return (float)(kInf ? s : sqrt(s));
}

// Grid: K L workgroups, one per (worker, tensor).
template <bool kInf>
__global__ __launch_bounds__(kBlock) void k_grad_tensors(DevLayout lay, GradsDev g,
                                                         float* __restrict__ tensor_norms) {
  const int l = (int)(blockIdx.x % (unsigned)lay.L), k = (int)(blockIdx.x / (unsigned)lay.L);
  const TensorInfo t = lay.tensors[l];
  const double s = block_join<kInf>(g.part + (int64_t)k * lay.n_tiles + t.first_tile, t.ntiles);
  if (threadIdx.x != 0) return;
  g.tpart[blockIdx.x] = s;
  if (tensor_norms != nullptr) tensor_norms[blockIdx.x] = norm_of<kInf>(s);
}

// Grid: K workgroups.
template <bool kInf>
__global__ __launch_bounds__(kBlock) void k_grad_norms(DevLayout lay, GradsDev g,
                                                       float* __restrict__ norms) {
  const double s = block_join<kInf>(g.tpart + (int64_t)blockIdx.x * lay.L, lay.L);
  if (threadIdx.x == 0) norms[blockIdx.x] = norm_of<kInf>(s);
}

// c v in the gradient's own type.  The product is rounded to fp32 first, in every
// instruction the compiler may choose (its fused forms for fp16 round once).
template <int kType>
__device__ __forceinline__ typename Elem<kType>::T scaled(typename Elem<kType>::T v, float c) {
  float f = Elem<kType>::to_f32(v) * c;
  if (kType == kF16) asm("" : "+v"(f));
  return Elem<kType>::of_f32(f);
}

// Grid: as k_grad_tiles.  kRows: into the fp32 rows of the layout.
template <int kType, bool kRows>
__global__ __launch_bounds__(kBlock) void k_clip(DevLayout lay, GradsDev g, float max_norm,
                                                 const float* __restrict__ norms,
                                                 float* __restrict__ out) {
  const unsigned per = (unsigned)((lay.n_tiles + kWaves - 1) / kWaves);
  const int k = (int)(blockIdx.x / per);
  const int64_t ti = (int64_t)(blockIdx.x % per) * kWaves + wave_id();
  const float c = clip_factor(max_norm, norms[k]);
  if (!kRows && c == 1.0f) return;  // in place, v * 1 is v
  if (ti >= lay.n_tiles) return;
  const int lane = lane_id();
  const Tile tile = lay.tiles[ti];
  const Span<kType> sp(lay, g, k, tile);
  typedef Elem<kType> E;
  typedef typename E::T T;
  const Buf b = sp.body();
  float* row = kRows ? out + (int64_t)k * lay.d_pad + tile.start : nullptr;
  for (int v0 = 0; v0 < sp.nvec; v0 += kGU * kWave) {
    u32x4 raw[kGU];
#pragma unroll
    for (int u = 0; u < kGU; ++u)
      raw[u] = __builtin_amdgcn_raw_buffer_load_b128(b, (v0 + u * kWave + lane) * 16, 0, kAuxNT);
#pragma unroll
    for (int u = 0; u < kGU; ++u) {
      const int i = v0 + u * kWave + lane;
      T v[E::kVec];
      __builtin_memcpy(v, &raw[u], 16);
      if (kRows) {
        if (i < sp.nvec) {
#pragma unroll
          for (int j = 0; j < E::kVec; ++j)
            st_nt(row + sp.head + i * E::kVec + j, E::to_f32(v[j]) * c);
        }
      } else {
#pragma unroll
        for (int j = 0; j < E::kVec; ++j) v[j] = scaled<kType>(v[j], c);
        __builtin_memcpy(&raw[u], v, 16);
        __builtin_amdgcn_raw_buffer_store_b128(raw[u], b, i * 16, 0, kAuxNT);
      }
    }
  }
  const int tail0 = sp.head + sp.nvec * E::kVec;
  if (lane < sp.head) {
    const T v = sp.p[lane];
    if (kRows) row[lane] = E::to_f32(v) * c; else sp.p[lane] = scaled<kType>(v, c);
  }
  if (lane < sp.tail) {
    const T v = sp.p[tail0 + lane];
    if (kRows) row[tail0 + lane] = E::to_f32(v) * c; else sp.p[tail0 + lane] = scaled<kType>(v, c);
  }
}

}  // namespace

hipError_t launch_grad_norm(const DevLayout& lay, const GradsDev& g, bool inf, float* norms,
                            float* tensor_norms, hipStream_t s) {
  const LaunchEvents ev;
  const dim3 tiles(per_wave_grid(lay) * (unsigned)g.K), tens((unsigned)g.K * (unsigned)lay.L);
#define SAEF_GN(T, I) SAEF_LAUNCH((k_grad_tiles<T, I>), tiles, dim3(kBlock), 0, s, lay, g)
  if (g.dtype == kF32) { if (inf) SAEF_GN(kF32, true); else SAEF_GN(kF32, false); }
  else if (g.dtype == kBF16) { if (inf) SAEF_GN(kBF16, true); else SAEF_GN(kBF16, false); }
  else { if (inf) SAEF_GN(kF16, true); else SAEF_GN(kF16, false); }
#undef SAEF_GN
  if (inf) {
    SAEF_LAUNCH(k_grad_tensors<true>, tens, dim3(kBlock), 0, s, lay, g, tensor_norms);
    SAEF_LAUNCH(k_grad_norms<true>, dim3(g.K), dim3(kBlock), 0, s, lay, g, norms);
  } else {
    SAEF_LAUNCH(k_grad_tensors<false>, tens, dim3(kBlock), 0, s, lay, g, tensor_norms);
    SAEF_LAUNCH(k_grad_norms<false>, dim3(g.K), dim3(kBlock), 0, s, lay, g, norms);
  }
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
