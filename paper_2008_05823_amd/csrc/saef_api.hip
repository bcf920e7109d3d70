// C ABI of the SAEF library: argument checks, the layout object and the
// order in which the kernels of one SAEF iteration are enqueued.
#include <algorithm>
#include <cmath>
#include <cstdint>
#include <cstring>
#include <initializer_list>
#include <mutex>
#include <new>
#include <utility>
#include <vector>

#include "saef.h"
#include "saef_clip.h"
#include "saef_group_norm.h"
#include "saef_internal.h"
#include "saef_topk.h"

using saef::DevLayout;
using saef::TensorInfo;
using saef::Tile;

// Kernel kinds timed by saef_profile_enable (step ahead, compression, worker
// scales, aggregation, server scales, averaging, mismatch).
constexpr int kProfileKinds = 7;

struct saef_layout {
  int device = 0;
  int32_t L = 0;
  int32_t k_max = 0;
  int64_t d_pad = 0;
  std::vector<int64_t> off, n;
  std::vector<TensorInfo> tensors;  // host copy of the tensor table (tiles per tensor)
  DevLayout dev{};
  void* mem_tiles = nullptr;
  void* mem_tensors = nullptr;
  void* mem_part = nullptr;
  void* mem_part2 = nullptr;
  void* mem_status = nullptr;
  // measurement: event pairs recorded around the kernels of saef_round
  std::vector<hipEvent_t> ev_start, ev_stop;
  std::vector<int> ev_kind;
  size_t ev_used = 0;
  uint32_t ev_mask = 0;  // kinds being timed
  int32_t ev_every = 1;  // every ev_every-th dispatch of a timed kind is stamped
  int64_t ev_seen[kProfileKinds] = {};  // dispatches of each kind since enable
};

// A Top-K plan: the kept count of every tensor and the selection scratch.
struct saef_topk {
  const saef_layout* layout = nullptr;
  std::vector<int64_t> keep;
  int64_t total_keep = 0;
  saef::TkDev dev{};
  void* mem_chunks = nullptr;
  void* mem_tens = nullptr;
  void* mem_groups = nullptr;
  void* mem_sgroups = nullptr;
  void* mem_thist = nullptr;
  void* mem_ghist = nullptr;
  void* mem_sghist = nullptr;
  void* mem_sel = nullptr;
  void* mem_tile_cnt = nullptr;
  void* mem_cand = nullptr;
  void* mem_lcnt = nullptr;
  void* mem_rhist = nullptr;
  void* mem_tile_cand = nullptr;
  void* mem_seg = nullptr;
  void* mem_arrived = nullptr;
  void* mem_large = nullptr;
  void* mem_spec = nullptr;
  // the side stream (default priority) and fork/join events of the worker
  // compression's two row groups and of the pipelined iteration end
  saef::TkStreams side{};
  saef::TkPart all{};               // every tensor
  std::vector<saef::TkPart> pipe;   // the iteration end's parts (empty: not pipelined)
};

// Where K workers' gradients lie, and the scratch of their norms.
struct saef_grads {
  const saef_layout* layout = nullptr;
  int32_t K = 0;
  int32_t dtype = 0;
  // the tensors' memory, in order of address (none overlap)
  std::vector<std::pair<uintptr_t, uintptr_t>> spans;
  saef::GradsDev dev{};
  void* mem_ptr = nullptr;
  void* mem_part = nullptr;
  void* mem_runs = nullptr;
};

// The shape of a group norm and the scratch of its sums.
struct saef_group_norm {
  int device = 0;
  int32_t dtype = 0;
  int32_t act = 0;
  saef::GroupNormDev dev{};
  saef::GroupNormHeld fwd{}, bwd{};
  void* mem_part = nullptr;
  void* mem_pieces = nullptr;
};

namespace {

// ---- scratch of the allocation-free iteration (saef_round_noalloc) --------
// The tile partial sums and their second level live in this file-scope
// device array instead of the layout's buffers.  Host code never uses the
// array's name as an address: saef_layout_create looks up its device
// address once per device (hipGetSymbolAddress, with that device current)
// and saef_round_noalloc passes that address to the kernels.
constexpr size_t kScratchBytes = size_t(32) << 20;
constexpr int kMaxDevices = 64;
__device__ __align__(256) unsigned char scratch[kScratchBytes];
std::mutex g_scratch_mu;
void* g_scratch_ptr[kMaxDevices] = {};
bool g_scratch_tried[kMaxDevices] = {};

// Looks up `scratch` on the current device (device `dev`) once.
void scratch_init(int dev) {
  if (dev < 0 || dev >= kMaxDevices) return;
  std::lock_guard<std::mutex> lock(g_scratch_mu);
  if (g_scratch_tried[dev]) return;
  g_scratch_tried[dev] = true;
  void* p = nullptr;
  if (hipGetSymbolAddress(&p, HIP_SYMBOL(scratch)) == hipSuccess) g_scratch_ptr[dev] = p;
}

void* scratch_of(int dev) {
  if (dev < 0 || dev >= kMaxDevices) return nullptr;
  std::lock_guard<std::mutex> lock(g_scratch_mu);
  return g_scratch_ptr[dev];
}

// The parts of the pipelined Top-K iteration end: runs of whole tensors in
// order (SAEF_TK_PARTS of them, fewer when there are fewer tensors; one part
// means no pipeline), cut where the running element count passes the first
// part's share of d (SAEF_TK_FIRST_PCT percent), then equal shares of the
// rest.  At resnet50 K = 8 a 60% share took 836 us per Top-1% iteration and
// 1057 at Top-10%, 55% 844 and 1069, 45% 848 and 1064, 70% 854 against 851 (an
// earlier build); three parts lost (913 against 858).
#ifndef SAEF_TK_PARTS
#define SAEF_TK_PARTS 2
#endif
#ifndef SAEF_TK_FIRST_PCT
#define SAEF_TK_FIRST_PCT 60
#endif
std::vector<saef::TkPart> pipeline_parts(const saef_layout* layout,
                                         const std::vector<saef::TkTensor>& tens) {
  const int32_t L = layout->L;
  const int parts = std::min<int>(SAEF_TK_PARTS, L);
  std::vector<saef::TkPart> out;
  if (parts < 2) return out;
  int64_t d = 0;
  for (int32_t l = 0; l < L; ++l) d += layout->n[l];
  int32_t l0 = 0;
  int64_t cum = 0;
  for (int i = 0; i < parts; ++i) {
    int32_t l1 = l0;
    if (i == parts - 1) {
      l1 = L;
    } else {
      // the running count's target after part i (in parts of 100 * (parts - 1))
      const int64_t first = SAEF_TK_FIRST_PCT * (parts - 1);
      const int64_t target = first + (100 - SAEF_TK_FIRST_PCT) * i;
      // at least one tensor, and one left for each later part
      while (l1 < L - (parts - 1 - i) && (l1 == l0 || cum * 100 * (parts - 1) < d * target))
        cum += layout->n[l1++];
    }
    const saef::TkTensor& a = tens[l0];
    const saef::TkTensor& b = tens[l1 - 1];
    const saef::TensorInfo& ta = layout->tensors[l0];
    const saef::TensorInfo& tb = layout->tensors[l1 - 1];
    out.push_back(saef::TkPart{l0, l1, ta.first_tile, tb.first_tile + tb.ntiles, a.first_group,
                               b.first_group + b.ngroups, a.first_sgroup,
                               b.first_sgroup + b.nsgroups, a.first_chunk,
                               b.first_chunk + b.nchunks, a.large,
                               b.large + (b.ngroups > 0 ? 1 : 0)});
    l0 = l1;
  }
  return out;
}

// Elements per work tile of a tensor of n elements: kTileElems, or more for
// very large tensors so that no tensor has more than kMaxTilesPerTensor tiles
// (bounds the number of partial sums the finalize kernel adds per tensor).
int64_t tile_elems(int64_t n) {
  int64_t t = saef::kTileElems;
  if (n > t * saef::kMaxTilesPerTensor) {
    t = (n + saef::kMaxTilesPerTensor - 1) / saef::kMaxTilesPerTensor;
    t = (t + 63) / 64 * 64;
  }
  return t;
}

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

// [p, p + bytes) and [q, q + qbytes) overlap?
bool overlap(const void* p, size_t bytes, const void* q, size_t qbytes) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(q);
  return a < b + qbytes && b < a + bytes;
}

// [p, p + bytes) shares memory with one of the (non-null) ranges?
struct Range {
  const void* p;
  size_t bytes;
};
bool overlap_any(const void* p, size_t bytes, std::initializer_list<Range> with) {
  for (const Range& r : with)
    if (r.p != nullptr && overlap(p, bytes, r.p, r.bytes)) return true;
  return false;
}

// Largest grid (workgroups in x) a launch may use.
constexpr int64_t kMaxGrid = 2147483647;

int check_common(const saef_layout* lay, int32_t K) {
  if (lay == nullptr) return SAEF_EINVAL;
  if (K < 1 || K > lay->k_max) return SAEF_EINVAL;
  // the per-(tile, worker) grids (tiles rounded up to whole groups of runs)
  // must fit the launch limit
  if (saef::run_padded_tiles(lay->dev.n_tiles * saef::kStepSplit) * (int64_t)K > kMaxGrid)
    return SAEF_EINVAL;
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess) return SAEF_EHIP;
  if (dev != lay->device) return SAEF_EINVAL;
  return SAEF_OK;
}

// What gradients may be clipped to.
bool clip_bound_ok(float max_norm) { return std::isfinite(max_norm) && max_norm >= 0.0f; }

bool f32_ok(const float* p) { return p != nullptr && aligned(p, 4); }
bool u64_ok(const uint64_t* p) { return p != nullptr && aligned(p, 8); }

int hip_rc(hipError_t e) { return e == hipSuccess ? SAEF_OK : SAEF_EHIP; }

void release_events(saef_layout* l) {
  for (hipEvent_t e : l->ev_start) (void)hipEventDestroy(e);
  for (hipEvent_t e : l->ev_stop) (void)hipEventDestroy(e);
  l->ev_start.clear();
  l->ev_stop.clear();
  l->ev_kind.clear();
  l->ev_used = 0;
}

// Launches one kernel of saef_round; while the layout is being profiled and
// an event pair is free, the dispatch stamps its start and end into the pair.
template <typename F>
hipError_t timed(const saef_layout* cl, int kind, F&& launch) {
  saef_layout* l = const_cast<saef_layout*>(cl);
  saef::LaunchEvents ev;
  const bool sel = ((l->ev_mask >> kind) & 1u) != 0;
  const bool rec = sel && l->ev_used < l->ev_start.size() && l->ev_seen[kind] % l->ev_every == 0;
  if (rec) {
    ev.start = l->ev_start[l->ev_used];
    ev.stop = l->ev_stop[l->ev_used];
  }
  hipError_t err = launch(ev);
  if (err != hipSuccess) return err;
  if (sel) ++l->ev_seen[kind];
  if (rec) {
    l->ev_kind[l->ev_used] = kind;
    ++l->ev_used;
  }
  return hipSuccess;
}

void free_layout(saef_layout* l) {
  if (l == nullptr) return;
  release_events(l);
  (void)hipFree(l->mem_tiles);
  (void)hipFree(l->mem_tensors);
  (void)hipFree(l->mem_part);
  (void)hipFree(l->mem_part2);
  (void)hipFree(l->mem_status);
  delete l;
}

void free_topk(saef_topk* p) {
  if (p == nullptr) return;
  if (p->side.stream != nullptr) {
    (void)hipStreamSynchronize(p->side.stream);
    (void)hipStreamDestroy(p->side.stream);
  }
  if (p->side.fork != nullptr) (void)hipEventDestroy(p->side.fork);
  if (p->side.join != nullptr) (void)hipEventDestroy(p->side.join);
  for (void* q : {p->mem_chunks, p->mem_tens, p->mem_groups, p->mem_sgroups, p->mem_thist,
                  p->mem_ghist, p->mem_sghist, p->mem_sel, p->mem_tile_cnt, p->mem_lcnt,
                  p->mem_rhist, p->mem_tile_cand, p->mem_seg, p->mem_arrived, p->mem_large,
                  p->mem_cand, p->mem_spec})
    (void)hipFree(q);
  delete p;
}

}  // namespace

extern "C" {

int saef_layout_create(const int64_t* off, const int64_t* n, int32_t L, int64_t d_pad,
                       int32_t k_max, saef_layout** out) {
  if (out == nullptr) return SAEF_EINVAL;
  *out = nullptr;
  if (off == nullptr || n == nullptr || L < 1 || d_pad < 64 || d_pad % 64 != 0) return SAEF_EINVAL;
  if (k_max < 1 || k_max > 4096) return SAEF_EINVAL;
  // tensors: 64-aligned, non-empty, in range, non-overlapping
  std::vector<int32_t> order(L);
  for (int32_t l = 0; l < L; ++l) {
    if (off[l] < 0 || off[l] % 64 != 0) return SAEF_EINVAL;
    if (n[l] < 1 || n[l] > saef::kMaxTensor) return SAEF_EINVAL;
    if (off[l] > d_pad - n[l]) return SAEF_EINVAL;
    order[l] = l;
  }
  std::sort(order.begin(), order.end(), [&](int32_t a, int32_t b) { return off[a] < off[b]; });
  for (int32_t i = 1; i < L; ++i)
    if (off[order[i - 1]] + n[order[i - 1]] > off[order[i]]) return SAEF_EINVAL;

  saef_layout* lay = new (std::nothrow) saef_layout();
  if (lay == nullptr) return SAEF_EHIP;
  if (hipGetDevice(&lay->device) != hipSuccess) {
    delete lay;
    return SAEF_EHIP;
  }
  scratch_init(lay->device);  // the allocation-free iteration's scratch on this device
  lay->L = L;
  lay->k_max = k_max;
  lay->d_pad = d_pad;
  lay->off.assign(off, off + L);
  lay->n.assign(n, n + L);

  std::vector<Tile> tiles;
  std::vector<TensorInfo> tensors(L);
  for (int32_t l = 0; l < L; ++l) {
    const int64_t te = tile_elems(n[l]);
    const int64_t nt = (n[l] + te - 1) / te;
    tensors[l] = TensorInfo{off[l], n[l], (int32_t)tiles.size(), (int32_t)nt};
    for (int64_t j = 0; j < nt; ++j) {
      const int64_t c = std::min(te, n[l] - j * te);
      tiles.push_back(Tile{off[l] + j * te, l, (int32_t)c});
    }
  }
  const size_t n_rows = (size_t)k_max + 1;
  const size_t part_bytes = n_rows * tiles.size() * 2 * sizeof(unsigned long long);
  int32_t max_tiles = 1;
  for (int32_t l = 0; l < L; ++l) max_tiles = std::max(max_tiles, tensors[l].ntiles);
  const int32_t fin_split = (max_tiles + saef::kFinChunk - 1) / saef::kFinChunk;
  const size_t part2_bytes = n_rows * L * fin_split * 2 * sizeof(unsigned long long);
  hipError_t err = hipSuccess;
  err = hipMalloc(&lay->mem_tiles, tiles.size() * sizeof(Tile));
  if (err == hipSuccess) err = hipMalloc(&lay->mem_tensors, tensors.size() * sizeof(TensorInfo));
  if (err == hipSuccess) err = hipMalloc(&lay->mem_part, part_bytes);
  if (err == hipSuccess) err = hipMalloc(&lay->mem_part2, part2_bytes);
  if (err == hipSuccess) err = hipMalloc(&lay->mem_status, sizeof(int));
  if (err == hipSuccess)
    err = hipMemcpy(lay->mem_tiles, tiles.data(), tiles.size() * sizeof(Tile),
                    hipMemcpyHostToDevice);
  if (err == hipSuccess)
    err = hipMemcpy(lay->mem_tensors, tensors.data(), tensors.size() * sizeof(TensorInfo),
                    hipMemcpyHostToDevice);
  if (err == hipSuccess) err = hipMemset(lay->mem_part, 0, part_bytes);
  if (err == hipSuccess) err = hipMemset(lay->mem_status, 0, sizeof(int));
  if (err == hipSuccess) err = hipDeviceSynchronize();
  if (err != hipSuccess) {
    free_layout(lay);
    return SAEF_EHIP;
  }
  DevLayout& d = lay->dev;
  lay->tensors = tensors;
  d.tiles = static_cast<const Tile*>(lay->mem_tiles);
  d.tensors = static_cast<const TensorInfo*>(lay->mem_tensors);
  d.part = static_cast<unsigned long long*>(lay->mem_part);
  d.part2 = static_cast<unsigned long long*>(lay->mem_part2);
  d.max_tiles = max_tiles;
  d.fin_split = fin_split;
  d.status = static_cast<int*>(lay->mem_status);
  d.n_tiles = (int64_t)tiles.size();
  d.d_pad = d_pad;
  d.L = L;
  d.k_max = k_max;
  *out = lay;
  return SAEF_OK;
}

int saef_layout_destroy(saef_layout* layout) {
  if (layout == nullptr) return SAEF_EINVAL;
  free_layout(layout);
  return SAEF_OK;
}

int saef_layout_info(const saef_layout* layout, int32_t* L, int64_t* d_pad, int32_t* k_max,
                     int64_t* n_tiles) {
  if (layout == nullptr) return SAEF_EINVAL;
  if (L) *L = layout->L;
  if (d_pad) *d_pad = layout->d_pad;
  if (k_max) *k_max = layout->k_max;
  if (n_tiles) *n_tiles = layout->dev.n_tiles;
  return SAEF_OK;
}

}  // extern "C"

namespace {

// saef_compress / saef_compress_momentum (m == nullptr: no momentum).
int compress_impl(const saef_layout* layout, int32_t K, float lr, float mu, const float* g,
                  float* m, float* e, uint64_t* signs, float* scales, hipStream_t stream) {
  int rc = check_common(layout, K);
  if (rc != SAEF_OK) return rc;
  if (!f32_ok(g) || !f32_ok(e) || !u64_ok(signs) || !f32_ok(scales) || !std::isfinite(lr))
    return SAEF_EINVAL;
  const size_t vb = (size_t)K * layout->d_pad * sizeof(float);
  if (overlap(g, vb, e, vb)) return SAEF_EINVAL;
  if (m != nullptr && (!f32_ok(m) || overlap(m, vb, g, vb) || overlap(m, vb, e, vb)))
    return SAEF_EINVAL;
  rc = hip_rc(
      saef::launch_compress(layout->dev, K, lr, mu, g, m, e, signs, scales, false, stream));
  if (rc != SAEF_OK) return rc;
  // e <- Delta - C(Delta); small layouts: the scales as well
  const bool fold = saef::folds_scales(layout->dev, K);
  if (!fold) rc = hip_rc(saef::launch_finalize(layout->dev, K, false, scales, stream));
  if (rc != SAEF_OK) return rc;
  return hip_rc(saef::launch_materialize(layout->dev, K, SAEF_MODE_DC, e, signs, scales, e,
                                         nullptr, nullptr, nullptr, nullptr, nullptr, nullptr,
                                         fold, stream));
}

// [p, p + bytes) shares memory with one of the gradients?
bool meets_grads(const saef_grads* g, const void* p, size_t bytes) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(p);
  // the first gradient that ends after p
  const auto it = std::upper_bound(
      g->spans.begin(), g->spans.end(), a,
      [](uintptr_t v, const std::pair<uintptr_t, uintptr_t>& s) { return v < s.second; });
  return it != g->spans.end() && it->first < a + bytes;
}

bool mu_ok(float mu) { return mu >= 0.0f && mu < 1.0f; }

}  // namespace

extern "C" {

int saef_compress(const saef_layout* layout, int32_t K, float lr, const float* g, float* e,
                  uint64_t* signs, float* scales, hipStream_t stream) {
  return compress_impl(layout, K, lr, 0.0f, g, nullptr, e, signs, scales, stream);
}

int saef_compress_momentum(const saef_layout* layout, int32_t K, float lr, float mu,
                           const float* g, float* m, float* e, uint64_t* signs, float* scales,
                           hipStream_t stream) {
  if (!mu_ok(mu) || m == nullptr) return SAEF_EINVAL;
  return compress_impl(layout, K, lr, mu, g, m, e, signs, scales, stream);
}

int saef_aggregate(const saef_layout* layout, int32_t K, int32_t mode, const uint64_t* signs,
                   const float* scales, float* avg, float* e_srv, uint64_t* srv_signs,
                   float* srv_scales, float* x, hipStream_t stream) {
  int rc = check_common(layout, K);
  if (rc != SAEF_OK) return rc;
  if (mode != SAEF_MODE_SC && mode != SAEF_MODE_DC) return SAEF_EINVAL;
  if (!u64_ok(signs) || !f32_ok(scales) || !f32_ok(x)) return SAEF_EINVAL;
  if (avg != nullptr && !aligned(avg, 4)) return SAEF_EINVAL;
  if (mode == SAEF_MODE_DC && (!f32_ok(e_srv) || !u64_ok(srv_signs) || !f32_ok(srv_scales)))
    return SAEF_EINVAL;
  rc = hip_rc(saef::launch_aggregate(layout->dev, K, mode, signs, const_cast<float*>(scales),
                                     false, avg, e_srv, srv_signs, srv_scales, x, false, stream));
  if (rc != SAEF_OK || mode == SAEF_MODE_SC) return rc;
  // e_srv <- Delta - C(Delta), x <- x - C(Delta); small layouts: the scales as well
  const bool fold = saef::folds_scales(layout->dev, 1);
  if (!fold) rc = hip_rc(saef::launch_finalize(layout->dev, K, true, srv_scales, stream));
  if (rc != SAEF_OK) return rc;
  return hip_rc(saef::launch_materialize(layout->dev, 0, SAEF_MODE_DC, nullptr, nullptr,
                                         nullptr, nullptr, e_srv, x, srv_signs, srv_scales,
                                         e_srv, x, fold, stream));
}

int saef_step_ahead(const saef_layout* layout, int32_t K, const float* x, const float* e,
                    float* xh, hipStream_t stream) {
  int rc = check_common(layout, K);
  if (rc != SAEF_OK) return rc;
  if (!f32_ok(x) || !f32_ok(e) || !f32_ok(xh)) return SAEF_EINVAL;
  const size_t vb = (size_t)K * layout->d_pad * sizeof(float);
  if (overlap(xh, vb, x, layout->d_pad * sizeof(float)) || overlap(xh, vb, e, vb))
    return SAEF_EINVAL;
  return hip_rc(saef::launch_step_ahead(layout->dev, K, x, nullptr, nullptr, false,
                                        const_cast<float*>(e), nullptr, nullptr, false, false, xh,
                                        stream));
}

int saef_error_average(const saef_layout* layout, int32_t K, float* e, hipStream_t stream) {
  int rc = check_common(layout, K);
  if (rc != SAEF_OK) return rc;
  if (!f32_ok(e)) return SAEF_EINVAL;
  return hip_rc(saef::launch_step_ahead(layout->dev, K, nullptr, nullptr, nullptr, false, e,
                                        nullptr, nullptr, false, true, nullptr, stream));
}

}  // extern "C"

namespace {

// saef_round / saef_round_momentum (m == nullptr: no momentum).
// The first half of iteration t (Algorithm 1 up to the gradient): error
// averaging when due, the mismatch bounds when requested, then the point
// where the gradient is taken (step ahead, or the weights themselves for
// local error feedback).  The state is in saef_round's pending form.
int round_begin_impl(const saef_layout* layout, int64_t t, int64_t period, int32_t K,
                     int32_t mode, int32_t variant, float* e, const float* e_srv, const float* x,
                     float* xh, const uint64_t* signs, const float* scales,
                     const uint64_t* srv_signs, const float* srv_scales, double* mismatch,
                     hipStream_t stream, const DevLayout* dev = nullptr) {
  int rc = check_common(layout, K);
  if (rc != SAEF_OK) return rc;
  if (t < 0 || period < 0) return SAEF_EINVAL;
  if (mode != SAEF_MODE_SC && mode != SAEF_MODE_DC) return SAEF_EINVAL;
  if (variant != SAEF_VARIANT_EF && variant != SAEF_VARIANT_SAEF) return SAEF_EINVAL;
  const bool pending = t > 0;  // at t == 0 the state is plain (Algorithm 1 initialisation)
  const bool averaging = period > 0 && (t + 1) % period == 0;
  const bool dc = mode == SAEF_MODE_DC;
  if (!f32_ok(e) || !f32_ok(x) || !f32_ok(xh)) return SAEF_EINVAL;
  if (pending && (!u64_ok(signs) || !f32_ok(scales))) return SAEF_EINVAL;
  if (pending && dc && (!u64_ok(srv_signs) || !f32_ok(srv_scales))) return SAEF_EINVAL;
  if (mismatch != nullptr && (!aligned(mismatch, 8) || (dc && !f32_ok(e_srv))))
    return SAEF_EINVAL;
  const size_t vb = (size_t)K * layout->d_pad * sizeof(float);
  const size_t xb = layout->d_pad * sizeof(float);
  const size_t hb = variant == SAEF_VARIANT_SAEF ? vb : xb;
  if (overlap(xh, hb, x, xb) || overlap(xh, hb, e, vb) ||
      (e_srv != nullptr && overlap(xh, hb, e_srv, xb)))
    return SAEF_EINVAL;
  if (mismatch != nullptr) {
    const size_t mb = 2 * (size_t)layout->L * sizeof(double);
    if (overlap(mismatch, mb, e, vb) || overlap(mismatch, mb, xh, hb) ||
        overlap(mismatch, mb, x, xb) || (e_srv != nullptr && overlap(mismatch, mb, e_srv, xb)))
      return SAEF_EINVAL;
  }
  const DevLayout& d = dev != nullptr ? *dev : layout->dev;
  if (variant == SAEF_VARIANT_SAEF) {
    // error averaging (when due) and step ahead, applying last iteration's
    // pending corrections to e and (double-way) x
    rc = hip_rc(timed(layout, averaging ? 5 : 0, [&](const saef::LaunchEvents& ev) {
      return saef::launch_step_ahead(d, K, x, srv_signs, srv_scales, pending && dc, e, signs,
                                     scales, pending, averaging, xh, stream, ev);
    }));
    if (rc != SAEF_OK) return rc;
  } else if (averaging) {
    // local error feedback with error averaging: average only
    rc = hip_rc(timed(layout, 5, [&](const saef::LaunchEvents& ev) {
      return saef::launch_step_ahead(d, K, x, srv_signs, srv_scales, false, e, signs, scales,
                                     pending, true, nullptr, stream, ev);
    }));
    if (rc != SAEF_OK) return rc;
  }
  if (mismatch != nullptr) {
    // the errors are plain after an averaging step
    rc = hip_rc(timed(layout, 6, [&](const saef::LaunchEvents& ev) {
      return saef::launch_mismatch(d, K, mode, e, signs, scales, pending && !averaging, e_srv,
                                   srv_signs, srv_scales, pending && dc, mismatch, stream, ev);
    }));
    if (rc != SAEF_OK) return rc;
  }
  if (variant == SAEF_VARIANT_SAEF) return SAEF_OK;
  // local error feedback: the gradient is taken at x_t itself (one row)
  return hip_rc(timed(layout, 0, [&](const saef::LaunchEvents& ev) {
    return saef::launch_weights(d, x, srv_signs, srv_scales, pending && dc, xh, stream, ev);
  }));
}

// The second half of iteration t: worker compression (momentum update first
// when m is given), worker scales, server aggregation and compression,
// server scales.  e is plain when the first half averaged it.  xh non-null
// (saef_round, no averaging due): the first half's step ahead, in the same
// pass as the compression.
int round_end_impl(const saef_layout* layout, int64_t t, int64_t period, int32_t K, float lr,
                   float mu, int32_t mode, const float* g, float* m, float* e, float* e_srv,
                   float* x, uint64_t* signs, float* scales, uint64_t* srv_signs,
                   float* srv_scales, hipStream_t stream, const DevLayout* dev = nullptr,
                   float* xh = nullptr, float max_norm = 0.0f, const float* norms = nullptr) {
  int rc = check_common(layout, K);
  if (rc != SAEF_OK) return rc;
  if (t < 0 || period < 0 || !std::isfinite(lr)) return SAEF_EINVAL;
  if (mode != SAEF_MODE_SC && mode != SAEF_MODE_DC) return SAEF_EINVAL;
  if (!f32_ok(g) || !f32_ok(e) || !f32_ok(x) || !u64_ok(signs) || !f32_ok(scales))
    return SAEF_EINVAL;
  if (mode == SAEF_MODE_DC && (!f32_ok(e_srv) || !u64_ok(srv_signs) || !f32_ok(srv_scales)))
    return SAEF_EINVAL;
  const size_t vb = (size_t)K * layout->d_pad * sizeof(float);
  const size_t xb = layout->d_pad * sizeof(float);
  if (overlap(g, vb, e, vb) || overlap(g, vb, x, xb) || overlap(e, vb, x, xb)) return SAEF_EINVAL;
  if (m != nullptr && (!f32_ok(m) || overlap(m, vb, g, vb) || overlap(m, vb, e, vb) ||
                       overlap(m, vb, x, xb)))
    return SAEF_EINVAL;
  if (norms != nullptr) {
    // read while all of these are written
    const size_t wb = (size_t)layout->d_pad / 64 * sizeof(uint64_t);
    const size_t sb = (size_t)layout->L * sizeof(float);
    if (!aligned(norms, 4) || !clip_bound_ok(max_norm) ||
        overlap_any(norms, K * sizeof(float),
                    {{e, vb}, {m, vb}, {x, xb}, {signs, K * wb}, {scales, K * sb}, {e_srv, xb},
                     {srv_signs, wb}, {srv_scales, sb}}))
      return SAEF_EINVAL;
  }

  const bool pending = t > 0;
  const bool averaging = period > 0 && (t + 1) % period == 0;
  const bool dc = mode == SAEF_MODE_DC;
  const DevLayout& d = dev != nullptr ? *dev : layout->dev;
  // [gradient slot: g was computed by the caller at the first half's xh]
  rc = hip_rc(timed(layout, 1, [&](const saef::LaunchEvents& ev) {
    if (xh != nullptr)
      return saef::launch_worker(d, K, lr, mu, g, m, e, signs, scales, pending, x, srv_signs,
                                 srv_scales, pending && dc, xh, stream, ev);
    return saef::launch_compress(d, K, lr, mu, g, m, e, signs, scales, pending && !averaging,
                                 stream, ev, max_norm, norms);
  }));
  if (rc != SAEF_OK) return rc;
  // Small layouts: the aggregation adds up the worker partials itself, one
  // dependent launch less.
  const bool fold = saef::folds_scales(d, K);
  if (!fold)
    rc = hip_rc(timed(layout, 2, [&](const saef::LaunchEvents& ev) {
      return saef::launch_finalize(d, K, false, scales, stream, ev);
    }));
  if (rc != SAEF_OK) return rc;
  // server aggregation, server compression; x keeps its correction pending
  rc = hip_rc(timed(layout, 3, [&](const saef::LaunchEvents& ev) {
    return saef::launch_aggregate(d, K, mode, signs, scales, fold, nullptr, e_srv, srv_signs,
                                  srv_scales, x, pending && dc, stream, ev);
  }));
  if (rc != SAEF_OK || !dc) return rc;
  return hip_rc(timed(layout, 4, [&](const saef::LaunchEvents& ev) {
    return saef::launch_finalize(d, K, true, srv_scales, stream, ev);
  }));
}

int round_impl(const saef_layout* layout, int64_t t, int64_t period, int32_t K, float lr,
               float mu, int32_t mode, const float* g, float* m, float* e, float* e_srv,
               float* x, float* xh, uint64_t* signs, float* scales, uint64_t* srv_signs,
               float* srv_scales, hipStream_t stream, const DevLayout* dev = nullptr) {
  // check both halves' arguments before anything is enqueued
  int rc = check_common(layout, K);
  if (rc != SAEF_OK) return rc;
  if (t < 0 || period < 0 || !std::isfinite(lr)) return SAEF_EINVAL;
  if (mode != SAEF_MODE_SC && mode != SAEF_MODE_DC) return SAEF_EINVAL;
  if (!f32_ok(g) || !f32_ok(e) || !f32_ok(x) || !f32_ok(xh) || !u64_ok(signs) || !f32_ok(scales))
    return SAEF_EINVAL;
  if (mode == SAEF_MODE_DC && (!f32_ok(e_srv) || !u64_ok(srv_signs) || !f32_ok(srv_scales)))
    return SAEF_EINVAL;
  const size_t vb = (size_t)K * layout->d_pad * sizeof(float);
  const size_t xb = layout->d_pad * sizeof(float);
  if (overlap(xh, vb, x, xb) || overlap(xh, vb, e, vb) || overlap(xh, vb, g, vb) ||
      overlap(g, vb, e, vb) || overlap(g, vb, x, xb) || overlap(e, vb, x, xb))
    return SAEF_EINVAL;
  if (m != nullptr && (!f32_ok(m) || overlap(m, vb, g, vb) || overlap(m, vb, e, vb) ||
                       overlap(m, vb, xh, vb) || overlap(m, vb, x, xb)))
    return SAEF_EINVAL;
  if (e_srv != nullptr && overlap(xh, vb, e_srv, xb)) return SAEF_EINVAL;
  // The gradient is in place, so off the averaging iterations the step ahead
  // shares its pass over e with the compression (resnet50 K = 8: one kernel
  // of 555 us for one of 280 and one of 400).
  // (Not when xh shares memory with a message: the step ahead goes first then.)
  const size_t wb = (size_t)layout->d_pad / 64 * sizeof(uint64_t), sb = layout->L * sizeof(float);
  const bool apart = !overlap_any(xh, vb, {{signs, K * wb}, {scales, K * sb}, {srv_signs, wb},
                                           {srv_scales, sb}});
  if (apart && (period == 0 || (t + 1) % period != 0))
    return round_end_impl(layout, t, period, K, lr, mu, mode, g, m, e, e_srv, x, signs, scales,
                          srv_signs, srv_scales, stream, dev, xh);
  rc = round_begin_impl(layout, t, period, K, mode, SAEF_VARIANT_SAEF, e, e_srv, x, xh, signs,
                        scales, srv_signs, srv_scales, nullptr, stream, dev);
  if (rc != SAEF_OK) return rc;
  return round_end_impl(layout, t, period, K, lr, mu, mode, g, m, e, e_srv, x, signs, scales,
                        srv_signs, srv_scales, stream, dev);
}

}  // namespace

extern "C" {

int saef_round(const saef_layout* layout, int64_t t, int64_t period, int32_t K, float lr,
               int32_t mode, const float* g, float* e, float* e_srv, float* x, float* xh,
               uint64_t* signs, float* scales, uint64_t* srv_signs, float* srv_scales,
               hipStream_t stream) {
  return round_impl(layout, t, period, K, lr, 0.0f, mode, g, nullptr, e, e_srv, x, xh, signs,
                    scales, srv_signs, srv_scales, stream);
}

int saef_round_noalloc(const saef_layout* layout, int64_t t, int64_t period, int32_t K, float lr,
                       int32_t mode, const float* g, float* e, float* e_srv, float* x, float* xh,
                       uint64_t* signs, float* scales, uint64_t* srv_signs, float* srv_scales,
                       hipStream_t stream) {
  int rc = check_common(layout, K);
  if (rc != SAEF_OK) return rc;
  // the tile partial sums of K worker rows and the server row, and their
  // second level, must fit the static scratch
  const DevLayout& ld = layout->dev;
  const size_t rows = (size_t)K + 1;
  const size_t part_bytes = rows * (size_t)ld.n_tiles * 2 * sizeof(unsigned long long);
  const size_t part2_bytes = rows * (size_t)ld.L * (size_t)ld.fin_split * 2 *
                             sizeof(unsigned long long);
  const size_t part_pad = (part_bytes + 255) / 256 * 256;
  if (part_pad + part2_bytes > kScratchBytes) return SAEF_EINVAL;
  unsigned char* base = static_cast<unsigned char*>(scratch_of(layout->device));
  if (base == nullptr) return SAEF_EHIP;
  DevLayout d = ld;
  d.part = reinterpret_cast<unsigned long long*>(base);
  d.part2 = reinterpret_cast<unsigned long long*>(base + part_pad);
  d.k_max = K;  // the server's partial sums go to row K of the scratch
  return round_impl(layout, t, period, K, lr, 0.0f, mode, g, nullptr, e, e_srv, x, xh, signs,
                    scales, srv_signs, srv_scales, stream, &d);
}

int saef_round_momentum(const saef_layout* layout, int64_t t, int64_t period, int32_t K,
                        float lr, float mu, int32_t mode, const float* g, float* m, float* e,
                        float* e_srv, float* x, float* xh, uint64_t* signs, float* scales,
                        uint64_t* srv_signs, float* srv_scales, hipStream_t stream) {
  if (!mu_ok(mu) || m == nullptr) return SAEF_EINVAL;
  return round_impl(layout, t, period, K, lr, mu, mode, g, m, e, e_srv, x, xh, signs, scales,
                    srv_signs, srv_scales, stream);
}

int saef_round_begin(const saef_layout* layout, int64_t t, int64_t period, int32_t K,
                     int32_t mode, int32_t variant, float* e, const float* e_srv, const float* x,
                     float* xh, const uint64_t* signs, const float* scales,
                     const uint64_t* srv_signs, const float* srv_scales, double* mismatch,
                     hipStream_t stream) {
  return round_begin_impl(layout, t, period, K, mode, variant, e, e_srv, x, xh, signs, scales,
                          srv_signs, srv_scales, mismatch, stream);
}

int saef_round_end(const saef_layout* layout, int64_t t, int64_t period, int32_t K, float lr,
                   float mu, int32_t mode, const float* g, float* m, float* e, float* e_srv,
                   float* x, uint64_t* signs, float* scales, uint64_t* srv_signs,
                   float* srv_scales, hipStream_t stream) {
  if (m == nullptr ? mu != 0.0f : !mu_ok(mu)) return SAEF_EINVAL;
  return round_end_impl(layout, t, period, K, lr, mu, mode, g, m, e, e_srv, x, signs, scales,
                        srv_signs, srv_scales, stream);
}

int saef_round_end_clipped(const saef_layout* layout, int64_t t, int64_t period, int32_t K,
                           float lr, float mu, int32_t mode, float max_norm, const float* norms,
                           const float* g, float* m, float* e, float* e_srv, float* x,
                           uint64_t* signs, float* scales, uint64_t* srv_signs,
                           float* srv_scales, hipStream_t stream) {
  if (m == nullptr ? mu != 0.0f : !mu_ok(mu)) return SAEF_EINVAL;
  if (norms == nullptr) return SAEF_EINVAL;
  return round_end_impl(layout, t, period, K, lr, mu, mode, g, m, e, e_srv, x, signs, scales,
                        srv_signs, srv_scales, stream, nullptr, nullptr, max_norm, norms);
}

int saef_grads_create(const saef_layout* layout, int32_t K, int32_t dtype, void* const* ptr,
                      saef_grads** out) {
  if (out == nullptr) return SAEF_EINVAL;
  *out = nullptr;
  int rc = check_common(layout, K);
  if (rc != SAEF_OK) return rc;
  if (ptr == nullptr || dtype < SAEF_F32 || dtype > SAEF_F16) return SAEF_EINVAL;
  // a launch has at most 2^32 - 1 threads: a wave per (tile, worker), a workgroup per
  // (tensor, worker) and one per worker
  if ((double)K * (layout->dev.n_tiles + saef::kWaves) * saef::kWave >= 4294967296.0 ||
      (double)K * (layout->L + 1.0) * saef::kBlock >= 4294967296.0)
    return SAEF_EINVAL;
  const size_t es = (size_t)saef::dtype_bytes(dtype);
  const size_t rows = (size_t)K * layout->L;
  saef_grads* g = nullptr;
  try {
    g = new saef_grads();
    for (size_t i = 0; i < rows; ++i) {
      if (ptr[i] == nullptr || !aligned(ptr[i], es)) {
        delete g;
        return SAEF_EINVAL;
      }
      const uintptr_t a = reinterpret_cast<uintptr_t>(ptr[i]);
      g->spans.emplace_back(a, a + es * (size_t)layout->n[i % layout->L]);
    }
    std::sort(g->spans.begin(), g->spans.end());
  } catch (const std::bad_alloc&) {
    delete g;
    return SAEF_EHIP;
  }
  for (size_t i = 1; i < rows; ++i)
    if (g->spans[i - 1].second > g->spans[i].first) {
      delete g;
      return SAEF_EINVAL;
    }
  g->layout = layout;
  g->K = K;
  g->dtype = dtype;
  hipError_t err = hipMalloc(&g->mem_ptr, rows * sizeof(void*));
  // Runs of tiles: enough waves to fill the GPU a few times over (1 M tiles of 2^28 x
  // 8 in runs of 32 1287 us, of 4 1356, one by one 1340; bert_base bf16 x 4 of 8
  // 146, one by one 196).  A worker of few tiles has one workgroup, in one launch.
  const int64_t pairs = layout->dev.n_tiles * K;
  const bool small = layout->dev.n_tiles <= saef::kSmallTiles;
  int32_t run_tiles = 1;
  while (run_tiles < 32 && pairs / run_tiles > 32768) run_tiles *= 2;
  const int64_t runs = small ? 0 : (layout->dev.n_tiles + run_tiles - 1) / run_tiles;
  // What is read for the norm is read again to be clipped.  Up to 1 GB leaving it in
  // the last-level cache pays over both (resnet56 x 8 15.1 us against 19.2, bert_base
  // bf16 x 4 570 against 589, resnet50 x 8 394 both ways); beyond, loads that pass it
  // by are faster (2^28 x 8: the norm 1290 against 1446).
  const int32_t cached = (double)K * layout->d_pad * es <= 1073741824.0;
  if (err == hipSuccess && !small)
    err = hipMalloc(&g->mem_part, (size_t)K * layout->dev.n_tiles * sizeof(double));
  if (err == hipSuccess && !small)
    err = hipMalloc(&g->mem_runs, (size_t)K * runs * sizeof(double));
  if (err == hipSuccess)
    err = hipMemcpy(g->mem_ptr, ptr, rows * sizeof(void*), hipMemcpyHostToDevice);
  if (err != hipSuccess) {
    (void)saef_grads_destroy(g);
    return SAEF_EHIP;
  }
  g->dev = saef::GradsDev{static_cast<void* const*>(g->mem_ptr), static_cast<double*>(g->mem_part),
                          static_cast<double*>(g->mem_runs), runs, run_tiles, cached, K, dtype};
  *out = g;
  return SAEF_OK;
}

int saef_grads_destroy(saef_grads* grads) {
  if (grads == nullptr) return SAEF_EINVAL;
  for (void* q : {grads->mem_ptr, grads->mem_part, grads->mem_runs}) (void)hipFree(q);
  delete grads;
  return SAEF_OK;
}

int saef_grad_norm(const saef_grads* grads, int32_t norm_type, float* norms, float* tensor_norms,
                   hipStream_t stream) {
  if (grads == nullptr) return SAEF_EINVAL;
  int rc = check_common(grads->layout, grads->K);
  if (rc != SAEF_OK) return rc;
  if (norm_type != SAEF_NORM_2 && norm_type != SAEF_NORM_INF) return SAEF_EINVAL;
  const size_t nb = (size_t)grads->K * sizeof(float), tb = nb * grads->layout->L;
  if (!f32_ok(norms) || !aligned(tensor_norms, 4) || meets_grads(grads, norms, nb))
    return SAEF_EINVAL;
  if (tensor_norms != nullptr &&
      (overlap(norms, nb, tensor_norms, tb) || meets_grads(grads, tensor_norms, tb)))
    return SAEF_EINVAL;
  return hip_rc(saef::launch_grad_norm(grads->layout->dev, grads->dev, norm_type == SAEF_NORM_INF,
                                       norms, tensor_norms, stream));
}

int saef_clip(const saef_grads* grads, float max_norm, const float* norms, float* out,
              hipStream_t stream) {
  if (grads == nullptr) return SAEF_EINVAL;
  int rc = check_common(grads->layout, grads->K);
  if (rc != SAEF_OK) return rc;
  const size_t nb = (size_t)grads->K * sizeof(float);
  if (!clip_bound_ok(max_norm) || !f32_ok(norms) || !aligned(out, 4)) return SAEF_EINVAL;
  if (meets_grads(grads, norms, nb)) return SAEF_EINVAL;
  if (out != nullptr) {
    const size_t vb = (size_t)grads->K * grads->layout->d_pad * sizeof(float);
    if (overlap(out, vb, norms, nb) || meets_grads(grads, out, vb)) return SAEF_EINVAL;
  }
  return hip_rc(saef::launch_clip(grads->layout->dev, grads->dev, max_norm, norms, out, stream));
}

int saef_materialize(const saef_layout* layout, int32_t K, int32_t mode, const float* e,
                     const float* e_srv, const float* x, const uint64_t* signs,
                     const float* scales, const uint64_t* srv_signs, const float* srv_scales,
                     float* e_out, float* e_srv_out, float* x_out, hipStream_t stream) {
  int rc = check_common(layout, K);
  if (rc != SAEF_OK) return rc;
  if (mode != SAEF_MODE_SC && mode != SAEF_MODE_DC) return SAEF_EINVAL;
  if (e_out != nullptr && (!f32_ok(e_out) || !f32_ok(e) || !u64_ok(signs) || !f32_ok(scales)))
    return SAEF_EINVAL;
  if (x_out != nullptr && (!f32_ok(x_out) || !f32_ok(x))) return SAEF_EINVAL;
  if (e_srv_out != nullptr && !f32_ok(e_srv_out)) return SAEF_EINVAL;
  if (mode == SAEF_MODE_DC && (e_srv_out != nullptr || x_out != nullptr) &&
      (!u64_ok(srv_signs) || !f32_ok(srv_scales)))
    return SAEF_EINVAL;
  if (mode == SAEF_MODE_DC && e_srv_out != nullptr && !f32_ok(e_srv)) return SAEF_EINVAL;
  return hip_rc(saef::launch_materialize(layout->dev, K, mode, e, signs,
                                         const_cast<float*>(scales), e_out, e_srv, x, srv_signs,
                                         const_cast<float*>(srv_scales), e_srv_out, x_out, false,
                                         stream));
}

int saef_profile_enable(saef_layout* layout, int32_t capacity, uint32_t kind_mask,
                        int32_t every) {
  if (layout == nullptr || capacity < 0 || capacity > (1 << 20) || every < 1) return SAEF_EINVAL;
  release_events(layout);
  layout->ev_mask = kind_mask;
  layout->ev_every = every;
  for (int i = 0; i < kProfileKinds; ++i) layout->ev_seen[i] = 0;
  for (int32_t i = 0; i < capacity; ++i) {
    hipEvent_t a = nullptr, b = nullptr;
    if (hipEventCreate(&a) != hipSuccess) return SAEF_EHIP;
    if (hipEventCreate(&b) != hipSuccess) {
      (void)hipEventDestroy(a);
      return SAEF_EHIP;
    }
    layout->ev_start.push_back(a);
    layout->ev_stop.push_back(b);
    layout->ev_kind.push_back(-1);
  }
  layout->ev_used = 0;
  return SAEF_OK;
}

int saef_stream_probe(const float* a, const float* b, float* c, int64_t n,
                      hipStream_t stream) {
  if (n < 1 || n > (int64_t)saef::kTileElems * 2147483647) return SAEF_EINVAL;
  if (!f32_ok(a) || (b != nullptr && !f32_ok(b)) || !f32_ok(c)) return SAEF_EINVAL;
  const size_t vb = (size_t)n * sizeof(float);
  if (b != nullptr && (overlap(c, vb, a, vb) || overlap(c, vb, b, vb))) return SAEF_EINVAL;
  if (b == nullptr && c != a && overlap(c, vb, a, vb)) return SAEF_EINVAL;
  return hip_rc(saef::launch_stream_probe(a, b, c, n, stream));
}

int saef_profile_read(saef_layout* layout, int32_t* counts, double* total_ms) {
  if (layout == nullptr || counts == nullptr || total_ms == nullptr) return SAEF_EINVAL;
  for (int i = 0; i < kProfileKinds; ++i) {
    counts[i] = 0;
    total_ms[i] = 0.0;
  }
  for (size_t i = 0; i < layout->ev_used; ++i) {
    if (hipEventSynchronize(layout->ev_stop[i]) != hipSuccess) return SAEF_EHIP;
    float ms = 0.0f;
    if (hipEventElapsedTime(&ms, layout->ev_start[i], layout->ev_stop[i]) != hipSuccess)
      return SAEF_EHIP;
    const int k = layout->ev_kind[i];
    if (k >= 0 && k < kProfileKinds) {
      counts[k] += 1;
      total_ms[k] += ms;
    }
  }
  layout->ev_used = 0;
  return SAEF_OK;
}

int saef_topk_create(const saef_layout* layout, const int64_t* keep, saef_topk** out) {
  if (out == nullptr) return SAEF_EINVAL;
  *out = nullptr;
  if (layout == nullptr || keep == nullptr) return SAEF_EINVAL;
  if (!saef::kTkUsable) return SAEF_EINVAL;  // a build with other than 2048-element tiles
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess) return SAEF_EHIP;
  if (dev != layout->device) return SAEF_EINVAL;
  const int32_t L = layout->L;
  for (int32_t l = 0; l < L; ++l)
    if (keep[l] < 1 || keep[l] > layout->n[l]) return SAEF_EINVAL;
  saef_topk* p = new (std::nothrow) saef_topk();
  if (p == nullptr) return SAEF_EHIP;
  p->layout = layout;
  p->keep.assign(keep, keep + L);
  // server chunks (kTkChunk elements); for large tensors
  // (below) tile groups (kTkGroup tiles), and for those with more than
  // kTkGroup groups (huge) super-groups (kTkGroup groups)
  std::vector<saef::TkChunk> chunks;
  std::vector<saef::TkTensor> tens(L);
  std::vector<saef::TkGroup> groups, sgroups;
  std::vector<int32_t> large;
  // A tensor of up to small_tiles tiles is selected by one workgroup of one
  // kernel; the others are large.  One workgroup takes up to a group of
  // tiles; where larger tensors need the other kernels anyway, only a
  // quarter (beyond, spreading the tiles over workgroups is faster).
  int32_t small_tiles = saef::kTkGroup;
  for (int32_t l = 0; l < L; ++l)
    if (layout->tensors[l].ntiles > saef::kTkGroup) small_tiles = saef::kTkSmall;
  for (int32_t l = 0; l < L; ++l) {
    const int64_t n = layout->n[l];
    const int64_t nc = (n + saef::kTkChunk - 1) / saef::kTkChunk;
    const int32_t first_tile = layout->tensors[l].first_tile, ntiles = layout->tensors[l].ntiles;
    const int32_t ng =
        ntiles > small_tiles ? (ntiles + saef::kTkGroup - 1) / saef::kTkGroup : 0;
    const int32_t nsg = ng > saef::kTkGroup ? (ng + saef::kTkGroup - 1) / saef::kTkGroup : 0;
    tens[l] = saef::TkTensor{p->total_keep,          keep[l],
                             (int32_t)chunks.size(), (int32_t)nc,
                             (int32_t)groups.size(), ng,
                             (int32_t)sgroups.size(), nsg,
                             (int32_t)large.size(),   0};
    if (ng > 0) large.push_back(l);
    p->total_keep += keep[l];
    for (int64_t c = 0; c < nc; ++c)
      chunks.push_back(saef::TkChunk{layout->off[l] + c * saef::kTkChunk, l,
                                     (int32_t)std::min<int64_t>(saef::kTkChunk,
                                                                n - c * saef::kTkChunk)});
    for (int32_t s = 0; s < nsg; ++s)
      sgroups.push_back(saef::TkGroup{l, (int32_t)groups.size() + s * saef::kTkGroup,
                                      std::min(saef::kTkGroup, ng - s * saef::kTkGroup), 0});
    for (int32_t g = 0; g < ng; ++g)
      groups.push_back(saef::TkGroup{l, first_tile + g * saef::kTkGroup,
                                     std::min(saef::kTkGroup, ntiles - g * saef::kTkGroup), 0});
  }
  p->all = saef::TkPart{0, L, 0, (int32_t)layout->dev.n_tiles, 0, (int32_t)groups.size(),
                        0, (int32_t)sgroups.size(), 0, (int32_t)chunks.size(),
                        0, (int32_t)large.size()};
  p->pipe = pipeline_parts(layout, tens);
  const size_t rows = (size_t)layout->k_max + 1;
  if ((int64_t)std::max(chunks.size(), groups.size() * saef::kTkGatherSplit) * (int64_t)rows >
      kMaxGrid) {
    free_topk(p);
    return SAEF_EINVAL;
  }
  const size_t n_tiles = (size_t)layout->dev.n_tiles;
  const size_t thist_bytes = rows * n_tiles * saef::kTkHistPad * sizeof(uint16_t);
  const size_t ghist_bytes = rows * groups.size() * saef::kTkHistPad * sizeof(uint32_t);
  const size_t sghist_bytes = rows * sgroups.size() * saef::kTkHistPad * sizeof(uint32_t);
  const size_t sel_bytes = rows * L * sizeof(saef::TkSel);
  const size_t cnt_bytes = rows * n_tiles * sizeof(uint32_t);
  // candidate slots: at most every element of a tensor (8 B each) per row
  const size_t cand_bytes = rows * (size_t)layout->d_pad * sizeof(unsigned long long);
  const size_t rhist_bytes = rows * large.size() * saef::kTkRefineLevels * saef::kTkBins * sizeof(uint32_t);
  // speculative candidate lists of the worker rows and the server row
  const size_t spec_bytes =
      (size_t)(layout->k_max + 1) * n_tiles * saef::kTkSpecCap * sizeof(unsigned long long);
  hipError_t err = hipMalloc(&p->mem_chunks, chunks.size() * sizeof(saef::TkChunk));
  if (err == hipSuccess) err = hipMalloc(&p->mem_tens, tens.size() * sizeof(saef::TkTensor));
  if (err == hipSuccess && !groups.empty())
    err = hipMalloc(&p->mem_groups, groups.size() * sizeof(saef::TkGroup));
  if (err == hipSuccess && !sgroups.empty())
    err = hipMalloc(&p->mem_sgroups, sgroups.size() * sizeof(saef::TkGroup));
  if (err == hipSuccess) err = hipMalloc(&p->mem_thist, thist_bytes);
  if (err == hipSuccess && ghist_bytes) err = hipMalloc(&p->mem_ghist, ghist_bytes);
  if (err == hipSuccess && sghist_bytes) err = hipMalloc(&p->mem_sghist, sghist_bytes);
  if (err == hipSuccess) err = hipMalloc(&p->mem_sel, sel_bytes);
  if (err == hipSuccess) err = hipMalloc(&p->mem_tile_cnt, cnt_bytes);
  if (err == hipSuccess) err = hipMalloc(&p->mem_cand, cand_bytes);
  if (err == hipSuccess) err = hipMalloc(&p->mem_lcnt, cnt_bytes);
  if (err == hipSuccess && rhist_bytes) err = hipMalloc(&p->mem_rhist, rhist_bytes);
  if (err == hipSuccess && rhist_bytes) err = hipMalloc(&p->mem_tile_cand, cnt_bytes);
  if (err == hipSuccess && !large.empty()) {
    const size_t seg_bytes = rows * groups.size() * saef::kTkGatherSplit * sizeof(uint32_t);
    err = hipMalloc(&p->mem_seg, seg_bytes);
    if (err == hipSuccess) err = hipMemset(p->mem_seg, 0, seg_bytes);
    const size_t arrived_bytes = rows * large.size() * sizeof(uint32_t);
    if (err == hipSuccess) err = hipMalloc(&p->mem_arrived, arrived_bytes);
    if (err == hipSuccess) err = hipMemset(p->mem_arrived, 0, arrived_bytes);
    if (err == hipSuccess) err = hipMalloc(&p->mem_large, large.size() * sizeof(int32_t));
    if (err == hipSuccess)
      err = hipMemcpy(p->mem_large, large.data(), large.size() * sizeof(int32_t),
                      hipMemcpyHostToDevice);
  }
  if (err == hipSuccess) err = hipMalloc(&p->mem_spec, spec_bytes);
  if (err == hipSuccess)
    err = hipMemcpy(p->mem_chunks, chunks.data(), chunks.size() * sizeof(saef::TkChunk),
                    hipMemcpyHostToDevice);
  if (err == hipSuccess)
    err = hipMemcpy(p->mem_tens, tens.data(), tens.size() * sizeof(saef::TkTensor),
                    hipMemcpyHostToDevice);
  if (err == hipSuccess && !groups.empty())
    err = hipMemcpy(p->mem_groups, groups.data(), groups.size() * sizeof(saef::TkGroup),
                    hipMemcpyHostToDevice);
  if (err == hipSuccess && !sgroups.empty())
    err = hipMemcpy(p->mem_sgroups, sgroups.data(), sgroups.size() * sizeof(saef::TkGroup),
                    hipMemcpyHostToDevice);
  if (err == hipSuccess) {
    // zero state (the first call's window starts at the bottom of the key
    // range), and the per-tensor speculative-list switch
    std::vector<saef::TkSel> sel0(rows * L);
    for (size_t r = 0; r < rows; ++r)
      for (int32_t l = 0; l < L; ++l) {
        saef::TkSel z{};
        z.lists = p->keep[l] * saef::kTkSpecMaxShare <= layout->n[l] ? 1u : 0u;
        sel0[r * L + l] = z;
      }
    err = hipMemcpy(p->mem_sel, sel0.data(), sel_bytes, hipMemcpyHostToDevice);
  }
  if (err == hipSuccess) err = hipStreamCreateWithFlags(&p->side.stream, hipStreamNonBlocking);
  if (err == hipSuccess) err = hipEventCreateWithFlags(&p->side.fork, hipEventDisableTiming);
  if (err == hipSuccess) err = hipEventCreateWithFlags(&p->side.join, hipEventDisableTiming);
  if (err == hipSuccess) err = hipDeviceSynchronize();
  if (err != hipSuccess) {
    free_topk(p);
    return SAEF_EHIP;
  }
  saef::TkDev& d = p->dev;
  d.chunks = static_cast<const saef::TkChunk*>(p->mem_chunks);
  d.tens = static_cast<const saef::TkTensor*>(p->mem_tens);
  d.groups = static_cast<const saef::TkGroup*>(p->mem_groups);
  d.sgroups = static_cast<const saef::TkGroup*>(p->mem_sgroups);
  d.thist = static_cast<uint16_t*>(p->mem_thist);
  d.ghist = static_cast<uint32_t*>(p->mem_ghist);
  d.sghist = static_cast<uint32_t*>(p->mem_sghist);
  d.sel = static_cast<saef::TkSel*>(p->mem_sel);
  d.tile_cnt = static_cast<uint32_t*>(p->mem_tile_cnt);
  d.cand = static_cast<unsigned long long*>(p->mem_cand);
  d.lcnt = static_cast<uint32_t*>(p->mem_lcnt);
  d.rhist = static_cast<uint32_t*>(p->mem_rhist);
  d.spec = static_cast<unsigned long long*>(p->mem_spec);
  d.n_chunks = (int64_t)chunks.size();
  d.n_groups = (int64_t)groups.size();
  d.n_sgroups = (int64_t)sgroups.size();
  d.tile_cand = static_cast<uint32_t*>(p->mem_tile_cand);
  d.seg = static_cast<uint32_t*>(p->mem_seg);
  d.arrived = static_cast<uint32_t*>(p->mem_arrived);
  d.large = static_cast<const int32_t*>(p->mem_large);
  d.n_large = (int64_t)large.size();
  d.levels = sgroups.empty() ? 0 : saef::kTkRefineLevels;
  for (int32_t l = 0; l < L; ++l)
    if (tens[l].ngroups == 0 && layout->tensors[l].ntiles > saef::kTkPickTiles) d.pick_wide = 1;
  d.alone = layout->dev.n_tiles * layout->k_max < saef::kTkSplitTiles ? 1 : 0;
  d.total_keep = p->total_keep;
  *out = p;
  return SAEF_OK;
}

int saef_topk_destroy(saef_topk* plan) {
  if (plan == nullptr) return SAEF_EINVAL;
  free_topk(plan);
  return SAEF_OK;
}

int saef_topk_info(const saef_topk* plan, int64_t* total_keep) {
  if (plan == nullptr) return SAEF_EINVAL;
  if (total_keep) *total_keep = plan->total_keep;
  return SAEF_OK;
}

namespace {

// The argument checks of saef_topk_compress.
int topk_compress_check(const saef_topk* plan, int32_t K, float lr, float mu, const float* g,
                        const float* m, const float* e, const uint64_t* sel,
                        const uint32_t* rank, const float* vals) {
  if (plan == nullptr) return SAEF_EINVAL;
  const saef_layout* layout = plan->layout;
  int rc = check_common(layout, K);
  if (rc != SAEF_OK) return rc;
  if (!std::isfinite(lr) || (m == nullptr ? mu != 0.0f : !mu_ok(mu))) return SAEF_EINVAL;
  if (!f32_ok(g) || !f32_ok(e) || !u64_ok(sel) || rank == nullptr || !aligned(rank, 4) ||
      !f32_ok(vals))
    return SAEF_EINVAL;
  const size_t vb = (size_t)K * layout->d_pad * sizeof(float);
  const size_t wb = (size_t)K * (layout->d_pad / 64) * sizeof(uint64_t);
  const size_t rb = (size_t)K * (layout->d_pad / 64) * sizeof(uint32_t);
  const size_t mb = (size_t)K * plan->total_keep * sizeof(float);
  if (overlap(g, vb, e, vb) || overlap(vals, mb, e, vb) || overlap(vals, mb, g, vb) ||
      overlap(sel, wb, e, vb) || overlap(rank, rb, e, vb) || overlap(rank, rb, vals, mb) ||
      overlap(sel, wb, vals, mb) || overlap(sel, wb, rank, rb))
    return SAEF_EINVAL;
  if (m != nullptr && (!f32_ok(m) || overlap(m, vb, g, vb) || overlap(m, vb, e, vb) ||
                       overlap(m, vb, vals, mb)))
    return SAEF_EINVAL;
  return SAEF_OK;
}

// saef_topk_compress with the pending flags of launch_topk_compress.
int topk_compress(const saef_topk* plan, int32_t K, float lr, float mu, const float* g,
                  float* m, float* e, uint64_t* sel, uint32_t* rank, float* vals, bool pend_in,
                  bool pend_out, const saef::TkStep& st, hipStream_t stream) {
  const int rc = topk_compress_check(plan, K, lr, mu, g, m, e, sel, rank, vals);
  if (rc != SAEF_OK) return rc;
  const saef_layout* layout = plan->layout;
  return hip_rc(timed(layout, 1, [&](const saef::LaunchEvents& ev) {
    return saef::launch_topk_compress(layout->dev, plan->dev, plan->all, K, lr, mu, g, m, e, sel,
                                      rank, vals, pend_in, pend_out, st, stream,
                                      layout->dev.n_tiles * K >= saef::kTkSplitTiles
                                          ? plan->side
                                          : saef::TkStreams(),
                                      ev);
  }));
}

// The argument checks of saef_topk_aggregate.
int topk_aggregate_check(const saef_topk* plan, int32_t K, int32_t mode, const uint64_t* sel,
                         const uint32_t* rank, const float* vals, const float* avg,
                         const float* e_srv, const uint64_t* srv_sel, const uint32_t* srv_rank,
                         const float* srv_vals, const float* x) {
  if (plan == nullptr) return SAEF_EINVAL;
  const saef_layout* layout = plan->layout;
  int rc = check_common(layout, K);
  if (rc != SAEF_OK) return rc;
  if (mode != SAEF_MODE_SC && mode != SAEF_MODE_DC) return SAEF_EINVAL;
  if (!u64_ok(sel) || rank == nullptr || !aligned(rank, 4) || !f32_ok(vals) || !f32_ok(x))
    return SAEF_EINVAL;
  if (avg != nullptr && !f32_ok(avg)) return SAEF_EINVAL;
  const size_t xb = layout->d_pad * sizeof(float);
  const size_t wb1 = (layout->d_pad / 64) * sizeof(uint64_t);
  const size_t rb1 = (layout->d_pad / 64) * sizeof(uint32_t);
  const size_t mb1 = plan->total_keep * sizeof(float);
  if (mode == SAEF_MODE_DC) {
    if (!f32_ok(e_srv) || !u64_ok(srv_sel) || srv_rank == nullptr || !aligned(srv_rank, 4) ||
        !f32_ok(srv_vals))
      return SAEF_EINVAL;
    if (overlap(e_srv, xb, x, xb) || overlap(srv_vals, mb1, x, xb) ||
        overlap(srv_vals, mb1, e_srv, xb) || overlap(srv_sel, wb1, x, xb) ||
        overlap(srv_sel, wb1, e_srv, xb) || overlap(srv_rank, rb1, x, xb) ||
        overlap(srv_rank, rb1, e_srv, xb) || overlap(srv_rank, rb1, srv_vals, mb1))
      return SAEF_EINVAL;
  }
  if (avg != nullptr && (overlap(avg, xb, x, xb) || (e_srv && overlap(avg, xb, e_srv, xb))))
    return SAEF_EINVAL;
  return SAEF_OK;
}

}  // namespace

int saef_topk_compress(const saef_topk* plan, int32_t K, float lr, float mu, const float* g,
                       float* m, float* e, uint64_t* sel, uint32_t* rank, float* vals,
                       hipStream_t stream) {
  return topk_compress(plan, K, lr, mu, g, m, e, sel, rank, vals, false, false, saef::TkStep(),
                       stream);
}

int saef_topk_materialize(const saef_topk* plan, int32_t K, float* e, const uint64_t* sel,
                          hipStream_t stream) {
  if (plan == nullptr) return SAEF_EINVAL;
  const saef_layout* layout = plan->layout;
  int rc = check_common(layout, K);
  if (rc != SAEF_OK) return rc;
  if (!f32_ok(e) || !u64_ok(sel)) return SAEF_EINVAL;
  const size_t vb = (size_t)K * layout->d_pad * sizeof(float);
  const size_t wb = (size_t)K * (layout->d_pad / 64) * sizeof(uint64_t);
  if (overlap(sel, wb, e, vb)) return SAEF_EINVAL;
  return hip_rc(saef::launch_topk_materialize(layout->dev, K, e, sel, stream));
}

int saef_topk_aggregate(const saef_topk* plan, int32_t K, int32_t mode, const uint64_t* sel,
                        const uint32_t* rank, const float* vals, float* avg, float* e_srv,
                        uint64_t* srv_sel, uint32_t* srv_rank, float* srv_vals, float* x,
                        hipStream_t stream) {
  const int rc = topk_aggregate_check(plan, K, mode, sel, rank, vals, avg, e_srv, srv_sel,
                                     srv_rank, srv_vals, x);
  if (rc != SAEF_OK) return rc;
  const saef_layout* layout = plan->layout;
  return hip_rc(timed(layout, 3, [&](const saef::LaunchEvents& ev) {
    return saef::launch_topk_aggregate(layout->dev, plan->dev, plan->all, K, mode, sel, rank,
                                       vals, avg, e_srv, srv_sel, srv_rank, srv_vals, x, stream,
                                       ev);
  }));
}

namespace {

// The argument checks of saef_topk_round_begin.
int topk_begin_check(const saef_topk* plan, int64_t t, int64_t period, int32_t K, int32_t mode,
                     int32_t variant, const float* e, const uint64_t* sel, const float* e_srv,
                     const float* x, const float* xh, const double* mismatch) {
  if (plan == nullptr) return SAEF_EINVAL;
  const saef_layout* layout = plan->layout;
  int rc = check_common(layout, K);
  if (rc != SAEF_OK) return rc;
  if (t < 0 || period < 0) return SAEF_EINVAL;
  if (mode != SAEF_MODE_SC && mode != SAEF_MODE_DC) return SAEF_EINVAL;
  if (variant != SAEF_VARIANT_EF && variant != SAEF_VARIANT_SAEF) return SAEF_EINVAL;
  if (!f32_ok(e) || !f32_ok(x) || !f32_ok(xh)) return SAEF_EINVAL;
  // after t = 0, e holds the previous iteration's Delta with its kept
  // elements (the selection words sel) pending
  const bool pending = t > 0;
  if (pending && !u64_ok(sel)) return SAEF_EINVAL;
  if (mismatch != nullptr && (!aligned(mismatch, 8) || (mode == SAEF_MODE_DC && !f32_ok(e_srv))))
    return SAEF_EINVAL;
  const size_t vb = (size_t)K * layout->d_pad * sizeof(float);
  const size_t xb = layout->d_pad * sizeof(float);
  const size_t hb = variant == SAEF_VARIANT_SAEF ? vb : xb;
  if (overlap(xh, hb, x, xb) || overlap(xh, hb, e, vb) || overlap(e, vb, x, xb) ||
      (e_srv != nullptr && overlap(xh, hb, e_srv, xb)))
    return SAEF_EINVAL;
  if (mismatch != nullptr) {
    const size_t mb = 2 * (size_t)layout->L * sizeof(double);
    if (overlap(mismatch, mb, e, vb) || overlap(mismatch, mb, xh, hb) ||
        overlap(mismatch, mb, x, xb) || (e_srv != nullptr && overlap(mismatch, mb, e_srv, xb)))
      return SAEF_EINVAL;
  }
  if (pending) {
    const size_t wb = (size_t)K * (layout->d_pad / 64) * sizeof(uint64_t);
    if (overlap(sel, wb, e, vb) || overlap(sel, wb, xh, hb) || overlap(sel, wb, x, xb))
      return SAEF_EINVAL;
  }
  return SAEF_OK;
}

// The argument checks of saef_topk_round_end, both halves of it.
int topk_end_check(const saef_topk* plan, int64_t t, int64_t period, int32_t K, float lr,
                   float mu, int32_t mode, const float* g, const float* m, const float* e,
                   const float* e_srv, const float* x, const uint64_t* sel, const uint32_t* rank,
                   const float* vals, const uint64_t* srv_sel, const uint32_t* srv_rank,
                   const float* srv_vals) {
  if (plan == nullptr || t < 0 || period < 0) return SAEF_EINVAL;
  int rc = topk_compress_check(plan, K, lr, mu, g, m, e, sel, rank, vals);
  if (rc == SAEF_OK)
    rc = topk_aggregate_check(plan, K, mode, sel, rank, vals, nullptr, e_srv, srv_sel, srv_rank,
                              srv_vals, x);
  if (rc != SAEF_OK) return rc;
  const size_t vb = (size_t)K * plan->layout->d_pad * sizeof(float);
  const size_t xb = plan->layout->d_pad * sizeof(float);
  return overlap(g, vb, x, xb) || overlap(e, vb, x, xb) ? SAEF_EINVAL : SAEF_OK;
}

// saef_topk_round_end; st: the step ahead taken along by the Delta pass.
int topk_round_end(const saef_topk* plan, int64_t t, int64_t period, int32_t K, float lr,
                   float mu, int32_t mode, const float* g, float* m, float* e, float* e_srv,
                   float* x, uint64_t* sel, uint32_t* rank, float* vals, uint64_t* srv_sel,
                   uint32_t* srv_rank, float* srv_vals, const saef::TkStep& st,
                   hipStream_t stream) {
  int rc = topk_end_check(plan, t, period, K, lr, mu, mode, g, m, e, e_srv, x, sel, rank, vals,
                          srv_sel, srv_rank, srv_vals);
  if (rc != SAEF_OK) return rc;
  const saef_layout* layout = plan->layout;
  // e is pending unless t = 0 or this iteration's averaging wrote it plain;
  // the compression leaves its own kept elements pending
  const bool averaging = period > 0 && (t + 1) % period == 0;
  const bool pend_in = t > 0 && !averaging;
  if (plan->pipe.size() >= 2 && layout->dev.n_tiles * K >= saef::kTkSplitTiles) {
    // pipelined over the plan's parts: one timed span (kind 1) from the
    // first Delta pass to the last kernel on the caller's stream
    return hip_rc(timed(layout, 1, [&](const saef::LaunchEvents& ev) {
      return saef::launch_topk_round_end(layout->dev, plan->dev, plan->pipe.data(),
                                         (int)plan->pipe.size(), K, lr, mu, mode, g, m, e, sel,
                                         rank, vals, pend_in, e_srv, srv_sel, srv_rank, srv_vals,
                                         x, st, stream, plan->side, ev);
    }));
  }
  rc = topk_compress(plan, K, lr, mu, g, m, e, sel, rank, vals, pend_in, true, st, stream);
  if (rc != SAEF_OK) return rc;
  return saef_topk_aggregate(plan, K, mode, sel, rank, vals, nullptr, e_srv, srv_sel, srv_rank,
                             srv_vals, x, stream);
}

}  // namespace

int saef_topk_round_begin(const saef_topk* plan, int64_t t, int64_t period, int32_t K,
                          int32_t mode, int32_t variant, float* e, const uint64_t* sel,
                          const float* e_srv, const float* x, float* xh, double* mismatch,
                          hipStream_t stream) {
  const int rc0 = topk_begin_check(plan, t, period, K, mode, variant, e, sel, e_srv, x, xh,
                                   mismatch);
  if (rc0 != SAEF_OK) return rc0;
  const saef_layout* layout = plan->layout;
  const bool pending = t > 0;
  int rc = SAEF_OK;
  const bool averaging = period > 0 && (t + 1) % period == 0;
  const DevLayout& d = layout->dev;
  const int dec = pending ? saef::kDecZero : saef::kDecPlain;
  if (variant == SAEF_VARIANT_SAEF || averaging) {
    float* h = variant == SAEF_VARIANT_SAEF ? xh : nullptr;
    rc = hip_rc(timed(layout, averaging ? 5 : 0, [&](const saef::LaunchEvents& ev) {
      return saef::launch_step_ahead(d, K, x, nullptr, nullptr, false, e, sel, nullptr, dec,
                                     averaging, h, stream, ev);
    }));
    if (rc != SAEF_OK) return rc;
  }
  if (mismatch != nullptr && pending && !averaging) {
    // the bounds read the plain errors: set the pending elements to 0 in place
    // (the next reader's zeroing of them is then a no-op)
    rc = hip_rc(saef::launch_topk_materialize(d, K, e, sel, stream));
    if (rc != SAEF_OK) return rc;
  }
  if (mismatch != nullptr) {
    rc = hip_rc(timed(layout, 6, [&](const saef::LaunchEvents& ev) {
      return saef::launch_mismatch(d, K, mode, e, nullptr, nullptr, false, e_srv, nullptr,
                                   nullptr, false, mismatch, stream, ev);
    }));
    if (rc != SAEF_OK) return rc;
  }
  if (variant == SAEF_VARIANT_SAEF) return SAEF_OK;
  return hip_rc(timed(layout, 0, [&](const saef::LaunchEvents& ev) {
    return saef::launch_weights(d, x, nullptr, nullptr, false, xh, stream, ev);
  }));
}

int saef_topk_round_end(const saef_topk* plan, int64_t t, int64_t period, int32_t K, float lr,
                        float mu, int32_t mode, const float* g, float* m, float* e, float* e_srv,
                        float* x, uint64_t* sel, uint32_t* rank, float* vals, uint64_t* srv_sel,
                        uint32_t* srv_rank, float* srv_vals, hipStream_t stream) {
  return topk_round_end(plan, t, period, K, lr, mu, mode, g, m, e, e_srv, x, sel, rank, vals,
                        srv_sel, srv_rank, srv_vals, saef::TkStep(), stream);
}

int saef_topk_round(const saef_topk* plan, int64_t t, int64_t period, int32_t K, float lr,
                    float mu, int32_t mode, const float* g, float* m, float* e, float* e_srv,
                    float* x, float* xh, uint64_t* sel, uint32_t* rank, float* vals,
                    uint64_t* srv_sel, uint32_t* srv_rank, float* srv_vals, hipStream_t stream) {
  if (plan == nullptr) return SAEF_EINVAL;
  const saef_layout* layout = plan->layout;
  int rc = check_common(layout, K);
  if (rc != SAEF_OK) return rc;
  if (!f32_ok(xh) || !f32_ok(g)) return SAEF_EINVAL;
  const size_t vb = (size_t)K * layout->d_pad * sizeof(float);
  if (overlap(xh, vb, g, vb)) return SAEF_EINVAL;
  // The gradient is in place: off the averaging iterations the Delta pass
  // takes the step ahead along, unless xh shares memory with something that
  // the rest of the iteration writes (then the step ahead goes first).
  const size_t W = layout->d_pad / 64;
  const bool apart =
      !overlap_any(xh, vb, {{m, vb}, {sel, K * W * 8}, {rank, K * W * 4},
                            {vals, (size_t)K * plan->total_keep * sizeof(float)},
                            {srv_sel, W * 8}, {srv_rank, W * 4},
                            {srv_vals, (size_t)plan->total_keep * sizeof(float)}});
  // both halves' arguments are checked before anything is enqueued
  rc = topk_begin_check(plan, t, period, K, mode, SAEF_VARIANT_SAEF, e, sel, e_srv, x, xh,
                        nullptr);
  if (rc == SAEF_OK)
    rc = topk_end_check(plan, t, period, K, lr, mu, mode, g, m, e, e_srv, x, sel, rank, vals,
                        srv_sel, srv_rank, srv_vals);
  if (rc != SAEF_OK) return rc;
  if (apart && (period == 0 || (t + 1) % period != 0))
    return topk_round_end(plan, t, period, K, lr, mu, mode, g, m, e, e_srv, x, sel, rank, vals,
                          srv_sel, srv_rank, srv_vals, saef::TkStep{x, xh}, stream);
  rc = saef_topk_round_begin(plan, t, period, K, mode, SAEF_VARIANT_SAEF, e, sel, e_srv, x, xh,
                             nullptr, stream);
  if (rc != SAEF_OK) return rc;
  // [gradient slot: g was computed by the caller at xh]
  return saef_topk_round_end(plan, t, period, K, lr, mu, mode, g, m, e, e_srv, x, sel, rank,
                             vals, srv_sel, srv_rank, srv_vals, stream);
}

int saef_status(const saef_layout* layout, hipStream_t stream) {
  if (layout == nullptr) return SAEF_EINVAL;
  if (hipStreamSynchronize(stream) != hipSuccess) return SAEF_EHIP;
  int flag = 0;
  if (hipMemcpy(&flag, layout->dev.status, sizeof(int), hipMemcpyDeviceToHost) != hipSuccess)
    return SAEF_EHIP;
  if (flag != 0 && hipMemset(layout->dev.status, 0, sizeof(int)) != hipSuccess) return SAEF_EHIP;
  return (flag & saef::kStatusRange) ? SAEF_ERANGE : SAEF_OK;
}

}  // extern "C"

// ---------------------------------------------------------------- group norm

namespace {

// How the kernels that read the features twice cut a shape: the vector width, the
// channels of a workgroup and the workgroups over the pixels of a sample.
void cut_group_norm(saef::GroupNormDev& d, int dtype) {
  const int32_t full = 16 / saef::dtype_bytes(dtype);
  const int32_t common = std::min(full, d.C & -d.C);
  d.vec = full;
  if (common == full) {
    // rows of 512 bytes, of whole groups where that is no more than twice as long
    const int32_t unit = d.Cg / std::min(full, d.Cg & -d.Cg) * full, row = 32 * full;
    d.slab = std::min(d.C, unit <= 2 * row ? (row + unit - 1) / unit * unit : row);
  } else if (d.C / common <= saef::kBlock) {
    // vectors that straddle pixels: the period of their channels is C / common threads
    d.slab = d.C;
  } else {
    d.vec = 1;
    d.slab = saef::kBlock;
  }
  d.slabs = (d.C + d.slab - 1) / d.slab;
  // About 2 workgroups for each of the 256 CUs (more make the second pass join more
  // sums: 50 MB forward 20.6 us, 24 with 4), of at least 8 vectors a thread, and at most
  // 32, or 64 where half of the threads have no whole pixels (the backward sums add a
  // thread's values in fp32, and long workgroups leave CUs idle at the end: 256 samples of
  // 1.6 MB forward 218 us, 226 with twice as many).
  const int64_t wgs = 512;
  const int64_t items = (int64_t)d.K * d.N * d.slabs, round = (int64_t)saef::kBlock * d.vec;
  const int64_t most = d.P * d.slab / (round * 8), least = d.P * d.slab / (round * 32) + 1;
  d.splits = (int32_t)std::max(least, std::min((wgs + items - 1) / items, most));
  d.split_pixels = (d.P + d.splits - 1) / d.splits;
  d.backwards = (double)d.K * d.N * d.P * d.C * saef::dtype_bytes(dtype) > 268435456.0;
}

// Whether, and how, features are held in registers between the sums and the
// result.
saef::GroupNormHeld hold_group_norm(const saef::GroupNormDev& d, int dtype, bool back) {
  const int32_t es = saef::dtype_bytes(dtype), vec = 16 / es;
  const saef::GroupNormHeld none{0, 0, 0, 0};
  if (d.P > (int64_t(1) << 31) / es / d.C - 1) return none;
  if (d.C % vec != 0) {
    // Vectors straddle pixels: the threads whose channels repeat take a whole sample, of
    // one vector at least.  128 samples of 64 x 33 in f32: forward 7.3 us, backward 11.6;
    // read twice 10.0 and 11.7.  2048 samples of 240 x 30: 22 and 53; 35 and 83.
    if (d.P * d.C < vec) return none;
    const int32_t period = d.C / std::min(vec, d.C & -d.C);
    for (int32_t threads : {64, 128, 256, 512})
      for (int32_t vectors : {4, 8}) {
        const int64_t held = (int64_t)(threads / period) * period * vectors * vec;
        if (held < d.P * d.C || held == 0) continue;
        // The most registers with 8 values a vector: a workgroup a CU, so one round of
        // them gains (256 samples of 196 x 84 in bf16 12.2 and 19.9 us, read twice 13.4
        // and 22.1) and more do not (512 of them 22.7 and 34; 17.9 and 25.4).  In f32
        // more do (512 samples of 500 x 30: 13.9 and 25.7; 19.6 and 38).
        if (vec == 8 && threads * vectors == 4096 && (int64_t)d.K * d.N > 256) return none;
        const saef::GroupNormHeld h{threads, vectors, d.C, 1};
        if (saef::group_norm_held_lds(d, h, dtype, back) <= saef::kMostLds) return h;
      }
    return none;
  }
  const int32_t unit = d.Cg / std::min(vec, d.Cg & -d.Cg) * vec;  // whole groups and vectors
  // Small workgroups first, then long rows (256 samples of 196 x 1024 in bf16: forward
  // 42 us with 256 threads and 256 bytes, 54 with 512 and 128; rows of 64 bytes took
  // 70); shorter ones only where there are no more channels.  What fits is faster this
  // way than in two passes: that shape 42 against 59 us, backward 72 against 109;
  // 784 x 512, in 512 threads, 91 against 108; 128 samples of 64 x 64 in fp32 7.7
  // against 10.
  for (int32_t most : {256, 512})
    for (int32_t row : {256, 128}) {
      int32_t slab = std::min(d.C, (row / es + unit - 1) / unit * unit);
      // a pixel or few: wider slabs
      while (slab < d.C && d.P * slab < 512 * vec) slab = std::min(d.C, 2 * slab);
      const int32_t cols = slab / vec;
      for (int32_t vectors : {4, 8, 16}) {
        if (vectors == 16 && back) continue;  // (their values do not fit the registers)
        const int64_t threads = ((d.P + vectors - 1) / vectors * cols + 63) / 64 * 64;
        if (threads > most) continue;
        const saef::GroupNormHeld h{(int32_t)threads, vectors, slab, (d.C + slab - 1) / slab};
        if (saef::group_norm_held_lds(d, h, dtype, back) <= saef::kMostLds) return h;
      }
    }
  return none;
}

struct GnSizes {
  size_t features, params, stats;  // bytes
};
GnSizes gn_sizes(const saef_group_norm* p, int64_t ld) {
  const saef::GroupNormDev& d = p->dev;
  return {(size_t)d.K * d.N * d.P * d.C * saef::dtype_bytes(p->dtype),
          ((size_t)(d.K - 1) * ld + d.C) * sizeof(float), (size_t)d.K * d.N * d.G * sizeof(float)};
}

// A row of a (K rows of C values, ld apart) shares memory with one of b?  They may
// lie in one another's gaps.
bool rows_meet(const saef_group_norm* p, const float* a, const float* b, int64_t ld) {
  const size_t bytes = gn_sizes(p, ld).params;
  if (!overlap(a, bytes, b, bytes)) return false;
  const uintptr_t pa = reinterpret_cast<uintptr_t>(a), pb = reinterpret_cast<uintptr_t>(b);
  const uintptr_t row = (uintptr_t)p->dev.C * sizeof(float), step = (uintptr_t)ld * sizeof(float);
  const uintptr_t apart = (pa < pb ? pb - pa : pa - pb) % step;
  return apart < row || apart > step - row;
}

int check_group_norm(const saef_group_norm* p) {
  if (p == nullptr) return SAEF_EINVAL;
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess) return SAEF_EHIP;
  return dev == p->device ? SAEF_OK : SAEF_EINVAL;
}

}  // namespace

extern "C" {

int saef_group_norm_create(int32_t K, int64_t N, int64_t P, int32_t C, int32_t G, int32_t dtype,
                           int32_t act, float eps, saef_group_norm** out) {
  if (out == nullptr) return SAEF_EINVAL;
  *out = nullptr;
  if (K < 1 || K > 4096 || N < 1 || P < 1 || C < 1 || C > 65536 || G < 1 || C % G != 0)
    return SAEF_EINVAL;
  if (dtype < SAEF_F32 || dtype > SAEF_F16) return SAEF_EINVAL;
  if (act < SAEF_ACT_NONE || act > SAEF_ACT_SILU) return SAEF_EINVAL;
  if (!std::isfinite(eps) || !(eps > 0.0f)) return SAEF_EINVAL;
  const int64_t most = int64_t(1) << 40;  // elements of the features
  if (N > most / K || P > most / ((int64_t)K * N) || C > most / ((int64_t)K * N * P))
    return SAEF_EINVAL;
  saef::GroupNormDev d{};
  d.K = K;
  d.N = N;
  d.P = P;
  d.C = C;
  d.G = G;
  d.Cg = C / G;
  d.eps = eps;
  cut_group_norm(d, dtype);
  const saef::GroupNormHeld fwd = hold_group_norm(d, dtype, false);
  const saef::GroupNormHeld bwd = hold_group_norm(d, dtype, true);
  // a launch has at most 2^32 - 1 threads
  const double items = (double)K * (double)N;
  const double params = (double)K * ((C + saef::kWave - 1) / saef::kWave);
  if ((items * d.slabs * d.splits + params) * saef::kBlock >= 4294967296.0 ||
      params * saef::kParamWaves * saef::kWave >= 4294967296.0 ||
      items * fwd.slabs * fwd.threads >= 4294967296.0 ||
      items * bwd.slabs * bwd.threads >= 4294967296.0)
    return SAEF_EINVAL;
  saef_group_norm* p = new (std::nothrow) saef_group_norm();
  if (p == nullptr) return SAEF_EHIP;
  p->dtype = dtype;
  p->act = act;
  p->fwd = fwd;
  p->bwd = bwd;
  hipError_t err = hipGetDevice(&p->device);
  const size_t rows = (size_t)K * N * d.splits, pair = 2 * sizeof(double);
  if (err == hipSuccess) err = hipMalloc(&p->mem_part, rows * C * 2 * sizeof(float));
  if (err == hipSuccess) err = hipMalloc(&p->mem_pieces, rows * (G + d.slabs - 1) * pair);
  if (err != hipSuccess) {
    (void)saef_group_norm_destroy(p);
    return SAEF_EHIP;
  }
  d.part = static_cast<float*>(p->mem_part);
  d.pieces = static_cast<double*>(p->mem_pieces);
  p->dev = d;
  *out = p;
  return SAEF_OK;
}

int saef_group_norm_destroy(saef_group_norm* plan) {
  if (plan == nullptr) return SAEF_EINVAL;
  (void)hipFree(plan->mem_part);
  (void)hipFree(plan->mem_pieces);
  delete plan;
  return SAEF_OK;
}

int saef_group_norm_forward(const saef_group_norm* plan, const void* x, const float* gamma,
                            const float* beta, int64_t ld, void* y, float* mean, float* rstd,
                            hipStream_t stream) {
  int rc = check_group_norm(plan);
  if (rc != SAEF_OK) return rc;
  const size_t es = (size_t)saef::dtype_bytes(plan->dtype);
  if (x == nullptr || y == nullptr || !aligned(x, es) || !aligned(y, es)) return SAEF_EINVAL;
  if (!f32_ok(gamma) || !f32_ok(beta) || !f32_ok(mean) || !f32_ok(rstd)) return SAEF_EINVAL;
  if (ld < plan->dev.C || ld > (int64_t(1) << 40)) return SAEF_EINVAL;
  const GnSizes z = gn_sizes(plan, ld);
  const Range in[3] = {{x, z.features}, {gamma, z.params}, {beta, z.params}};
  for (const Range& r : in)
    if (overlap_any(r.p, r.bytes, {{y, z.features}, {mean, z.stats}, {rstd, z.stats}}))
      return SAEF_EINVAL;
  if (overlap_any(y, z.features, {{mean, z.stats}, {rstd, z.stats}}) ||
      overlap(mean, z.stats, rstd, z.stats))
    return SAEF_EINVAL;
  return hip_rc(saef::launch_group_norm_forward(plan->dev, plan->fwd, plan->dtype, plan->act, x,
                                                gamma, beta, ld, y, mean, rstd, stream));
}

int saef_group_norm_backward(const saef_group_norm* plan, const void* dy, const void* x,
                             const float* gamma, const float* beta, int64_t ld,
                             const float* mean, const float* rstd, void* dx, float* dgamma,
                             float* dbeta, int64_t ldg, hipStream_t stream) {
  int rc = check_group_norm(plan);
  if (rc != SAEF_OK) return rc;
  const size_t es = (size_t)saef::dtype_bytes(plan->dtype);
  for (const void* p : {dy, x, (const void*)dx})
    if (p == nullptr || !aligned(p, es)) return SAEF_EINVAL;
  for (const float* p : {gamma, beta, mean, rstd, (const float*)dgamma, (const float*)dbeta})
    if (!f32_ok(p)) return SAEF_EINVAL;
  const int64_t most = int64_t(1) << 40;
  if (ld < plan->dev.C || ld > most || ldg < plan->dev.C || ldg > most) return SAEF_EINVAL;
  const GnSizes z = gn_sizes(plan, ld);
  const size_t gb = gn_sizes(plan, ldg).params;
  const Range in[6] = {{dy, z.features},  {x, z.features}, {gamma, z.params},
                       {beta, z.params}, {mean, z.stats}, {rstd, z.stats}};
  for (const Range& r : in)
    if (overlap_any(r.p, r.bytes, {{dx, z.features}, {dgamma, gb}, {dbeta, gb}}))
      return SAEF_EINVAL;
  if (overlap_any(dx, z.features, {{dgamma, gb}, {dbeta, gb}}) ||
      rows_meet(plan, dgamma, dbeta, ldg))
    return SAEF_EINVAL;
  return hip_rc(saef::launch_group_norm_backward(plan->dev, plan->bwd, plan->dtype, plan->act, dy,
                                                 x, gamma, beta, ld, mean, rstd, dx, dgamma,
                                                 dbeta, ldg, stream));
}

}  // extern "C"
