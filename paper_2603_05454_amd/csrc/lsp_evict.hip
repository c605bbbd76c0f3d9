// lsp_kv_evict: cuts the cache of a sequence back to `keep` rows, those of most accumulated attention weight, for every layer
// and KV head by itself.
//
// Which rows stay: the first `first`, the last `recent`, and of the others the largest weights (equal ones: the lower row).  A
// radix select over the weights' bits, mapped to whole numbers of the same order, finds the smallest weight that stays, 8
// bits a pass.
//
// Where they go: keys carry their positions and the attention has no mask, so the order of cached rows means nothing.  Rows
// below `keep` that stay do not move; each row from `keep` on that stays goes into the place of one below that leaves (the n-th of
// one to the n-th of the other).  That moves at most P - keep rows, where closing the gaps in order moves every row behind the first
// one.  Sources are all at or above `keep` and destinations below, so nothing that is read is written.
#include "lsp_common.h"

namespace lsp {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;
constexpr int kMaxLayersPerLaunch = 32;
struct CachePtrs {
  char *at[2 * kMaxLayersPerLaunch];  // K then V per layer
};

struct EvictArgs {
  const float *weights;  // [layers, B, Hkv, C], the launch's first layer
  float *new_weights;
  int32_t *kept_index;  // [layers, B, Hkv, keep] or null
  const int32_t *prefix_len;
  int32_t *moves;  // per unit (layer, sequence, KV head): count, then `room` destinations, then `room` sources
  int32_t B, Hkv, C, keep, high, first, recent, room;
};

// Whole numbers in the order of the weights: -0 as 0, NaN below everything.
__device__ __forceinline__ uint32_t order_of(float w) {
  const uint32_t u = __float_as_uint(w + 0.f);
  if ((u & 0x7fffffffu) > 0x7f800000u) return 0;
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Sum over the workgroup of the flags of the threads before this one; `all`: of all of them.
__device__ __forceinline__ int place_in_group(bool flag, int *s_wave, int &all) {
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
  const unsigned long long m = __ballot(flag);
  if (lane == 0) s_wave[wave] = __popcll(m);
  __syncthreads();
  int before = __popcll(m & ((1ull << lane) - 1));
  all = 0;
  for (int w = 0; w < kThreads / kWave; ++w) {
    if (w < wave) before += s_wave[w];
    all += s_wave[w];
  }
  __syncthreads();
  return before;
}

__global__ __launch_bounds__(kThreads) void evict_select_kernel(EvictArgs a) {
  __shared__ int s_count[256], s_wave[kThreads / kWave], s_digit, s_left;
  const int tid = threadIdx.x, b = blockIdx.y, unit = (blockIdx.z * a.B + b) * a.Hkv + blockIdx.x;
  const int P = min(max(a.prefix_len[b], 0), a.C);
  const float *w = a.weights + int64_t(unit) * a.C;
  float *nw = a.new_weights + int64_t(unit) * a.C;
  int32_t *kept = a.kept_index == nullptr ? nullptr : a.kept_index + int64_t(unit) * a.keep;
  int32_t *moves = a.moves + int64_t(unit) * (1 + 2 * a.room), *holes = moves + 1, *sources = moves + 1 + a.room;
  if (P <= a.high) {  // nothing leaves
    for (int t = tid; t < P; t += kThreads) nw[t] = w[t];
    if (kept != nullptr)
      for (int t = tid; t < a.keep; t += kThreads) kept[t] = t < P ? t : -1;
    if (tid == 0) moves[0] = 0;
    return;
  }
  // rows [first, end) compete for `left` places
  const int end = P - a.recent;
  int left = a.keep - a.first - a.recent;
  uint32_t found = 0, mask = 0;  // the digits found so far
  for (int shift = 24; shift >= 0 && left > 0; shift -= 8) {
    s_count[tid] = 0;
    __syncthreads();
    for (int t = a.first + tid; t < end; t += kThreads) {
      const uint32_t u = order_of(w[t]);
      if ((u & mask) == found) atomicAdd(&s_count[u >> shift & 255], 1);
    }
    __syncthreads();
    if (tid == 0) {
      int d = 255, above = 0;
      for (; d > 0 && above + s_count[d] < left; --d) above += s_count[d];
      s_digit = d;
      s_left = left - above;
    }
    __syncthreads();
    found |= uint32_t(s_digit) << shift;
    mask |= 255u << shift;
    left = s_left;
    __syncthreads();
  }
  // `left` of the rows equal to `found` stay, the lowest ones; with no place for any, none does
  const bool none = a.keep == a.first + a.recent;
  int equal_before = 0, nh = 0, ns = 0;
  for (int t0 = 0; t0 < P; t0 += kThreads) {
    const int t = t0 + tid;
    const uint32_t u = t >= a.first && t < end ? order_of(w[t]) : 0;
    const bool in = t >= a.first && t < end, equal = in && !none && u == found;
    int all;
    const int e = equal_before + place_in_group(equal, s_wave, all);
    equal_before += all;
    const bool stays = t < P && (!in || (!none && (u > found || (equal && e < left))));
    const bool hole = t < a.keep && !stays, moved = t >= a.keep && stays;
    const int h = nh + place_in_group(hole, s_wave, all);
    nh += all;
    const int s = ns + place_in_group(moved, s_wave, all);
    ns += all;
    if (hole) holes[h] = t;
    if (moved) sources[s] = t;
    if (stays && t < a.keep) {
      nw[t] = w[t];
      if (kept != nullptr) kept[t] = t;
    }
  }
  __syncthreads();  // (holes and sources are as many: `keep` rows stay)
  for (int k = tid; k < nh; k += kThreads) {
    nw[holes[k]] = w[sources[k]];
    if (kept != nullptr) kept[holes[k]] = sources[k];
  }
  if (tid == 0) moves[0] = nh;
}

// One moved row of a unit, K and V, per workgroup and round.
__global__ __launch_bounds__(kWave) void evict_move_kernel(EvictArgs a, CachePtrs p, int row_bytes, int64_t cache_row_bytes, int64_t cache_batch_bytes) {
  const int unit = blockIdx.x, b = unit / a.Hkv % a.B, g = unit % a.Hkv, l = unit / a.Hkv / a.B;
  const int32_t *moves = a.moves + int64_t(unit) * (1 + 2 * a.room);
  const int n = moves[0];
  char *base = p.at[2 * l + blockIdx.z] + int64_t(b) * cache_batch_bytes + int64_t(g) * row_bytes;
  for (int k = blockIdx.y; k < n; k += gridDim.y) {
    const int dst = moves[1 + k], src = moves[1 + a.room + k];
    for (int o = threadIdx.x * 16; o < row_bytes; o += kWave * 16)
      *reinterpret_cast<u32x4 *>(base + dst * cache_row_bytes + o) = *reinterpret_cast<const u32x4 *>(base + src * cache_row_bytes + o);
  }
}

__global__ void evict_length_kernel(int B, int C, int keep, int high, const int32_t *prefix_len, int32_t *new_len) {
  const int b = blockIdx.x * blockDim.x + threadIdx.x;
  if (b >= B) return;
  const int P = min(max(prefix_len[b], 0), C);
  new_len[b] = P > high ? keep : P;
}

// rows that can move at most
int32_t room_of(const lsp_evict_desc *d) { return d->keep < d->C - d->keep ? d->keep : d->C - d->keep; }
int32_t layers_at_once(int32_t n) { return n < kMaxLayersPerLaunch ? n : kMaxLayersPerLaunch; }

int32_t check(const lsp_evict_desc *d) {
  LSP_CHECK_ARG(d != nullptr, "lsp_kv_evict: null descriptor");
  LSP_CHECK_ARG(d->kv_dtype == LSP_F32 || d->kv_dtype == LSP_BF16, "lsp_kv_evict: unknown kv_dtype %d", d->kv_dtype);
  LSP_CHECK_ARG(d->B > 0 && d->B <= 65535 && d->Hkv > 0 && d->Hkv <= 65535 && d->D > 0 && d->C > 0 && d->num_layers > 0, "lsp_kv_evict: bad dimension");
  LSP_CHECK_ARG(d->keep > 0 && d->keep <= d->C, "lsp_kv_evict: keep must be 1..C (got %d, C = %d)", d->keep, d->C);
  LSP_CHECK_ARG(d->high >= d->keep, "lsp_kv_evict: high = %d is below keep = %d", d->high, d->keep);
  LSP_CHECK_ARG(d->first >= 0 && d->recent >= 0 && int64_t(d->first) + d->recent <= d->keep,
                "lsp_kv_evict: first + recent must be 0..keep (got %d + %d of %d)", d->first, d->recent, d->keep);
  LSP_CHECK_ARG(int64_t(d->B) * d->Hkv * layers_at_once(d->num_layers) < int64_t(1) << 31, "lsp_kv_evict: too many heads");
  return LSP_OK;
}

}  // namespace
}  // namespace lsp

extern "C" size_t lsp_kv_evict_workspace_bytes(const lsp_evict_desc *d) {
  if (lsp::check(d) != LSP_OK) return 0;
  return size_t(lsp::layers_at_once(d->num_layers)) * d->B * d->Hkv * (1 + 2 * size_t(lsp::room_of(d))) * sizeof(int32_t);
}

extern "C" int32_t lsp_kv_evict(const lsp_evict_desc *d, const float *weights, const int32_t *prefix_len, void *const *k_cache_layers,
                                void *const *v_cache_layers, float *new_weights, int32_t *new_len, int32_t *kept_index, void *workspace,
                                size_t workspace_bytes, void *stream) {
  using namespace lsp;
  const int32_t rc = check(d);
  if (rc != LSP_OK) return rc;
  LSP_CHECK_ARG(weights && prefix_len && k_cache_layers && v_cache_layers && new_weights && new_len, "lsp_kv_evict: null pointer");
  const int64_t es = int64_t(elem_size(d->kv_dtype)), row_bytes = d->D * es, cache_row_bytes = d->Hkv * row_bytes;
  LSP_CHECK_ARG(row_bytes % 16 == 0, "lsp_kv_evict: a head's row of %lld bytes is not a multiple of 16", (long long)row_bytes);
  const int64_t cache_bb = d->cache_batch_stride ? d->cache_batch_stride * es : d->C * cache_row_bytes;
  LSP_CHECK_ARG(cache_bb % 16 == 0 && cache_bb >= d->C * cache_row_bytes, "lsp_kv_evict: bad batch stride");
  for (int l = 0; l < d->num_layers; ++l) {
    LSP_CHECK_ARG(k_cache_layers[l] && v_cache_layers[l], "lsp_kv_evict: null K/V pointer in layer %d", l);
    LSP_CHECK_ARG(aligned16(k_cache_layers[l]) && aligned16(v_cache_layers[l]), "lsp_kv_evict: K/V pointer of layer %d is not 16-byte aligned", l);
  }
  const size_t need = lsp_kv_evict_workspace_bytes(d);
  if (workspace == nullptr || workspace_bytes < need || !aligned16(workspace)) {
    set_error("lsp_kv_evict: workspace of %zu bytes (16-byte aligned) required, got %zu", need, workspace_bytes);
    return LSP_ERR_WORKSPACE;
  }
  hipStream_t st = static_cast<hipStream_t>(stream);
  EvictArgs a = {weights, new_weights, kept_index, prefix_len, static_cast<int32_t *>(workspace), d->B, d->Hkv, d->C, d->keep, d->high, d->first, d->recent, room_of(d)};
  for (int l0 = 0; l0 < d->num_layers; l0 += kMaxLayersPerLaunch) {
    const int nl = layers_at_once(d->num_layers - l0);
    const int64_t units = int64_t(l0) * d->B * d->Hkv;
    a.weights = weights + units * d->C;
    a.new_weights = new_weights + units * d->C;
    a.kept_index = kept_index == nullptr ? nullptr : kept_index + units * d->keep;
    CachePtrs p;
    for (int l = 0; l < kMaxLayersPerLaunch; ++l) {
      const int s = l < nl ? l0 + l : l0;
      p.at[2 * l] = static_cast<char *>(k_cache_layers[s]);
      p.at[2 * l + 1] = static_cast<char *>(v_cache_layers[s]);
    }
    evict_select_kernel<<<dim3(d->Hkv, d->B, nl), kThreads, 0, st>>>(a);
    LSP_CHECK_LAUNCH("lsp_kv_evict: selection launch");
    evict_move_kernel<<<dim3(nl * d->B * d->Hkv, 16, 2), kWave, 0, st>>>(a, p, int(row_bytes), cache_row_bytes, cache_bb);
    LSP_CHECK_LAUNCH("lsp_kv_evict: copy launch");
  }
  evict_length_kernel<<<(d->B + 255) / 256, 256, 0, st>>>(d->B, d->C, d->keep, d->high, prefix_len, new_len);
  LSP_CHECK_LAUNCH("lsp_kv_evict: length launch");
  return LSP_OK;
}
