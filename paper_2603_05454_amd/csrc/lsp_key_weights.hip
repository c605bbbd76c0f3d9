// lsp_attn_key_weights: the attention mass that every key received from the active queries of its group.
//
// With c = scale log2(e) and L[h,i] the base-2 logarithm of the sum over all keys of 2^(c q.k):
//   mass[g,t] = sum over heads h of group g and rows i < N of 2^(c q[i,h].k[t,g] - L[h,i])
// Two kernels: one computes L of every row, the other the sums down the columns, each from its own product of queries and
// keys.  (The products kept instead would be 1.3e9 numbers a layer at 8 x 1024 rows of 32 heads on 4096.)
#include <math.h>

#include "lsp_attn.h"

namespace lsp {
namespace {

constexpr float kLog2e = 1.4426950408889634f;

struct WeightArgs {
  const int32_t *prefix_len, *suffix_len;
  int32_t B, S, Hq, Hkv, D, C, rep;
  float scale, decay;
  int64_t qs[3], ks[3], cs[3];
  float *row_log;  // [layers of the launch, B, Hq, S]
  float *weights;  // of the launch's first layer: [layers, B, Hkv, C]
};
struct WeightLayers {
  const void *q[kMaxAttnLayers], *k_suf[kMaxAttnLayers], *k_cache[kMaxAttnLayers];
};

__device__ __forceinline__ float element(const float *p) { return *p; }
__device__ __forceinline__ float element(const uint16_t *p) { return bf16_to_f32(*p); }

template <typename T>
__device__ __forceinline__ const T *key_row(const WeightArgs &a, const WeightLayers &L, int l, int b, int g, int t, int P) {
  if (t < P) return static_cast<const T *>(L.k_cache[l]) + b * a.cs[0] + int64_t(t) * a.cs[1] + g * a.cs[2];
  return static_cast<const T *>(L.k_suf[l]) + b * a.ks[0] + int64_t(t - P) * a.ks[1] + g * a.ks[2];
}
template <typename T>
__device__ __forceinline__ float dot(const T *x, const T *y, int D) {
  float s = 0.f;
  for (int d = 0; d < D; ++d) s = fmaf(element(x + d), element(y + d), s);
  return s;
}

// One wave per row.
template <typename T>
__global__ __launch_bounds__(kWave) void row_log_kernel(WeightArgs a, WeightLayers L) {
  const int i = blockIdx.x, h = blockIdx.y % a.Hq, b = blockIdx.y / a.Hq, l = blockIdx.z;
  const int N = min(max(a.suffix_len[b], 0), a.S), P = min(max(a.prefix_len[b], 0), a.C);
  if (i >= N) return;
  const T *q = static_cast<const T *>(L.q[l]) + b * a.qs[0] + i * a.qs[1] + h * a.qs[2];
  float m = -INFINITY, s = 0.f;
  for (int t = threadIdx.x; t < P + N; t += kWave) {
    const float x = dot(q, key_row<T>(a, L, l, b, h / a.rep, t, P), a.D) * a.scale * kLog2e;
    const float n = fmaxf(m, x);
    s = s * exp2f(m - n) + exp2f(x - n);
    m = n;
  }
  float M = m;
  for (int k = 1; k < kWave; k <<= 1) M = fmaxf(M, __shfl_xor(M, k));
  s *= exp2f(m - M);
  for (int k = 1; k < kWave; k <<= 1) s += __shfl_xor(s, k);
  if (threadIdx.x == 0) a.row_log[((int64_t(l) * a.B + b) * a.Hq + h) * a.S + i] = M + log2f(s);
}

// One key per lane.
template <typename T>
__global__ __launch_bounds__(kWave) void key_sum_kernel(WeightArgs a, WeightLayers L) {
  const int t = blockIdx.x * kWave + threadIdx.x, g = blockIdx.y % a.Hkv, b = blockIdx.y / a.Hkv, l = blockIdx.z;
  const int N = min(max(a.suffix_len[b], 0), a.S), P = min(max(a.prefix_len[b], 0), a.C);
  if (N == 0 || t >= min(P + N, a.C)) return;
  const T *k = key_row<T>(a, L, l, b, g, t, P);
  float sum = 0.f;
  for (int h = g * a.rep; h < (g + 1) * a.rep; ++h)
    for (int i = 0; i < N; ++i) {
      const T *q = static_cast<const T *>(L.q[l]) + b * a.qs[0] + i * a.qs[1] + h * a.qs[2];
      sum += exp2f(dot(q, k, a.D) * a.scale * kLog2e - a.row_log[((int64_t(l) * a.B + b) * a.Hq + h) * a.S + i]);
    }
  float *w = a.weights + ((int64_t(l) * a.B + b) * a.Hkv + g) * a.C + t;
  *w = t < P && a.decay != 0.f ? a.decay * *w + sum : sum;
}

int layers_at_once(int32_t n) { return n < kMaxAttnLayers ? n : kMaxAttnLayers; }
size_t row_log_bytes(const lsp_attn_desc *d, int32_t num_layers) {
  return size_t(layers_at_once(num_layers)) * d->B * d->Hq * d->S * sizeof(float);
}

}  // namespace
}  // namespace lsp

extern "C" size_t lsp_attn_key_weights_workspace_bytes(const lsp_attn_desc *d, int32_t num_layers) {
  if (d == nullptr || num_layers <= 0 || d->B <= 0 || d->S <= 0 || d->Hq <= 0) return 0;
  return lsp::row_log_bytes(d, num_layers);
}

extern "C" int32_t lsp_attn_key_weights(const lsp_attn_desc *d, int32_t num_layers, const void *const *q_layers,
                                        const void *const *k_suf_layers, const void *const *k_cache_layers,
                                        const int32_t *prefix_len, const int32_t *suffix_len, float decay, float *weights,
                                        void *workspace, size_t workspace_bytes, void *stream) {
  using namespace lsp;
  AttnArgs at;
  const int32_t rc = check_attn(d, at);
  if (rc != LSP_OK) return rc;
  LSP_CHECK_ARG(num_layers > 0, "lsp_attn_key_weights: num_layers must be positive");
  LSP_CHECK_ARG(q_layers && k_suf_layers && k_cache_layers && prefix_len && suffix_len && weights, "lsp_attn_key_weights: null pointer");
  LSP_CHECK_ARG(decay >= 0.f && decay <= 1.f, "lsp_attn_key_weights: decay must be in [0, 1] (got %g)", double(decay));
  LSP_CHECK_ARG(int64_t(d->B) * d->Hq <= 65535, "lsp_attn_key_weights: B * Hq must be <= 65535");
  for (int l = 0; l < num_layers; ++l) {
    LSP_CHECK_ARG(q_layers[l] && k_suf_layers[l] && k_cache_layers[l], "lsp_attn_key_weights: null operand in layer %d", l);
    LSP_CHECK_ARG(aligned16(q_layers[l]) && aligned16(k_suf_layers[l]) && aligned16(k_cache_layers[l]),
                  "lsp_attn_key_weights: operands of layer %d must be 16-byte aligned", l);
  }
  if (d->D != 64 && d->D != 128) {
    set_error("lsp_attn_key_weights: head_dim %d is not built (64 or 128)", d->D);
    return LSP_ERR_UNSUPPORTED;
  }
  const size_t need = row_log_bytes(d, num_layers);
  if (workspace == nullptr || workspace_bytes < need || !aligned16(workspace)) {
    set_error("lsp_attn_key_weights: workspace of %zu bytes (16-byte aligned) required, got %zu", need, workspace_bytes);
    return LSP_ERR_WORKSPACE;
  }
  WeightArgs a = {prefix_len, suffix_len, at.B, at.S, at.Hq, at.Hkv, at.D, at.C, at.Hq / at.Hkv, at.scale, decay, {}, {}, {}, static_cast<float *>(workspace), weights};
  for (int k = 0; k < 3; ++k) a.qs[k] = at.qs[k], a.ks[k] = at.ks[k], a.cs[k] = at.cs[k];
  hipStream_t st = static_cast<hipStream_t>(stream);
  const int keys = at.C;
  for (int l0 = 0; l0 < num_layers; l0 += kMaxAttnLayers) {
    const int nl = layers_at_once(num_layers - l0);
    WeightLayers L;
    for (int l = 0; l < kMaxAttnLayers; ++l) {
      const int s = l < nl ? l0 + l : l0;
      L.q[l] = q_layers[s]; L.k_suf[l] = k_suf_layers[s]; L.k_cache[l] = k_cache_layers[s];
    }
    a.weights = weights + int64_t(l0) * at.B * at.Hkv * at.C;
    const dim3 rows(at.S, at.B * at.Hq, nl), cols((keys + kWave - 1) / kWave, at.B * at.Hkv, nl);
    if (d->dtype == LSP_BF16) {
      row_log_kernel<uint16_t><<<rows, kWave, 0, st>>>(a, L);
      LSP_CHECK_LAUNCH("lsp_attn_key_weights: row launch");
      key_sum_kernel<uint16_t><<<cols, kWave, 0, st>>>(a, L);
    } else {
      row_log_kernel<float><<<rows, kWave, 0, st>>>(a, L);
      LSP_CHECK_LAUNCH("lsp_attn_key_weights: row launch");
      key_sum_kernel<float><<<cols, kWave, 0, st>>>(a, L);
    }
    LSP_CHECK_LAUNCH("lsp_attn_key_weights: column launch");
  }
  return LSP_OK;
}
