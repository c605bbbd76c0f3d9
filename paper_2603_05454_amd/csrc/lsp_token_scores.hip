// lsp_token_scores: log probability of a given token, entropy and the most likely alternatives of every active row of the logits.
//
// With m the row's maximum, s = sum exp(z - m) and t = sum exp(z - m) (z - m):
//   log p(v) = z[v] - m - log s          entropy = log s - t / s
// and the alternatives are the first K entries in the order (value descending, index ascending).
#include <float.h>
#include <limits.h>

#include "lsp_common.h"

namespace lsp {
namespace {

constexpr int kMaxAlt = 32;
constexpr int kThreads = 256;

__device__ __forceinline__ float element(const float *p) { return *p; }
__device__ __forceinline__ float element(const uint16_t *p) { return bf16_to_f32(*p); }

// One workgroup per row, a pass for the statistics and one for each alternative.
template <typename T>
__global__ __launch_bounds__(kThreads) void token_scores_kernel(const T *__restrict__ logits, int S, int V, int64_t row_stride,
                                                                int64_t batch_stride, const int32_t *__restrict__ suffix_len,
                                                                const int32_t *__restrict__ token_id, int K, float *__restrict__ logprob,
                                                                float *__restrict__ entropy, int32_t *__restrict__ alt_id,
                                                                float *__restrict__ alt_logprob) {
  __shared__ float s_a[kThreads], s_b[kThreads];
  __shared__ int s_i[kThreads];
  const int i = blockIdx.x, b = blockIdx.y, tid = threadIdx.x;
  if (suffix_len != nullptr && i >= suffix_len[b]) return;
  const T *z = logits + int64_t(b) * batch_stride + int64_t(i) * row_stride;
  const int64_t o = int64_t(b) * S + i;

  float m = -INFINITY;
  for (int v = tid; v < V; v += kThreads) m = fmaxf(m, element(z + v));
  s_a[tid] = m;
  __syncthreads();
  for (int h = kThreads / 2; h > 0; h >>= 1) {
    if (tid < h) s_a[tid] = fmaxf(s_a[tid], s_a[tid + h]);
    __syncthreads();
  }
  m = s_a[0];
  __syncthreads();
  float s = 0.f, t = 0.f;
  for (int v = tid; v < V; v += kThreads) {
    const float x = element(z + v);
    if (x == -INFINITY) continue;  // probability 0 (and, where nothing else is there, no difference to it)
    const float e = __expf(x - m);
    s += e;
    if (e > 0.f) t += e * (x - m);
  }
  s_a[tid] = s;
  s_b[tid] = t;
  __syncthreads();
  for (int h = kThreads / 2; h > 0; h >>= 1) {
    if (tid < h) s_a[tid] += s_a[tid + h], s_b[tid] += s_b[tid + h];
    __syncthreads();
  }
  s = s_a[0];
  t = s_b[0];
  __syncthreads();
  const bool none = m == -INFINITY;
  const float log_s = __logf(s);
  auto log_p = [&](float x) { return none || x == -INFINITY ? -INFINITY : (x - m) - log_s; };
  if (tid == 0) {
    entropy[o] = none ? 0.f : log_s - t / s;
    if (token_id != nullptr) {
      const int id = token_id[o];
      logprob[o] = id < 0 || id >= V ? -INFINITY : log_p(element(z + id));
    }
  }
  float last = INFINITY;  // the alternative found before
  int last_i = -1;
  for (int k = 0; k < K; ++k) {
    float x = -INFINITY;
    int at = INT_MAX;
    for (int v = tid; v < V; v += kThreads) {
      const float y = element(z + v);
      const bool left = y < last || (y == last && v > last_i);
      if (left && (y > x || (y == x && v < at))) x = y, at = v;
    }
    s_a[tid] = x;
    s_i[tid] = at;
    __syncthreads();
    for (int h = kThreads / 2; h > 0; h >>= 1) {
      if (tid < h && (s_a[tid + h] > s_a[tid] || (s_a[tid + h] == s_a[tid] && s_i[tid + h] < s_i[tid]))) {
        s_a[tid] = s_a[tid + h];
        s_i[tid] = s_i[tid + h];
      }
      __syncthreads();
    }
    last = s_a[0];
    last_i = s_i[0];
    __syncthreads();
    if (tid == 0) {
      alt_id[o * K + k] = last_i == INT_MAX ? -1 : last_i;
      alt_logprob[o * K + k] = last_i == INT_MAX ? -INFINITY : log_p(last);
    }
  }
}

}  // namespace
}  // namespace lsp

extern "C" size_t lsp_token_scores_workspace_bytes(int32_t B, int32_t S, int32_t V, int32_t num_alt) { return 0; }

extern "C" int32_t lsp_token_scores(int32_t dtype, const void *logits, int32_t B, int32_t S, int32_t V, int64_t row_stride,
                                    int64_t batch_stride, const int32_t *suffix_len, const int32_t *token_id, int32_t num_alt,
                                    float *logprob, float *entropy, int32_t *alt_id, float *alt_logprob, void *workspace,
                                    size_t workspace_bytes, void *stream) {
  using namespace lsp;
  LSP_CHECK_ARG(dtype == LSP_F32 || dtype == LSP_BF16, "lsp_token_scores: unknown dtype %d", dtype);
  LSP_CHECK_ARG(B > 0 && S > 0 && V > 0, "lsp_token_scores: need B>0, S>0, V>0 (got %d %d %d)", B, S, V);
  LSP_CHECK_ARG(B <= 65535 && S <= 65535, "lsp_token_scores: B and S must be <= 65535");
  LSP_CHECK_ARG(num_alt >= 0 && num_alt <= kMaxAlt, "lsp_token_scores: num_alt must be 0..%d (got %d)", kMaxAlt, num_alt);
  LSP_CHECK_ARG(logits && entropy, "lsp_token_scores: null pointer");
  LSP_CHECK_ARG((token_id != nullptr) == (logprob != nullptr), "lsp_token_scores: token_id and logprob come together");
  LSP_CHECK_ARG(num_alt == 0 || (alt_id && alt_logprob), "lsp_token_scores: alternatives need alt_id and alt_logprob");
  if (row_stride == 0) row_stride = V;
  if (batch_stride == 0) batch_stride = int64_t(S) * row_stride;
  LSP_CHECK_ARG(row_stride >= V && batch_stride >= 0, "lsp_token_scores: bad strides");
  LSP_CHECK_ARG((reinterpret_cast<uintptr_t>(logits) & (elem_size(dtype) - 1)) == 0, "lsp_token_scores: logits misaligned");
  hipStream_t st = static_cast<hipStream_t>(stream);
  const dim3 grid(S, B);
  if (dtype == LSP_BF16)
    token_scores_kernel<uint16_t><<<grid, kThreads, 0, st>>>(static_cast<const uint16_t *>(logits), S, V, row_stride, batch_stride, suffix_len,
                                                             token_id, num_alt, logprob, entropy, alt_id, alt_logprob);
  else
    token_scores_kernel<float><<<grid, kThreads, 0, st>>>(static_cast<const float *>(logits), S, V, row_stride, batch_stride, suffix_len,
                                                          token_id, num_alt, logprob, entropy, alt_id, alt_logprob);
  LSP_CHECK_LAUNCH("lsp_token_scores: launch");
  return LSP_OK;
}
