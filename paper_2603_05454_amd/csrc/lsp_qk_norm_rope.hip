// lsp_qk_norm_rope: norms of heads and position rotation of a step's queries and keys in one pass.
//
// y = x rsqrt(mean(x^2) + eps) w over a head, then pairs (y_a, y_b) -> (y_a cos t - y_b sin t, y_b cos t + y_a sin t) with t = position * inv_freq[i].
// Bound by the bytes of the rows, read once and written once.  All heads of a row turn by the same angles: a workgroup works them out once, a thread
// each, into LDS.  The product position * inv_freq is taken in 64 bits (in 32 the angle of position 100 000 is off by up to 0.004) and reduced there to
// an eighth of a turn about a quarter; sine and cosine of that are their power series in 32 bits, to x^9 and x^10, whose next terms are below
// 2e-9 and 1.2e-10.  Everything behind is 32 bits, rounded once.  8192 rows of 64 heads of 128, 268 MB in and out, take 41 us (6.5 TB/s); one row 2.6 us.
#include <math.h>

#include "lsp_q8.h"

namespace lsp {
namespace {

constexpr int kThreads = 256;

struct RopeArgs {
  const char *q, *k;
  char *q_out, *k_out;
  const float *q_weight, *k_weight, *inv_freq;
  const int32_t *prefix_len, *suffix_len, *positions;
  int32_t S, Hq, heads, half;  // half: pairs that turn
  float eps;
  int64_t qs[3], ks[3], qo[3], ko[3];  // bytes: sequence, row, head
};

// cos and sin of position * frequency
__device__ __forceinline__ f32x2 turn(int position, float frequency) {
  const double t = double(position) * double(frequency), quarters = rint(t * 0.63661977236758134308);
  // pi / 2 in two parts
  const float x = float(fma(-quarters, 6.123233995736766036e-17, fma(-quarters, 1.5707963267948965580, t)));
  const int n = int(int64_t(quarters) & 3);
  const float z = x * x;
  const float s = fmaf(x * z, fmaf(z, fmaf(z, fmaf(z, 1.f / 362880.f, -1.f / 5040.f), 1.f / 120.f), -1.f / 6.f), x);
  const float c = fmaf(z, fmaf(z, fmaf(z, fmaf(z, fmaf(z, -1.f / 3628800.f, 1.f / 40320.f), -1.f / 720.f), 1.f / 24.f), -0.5f), 1.f);
  const float a = n & 1 ? s : c, b = n & 1 ? c : s;
  return f32x2{(n + 1) & 2 ? -a : a, n & 2 ? -b : b};
}

template <typename T>
struct Piece;  // 16 bytes of a row
template <>
struct Piece<uint16_t> {
  static constexpr int kN = 8;
  static __device__ __forceinline__ void load(const char *p, float *x) {
    const u32x4 w = *reinterpret_cast<const u32x4 *>(p);
#pragma unroll
    for (int k = 0; k < 4; ++k) x[2 * k] = bf16_lo(w[k]), x[2 * k + 1] = bf16_hi(w[k]);
  }
  static __device__ __forceinline__ void store(char *p, const float *x) {
    bf16x8 v;
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = __bf16(x[k]);
    *reinterpret_cast<bf16x8 *>(p) = v;
  }
};
template <>
struct Piece<float> {
  static constexpr int kN = 4;
  static __device__ __forceinline__ void load(const char *p, float *x) {
    const f32x4 w = *reinterpret_cast<const f32x4 *>(p);
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] = w[k];
  }
  static __device__ __forceinline__ void store(char *p, const float *x) { *reinterpret_cast<f32x4 *>(p) = f32x4{x[0], x[1], x[2], x[3]}; }
};

// A thread has two pieces of a head, those that turn with each other: pieces j and j + R/2 elements on, or neighbours where neighbours are paired (and
// where nothing turns).  ROWS rows of a sequence to a workgroup.
template <typename T, int D, int ROWS>
__global__ __launch_bounds__(kThreads) void norm_rope_kernel(RopeArgs a, bool interleaved) {
  constexpr int N = Piece<T>::kN, kLanes = D / (2 * N);
  __shared__ f32x2 s_turn[ROWS * D / 2];
  const int b = blockIdx.y, u0 = blockIdx.x * ROWS;
  const int n = a.suffix_len ? min(max(a.suffix_len[b], 0), a.S) : a.S, rows = min(ROWS, n - u0);
  if (rows <= 0) return;
  const int P = a.prefix_len ? a.prefix_len[b] : 0;
  for (int i = threadIdx.x; i < rows * a.half; i += kThreads) {
    const int r = ROWS == 1 ? 0 : i / a.half, p = i - r * a.half;
    s_turn[r * (D / 2) + p] = turn(a.positions ? a.positions[int64_t(b) * a.S + u0 + r] : P + u0 + r, a.inv_freq[p]);
  }
  __syncthreads();
  const int j = threadIdx.x % kLanes;
  // elements of a head that the pieces begin with
  const int turning = a.half / N;     // threads of a head whose pieces turn
  const bool turns = j < turning, apart = turns && !interleaved;
  const int d0 = apart ? j * N : 2 * j * N, d1 = apart ? d0 + a.half : d0 + N;
  const int items = rows * a.heads;
  for (int it = threadIdx.x / kLanes; it < items; it += kThreads / kLanes) {
    const int r = ROWS == 1 ? 0 : it / a.heads, h = it - r * a.heads, u = u0 + r;
    const bool key = h >= a.Hq;
    const char *from = key ? a.k + b * a.ks[0] + u * a.ks[1] + (h - a.Hq) * a.ks[2] : a.q + b * a.qs[0] + u * a.qs[1] + h * a.qs[2];
    char *to = key ? a.k_out + b * a.ko[0] + u * a.ko[1] + (h - a.Hq) * a.ko[2] : a.q_out + b * a.qo[0] + u * a.qo[1] + h * a.qo[2];
    float x[2 * N];
    Piece<T>::load(from + d0 * int(sizeof(T)), x);
    Piece<T>::load(from + d1 * int(sizeof(T)), x + N);
    const float *w = key ? a.k_weight : a.q_weight;
    if (w) {
      float sum = 0.f;
#pragma unroll
      for (int e = 0; e < 2 * N; ++e) sum = fmaf(x[e], x[e], sum);
#pragma unroll
      for (int m = 1; m < kLanes; m <<= 1) sum += __shfl_xor(sum, m);
      const float f = 1.f / sqrtf(sum * (1.f / D) + a.eps);
#pragma unroll
      for (int e = 0; e < N; ++e) x[e] *= f * w[d0 + e], x[N + e] *= f * w[d1 + e];
    }
    if (turns) {
      const f32x2 *t = s_turn + r * (D / 2) + j * N;
      if (interleaved) {
#pragma unroll
        for (int e = 0; e < N; ++e) {
          const float p = x[2 * e], q = x[2 * e + 1];
          x[2 * e] = p * t[e][0] - q * t[e][1];
          x[2 * e + 1] = q * t[e][0] + p * t[e][1];
        }
      } else {
#pragma unroll
        for (int e = 0; e < N; ++e) {
          const float p = x[e], q = x[N + e];
          x[e] = p * t[e][0] - q * t[e][1];
          x[N + e] = q * t[e][0] + p * t[e][1];
        }
      }
    }
    Piece<T>::store(to + d0 * int(sizeof(T)), x);
    Piece<T>::store(to + d1 * int(sizeof(T)), x + N);
  }
}

template <typename T>
void launch(const RopeArgs &a, int B, int D, bool interleaved, hipStream_t st) {
  // A workgroup has one row where its heads are work for all threads (8192 rows of 64 heads of 128: 41 us, with four rows 44; 1024 of 32 heads 5.6 and 7.4), or
  // where rows are few (512 of 10 heads: 4.0 and 4.7); else four, which share the angles' latency (8192 rows of 10 heads: 12.5 with one, 10.2).
  // (A launch has fewer than 2^32 threads in x: the most rows that the call takes are four to a workgroup in any case.)
  const bool few = (a.heads * (D * int64_t(sizeof(T)) / 32) >= kThreads || int64_t(B) * a.S <= 2048) && int64_t(a.S) * kThreads < int64_t(1) << 32;
  const dim3 grid(unsigned(few ? a.S : (a.S + 3) / 4), unsigned(B));
  if (D == 64) {
    if (few) norm_rope_kernel<T, 64, 1><<<grid, kThreads, 0, st>>>(a, interleaved);
    else norm_rope_kernel<T, 64, 4><<<grid, kThreads, 0, st>>>(a, interleaved);
  } else {
    if (few) norm_rope_kernel<T, 128, 1><<<grid, kThreads, 0, st>>>(a, interleaved);
    else norm_rope_kernel<T, 128, 4><<<grid, kThreads, 0, st>>>(a, interleaved);
  }
}

// outer strides in elements, all 0 for a dense buffer -> bytes
bool byte_strides(const int64_t in[3], int64_t S, int64_t H, int64_t D, int64_t es, int64_t out[3]) {
  int64_t s[3] = {S * H * D, H * D, D};
  if (in[0] != 0 || in[1] != 0 || in[2] != 0) {
    if (in[2] < D || in[1] <= 0 || in[0] < 0) return false;
    for (int k = 0; k < 3; ++k) s[k] = in[k];
  }
  for (int k = 0; k < 3; ++k) {
    out[k] = s[k] * es;
    if (out[k] % 16 != 0) return false;
  }
  return true;
}

}  // namespace
}  // namespace lsp

extern "C" int32_t lsp_qk_norm_rope(const lsp_qk_norm_rope_desc *d, const void *q, const void *k, const float *q_weight, const float *k_weight,
                                    const float *inv_freq, const int32_t *prefix_len, const int32_t *suffix_len, const int32_t *positions,
                                    void *q_out, void *k_out, void *stream) {
  using namespace lsp;
  const char *what = "lsp_qk_norm_rope";
  LSP_CHECK_ARG(d != nullptr, "%s: null descriptor", what);
  LSP_CHECK_ARG(d->dtype == LSP_F32 || d->dtype == LSP_BF16, "%s: unknown dtype %d", what, d->dtype);
  LSP_CHECK_ARG(d->B > 0 && d->S > 0 && d->Hq > 0 && d->Hkv > 0 && d->D > 0, "%s: non-positive dimension", what);
  LSP_CHECK_ARG(d->B <= 65535 && d->Hq <= 65535 && d->Hkv <= 65535 && d->S <= 1 << 24, "%s: B, Hq and Hkv must be <= 65535, S <= 2^24", what);
  if (d->D != 64 && d->D != 128) {
    set_error("%s: head_dim %d (64 and 128 are built)", what, d->D);
    return LSP_ERR_UNSUPPORTED;
  }
  LSP_CHECK_ARG(d->R >= 0 && d->R <= d->D && d->R % 16 == 0, "%s: R must be a multiple of 16 from 0 to D", what);
  LSP_CHECK_ARG(d->eps >= 0.f && isfinite(d->eps), "%s: bad eps", what);
  LSP_CHECK_ARG(q && k && q_out && k_out && (inv_freq || d->R == 0), "%s: null pointer", what);
  LSP_CHECK_ARG((q_weight == nullptr) == (k_weight == nullptr), "%s: the norms' weights come together", what);
  LSP_CHECK_ARG(aligned16(q) && aligned16(k) && aligned16(q_out) && aligned16(k_out), "%s: pointers must be 16-byte aligned", what);
  RopeArgs a;
  const int64_t es = int64_t(elem_size(d->dtype));
  LSP_CHECK_ARG(byte_strides(d->q_stride, d->S, d->Hq, d->D, es, a.qs) && byte_strides(d->k_stride, d->S, d->Hkv, d->D, es, a.ks) &&
                    byte_strides(d->q_out_stride, d->S, d->Hq, d->D, es, a.qo) && byte_strides(d->k_out_stride, d->S, d->Hkv, d->D, es, a.ko),
                "%s: bad strides, or no multiples of 16 bytes", what);
  LSP_CHECK_ARG(d->B == 1 || (a.qo[0] > 0 && a.ko[0] > 0), "%s: an output must not be shared by sequences", what);
  a.q = static_cast<const char *>(q); a.k = static_cast<const char *>(k);
  a.q_out = static_cast<char *>(q_out); a.k_out = static_cast<char *>(k_out);
  a.q_weight = q_weight; a.k_weight = k_weight; a.inv_freq = inv_freq;
  a.prefix_len = prefix_len; a.suffix_len = suffix_len; a.positions = positions;
  a.S = d->S; a.Hq = d->Hq; a.heads = d->Hq + d->Hkv; a.half = d->R / 2; a.eps = d->eps;
  if (d->dtype == LSP_F32) launch<float>(a, d->B, d->D, d->interleaved != 0, static_cast<hipStream_t>(stream));
  else launch<uint16_t>(a, d->B, d->D, d->interleaved != 0, static_cast<hipStream_t>(stream));
  LSP_CHECK_LAUNCH("lsp_qk_norm_rope: launch");
  return LSP_OK;
}
