// lsp_kv_append_q8, lsp_kv_read_q8: committed rows quantised as they are written into a cache, and read back.
//
// A block is 32 rows of one head, one wave's.  With a = the largest finite magnitude of its new rows and 448 that of e4m3, E is the smallest
// exponent byte with a <= 448 * 2^(E - 127); powers of two cost an e4m3 value nothing (its own exponent takes them up) and make multiplying by a
// scale, and rounding again under a larger one, exact but for what becomes subnormal.  Bound by the bytes: 16 bits read and 8 written for each number, or the other way
// round (the prompt below: 6.0 TB/s written, 5.1 read back; a large copy reaches 4.9).
#include <type_traits>

#include "lsp_q8.h"

namespace lsp {

int32_t check_q8(const char *what, const lsp_attn_desc *d, bool queries, AttnArgs &a) {
  LSP_CHECK_ARG(d != nullptr, "%s: null descriptor", what);
  lsp_attn_desc c = *d;
  if (!queries) {
    c.Hq = c.Hkv;
    for (int k = 0; k < 3; ++k) c.q_stride[k] = c.o_stride[k] = 0;
    c.scale = 0.f;
  }
  const int32_t rc = check_attn(&c, a);
  if (rc != LSP_OK) return rc;
  LSP_CHECK_ARG(a.cs[0] % 16 == 0 && a.cs[1] % 16 == 0 && a.cs[2] % 16 == 0, "%s: cache strides must be multiples of 16 bytes", what);
  LSP_CHECK_ARG(a.C <= 1 << 30 && a.S <= 1 << 30 && (a.S / kQ8Block + int64_t(2)) * a.Hkv < int64_t(1) << 31,
                "%s: C and S must be <= 2^30, S / 32 * Hkv < 2^31", what);
  if (a.D != 64 && a.D != 128) {
    set_error("%s: head_dim %d (64 and 128 are built)", what, a.D);
    return LSP_ERR_UNSUPPORTED;
  }
  return LSP_OK;
}

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
// Workgroups of a launch, where there is work for them: sixteen waves to a SIMD's worth are in flight or next.
constexpr int64_t kGroups = 4096;

struct KvArgs {
  const int32_t *from, *to;  // append: commit_len and prefix_len; read: first and last row
  int32_t B, S, Hkv, C, blocks;
  Div by_heads;
  int64_t ss[3], cs[3];  // bytes: sequence, row, head of a suffix (or output) buffer, of a cache
};

// eight numbers of a row
struct Eight {
  float x[8];
};
// ONCE: nontemporal.  Where the buffers are larger than the last cache (256 MB), what a call reads or writes once need not stay there: 4 x 4096 rows of 32 heads
// in two layers, 0.8 GB, are appended in 131 to 135 us so and 148 without, and appended and read back in 294 and 314; where they are smaller it is better kept: 64
// rows of 8 sequences in four layers 36 and 31 us.  It goes by the size of the buffers: how many of their rows a call commits only the device knows, and a step that commits a
// few rows of large buffers goes nontemporally as well.  The reading's own writes are plain ones: 156 us against 167.
constexpr int64_t kLastCache = int64_t(256) << 20;
template <bool ONCE, typename V>
__device__ __forceinline__ V load_once(const char *p) {
  if constexpr (ONCE) return __builtin_nontemporal_load(reinterpret_cast<const V *>(p));
  else return *reinterpret_cast<const V *>(p);
}
template <bool ONCE, typename V>
__device__ __forceinline__ void store_once(char *p, V x) {
  if constexpr (ONCE) __builtin_nontemporal_store(x, reinterpret_cast<V *>(p));
  else *reinterpret_cast<V *>(p) = x;
}
template <bool ONCE>
__device__ __forceinline__ Eight load8(const char *p, const uint16_t *) {
  const u32x4 w = load_once<ONCE, u32x4>(p);
  Eight r;
#pragma unroll
  for (int k = 0; k < 4; ++k) r.x[2 * k] = bf16_lo(w[k]), r.x[2 * k + 1] = bf16_hi(w[k]);
  return r;
}
template <bool ONCE>
__device__ __forceinline__ Eight load8(const char *p, const float *) {
  const f32x4 a = load_once<ONCE, f32x4>(p), b = load_once<ONCE, f32x4>(p + 16);
  return {{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]}};
}

// to the nearest e4m3 value; NaN and infinities, which e4m3 does not have, become NaN
__device__ __forceinline__ float in_range(float x, float inverse) {
  const float y = fminf(fmaxf(x * inverse, -448.f), 448.f);
  return fabsf(x) <= 3.402823466e38f ? y : __builtin_nanf("");
}
__device__ __forceinline__ u32x2 round8(const Eight &v, float inverse) {
  u32x2 r;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(in_range(v.x[4 * k], inverse), in_range(v.x[4 * k + 1], inverse), 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(in_range(v.x[4 * k + 2], inverse), in_range(v.x[4 * k + 3], inverse), w, true);
    r[k] = uint32_t(w);
  }
  return r;
}
__device__ __forceinline__ Eight values8(u32x2 w, float scale) {
  Eight r;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(int(w[k]), false), b = __builtin_amdgcn_cvt_pk_f32_fp8(int(w[k]), true);
    r.x[4 * k] = a[0] * scale, r.x[4 * k + 1] = a[1] * scale, r.x[4 * k + 2] = b[0] * scale, r.x[4 * k + 3] = b[1] * scale;
  }
  return r;
}

__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
  for (int m = 1; m < kWave; m <<= 1) x = fmaxf(x, __shfl_xor(x, m));
  return x;
}

// the smallest E with a <= 448 * 2^(E - 127): 448 = 1.75 * 2^8
__device__ __forceinline__ int exponent_of(float a) {
  const uint32_t u = __float_as_uint(a);
  const int E = int(u >> 23) - ((u & 0x7fffffu) <= 0x600000u ? 8 : 7);
  return min(max(E, 1), kQ8Most);
}

// A lane has eight numbers (16 or 32 bytes) of every fourth row (of every eighth, where heads are of 64), so that a wave's loads are of whole rows and
// the block is in registers between its maximum and its rounding: one pass over the new rows.
template <typename T, int D, bool ONCE>
__global__ __launch_bounds__(kThreads) void append_kernel(KvArgs a, Q8Layers L) {
  constexpr int kLanes = D / 8, kRows = kWave / kLanes, kSteps = kQ8Block / kRows;
  const int b = blockIdx.z, l = blockIdx.y >> 1, lane = threadIdx.x & (kWave - 1);
  const int P = min(max(a.to[b], 0), a.C), n = min(min(max(a.from[b], 0), a.S), P), P0 = P - n;
  if (n == 0) return;
  const bool values = blockIdx.y & 1;
  const char *suf = (values ? L.of[l].v_suf : L.of[l].k_suf) + b * a.ss[0];
  char *cache = (values ? L.of[l].v_cache : L.of[l].k_cache) + b * a.cs[0];
  uint8_t *scales = (values ? L.of[l].v_scale : L.of[l].k_scale) + int64_t(b) * a.Hkv * a.blocks;
  const int first = P0 / kQ8Block, items = ((P - 1) / kQ8Block - first + 1) * a.Hkv;
  const int r = lane / kLanes, d = (lane % kLanes) * 8;
  for (int it = blockIdx.x * kWaves + threadIdx.x / kWave; it < items; it += gridDim.x * kWaves) {
    const int q = quotient(it, a.by_heads), blk = first + q, g = it - q * a.Hkv, t0 = blk * kQ8Block;
    Eight x[kSteps];
    float most = 0.f;
#pragma unroll
    for (int k = 0; k < kSteps; ++k)  // (rows that are not new repeat one that is)
      x[k] = load8<ONCE>(suf + int64_t(min(max(t0 + k * kRows + r, P0), P - 1) - P0) * a.ss[1] + g * a.ss[2] + d * int(sizeof(T)), static_cast<T *>(nullptr));
#pragma unroll
    for (int k = 0; k < kSteps; ++k)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float m = fabsf(x[k].x[e]);
        most = fmaxf(most, m <= 3.402823466e38f ? m : 0.f);
      }
    int E = exponent_of(wave_max(most));
    char *to = cache + g * a.cs[2] + d;
    uint8_t *s = scales + int64_t(g) * a.blocks + blk;
    if (t0 < P0) {  // the rows that are there stay under the scale they have, or are rounded again under a larger one
      const int old = *s;
      if (old >= E) E = old;
      else {
        const float by = q8_scale(uint32_t(max(127 + old - E, 1)));
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
          const int t = t0 + k * kRows + r;
          if (t < P0) {
            u32x2 *p = reinterpret_cast<u32x2 *>(to + int64_t(t) * a.cs[1]);
            *p = round8(values8(*p, 1.f), by);
          }
        }
      }
    }
    const float inverse = q8_scale(uint32_t(max(254 - E, 1)));
#pragma unroll
    for (int k = 0; k < kSteps; ++k) {
      const int t = t0 + k * kRows + r;
      if (t >= P0 && t < P) store_once<ONCE>(to + int64_t(t) * a.cs[1], round8(x[k], inverse));
    }
    if (lane == 0) *s = uint8_t(E);
  }
}

// A lane's 16 values are 32 or 64 bytes, two or four stores, in each of which neighbouring lanes are as far apart: fp32 rows, 5 x 333 of 4 heads of 64 in four layers
// (15 MB), take 7.9 us, where the append that reads as much takes 5.4.
__device__ __forceinline__ void store16(char *p, u32x4 w, float scale, const uint16_t *) {
  u32x4 o[2];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    o[k >> 1][2 * (k & 1)] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[k], scale, false));
    o[k >> 1][2 * (k & 1) + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[k], scale, true));
  }
  reinterpret_cast<u32x4 *>(p)[0] = o[0];
  reinterpret_cast<u32x4 *>(p)[1] = o[1];
}
__device__ __forceinline__ void store16(char *p, u32x4 w, float scale, const float *) {
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const Eight v = values8(u32x2{w[2 * k], w[2 * k + 1]}, scale);
    reinterpret_cast<f32x4 *>(p)[2 * k] = f32x4{v.x[0], v.x[1], v.x[2], v.x[3]};
    reinterpret_cast<f32x4 *>(p)[2 * k + 1] = f32x4{v.x[4], v.x[5], v.x[6], v.x[7]};
  }
}

constexpr int kAtOnce = 4;
// 16 values a lane and step, four steps at once (of 32 layers' 8 x 64 rows 76 us, with two 83, with eight 81), what is left singly.
template <typename T, int D, bool ONCE>
__global__ __launch_bounds__(kThreads) void read_kernel(KvArgs a, Q8Layers L) {
  constexpr int kLanes = D / 16, kHeads = kThreads / kLanes;
  const int b = blockIdx.z, l = blockIdx.y >> 1;
  const int first = min(max(a.from[b], 0), a.C), end = min(max(a.to[b], first), a.C), n = min(end - first, a.S);
  const bool values = blockIdx.y & 1;
  char *out = (values ? L.of[l].out : const_cast<char *>(L.of[l].q)) + b * a.ss[0];
  const char *cache = (values ? L.of[l].v_cache : L.of[l].k_cache) + b * a.cs[0];
  const uint8_t *scales = (values ? L.of[l].v_scale : L.of[l].k_scale) + int64_t(b) * a.Hkv * a.blocks;
  const int d = (threadIdx.x % kLanes) * 16;
  const int items = n * a.Hkv, step = gridDim.x * kHeads;
  int it = blockIdx.x * kHeads + threadIdx.x / kLanes;
  auto some = [&](auto count) {
    constexpr int N = decltype(count)::value;
    u32x4 w[N];
    uint32_t E[N];
    char *to[N];
#pragma unroll
    for (int k = 0; k < N; ++k, it += step) {
      const int i = quotient(it, a.by_heads), g = it - i * a.Hkv, t = first + i;
      w[k] = load_once<ONCE, u32x4>(cache + int64_t(t) * a.cs[1] + g * a.cs[2] + d);
      E[k] = scales[int64_t(g) * a.blocks + t / kQ8Block];
      to[k] = out + int64_t(i) * a.ss[1] + g * a.ss[2] + d * int(sizeof(T));
    }
#pragma unroll
    for (int k = 0; k < N; ++k) store16(to[k], w[k], q8_scale(E[k]), static_cast<T *>(nullptr));
  };
  while (it + int64_t(kAtOnce - 1) * step < items) some(std::integral_constant<int, kAtOnce>());
  while (it < items) some(std::integral_constant<int, 1>());
}

KvArgs kv_args(const AttnArgs &a, const lsp_attn_desc *d, const int32_t *from, const int32_t *to) {
  KvArgs k;
  k.from = from; k.to = to;
  k.B = a.B; k.S = a.S; k.Hkv = a.Hkv; k.C = a.C; k.blocks = (a.C + kQ8Block - 1) / kQ8Block;
  k.by_heads = div_by(a.Hkv);
  for (int j = 0; j < 3; ++j) {
    k.ss[j] = a.ks[j] * int64_t(elem_size(d->dtype));
    k.cs[j] = a.cs[j];
  }
  return k;
}

template <bool ONCE>
void launch_append(int32_t dtype, int D, dim3 grid, hipStream_t st, const KvArgs &k, const Q8Layers &L) {
  if (dtype == LSP_F32) {
    if (D == 64) append_kernel<float, 64, ONCE><<<grid, kThreads, 0, st>>>(k, L);
    else append_kernel<float, 128, ONCE><<<grid, kThreads, 0, st>>>(k, L);
  } else {
    if (D == 64) append_kernel<uint16_t, 64, ONCE><<<grid, kThreads, 0, st>>>(k, L);
    else append_kernel<uint16_t, 128, ONCE><<<grid, kThreads, 0, st>>>(k, L);
  }
}
template <bool ONCE>
void launch_read(int32_t dtype, int D, dim3 grid, hipStream_t st, const KvArgs &k, const Q8Layers &L) {
  if (dtype == LSP_F32) {
    if (D == 64) read_kernel<float, 64, ONCE><<<grid, kThreads, 0, st>>>(k, L);
    else read_kernel<float, 128, ONCE><<<grid, kThreads, 0, st>>>(k, L);
  } else {
    if (D == 64) read_kernel<uint16_t, 64, ONCE><<<grid, kThreads, 0, st>>>(k, L);
    else read_kernel<uint16_t, 128, ONCE><<<grid, kThreads, 0, st>>>(k, L);
  }
}
// whether the buffers of a launch, beside the caches, are larger than the last cache; bytes: of a head's row
bool is_large(const KvArgs &k, int layers, size_t bytes) { return double(2 * layers) * k.B * k.S * k.Hkv * double(bytes) > double(kLastCache); }

// workgroups in x: all that there is work for, or what makes kGroups of them
dim3 grid_of(const KvArgs &k, int layers, int64_t most) {
  const int64_t yz = int64_t(2) * layers * k.B, want = (kGroups + yz - 1) / yz;
  return dim3(unsigned(want < 1 ? 1 : want < most ? want : most), unsigned(2 * layers), unsigned(k.B));
}

}  // namespace
}  // namespace lsp

extern "C" int32_t lsp_kv_append_q8(const lsp_attn_desc *d, int32_t num_layers, const void *const *k_suf_layers, const void *const *v_suf_layers,
                                    void *const *k_cache_layers, void *const *v_cache_layers, void *const *k_scale_layers,
                                    void *const *v_scale_layers, const int32_t *commit_len, const int32_t *prefix_len, void *stream) {
  using namespace lsp;
  const char *what = "lsp_kv_append_q8";
  AttnArgs a;
  const int32_t rc = check_q8(what, d, false, a);
  if (rc != LSP_OK) return rc;
  LSP_CHECK_ARG(num_layers > 0, "%s: num_layers must be positive", what);
  LSP_CHECK_ARG(k_suf_layers && v_suf_layers && k_cache_layers && v_cache_layers && k_scale_layers && v_scale_layers && commit_len && prefix_len,
                "%s: null pointer", what);
  LSP_CHECK_ARG(a.B == 1 || a.cs[0] > 0, "%s: a cache must not be shared by sequences", what);
  for (int l = 0; l < num_layers; ++l) {
    LSP_CHECK_ARG(k_suf_layers[l] && v_suf_layers[l] && k_cache_layers[l] && v_cache_layers[l] && k_scale_layers[l] && v_scale_layers[l],
                  "%s: null operand in layer %d", what, l);
    LSP_CHECK_ARG(aligned16(k_suf_layers[l]) && aligned16(v_suf_layers[l]) && aligned16(k_cache_layers[l]) && aligned16(v_cache_layers[l]),
                  "%s: operands of layer %d must be 16-byte aligned", what, l);
  }
  const KvArgs k = kv_args(a, d, commit_len, prefix_len);
  const int64_t most = ((a.S + int64_t(2 * kQ8Block) - 1) / kQ8Block * a.Hkv + kWaves - 1) / kWaves;
  for (int l0 = 0; l0 < num_layers; l0 += kMaxAttnLayers) {
    const int nl = num_layers - l0 < kMaxAttnLayers ? num_layers - l0 : kMaxAttnLayers;
    Q8Layers L = {};
    for (int l = 0; l < nl; ++l) {
      L.of[l].k_suf = static_cast<const char *>(k_suf_layers[l0 + l]); L.of[l].v_suf = static_cast<const char *>(v_suf_layers[l0 + l]);
      L.of[l].k_cache = static_cast<char *>(k_cache_layers[l0 + l]); L.of[l].v_cache = static_cast<char *>(v_cache_layers[l0 + l]);
      L.of[l].k_scale = static_cast<uint8_t *>(k_scale_layers[l0 + l]); L.of[l].v_scale = static_cast<uint8_t *>(v_scale_layers[l0 + l]);
    }
    const dim3 grid = grid_of(k, nl, most);
    const bool once = is_large(k, nl, elem_size(d->dtype) * a.D);
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (once) launch_append<true>(d->dtype, a.D, grid, st, k, L);
    else launch_append<false>(d->dtype, a.D, grid, st, k, L);
    LSP_CHECK_LAUNCH("lsp_kv_append_q8: launch");
  }
  return LSP_OK;
}

extern "C" int32_t lsp_kv_read_q8(const lsp_attn_desc *d, int32_t num_layers, const void *const *k_cache_layers, const void *const *v_cache_layers,
                                  const void *const *k_scale_layers, const void *const *v_scale_layers, const int32_t *first_row,
                                  const int32_t *end_row, void *const *k_out_layers, void *const *v_out_layers, void *stream) {
  using namespace lsp;
  const char *what = "lsp_kv_read_q8";
  AttnArgs a;
  const int32_t rc = check_q8(what, d, false, a);
  if (rc != LSP_OK) return rc;
  LSP_CHECK_ARG(num_layers > 0, "%s: num_layers must be positive", what);
  LSP_CHECK_ARG(k_cache_layers && v_cache_layers && k_scale_layers && v_scale_layers && first_row && end_row && k_out_layers && v_out_layers,
                "%s: null pointer", what);
  LSP_CHECK_ARG(a.B == 1 || a.ks[0] > 0, "%s: an output must not be shared by sequences", what);
  LSP_CHECK_ARG(int64_t(a.S < a.C ? a.S : a.C) * a.Hkv < int64_t(1) << 30, "%s: min(S, C) * Hkv must be < 2^30", what);
  for (int l = 0; l < num_layers; ++l) {
    LSP_CHECK_ARG(k_cache_layers[l] && v_cache_layers[l] && k_scale_layers[l] && v_scale_layers[l] && k_out_layers[l] && v_out_layers[l],
                  "%s: null operand in layer %d", what, l);
    LSP_CHECK_ARG(aligned16(k_cache_layers[l]) && aligned16(v_cache_layers[l]) && aligned16(k_out_layers[l]) && aligned16(v_out_layers[l]),
                  "%s: operands of layer %d must be 16-byte aligned", what, l);
  }
  const KvArgs k = kv_args(a, d, first_row, end_row);
  const int heads = kThreads / (a.D / 16);
  const int64_t most = (int64_t(a.S < a.C ? a.S : a.C) * a.Hkv + heads - 1) / heads;
  for (int l0 = 0; l0 < num_layers; l0 += kMaxAttnLayers) {
    const int nl = num_layers - l0 < kMaxAttnLayers ? num_layers - l0 : kMaxAttnLayers;
    Q8Layers L = {};
    for (int l = 0; l < nl; ++l) {
      L.of[l].k_cache = static_cast<char *>(const_cast<void *>(k_cache_layers[l0 + l])); L.of[l].v_cache = static_cast<char *>(const_cast<void *>(v_cache_layers[l0 + l]));
      L.of[l].k_scale = static_cast<uint8_t *>(const_cast<void *>(k_scale_layers[l0 + l])); L.of[l].v_scale = static_cast<uint8_t *>(const_cast<void *>(v_scale_layers[l0 + l]));
      L.of[l].q = static_cast<char *>(k_out_layers[l0 + l]); L.of[l].out = static_cast<char *>(v_out_layers[l0 + l]);
    }
    const dim3 grid = grid_of(k, nl, most);
    const bool once = is_large(k, nl, elem_size(d->dtype) * a.D);
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (once) launch_read<true>(d->dtype, a.D, grid, st, k, L);
    else launch_read<false>(d->dtype, a.D, grid, st, k, L);
    LSP_CHECK_LAUNCH("lsp_kv_read_q8: launch");
  }
  return LSP_OK;
}
