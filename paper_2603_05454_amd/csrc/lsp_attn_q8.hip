// lsp_attn_step_q8: attention of the active rows over [cached rows in 8 bits || suffix rows].
//
// A unit is (layer, sequence, KV head); the rows of all heads of its group are one list (entry e: row e / rep of head e % rep), since they meet
// the same keys.  A wave has tiles of 16 entries and goes over blocks of 32 keys, those that share a scale:
//   S^T = K Q^T   v_mfma_f32_16x16x32_bf16, keys x entries: a lane's scores are of ONE entry, and of those keys of which
//   O^T += V^T P^T  has its probabilities as operand: they go from one product to the other in the lane's registers.
// The order of a head's elements and of a block's keys within the products is of no matter, so both operands are taken as a lane loads them: 16 bytes of a
// key's row; a few elements of eight keys' rows, turned in registers, a byte each, before they become bf16 (v_cvt_scalef32_pk_bf16_fp8, with the
// block's scale: exact).
#include <math.h>

#include "lsp_q8.h"

namespace lsp {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kWaves = 8;
constexpr int kThreads = kWaves * kWave;
constexpr float kLag = 8.f;  // octaves that a maximum may exceed the reference by before that moves

struct Q8AttnArgs {
  const int32_t *prefix_len, *suffix_len;
  int32_t B, S, Hkv, C, rep, blocks, units, tiles;
  float c;  // scale log2(e)
  Div by_tiles, by_heads, by_units, by_rep;
  int64_t qs[3], ks[3], cs[3], os[3];  // bytes: sequence, row, head
};

__device__ __forceinline__ uint32_t word(bf16x2 x) { return __builtin_bit_cast(uint32_t, x); }
__device__ __forceinline__ bf16x8 fragment(uint32_t a, uint32_t b, uint32_t c, uint32_t d) { return __builtin_bit_cast(bf16x8, u32x4{a, b, c, d}); }
// four e4m3 values -> two words of bf16
__device__ __forceinline__ uint32_t low(uint32_t w, float s) { return word(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, s, false)); }
__device__ __forceinline__ uint32_t high(uint32_t w, float s) { return word(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, s, true)); }
__device__ __forceinline__ uint32_t pick(uint32_t hi, uint32_t lo, uint32_t sel) { return __builtin_amdgcn_perm(hi, lo, sel); }

__device__ __forceinline__ float across(float x, bool sum) {  // over the four lanes that have an entry
#pragma unroll
  for (int m = 16; m < 64; m <<= 1) {
    const float y = __shfl_xor(x, m);
    x = sum ? x + y : fmaxf(x, y);
  }
  return x;
}

// Lanes l % 16 = r, l / 16 = h.  Of the keys: rows 16 k + r of the block, elements 64 i + 16 h of 16; of the values: rows 16 k + 4 h + e, of which
// VJ elements from VJ r on.
template <int D>
struct Keys {
  static constexpr int KI = D / 64, KC = D / 32, VJ = D / 16;
  bf16x8 k[2][KC], v[VJ];

  // row of the block that element e (of eight) of a lane's values is of
  static __device__ __forceinline__ int value_row(int h, int e) { return 16 * (e >> 2) + 4 * h + (e & 3); }

  __device__ __forceinline__ void cached(const char *kp, const char *vp, int64_t row, int last, float ks, float vs, int r, int h) {
    u32x4 kw[2][KI];
    uint32_t w[8][VJ / 4];
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int i = 0; i < KI; ++i) kw[b][i] = *reinterpret_cast<const u32x4 *>(kp + min(16 * b + r, last) * row + 64 * i + 16 * h);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t *p = reinterpret_cast<const uint32_t *>(vp + min(value_row(h, e), last) * row + VJ * r);
#pragma unroll
      for (int j = 0; j < VJ / 4; ++j) w[e][j] = p[j];
    }
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int i = 0; i < KI; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
          k[b][2 * i + j] = fragment(low(kw[b][i][2 * j], ks), high(kw[b][i][2 * j], ks), low(kw[b][i][2 * j + 1], ks), high(kw[b][i][2 * j + 1], ks));
#pragma unroll
    for (int q = 0; q < VJ / 4; ++q) {
      uint32_t t[4][2];  // element j of keys 4 m to 4 m + 3
#pragma unroll
      for (int m = 0; m < 2; ++m) {
        const uint32_t a = w[4 * m][q], b = w[4 * m + 1][q], c = w[4 * m + 2][q], d = w[4 * m + 3][q];
        const uint32_t ab = pick(b, a, 0x05010400), cd = pick(d, c, 0x05010400), ab2 = pick(b, a, 0x07030602), cd2 = pick(d, c, 0x07030602);
        t[0][m] = pick(cd, ab, 0x05040100);
        t[1][m] = pick(cd, ab, 0x07060302);
        t[2][m] = pick(cd2, ab2, 0x05040100);
        t[3][m] = pick(cd2, ab2, 0x07060302);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) v[4 * q + j] = fragment(low(t[j][0], vs), high(t[j][0], vs), low(t[j][1], vs), high(t[j][1], vs));
    }
  }

  __device__ __forceinline__ void suffix(const char *kp, const char *vp, int64_t row, int last, int r, int h) {
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int c = 0; c < KC; ++c)
        k[b][c] = *reinterpret_cast<const bf16x8 *>(kp + min(16 * b + r, last) * row + 128 * (c >> 1) + 32 * h + 16 * (c & 1));
    uint32_t w[8][VJ / 2];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t *p = reinterpret_cast<const uint32_t *>(vp + min(value_row(h, e), last) * row + 2 * VJ * r);
#pragma unroll
      for (int j = 0; j < VJ / 2; ++j) w[e][j] = p[j];
    }
#pragma unroll
    for (int j = 0; j < VJ; ++j) {
      uint32_t t[4];
#pragma unroll
      for (int m = 0; m < 4; ++m) t[m] = pick(w[2 * m + 1][j >> 1], w[2 * m][j >> 1], j & 1 ? 0x07060302 : 0x05040100);
      v[j] = fragment(t[0], t[1], t[2], t[3]);
    }
  }
};

// NB tiles of 16 entries
template <int D, int NB>
struct Rows {
  static constexpr int KC = D / 32, VJ = D / 16;
  bf16x8 q[NB][KC];
  f32x4 o[NB][VJ];   // o[n][j][i]: element 4 VJ h + VJ i + j of entry r
  float m[NB], l[NB];  // reference (base 2, scaled), this lane's part of the sum

  __device__ __forceinline__ void start(const Q8AttnArgs &a, const char *q0, int entry, int entries, int r, int h) {
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      const int e = min(entry + 16 * n + r, entries - 1), u = quotient(e, a.by_rep);
      const char *p = q0 + u * a.qs[1] + (e - u * a.rep) * a.qs[2];
#pragma unroll
      for (int c = 0; c < KC; ++c) q[n][c] = *reinterpret_cast<const bf16x8 *>(p + 128 * (c >> 1) + 32 * h + 16 * (c & 1));
#pragma unroll
      for (int j = 0; j < VJ; ++j) o[n][j] = f32x4{0.f, 0.f, 0.f, 0.f};
      m[n] = -INFINITY;
      l[n] = 0.f;
    }
  }

  // valid: keys of the block that there are
  __device__ __forceinline__ void meet(const Keys<D> &x, float c, int valid, int h) {
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      f32x4 s[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
      for (int k = 0; k < KC; ++k)
#pragma unroll
        for (int b = 0; b < 2; ++b) s[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x.k[b][k], q[n][k], s[b], 0, 0, 0);
      if (valid < kQ8Block)
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int i = 0; i < 4; ++i) s[b][i] = 16 * b + 4 * h + i < valid ? s[b][i] : -INFINITY;
      float most = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])), fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
      most = across(most, false) * c;
      if (__any(most > m[n] + kLag)) {
        const float to = fmaxf(m[n], most), f = to > m[n] ? __builtin_amdgcn_exp2f(m[n] - to) : 1.f;
        m[n] = to;
        l[n] *= f;
#pragma unroll
        for (int j = 0; j < VJ; ++j) o[n][j] *= f;
      }
      float p[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        p[e] = __builtin_amdgcn_exp2f(fmaf(s[e >> 2][e & 3], c, -m[n]));
        l[n] += p[e];
      }
      bf16x8 P;
#pragma unroll
      for (int e = 0; e < 8; ++e) P[e] = __bf16(p[e]);
#pragma unroll
      for (int j = 0; j < VJ; ++j) o[n][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x.v[j], P, o[n][j], 0, 0, 0);
    }
  }
};

template <int D, int NB>
__global__ __launch_bounds__(kThreads) void attn_q8_kernel(Q8AttnArgs a, Q8Layers L) {
  constexpr int VJ = D / 16;
  __shared__ f32x4 s_o[kWaves][VJ][kWave];
  __shared__ float s_m[kWaves][16], s_l[kWaves][16];
  const int id = workgroup_id(), lane = threadIdx.x & (kWave - 1), r = lane & 15, h = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  // the tiles of a unit on one XCD
  const int m8 = id >> 3, turn = quotient(m8, a.by_tiles), tile = m8 - turn * a.tiles, unit = turn * 8 + (id & 7);
  if (unit >= a.units) return;
  const int per_layer = a.B * a.Hkv, layer = quotient(unit, a.by_units), in_layer = unit - layer * per_layer;
  const int b = quotient(in_layer, a.by_heads), g = in_layer - b * a.Hkv;
  const int N = min(max(a.suffix_len[b], 0), a.S), P = min(max(a.prefix_len[b], 0), a.C);
  const int entries = N * a.rep, entry = tile * 16 * NB;
  if (entry >= entries) return;

  Rows<D, NB> rows;
  rows.start(a, L.q[layer] + b * a.qs[0] + g * a.rep * a.qs[2], entry, entries, r, h);
  const char *kc = L.k_cache[layer] + b * a.cs[0] + g * a.cs[2], *vc = L.v_cache[layer] + b * a.cs[0] + g * a.cs[2];
  const char *ks = L.k_suf[layer] + b * a.ks[0] + g * a.ks[2], *vs = L.v_suf[layer] + b * a.ks[0] + g * a.ks[2];
  const int64_t scales = (int64_t(b) * a.Hkv + g) * a.blocks;
  const uint8_t *ke = L.k_scale[layer] + scales, *ve = L.v_scale[layer] + scales;
  const int cached = (P + kQ8Block - 1) / kQ8Block, all = cached + (N + kQ8Block - 1) / kQ8Block;
  for (int s = wave; s < all; s += kWaves) {
    Keys<D> x;
    int valid;
    if (s < cached) {
      valid = P - s * kQ8Block;
      const int64_t at = int64_t(s) * kQ8Block * a.cs[1];
      x.cached(kc + at, vc + at, a.cs[1], valid - 1, q8_scale(ke[s]), q8_scale(ve[s]), r, h);
    } else {
      const int t = s - cached;
      valid = N - t * kQ8Block;
      const int64_t at = int64_t(t) * kQ8Block * a.ks[1];
      x.suffix(ks + at, vs + at, a.ks[1], valid - 1, r, h);
    }
    rows.meet(x, a.c, valid, h);
  }

  // the waves' parts, joined in LDS: wave w adds what all have in place w of their lanes
  char *out = L.out[layer] + b * a.os[0] + g * a.rep * a.os[2];
#pragma unroll
  for (int n = 0; n < NB; ++n) {
    const float l = across(rows.l[n], true);
    if (n > 0) __syncthreads();
    if (h == 0) s_m[wave][r] = rows.m[n], s_l[wave][r] = l;
    __syncthreads();
    float m = -INFINITY, sum = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) m = fmaxf(m, s_m[w][r]);
#pragma unroll
    for (int w = 0; w < kWaves; ++w) sum += s_l[w][r] > 0.f || s_l[w][r] != s_l[w][r] ? s_l[w][r] * __builtin_amdgcn_exp2f(s_m[w][r] - m) : 0.f;
    const float f = l > 0.f ? __builtin_amdgcn_exp2f(rows.m[n] - m) : l;  // (a wave that met no key has zeros)
#pragma unroll
    for (int p = 0; p < VJ; ++p) {  // elements 4 p to 4 p + 3 of the lane's 4 VJ
      f32x4 x;
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] = f * rows.o[n][(4 * p + j) % VJ][(4 * p + j) / VJ];
      s_o[wave][p][lane] = x;
    }
    __syncthreads();
    if (wave < VJ) {
      f32x4 x = s_o[0][wave][lane];
#pragma unroll
      for (int w = 1; w < kWaves; ++w) x += s_o[w][wave][lane];
      const int e = entry + 16 * n + r;
      if (e < entries) {
        const int u = quotient(e, a.by_rep);
        const float inv = 1.f / sum;
        typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
        *reinterpret_cast<bf16x4 *>(out + u * a.os[1] + (e - u * a.rep) * a.os[2] + 2 * (4 * VJ * h + 4 * wave)) =
            bf16x4{__bf16(x[0] * inv), __bf16(x[1] * inv), __bf16(x[2] * inv), __bf16(x[3] * inv)};
      }
    }
  }
}

int32_t launch(const Q8AttnArgs &args, int D, const Q8Layers &L, int layers, hipStream_t st) {
  Q8AttnArgs a = args;
  a.units = layers * a.B * a.Hkv;
  const int NB = int64_t(a.rep) * a.S > 16 ? 2 : 1;
  const int64_t tiles = (int64_t(a.rep) * a.S + 16 * NB - 1) / (16 * NB), nwg = (int64_t(a.units) + 7) / 8 * 8 * tiles;
  LSP_CHECK_ARG(nwg < kMaxGrid, "lsp_attn_step_q8: too many rows for one launch");
  a.tiles = int32_t(tiles);
  a.by_tiles = div_by(tiles);
  a.by_heads = div_by(a.Hkv);
  a.by_units = div_by(int64_t(a.B) * a.Hkv);
  a.by_rep = div_by(a.rep);
  const dim3 grid = grid_of(nwg);
  if (D == 64) {
    if (NB == 1) attn_q8_kernel<64, 1><<<grid, kThreads, 0, st>>>(a, L);
    else attn_q8_kernel<64, 2><<<grid, kThreads, 0, st>>>(a, L);
  } else {
    if (NB == 1) attn_q8_kernel<128, 1><<<grid, kThreads, 0, st>>>(a, L);
    else attn_q8_kernel<128, 2><<<grid, kThreads, 0, st>>>(a, L);
  }
  LSP_CHECK_LAUNCH("lsp_attn_step_q8: launch");
  return LSP_OK;
}

}  // namespace
}  // namespace lsp

extern "C" size_t lsp_attn_q8_workspace_bytes(const lsp_attn_desc *d, int32_t num_layers) { return 0; }

extern "C" int32_t lsp_attn_step_q8_layers(const lsp_attn_desc *d, int32_t num_layers, const void *const *q_layers, const void *const *k_suf_layers,
                                           const void *const *v_suf_layers, const void *const *k_cache_layers, const void *const *v_cache_layers,
                                           const void *const *k_scale_layers, const void *const *v_scale_layers, const int32_t *prefix_len,
                                           const int32_t *suffix_len, void *const *out_layers, void *workspace, size_t workspace_bytes,
                                           void *stream) {
  using namespace lsp;
  const char *what = "lsp_attn_step_q8";
  AttnArgs c;
  const int32_t rc = check_q8(what, d, true, c);
  if (rc != LSP_OK) return rc;
  if (d->dtype != LSP_BF16) {
    set_error("%s: bf16 queries only", what);
    return LSP_ERR_UNSUPPORTED;
  }
  LSP_CHECK_ARG(num_layers > 0, "%s: num_layers must be positive", what);
  LSP_CHECK_ARG(q_layers && k_suf_layers && v_suf_layers && k_cache_layers && v_cache_layers && k_scale_layers && v_scale_layers && out_layers &&
                    prefix_len && suffix_len,
                "%s: null pointer", what);
  LSP_CHECK_ARG(c.B == 1 || c.os[0] > 0, "%s: the output must not be shared by sequences", what);
  LSP_CHECK_ARG(int64_t(kMaxAttnLayers) * c.B * c.Hkv < int64_t(1) << 31 && int64_t(c.S) * (c.Hq / c.Hkv) <= 1 << 30,
                "%s: B * Hkv must be < 2^26, S * Hq / Hkv <= 2^30", what);
  for (int l = 0; l < num_layers; ++l) {
    LSP_CHECK_ARG(q_layers[l] && k_suf_layers[l] && v_suf_layers[l] && k_cache_layers[l] && v_cache_layers[l] && k_scale_layers[l] &&
                      v_scale_layers[l] && out_layers[l],
                  "%s: null operand in layer %d", what, l);
    LSP_CHECK_ARG(aligned16(q_layers[l]) && aligned16(k_suf_layers[l]) && aligned16(v_suf_layers[l]) && aligned16(k_cache_layers[l]) &&
                      aligned16(v_cache_layers[l]) && aligned16(out_layers[l]),
                  "%s: operands of layer %d must be 16-byte aligned", what, l);
  }
  Q8AttnArgs a = {};
  a.prefix_len = prefix_len; a.suffix_len = suffix_len;
  a.B = c.B; a.S = c.S; a.Hkv = c.Hkv; a.C = c.C; a.rep = c.Hq / c.Hkv; a.blocks = (c.C + kQ8Block - 1) / kQ8Block;
  a.c = c.scale * kLog2e;
  for (int k = 0; k < 3; ++k) a.qs[k] = 2 * c.qs[k], a.ks[k] = 2 * c.ks[k], a.cs[k] = c.cs[k], a.os[k] = 2 * c.os[k];
  for (int l0 = 0; l0 < num_layers; l0 += kMaxAttnLayers) {
    const int nl = num_layers - l0 < kMaxAttnLayers ? num_layers - l0 : kMaxAttnLayers;
    Q8Layers L = {};
    for (int l = 0; l < nl; ++l) {
      L.q[l] = static_cast<const char *>(q_layers[l0 + l]);
      L.k_suf[l] = static_cast<const char *>(k_suf_layers[l0 + l]); L.v_suf[l] = static_cast<const char *>(v_suf_layers[l0 + l]);
      L.k_cache[l] = static_cast<char *>(const_cast<void *>(k_cache_layers[l0 + l])); L.v_cache[l] = static_cast<char *>(const_cast<void *>(v_cache_layers[l0 + l]));
      L.k_scale[l] = static_cast<uint8_t *>(const_cast<void *>(k_scale_layers[l0 + l])); L.v_scale[l] = static_cast<uint8_t *>(const_cast<void *>(v_scale_layers[l0 + l]));
      L.out[l] = static_cast<char *>(out_layers[l0 + l]);
    }
    const int32_t r = launch(a, c.D, L, nl, static_cast<hipStream_t>(stream));
    if (r != LSP_OK) return r;
  }
  return LSP_OK;
}

extern "C" int32_t lsp_attn_step_q8(const lsp_attn_desc *d, const void *q, const void *k_suf, const void *v_suf, const void *k_cache, const void *v_cache,
                                    const uint8_t *k_scale, const uint8_t *v_scale, const int32_t *prefix_len, const int32_t *suffix_len, void *out,
                                    void *workspace, size_t workspace_bytes, void *stream) {
  const void *ke = k_scale, *ve = v_scale;
  return lsp_attn_step_q8_layers(d, 1, &q, &k_suf, &v_suf, &k_cache, &v_cache, &ke, &ve, prefix_len, suffix_len, &out, workspace, workspace_bytes, stream);
}
