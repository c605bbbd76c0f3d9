// lsp_token_scores: log probability of a given token, entropy and the most likely alternatives of every active row of the logits,
// from one pass over the row.
//
// With m the row's maximum, s = sum exp(z - m) and t = sum exp(z - m) (z - m) / ln 2:
//   log p(v) = z[v] - m - log s          entropy = log s - ln 2 t / s
// A lane keeps both sums against a reference of its own that follows its maximum at most kLagOctaves behind (so that the branch that
// moves it is cold), and they are taken to the row's maximum at the end: with r = m log2(e) + x, s' = s 2^x, t' = 2^x (t + x s).
//
// The alternatives are the K first entries in the order (value descending, index ascending).  A pass that compared every entry with the K-th
// best so far would enter its rare branch for most groups of loads (the best K of the first half row are behind every second one of them).
// Instead every 16-byte vector's maximum goes to LDS, one store for two of them, and selection waits for the end:
//   the first K entries lie in the K vectors that come first by (maximum descending, position ascending).
// (Let x lie in none of them.  Each of those vectors holds an entry equal to its maximum, which is larger than x, or as large and in
// an earlier vector: K entries come before x.)  Those vectors are read once more, and their entries ranked by counting.
// Which vectors: at least K lanes hold a maximum of their own of at least T, if T is the smallest over the waves of each wave's
// (K / waves)-th largest lane maximum; vectors below T are out, and usually few more than K are left.  If more are left than there are threads
// (rows of equal entries), a search bit by bit finds the K-th one exactly.
//
// What bounds it: HBM with many rows (each byte read once: 8 x 1024 bf16 rows of 152 064 entries with 20 alternatives, 2.5 GB, 388 us = 6.4 TB/s,
// a bare read's rate; 438 us with ordinary instead of non-temporal loads).  With few, latencies: the trip through a row, the
// vectors read once more, ranks, and the segments' meeting, 1-4 us each (one row of 126 464 entries 9.5 us, 127 of them 16.4, 364 fp32 rows of 30 001
// 15.1).  Where few rows are active they are cut into segments, whose results meet in the workspace as in confidence_split_kernel
// (numbers with the call's tag beside them).
#include <float.h>
#include <limits.h>

#include <type_traits>

#include "lsp_common.h"

namespace lsp {
namespace {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
// An entropy loses 2^-24 of x s in t + x s: 5e-7 at 8 octaves, 2e-6 at the confidence pass's 32, whose sum has no such term.
constexpr float kLagOctaves = 8.0f;
// Entries below this are kept out of products (-inf, and the lowest values, whose product with log2(e) is): a group of loads that holds one
// takes a way of its own.
constexpr float kLow = -1e37f;
// Maxima farther from 0 than 2^26: the reference is a rounded product, and the maximum's own exponent its rounding error, up to half a step of it. That is 4 octaves
// here and 512 at 1e10, where 2^512 is infinite.
constexpr float kFar = 67108864.f;
constexpr int kMaxAlt = 32;
constexpr int kRankStep = 16;   // entries that are read at a time
constexpr int kMinCut = 16384;  // rows of at most this many entries are not cut

template <typename T>
struct Vec;
template <>
struct Vec<float> {
  static constexpr int N = 4;
  typedef u32x2 Pair;  // maxima of two vectors
  static __device__ __forceinline__ void unpack(const u32x4 &w, float (&x)[4]) {
    x[0] = __uint_as_float(w.x); x[1] = __uint_as_float(w.y);
    x[2] = __uint_as_float(w.z); x[3] = __uint_as_float(w.w);
  }
  static __device__ __forceinline__ Pair pack(float a, float b) { return Pair{__float_as_uint(a), __float_as_uint(b)}; }
  static __device__ __forceinline__ float first(Pair p) { return __uint_as_float(p.x); }
  static __device__ __forceinline__ float second(Pair p) { return __uint_as_float(p.y); }
  static __device__ __forceinline__ float scalar(const float *p) { return *p; }
};
template <>
struct Vec<uint16_t> {
  static constexpr int N = 8;
  typedef uint32_t Pair;
  static __device__ __forceinline__ void unpack(const u32x4 &w, float (&x)[8]) {
    x[0] = bf16_lo(w.x); x[1] = bf16_hi(w.x);
    x[2] = bf16_lo(w.y); x[3] = bf16_hi(w.y);
    x[4] = bf16_lo(w.z); x[5] = bf16_hi(w.z);
    x[6] = bf16_lo(w.w); x[7] = bf16_hi(w.w);
  }
  static __device__ __forceinline__ Pair pack(float a, float b) { return __float_as_uint(a) >> 16 | (__float_as_uint(b) & 0xffff0000u); }
  static __device__ __forceinline__ float first(Pair p) { return bf16_lo(p); }
  static __device__ __forceinline__ float second(Pair p) { return bf16_hi(p); }
  static __device__ __forceinline__ float scalar(const uint16_t *p) { return bf16_to_f32(*p); }
};

// Whole numbers in the order of the values, all at least 1 (0 is below every value); -0 as 0.
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);
  return u & 0x80000000u ? max(~u, 1u) : u | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k); }
// An entry: better ones are larger, no two are equal.
__device__ __forceinline__ uint64_t entry_of(uint32_t key, int index) { return uint64_t(key) << 32 | uint32_t(~index); }

__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(d) : "v"(a), "v"(b), "v"(c));
  return d;
}
__device__ __forceinline__ float min3(float a, float b, float c) {
  float d;
  asm("v_min3_f32 %0, %1, %2, %3" : "=v"(d) : "v"(a), "v"(b), "v"(c));
  return d;
}

// Reductions over a wave on the DPP network, valid in every lane (as in the confidence pass).
template <typename V, typename Op>
__device__ __forceinline__ V wave_reduce(V v, Op op) {
  static_assert(sizeof(V) == 4, "one register");
  auto bits = [](V x) { int i; __builtin_memcpy(&i, &x, 4); return i; };
  auto from = [](int i) { V x; __builtin_memcpy(&x, &i, 4); return x; };
#define LSP_DPP_STEP(ctrl) v = op(v, from(__builtin_amdgcn_update_dpp(bits(v), bits(v), ctrl, 0xf, 0xf, false)))
  LSP_DPP_STEP(0xb1);   // quad_perm [1,0,3,2]
  LSP_DPP_STEP(0x4e);   // quad_perm [2,3,0,1]
  LSP_DPP_STEP(0x114);  // row_shr:4
  LSP_DPP_STEP(0x118);  // row_shr:8
  LSP_DPP_STEP(0x142);  // row_bcast:15
  LSP_DPP_STEP(0x143);  // row_bcast:31
#undef LSP_DPP_STEP
  return from(__builtin_amdgcn_readlane(bits(v), kWave - 1));
}
__device__ __forceinline__ float wave_max(float v) { return wave_reduce(v, [](float a, float b) { return fmaxf(a, b); }); }
__device__ __forceinline__ float wave_sum(float v) { return wave_reduce(v, [](float a, float b) { return a + b; }); }
__device__ __forceinline__ uint32_t wave_max(uint32_t v) { return wave_reduce(v, [](uint32_t a, uint32_t b) { return max(a, b); }); }
__device__ __forceinline__ int wave_sum(int v) { return wave_reduce(v, [](int a, int b) { return a + b; }); }

struct Stat {  // of some entries: maximum m, s = sum 2^(x log2e - r), t = sum of these terms times their exponents
  float m, s, t;
};
// Takes sums to the reference M log2(e) from theirs, which is x above it.
__device__ __forceinline__ void take_to(Stat &a, float x) {
  const float f = __builtin_amdgcn_exp2f(x);
  a.t = f > 0.f ? f * __builtin_fmaf(x, a.s, a.t) : 0.f;
  a.s = f > 0.f ? f * a.s : 0.f;
}
// Over the lanes, each relative to its own maximum (idle lanes: -inf, 0, 0).
__device__ __forceinline__ Stat merge_stats(Stat a) {
  Stat r;
  r.m = wave_max(a.m);
  take_to(a, a.m == -INFINITY ? -INFINITY : (a.m - r.m) * kLog2e);
  r.s = wave_sum(a.s);
  r.t = wave_sum(a.t);
  return r;
}

// Threads of a workgroup share: the maxima of a tile's vectors and, when these are done with, the entries to be ranked (dynamic LDS), and
template <int NT>
struct Shared {
  Stat stat[NT / kWave];
  uint32_t wave_key[NT / kWave];
  int wave_count[NT / kWave];
  int vectors[NT];  // vectors that are left
  int count, entries;
  uint64_t best[kMaxAlt];  // the entries found so far, best first; 0: none
};
// Vectors of a tile.  19456 pairs of bytes or half as many of four are 38 KB: four workgroups share a compute unit, and bf16 rows of up to 155 648
// entries are one tile.
constexpr int kTileBytes = 38912;
template <typename T, int NT>
__host__ __device__ constexpr int tile_vectors() {
  return kTileBytes / int(sizeof(T)) / (2 * NT) * (2 * NT);
}
template <typename T, int NT, bool ALT>
inline size_t dynamic_lds(int64_t elements) {
  const int64_t group = 2 * NT, vectors = (elements / Vec<T>::N + group - 1) / group * group;
  const int64_t maxima = (vectors < tile_vectors<T, NT>() ? vectors : tile_vectors<T, NT>()) * int64_t(sizeof(T));
  const int64_t entries = (NT * Vec<T>::N + kMaxAlt + 16 + kRankStep) * 8, merged = ((3 + 2 * kMaxAlt) * 8 + 17 * kMaxAlt + kRankStep) * 8;
  const int64_t least = elements > kMinCut && merged > entries ? merged : entries;  // (only rows that are cut meet)
  return !ALT ? size_t(merged) : size_t(maxima > least ? maxima : least);
}

// Sum over the workgroup; every thread calls it.
template <int NT>
__device__ __forceinline__ int group_sum(Shared<NT> &sh, int n) {
  if (NT == kWave) return wave_sum(n);
  const int w = wave_sum(n);
  if ((threadIdx.x & (kWave - 1)) == 0) sh.wave_count[threadIdx.x / kWave] = w;
  __syncthreads();
  int all = 0;
#pragma unroll
  for (int k = 0; k < NT / kWave; ++k) all += sh.wave_count[k];
  __syncthreads();
  return all;
}

// The best K of `n` entries in LDS and of sh.best go to sh.best.  Every thread calls it, after a barrier; there is room for K + kRankStep entries more.
// Sixteen are read at a time: one by one the trip to LDS is waited for at each (8 rows of 82 303 entries, cut into 16 segments, 20 alternatives, eight at a
// time: 19.2 -> 15.0 us).
template <int NT>
__device__ __forceinline__ void rank_entries(Shared<NT> &sh, uint64_t *entries, int n, int K) {
  typedef uint64_t u64x2 __attribute__((ext_vector_type(2)));
  const int tid = threadIdx.x;
  if (tid < K + kRankStep) entries[n + tid] = tid < K ? sh.best[tid] : 0;
  n += K;
  __syncthreads();
  if (tid < K) sh.best[tid] = 0;
  __syncthreads();
  for (int e = tid; e < n; e += NT) {
    const uint64_t mine = entries[e];
    int before = 0;
    for (int k = 0; k < n; k += kRankStep) {
      u64x2 x[kRankStep / 2];
#pragma unroll
      for (int i = 0; i < kRankStep / 2; ++i) x[i] = *reinterpret_cast<const u64x2 *>(entries + k + 2 * i);
#pragma unroll
      for (int i = 0; i < kRankStep / 2; ++i) before += (x[i].x > mine) + (x[i].y > mine);
    }
    if (before < K && mine != 0) sh.best[before] = mine;
  }
  __syncthreads();
}

// One workgroup: statistics and best K of the elements [c0, c1) of a row.  The statistics are valid in wave 0, sh.best everywhere.
template <typename T, int NT, bool ALT>
__device__ __forceinline__ Stat scan_segment(const T *row, int c0, int c1, int K, Shared<NT> &sh, char *lds) {
  constexpr int N = Vec<T>::N, U = 2, G = NT * U;
  typedef typename Vec<T>::Pair Pair;
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
  Pair *maxima = reinterpret_cast<Pair *>(lds);
  uint64_t *entries = reinterpret_cast<uint64_t *>(lds);

  // an unaligned head, 16-byte vectors, and a tail
  const int len = c1 - c0;
  const int head = min(int(((16u - (unsigned(reinterpret_cast<uintptr_t>(row + c0)) & 15u)) & 15u) / sizeof(T)), len);
  const int nvec = (len - head) / N, vbase = c0 + head, tail0 = vbase + nvec * N;
  const u32x4 *vp = reinterpret_cast<const u32x4 *>(row + vbase);
  if (ALT && tid < kMaxAlt) sh.best[tid] = 0;

  Stat a = {-INFINITY, 0.f, 0.f};
  float r = -FLT_MAX;  // reference of s and t: some earlier maximum times log2(e), rounded
  auto settle = [&]() {
    const float mc = a.m * kLog2e;
    if (mc - r > kLagOctaves) {
      take_to(a, r - mc);
      r = mc;
    }
  };
  auto add = [&](float x, bool careful) {
    float d = __builtin_fmaf(x, kLog2e, -r);
    if (careful) d = fmaxf(d, -1000.f);
    const float e = __builtin_amdgcn_exp2f(d);
    a.s += e;
    a.t = __builtin_fmaf(e, d, a.t);
  };
  auto one = [&](float x) {
    a.m = fmaxf(a.m, x);
    settle();
    add(x, true);
  };
  const bool has_head = tid < head, has_tail = tid < c1 - tail0;
  float at_head = 0.f, at_tail = 0.f;
  if (has_head) one(at_head = Vec<T>::scalar(row + c0 + tid));
  if (has_tail) one(at_tail = Vec<T>::scalar(row + tail0 + tid));

  auto statistics = [&]() {  // lanes, then waves
    Stat own = a;
    const float top = wave_max(a.m);
    take_to(own, a.m == -INFINITY ? -INFINITY : __builtin_fmaf(-top, kLog2e, r));  // (the product unrounded inside the fma)
    Stat of_wave = {top, wave_sum(own.s), wave_sum(own.t)};
    if (NT == kWave) return of_wave;
    if (lane == 0) sh.stat[wave] = of_wave;
    __syncthreads();
    Stat w = {-INFINITY, 0.f, 0.f};
    if (lane < NT / kWave) w = sh.stat[lane];
    return merge_stats(w);
  };
  Stat all;
  const std::false_type full;
  const std::true_type maybe_partial;
  // Lanes past the end of a last, partial group read the last vector again, with -inf in the place of its values.
  for (int v0 = 0; v0 < nvec || (ALT && v0 == 0); v0 += tile_vectors<T, NT>()) {
    const int v1 = min(nvec, v0 + tile_vectors<T, NT>()), ngroups = (v1 - v0 + G - 1) / G;
    float lane_max = -INFINITY;  // of the tile
    auto load_group = [&](u32x4 (&buf)[U], int g, auto last) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int v = v0 + g * G + u * NT + tid;
        buf[u] = __builtin_nontemporal_load(vp + (decltype(last)::value ? min(v, v1 - 1) : v));
      }
    };
    auto process_group = [&](const u32x4 (&buf)[U], int g, auto last) {
      float x[U][N], top[U], low = 0.f;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        Vec<T>::unpack(buf[u], x[u]);
        if (decltype(last)::value && v0 + g * G + u * NT + tid >= v1) {
#pragma unroll
          for (int k = 0; k < N; ++k) x[u][k] = -INFINITY;
        }
        top[u] = max3(x[u][0], x[u][1], x[u][2]);
        low = min3(low, x[u][0], x[u][1]);
#pragma unroll
        for (int k = 3; k + 1 < N; k += 2) top[u] = max3(top[u], x[u][k], x[u][k + 1]);
        if (N % 2 == 0) top[u] = max3(top[u], x[u][N - 1], x[u][N - 1]);
#pragma unroll
        for (int k = 2; k < N; k += 2) low = min3(low, x[u][k], x[u][k + 1]);
      }
      if (ALT) maxima[g * NT + tid] = Vec<T>::pack(top[0], top[1]);
      lane_max = max3(lane_max, top[0], top[1]);
      a.m = fmaxf(a.m, lane_max);
      settle();
      if (__any(low < kLow)) {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int k = 0; k < N; ++k) add(x[u][k], true);
      } else {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int k = 0; k < N; ++k) add(x[u][k], false);
      }
    };
    if (ngroups > 0) {
      u32x4 ping[U], pong[U];
      if (ngroups == 1) load_group(ping, 0, maybe_partial); else load_group(ping, 0, full);
      int g = 0;
      for (; g + 3 < ngroups; g += 2) {  // groups g+1 and g+2 are full
        load_group(pong, g + 1, full);
        process_group(ping, g, full);
        load_group(ping, g + 2, full);
        process_group(pong, g + 1, full);
      }
      // one to three groups left; only the very last may be partial
      if (g + 2 < ngroups) {
        load_group(pong, g + 1, full);
        process_group(ping, g, full);
        load_group(ping, g + 2, maybe_partial);
        process_group(pong, g + 1, full);
        process_group(ping, g + 2, maybe_partial);
      } else if (g + 1 < ngroups) {
        load_group(pong, g + 1, maybe_partial);
        process_group(ping, g, full);
        process_group(pong, g + 1, maybe_partial);
      } else {
        process_group(ping, g, maybe_partial);
      }
    }
    if (!ALT) continue;

    // ---- the tile's part of the best K ----
    auto each = [&](auto f) {  // (key, vector of the tile) of each of the thread's own vectors
      for (int g = 0; g < ngroups; ++g) {
        const Pair p = maxima[g * NT + tid];
        const int v = g * G + tid;
        if (v0 + v < v1) f(key_of(Vec<T>::first(p)), v);
        if (v0 + v + NT < v1) f(key_of(Vec<T>::second(p)), v + NT);
      }
    };
    constexpr int kWaves = NT / kWave;
    uint32_t mine = key_of(lane_max), kth = 0;
    for (int j = 0; j < K; j += kWaves) {
      kth = wave_max(mine);
      const unsigned long long holders = __ballot(mine == kth);
      if (lane == __builtin_ctzll(holders)) mine = 0;
    }
    if (tid == 0) sh.count = sh.entries = 0;
    if (lane == 0) sh.wave_key[wave] = kth;
    __syncthreads();
    uint32_t least = sh.wave_key[0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) least = min(least, sh.wave_key[w]);
    // an entry of a later tile has to be larger than the K-th best of those before
    least = max(max(least, uint32_t(sh.best[K - 1] >> 32) + 1), 1u);
    if (key_of(lane_max) >= least)
      each([&](uint32_t k, int v) {
        if (k >= least) {
          const int at = atomicAdd(&sh.count, 1);
          if (at < NT) sh.vectors[at] = v;
        }
      });
    __syncthreads();
    int left = sh.count;
    if (left > NT) {  // (uniform) the K-th largest key, then the place up to which vectors with that key are in
      auto number = [&](auto in) {
        int n = 0;
        each([&](uint32_t k, int v) { n += in(k, v); });
        return group_sum<NT>(sh, n);
      };
      least = 0;
      for (uint32_t bit = 0x80000000u; bit != 0; bit >>= 1)
        if (number([&](uint32_t k, int) { return k >= (least | bit); }) >= K) least |= bit;
      const int equal = K - number([&](uint32_t k, int) { return k > least; });
      int upto = 0;
      for (int bit = 1 << 16; bit != 0; bit >>= 1)  // the largest with fewer than `equal` of them before it
        if (number([&](uint32_t k, int v) { return k == least && v < (upto | bit); }) < equal) upto |= bit;
      if (tid == 0) sh.count = 0;
      __syncthreads();
      each([&](uint32_t k, int v) {
        if (k > least || (k == least && v <= upto)) sh.vectors[atomicAdd(&sh.count, 1)] = v;
      });
      __syncthreads();
      left = sh.count;
    }
    const int again = v0 + (tid < left ? sh.vectors[tid] : 0);
    u32x4 entered = {};
    if (tid < left) entered = vp[again];
    if (v1 == nvec) all = statistics();  // (while they come)
    // (the maxima's place becomes the entries')
    auto enter = [&](float x, int index) {
      const uint32_t k = key_of(x);
      if (k >= least) entries[atomicAdd(&sh.entries, 1)] = entry_of(k, index);
    };
    if (tid < left) {
      float x[N];
      Vec<T>::unpack(entered, x);
#pragma unroll
      for (int k = 0; k < N; ++k) enter(x[k], vbase + again * N + k);
    }
    if (v0 == 0 && has_head) enter(at_head, c0 + tid);
    if (v1 == nvec && has_tail) enter(at_tail, tail0 + tid);
    __syncthreads();
    rank_entries<NT>(sh, entries, sh.entries, K);
  }

  if (!ALT) all = statistics();
  if (fabsf(all.m) > kFar && all.m > -INFINITY) {  // (uniform) sums that may have overflowed, or be of nothing: differences first
    __syncthreads();
    Stat w = {all.m, 0.f, 0.f};
    for (int c = c0 + tid; c < c1; c += NT) {
      const float d = fmaxf((Vec<T>::scalar(row + c) - all.m) * kLog2e, -1000.f), e = __builtin_amdgcn_exp2f(d);
      w.s += e;
      w.t = __builtin_fmaf(e, d, w.t);
    }
    all.s = wave_sum(w.s);
    all.t = wave_sum(w.t);
    if (NT > kWave) {
      if (lane == 0) sh.stat[wave] = all;
      __syncthreads();
      all.s = all.t = 0.f;
      for (int k = 0; k < NT / kWave; ++k) all.s += sh.stat[k].s, all.t += sh.stat[k].t;
    }
  }
  return all;
}

struct ScoreArgs {
  int32_t B, S, V, K;
  int64_t row_stride, batch_stride;
  const int32_t *suffix_len, *token_id;
  float *logprob, *entropy;
  int32_t *alt_id;
  float *alt_logprob;
};

// Threads of wave 0 store a row's results.
template <typename T>
__device__ __forceinline__ void store_row(const ScoreArgs &a, const T *row, int64_t o, const Stat &st, const uint64_t *best) {
  const int lane = threadIdx.x;
  const bool none = st.m == -INFINITY;
  const float log_s = logf(st.s);
  auto log_p = [&](float x) { return none ? -INFINITY : (x - st.m) - log_s; };
  if (lane < a.K) {
    const uint64_t e = best[lane];
    a.alt_id[o * a.K + lane] = e == 0 ? -1 : ~int32_t(uint32_t(e));
    a.alt_logprob[o * a.K + lane] = e == 0 ? -INFINITY : log_p(value_of(uint32_t(e >> 32)));
  }
  if (lane == 0) a.entropy[o] = none ? 0.f : log_s - kLn2 * (st.t / st.s);
  if (lane == 1 && a.token_id != nullptr) {
    const int id = a.token_id[o];
    a.logprob[o] = id < 0 || id >= a.V ? -INFINITY : log_p(Vec<T>::scalar(row + id));
  }
}

// One workgroup per row of the buffer.
template <typename T, int NT, bool ALT>
__global__ __launch_bounds__(NT) void token_scores_kernel(const T *__restrict__ logits, ScoreArgs a) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  __shared__ Shared<NT> sh;
  const int i = blockIdx.x, b = blockIdx.y;
  if (a.suffix_len != nullptr && i >= a.suffix_len[b]) return;
  const T *row = logits + int64_t(b) * a.batch_stride + int64_t(i) * a.row_stride;
  const Stat st = scan_segment<T, NT, ALT>(row, 0, a.V, a.K, sh, lds);
  if (threadIdx.x < kWave) store_row(a, row, int64_t(b) * a.S + i, st, sh.best);
}

// Rows in up to 2^kMaxLog2 segments, as many as the number of active rows leaves compute units for: kSplitTarget workgroups of 256 threads or half as
// many of 512, which buffers of fewer than kSplitRows rows take (workgroups of 512 up to kSplitTarget: the same times).
constexpr int kSplitTarget = 512;
constexpr int kMaxLog2 = 4;
constexpr int kMinSegment = 4096;
constexpr int kSplitRows = 512;
constexpr int kMaxScannedBatch = 256;
constexpr int64_t kMaxSplitGrid = int64_t(1) << 22;
__host__ __device__ constexpr int segment_words(int K) { return 3 + 2 * K; }
constexpr size_t split_bytes(int K) { return size_t(kSplitTarget) * segment_words(K) * sizeof(uint64_t); }

// Position among the active rows: how many there are, and sequence and row of the n-th.
struct ActiveRows {
  int lane, total = 0, upto = 0, n = 0;
  const ScoreArgs &a;
  __device__ __forceinline__ ActiveRows(const ScoreArgs &args) : lane(threadIdx.x & (kWave - 1)), a(args) {
    if (a.suffix_len == nullptr) total = a.B * a.S;
    else
      for (int b0 = 0; b0 < a.B; b0 += kWave) total += scan(b0);
  }
  __device__ __forceinline__ int scan(int b0) {
    const int b = b0 + lane;
    n = b < a.B ? min(max(a.suffix_len[b], 0), a.S) : 0;
    upto = n;
    upto += __builtin_amdgcn_update_dpp(0, upto, 0x111, 0xf, 0xf, false);  // row_shr:1
    upto += __builtin_amdgcn_update_dpp(0, upto, 0x112, 0xf, 0xf, false);  // row_shr:2
    upto += __builtin_amdgcn_update_dpp(0, upto, 0x114, 0xf, 0xf, false);  // row_shr:4
    upto += __builtin_amdgcn_update_dpp(0, upto, 0x118, 0xf, 0xf, false);  // row_shr:8
    upto += __builtin_amdgcn_update_dpp(0, upto, 0x142, 0xa, 0xf, false);  // row_bcast:15 into rows 1 and 3
    upto += __builtin_amdgcn_update_dpp(0, upto, 0x143, 0xc, 0xf, false);  // row_bcast:31 into rows 2 and 3
    return __builtin_amdgcn_readlane(upto, kWave - 1);
  }
  __device__ __forceinline__ void place(int row, int &b, int &i) {
    b = 0;
    i = row;
    if (a.suffix_len == nullptr) {
      b = row / a.S;
      i = row - b * a.S;
      return;
    }
    if (a.B > kWave)
      for (;; b += kWave) {
        const int t = scan(b);
        if (i < t) break;
        i -= t;
      }
    const int s = __popcll(__ballot(upto <= i));
    i -= __builtin_amdgcn_readlane(upto, s) - __builtin_amdgcn_readlane(n, s);
    b += s;
  }
};

template <typename T, int NT, bool ALT>
__global__ __launch_bounds__(NT) void token_scores_split_kernel(const T *__restrict__ logits, ScoreArgs a, int max_log2, uint32_t tag, uint64_t *segments) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  __shared__ Shared<NT> sh;
  const int tid = threadIdx.x, lane = tid & (kWave - 1);
  ActiveRows active(a);
  int k = 0;
  while (k < max_log2 && active.total << (k + 1) <= kSplitTarget * 256 / NT) ++k;
  const int row_n = int(blockIdx.x >> k), seg = int(blockIdx.x) & ((1 << k) - 1);
  if (row_n >= active.total) return;
  int b, i;
  active.place(row_n, b, i);
  const T *row = logits + int64_t(b) * a.batch_stride + int64_t(i) * a.row_stride;
  const int len = (((a.V + (1 << k) - 1) >> k) + 63) & ~63, c0 = min(a.V, seg * len);
  Stat st = scan_segment<T, NT, ALT>(row, c0, min(a.V, c0 + len), a.K, sh, lds);
  if (k > 0) {
    const int words = segment_words(a.K), all = words << k;
    uint64_t *w = segments + int64_t(row_n) * all;
    if (tid < words) {
      const uint32_t mine = tid == 0   ? __float_as_uint(st.m)
                            : tid == 1 ? __float_as_uint(st.s)
                            : tid == 2 ? __float_as_uint(st.t)
                                       : uint32_t(sh.best[(tid - 3) >> 1] >> (tid & 1 ? 32 : 0));
      __hip_atomic_store(w + seg * words + tid, uint64_t(mine) << 32 | tag, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // they are where every workgroup sees them
    __syncthreads();
    uint32_t *got = reinterpret_cast<uint32_t *>(lds);
    bool there = true;
    for (int j = tid; j < all; j += NT) {
      const uint64_t x = __hip_atomic_load(w + j, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      there = there && uint32_t(x) == tag;
      got[j] = uint32_t(x >> 32);
    }
    if (!__syncthreads_and(there)) return;
    for (int j = tid; j < all; j += NT) __hip_atomic_store(w + j, uint64_t(0), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    Stat part = {-INFINITY, 0.f, 0.f};
    if (lane < 1 << k) part = {__uint_as_float(got[lane * words]), __uint_as_float(got[lane * words + 1]), __uint_as_float(got[lane * words + 2])};
    st = merge_stats(part);
    if (ALT) {
      uint64_t *entries = reinterpret_cast<uint64_t *>(lds) + ((all + 3) >> 2) * 2;  // (16-byte aligned)
      for (int j = tid; j < a.K << k; j += NT) {
        const int s = j / a.K, e = j - s * a.K;
        entries[j] = uint64_t(got[s * words + 3 + 2 * e]) << 32 | got[s * words + 4 + 2 * e];
      }
      if (tid < a.K) sh.best[tid] = 0;
      __syncthreads();
      rank_entries<NT>(sh, entries, a.K << k, a.K);
    }
  }
  if (tid < kWave) store_row(a, row, int64_t(b) * a.S + i, st, sh.best);
}

struct Plan {
  int nt;        // threads of a workgroup
  int max_log2;  // rows may be cut into up to 2^max_log2 segments
};
inline Plan plan(int64_t rows, int V, int elem_bytes) {
  Plan p = {64, 0};
  const int64_t nvec = int64_t(V) * elem_bytes / 16;
  if (nvec >= 64 * 32) p.nt = 256;
  if (p.nt == 256)
    while (V > kMinCut && p.max_log2 < kMaxLog2 && (V >> (p.max_log2 + 1)) >= kMinSegment) ++p.max_log2;
  if (p.max_log2 > 0 && rows < kSplitRows) p.nt = 512;
  return p;
}

template <typename T, bool ALT>
int32_t launch(const Plan &p, bool split, const T *z, const ScoreArgs &a, void *workspace, hipStream_t st) {
  const int64_t rows = int64_t(a.B) * a.S;
  auto whole = [&](auto kernel, int nt, size_t bytes) { kernel<<<dim3(a.S, a.B), nt, bytes, st>>>(z, a); };
  auto cut = [&](auto kernel, int nt, size_t bytes) {
    const int64_t most = rows << p.max_log2, target = int64_t(kSplitTarget) * 256 / nt;
    const int64_t grid = rows > target ? rows : most < target ? most : target;
    kernel<<<unsigned(grid), nt, bytes, st>>>(z, a, p.max_log2, call_tag(), static_cast<uint64_t *>(workspace));
  };
  if (split && p.nt == 512) cut(token_scores_split_kernel<T, 512, ALT>, 512, dynamic_lds<T, 512, ALT>(a.V));
  else if (split) cut(token_scores_split_kernel<T, 256, ALT>, 256, dynamic_lds<T, 256, ALT>(a.V));
  else if (p.nt == 64) whole(token_scores_kernel<T, 64, ALT>, 64, dynamic_lds<T, 64, ALT>(a.V));
  else whole(token_scores_kernel<T, 256, ALT>, 256, dynamic_lds<T, 256, ALT>(a.V));
  LSP_CHECK_LAUNCH("lsp_token_scores: launch");
  return LSP_OK;
}

}  // namespace
}  // namespace lsp

extern "C" size_t lsp_token_scores_workspace_bytes(int32_t B, int32_t S, int32_t V, int32_t num_alt) {
  if (B <= 0 || S <= 0 || V <= 0 || num_alt < 0 || num_alt > lsp::kMaxAlt) return 0;
  // the dtype is not an argument here: enough for either
  const int64_t rows = int64_t(B) * S;
  return lsp::plan(rows, V, 2).max_log2 > 0 || lsp::plan(rows, V, 4).max_log2 > 0 ? lsp::split_bytes(num_alt) : 0;
}

extern "C" int32_t lsp_token_scores(int32_t dtype, const void *logits, int32_t B, int32_t S, int32_t V, int64_t row_stride,
                                    int64_t batch_stride, const int32_t *suffix_len, const int32_t *token_id, int32_t num_alt,
                                    float *logprob, float *entropy, int32_t *alt_id, float *alt_logprob, void *workspace,
                                    size_t workspace_bytes, void *stream) {
  using namespace lsp;
  LSP_CHECK_ARG(dtype == LSP_F32 || dtype == LSP_BF16, "lsp_token_scores: unknown dtype %d", dtype);
  LSP_CHECK_ARG(B > 0 && S > 0 && V > 0, "lsp_token_scores: need B>0, S>0, V>0 (got %d %d %d)", B, S, V);
  LSP_CHECK_ARG(B <= 65535 && S <= 65535, "lsp_token_scores: B and S must be <= 65535");
  LSP_CHECK_ARG(V <= 1 << 30, "lsp_token_scores: V must be <= 2^30");
  LSP_CHECK_ARG(num_alt >= 0 && num_alt <= kMaxAlt, "lsp_token_scores: num_alt must be 0..%d (got %d)", kMaxAlt, num_alt);
  LSP_CHECK_ARG(logits && entropy, "lsp_token_scores: null pointer");
  LSP_CHECK_ARG((token_id != nullptr) == (logprob != nullptr), "lsp_token_scores: token_id and logprob come together");
  LSP_CHECK_ARG(num_alt == 0 || (alt_id && alt_logprob), "lsp_token_scores: alternatives need alt_id and alt_logprob");
  if (row_stride == 0) row_stride = V;
  if (batch_stride == 0) batch_stride = int64_t(S) * row_stride;
  LSP_CHECK_ARG(row_stride >= V && batch_stride >= 0, "lsp_token_scores: bad strides");
  LSP_CHECK_ARG((reinterpret_cast<uintptr_t>(logits) & (elem_size(dtype) - 1)) == 0, "lsp_token_scores: logits misaligned");
  const int64_t rows = int64_t(B) * S;
  const Plan p = plan(rows, V, int(elem_size(dtype)));
  const bool room = workspace != nullptr && workspace_bytes >= split_bytes(num_alt) && aligned16(workspace);
  const bool split = p.max_log2 > 0 && room && (suffix_len == nullptr || B <= kMaxScannedBatch) && rows <= kMaxSplitGrid;
  const ScoreArgs a = {B, S, V, num_alt, row_stride, batch_stride, suffix_len, token_id, logprob, entropy, alt_id, alt_logprob};
  hipStream_t st = static_cast<hipStream_t>(stream);
  const auto *zb = static_cast<const uint16_t *>(logits);
  const auto *zf = static_cast<const float *>(logits);
  if (dtype == LSP_BF16) return num_alt ? launch<uint16_t, true>(p, split, zb, a, workspace, st) : launch<uint16_t, false>(p, split, zb, a, workspace, st);
  return num_alt ? launch<float, true>(p, split, zf, a, workspace, st) : launch<float, false>(p, split, zf, a, workspace, st);
}
