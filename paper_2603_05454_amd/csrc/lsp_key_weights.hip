// lsp_attn_key_weights: the attention mass that every key received from the active queries of its group.
//
// With c = scale log2(e) and L[h,i] the base-2 logarithm of the sum over all keys of 2^(c q.k):
//   mass[g,t] = sum over heads h of group g and rows i < N of 2^(c q[i,h].k[t,g] - L[h,i])
//
// Units are (layer, sequence, KV head); the rows of all heads of a group are one list (entry e: row e % N of head e / N), since they meet the same
// keys.  Three kernels, each of which takes the units whose lengths, known on the device alone, are its own:
//   few_rows_kernel   up to 64 rows and as many keys as eight waves have registers for scores of (2048 with 32 rows, 768 with 64): one product, one
//                     exponential a score.  Bound by the bytes of the keys: 8 layers of 32 heads, 16 x 21 rows on 1536 keys, 1.7 GB, 324 us = 5.2 TB/s.
//   row_log_kernel    L of every other row, and
//   key_sum_kernel    the sums down the columns, each from its own product of queries and keys.  (The products kept between them would be 1.3e9 numbers a layer
//                     at 8 x 1024 rows of 32 heads on 5120 keys.)  Bound by instructions and power: there 376 and 388 us, 0.92 PFLOP/s, with vector
//                     instructions in 55-64 % of the cycles, matrix instructions in 43-45 %, at 1.95 GHz.  The two do not overlap further in any order that
//                     was tried (all of the one, then all of the other; halves; exponents, powers and additions a step apart: 753-774 us
//                     in all for 735), and the attention of the same products, by hand and with half the exponentials, takes 595 us, at the power limit.
// More rows than there are keys for, or fewer: both of the latter divide what is long, rows or keys, among workgroups that the others leave free
// (kGroups); one layer of 4 x 497 rows of 28 heads on 4 KV heads and 1500 keys 80 -> 55 us.
//
// The last two are the same loop with the operands exchanged.  A wave holds NS blocks of 32 rows of one operand as matrix fragments in registers (queries for
// the logarithms, keys for the sums) and all four waves of the workgroup read the other one from LDS, 32 rows at a time, from a ring that
// is filled by loads that go straight to LDS.  Scores come out transposed, keys x queries (v_mfma_f32_32x32x16_bf16, or 32x32x2 in fp32),
// so a lane's 16 scores are of ONE query: its reference and sum, or its L, are per-lane numbers, and nothing crosses lanes in the loop:
// the logarithm joins two lanes at the end, the sums of a key stay one register for each of the wave's 32 x NS keys and are reduced over
// 32 lanes once.  Scores, exponentials and sums are fp32, in an order that sizes alone decide.
#include <math.h>

#include <type_traits>

#include "lsp_attn.h"

namespace lsp {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kWaves = 4;
constexpr int kThreads = kWaves * kWave;
constexpr int kStages = 4;           // of the ring
constexpr int kLogs = 4096;          // rows whose L are in LDS at a time
constexpr int kMaxParts = 16;        // of the keys, for the logarithms of few rows
constexpr int kPartKeys = 128;       // a part has at least
constexpr int kPartRows = 128;       // a part of the rows, for the sums of few keys, has at least
constexpr int kGroups = 512;         // workgroups that a launch is divided into where it can be: two to a compute unit
// Keys of more bytes than this (as many as the attention's K/V, which are twice that) are loaded with the non-temporal hint: in the case above
// 343 -> 332 us.
constexpr int64_t kOnceBytes = int64_t(160) << 20;
constexpr float kFarBelow = -1.7e38f;  // a reference below all scores

struct WeightArgs {
  const int32_t *prefix_len, *suffix_len;
  int32_t B, S, Hkv, C, rep;
  int32_t units, groups, spread, max_parts;  // (layer, sequence, KV head)s; workgroups of one; each unit in 2^spread pieces
  int32_t log_rows;  // rows of a workgroup of row_log_kernel
  uint32_t tag;      // of the call, beside numbers that workgroups hand over
  float scale, decay;
  int64_t qs[3], ks[3], cs[3];  // bytes: batch, row, head
  float *row_log;   // [max_parts, units, rep * S]
  uint64_t *sums;   // [kGroups, 256]: parts of sums, or null
  float *weights;   // of the launch's first layer: [layers, B, Hkv, C]
};
struct WeightLayers {
  const char *q[kMaxAttnLayers], *k_suf[kMaxAttnLayers], *k_cache[kMaxAttnLayers];
};

// Geometry of a tile of 32 rows in LDS.  16-byte pieces of a row are exchanged so that the 32 lanes that read the same piece of 32 rows meet
// all banks alike: piece p of row r is at p ^ (r % 16) of its 256 bytes; where two rows share 256 bytes, at (8 (r % 2) + p) ^ (r / 2 % 8).
template <typename T, int D>
struct Tile {
  static constexpr int kRowBytes = D * int(sizeof(T));     // 128, 256 or 512
  static constexpr int kFrags = kRowBytes / 32;            // pieces of a row that a lane has: lane l those of row l % 32 with number % 2 = l / 32
  static constexpr int kBytes = 32 * kRowBytes;
  static constexpr int kLoads = kFrags / kWaves;           // wave-wide loads of 1 KB that a wave makes for a tile
  // where lane's fragment c is
  static __device__ __forceinline__ int frag_at(int lane, int c) {
    const int r = lane & 31, p = 2 * c + (lane >> 5);
    if (kRowBytes == 128) return (r >> 1) * 256 + 16 * ((8 * (r & 1) + p) ^ (r >> 1 & 7));
    return r * kRowBytes + (p >> 4) * 256 + 16 * ((p & 15) ^ (r & 15));
  }
  // row and byte of it that belong to 16-byte place y
  static __device__ __forceinline__ void place(int y, int &row, int &byte) {
    const int line = y >> 4, x = y & 15;
    if (kRowBytes == 128) {
      const int z = x ^ (line & 7);
      row = 2 * line + (z >> 3);
      byte = 16 * (z & 7);
    } else {
      constexpr int kLines = kRowBytes < 256 ? 1 : kRowBytes / 256;
      row = line / kLines;
      byte = 256 * (line % kLines) + 16 * (x ^ (row & 15));
    }
  }
  // byte that belongs to place 64 k + y, from place y's, y < 64 (its row: 1024 / kRowBytes k on)
  static __device__ __forceinline__ int byte_of(int byte, int k) {
    return byte ^ 16 * (kRowBytes == 128 ? 4 * k & 4 : kRowBytes == 256 ? 4 * k & 12 : 2 * k & 14);
  }
};

// scores += A x B for one fragment of each
__device__ __forceinline__ void step(f32x16 &s, const u32x4 &a, const u32x4 &b, const uint16_t *) {
  s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), s, 0, 0, 0);
}
__device__ __forceinline__ void step(f32x16 &s, const u32x4 &a, const u32x4 &b, const float *) {
  const f32x4 x = __builtin_bit_cast(f32x4, a), y = __builtin_bit_cast(f32x4, b);
#pragma unroll
  for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_32x32x2f32(x[e], y[e], s, 0, 0, 0);
}
// row of the product that register r of a lane holds (its column: lane % 32)
__device__ __forceinline__ int product_row(int lane, int r) { return 8 * (r >> 2) + 4 * (lane >> 5) + (r & 3); }

// v_maximum3_f32.  (Not in asm: the compiler has to see that it reads what a matrix instruction wrote, and wait for that.)
__device__ __forceinline__ float max3(float a, float b, float c) { return __builtin_elementwise_maximum(__builtin_elementwise_maximum(a, b), c); }

// Sum over lane % 32 of 16 numbers: lane l gets the one with number l % 16.  Every step halves what a lane has to send: the partner is the
// mirror image within 16, 8, 4 and 2 lanes, so that it agrees in the bits that earlier steps went by (46 instructions, 80 for each by itself).
template <int CTRL, int HALF>
__device__ __forceinline__ void fold(float (&x)[16], int lane) {
  const bool upper = lane & HALF;
#pragma unroll
  for (int r = 0; r < HALF; ++r) {
    const float keep = upper ? x[r + HALF] : x[r], send = upper ? x[r] : x[r + HALF];
    x[r] = keep + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(send), CTRL, 0xf, 0xf, true));
  }
}
__device__ __forceinline__ float sum_of_lanes(float (&x)[16], int lane) {
  fold<0x140, 8>(x, lane);  // row_mirror
  fold<0x141, 4>(x, lane);  // row_half_mirror
  fold<0x1b, 2>(x, lane);   // quad_perm [3,2,1,0]
  fold<0xb1, 1>(x, lane);   // quad_perm [1,0,3,2]
  return x[0] + __shfl_xor(x[0], 16);
}

// The compiler may not put off what makes x to behind a later branch, away from the matrix instructions it is meant to run beside.
__device__ __forceinline__ void stays_here(float &x) { asm volatile("" : "+v"(x)); }

struct Unit {
  int n, l, b, g, w, N, P, rows, keys;  // number, its parts, workgroup of it, lengths, rows of all heads, keys
  bool valid;
};
__device__ __forceinline__ Unit unit_at(const WeightArgs &a, int n) {
  Unit u;
  u.n = n;
  u.valid = n < a.units;
  u.g = n % a.Hkv;
  u.b = n / a.Hkv % a.B;
  u.l = n / a.Hkv / a.B;
  u.w = u.N = u.P = 0;
  if (u.valid) {
    u.N = min(max(a.suffix_len[u.b], 0), a.S);
    u.P = min(max(a.prefix_len[u.b], 0), a.C);
  }
  u.rows = a.rep * u.N;
  u.keys = u.P + u.N;
  return u;
}
// The workgroups of a unit read the same stream: ids that are equal modulo 8 share an XCD's L2.
__device__ __forceinline__ Unit unit_of(const WeightArgs &a, int id) {
  const int per_piece = a.groups >> a.spread, rest = id >> 3, piece = rest / per_piece * 8 + (id & 7);
  Unit u = unit_at(a, piece >> a.spread);
  u.w = ((rest % per_piece) << a.spread) + (piece & ((1 << a.spread) - 1));
  return u;
}
// `most`: pieces of work that a unit may have.  They are dealt out to as many workgroups as there are, which find out how many there
// are from the lengths; with more than kGroups in all, few of them find none.
int64_t place_grid(WeightArgs &a, int64_t most) {
  a.spread = 0;
  if (a.units < 32)
    while ((a.units << a.spread) % 8 != 0) ++a.spread;
  const int64_t g = (2 * kGroups + a.units - 1) / a.units, one = int64_t(1) << a.spread;
  a.groups = int32_t(((g < most ? g : most) + one - 1) / one * one);
  return ((int64_t(a.units) << a.spread) + 7) / 8 * 8 * (a.groups >> a.spread);
}
// Parts of the keys of a unit, for the logarithms of its rows: both kernels go by this.
__device__ __forceinline__ int key_parts(const WeightArgs &a, const Unit &u) {
  const int groups = a.units * ((u.rows + a.log_rows - 1) / a.log_rows);
  return max(1, min(min(kGroups / groups, a.max_parts), u.keys / kPartKeys));
}
// Parts of its rows, for the sums of `tiles` groups of keys.
__device__ __forceinline__ int row_parts(const WeightArgs &a, const Unit &u, int tiles) {
  return a.sums == nullptr ? 1 : max(1, min(kGroups / (a.units * tiles), u.rows / kPartRows));
}

// Units of up to 64 rows: their scores are kept (few_rows_kernel), or, with more keys than registers, made twice by waves that share the keys
// (few_rows_stream).
constexpr int kFewRows = 64;
template <typename T, int D>
constexpr int kFewRowsOf = Tile<T, D>::kRowBytes == 512 ? 32 : kFewRows;  // (as many as there are registers for)
constexpr int kFewWaves = 8;
template <int RS>
constexpr int kFewTiles = RS == 1 ? 8 : 3;  // a wave's: 128 or 96 registers of scores
template <typename T, int D>
__host__ __device__ constexpr bool keeps_scores(int64_t rows, int64_t keys) {
  return Tile<T, D>::kRowBytes <= 256 && rows <= kFewRows && keys <= kFewWaves * 32 * (rows <= 32 ? kFewTiles<1> : kFewTiles<2>);
}

// A ring of tiles.  fetch(tile, place's row, place's byte) says where a lane's 16 bytes are.
template <typename T, int D>
struct Ring {
  typedef Tile<T, D> G;
  char *lds;
  int wave, row[G::kLoads], byte[G::kLoads];
  __device__ __forceinline__ Ring(char *at) : lds(at) {
    wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
#pragma unroll
    for (int k = 0; k < G::kLoads; ++k) G::place((k * kWaves + wave) * kWave + (threadIdx.x & (kWave - 1)), row[k], byte[k]);
  }
  template <typename F>
  __device__ __forceinline__ void ask(int stage, F fetch) {
#pragma unroll
    for (int k = 0; k < G::kLoads; ++k)
      __builtin_amdgcn_global_load_lds(fetch(k, row[k], byte[k]),
                                       (__attribute__((address_space(3))) void *)(lds + stage * G::kBytes + (k * kWaves + wave) * 1024), 16, 0, 0);
  }
  // all but the newest TILES tiles asked for are there, for every wave, and what it read before is in registers
  template <int TILES>
  static __device__ __forceinline__ void wait() {
    constexpr int kCount = TILES * G::kLoads;
    __builtin_amdgcn_s_waitcnt(0x0070 | (kCount & 15) | (kCount >> 4) << 14);  // vmcnt(kCount) lgkmcnt(0)
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  }
  __device__ __forceinline__ void read(u32x4 (&f)[G::kFrags], int stage, const int (&at)[G::kFrags]) const {
#pragma unroll
    for (int c = 0; c < G::kFrags; ++c) f[c] = *reinterpret_cast<const u32x4 *>(lds + stage * G::kBytes + at[c]);
  }
};

// A lane's fragments of one row.
template <int F>
__device__ __forceinline__ void load_row(u32x4 (&f)[F], const char *row, int lane) {
#pragma unroll
  for (int c = 0; c < F; ++c) f[c] = *reinterpret_cast<const u32x4 *>(row + 32 * c + 16 * (lane >> 5));
}

// (tiles beyond the end are asked for again as the last one, so that as many loads are under way everywhere)
template <typename Ask>
__device__ __forceinline__ void fill(int first, int end, Ask ask) {
#pragma unroll
  for (int k = 0; k < kStages; ++k) ask(min(first + k, end - 1), k);
}

// The wave's NS blocks (`own`) times each of the tiles [first, end) of the stream, one product behind the other: while the matrix cores make one,
// the vector units use the one before.  Tile j + 1 is read from the ring at the start of tile j's last product, so that its barrier is also the one
// behind which tile j's stage is free.
// The first tiles have been asked for (fill).
// begin(parity of a tile, tile) comes before a tile's first product.  Of a product, with its block and its tile, the next one's first half goes by
// ready() (READY) and its second half, or all of it, by use(product, block, parity, first, end): numbers [first, end) of 16.
// STREAM_ROWS: the products' rows are the stream's (its columns otherwise).
template <bool STREAM_ROWS, bool READY, typename T, int D, int NS, typename Ask, typename Begin, typename Ready, typename Use>
__device__ __forceinline__ void run_pipeline(Ring<T, D> &ring, int first, int end, const int (&at)[Tile<T, D>::kFrags], bool live,
                                             const u32x4 (&own)[NS][Tile<T, D>::kFrags], float nothing, Ask ask, Begin begin, Ready ready, Use use) {
  typedef Tile<T, D> G;
  constexpr int F = G::kFrags;
  Ring<T, D>::template wait<kStages - 1>();
  auto next = [&](int j, int stage) {  // tile j + 1 is there, tile j's stage takes tile j + kStages
    Ring<T, D>::template wait<kStages - 2>();
    ask(min(j + kStages, end - 1), stage);
  };
  if (!live) {
    for (int j = first, stage = 0; j < end; ++j, stage = (stage + 1) % kStages) next(j, stage);
    __builtin_amdgcn_s_waitcnt(0x0F70);
    return;
  }
  constexpr bool kAhead = G::kRowBytes < 512;  // (there are no registers for two tiles of these)
  u32x4 x[kAhead ? 2 : 1][F];
  f32x16 s[2];
#pragma unroll
  for (int r = 0; r < 16; ++r) s[1][r] = nothing;
  ring.read(x[0], 0, at);
  auto tile = [&](int j, auto place) {
    constexpr int kStage = decltype(place)::value, P = kStage & 1;
    begin(P, j);
#pragma unroll
    for (int n = 0; n < NS; ++n) {
      if (kAhead && n == NS - 1) {
        next(j, kStage);
        ring.read(x[1 - P], (kStage + 1) % kStages, at);
      }
      // (the product before: block `before` of this tile or the one before)
      const int cur = NS == 2 ? n : P, before = NS == 2 ? 1 - n : 0, its_parity = NS == 2 && n == 1 ? P : 1 - P;
      f32x16 &now = s[cur], &old = s[1 - cur];
      auto make = [&](int c) {
        if (STREAM_ROWS) step(now, x[kAhead ? P : 0][c], own[n][c], static_cast<const T *>(nullptr));
        else step(now, own[n][c], x[kAhead ? P : 0][c], static_cast<const T *>(nullptr));
      };
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int r = 0; r < 16; ++r) now[r] = 0.f;
      constexpr int kFrom = READY ? F / 2 : 0, kEach = 16 / (F - kFrom), kMatrix = sizeof(T) == 2 ? 1 : 4;
#pragma unroll
      for (int c = 0; c < kFrom; ++c) make(c);
      if (READY) ready(old, before, NS == 2 && n == 1 ? j : j - 1);
#pragma unroll
      for (int c = kFrom; c < F; ++c) {
        make(c);
        use(old, before, its_parity, (c - kFrom) * kEach, (c - kFrom + 1) * kEach);
      }
      // matrix, vector and exponential instructions in turn
#pragma unroll
      for (int c = kFrom; c < F; ++c) {
        __builtin_amdgcn_sched_group_barrier(0x008, kMatrix, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x002, kEach + 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x400, kEach, 0);
        __builtin_amdgcn_sched_group_barrier(0x002, kEach, 0);
      }
    }
    if (!kAhead) {
      next(j, kStage);
      ring.read(x[0], (kStage + 1) % kStages, at);
    }
  };
  static_assert(kStages == 4, "a round of the loop");
  for (int j = first;; j += kStages) {
    tile(j, std::integral_constant<int, 0>());
    if (j + 1 == end) break;
    tile(j + 1, std::integral_constant<int, 1>());
    if (j + 2 == end) break;
    tile(j + 2, std::integral_constant<int, 2>());
    if (j + 3 == end) break;
    tile(j + 3, std::integral_constant<int, 3>());
    if (j + 4 == end) break;
  }
  const bool last_is_even = (end - first) & 1;
  // the last product
  auto finish = [&](f32x16 &last, int parity) {
    if (READY) ready(last, NS - 1, end - 1);
    use(last, NS - 1, parity, 0, 16);
  };
  if (NS == 2) {
    if (last_is_even) finish(s[1], 0); else finish(s[1], 1);
  } else {
    if (last_is_even) finish(s[0], 0); else finish(s[1], 1);
  }
  __builtin_amdgcn_s_waitcnt(0x0F70);  // nothing is still on its way into LDS
}

struct Operands {
  const char *q, *kc, *ks;  // of the unit: first head of its group, its KV head
  __device__ __forceinline__ Operands(const WeightArgs &a, const WeightLayers &L, const Unit &u)
      : q(L.q[u.l] + u.b * a.qs[0] + u.g * a.rep * a.qs[2]), kc(L.k_cache[u.l] + u.b * a.cs[0] + u.g * a.cs[2]),
        ks(L.k_suf[u.l] + u.b * a.ks[0] + u.g * a.ks[2]) {}
  __device__ __forceinline__ const char *row(const WeightArgs &a, const Unit &u, int e) const {  // entry e of the list of rows
    const int h = e / u.N;
    return q + (e - h * u.N) * a.qs[1] + h * a.qs[2];
  }
  __device__ __forceinline__ const char *key(const WeightArgs &a, const Unit &u, int t) const {
    return t < u.P ? kc + t * a.cs[1] : ks + (t - u.P) * a.ks[1];
  }
};
__device__ __forceinline__ int64_t logs_at(const WeightArgs &a, const Unit &u, int part) { return (int64_t(part) * a.units + u.n) * (int64_t(a.rep) * a.S); }
// a row's logarithm from those of the parts of the keys
__device__ __forceinline__ float row_log_of(const WeightArgs &a, const Unit &u, int parts, int e) {
  const float *at = a.row_log + logs_at(a, u, 0) + e;
  const int64_t stride = int64_t(a.units) * a.rep * a.S;
  if (parts == 1) return *at;
  float x[kMaxParts], top = -INFINITY, sum = 0.f;
#pragma unroll
  for (int p = 0; p < kMaxParts; ++p) x[p] = p < parts ? at[p * stride] : -INFINITY;
#pragma unroll
  for (int p = 0; p < kMaxParts; ++p) top = fmaxf(top, x[p]);
#pragma unroll
  for (int p = 0; p < kMaxParts; ++p) sum += __builtin_amdgcn_exp2f(x[p] - top);
  return top + __builtin_amdgcn_logf(sum);
}
// Lanes with l % 32 < 16 have a key's mass.
__device__ __forceinline__ void store_mass(const WeightArgs &a, const Unit &u, int t, float mass, int lane) {
  if ((lane & 16) || t >= min(u.keys, a.C)) return;
  float *w = a.weights + int64_t(u.n) * a.C + t;
  *w = t < u.P && a.decay != 0.f ? __builtin_fmaf(a.decay, *w, mass) : mass;
}
// a lane's running sum over keys of 2^(score - ref), in two chains of additions
struct LogSum {
  float ref = kFarBelow, sum = 0.f, sum2 = 0.f;
  // the reference for these scores too (seldom moved: sums of 2^8 at most for each key are far from the end of fp32's range)
  __device__ __forceinline__ void cover(const f32x16 &s, float sc) {
    float top = max3(s[0], s[1], s[2]);
#pragma unroll
    for (int r = 3; r < 15; r += 2) top = max3(top, s[r], s[r + 1]);
    top = max3(top, s[15], s[15]) * sc;
    if (__any(top > ref + 8.f)) {
      const float to = fmaxf(top, ref), f = __builtin_amdgcn_exp2f(ref - to);
      sum *= f;
      sum2 *= f;
      ref = to;
    }
  }
  __device__ __forceinline__ void add(const f32x16 &s, float sc, int r0, int r1) {
#pragma unroll
    for (int r = r0; r < r1; ++r) {
      float &to = r & 1 ? sum : sum2;
      to += __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], sc, -ref));
      stays_here(to);
    }
  }
  // with the other half of the keys, which lane +- 32 has
  __device__ __forceinline__ void join() {
    const float top = fmaxf(ref, __shfl_xor(ref, 32));
    sum = (sum + sum2) * __builtin_amdgcn_exp2f(ref - top);
    sum += __shfl_xor(sum, 32);
    ref = top;
  }
};
__device__ __forceinline__ void mask_keys(f32x16 &s, int first, int keys, int lane) {
  if (first + 32 > keys) {
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = first + product_row(lane, r) < keys ? s[r] : -INFINITY;
  }
}

// ---- few rows ----------------------------------------------------------------------
// The rows (32 RS of them at most) are every wave's; the waves share the keys, in tiles of 32 that each fetches for itself.
template <typename T, int D, bool ONCE = false>  // ONCE: non-temporal loads
struct OwnTiles {
  typedef Tile<T, D> G;
  static constexpr int kLoads = G::kBytes / 1024, kDepth = 2;  // tiles ahead
  char *lds;
  int lane;
  __device__ __forceinline__ OwnTiles(char *base, int wave, int ln) : lds(base + wave * kDepth * G::kBytes), lane(ln) {}
  __device__ __forceinline__ void ask(const WeightArgs &a, const Unit &u, const Operands &o, int j, int stage) const {
    int own_lane = lane;
    asm volatile("" : "+v"(own_lane));  // (places are computed anew for every tile: kept, they take the registers of scores)
    // Load k takes the rows kRows k on from the first one's, with pieces exchanged by k alone (Tile::place).
    constexpr int kRows = 1024 / G::kRowBytes;
    int row, byte;
    G::place(own_lane, row, byte);
    const int t = 32 * j;
    auto load = [&](int k, const char *at) {
      __builtin_amdgcn_global_load_lds(at, (__attribute__((address_space(3))) void *)(lds + stage * G::kBytes + k * 1024), 16, 0, ONCE ? 2 : 0);
    };
    auto whole = [&](const char *base, int64_t stride) {  // (per load three vector instructions; 25 where rows are looked up one by one)
      const uint32_t first = uint32_t(row) * uint32_t(stride);
#pragma unroll
      for (int k = 0; k < kLoads; ++k) load(k, base + k * kRows * stride + (first + uint32_t(G::byte_of(byte, k))));
    };
    if (t + 32 <= u.P) whole(o.kc + t * a.cs[1], a.cs[1]);
    else if (t >= u.P && t + 32 <= u.keys) whole(o.ks + (t - u.P) * a.ks[1], a.ks[1]);
    else {
#pragma unroll
      for (int k = 0; k < kLoads; ++k) load(k, o.key(a, u, min(t + row + k * kRows, u.keys - 1)) + G::byte_of(byte, k));
    }
  }
  // The tile in `stage`, which may be written again then; `newer`: one asked for later may be under way.
  __device__ __forceinline__ void read(u32x4 (&kf)[G::kFrags], int stage, bool newer) const {
    if (newer) __builtin_amdgcn_s_waitcnt(0x0F70 | (kLoads & 15) | (kLoads >> 4) << 14);
    else __builtin_amdgcn_s_waitcnt(0x0F70);
    int own_lane = lane;
    asm volatile("" : "+v"(own_lane)::"memory");
#pragma unroll
    for (int c = 0; c < G::kFrags; ++c) kf[c] = *reinterpret_cast<const u32x4 *>(lds + stage * G::kBytes + G::frag_at(own_lane, c));
    __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
    asm volatile("" ::: "memory");
  }
};
template <int RS, int F>
__device__ __forceinline__ void load_rows(u32x4 (&qf)[RS][F], const WeightArgs &a, const Unit &u, const Operands &o, int lane) {
#pragma unroll
  for (int n = 0; n < RS; ++n) load_row(qf[n], o.row(a, u, min(32 * n + (lane & 31), u.rows - 1)), lane);
}
template <typename T, int F>
__device__ __forceinline__ void multiply(f32x16 &s, const u32x4 (&kf)[F], const u32x4 (&qf)[F]) {
#pragma unroll
  for (int r = 0; r < 16; ++r) s[r] = 0.f;
#pragma unroll
  for (int c = 0; c < F; ++c) step(s, kf[c], qf[c], static_cast<const T *>(nullptr));
}

// All of the unit's scores are kept in registers, so that K is read once and every score and exponential computed once.  Maxima and sums of the
// rows meet in LDS.  first_tiles() asks for the first ones, if that has not been done (`asked`); when the last are done with, before_end() is called.
template <typename T, int D, int RS, bool ONCE, typename FirstTiles, typename BeforeEnd>
__device__ __forceinline__ void few_rows_body(const WeightArgs &a, const Unit &u, const Operands &o, const OwnTiles<T, D, ONCE> &own, int wave, float *s_row,
                                              bool asked, FirstTiles first_tiles, BeforeEnd before_end) {
  typedef Tile<T, D> G;
  constexpr int kTiles = kFewTiles<RS>, kDepth = OwnTiles<T, D>::kDepth;
  const int lane = own.lane, tiles = (u.keys + 31) / 32, cols = min(u.keys, a.C);
  u32x4 qf[RS][G::kFrags];
  load_rows(qf, a, u, o, lane);
  if (!asked) first_tiles();
  f32x16 s[kTiles][RS];
  float top[RS], sum[RS];
#pragma unroll
  for (int n = 0; n < RS; ++n) top[n] = -INFINITY, sum[n] = 0.f;
#pragma unroll
  for (int k = 0; k < kTiles; ++k) {
    const int j = wave + k * kFewWaves;
    if (j < tiles) {
      u32x4 kf[G::kFrags];
      own.read(kf, k % kDepth, j + kFewWaves < tiles && !(k == 0 && asked));  // (the rows may be newer than the first two)
      if (j + kDepth * kFewWaves < tiles) own.ask(a, u, o, j + kDepth * kFewWaves, k % kDepth);
#pragma unroll
      for (int n = 0; n < RS; ++n) {
        multiply<T>(s[k][n], kf, qf[n]);
        mask_keys(s[k][n], 32 * j, u.keys, lane);
#pragma unroll
        for (int r = 0; r < 16; r += 2) top[n] = max3(top[n], s[k][n][r], s[k][n][r + 1]);
      }
    }
  }
  // what the weights were, before the next unit's tiles are asked for: loads come back in order
  float *w = a.weights + int64_t(u.n) * a.C, was[kTiles];
#pragma unroll
  for (int k = 0; k < kTiles; ++k) {
    const int t = 32 * (wave + k * kFewWaves) + product_row(lane, lane & 15);
    was[k] = a.decay != 0.f && t < u.P ? w[t] : 0.f;
  }
  before_end();
  // of each row over all waves; lanes l and l + 32 have the same row
  auto over_waves = [&](int slot, float (&x)[RS], auto op) {
    float *at = s_row + slot * kFewWaves * kFewRows;
#pragma unroll
    for (int n = 0; n < RS; ++n) {
      x[n] = op(x[n], __shfl_xor(x[n], 32));
      if (lane < 32) at[wave * kFewRows + 32 * n + lane] = x[n];
    }
    __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0): a plain barrier, loads stay under way
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
#pragma unroll
    for (int n = 0; n < RS; ++n) {
      x[n] = at[32 * n + (lane & 31)];
#pragma unroll
      for (int v = 1; v < kFewWaves; ++v) x[n] = op(x[n], at[v * kFewRows + 32 * n + (lane & 31)]);
    }
  };
  over_waves(0, top, [](float x, float y) { return fmaxf(x, y); });
  const float sc = a.scale * kLog2e;
#pragma unroll
  for (int k = 0; k < kTiles; ++k)
    if (wave + k * kFewWaves < tiles) {
#pragma unroll
      for (int n = 0; n < RS; ++n)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          s[k][n][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[k][n][r], sc, -top[n] * sc));
          sum[n] += s[k][n][r];
        }
    }
  over_waves(1, sum, [](float x, float y) { return x + y; });
#pragma unroll
  for (int n = 0; n < RS; ++n) sum[n] = 32 * n + (lane & 31) < u.rows ? 1.f / sum[n] : 0.f;
#pragma unroll
  for (int k = 0; k < kTiles; ++k) {
    const int j = wave + k * kFewWaves;
    if (j < tiles) {
      float x[16];
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        x[r] = s[k][0][r] * sum[0];
        if (RS == 2) x[r] = __builtin_fmaf(s[k][RS - 1][r], sum[RS - 1], x[r]);
      }
      const float mass = sum_of_lanes(x, lane);
      const int t = 32 * j + product_row(lane, lane & 15);
      if (!(lane & 16) && t < cols) w[t] = t < u.P ? __builtin_fmaf(a.decay, was[k], mass) : mass;
    }
  }
}

// One workgroup to a compute unit (128 KB of tiles on their way), which goes on to the units that are left; the next one's first tiles are fetched
// while this one's sums are formed.
template <typename T, int D, bool ONCE, typename NextOf>
__device__ __forceinline__ void few_rows_units(const WeightArgs &a, const WeightLayers &L, Unit u, char *lds, float *s_row, NextOf next_of) {
  const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const OwnTiles<T, D, ONCE> own(lds, wave, lane);
  auto fetch = [&](const Unit &u) {
    const Operands o(a, L, u);
#pragma unroll
    for (int k = 0; k < OwnTiles<T, D>::kDepth; ++k)
      if (32 * (wave + k * kFewWaves) < u.keys) own.ask(a, u, o, wave + k * kFewWaves, k);
  };
  for (bool asked = false; u.valid; asked = true) {
    const Unit next = next_of(u.n + gridDim.x);
    const Operands o(a, L, u);
    auto first_tiles = [&]() { fetch(u); };
    auto before_end = [&]() {
      if (next.valid) fetch(next);
    };
    if (u.rows <= 32) few_rows_body<T, D, 1, ONCE>(a, u, o, own, wave, s_row, asked, first_tiles, before_end);
    else few_rows_body<T, D, 2, ONCE>(a, u, o, own, wave, s_row, asked, first_tiles, before_end);
    u = next;
  }
}
template <typename T, int D>
__global__ __launch_bounds__(kFewWaves *kWave) __attribute__((amdgpu_waves_per_eu(2, 2))) void few_rows_kernel(WeightArgs a, WeightLayers L) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  __shared__ float s_row[2 * kFewWaves * kFewRows];
  auto next_of = [&](int n) {
    for (;; n += gridDim.x) {
      const Unit u = unit_at(a, n);
      if (!u.valid || (u.N > 0 && keeps_scores<T, D>(u.rows, u.keys))) return u;
    }
  };
  const Unit u = next_of(blockIdx.x);
  if (!u.valid) return;
  // (by the first unit's keys: the others' are about as many)
  if (int64_t(a.units) * u.keys * Tile<T, D>::kRowBytes > kOnceBytes) few_rows_units<T, D, true>(a, L, u, lds, s_row, next_of);
  else few_rows_units<T, D, false>(a, L, u, lds, s_row, next_of);
}

// More keys than that: what the waves have of a part of them is streamed, for the rows' logarithms (SUMS = false) and then for the sums.
template <bool SUMS, typename T, int D, int RS>
__device__ __forceinline__ void few_rows_stream(const WeightArgs &a, const WeightLayers &L, const Unit &u, int part, int parts, char *lds) {
  typedef Tile<T, D> G;
  constexpr int kDepth = OwnTiles<T, D>::kDepth;
  const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int tiles = (u.keys + 31) / 32, first = int(int64_t(tiles) * part / parts), end = int(int64_t(tiles) * (part + 1) / parts);
  const Operands o(a, L, u);
  const OwnTiles<T, D> own(lds, wave, lane);
#pragma unroll
  for (int k = 0; k < kDepth; ++k)
    if (first + wave + k * kWaves < end) own.ask(a, u, o, first + wave + k * kWaves, k);
  u32x4 qf[RS][G::kFrags];
  load_rows(qf, a, u, o, lane);
  const float sc = a.scale * kLog2e;
  LogSum to[RS];
  if (SUMS) {
#pragma unroll
    for (int n = 0; n < RS; ++n) to[n].ref = 32 * n + (lane & 31) < u.rows ? row_log_of(a, u, parts, 32 * n + (lane & 31)) : INFINITY;
  }
  int stage = 0;
  for (int j = first + wave; j < end; j += kWaves, stage ^= 1) {
    u32x4 kf[G::kFrags];
    own.read(kf, stage, j + kWaves < end && j > first + wave);
    const int t = 32 * j + product_row(lane, lane & 15);
    float *w = a.weights + int64_t(u.n) * a.C + t;
    const float was = SUMS && a.decay != 0.f && t < u.P ? *w : 0.f;  // (before the next tile: loads come back in order)
    if (j + kDepth * kWaves < end) own.ask(a, u, o, j + kDepth * kWaves, stage);
    f32x16 s[RS];
#pragma unroll
    for (int n = 0; n < RS; ++n) multiply<T>(s[n], kf, qf[n]);
    if (SUMS) {
      float x[16];
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        x[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[0][r], sc, -to[0].ref));
        if (RS == 2) x[r] += __builtin_amdgcn_exp2f(__builtin_fmaf(s[RS - 1][r], sc, -to[RS - 1].ref));
      }
      const float mass = sum_of_lanes(x, lane);
      if (!(lane & 16) && t < min(u.keys, a.C)) *w = t < u.P ? __builtin_fmaf(a.decay, was, mass) : mass;
    } else {
#pragma unroll
      for (int n = 0; n < RS; ++n) {
        mask_keys(s[n], 32 * j, u.keys, lane);
        to[n].cover(s[n], sc);
        to[n].add(s[n], sc, 0, 16);
      }
    }
  }
  if (SUMS) return;
  // (every wave is done with its tiles: their place takes references and sums)
  float *refs = reinterpret_cast<float *>(lds), *sums = refs + kWaves * kFewRows;
  __syncthreads();
#pragma unroll
  for (int n = 0; n < RS; ++n) {
    to[n].join();
    if (lane < 32) {
      refs[wave * kFewRows + 32 * n + lane] = to[n].ref;
      sums[wave * kFewRows + 32 * n + lane] = to[n].sum;
    }
  }
  __syncthreads();
  const int e = threadIdx.x;
  if (e < u.rows) {
    float top = refs[e], sum = 0.f;
#pragma unroll
    for (int v = 1; v < kWaves; ++v) top = fmaxf(top, refs[v * kFewRows + e]);
#pragma unroll
    for (int v = 0; v < kWaves; ++v) sum += sums[v * kFewRows + e] * __builtin_amdgcn_exp2f(refs[v * kFewRows + e] - top);
    a.row_log[logs_at(a, u, part) + e] = top + __builtin_amdgcn_logf(sum);
  }
}

// ---- more rows ---------------------------------------------------------------------
template <typename T, int D, int NS>
__device__ __forceinline__ void row_logs(const WeightArgs &a, const WeightLayers &L, const Unit &u, int w, int part, int parts, char *lds) {
  typedef Tile<T, D> G;
  const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), e1 = (w * kWaves + wave) * 32 * NS;
  const Operands o(a, L, u);
  u32x4 qf[NS][G::kFrags];
#pragma unroll
  for (int n = 0; n < NS; ++n) load_row(qf[n], o.row(a, u, min(e1 + 32 * n + (lane & 31), u.rows - 1)), lane);
  int at[G::kFrags];
#pragma unroll
  for (int c = 0; c < G::kFrags; ++c) at[c] = G::frag_at(lane, c);
  Ring<T, D> ring(lds);
  int from_cache[G::kLoads], from_suffix[G::kLoads];  // within a tile, from its first row
#pragma unroll
  for (int k = 0; k < G::kLoads; ++k) {
    from_cache[k] = ring.row[k] * int(a.cs[1]) + ring.byte[k];
    from_suffix[k] = ring.row[k] * int(a.ks[1]) + ring.byte[k];
  }
  auto ask = [&](int j, int stage) {
    const int t = 32 * j;
    if (t + 32 <= u.P) {
      const char *base = o.kc + t * a.cs[1];
      ring.ask(stage, [&](int k, int, int) { return base + from_cache[k]; });
    } else if (t >= u.P && t + 32 <= u.keys) {
      const char *base = o.ks + (t - u.P) * a.ks[1];
      ring.ask(stage, [&](int k, int, int) { return base + from_suffix[k]; });
    } else {
      ring.ask(stage, [&](int, int row, int byte) { return o.key(a, u, min(t + row, u.keys - 1)) + byte; });
    }
  };
  const float sc = a.scale * kLog2e;
  const int tiles = (u.keys + 31) / 32, first = int(int64_t(tiles) * part / parts), end = int(int64_t(tiles) * (part + 1) / parts);
  LogSum to[NS];
  fill(first, end, ask);
  run_pipeline<true, true, T, D, NS>(
      ring, first, end, at, e1 < u.rows, qf, -INFINITY, ask, [](int, int) {},
      [&](f32x16 &s, int n, int j) {
        mask_keys(s, 32 * j, u.keys, lane);
        to[n].cover(s, sc);
      },
      [&](const f32x16 &s, int n, int, int r0, int r1) { to[n].add(s, sc, r0, r1); });
#pragma unroll
  for (int n = 0; n < NS; ++n) {
    to[n].join();
    const int e = e1 + 32 * n + (lane & 31);
    if (lane < 32 && e < u.rows) a.row_log[logs_at(a, u, part) + e] = to[n].ref + __builtin_amdgcn_logf(to[n].sum);
  }
  __syncthreads();  // (the ring may be filled anew)
}

template <typename T, int D, int NS>
__global__ __launch_bounds__(kThreads, 2) void row_log_kernel(WeightArgs a, WeightLayers L) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  const Unit u = unit_of(a, blockIdx.x);
  if (!u.valid || u.N == 0 || keeps_scores<T, D>(u.rows, u.keys)) return;
  const int parts = key_parts(a, u);
  if (u.rows <= kFewRowsOf<T, D>) {
    for (int part = u.w; part < parts; part += a.groups) {
      if (part != u.w) __syncthreads();
      if (u.rows <= 32) few_rows_stream<false, T, D, 1>(a, L, u, part, parts, lds);
      else few_rows_stream<false, T, D, kFewRowsOf<T, D> / 32>(a, L, u, part, parts, lds);
    }
    return;
  }
  const int pieces = (u.rows + 32 * NS * kWaves - 1) / (32 * NS * kWaves) * parts;
  for (int i = u.w; i < pieces; i += a.groups) row_logs<T, D, NS>(a, L, u, i / parts, i % parts, parts, lds);
}

// Sums of 32 NS keys for each wave over a part of the rows.  Parts meet in the workspace: every number is written with the call's tag beside it, and a
// thread that finds all parts of a key there adds them, in order, and clears the tags, so that a graph may be replayed (see confidence_split_kernel).
template <typename T, int D, int NS>
__device__ __forceinline__ void key_sums(const WeightArgs &a, const WeightLayers &L, const Unit &u, int w, int part, int parts, int log_parts, char *lds) {
  typedef Tile<T, D> G;
  const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), t1 = (w * kWaves + wave) * 32 * NS;
  const int cols = min(u.keys, a.C), row_tiles = (u.rows + 31) / 32;
  const int from = 32 * int(int64_t(row_tiles) * part / parts), to = min(u.rows, 32 * int(int64_t(row_tiles) * (part + 1) / parts));
  const Operands o(a, L, u);
  float *logs = reinterpret_cast<float *>(lds + kStages * G::kBytes);
  u32x4 kf[NS][G::kFrags];
#pragma unroll
  for (int n = 0; n < NS; ++n) load_row(kf[n], o.key(a, u, min(t1 + 32 * n + (lane & 31), cols - 1)), lane);
  int at[G::kFrags];
#pragma unroll
  for (int c = 0; c < G::kFrags; ++c) at[c] = G::frag_at(lane, c);
  const float sc = a.scale * kLog2e;
  float mass[NS][16];
#pragma unroll
  for (int n = 0; n < NS; ++n)
#pragma unroll
    for (int r = 0; r < 16; ++r) mass[n][r] = 0.f;

  Ring<T, D> ring(lds);
  int in_tile[G::kLoads];  // within a tile of one head, from its first row
#pragma unroll
  for (int k = 0; k < G::kLoads; ++k) in_tile[k] = ring.row[k] * int(a.qs[1]) + ring.byte[k];
  const bool near = a.qs[1] <= 1 << 25;  // (a tile's bytes fit 32 bits)
  for (int chunk = from; chunk < to; chunk += kLogs) {
    const int here = min(to - chunk, kLogs), tiles = (here + 31) / 32;
    // row and address of the first entry of the next tile to be asked for
    int pos, asked = 0;
    const char *base;
    auto to_entry = [&](int e) {
      const int h = e / u.N;
      pos = e - h * u.N;
      base = o.q + pos * a.qs[1] + h * a.qs[2];
    };
    to_entry(chunk);
    auto ask = [&](int j, int stage) {
      if (j < asked) return ring.ask(stage, [&](int, int, int byte) { return o.q + byte; });  // (behind the last one: any row)
      ++asked;
      if (pos + 32 <= u.N && near) {
        ring.ask(stage, [&](int k, int, int) { return base + in_tile[k]; });
        pos += 32;
        base += 32 * a.qs[1];
        if (pos < u.N) return;
      } else {
        ring.ask(stage, [&](int, int row, int byte) { return o.row(a, u, min(chunk + 32 * j + row, u.rows - 1)) + byte; });
      }
      to_entry(chunk + 32 * (j + 1));
    };
    fill(0, tiles, ask);
    for (int e = threadIdx.x; e < 32 * tiles; e += kThreads) logs[e] = e < here ? row_log_of(a, u, log_parts, chunk + e) : INFINITY;  // (rows that are not there: 0)
    float log[2] = {INFINITY, INFINITY};
    run_pipeline<false, false, T, D, NS>(
        ring, 0, tiles, at, t1 < cols, kf, 0.f, ask, [&](int parity, int j) { log[parity] = logs[32 * j + (lane & 31)]; }, [](f32x16 &, int, int) {},
        [&](const f32x16 &s, int n, int parity, int r0, int r1) {
#pragma unroll
          for (int r = r0; r < r1; ++r) {
            mass[n][r] += __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], sc, -log[parity]));
            stays_here(mass[n][r]);
          }
        });
    __syncthreads();  // (ring and logarithms may be filled anew)
  }
  if (parts == 1) {
#pragma unroll
    for (int n = 0; n < NS; ++n) store_mass(a, u, t1 + 32 * n + product_row(lane, lane & 15), sum_of_lanes(mass[n], lane), lane);
    return;
  }
  constexpr int kKeys = 32 * NS * kWaves;
  uint64_t *mine = a.sums + (int64_t(u.n) * (kGroups / a.units) + w * parts) * 256;
#pragma unroll
  for (int n = 0; n < NS; ++n) {
    const float x = sum_of_lanes(mass[n], lane);
    if (!(lane & 16))
      __hip_atomic_store(mine + part * 256 + (wave * NS + n) * 32 + product_row(lane, lane & 15), uint64_t(__float_as_uint(x)) << 32 | a.tag, __ATOMIC_RELAXED,
                         __HIP_MEMORY_SCOPE_AGENT);
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // they are where every workgroup sees them
  __syncthreads();
  const int i = threadIdx.x;
  if (i >= kKeys) return;
  bool there = true;
  float sum = 0.f;
  for (int p = 0; p < parts; ++p) {
    const uint64_t x = __hip_atomic_load(mine + p * 256 + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    there = there && uint32_t(x) == a.tag;
    sum += __uint_as_float(uint32_t(x >> 32));
  }
  // Two workgroups may find them all: whoever takes the first part's number away adds the sum to the weight, once.
  if (!there || uint32_t(__hip_atomic_exchange(mine + i, uint64_t(0), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT)) != a.tag) return;
  for (int p = 1; p < parts; ++p) __hip_atomic_store(mine + p * 256 + i, uint64_t(0), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  store_mass(a, u, w * kKeys + i, sum, 0);
}

template <typename T, int D, int NS>
__global__ __launch_bounds__(kThreads, 2) void key_sum_kernel(WeightArgs a, WeightLayers L) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  const Unit u = unit_of(a, blockIdx.x);
  if (!u.valid || u.N == 0 || keeps_scores<T, D>(u.rows, u.keys)) return;
  const int log_parts = key_parts(a, u);
  if (u.rows <= kFewRowsOf<T, D>) {
    for (int part = u.w; part < log_parts; part += a.groups) {
      if (u.rows <= 32) few_rows_stream<true, T, D, 1>(a, L, u, part, log_parts, lds);
      else few_rows_stream<true, T, D, kFewRowsOf<T, D> / 32>(a, L, u, part, log_parts, lds);
    }
    return;
  }
  const int tiles = (min(u.keys, a.C) + 32 * NS * kWaves - 1) / (32 * NS * kWaves), parts = row_parts(a, u, tiles);
  for (int i = u.w; i < tiles * parts; i += a.groups) key_sums<T, D, NS>(a, L, u, i / parts, i % parts, parts, log_parts, lds);
}

int layers_at_once(int32_t n) { return n < kMaxAttnLayers ? n : kMaxAttnLayers; }
int max_parts(const lsp_attn_desc *d, int32_t num_layers) {
  const int64_t units = int64_t(layers_at_once(num_layers)) * d->B * d->Hkv, keys = (int64_t(d->C) + d->S) / kPartKeys;
  const int64_t n = units < kGroups ? kGroups / units : 1;
  return int(n < keys ? (n < kMaxParts ? n : kMaxParts) : (keys < 1 ? 1 : keys < kMaxParts ? keys : kMaxParts));
}
size_t row_log_bytes(const lsp_attn_desc *d, int32_t num_layers) {
  return (size_t(max_parts(d, num_layers)) * layers_at_once(num_layers) * d->B * d->Hq * d->S * sizeof(float) + 15) & ~size_t(15);
}
size_t sums_bytes(const lsp_attn_desc *d, int32_t num_layers) {
  return int64_t(layers_at_once(num_layers)) * d->B * d->Hkv <= kGroups / 2 ? size_t(kGroups) * 256 * sizeof(uint64_t) : 0;
}

template <typename T, int D>
int32_t launch(WeightArgs a, const WeightLayers &L, hipStream_t st) {
  constexpr int kMost = Tile<T, D>::kRowBytes == 512 ? 1 : 2;  // (64 registers a block)
  constexpr int kTile = Tile<T, D>::kBytes, kOwn = OwnTiles<T, D>::kDepth * kTile;
  constexpr int kRing = kStages * kTile, kLogBytes = kLogs * int(sizeof(float));
  constexpr int kRowLds = kRing > kWaves * kOwn ? kRing : kWaves * kOwn, kSumLds = kRing + kLogBytes > kWaves * kOwn ? kRing + kLogBytes : kWaves * kOwn;
  static std::atomic<uint64_t> done[5];
  auto start = [&](auto kernel, std::atomic<uint64_t> &mark, int threads, int64_t grid, int bytes) -> int32_t {
    const int32_t rc = ensure_dynamic_lds(reinterpret_cast<const void *>(kernel), bytes, mark, "lsp_attn_key_weights");
    if (rc != LSP_OK) return rc;
    kernel<<<unsigned(grid), threads, bytes, st>>>(a, L);
    LSP_CHECK_LAUNCH("lsp_attn_key_weights: launch");
    return LSP_OK;
  };
  const int64_t rows = int64_t(a.rep) * a.S, cols = a.C;
  if constexpr (Tile<T, D>::kRowBytes <= 256) {
    const int32_t rc = start(few_rows_kernel<T, D>, done[4], kFewWaves * kWave, a.units < 256 ? a.units : 256, kFewWaves * kOwn);
    if (rc != LSP_OK) return rc;
    if (keeps_scores<T, D>(rows, cols + a.S)) return LSP_OK;  // whatever the lengths
  }
  // Two blocks of 32 to a wave, which halves what is read from LDS for a product, where that leaves work for all.
  auto groups = [](int64_t n, int ns) { return (n + 32 * ns * kWaves - 1) / (32 * ns * kWaves); };
  const bool two_rows = kMost == 2 && a.units * groups(rows, 2) * ((cols + 511) / 512) >= 512, two_cols = kMost == 2 && a.units * groups(cols, 2) * ((rows + 511) / 512) >= 512;
  a.log_rows = 32 * kWaves * (two_rows ? 2 : 1);
  int64_t grid = place_grid(a, groups(rows, two_rows ? 2 : 1) * a.max_parts);
  const int32_t rc = two_rows ? start(row_log_kernel<T, D, kMost>, done[0], kThreads, grid, kRowLds) : start(row_log_kernel<T, D, 1>, done[1], kThreads, grid, kRowLds);
  if (rc != LSP_OK) return rc;
  const int64_t tiles = groups(cols, two_cols ? 2 : 1), few = a.max_parts;
  grid = place_grid(a, tiles * (rows / kPartRows + 1) > few ? tiles * (rows / kPartRows + 1) : few);
  return two_cols ? start(key_sum_kernel<T, D, kMost>, done[2], kThreads, grid, kSumLds) : start(key_sum_kernel<T, D, 1>, done[3], kThreads, grid, kSumLds);
}

}  // namespace
}  // namespace lsp

extern "C" size_t lsp_attn_key_weights_workspace_bytes(const lsp_attn_desc *d, int32_t num_layers) {
  if (d == nullptr || num_layers <= 0 || d->B <= 0 || d->S <= 0 || d->Hq <= 0 || d->Hkv <= 0 || d->C <= 0) return 0;
  return lsp::row_log_bytes(d, num_layers) + lsp::sums_bytes(d, num_layers);
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
  LSP_CHECK_ARG(int64_t(d->C) + d->S <= 1 << 30 && int64_t(d->Hq / d->Hkv) * d->S <= 1 << 30, "lsp_attn_key_weights: C + S and S * Hq / Hkv must be <= 2^30");
  for (int l = 0; l < num_layers; ++l) {
    LSP_CHECK_ARG(q_layers[l] && k_suf_layers[l] && k_cache_layers[l], "lsp_attn_key_weights: null operand in layer %d", l);
    LSP_CHECK_ARG(aligned16(q_layers[l]) && aligned16(k_suf_layers[l]) && aligned16(k_cache_layers[l]),
                  "lsp_attn_key_weights: operands of layer %d must be 16-byte aligned", l);
  }
  if (d->D != 64 && d->D != 128) {
    set_error("lsp_attn_key_weights: head_dim %d is not built (64 or 128)", d->D);
    return LSP_ERR_UNSUPPORTED;
  }
  const size_t need = row_log_bytes(d, num_layers) + sums_bytes(d, num_layers);
  if (workspace == nullptr || workspace_bytes < need || !aligned16(workspace)) {
    set_error("lsp_attn_key_weights: workspace of %zu bytes (16-byte aligned) required, got %zu", need, workspace_bytes);
    return LSP_ERR_WORKSPACE;
  }
  WeightArgs a = {};
  a.prefix_len = prefix_len; a.suffix_len = suffix_len;
  a.B = at.B; a.S = at.S; a.Hkv = at.Hkv; a.C = at.C; a.rep = at.Hq / at.Hkv;
  a.scale = at.scale; a.decay = decay;
  const int64_t es = int64_t(elem_size(d->dtype));
  for (int k = 0; k < 3; ++k) a.qs[k] = at.qs[k] * es, a.ks[k] = at.ks[k] * es, a.cs[k] = at.cs[k] * es;
  a.row_log = static_cast<float *>(workspace);
  if (sums_bytes(d, num_layers) > 0) a.sums = reinterpret_cast<uint64_t *>(static_cast<char *>(workspace) + row_log_bytes(d, num_layers));
  a.max_parts = max_parts(d, num_layers);
  hipStream_t st = static_cast<hipStream_t>(stream);
  for (int l0 = 0; l0 < num_layers; l0 += kMaxAttnLayers) {
    const int layers = layers_at_once(num_layers - l0);
    a.units = layers * a.B * a.Hkv;
    a.tag = call_tag();
    WeightLayers L;
    for (int l = 0; l < kMaxAttnLayers; ++l) {
      const int s = l < layers ? l0 + l : l0;  // unused slots repeat a valid layer
      L.q[l] = static_cast<const char *>(q_layers[s]);
      L.k_suf[l] = static_cast<const char *>(k_suf_layers[s]);
      L.k_cache[l] = static_cast<const char *>(k_cache_layers[s]);
    }
    a.weights = weights + int64_t(l0) * at.B * at.Hkv * at.C;
    const int32_t r = d->dtype == LSP_BF16 ? (d->D == 64 ? launch<uint16_t, 64>(a, L, st) : launch<uint16_t, 128>(a, L, st))
                                           : (d->D == 64 ? launch<float, 64>(a, L, st) : launch<float, 128>(a, L, st));
    if (r != LSP_OK) return r;
  }
  return LSP_OK;
}
