// lsp_attn_key_weights: the attention mass that every key received from the active queries of its group.
//
// With c = scale log2(e) and L[h,i] the base-2 logarithm of the sum over all keys of 2^(c q.k):
//   mass[g,t] = sum over heads h of group g and rows i < N of 2^(c q[i,h].k[t,g] - L[h,i])
// Two kernels: row_log_kernel computes L of every row, key_sum_kernel the sums down the columns, each from its own product of queries
// and keys.  (The products kept instead would be 1.3e9 numbers a layer at 8 x 1024 rows of 32 heads on 4096.)
//
// Both are the same loop with the operands exchanged.  A wave holds NS blocks of 32 rows of one operand as matrix fragments in registers (queries for
// the logarithms, keys for the sums) and all four waves of the workgroup read the other one from LDS, 32 rows at a time, from a ring that
// is filled by loads that go straight to LDS.  Scores come out transposed, keys x queries (v_mfma_f32_32x32x16_bf16, or 32x32x2 in fp32),
// so a lane's 16 scores are of ONE query: its reference and sum, or its L, are per-lane numbers, and nothing crosses lanes in the loop:
// the logarithm joins two lanes at the end, the sums of a key stay one register for each of the wave's 32 x NS keys and are reduced over
// 32 lanes once.  The rows of all heads of a group are one list (entry e: row e % N of head e / N), since they meet the same keys.
// Everything is summed in fp32, in an order that sizes alone decide.
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
constexpr int kMaxParts = 16;        // of the keys, where rows are few
constexpr int kPartKeys = 128;       // a part has at least
constexpr int kEnough = 512;         // workgroups: two to a compute unit
constexpr float kFarBelow = -1.7e38f;  // a reference below all scores

struct WeightArgs {
  const int32_t *prefix_len, *suffix_len;
  int32_t B, S, Hq, Hkv, D, C, rep, layers;
  int32_t units, tiles, spread, max_parts;  // (layer, sequence, KV head)s; workgroups of one; each unit in 2^spread pieces
  float scale, decay;
  int64_t qs[3], ks[3], cs[3];  // bytes: batch, row, head
  float *row_log;  // [max_parts, units, rep * S]
  float *weights;  // of the launch's first layer: [layers, B, Hkv, C]
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

__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(d) : "v"(a), "v"(b), "v"(c));
  return d;
}

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
  int l, b, g, w, N, P;
  bool valid;
};
// Workgroups of a unit read the same stream; ids that are equal modulo 8 share an XCD's L2.
__device__ __forceinline__ Unit unit_of(const WeightArgs &a, int n) {
  const int pieces = a.units << a.spread, per_piece = (a.tiles + (1 << a.spread) - 1) >> a.spread;
  const int rest = n >> 3, piece = rest / per_piece * 8 + (n & 7), u = piece >> a.spread;
  Unit r;
  r.w = ((rest % per_piece) << a.spread) + (piece & ((1 << a.spread) - 1));
  r.valid = piece < pieces && r.w < a.tiles;
  r.g = u % a.Hkv;
  r.b = u / a.Hkv % a.B;
  r.l = u / a.Hkv / a.B;
  r.N = r.P = 0;
  if (r.valid) {
    r.N = min(max(a.suffix_len[r.b], 0), a.S);
    r.P = min(max(a.prefix_len[r.b], 0), a.C);
  }
  return r;
}
int64_t place_grid(WeightArgs &a) {
  a.spread = 0;
  if (a.units < 32)
    while ((a.units << a.spread) % 8 != 0) ++a.spread;
  const int64_t pieces8 = ((int64_t(a.units) << a.spread) + 7) / 8, per_piece = (a.tiles + (1 << a.spread) - 1) >> a.spread;
  return pieces8 * 8 * per_piece;
}
// Parts of the keys of a sequence: both kernels go by this.
__device__ __forceinline__ int parts_of(const WeightArgs &a, int rows, int keys, int rows_of_group) {
  if (a.max_parts == 1 || rows > kLogs) return 1;
  const int groups = a.units * ((rows + rows_of_group - 1) / rows_of_group);
  return max(1, min(min(kEnough / groups, a.max_parts), keys / kPartKeys));
}

// Which units few_rows_kernel takes; the other two leave these alone.
constexpr int kFewWaves = 8;
template <int RS>
constexpr int kFewTiles = RS == 1 ? 8 : 4;  // a wave's: 128 registers of scores
template <typename T, int D>
constexpr bool kHasFew = Tile<T, D>::kRowBytes <= 256;
template <int RS>
__host__ __device__ constexpr int few_keys() { return kFewWaves * 32 * kFewTiles<RS>; }
// blocks of 32 rows (0: too many, or too many keys)
template <typename T, int D>
__host__ __device__ constexpr int few_rows(int64_t rows, int64_t keys) {
  return !kHasFew<T, D> ? 0 : rows <= 32 && keys <= few_keys<1>() ? 1 : rows <= 64 && keys <= few_keys<2>() ? 2 : 0;
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

// The wave's NS blocks (`own`) times each of the tiles [first, end) of the stream, one product behind the other: while the matrix cores make one,
// the vector units use the one before.  Tile j + 1 is read from the ring at the start of tile j's last product, so that its barrier is also the one
// behind which tile j's stage is free.
// begin(parity of a tile, tile) comes before a tile's first product.  Of a product, with its block and its tile, the next one's first half goes by
// ready() (READY) and its second half, or all of it, by use(product, block, parity, first, end): numbers [first, end) of 16.
// STREAM_ROWS: the products' rows are the stream's (its columns otherwise).
template <bool STREAM_ROWS, bool READY, typename T, int D, int NS, typename Ask, typename Begin, typename Ready, typename Use>
__device__ __forceinline__ void run_pipeline(Ring<T, D> &ring, int first, int end, const int (&at)[Tile<T, D>::kFrags], bool live,
                                             const u32x4 (&own)[NS][Tile<T, D>::kFrags], float nothing, Ask ask, Begin begin, Ready ready, Use use) {
  typedef Tile<T, D> G;
  constexpr int F = G::kFrags;
  // (tiles beyond the end are asked for again as the last one, so that as many loads are under way everywhere)
#pragma unroll
  for (int k = 0; k < kStages; ++k) ask(min(first + k, end - 1), k);
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

template <typename T, int D, int NS>
__global__ __launch_bounds__(kThreads, 2) void row_log_kernel(WeightArgs a, WeightLayers L) {
  typedef Tile<T, D> G;
  extern __shared__ __attribute__((aligned(16))) char lds[];
  const Unit u = unit_of(a, blockIdx.x);
  if (!u.valid) return;
  const int rows = a.rep * u.N, keys = u.P + u.N, e0 = u.w * kWaves * 32 * NS;
  if (e0 >= rows || few_rows<T, D>(rows, keys)) return;
  const int parts = parts_of(a, rows, keys, kWaves * 32 * NS), part = blockIdx.y;
  if (part >= parts) return;
  const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), e1 = e0 + wave * 32 * NS;
  const char *q = L.q[u.l] + u.b * a.qs[0], *kc = L.k_cache[u.l] + u.b * a.cs[0] + u.g * a.cs[2], *ks = L.k_suf[u.l] + u.b * a.ks[0] + u.g * a.ks[2];

  u32x4 qf[NS][G::kFrags];
#pragma unroll
  for (int n = 0; n < NS; ++n) {
    const int e = min(e1 + 32 * n + (lane & 31), rows - 1), h = e / u.N, i = e - h * u.N;
    load_row(qf[n], q + i * a.qs[1] + (u.g * a.rep + h) * a.qs[2], lane);
  }
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
      const char *base = kc + t * a.cs[1];
      ring.ask(stage, [&](int k, int, int) { return base + from_cache[k]; });
    } else if (t >= u.P && t + 32 <= keys) {
      const char *base = ks + (t - u.P) * a.ks[1];
      ring.ask(stage, [&](int k, int, int) { return base + from_suffix[k]; });
    } else {
      ring.ask(stage, [&](int, int row, int byte) {
        const int r = min(t + row, keys - 1);
        return (r < u.P ? kc + r * a.cs[1] : ks + (r - u.P) * a.ks[1]) + byte;
      });
    }
  };
  const float sc = a.scale * kLog2e;
  float ref[NS], sum[NS], sum2[NS];  // (two chains of additions)
#pragma unroll
  for (int n = 0; n < NS; ++n) ref[n] = kFarBelow, sum[n] = sum2[n] = 0.f;
  const int tiles = (keys + 31) / 32;
  run_pipeline<true, true, T, D, NS>(
      ring, int(int64_t(tiles) * part / parts), int(int64_t(tiles) * (part + 1) / parts), at, e1 < rows, qf, -INFINITY, ask, [](int, int) {},
      [&](f32x16 &s, int n, int j) {
        if (32 * j + 32 > keys) {
#pragma unroll
          for (int r = 0; r < 16; ++r) s[r] = 32 * j + product_row(lane, r) < keys ? s[r] : -INFINITY;
        }
        float top = max3(s[0], s[1], s[2]);
#pragma unroll
        for (int r = 3; r < 15; r += 2) top = max3(top, s[r], s[r + 1]);
        top = fmaxf(top, s[15]) * sc;
        if (__any(top > ref[n] + 8.f)) {  // (seldom: sums of 2^8 at most for each key are far from the end of fp32's range)
          const float to = fmaxf(top, ref[n]);
          const float f = __builtin_amdgcn_exp2f(ref[n] - to);
          sum[n] *= f;
          sum2[n] *= f;
          ref[n] = to;
        }
      },
      [&](const f32x16 &s, int n, int, int r0, int r1) {
#pragma unroll
        for (int r = r0; r < r1; ++r) {
          float &to = r & 1 ? sum[n] : sum2[n];
          to += __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], sc, -ref[n]));
          stays_here(to);
        }
      });
#pragma unroll
  for (int n = 0; n < NS; ++n) {
    const float other = __shfl_xor(ref[n], 32), top = fmaxf(ref[n], other);
    float all = (sum[n] + sum2[n]) * __builtin_amdgcn_exp2f(ref[n] - top);
    all += __shfl_xor(all, 32);
    const int e = e1 + 32 * n + (lane & 31);
    if (lane < 32 && e < rows)
      a.row_log[(int64_t(part) * a.units + (u.l * a.B + u.b) * a.Hkv + u.g) * (int64_t(a.rep) * a.S) + e] = top + __builtin_amdgcn_logf(all);
  }
}

// Lanes with l % 32 < 16 have a key's mass.
__device__ __forceinline__ void store_mass(const WeightArgs &a, float *w, int t, int cols, int P, float mass, int lane) {
  if ((lane & 16) || t >= cols) return;
  w[t] = t < P && a.decay != 0.f ? __builtin_fmaf(a.decay, w[t], mass) : mass;
}

template <typename T, int D, int NS>
__global__ __launch_bounds__(kThreads, 2) void key_sum_kernel(WeightArgs a, WeightLayers L, int log_rows) {
  typedef Tile<T, D> G;
  extern __shared__ __attribute__((aligned(16))) char lds[];
  const Unit u = unit_of(a, blockIdx.x);
  if (!u.valid) return;
  const int rows = a.rep * u.N, keys = u.P + u.N, cols = min(keys, a.C), t0 = u.w * kWaves * 32 * NS;
  if (rows == 0 || t0 >= cols || few_rows<T, D>(rows, keys)) return;
  const int parts = parts_of(a, rows, keys, log_rows);
  const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), t1 = t0 + wave * 32 * NS;
  const char *q = L.q[u.l] + u.b * a.qs[0] + u.g * a.rep * a.qs[2], *kc = L.k_cache[u.l] + u.b * a.cs[0] + u.g * a.cs[2],
             *ks = L.k_suf[u.l] + u.b * a.ks[0] + u.g * a.ks[2];
  float *logs = reinterpret_cast<float *>(lds + kStages * G::kBytes);
  const float *row_log = a.row_log + ((u.l * a.B + u.b) * a.Hkv + u.g) * (int64_t(a.rep) * a.S);
  const int64_t part_stride = int64_t(a.units) * a.rep * a.S;

  u32x4 kf[NS][G::kFrags];
#pragma unroll
  for (int n = 0; n < NS; ++n) {
    const int t = min(t1 + 32 * n + (lane & 31), cols - 1);
    load_row(kf[n], t < u.P ? kc + t * a.cs[1] : ks + (t - u.P) * a.ks[1], lane);
  }
  int at[G::kFrags];
#pragma unroll
  for (int c = 0; c < G::kFrags; ++c) at[c] = G::frag_at(lane, c);
  const float sc = a.scale * kLog2e;
  const bool live = t1 < cols;
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
  for (int chunk = 0; chunk < rows; chunk += kLogs) {
    const int here = min(rows - chunk, kLogs), padded = (here + 31) & ~31;
    if (chunk > 0) __syncthreads();
    for (int e = threadIdx.x; e < padded; e += kThreads) {
      float x = INFINITY;  // rows that are not there: probability 0
      if (e < here) {
        x = row_log[chunk + e];
        if (parts > 1) {
          float top = x, sum = 0.f;
          for (int p = 1; p < parts; ++p) top = fmaxf(top, row_log[p * part_stride + chunk + e]);
          for (int p = 0; p < parts; ++p) sum += __builtin_amdgcn_exp2f(row_log[p * part_stride + chunk + e] - top);
          x = top + __builtin_amdgcn_logf(sum);
        }
      }
      logs[e] = x;
    }
    const int tiles = padded / 32;
    // row and address of the first entry of the next tile to be asked for
    int pos, asked = 0;
    const char *base;
    auto to_entry = [&](int e) {
      const int h = e / u.N;
      pos = e - h * u.N;
      base = q + pos * a.qs[1] + h * a.qs[2];
    };
    to_entry(chunk);
    auto ask = [&](int j, int stage) {
      if (j < asked) return ring.ask(stage, [&](int, int, int byte) { return q + byte; });  // (behind the last one: any row)
      ++asked;
      if (pos + 32 <= u.N && near) {
        ring.ask(stage, [&](int k, int, int) { return base + in_tile[k]; });
        pos += 32;
        base += 32 * a.qs[1];
        if (pos < u.N) return;
      } else {
        ring.ask(stage, [&](int, int row, int byte) {
          const int e = min(chunk + 32 * j + row, rows - 1), h = e / u.N;
          return q + (e - h * u.N) * a.qs[1] + h * a.qs[2] + byte;
        });
      }
      to_entry(chunk + 32 * (j + 1));
    };
    __syncthreads();  // (the logarithms are there)
    float log[2] = {INFINITY, INFINITY};
    run_pipeline<false, false, T, D, NS>(
        ring, 0, tiles, at, live, kf, 0.f, ask, [&](int parity, int j) { log[parity] = logs[32 * j + (lane & 31)]; }, [](f32x16 &, int, int) {},
        [&](const f32x16 &s, int n, int parity, int r0, int r1) {
#pragma unroll
          for (int r = r0; r < r1; ++r) {
            mass[n][r] += __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], sc, -log[parity]));
            stays_here(mass[n][r]);
          }
        });
  }
  // over the 32 lanes that hold the same keys
  float *w = a.weights + ((u.l * a.B + u.b) * int64_t(a.Hkv) + u.g) * a.C;
#pragma unroll
  for (int n = 0; n < NS; ++n) {
    store_mass(a, w, t1 + 32 * n + product_row(lane, lane & 15), cols, u.P, sum_of_lanes(mass[n], lane), lane);
  }
}

// Few rows: all of a unit's scores are kept in registers, so that K is read once and every score and exponential computed once.  The rows
// (32 RS of them at most) are every wave's; the waves share the keys, in tiles of 32 that each fetches for itself, two ahead.  Maxima and sums of
// the rows meet in LDS.
template <typename T, int D>
constexpr int kFewStages = Tile<T, D>::kRowBytes == 128 ? 4 : 2;

template <typename T, int D, int RS>
__device__ __forceinline__ void few_rows_body(const WeightArgs &a, const WeightLayers &L, const Unit &u, char *lds) {
  typedef Tile<T, D> G;
  constexpr int kLoads = G::kBytes / 1024, kStages2 = kFewStages<T, D>, kTiles = kFewTiles<RS>;
  __shared__ float s_row[2][kFewWaves][32 * RS];
  const int rows = a.rep * u.N, keys = u.P + u.N, tiles = (keys + 31) / 32, cols = min(keys, a.C);
  const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const char *q = L.q[u.l] + u.b * a.qs[0], *kc = L.k_cache[u.l] + u.b * a.cs[0] + u.g * a.cs[2], *ks = L.k_suf[u.l] + u.b * a.ks[0] + u.g * a.ks[2];
  char *own = lds + wave * kStages2 * G::kBytes;
  auto ask = [&](int j, int stage) {
#pragma unroll
    for (int k = 0; k < kLoads; ++k) {
      int row, byte;
      G::place(k * kWave + lane, row, byte);
      const int t = min(32 * j + row, keys - 1);
      __builtin_amdgcn_global_load_lds((t < u.P ? kc + t * a.cs[1] : ks + (t - u.P) * a.ks[1]) + byte,
                                       (__attribute__((address_space(3))) void *)(own + stage * G::kBytes + k * 1024), 16, 0, 0);
    }
  };
  u32x4 qf[RS][G::kFrags];
#pragma unroll
  for (int n = 0; n < RS; ++n) {
    const int e = min(32 * n + (lane & 31), rows - 1), h = e / u.N, i = e - h * u.N;
    load_row(qf[n], q + i * a.qs[1] + (u.g * a.rep + h) * a.qs[2], lane);
  }
#pragma unroll
  for (int k = 0; k < kStages2; ++k)
    if (wave + k * kFewWaves < tiles) ask(wave + k * kFewWaves, k);

  f32x16 s[kTiles][RS];
  float top[RS];
#pragma unroll
  for (int n = 0; n < RS; ++n) top[n] = -INFINITY;
#pragma unroll
  for (int k = 0; k < kTiles; ++k) {
    const int j = wave + k * kFewWaves;
    if (j < tiles) {
      const int stage = k % kStages2;
      // the newer tiles that were asked for may be under way
      if (kStages2 == 4 && j + 3 * kFewWaves < tiles) __builtin_amdgcn_s_waitcnt(0x0F70 | 3 * kLoads);
      else if (kStages2 == 2 && j + kFewWaves < tiles) __builtin_amdgcn_s_waitcnt(0x0F70 | kLoads);
      else __builtin_amdgcn_s_waitcnt(0x0F70);
      asm volatile("" ::: "memory");
      u32x4 kf[G::kFrags];
#pragma unroll
      for (int c = 0; c < G::kFrags; ++c) kf[c] = *reinterpret_cast<const u32x4 *>(own + stage * G::kBytes + G::frag_at(lane, c));
      __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0): the stage may be written again
      asm volatile("" ::: "memory");
      if (k + kStages2 < kTiles && j + kStages2 * kFewWaves < tiles) ask(j + kStages2 * kFewWaves, stage);
#pragma unroll
      for (int n = 0; n < RS; ++n) {
#pragma unroll
        for (int r = 0; r < 16; ++r) s[k][n][r] = 0.f;
#pragma unroll
        for (int c = 0; c < G::kFrags; ++c) step(s[k][n], kf[c], qf[n][c], static_cast<const T *>(nullptr));
        if (32 * j + 32 > keys) {
#pragma unroll
          for (int r = 0; r < 16; ++r) s[k][n][r] = 32 * j + product_row(lane, r) < keys ? s[k][n][r] : -INFINITY;
        }
#pragma unroll
        for (int r = 0; r < 16; r += 2) top[n] = max3(top[n], s[k][n][r], s[k][n][r + 1]);
      }
    }
  }
  // of each row over all waves; lanes l and l + 32 have the same row
  auto over_waves = [&](int slot, float (&x)[RS], auto op) {
#pragma unroll
    for (int n = 0; n < RS; ++n) {
      x[n] = op(x[n], __shfl_xor(x[n], 32));
      if (lane < 32) s_row[slot][wave][32 * n + lane] = x[n];
    }
    __syncthreads();
#pragma unroll
    for (int n = 0; n < RS; ++n) {
      x[n] = s_row[slot][0][32 * n + (lane & 31)];
#pragma unroll
      for (int w = 1; w < kFewWaves; ++w) x[n] = op(x[n], s_row[slot][w][32 * n + (lane & 31)]);
    }
  };
  over_waves(0, top, [](float x, float y) { return fmaxf(x, y); });
  const float sc = a.scale * kLog2e;
  float sum[RS];
#pragma unroll
  for (int n = 0; n < RS; ++n) sum[n] = 0.f;
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
  for (int n = 0; n < RS; ++n) sum[n] = 32 * n + (lane & 31) < rows ? 1.f / sum[n] : 0.f;
  float *w = a.weights + ((u.l * a.B + u.b) * int64_t(a.Hkv) + u.g) * a.C;
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
      store_mass(a, w, 32 * j + product_row(lane, lane & 15), cols, u.P, sum_of_lanes(x, lane), lane);
    }
  }
}

template <typename T, int D>
__global__ __launch_bounds__(kFewWaves *kWave) __attribute__((amdgpu_waves_per_eu(2, 2))) void few_rows_kernel(WeightArgs a, WeightLayers L) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  const Unit u = unit_of(a, blockIdx.x);
  if (!u.valid || u.N == 0) return;
  const int blocks = few_rows<T, D>(a.rep * int64_t(u.N), u.P + u.N);
  if (blocks == 1) few_rows_body<T, D, 1>(a, L, u, lds);
  else if (blocks == 2) few_rows_body<T, D, 2>(a, L, u, lds);
}

int layers_at_once(int32_t n) { return n < kMaxAttnLayers ? n : kMaxAttnLayers; }
int max_parts(const lsp_attn_desc *d, int32_t num_layers) {
  const int64_t units = int64_t(layers_at_once(num_layers)) * d->B * d->Hkv, keys = (int64_t(d->C) + d->S) / kPartKeys;
  const int64_t n = units < kEnough ? kEnough / units : 1;
  return int(n < keys ? (n < kMaxParts ? n : kMaxParts) : (keys < 1 ? 1 : keys < kMaxParts ? keys : kMaxParts));
}
size_t row_log_bytes(const lsp_attn_desc *d, int32_t num_layers) {
  return size_t(max_parts(d, num_layers)) * layers_at_once(num_layers) * d->B * d->Hq * d->S * sizeof(float);
}

template <typename T, int D>
int32_t launch(WeightArgs a, const WeightLayers &L, hipStream_t st) {
  constexpr int kMost = D * sizeof(T) == 512 ? 1 : 2;  // (512-byte rows: 64 registers a block)
  constexpr int kRing = kStages * Tile<T, D>::kBytes, kLds = kRing + kLogs * int(sizeof(float));
  static std::atomic<uint64_t> done[5];
  auto start = [&](auto kernel, std::atomic<uint64_t> &mark, int threads, int64_t tiles, int bytes, int parts, auto... more) -> int32_t {
    const int32_t rc = ensure_dynamic_lds(reinterpret_cast<const void *>(kernel), bytes, mark, "lsp_attn_key_weights");
    if (rc != LSP_OK) return rc;
    a.tiles = int(tiles);
    const int64_t grid = place_grid(a);
    if (grid > (int64_t(1) << 23)) {
      set_error("lsp_attn_key_weights: %lld workgroups are too many", (long long)grid);
      return LSP_ERR_UNSUPPORTED;
    }
    kernel<<<dim3(unsigned(grid), parts), threads, bytes, st>>>(a, L, more...);
    LSP_CHECK_LAUNCH("lsp_attn_key_weights: launch");
    return LSP_OK;
  };
  const int64_t rows = int64_t(a.rep) * a.S, cols = a.C;
  if constexpr (kHasFew<T, D>) {
    constexpr int kBytes = kFewWaves * kFewStages<T, D> * Tile<T, D>::kBytes;
    const int32_t rc = start(few_rows_kernel<T, D>, done[4], kFewWaves * kWave, 1, kBytes, 1);
    if (rc != LSP_OK) return rc;
    if (few_rows<T, D>(rows, cols + a.S)) return LSP_OK;  // whatever the lengths
  }
  // two blocks of 32 to a wave where that leaves two workgroups to a compute unit
  auto groups = [](int64_t n, int ns) { return (n + 32 * ns * kWaves - 1) / (32 * ns * kWaves); };
  const int row_blocks = kMost == 2 && a.units * groups(rows, 2) >= kEnough ? 2 : 1, col_blocks = kMost == 2 && a.units * groups(cols, 2) >= kEnough ? 2 : 1;
  const int log_rows = 32 * kWaves * row_blocks;
  const int32_t rc = row_blocks == 2 ? start(row_log_kernel<T, D, kMost>, done[0], kThreads, groups(rows, 2), kRing, a.max_parts)
                                     : start(row_log_kernel<T, D, 1>, done[1], kThreads, groups(rows, 1), kRing, a.max_parts);
  if (rc != LSP_OK) return rc;
  return col_blocks == 2 ? start(key_sum_kernel<T, D, kMost>, done[2], kThreads, groups(cols, 2), kLds, 1, log_rows)
                         : start(key_sum_kernel<T, D, 1>, done[3], kThreads, groups(cols, 1), kLds, 1, log_rows);
}

}  // namespace
}  // namespace lsp

extern "C" size_t lsp_attn_key_weights_workspace_bytes(const lsp_attn_desc *d, int32_t num_layers) {
  if (d == nullptr || num_layers <= 0 || d->B <= 0 || d->S <= 0 || d->Hq <= 0 || d->Hkv <= 0 || d->C <= 0) return 0;
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
  WeightArgs a = {};
  a.prefix_len = prefix_len; a.suffix_len = suffix_len;
  a.B = at.B; a.S = at.S; a.Hq = at.Hq; a.Hkv = at.Hkv; a.D = at.D; a.C = at.C; a.rep = at.Hq / at.Hkv;
  a.scale = at.scale; a.decay = decay;
  const int64_t es = int64_t(elem_size(d->dtype));
  for (int k = 0; k < 3; ++k) a.qs[k] = at.qs[k] * es, a.ks[k] = at.ks[k] * es, a.cs[k] = at.cs[k] * es;
  a.row_log = static_cast<float *>(workspace);
  a.max_parts = max_parts(d, num_layers);
  hipStream_t st = static_cast<hipStream_t>(stream);
  for (int l0 = 0; l0 < num_layers; l0 += kMaxAttnLayers) {
    a.layers = layers_at_once(num_layers - l0);
    a.units = a.layers * a.B * a.Hkv;
    WeightLayers L;
    for (int l = 0; l < kMaxAttnLayers; ++l) {
      const int s = l < a.layers ? l0 + l : l0;  // unused slots repeat a valid layer
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
