// lsp_kv_evict: cuts the cache of a sequence back to `keep` rows, those of most accumulated attention weight, for every layer
// and KV head by itself.
//
// Which rows stay: the first `first`, the last `recent`, and of the others the largest weights (equal ones: the lower row).  The weights'
// bits, mapped to whole numbers of the same order, are in registers (16 a thread, which is 8192 rows); the smallest that stays is
// found by halving the interval between the least and the largest, a count over the workgroup each time, until as many are at or above the
// middle as there are places, or until those between are at most 64, which are ranked by counting.  (A histogram of the weights' leading bits,
// which accumulated weights share, is a queue for few counters in LDS.)
// With ties at the end, the row up to which the equal ones stay is found in the same way.
//
// Which rows are the last: those at the end, as long as rows are only appended.  An eviction puts rows from the end among the others, so that a cache that is evicted from
// again needs its rows' positions.  They are kept beside the weights, for rows from `keep` on as "by place" (kByPlace), since those in front of the end were appended in
// order: a row at t is P - t rows old.  An append has nothing to write then, and an eviction writes the positions below `keep`.  They cost their bytes and one count more
// (4 rows to leave: one layer of four heads, 516 rows, 8.5 us by place, 13.1 by position; 32 layers of 8 x 4100 rows of 32 heads, 134 MB of positions, 149 and 218).
//
// Where they go: keys carry their positions and the attention has no mask, so the order of cached rows means nothing.  Rows
// below `keep` that stay do not move; each row from `keep` on that stays goes into the place of one below that leaves (the n-th of
// one to the n-th of the other).  That moves at most P - keep rows, where closing the gaps in order moves every row behind the first
// one.  Sources are all at or above `keep` and destinations below, so nothing that is read is written.
//
// What bounds it: HBM, for the rows that move (8 layers, 8 x about 4860 rows of 32 heads cut to 4096: 1.6 GB read and written in 310-361 us, about a
// large copy's rate), and where they are few the selection's chain of counts, each a trip to LDS and a barrier (one layer of four heads, 700 rows cut
// to 512: 9.2 us; 32 layers of 32 heads, 1280 rows cut to 1024: 59 us for 0.25 GB).  There it counts that loops end at the last row, and that
// waves add up on the DPP network: together 12.5 -> 9.2 us.  Few units (layer, sequence, KV head) with many rows to move take several workgroups
// each, which all find the same rows and move a part of them.
#include "lsp_attn.h"

namespace lsp {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint64_t u64x2 __attribute__((ext_vector_type(2)));

constexpr int kThreads = 512;
constexpr int kWaves = kThreads / kWave;
constexpr int kKeys = 16;                     // of a thread (with them 60 registers: four workgroups share a compute unit)
constexpr int kBlock = kThreads * kKeys;      // rows whose weights are in registers at a time
constexpr int kFew = kWave;                   // rows that are ranked by counting
constexpr int kWindow = 2048;                 // moves that are listed in LDS at a time
constexpr int kMaxParts = 16;                 // workgroups of a unit
constexpr int64_t kPartBytes = 256 << 10;     // to be moved, a workgroup's at least
constexpr int kEnough = 512;                  // workgroups
constexpr int kMaxLayersPerLaunch = 32;
constexpr int32_t kByPlace = INT32_MIN;
struct CachePtrs {
  char *at[2 * kMaxLayersPerLaunch];  // K then V per layer
};

struct EvictArgs {
  const float *weights;  // [layers, B, Hkv, C], the launch's first layer
  float *new_weights;
  int32_t *kept_index;  // [layers, B, Hkv, keep] or null
  int32_t *positions;   // as the weights, or null: then the last places are the last rows
  const int32_t *token_len, *prefix_len;
  // per unit, where another kernel writes weights and index (`later`): P, moves (-1: nothing leaves), `room` destinations, `room` sources
  int32_t *moves;
  int32_t *new_len;  // where they are written by the first launch (not over the lengths that all of them read), or null
  int32_t B, Hkv, C, keep, high, first, recent, room, parts, later;
  int32_t row_bytes;
  Div by_pieces;  // 16-byte pieces of a K row and a V row
  int64_t cache_row_bytes, cache_batch_bytes;
};

// Whole numbers from 1 on in the order of the weights: -0 as 0, NaN below everything.
__device__ __forceinline__ uint32_t order_of(float w) {
  const uint32_t u = __float_as_uint(w + 0.f);
  if ((u & 0x7fffffffu) > 0x7f800000u) return 1;
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// How many tokens are at or behind a row's: 1 for the last one.  (Unsigned differences: numbers that make no sense give some age.)
__device__ __forceinline__ int age_of(int32_t position, int32_t tokens, int rows, int t) {
  return position == kByPlace ? rows - t : int32_t(uint32_t(tokens) - uint32_t(position));
}
__device__ __forceinline__ int32_t position_of(int32_t position, int32_t tokens, int rows, int t) {
  return position == kByPlace ? int32_t(uint32_t(tokens) - uint32_t(rows - t)) : position;
}

// Over a wave on the DPP network: the maximum, in every lane, and the sum up to and with the lane.
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
#define LSP_DPP(x, ctrl, rows) uint32_t(__builtin_amdgcn_update_dpp(0, int(x), ctrl, rows, 0xf, false))
  v = max(v, LSP_DPP(v, 0x111, 0xf));  // row_shr:1
  v = max(v, LSP_DPP(v, 0x112, 0xf));  // row_shr:2
  v = max(v, LSP_DPP(v, 0x114, 0xf));  // row_shr:4
  v = max(v, LSP_DPP(v, 0x118, 0xf));  // row_shr:8
  v = max(v, LSP_DPP(v, 0x142, 0xa));  // row_bcast:15 into rows 1 and 3
  v = max(v, LSP_DPP(v, 0x143, 0xc));  // row_bcast:31 into rows 2 and 3
  return uint32_t(__builtin_amdgcn_readlane(int(v), kWave - 1));
}
__device__ __forceinline__ int sum_upto(int n) {
  uint32_t v = uint32_t(n);
  v += LSP_DPP(v, 0x111, 0xf);
  v += LSP_DPP(v, 0x112, 0xf);
  v += LSP_DPP(v, 0x114, 0xf);
  v += LSP_DPP(v, 0x118, 0xf);
  v += LSP_DPP(v, 0x142, 0xa);
  v += LSP_DPP(v, 0x143, 0xc);
#undef LSP_DPP
  return int(v);
}

// Numbers of all waves, of which each has one (in every lane).
struct Meeting {
  int *s;  // [2][kWaves]: two, so that one barrier is enough
  int turn = 0;
  __device__ __forceinline__ int *put(int x) {
    int *at = s + turn * kWaves;
    turn ^= 1;
    if ((threadIdx.x & (kWave - 1)) == 0) at[threadIdx.x / kWave] = x;
    __syncthreads();
    return at;
  }
  __device__ __forceinline__ int sum(int x) {
    const int *at = put(x);
    int r = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) r += at[w];
    return r;
  }
  __device__ __forceinline__ uint32_t most(uint32_t x) {
    const int *at = put(int(x));
    uint32_t r = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) r = max(r, uint32_t(at[w]));
    return r;
  }
};

// ONE: a unit's rows are one block, whose weights are read once.  AGED: the last rows go by positions.
template <bool ONE, bool AGED>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(ONE ? 8 : 1))) void evict_kernel(EvictArgs a, CachePtrs p) {
  __shared__ __attribute__((aligned(16))) int s_meet[2 * kWaves];
  __shared__ int s_places[2][kKeys * kWaves], s_total[2], s_src[kWindow];
  __shared__ __attribute__((aligned(16))) int s_dst[kWindow];
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
  const int g = blockIdx.x, b = blockIdx.y, l = blockIdx.z / a.parts, part = blockIdx.z - l * a.parts, unit = (l * a.B + b) * a.Hkv + g;
  const int P = min(max(a.prefix_len[b], 0), a.C);
  const float *w = a.weights + int64_t(unit) * a.C;
  float *nw = a.new_weights + int64_t(unit) * a.C;
  int32_t *kept = a.kept_index == nullptr ? nullptr : a.kept_index + int64_t(unit) * a.keep;
  int32_t *list = a.later ? a.moves + int64_t(unit) * (2 + 2 * int64_t(a.room)) : nullptr;
  if (a.new_len != nullptr && tid == 0 && g == 0 && l == 0 && part == 0) a.new_len[b] = P > a.high ? a.keep : P;
  if (P <= a.high) {  // nothing leaves
    if (part > 0) return;
    if (a.later) {
      if (tid == 0) list[0] = P, list[1] = -1;
      return;
    }
    if (nw != w)
      for (int t = tid; t < P; t += kThreads) nw[t] = w[t];
    if (kept != nullptr)
      for (int t = tid; t < a.keep; t += kThreads) kept[t] = t < P ? t : -1;
    return;
  }
  // rows [first, end) compete for `places` places, but those that are young (AGED); the others' key is 0
  const int blocks = ONE ? 1 : (P + kBlock - 1) / kBlock;
  int32_t *position = AGED ? a.positions + int64_t(unit) * a.C : nullptr;
  const int32_t tokens = AGED ? a.token_len[b] : 0;
  bool by_age = AGED;
  int end = AGED ? P : P - a.recent, places = a.keep - a.first - (AGED ? 0 : a.recent), rivals = end - a.first;
  uint32_t key[kKeys];
  // (a thread's number that the compiler takes for a new one: it would keep sixteen rows' numbers, addresses and flags from loop to loop, in
  // registers that would leave one workgroup to a compute unit)
  auto here_tid = [&]() {
    int x = tid;
    asm volatile("" : "+v"(x));
    return x;
  };
  auto load = [&](int blk) {
    const int own = here_tid();
#pragma unroll
    for (int r = 0; r < kKeys; ++r) {
      if (blk * kBlock + r * kThreads >= P) break;
      const int t = blk * kBlock + r * kThreads + own;
      key[r] = t >= a.first && t < end && (!AGED || !by_age || age_of(position[t], tokens, P, t) > a.recent) ? order_of(w[t]) : 0;
    }
  };
  if (ONE) load(0);
  Meeting meet = {s_meet};
  auto count = [&](auto in) {  // rows for which in(key, row)
    int n = 0;
    for (int blk = 0; blk < blocks; ++blk) {
      if (!ONE) load(blk);
      const int own = here_tid();
#pragma unroll
      for (int r = 0; r < kKeys; ++r) {
        if (blk * kBlock + r * kThreads >= P) break;
        n += __popcll(__ballot(in(key[r], blk * kBlock + r * kThreads + own)));
      }
    }
    return meet.sum(n);
  };
  if (AGED) {
    rivals = count([&](uint32_t k, int) { return k != 0; });
    places -= P - a.first - rivals;
    if (places < 0) {  // more rows than there is room for claim to be the last (positions that make no sense): those at the end are
      by_age = false;
      end = P - a.recent;
      places = a.keep - a.first - a.recent;
      rivals = end - a.first;
      if (ONE) load(0);
    }
  }
  uint32_t least = 0xffffffffu;  // what stays is above, or equal and up to row `upto`
  int upto = -1;
  if (places > 0) {
    uint32_t top = 0, low = 0;  // (low: of the complements)
    for (int blk = 0; blk < blocks; ++blk) {
      if (!ONE) load(blk);
#pragma unroll
      for (int r = 0; r < kKeys; ++r) {
        if (blk * kBlock + r * kThreads >= P) break;
        top = max(top, key[r]);
        low = max(low, key[r] == 0 ? 0u : ~key[r]);
      }
    }
    // at least `places` are at or above lo, fewer at or above hi
    uint32_t lo = ~meet.most(wave_max(low)), hi = meet.most(wave_max(top)) + 1;
    int from_lo = rivals, above = 0;  // how many
    while (hi - lo > 1 && from_lo != places && from_lo - above > kFew) {
      const uint32_t mid = lo + (hi - lo) / 2;
      const int n = count([&](uint32_t k, int) { return k >= mid; });
      if (n >= places) lo = mid, from_lo = n;
      else hi = mid, above = n;
    }
    least = lo;
    upto = P;
    if (from_lo != places && from_lo - above <= kFew) {  // those between are ranked
      uint64_t *few = reinterpret_cast<uint64_t *>(s_dst);
      if (tid < kFew) few[tid] = 0;
      if (tid == 0) s_total[0] = 0;
      __syncthreads();
      for (int blk = 0; blk < blocks; ++blk) {
        if (!ONE) load(blk);
        const int own = here_tid();
#pragma unroll
        for (int r = 0; r < kKeys; ++r) {
          if (blk * kBlock + r * kThreads >= P) break;
          if (key[r] >= lo && key[r] < hi) {
            const int at = atomicAdd(&s_total[0], 1);
            if (at < kFew) few[at] = uint64_t(key[r]) << 32 | uint32_t(~(blk * kBlock + r * kThreads + own));
          }
        }
      }
      __syncthreads();
      if (tid < kFew) {
        const uint64_t mine = few[tid];
        int before = 0;
#pragma unroll 4
        for (int k = 0; k < kFew; k += 2) {
          const u64x2 x = *reinterpret_cast<const u64x2 *>(few + k);
          before += (x.x > mine) + (x.y > mine);
        }
        if (before == places - above - 1) s_total[0] = int(mine >> 32), s_total[1] = ~int(uint32_t(mine));
      }
      __syncthreads();
      least = uint32_t(s_total[0]);
      upto = s_total[1];
      __syncthreads();
    } else if (from_lo != places) {  // equal ones: the largest row with fewer than as many equal ones before it as there are places left
      const int equal = places - above;
      upto = 0;
      int bit = 1;
      while (bit <= P / 2) bit *= 2;
      for (; bit > 0; bit >>= 1)
        if ((upto | bit) <= P && count([&](uint32_t k, int t) { return k == least && t < (upto | bit); }) < equal) upto |= bit;
    }
  }
  auto stays = [&](uint32_t k, int t) { return t < P && (k == 0 || k > least || (k == least && t <= upto)); };

  // The n-th row below `keep` that leaves is the place of the n-th one from there on that stays.
  int moves = kWindow;  // (known after the first round)
  for (int window = 0; window < moves; window += kWindow) {
    int nh = 0, ns = 0;  // in the blocks before
    for (int blk = 0; blk < blocks; ++blk) {
      if (!ONE) load(blk);
      uint32_t hole = 0, moved = 0;  // bit r: row r of the thread
      const int own = here_tid();
#pragma unroll
      for (int r = 0; r < kKeys; ++r) {
        if (blk * kBlock + r * kThreads >= P) break;
        const int t = blk * kBlock + r * kThreads + own;
        const bool s = stays(key[r], t);
        hole |= uint32_t(t < a.keep && !s) << r;
        moved |= uint32_t(t >= a.keep && s) << r;
        const int h = __popcll(__ballot(hole >> r & 1)), m = __popcll(__ballot(moved >> r & 1));
        if (lane == 0) {
          s_places[0][r * kWaves + wave] = h;
          s_places[1][r * kWaves + wave] = m;
        }
      }
      __syncthreads();
      if (wave < 2) {  // the numbers before each: two per lane
        int *at = s_places[wave];
        static_assert(kKeys * kWaves == 2 * kWave, "two per lane");
        const bool there = blk * kBlock + lane / (kWaves / 2) * kThreads < P;  // (those of the same r)
        const int x = there ? at[2 * lane] : 0, y = there ? at[2 * lane + 1] : 0, before = sum_upto(x + y);
        if (lane == kWave - 1) s_total[wave] = before;
        at[2 * lane] = before - x - y;
        at[2 * lane + 1] = before - y;
      }
      __syncthreads();
      const unsigned long long earlier = (1ull << lane) - 1;
      const int own2 = here_tid();
#pragma unroll
      for (int r = 0; r < kKeys; ++r) {
        if (blk * kBlock + r * kThreads >= P) break;
        const int t = blk * kBlock + r * kThreads + own2;
        const bool is_hole = hole >> r & 1, is_moved = moved >> r & 1;
        const unsigned long long holes = __ballot(is_hole), all_moved = __ballot(is_moved);
        if (is_hole) {
          const int n = nh + s_places[0][r * kWaves + wave] + __popcll(holes & earlier) - window;
          if (n >= 0 && n < kWindow) s_dst[n] = t;
        }
        if (is_moved) {
          const int n = ns + s_places[1][r * kWaves + wave] + __popcll(all_moved & earlier) - window;
          if (n >= 0 && n < kWindow) s_src[n] = t;
        }
        if (!a.later && window == 0 && t < a.keep && !is_hole) {
          if (nw != w) nw[t] = w[t];
          if (kept != nullptr) kept[t] = t;
          if (AGED && position[t] == kByPlace) position[t] = position_of(kByPlace, tokens, P, t);
        }
      }
      nh += s_total[0];
      ns += s_total[1];
      __syncthreads();
    }
    moves = nh;  // (= ns: `keep` rows stay)
    const int here = min(moves - window, kWindow);
    if (a.later && part == 0) {
      if (window == 0 && tid == 0) list[0] = P, list[1] = moves;
      for (int n = tid; n < here; n += kThreads) {
        list[2 + window + n] = s_dst[n];
        list[2 + a.room + window + n] = s_src[n];
      }
    }
    if (!a.later)  // (weights in registers: what is written here is not read again)
      for (int n = tid; n < here; n += kThreads) {
        nw[s_dst[n]] = w[s_src[n]];
        if (kept != nullptr) kept[s_dst[n]] = s_src[n];
        if (AGED) position[s_dst[n]] = position_of(position[s_src[n]], tokens, P, s_src[n]);
      }
    // the rows, K and V, 16 bytes a thread, four loads under way
    char *k_base = p.at[2 * l] + int64_t(b) * a.cache_batch_bytes + int64_t(g) * a.row_bytes;
    char *v_base = p.at[2 * l + 1] + int64_t(b) * a.cache_batch_bytes + int64_t(g) * a.row_bytes;
    constexpr int kAhead = 4;
    const int pieces = a.row_bytes / 8, items = here * pieces, step = kThreads * a.parts;
    for (int i0 = part * kThreads + tid; i0 < items; i0 += kAhead * step) {
      u32x4 x[kAhead];
      char *to[kAhead];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const int i = min(i0 + k * step, items - 1), n = quotient(i, a.by_pieces), at = (i - n * pieces) * 16;
        char *base = at < a.row_bytes ? k_base + at : v_base + (at - a.row_bytes);
        to[k] = base + s_dst[n] * a.cache_row_bytes;
        x[k] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(base + s_src[n] * a.cache_row_bytes));
      }
#pragma unroll
      for (int k = 0; k < kAhead; ++k)
        if (i0 + k * step < items) __builtin_nontemporal_store(x[k], reinterpret_cast<u32x4 *>(to[k]));
    }
    __syncthreads();
  }
  if (AGED && !a.later)  // (all that was there has been read)
    for (int t = a.keep + tid; t < P; t += kThreads) position[t] = kByPlace;
}

// Weights, index and positions of a unit whose workgroups, or whose blocks of rows, were several: they are read by all until the end.
constexpr int kLaterThreads = 256;
__global__ __launch_bounds__(kLaterThreads) void evict_weights_kernel(EvictArgs a, int32_t *new_len) {
  const int tid = threadIdx.x, unit = blockIdx.x, b = unit / a.Hkv % a.B;
  const float *w = a.weights + int64_t(unit) * a.C;
  float *nw = a.new_weights + int64_t(unit) * a.C;
  int32_t *kept = a.kept_index == nullptr ? nullptr : a.kept_index + int64_t(unit) * a.keep;
  const int32_t *list = a.moves + int64_t(unit) * (2 + 2 * int64_t(a.room));
  const int P = list[0], moves = list[1], rows = moves < 0 ? P : a.keep;
  if (nw != w)
    for (int t = tid; t < rows; t += kLaterThreads) nw[t] = w[t];
  if (kept != nullptr)
    for (int t = tid; t < a.keep; t += kLaterThreads) kept[t] = t < P ? t : -1;
  __syncthreads();
  for (int n = tid; n < moves; n += kLaterThreads) {
    const int dst = list[2 + n], src = list[2 + a.room + n];
    nw[dst] = w[src];
    if (kept != nullptr) kept[dst] = src;
  }
  if (a.positions != nullptr && moves >= 0) {
    int32_t *position = a.positions + int64_t(unit) * a.C;
    const int32_t tokens = a.token_len[b];
    for (int n = tid; n < moves; n += kLaterThreads) {
      const int dst = list[2 + n], src = list[2 + a.room + n];
      position[dst] = position_of(position[src], tokens, P, src);
    }
    __syncthreads();
    for (int t = tid; t < P; t += kLaterThreads) {
      if (t >= a.keep) position[t] = kByPlace;
      else if (position[t] == kByPlace) position[t] = position_of(kByPlace, tokens, P, t);
    }
  }
  if (new_len != nullptr && unit == b * a.Hkv && tid == 0) new_len[b] = rows;
}

__global__ void evict_length_kernel(int B, int C, int keep, int high, const int32_t *prefix_len, int32_t *new_len) {
  const int b = blockIdx.x * 256 + threadIdx.x;
  if (b >= B) return;
  const int P = min(max(prefix_len[b], 0), C);
  new_len[b] = P > high ? keep : P;
}

// rows that can move at most
int32_t room_of(const lsp_evict_desc *d) { return d->keep < d->C - d->keep ? d->keep : d->C - d->keep; }
int32_t layers_at_once(int32_t n) { return n < kMaxLayersPerLaunch ? n : kMaxLayersPerLaunch; }
// workgroups of a unit
int32_t parts_of(const lsp_evict_desc *d, int32_t layers) {
  const int64_t units = int64_t(layers) * d->B * d->Hkv, bytes = int64_t(room_of(d)) * d->D * int64_t(elem_size(d->kv_dtype)) * 2;
  const int64_t most = kEnough / units < kMaxParts ? kEnough / units : kMaxParts, n = bytes / kPartBytes < most ? bytes / kPartBytes : most;
  return n > 1 ? int32_t(n) : 1;
}
bool weights_later(const lsp_evict_desc *d, int32_t layers) { return d->C > kBlock || parts_of(d, layers) > 1; }

int32_t check(const lsp_evict_desc *d) {
  LSP_CHECK_ARG(d != nullptr, "lsp_kv_evict: null descriptor");
  LSP_CHECK_ARG(d->kv_dtype == LSP_F32 || d->kv_dtype == LSP_BF16, "lsp_kv_evict: unknown kv_dtype %d", d->kv_dtype);
  LSP_CHECK_ARG(d->B > 0 && d->B <= 65535 && d->Hkv > 0 && d->Hkv <= 65535 && d->D > 0 && d->C > 0 && d->num_layers > 0, "lsp_kv_evict: bad dimension");
  LSP_CHECK_ARG(d->D <= 65536 && d->C < 1 << 30, "lsp_kv_evict: D must be <= 65536 and C below 2^30");
  LSP_CHECK_ARG(d->keep > 0 && d->keep <= d->C, "lsp_kv_evict: keep must be 1..C (got %d, C = %d)", d->keep, d->C);
  LSP_CHECK_ARG(d->high >= d->keep, "lsp_kv_evict: high = %d is below keep = %d", d->high, d->keep);
  LSP_CHECK_ARG(d->first >= 0 && d->recent >= 0 && int64_t(d->first) + d->recent <= d->keep,
                "lsp_kv_evict: first + recent must be 0..keep (got %d + %d of %d)", d->first, d->recent, d->keep);
  LSP_CHECK_ARG(int64_t(d->B) * d->Hkv * layers_at_once(d->num_layers) < int64_t(1) << 23, "lsp_kv_evict: too many heads");
  return LSP_OK;
}

}  // namespace
}  // namespace lsp

extern "C" size_t lsp_kv_evict_workspace_bytes(const lsp_evict_desc *d) {
  if (lsp::check(d) != LSP_OK) return 0;
  // a launch for the last layers, of fewer units, may divide them further
  size_t most = 0;
  const int32_t rest = d->num_layers % lsp::kMaxLayersPerLaunch, sizes[2] = {lsp::layers_at_once(d->num_layers), rest};
  for (int32_t n : sizes) {
    const size_t bytes = n > 0 && lsp::weights_later(d, n) ? size_t(n) * d->B * d->Hkv * (2 + 2 * size_t(lsp::room_of(d))) * sizeof(int32_t) : 0;
    if (bytes > most) most = bytes;
  }
  return most;
}

namespace lsp {
namespace {
int32_t evict(const lsp_evict_desc *d, const float *weights, int32_t *positions, const int32_t *token_len, const int32_t *prefix_len,
              void *const *k_cache_layers, void *const *v_cache_layers, float *new_weights, int32_t *new_len, int32_t *kept_index, void *workspace,
              size_t workspace_bytes, void *stream) {
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
  if (need > 0 && (workspace == nullptr || workspace_bytes < need || !aligned16(workspace))) {
    set_error("lsp_kv_evict: workspace of %zu bytes (16-byte aligned) required, got %zu", need, workspace_bytes);
    return LSP_ERR_WORKSPACE;
  }
  hipStream_t st = static_cast<hipStream_t>(stream);
  EvictArgs a = {weights, new_weights, kept_index, positions, token_len, prefix_len, static_cast<int32_t *>(workspace), new_len == prefix_len ? nullptr : new_len, d->B, d->Hkv, d->C, d->keep, d->high, d->first, d->recent, room_of(d)};
  a.row_bytes = int32_t(row_bytes);
  a.by_pieces = div_by(row_bytes / 8);
  a.cache_row_bytes = cache_row_bytes;
  a.cache_batch_bytes = cache_bb;
  bool lengths_left = new_len == prefix_len;
  for (int l0 = 0; l0 < d->num_layers; l0 += kMaxLayersPerLaunch) {
    const int nl = layers_at_once(d->num_layers - l0);
    const int64_t units = int64_t(l0) * d->B * d->Hkv;
    a.weights = weights + units * d->C;
    a.new_weights = new_weights + units * d->C;
    a.kept_index = kept_index == nullptr ? nullptr : kept_index + units * d->keep;
    a.positions = positions == nullptr ? nullptr : positions + units * d->C;
    a.parts = parts_of(d, nl);
    a.later = weights_later(d, nl);
    CachePtrs p;
    for (int l = 0; l < kMaxLayersPerLaunch; ++l) {
      const int s = l < nl ? l0 + l : l0;
      p.at[2 * l] = static_cast<char *>(k_cache_layers[s]);
      p.at[2 * l + 1] = static_cast<char *>(v_cache_layers[s]);
    }
    const dim3 grid(d->Hkv, d->B, nl * a.parts);
    const auto kernel = d->C <= kBlock ? (positions ? evict_kernel<true, true> : evict_kernel<true, false>)
                                       : (positions ? evict_kernel<false, true> : evict_kernel<false, false>);
    kernel<<<grid, kThreads, 0, st>>>(a, p);
    LSP_CHECK_LAUNCH("lsp_kv_evict: launch");
    a.new_len = nullptr;
    if (a.later) {
      const bool last = lengths_left && l0 + nl == d->num_layers;  // (every layer goes by the lengths)
      evict_weights_kernel<<<nl * d->B * d->Hkv, kLaterThreads, 0, st>>>(a, last ? new_len : nullptr);
      LSP_CHECK_LAUNCH("lsp_kv_evict: weights launch");
      if (last) lengths_left = false;
    }
  }
  if (lengths_left) {
    evict_length_kernel<<<(d->B + 255) / 256, 256, 0, st>>>(d->B, d->C, d->keep, d->high, prefix_len, new_len);
    LSP_CHECK_LAUNCH("lsp_kv_evict: length launch");
  }
  return LSP_OK;
}
}  // namespace
}  // namespace lsp

extern "C" int32_t lsp_kv_evict(const lsp_evict_desc *d, const float *weights, const int32_t *prefix_len, void *const *k_cache_layers,
                                void *const *v_cache_layers, float *new_weights, int32_t *new_len, int32_t *kept_index, void *workspace,
                                size_t workspace_bytes, void *stream) {
  return lsp::evict(d, weights, nullptr, nullptr, prefix_len, k_cache_layers, v_cache_layers, new_weights, new_len, kept_index, workspace, workspace_bytes,
                    stream);
}

extern "C" int32_t lsp_kv_evict_positions(const lsp_evict_desc *d, const float *weights, int32_t *positions, const int32_t *token_len,
                                          const int32_t *prefix_len, void *const *k_cache_layers, void *const *v_cache_layers, float *new_weights,
                                          int32_t *new_len, int32_t *kept_index, void *workspace, size_t workspace_bytes, void *stream) {
  using namespace lsp;
  LSP_CHECK_ARG(positions && token_len, "lsp_kv_evict_positions: null pointer");
  const auto tokens = reinterpret_cast<uintptr_t>(token_len), lengths = reinterpret_cast<uintptr_t>(new_len), bytes = uintptr_t(d ? d->B : 0) * sizeof(int32_t);
  LSP_CHECK_ARG(tokens + bytes <= lengths || lengths + bytes <= tokens, "lsp_kv_evict_positions: token_len must not be new_len");
  return evict(d, weights, positions, token_len, prefix_len, k_cache_layers, v_cache_layers, new_weights, new_len, kept_index, workspace, workspace_bytes,
               stream);
}
