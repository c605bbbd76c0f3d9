// lsp_attn_step_q8: attention of the active rows over [cached rows in 8 bits || suffix rows], out = softmax(q K^T scale) V in one pass over the keys.
//
// A unit is (layer, sequence, KV head); the rows of all heads of its group are one list (entry e: row e / rep of head e % rep), since they meet
// the same keys.  Tiles of entries go over blocks of 32 keys, those that share a scale, with a running reference m and sum l of the weights 2^(s - m):
//   S^T = K Q^T   keys x entries: a lane's scores are of ONE entry, and of those keys of which
//   O^T += V^T P^T  has its probabilities as operand: they go from one product to the other in the lane's registers, rounded to bf16 (2^-8 of each).
// m moves only when a maximum exceeds it by more than 8 octaves: weights stay below 2^8, and sums seldom have to be multiplied.  A scale is a power of two,
// so that e4m3 values become bf16 exactly (v_cvt_scalef32_pk_bf16_fp8).  Sums are 32 bits.
// Short tiles (units of up to 64 entries) are bound by the cache's bytes: each wave takes blocks by itself.  Tall ones are bound by matrix and vector instructions: waves share
// blocks in LDS, made bf16 once for all.
#include <math.h>

#include <type_traits>

#include "lsp_q8.h"

namespace lsp {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLag = 8.f;      // octaves that a maximum may exceed the reference by before that moves
// The reference before the first key: a number, so that weights of scores of -infinity are 0 whatever stands before them.
constexpr float kLowest = -3.402823466e38f;
constexpr int kStep = 64;        // keys of a step: of the cache or of the suffix
constexpr int kShort = 64;       // entries of a unit up to which its tiles are short ones
constexpr int kTall = 128;       // entries up to which, beyond that, a tile has as many
constexpr int kTallest = 256;    // entries of a tile of the others (heads of 128)
constexpr int kXcds = 8;
constexpr int kSlots = 2048;     // parts of 32 entries in the workspace, for each of two kernels
// C + S beyond which keys are divided among workgroups at all, with up to so many units and with more: one row of 4 heads on 2000 keys takes 17.2 us in one part and 15.2 in
// several, on 12 000 68 and 18.6; but where units are work for all (256 of them on 1024 keys: 21.2 us) the kernel that would join the parts takes 3 us.
constexpr int kFewUnits = 64, kPartKeysFew = 1024, kPartKeys = 2048;
constexpr int kLeast = 4;        // steps of a part, at least
constexpr int kOnce = 2;         // of a buffer read: nontemporal, the caches need not keep it
// Steps of all short tiles from which on a workgroup's waves have up to four heads beside each other.  A row of the cache holds a head's 128 bytes beside
// the next one's: four waves that read the same rows fetch 512 bytes in a piece (16 x 21 rows on 1515 keys in 8 layers: 302 us; where a workgroup's waves
// divide one head's keys among themselves 362).  With less to do the waves divide the keys, so that more of them work.
constexpr float kBeside = 8192;

struct Q8AttnArgs {
  const int32_t *prefix_len, *suffix_len;
  int32_t B, S, Hkv, C, rep, blocks, per_seq;  // per_seq: units of a sequence, layers * Hkv
  int32_t heads;                               // log2 of the heads that a short tile's workgroup may have beside each other
  int32_t groups;                              // workgroups
  int32_t above, up_to, tall;                  // entries of the units that are this kernel's; of a tall tile
  float c;                                     // scale log2(e)
  Div by_heads, by_rep;
  int64_t qs[3], ks[3], cs[3], os[3];  // bytes: sequence, row, head
  float *parts;
};

__device__ __forceinline__ uint32_t word(bf16x2 x) { return __builtin_bit_cast(uint32_t, x); }
__device__ __forceinline__ bf16x8 fragment(uint32_t a, uint32_t b, uint32_t c, uint32_t d) { return __builtin_bit_cast(bf16x8, u32x4{a, b, c, d}); }
// four e4m3 values -> two words of bf16
__device__ __forceinline__ uint32_t low(uint32_t w, float s) { return word(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, s, false)); }
__device__ __forceinline__ uint32_t high(uint32_t w, float s) { return word(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, s, true)); }
__device__ __forceinline__ uint32_t pick(uint32_t hi, uint32_t lo, uint32_t sel) { return __builtin_amdgcn_perm(hi, lo, sel); }
// bytes j of four words, in order
__device__ __forceinline__ void turn_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d, uint32_t (&t)[4]) {
  const uint32_t ab = pick(b, a, 0x05010400), cd = pick(d, c, 0x05010400), ab2 = pick(b, a, 0x07030602), cd2 = pick(d, c, 0x07030602);
  t[0] = pick(cd, ab, 0x05040100);
  t[1] = pick(cd, ab, 0x07060302);
  t[2] = pick(cd2, ab2, 0x05040100);
  t[3] = pick(cd2, ab2, 0x07060302);
}

// The rows of a block or step, as a buffer: what is read beyond the last one that there is comes as 0.
struct Rows {
  __amdgpu_buffer_rsrc_t at;
  int row;
  __device__ __forceinline__ Rows(const char *base, int64_t stride, int first, int valid, int bytes)
      : at(__builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(base + first * stride), 0,
                                             __builtin_amdgcn_readfirstlane(valid > 0 ? (valid - 1) * int(stride) + bytes : 0), 0x00020000)),
        row(int(stride)) {}
};
// 16 or 8 bytes, `rows` behind byte v
__device__ __forceinline__ u32x4 load16(const Rows &r, int v, int rows) {
  return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r.at, v + rows * r.row, 0, 0));
}
__device__ __forceinline__ u32x2 load8(const Rows &r, int v, int rows) {
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(r.at, v + rows * r.row, 0, 0));
}
// The compiler takes what is made of x for new every time: it is not kept in registers from one step to the next.
__device__ __forceinline__ int anew(int x) {
  asm volatile("" : "+v"(x));
  return x;
}

// over the lanes l % 16: rows of 16 lanes are exchanged, then halves
template <typename F>
__device__ __forceinline__ float quad(float x, F f) {
  auto y = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = f(__uint_as_float(y[0]), __uint_as_float(y[1]));
  y = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return f(__uint_as_float(y[0]), __uint_as_float(y[1]));
}
__device__ __forceinline__ float quad_max(float x) {
  return quad(x, [](float a, float b) { return fmaxf(a, b); });
}
__device__ __forceinline__ float quad_sum(float x) {
  return quad(x, [](float a, float b) { return a + b; });
}

// ---- what there is to do ---------------------------------------------------------------
struct Lens {
  int N, P;
};
struct Shape {  // of a sequence's units
  int entries, rows, tiles, steps, cached;  // rows: entries of a tile; steps: of all keys, `cached` of them of the cache
};
__device__ __forceinline__ Shape shape_of(const Q8AttnArgs &a, Lens n) {
  Shape s;
  s.entries = n.N * a.rep;
  if (s.entries <= a.above || s.entries > a.up_to) s.entries = 0;
  s.rows = s.entries > kShort ? a.tall : s.entries > 16 ? 32 : 16;
  s.tiles = (s.entries + s.rows - 1) / s.rows;
  s.cached = (n.P + kStep - 1) / kStep;
  s.steps = s.cached + (n.N + kStep - 1) / kStep;
  return s;
}
__device__ __forceinline__ Lens lens_of(const Q8AttnArgs &a, int b) {
  if (b >= a.B) return {0, 0};
  return {min(max(a.suffix_len[b], 0), a.S), min(max(a.prefix_len[b], 0), a.C)};
}
__device__ __forceinline__ int first_lane(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ int at_lane(int x, int l) { return __builtin_amdgcn_readlane(x, l); }
// What f makes of lanes 0 to l, in lane l; f(x, none) = x.  By moves between lanes in registers: a plan's sums through LDS were 2 us of a call.
template <int MOVE, int ROWS, typename F>
__device__ __forceinline__ int meet_lane(int x, int none, F f) {
  return f(x, __builtin_amdgcn_update_dpp(none, x, MOVE, ROWS, 0xf, false));
}
template <typename F>
__device__ __forceinline__ int running(int x, int none, F f) {
  x = meet_lane<0x111, 0xf>(x, none, f);  // within 16 lanes from 1, 2, 4, 8 below
  x = meet_lane<0x112, 0xf>(x, none, f);
  x = meet_lane<0x114, 0xf>(x, none, f);
  x = meet_lane<0x118, 0xf>(x, none, f);
  x = meet_lane<0x142, 0xa>(x, none, f);  // lane 15 of the 16 below, then lane 31
  return meet_lane<0x143, 0xc>(x, none, f);
}
__device__ __forceinline__ int running_sum(int x) {
  return running(x, 0, [](int p, int q) { return p + q; });
}
__device__ __forceinline__ int wave_sum(int x) { return at_lane(running_sum(x), kWave - 1); }

// The sequences, 64 at a time, a lane each.
struct Plan {
  int chunk;          // steps of an item, at most
  int heads;          // log2 of the heads of a short item
  bool split;         // whether some tile is more than one item
  int b0;             // the first of the sequences that the lanes have
  Lens n;
  int end, base;      // running sum of the items of an XCD, those of sequences before b0
  int slot_end, slot_base;  // the same of the parts of 32 entries

  __device__ __forceinline__ int heads_of(const Shape &s) const { return s.rows > 32 ? 0 : heads; }
  // Items are dealt out to the XCDs by unit (of a short tile: by its heads); where a sequence's units are no multiple of 8, each unit's items to 2^pieces of them.
  __device__ __forceinline__ static int pieces_of(int units) { return 3 - min(__builtin_ctz(units), 3); }
  __device__ __forceinline__ int splits_of(const Shape &s) const { return split ? (s.steps + chunk - 1) / chunk : 1; }  // of a tile
  __device__ __forceinline__ void take(const Q8AttnArgs &a, int lane, bool first = false) {  // first: the lanes have the lengths already
    if (b0 > 0 || !first) n = lens_of(a, b0 + lane);
    const Shape s = shape_of(a, n);
    const int items = s.tiles * splits_of(s), units = a.per_seq >> heads_of(s), pieces = pieces_of(units);
    end = running_sum((units << pieces) / kXcds * ((items + (1 << pieces) - 1) >> pieces));
    slot_end = split ? running_sum(a.per_seq * items * ((s.rows + 31) / 32)) : 0;
  }
  // How long the items are: all keys of a tile, or, where workgroups would be without one, part of them.  Lane i looks at i + 1 parts (from 32 on at
  // multiples of 8).  A round of items takes its steps and about four steps' time to begin and end, joining the parts as much again.
  // false: there is nothing to do, as for one of two kernels often (which then ends as early as it can).
  __device__ __forceinline__ bool choose(const Q8AttnArgs &a, int lane) {
    chunk = 1 << 30;
    split = false;
    heads = 0;
    n = lens_of(a, lane);
    if (a.parts != nullptr || a.heads > 0) {
      int all = 0, slots = 0, most = 0;
      float work = 0.f;
      for (int b = 0; b < a.B; b += kWave) {
        const Shape x = shape_of(a, b == 0 ? n : lens_of(a, b + lane));
        all += a.per_seq * x.tiles;
        slots += a.per_seq * x.tiles * ((x.rows + 31) / 32);
        most = max(most, x.tiles > 0 ? x.steps : 0);
        work += x.rows > 32 ? 0.f : float(a.per_seq * x.tiles) * float(x.steps);
      }
      all = wave_sum(all);
      if (all == 0) return false;
      slots = wave_sum(slots);
      const bool divides = a.parts != nullptr && slots <= kSlots / 2;
      if (a.heads > 0) {
        const int total = at_lane(running(__float_as_int(work), 0, [](int p, int q) { return __float_as_int(__int_as_float(p) + __int_as_float(q)); }), kWave - 1);
        if (__int_as_float(total) >= kBeside) heads = a.heads;
        // fewer where workgroups would be without work (8 x 32 units on 2000 keys: 30 us, with four heads 52), unless keys are to be divided in any case
        while (heads > 0 && (all >> heads) < a.groups && (!divides || all >= a.groups)) --heads;
      }
      if (divides) {
        const int tiles = (all + (1 << heads) - 1) >> heads;
        most = at_lane(running(most, 0, [](int p, int q) { return max(p, q); }), kWave - 1);
        const int k = lane < 32 ? lane + 1 : 32 + 8 * (lane - 31), part = (most + k - 1) / k;
        const bool fits = k == 1 || (int64_t(slots) * k <= kSlots && part >= kLeast);
        const int64_t rounds = (int64_t(tiles) * k + a.groups - 1) / a.groups, cost = rounds * ((part << heads) + 4) + (k > 1 ? 4 + k / 8 : 0);
        const int least = fits ? int(min(cost, int64_t(1) << 24)) * kWave + lane : 0x7fffffff;
        const int best = at_lane(running(least, 0x7fffffff, [](int p, int q) { return min(p, q); }), kWave - 1) % kWave;
        if (best > 0) {
          const int k2 = best < 32 ? best + 1 : 32 + 8 * (best - 31);
          chunk = (most + k2 - 1) / k2;
          split = true;
        }
      }
    }
    return true;
  }
  __device__ __forceinline__ bool start(const Q8AttnArgs &a, int lane) {
    if (!choose(a, lane)) return false;
    b0 = base = slot_base = 0;
    take(a, lane, true);
    return true;
  }
  // Brings the lanes to the sequence of item q of an XCD's list: its lane, or -1 behind the last item.
  __device__ __forceinline__ int find(const Q8AttnArgs &a, int q, int lane) {
    for (;;) {
      const uint64_t behind = __ballot(q < base + end);
      if (behind != 0) return __builtin_ctzll(behind);
      base += __builtin_amdgcn_readlane(end, kWave - 1);
      slot_base += __builtin_amdgcn_readlane(slot_end, kWave - 1);
      b0 += kWave;
      if (b0 >= a.B) return -1;
      take(a, lane);
    }
  }
};

struct Item {
  int b, l, g, N, P, entries, entry, rows;
  int from, to, cached;  // steps
  int slot, next_slot;   // of its part, or -1: the item is all of a tile; how much further that of a short tile's next head is
  int heads;             // log2 of the heads of a short item
};

// Where a unit's rows are.
struct Unit {
  const char *q, *ks, *vs, *kc, *vc;
  const uint8_t *ke, *ve;
  char *out;
  __device__ __forceinline__ Unit(const Q8AttnArgs &a, const Q8Layers &L, const Item &t) {
    const Q8Layer &of = L.of[t.l];
    const int64_t c = t.b * a.cs[0] + t.g * a.cs[2], s = t.b * a.ks[0] + t.g * a.ks[2], e = (int64_t(t.b) * a.Hkv + t.g) * a.blocks;
    q = of.q + t.b * a.qs[0] + t.g * a.rep * a.qs[2];
    out = of.out + t.b * a.os[0] + t.g * a.rep * a.os[2];
    kc = of.k_cache + c; vc = of.v_cache + c;
    ks = of.k_suf + s; vs = of.v_suf + s;
    ke = of.k_scale + e; ve = of.v_scale + e;
  }
};
// entry e of a unit: its row and head
__device__ __forceinline__ int64_t entry_at(const Q8AttnArgs &a, int e, const int64_t (&s)[3]) {
  const int u = quotient(e, a.by_rep);
  return u * s[1] + (e - u * a.rep) * s[2];
}
// part of 32 entries: their sums, then reference and sum of weights of each
template <int D>
__device__ __forceinline__ float *part_at(const Q8AttnArgs &a, int slot, int row) { return a.parts + (int64_t(slot) + (row >> 5)) * 32 * (D + 2) + (row & 31) * D; }
template <int D>
__device__ __forceinline__ float *part_stats(const Q8AttnArgs &a, int slot, int row) { return a.parts + (int64_t(slot) + (row >> 5)) * 32 * (D + 2) + 32 * D + 2 * (row & 31); }

// ---- short tiles -----------------------------------------------------------------------
// v_mfma_f32_16x16x32_bf16.  The order of a head's elements and of a block's keys within the products is of no matter, so both operands are taken as a lane reads them: 16
// bytes of a key's row; a few elements of eight keys' rows, turned in registers, a byte each, before they become bf16.  Lanes l % 16 = r, l / 16 = h.  Of the keys: rows 16 k + r of the block, elements 64 i + 16 h of 16; of the values: rows 16 k + 4 h + e, of which
// VJ elements from VJ r on.
// A block of the cache comes to LDS by loads that go straight there, each of whole rows, and stays the wave's own: two blocks are on their way at any time, without a
// register (as loads to registers, of which neighbouring lanes belong to different rows, the 16 x 21 rows above took 395 us instead of 362).  Where a unit
// has one tile its keys are read once, and nontemporally (277 us instead of 302).  The 16-byte pieces in LDS are exchanged, those of keys at p ^ (row / 2 % 8)
// (heads of 64: row / 4 % 4), the values' rows with their neighbours where row / 4 is odd (heads of 64: at row ^ (row / 4 % 4)), so that
// what lanes read together lies in different banks.
template <int D>
struct Keys {
  static constexpr int KI = D / 64, KC = D / 32, VJ = D / 16;
  static constexpr int kBytes = kQ8Block * D, kLoads = kBytes / 1024, kRows = 1024 / D;  // of a block's keys or values; loads; rows of one
  u32x4 kw[2][KI];
  uint32_t w[8][VJ / 4];

  // row of the block that element e (of eight) of a lane's values is of
  static __device__ __forceinline__ int value_row(int h, int e) { return 16 * (e >> 2) + 4 * h + (e & 3); }

  // The lane's part of load 0 (the others are kRows rows further on; of keys of 128, every other one has its pieces 4 apart).
  static __device__ __forceinline__ int key_source(int lane, int row) {
    return D == 128 ? lane / 8 * row + 16 * (lane % 8 ^ lane / 16) : lane / 4 * row + 16 * (lane % 4 ^ lane / 16);
  }
  static __device__ __forceinline__ int value_source(int lane, int row) {
    const int p = D == 128 ? lane / 8 : lane / 4;
    return (p ^ (D == 128 ? p >> 2 : p >> 2 & 3)) * row + 16 * (D == 128 ? lane % 8 : lane % 4);
  }
  typedef __attribute__((address_space(3))) void *Lds;
  template <bool ONCE>
  static __device__ __forceinline__ void ask_keys(const Rows &k, int source, char *to) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(k.at, (Lds)(to + 1024 * i), 16, (D == 128 && (i & 1) ? source ^ 64 : source) + i * kRows * k.row, 0, 0,
                                               ONCE ? kOnce : 0);
  }
  template <bool ONCE>
  static __device__ __forceinline__ void ask_values(const Rows &v, int source, char *to) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) __builtin_amdgcn_raw_ptr_buffer_load_lds(v.at, (Lds)(to + 1024 * i), 16, source + i * kRows * v.row, 0, 0, ONCE ? kOnce : 0);
  }
  // What a lane reads first, in bytes of a slot.
  static __device__ __forceinline__ int key_place(int r, int h) { return D == 128 ? r * 128 + 16 * (h ^ r / 2 % 8) : r * 64 + 16 * (h ^ r / 4 % 4); }
  static __device__ __forceinline__ int value_place(int r, int h) { return D == 128 ? 4 * h * 128 + 8 * r : 4 * h * 64 + 4 * r; }
  // Waits for a block's keys (or values), behind which three times as many loads have been asked for, reads them and waits for that, in one.
  __device__ __forceinline__ void read_keys(uint32_t at) {
    if constexpr (D == 128) {
      asm volatile(
          "s_waitcnt vmcnt(12)\n\tds_read_b128 %0, %4 offset:%6\n\tds_read_b128 %1, %5 offset:%6\n\tds_read_b128 %2, %4 offset:%7\n\tds_read_b128 %3, %5 offset:%7\n\t"
          "s_waitcnt lgkmcnt(0)"
          : "=&v"(kw[0][0]), "=&v"(kw[0][1]), "=&v"(kw[1][0]), "=&v"(kw[1][1])
          : "v"(at), "v"(at ^ 64), "i"(0), "i"(2048)
          : "memory");
    } else {
      asm volatile("s_waitcnt vmcnt(6)\n\tds_read_b128 %0, %2 offset:%3\n\tds_read_b128 %1, %2 offset:%4\n\ts_waitcnt lgkmcnt(0)"
                   : "=&v"(kw[0][0]), "=&v"(kw[1][0])
                   : "v"(at), "i"(0), "i"(1024)
                   : "memory");
    }
  }
  __device__ __forceinline__ void read_values(uint32_t at, int h) {
    constexpr int V = kBytes;
    if constexpr (D == 128) {
      const uint32_t a = at + 128 * (h & 1), b = at + 128 - 128 * (h & 1);
      u32x2 x[8];
      asm volatile(
          "s_waitcnt vmcnt(12)\n\tds_read_b64 %0, %8 offset:%10\n\tds_read_b64 %1, %9 offset:%10\n\tds_read_b64 %2, %8 offset:%11\n\tds_read_b64 %3, %9 offset:%11\n\t"
          "ds_read_b64 %4, %8 offset:%12\n\tds_read_b64 %5, %9 offset:%12\n\tds_read_b64 %6, %8 offset:%13\n\tds_read_b64 %7, %9 offset:%13\n\ts_waitcnt lgkmcnt(0)"
          : "=&v"(x[0]), "=&v"(x[1]), "=&v"(x[2]), "=&v"(x[3]), "=&v"(x[4]), "=&v"(x[5]), "=&v"(x[6]), "=&v"(x[7])
          : "v"(a), "v"(b), "i"(V), "i"(V + 256), "i"(V + 2048), "i"(V + 2304)
          : "memory");
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i][0] = x[i][0], w[i][1] = x[i][1];
    } else {
      const uint32_t a0 = at + 64 * h, a1 = at + 64 * (h ^ 1), a2 = at + 64 * (h ^ 2), a3 = at + 64 * (h ^ 3);
      asm volatile(
          "s_waitcnt vmcnt(6)\n\tds_read_b32 %0, %8 offset:%12\n\tds_read_b32 %1, %9 offset:%12\n\tds_read_b32 %2, %10 offset:%12\n\tds_read_b32 %3, %11 offset:%12\n\t"
          "ds_read_b32 %4, %8 offset:%13\n\tds_read_b32 %5, %9 offset:%13\n\tds_read_b32 %6, %10 offset:%13\n\tds_read_b32 %7, %11 offset:%13\n\ts_waitcnt lgkmcnt(0)"
          : "=&v"(w[0][0]), "=&v"(w[1][0]), "=&v"(w[2][0]), "=&v"(w[3][0]), "=&v"(w[4][0]), "=&v"(w[5][0]), "=&v"(w[6][0]), "=&v"(w[7][0])
          : "v"(a0), "v"(a1), "v"(a2), "v"(a3), "i"(V), "i"(V + 1024)
          : "memory");
    }
  }
  __device__ __forceinline__ bf16x8 key(int b, int c, float s) const {
    const u32x4 x = kw[b][c >> 1];
    const int j = 2 * (c & 1);
    return fragment(low(x[j], s), high(x[j], s), low(x[j + 1], s), high(x[j + 1], s));
  }
  __device__ __forceinline__ void turned(int q, bf16x8 (&v)[4], float s) const {  // elements 4 q to 4 q + 3 of the lane's
    uint32_t t[2][4];  // element j of keys 4 m to 4 m + 3
#pragma unroll
    for (int m = 0; m < 2; ++m) turn_bytes(w[4 * m][q], w[4 * m + 1][q], w[4 * m + 2][q], w[4 * m + 3][q], t[m]);
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = fragment(low(t[0][j], s), high(t[0][j], s), low(t[1][j], s), high(t[1][j], s));
  }
};

// NB tiles of 16 entries
template <int D, int NB>
struct Short {
  static constexpr int KC = D / 32, VJ = D / 16;
  bf16x8 q[NB][KC];
  f32x4 o[NB][VJ];     // o[n][j][i]: element 4 VJ h + VJ i + j of entry r
  float m[NB], l[NB];  // reference (base 2, scaled), this lane's part of the sum

  __device__ __forceinline__ void start(const Q8AttnArgs &a, const char *q0, int entry, int entries, int r, int h) {
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      const char *p = q0 + entry_at(a, min(entry + 16 * n + r, entries - 1), a.qs);
#pragma unroll
      for (int c = 0; c < KC; ++c) q[n][c] = *reinterpret_cast<const bf16x8 *>(p + 128 * (c >> 1) + 32 * h + 16 * (c & 1));
#pragma unroll
      for (int j = 0; j < VJ; ++j) o[n][j] = f32x4{0.f, 0.f, 0.f, 0.f};
      m[n] = kLowest;
      l[n] = 0.f;
    }
  }
  // the queries are waited for here, not in a loop, where the wait would count what is under way by then
  __device__ __forceinline__ void arrived() {
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
      for (int c = 0; c < KC; ++c) asm volatile("" : "+v"(q[n][c]));
  }
  // scores of entries n -> probabilities; valid: keys of the block that there are
  __device__ __forceinline__ bf16x8 weigh(int n, f32x4 (&s)[2], float c, int valid, int h) {
    if (valid < kQ8Block)
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i) s[b][i] = 16 * b + 4 * h + i < valid ? s[b][i] : -INFINITY;
    float most = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])), fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
    most = quad_max(most) * c;
    if (__any(most > m[n] + kLag)) {
      const float to = fmaxf(m[n], most), f = to > m[n] ? __builtin_amdgcn_exp2f(m[n] - to) : 1.f;
      m[n] = to;
      l[n] *= f;
#pragma unroll
      for (int j = 0; j < VJ; ++j) o[n][j] *= f;
    }
    bf16x8 P;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float p = __builtin_amdgcn_exp2f(fmaf(s[e >> 2][e & 3], c, -m[n]));
      l[n] += p;
      P[e] = __bf16(p);
    }
    return P;
  }
  // A block that is in a slot: keys(x) and values(x) read it and answer their scale; what follows it there is asked for as soon as it is in registers.
  template <typename K, typename V>
  __device__ __forceinline__ void meet(float c, int valid, int h, K keys, V values) {
    Keys<D> x;
    const float ks = keys(x);
    f32x4 s[NB][2];
#pragma unroll
    for (int n = 0; n < NB; ++n) s[n][0] = s[n][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < KC; ++k)
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const bf16x8 f = x.key(b, k, ks);
#pragma unroll
        for (int n = 0; n < NB; ++n) s[n][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, q[n][k], s[n][b], 0, 0, 0);
      }
    bf16x8 P[NB];
#pragma unroll
    for (int n = 0; n < NB; ++n) P[n] = weigh(n, s[n], c, valid, h);
    const float vs = values(x);
#pragma unroll
    for (int p = 0; p < VJ / 4; ++p) {
      bf16x8 v[4];
      x.turned(p, v, vs);
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int n = 0; n < NB; ++n) o[n][4 * p + j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v[j], P[n], o[n][4 * p + j], 0, 0, 0);
    }
  }
  // 32 rows of the suffix
  __device__ __forceinline__ void meet_suffix(const Rows &kr, const Rows &vr, float c, int valid, int r, int h) {
    const int kv = anew(r * kr.row + 32 * h), vv = anew(4 * h * vr.row + 2 * VJ * r);
    f32x4 s[NB][2];
#pragma unroll
    for (int n = 0; n < NB; ++n) s[n][0] = s[n][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int k = 0; k < KC; ++k) {
        const bf16x8 f = __builtin_bit_cast(bf16x8, load16(kr, kv + 128 * (k >> 1) + 16 * (k & 1), 16 * b));
#pragma unroll
        for (int n = 0; n < NB; ++n) s[n][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, q[n][k], s[n][b], 0, 0, 0);
      }
    uint32_t w[8][VJ / 2];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if constexpr (VJ == 8) {
        const u32x4 x = load16(vr, vv, Keys<D>::value_row(0, e));
#pragma unroll
        for (int j = 0; j < 4; ++j) w[e][j] = x[j];
      } else {
        const u32x2 x = load8(vr, vv, Keys<D>::value_row(0, e));
        w[e][0] = x[0], w[e][1] = x[1];
      }
    }
    bf16x8 P[NB];
#pragma unroll
    for (int n = 0; n < NB; ++n) P[n] = weigh(n, s[n], c, valid, h);
#pragma unroll
    for (int j = 0; j < VJ; ++j) {
      uint32_t t[4];
#pragma unroll
      for (int m = 0; m < 4; ++m) t[m] = pick(w[2 * m + 1][j >> 1], w[2 * m][j >> 1], j & 1 ? 0x07060302 : 0x05040100);
      const bf16x8 v = fragment(t[0], t[1], t[2], t[3]);
#pragma unroll
      for (int n = 0; n < NB; ++n) o[n][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, P[n], o[n][j], 0, 0, 0);
    }
  }
};

// LDS of a workgroup.  Short tiles: two blocks' keys and values of each wave, then what the waves join.  Tall ones: 4 AHEAD blocks' keys [32][D] and 2 AHEAD
// steps' values [64][D], bf16.
template <int D, int WAVES>
union Joined {
  struct {
    f32x4 o[WAVES][D / 16][kWave];
    float m[WAVES][16], l[WAVES][16];
  };
  char slots[WAVES][4 * Keys<D>::kBytes];
};
template <int D, int AHEAD>
struct Staged {
  uint32_t k[4 * AHEAD][kQ8Block * D / 2], v[2 * AHEAD][kStep * D / 2];
};

template <int D, int NB, int WAVES, bool ONCE>
__device__ __forceinline__ void short_item(const Q8AttnArgs &a, const Q8Layers &L, Item t, Joined<D, WAVES> &s, int lane, int wave) {
  constexpr int VJ = D / 16;
  const int sub = wave & ((1 << t.heads) - 1), turn = wave >> t.heads, turns = WAVES >> t.heads;
  t.g += sub;
  t.slot += sub * t.next_slot;
  const Unit u(a, L, t);
  const int r = lane & 15, h = lane >> 4;
  // blocks of 32 keys: of the cache, the waves taking turns
  const int row = int(a.cs[1]), k_source = Keys<D>::key_source(lane, row), v_source = Keys<D>::value_source(lane, row);
  const int c_end = min(2 * min(t.to, t.cached), (t.P + kQ8Block - 1) / kQ8Block);
  char *slots = s.slots[wave];
  const uint32_t at = uint32_t(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char *)slots));
  const uint32_t k_at = at + Keys<D>::key_place(r, h), v_at = at + Keys<D>::value_place(r, h);
  // (beyond the last block the rows are none, and come as zeros: the waits count on as many loads everywhere)
  auto ask_keys = [&](int i, int j) {
    Keys<D>::template ask_keys<ONCE>(Rows(u.kc, a.cs[1], min(j, c_end - 1) * kQ8Block, min(t.P - j * kQ8Block, j < c_end ? kQ8Block : 0), D), anew(k_source),
                      slots + i * 2 * Keys<D>::kBytes);
  };
  auto ask_values = [&](int i, int j) {
    Keys<D>::template ask_values<ONCE>(Rows(u.vc, a.cs[1], min(j, c_end - 1) * kQ8Block, min(t.P - j * kQ8Block, j < c_end ? kQ8Block : 0), D), anew(v_source),
                        slots + i * 2 * Keys<D>::kBytes + Keys<D>::kBytes);
  };
  int j = 2 * t.from + turn;
  Short<D, NB> x;
  x.start(a, u.q, t.entry, t.entries, r, h);
  while (j < c_end) {  // 64 of the wave's blocks at a time: lane i has the exponents of the i-th
    int n = 0;
    const int end = min(c_end, j + kWave * turns), mine = min(j + lane * turns, c_end - 1);
    uint32_t ke = u.ke[mine], ve = u.ve[mine];
    ask_keys(0, j), ask_values(0, j), ask_keys(1, j + turns), ask_values(1, j + turns);
    asm volatile("" : "+v"(ke), "+v"(ve));
    x.arrived();
    for (int slot = 0;; slot ^= 1) {
      const int in_slot = slot * 2 * Keys<D>::kBytes;
      x.meet(a.c, t.P - j * kQ8Block, h,
             [&](Keys<D> &k) {
               k.read_keys(k_at + in_slot);
               ask_keys(slot, j + 2 * turns);
               return q8_scale(__builtin_amdgcn_readlane(ke, n));
             },
             [&](Keys<D> &k) {
               k.read_values(v_at + in_slot, h);
               ask_values(slot, j + 2 * turns);
               return q8_scale(__builtin_amdgcn_readlane(ve, n));
             });
      if (++n, (j += turns) >= end) break;
    }
    __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0): nothing comes to the slots any more
  }
  // of the suffix
  const int s_end = min(2 * (t.to - t.cached), (t.N + kQ8Block - 1) / kQ8Block);
  for (int i = 2 * max(t.from - t.cached, 0) + (turns - 1 - turn); i < s_end; i += turns) {
    const int valid = t.N - i * kQ8Block;
    x.meet_suffix(Rows(u.ks, a.ks[1], i * kQ8Block, min(valid, kQ8Block), 2 * D), Rows(u.vs, a.ks[1], i * kQ8Block, min(valid, kQ8Block), 2 * D), a.c, valid,
                  r, h);
  }

  // The waves' parts: what all have in a place of their lanes is added by one of them, each times what its reference is to the largest.  (A wave that met no key
  // has zeros; all reads at once, and those of other heads' waves are not used.)
  __syncthreads();
#pragma unroll
  for (int n = 0; n < NB; ++n) {
    const float l = quad_sum(x.l[n]);
    if (n > 0) __syncthreads();
    if (h == 0) s.m[wave][r] = x.m[n], s.l[wave][r] = l;
#pragma unroll
    for (int p = 0; p < VJ; ++p) {  // elements 4 p to 4 p + 3 of the lane's 4 VJ
      f32x4 y;
#pragma unroll
      for (int j = 0; j < 4; ++j) y[j] = x.o[n][(4 * p + j) % VJ][(4 * p + j) / VJ];
      s.o[wave][p][lane] = y;
    }
    __syncthreads();
    const int e = 16 * n + r;
    if (t.entry + e < t.entries) {
      float m = kLowest, sum = 0.f, f[WAVES], ls[WAVES];
#pragma unroll
      for (int k = 0; k < WAVES; ++k) {
        const int w = (sub + (k << t.heads)) % WAVES;
        f[k] = k < turns ? s.m[w][r] : kLowest;
        ls[k] = s.l[w][r];
        m = fmaxf(m, f[k]);
      }
#pragma unroll
      for (int k = 0; k < WAVES; ++k) {
        f[k] = __builtin_amdgcn_exp2f(f[k] - m);
        if (k < turns) sum += f[k] * ls[k];
      }
      for (int p = turn; p < VJ; p += turns) {
        f32x4 y = {0.f, 0.f, 0.f, 0.f}, o[WAVES];
#pragma unroll
        for (int k = 0; k < WAVES; ++k) o[k] = s.o[(sub + (k << t.heads)) % WAVES][p][lane];
#pragma unroll
        for (int k = 0; k < WAVES; ++k)
          if (k < turns) y += f[k] * o[k];
        const int d = 4 * VJ * h + 4 * p;
        if (t.slot < 0) {
          const float inv = 1.f / sum;
          *reinterpret_cast<bf16x4 *>(u.out + entry_at(a, t.entry + e, a.os) + 2 * d) =
              bf16x4{__bf16(y[0] * inv), __bf16(y[1] * inv), __bf16(y[2] * inv), __bf16(y[3] * inv)};
        } else {
          *reinterpret_cast<f32x4 *>(part_at<D>(a, t.slot, e) + d) = y;
          if (p == 0 && h == 0) *reinterpret_cast<f32x2 *>(part_stats<D>(a, t.slot, e)) = f32x2{m, sum};
        }
      }
    }
  }
}

// values of eight keys, four from p on and four that are NEXT words on, of one element a lane
typedef short s16x4 __attribute__((ext_vector_type(4)));
template <int NEXT>
__device__ __forceinline__ bf16x8 turned(const uint32_t *__restrict__ p) {
  typedef __attribute__((address_space(3))) s16x4 *At;
  const u32x2 a = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((At)(p)));
  const u32x2 b = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((At)(p + NEXT)));
  return fragment(a[0], a[1], b[0], b[1]);
}

// ---- tall tiles ------------------------------------------------------------------------
// Waves of 32 entries each, which share keys and values in LDS, bf16 by then.  The scores of a wave are keys x entries (32x32x16): lane l has those
// of entry l % 32 with keys 8 j + 4 h + i of 32, h = l / 32, and these are, eight at a time, the operand of the second product, whose other one is
// V^T: of one element those of keys 16 t + 8 x + 4 h + i.  Values lie in LDS as keys do, row by row, and are turned as they are read (ds_read_b64_tr_b16: lane
// s of 16 points at columns 4 (s % 4) of row s / 4 and receives column s of four rows).
// 16-byte pieces are exchanged against bank conflicts: piece p of a key's 256 bytes at p ^ (key % 16) (of 128: p ^ (key / 2 % 8)); of a value's at
// p ^ (4 (key % 4) + key % 2) (of 128: p ^ 4 (key / 2 % 2)): the four rows of a turning read then have all banks between them, and so have a write's two.
template <int D, int WAVES>
struct Tall {
  static constexpr int KC = D / 16, DB = D / 32;
  static constexpr int KP = D / 64;        // pieces of a block's keys that a thread has
  static constexpr int kSets = 8 / WAVES;  // of a step's two blocks

  // in words
  static __device__ __forceinline__ int key_piece(int key, int p) {
    return D == 128 ? key * 64 + 4 * (p ^ (key & 15)) : key * 32 + 4 * (p ^ (key >> 1 & 7));
  }
  static __device__ __forceinline__ int value_piece(int key, int p) {
    return D == 128 ? key * 64 + 4 * (p ^ (4 * (key & 3) + (key & 1))) : key * 32 + 4 * (p ^ 4 * (key >> 1 & 1));
  }
  // where a lane's part of the first transposed read is
  static __device__ __forceinline__ int value_start(int lane) {
    const int s = lane & 15;
    return value_piece(4 * (lane >> 5) + s / 4, 2 * (lane >> 4 & 1) + s % 4 / 2) + 2 * (s & 1);
  }

  // what a thread has on its way, of a block's keys and of one's values, or of two blocks': D / 8 elements of key tid / 8 % 32; and their exponents, a byte each
  uint32_t rk[kSets][4 * KP], rv[kSets][4 * KP], ke, ve;

  static __device__ __forceinline__ void load(uint32_t (&to)[4 * KP], const Rows &k, int tid, bool cached) {
    const int at = anew(tid / 8 % 32 * k.row + tid % 8 * (cached ? D / 8 : D / 4));
    if (!cached) {
#pragma unroll
      for (int p = 0; p < KP; ++p) {
        const u32x4 x = load16(k, at + 16 * p, 0);
#pragma unroll
        for (int j = 0; j < 4; ++j) to[4 * p + j] = x[j];
      }
    } else if constexpr (D == 128) {
      const u32x4 x = load16(k, at, 0);
#pragma unroll
      for (int j = 0; j < 4; ++j) to[j] = x[j];
    } else {
      const u32x2 x = load8(k, at, 0);
      to[0] = x[0], to[1] = x[1];
    }
  }
  // place: of the thread's first piece
  static __device__ __forceinline__ void store(const uint32_t (&from)[4 * KP], uint32_t *to, int place, float s, bool cached) {
    const int k0 = anew(place);
#pragma unroll
    for (int p = 0; p < KP; ++p)
      *reinterpret_cast<u32x4 *>(to + (k0 ^ 4 * p)) = cached ? u32x4{low(from[2 * p], s), high(from[2 * p], s), low(from[2 * p + 1], s), high(from[2 * p + 1], s)}
                                                             : u32x4{from[4 * p], from[4 * p + 1], from[4 * p + 2], from[4 * p + 3]};
  }
  static __device__ __forceinline__ int key_place(int tid) { return key_piece(tid / 8 % 32, KP * (tid % 8)); }
  static __device__ __forceinline__ int value_place(int tid) { return value_piece(tid / 8 % 32, KP * (tid % 8)); }
};

// What stands before it is issued before what stands behind.
__device__ __forceinline__ void here() { __builtin_amdgcn_sched_barrier(0); }

// Blocks of 32 keys: the scores of the next block (eight matrix instructions) stand beside the exponentials of this one, and this one's values (eight) beside
// the next one's maximum; a slice of vector instructions behind every matrix instruction, laid by hand.  Operands are read from LDS four
// instructions ahead.  A step is two blocks; step j writes what step j + AHEAD reads, its values and the keys of the blocks behind its first one, and waves meet every AHEAD
// steps: rings of 4 AHEAD blocks of keys and 2 AHEAD steps of values, half of which are read and half written between two meetings.  AHEAD is 2 where a workgroup has
// the compute unit to itself (8 x 1024 rows on 5120 keys, side by side: 726 us, 734 with 1).
template <int D, int WAVES, int AHEAD>
__device__ __forceinline__ void tall_item(const Q8AttnArgs &a, const Unit &u, const Item &t, Staged<D, AHEAD> &s, int lane, int wave) {
  typedef Tall<D, WAVES> T;
  constexpr int KC = T::KC, DB = T::DB;
  const int tid = wave * kWave + lane, r = lane & 31, h = lane >> 5;
  const int mine = t.entry + 32 * wave;
  const bool live = mine < t.entries;  // (a wave without entries stages with the others)
  bf16x8 q[KC];
  f32x16 o[DB];
  {
    const char *p = u.q + entry_at(a, min(mine + r, t.entries - 1), a.qs);
#pragma unroll
    for (int c = 0; c < KC; ++c) q[c] = *reinterpret_cast<const bf16x8 *>(p + 32 * c + 16 * h);
  }
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
  float m = kLowest, l = 0.f;

  const int last_block = (t.P + kQ8Block - 1) / kQ8Block - 1, end = 2 * t.to, second = wave / 4;  // (of eight waves four have the one of two blocks, four the other)
  auto valid_in = [&](int j) { return j < t.cached ? t.P - j * kStep : t.N - (j - t.cached) * kStep; };  // keys of step j that there are
  auto load_keys = [&](T &to, int i, int b) {  // block b
    const int j = b >> 1, valid = min(valid_in(j) - (b & 1) * kQ8Block, kQ8Block);
    if (b >= end || valid <= 0) return;
    if (j < t.cached) {
      T::load(to.rk[i], Rows(u.kc, a.cs[1], b * kQ8Block, valid, D), tid, true);
      to.ke = i == 0 ? u.ke[b] : to.ke | u.ke[b] << 8;
    } else {
      T::load(to.rk[i], Rows(u.ks, a.ks[1], (b - 2 * t.cached) * kQ8Block, valid, 2 * D), tid, false);
      to.ke = i == 0 ? 127 : to.ke | 127 << 8;
    }
  };
  auto load_values = [&](T &to, int j) {  // (those that are not there come as zeros, and have a scale)
    if (j >= t.to) return;
#pragma unroll
    for (int i = 0; i < T::kSets; ++i) {
      const int b = 2 * j + second + i, valid = min(valid_in(j) - (b & 1) * kQ8Block, kQ8Block);
      if (j < t.cached) {
        T::load(to.rv[i], Rows(u.vc, a.cs[1], b * kQ8Block, valid, D), tid, true);
        const uint32_t e = u.ve[min(b, last_block)];
        to.ve = i == 0 ? e : to.ve | e << 8;
      } else {
        T::load(to.rv[i], Rows(u.vs, a.ks[1], (b - 2 * t.cached) * kQ8Block, valid, 2 * D), tid, false);
        to.ve = 127;
      }
    }
  };
  auto store_keys = [&](const T &from, int i, int b) {
    if (b >= end) return;
    if (b < 2 * t.cached) T::store(from.rk[i], s.k[b & (4 * AHEAD - 1)], T::key_place(tid), q8_scale(i == 0 ? from.ke & 255 : from.ke >> 8), true);
    else T::store(from.rk[i], s.k[b & (4 * AHEAD - 1)], T::key_place(tid), 1.f, false);
  };
  auto store_values = [&](const T &from, int j) {
    if (j >= t.to) return;
#pragma unroll
    for (int i = 0; i < T::kSets; ++i) {
      uint32_t *to = s.v[j & (2 * AHEAD - 1)] + (second + i) * (kQ8Block * D / 2);
      if (j < t.cached) T::store(from.rv[i], to, T::value_place(tid), q8_scale(i == 0 ? from.ve & 255 : from.ve >> 8), true);
      else T::store(from.rv[i], to, T::value_place(tid), 1.f, false);
    }
  };
  auto mask = [&](f32x16 &z, int b) {
    const int valid = valid_in(b >> 1) - (b & 1) * kQ8Block;
    if (valid < kQ8Block)
#pragma unroll
      for (int i = 0; i < 16; ++i) z[i] = 8 * (i >> 2) + 4 * h + (i & 3) < valid ? z[i] : -INFINITY;
  };
  // the largest score of each entry, against the reference
  auto look = [&](float most) {
    const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(most), __float_as_uint(most), false, false);
    most = fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1])) * a.c;
    if (__any(most > m + kLag)) {
      const float to = fmaxf(m, most), f = to > m ? __builtin_amdgcn_exp2f(m - to) : 1.f;
      m = to;
      l *= f;
#pragma unroll
      for (int d = 0; d < DB; ++d) o[d] *= f;
    }
  };
  constexpr int kAhead = 4, kValues = 2 * DB;
  auto clear = [](f32x16 &z) {
#pragma unroll
    for (int i = 0; i < 16; ++i) z[i] = 0.f;
  };
  bf16x8 f[kAhead];  // operands on their way
  // block b: z are its scores, y becomes the next one's (MORE).  PAIR: 1 the next block's first operands are read at its end, 2 these have been
  auto block = [&](int b, f32x16 &z, f32x16 &y, auto more, auto pair) {
    constexpr bool MORE = decltype(more)::value;
    constexpr int PAIR = decltype(pair)::value;
    const uint32_t *k = s.k[(b + 1) & (4 * AHEAD - 1)], *v = s.v[b >> 1 & (2 * AHEAD - 1)] + (b & 1) * (kQ8Block * D / 2);
    const int k0 = anew(T::key_piece(r, h)), v0 = anew(T::value_start(lane));
    auto key = [&](int c) { return *reinterpret_cast<const bf16x8 *>(k + (k0 ^ 8 * c)); };
    auto value = [&](int i) { return turned<8 * D / 2>(v + (v0 ^ 16 * (i % DB)) + i / DB * (16 * D / 2)); };
    u32x4 P[2];
    float part[2] = {0.f, 0.f};
    if (MORE) {
      clear(y);
      if (PAIR != 2)
#pragma unroll
        for (int c = 0; c < kAhead; ++c) f[c] = key(c);
    }
    here();
#pragma unroll
    for (int c = 0; c < KC; ++c) {
      if (MORE) {
        y = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[c % kAhead], q[c], y, 0, 0, 0);
        if (c + kAhead < KC) f[c % kAhead] = key(c + kAhead);
      }
      if (c + kAhead >= KC) f[c % kAhead] = value(c + kAhead - KC);
#pragma unroll
      for (int i = 8 * c / KC; i < 8 * (c + 1) / KC; ++i) {
        bf16x2 two;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float p = __builtin_amdgcn_exp2f(fmaf(z[2 * i + e], a.c, -m));
          part[e] += p;
          two[e] = __bf16(p);
        }
        P[i >> 2][i & 3] = word(two);
        asm volatile("" : "+v"(P[i >> 2][i & 3]), "+v"(part[0]), "+v"(part[1]));  // (not later, behind the next branch)
      }
      here();
    }
    l += part[0] + part[1];
    if (MORE) mask(y, b + 1);
    float most = -INFINITY;
    here();
#pragma unroll
    for (int i = 0; i < kValues; ++i) {
      o[i % DB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[i % kAhead], __builtin_bit_cast(bf16x8, P[i / DB]), o[i % DB], 0, 0, 0);
      if (i + kAhead < kValues) f[i % kAhead] = value(i + kAhead);
      else if (PAIR == 1) f[i % kAhead] = *reinterpret_cast<const bf16x8 *>(s.k[(b + 2) & (4 * AHEAD - 1)] + (k0 ^ 8 * (i + kAhead - kValues)));
      if (MORE)
#pragma unroll
        for (int e = 16 * i / kValues; e < 16 * (i + 1) / kValues; e += 2) most = fmaxf(fmaxf(most, y[e]), y[e + 1]);
      here();
    }
    if (MORE) look(most);
  };

  const int b0 = 2 * t.from;
  // what step j stores.  (A new one each time: what a load leaves out is not the former's.)
  auto load_next = [&](int j) {
    T n;
    const int b = 2 * (j + AHEAD) + 1 + second;
    const int bv = 2 * (j + AHEAD) + second;
    if (j + 1 + AHEAD < min(t.to, t.cached)) {  // all of it of the cache: one run of loads
#pragma unroll
      for (int i = 0; i < T::kSets; ++i) T::load(n.rk[i], Rows(u.kc, a.cs[1], (b + i) * kQ8Block, min(t.P - (b + i) * kQ8Block, kQ8Block), D), tid, true);
#pragma unroll
      for (int i = 0; i < T::kSets; ++i) T::load(n.rv[i], Rows(u.vc, a.cs[1], (bv + i) * kQ8Block, kQ8Block, D), tid, true);
      if constexpr (T::kSets == 2) {
        uint16_t two;
        __builtin_memcpy(&two, u.ke + b, 2);
        n.ke = two;
        __builtin_memcpy(&two, u.ve + bv, 2);
        n.ve = two;
      } else {
        n.ke = u.ke[b], n.ve = u.ve[bv];
      }
    } else if (j + AHEAD >= t.cached && j + 1 + AHEAD < t.to) {
      const int at = (b - 2 * t.cached) * kQ8Block, at_v = (bv - 2 * t.cached) * kQ8Block;
#pragma unroll
      for (int i = 0; i < T::kSets; ++i) T::load(n.rk[i], Rows(u.ks, a.ks[1], at + i * kQ8Block, min(t.N - at - i * kQ8Block, kQ8Block), 2 * D), tid, false);
#pragma unroll
      for (int i = 0; i < T::kSets; ++i) T::load(n.rv[i], Rows(u.vs, a.ks[1], at_v + i * kQ8Block, kQ8Block, 2 * D), tid, false);
      n.ke = u.ke[0], n.ve = u.ve[0];  // (of no use, but a constant in their place would wait for the loads before)
    } else {
#pragma unroll
      for (int i = 0; i < T::kSets; ++i) load_keys(n, i, b + i);
      load_values(n, j + AHEAD);
    }
    return n;
  };
  auto store_next = [&](const T &n, int j) {
#pragma unroll
    for (int i = 0; i < T::kSets; ++i) store_keys(n, i, 2 * (j + AHEAD) + 1 + second + i);
    store_values(n, j + AHEAD);
  };
  {
    T n[AHEAD], last;
#pragma unroll
    for (int p = 0; p < AHEAD; ++p) {
#pragma unroll
      for (int i = 0; i < T::kSets; ++i) load_keys(n[p], i, b0 + 2 * p + second + i);
      load_values(n[p], t.from + p);
    }
    if (second == 0) load_keys(last, 0, b0 + 2 * AHEAD);
#pragma unroll
    for (int p = 0; p < AHEAD; ++p) {
#pragma unroll
      for (int i = 0; i < T::kSets; ++i) store_keys(n[p], i, b0 + 2 * p + second + i);
      store_values(n[p], t.from + p);
    }
    if (second == 0) store_keys(last, 0, b0 + 2 * AHEAD);
  }
  T next = load_next(t.from);
  __syncthreads();
  if (live) {
    f32x16 z, y;
    clear(z);
    {
      const uint32_t *k = s.k[b0 & (4 * AHEAD - 1)];
      const int k0 = T::key_piece(r, h);
#pragma unroll
      for (int c = 0; c < KC; ++c) z = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8 *>(k + (k0 ^ 8 * c)), q[c], z, 0, 0, 0);
      mask(z, b0);
      float most = fmaxf(z[0], z[1]);
#pragma unroll
      for (int i = 2; i < 16; i += 2) most = fmaxf(fmaxf(most, z[i]), z[i + 1]);
      look(most);
    }
    __syncthreads();  // (the first step writes over the first block's keys)
    for (int j = t.from; j + 1 < t.to; ++j) {
      store_next(next, j);
      next = load_next(j + 1);
      block(2 * j, z, y, std::true_type(), std::integral_constant<int, 1>());
      block(2 * j + 1, y, z, std::true_type(), std::integral_constant<int, 2>());
      if (AHEAD == 1 || (j - t.from) % AHEAD == AHEAD - 1) __syncthreads();
    }
    block(end - 2, z, y, std::true_type(), std::integral_constant<int, 0>());
    block(end - 1, y, z, std::false_type(), std::integral_constant<int, 0>());
  } else {  // (as many barriers)
    __syncthreads();
    for (int j = t.from; j + 1 < t.to; ++j) {
      store_next(next, j);
      next = load_next(j + 1);
      if (AHEAD == 1 || (j - t.from) % AHEAD == AHEAD - 1) __syncthreads();
    }
  }
  if (!live || mine + r >= t.entries) return;
  l += __shfl_xor(l, 32);
  // element 32 d + 8 j + 4 h + i
  if (t.slot < 0) {
    const float inv = 1.f / l;
    char *out = u.out + entry_at(a, mine + r, a.os);
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        *reinterpret_cast<bf16x4 *>(out + 2 * (32 * d + 8 * j + 4 * h)) =
            bf16x4{__bf16(o[d][4 * j] * inv), __bf16(o[d][4 * j + 1] * inv), __bf16(o[d][4 * j + 2] * inv), __bf16(o[d][4 * j + 3] * inv)};
  } else {
    float *to = part_at<D>(a, t.slot, 32 * wave + r);
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int j = 0; j < 4; ++j) *reinterpret_cast<f32x4 *>(to + 32 * d + 8 * j + 4 * h) = f32x4{o[d][4 * j], o[d][4 * j + 1], o[d][4 * j + 2], o[d][4 * j + 3]};
    if (h == 0) *reinterpret_cast<f32x2 *>(part_stats<D>(a, t.slot, 32 * wave + r)) = f32x2{m, l};
  }
}

// ---- kernels ---------------------------------------------------------------------------
// Workgroups that stay, and take every groups / 8-th item of their XCD's list.  In it: sequences; of a sequence this XCD's share of its units (so that what
// meets the same keys shares an L2); of a unit its tiles, their parts.  does(item)
template <typename F>
__device__ __forceinline__ void all_items(const Q8AttnArgs &a, const Q8Layers &L, int lane, F does) {
  const int xcd = blockIdx.x % kXcds, stride = a.groups / kXcds;
  Plan plan;
  if (!plan.start(a, lane)) return;
  for (int q = blockIdx.x / kXcds;; q += stride) {
    const int at = plan.find(a, q, lane);
    if (at < 0) break;
    Item t;
    t.b = plan.b0 + at;
    t.N = at_lane(plan.n.N, at);
    t.P = at_lane(plan.n.P, at);
    const Shape shape = shape_of(a, {t.N, t.P});
    t.entries = shape.entries;
    t.rows = shape.rows;
    t.cached = shape.cached;
    const int splits = plan.splits_of(shape), items = shape.tiles * splits;
    const int before = plan.base + (at > 0 ? at_lane(plan.end, max(at - 1, 0)) : 0), in_seq = q - before;
    const int heads = plan.heads_of(shape), pieces = plan.pieces_of(a.per_seq >> heads);
    const int per_piece = (items + (1 << pieces) - 1) >> pieces, piece = per_piece == 1 ? in_seq : in_seq / per_piece, list = piece * kXcds + xcd;
    const int unit = (list >> pieces) << heads, item = ((in_seq - piece * per_piece) << pieces) + (list & ((1 << pieces) - 1));
    if (item >= items) continue;
    t.b = first_lane(t.b);
    t.heads = heads;
    t.l = first_lane(quotient(unit, a.by_heads));
    t.g = first_lane(unit - t.l * a.Hkv);
    const int tile = splits == 1 ? item : item / splits, part = item - tile * splits;
    t.entry = first_lane(tile * t.rows);
    t.from = first_lane(part * plan.chunk);
    t.to = splits == 1 ? shape.steps : min(t.from + plan.chunk, shape.steps);
    t.slot = -1;
    t.next_slot = 0;
    if (splits > 1) {
      const int slots = plan.slot_base + (at > 0 ? at_lane(plan.slot_end, max(at - 1, 0)) : 0);
      t.slot = slots + (unit * items + item) * ((t.rows + 31) / 32);
      t.next_slot = items;  // (of a short tile: that of the next head)
    }
    does(t);
    __syncthreads();
  }
}

// Short tiles, and (TALL) tall ones of four waves.
template <int D, int WAVES, bool TALL>
__global__ __launch_bounds__(WAVES * kWave, 2) void attn_q8_kernel(Q8AttnArgs a, Q8Layers L) {
  union alignas(1024) Shared {
    Joined<D, WAVES> joined;
    Staged<TALL ? D : 64, 1> staged;
    __device__ Shared() {}
  };
  __shared__ Shared s;
  const int lane = threadIdx.x & (kWave - 1), wave = first_lane(threadIdx.x / kWave);
  all_items(a, L, lane, [&](const Item &t) {
    const int own = anew(lane);  // (what an item makes of it is not kept for the next one, in registers that the other kinds of items need)
    if (TALL && t.rows > 32) {
      if constexpr (TALL) tall_item<D, WAVES, 1>(a, Unit(a, L, t), t, s.staged, own, wave);
    } else if (t.rows == 32) {
      if (t.entries <= 32) short_item<D, 2, WAVES, true>(a, L, t, s.joined, own, wave);
      else short_item<D, 2, WAVES, false>(a, L, t, s.joined, own, wave);
    } else {
      short_item<D, 1, WAVES, true>(a, L, t, s.joined, own, wave);
    }
  });
}
// Tall tiles of eight waves.
template <int D>
__global__ __launch_bounds__(512, 2) void attn_q8_tall_kernel(Q8AttnArgs a, Q8Layers L) {
  __shared__ Staged<D, 2> s;
  const int lane = threadIdx.x & (kWave - 1), wave = first_lane(threadIdx.x / kWave);
  all_items(a, L, lane, [&](const Item &t) { tall_item<D, 8, 2>(a, Unit(a, L, t), t, s, anew(lane), wave); });
}

constexpr int kAtOnce = 8;
// The parts of divided tiles, joined: a wave to an entry, which has eight parts on their way at once.
template <int D>
__device__ __forceinline__ void join(const Q8AttnArgs &a, const Q8Layers &L, int lane) {
  Plan plan;
  if (!plan.choose(a, lane) || !plan.split) return;
  // entries of all units of sequences, instead of items of an XCD
  const int waves = gridDim.x * 4;
  int first = blockIdx.x * 4 + first_lane(threadIdx.x / kWave), slots = 0, before = 0;
  for (int b0 = 0; b0 < a.B; b0 += kWave) {
    plan.b0 = b0;
    plan.take(a, lane);
    const Shape mine = shape_of(a, plan.n);
    const int n = a.per_seq * mine.entries, splits_mine = plan.splits_of(mine), end = running_sum(n), all = at_lane(end, kWave - 1);
    for (; first < before + all; first += waves) {
      const int at = __builtin_ctzll(__ballot(first < before + end));
      const int entries = at_lane(mine.entries, at), splits = at_lane(splits_mine, at), rows = at_lane(mine.rows, at), tiles = at_lane(mine.tiles, at);
      if (splits <= 1) continue;
      const int i = first - before - (at_lane(end, at) - at_lane(n, at)), unit = i / entries, e = i - unit * entries, tile = e / rows;
      const int per_part = (rows + 31) / 32, items = tiles * splits;
      const int slot = slots + (at_lane(plan.slot_end, at) - a.per_seq * items * per_part) + (unit * items + tile * splits) * per_part;
      const int row = e - tile * rows;
      float m = kLowest;
      for (int k = lane; k < splits; k += kWave) m = fmaxf(m, part_stats<D>(a, slot + k * per_part, row)[0]);
      m = __int_as_float(at_lane(running(__float_as_int(m), __float_as_int(kLowest), [](int p, int q) { return __float_as_int(fmaxf(__int_as_float(p), __int_as_float(q))); }),
                                 kWave - 1));
      float o[D / kWave] = {}, sum = 0.f;
      for (int k0 = 0; k0 < splits; k0 += kAtOnce) {
        f32x2 st[kAtOnce];
        float p[kAtOnce][D / kWave];
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
          const int part = slot + min(k0 + k, splits - 1) * per_part;
          st[k] = *reinterpret_cast<const f32x2 *>(part_stats<D>(a, part, row));
#pragma unroll
          for (int j = 0; j < D / kWave; ++j) p[k][j] = part_at<D>(a, part, row)[lane * (D / kWave) + j];
        }
        here();
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
          const bool there = k0 + k < splits;
          const float f = __builtin_amdgcn_exp2f(st[k][0] - m);
          sum = there ? sum + st[k][1] * f : sum;
#pragma unroll
          for (int j = 0; j < D / kWave; ++j) o[j] = there ? o[j] + p[k][j] * f : o[j];
        }
      }
      Item t = {};
      t.b = b0 + at;
      t.l = quotient(unit, a.by_heads);
      t.g = unit - t.l * a.Hkv;
      const Unit u(a, L, t);
      const float inv = 1.f / sum;
      __bf16 *out = reinterpret_cast<__bf16 *>(u.out + entry_at(a, e, a.os)) + lane * (D / kWave);
#pragma unroll
      for (int j = 0; j < D / kWave; ++j) out[j] = __bf16(o[j] * inv);
    }
    before += all;
    slots += at_lane(plan.slot_end, kWave - 1);
  }
}

template <int D>
__global__ __launch_bounds__(256) void join_kernel(Q8AttnArgs a, Q8AttnArgs tallest, Q8Layers L) {
  const int lane = threadIdx.x & (kWave - 1);
  join<D>(a, L, lane);
  if (tallest.groups > 0) join<D>(tallest, L, lane);
}

bool divides(int64_t C, int64_t S, int64_t units) { return C + S > (units <= kFewUnits ? kPartKeysFew : kPartKeys); }
// whether some unit may have more entries than tiles of four waves are for
bool has_tallest(int64_t entries, int D) { return D == 128 && entries > kTall; }
size_t parts_bytes(int D) { return size_t(kSlots) * 32 * (D + 2) * sizeof(float); }

// Two workgroups of four waves, or one of eight, stay on each compute unit.  Units of more entries than 128 (heads of 128) have a kernel of their own, of eight waves and 256
// entries, so that every key that is made bf16 and laid out in LDS meets twice as many queries: 8 x 1024 rows on 5120 keys of 32 heads, 687 GFLOP, take 730 to 760 us
// (0.90 to 0.94 PFLOP/s, from card to card; 1.2 is what a large library product reaches; a process's first twenty launches are slower, 850 on average), 843 in tiles of 128
// where these took 736.  Of it the laying out is 110, the exponentials are 60:
// they, the matrix instructions and the power that both draw are what bounds it.
template <int D>
int32_t launch(const Q8AttnArgs &args, const Q8Layers &L, int layers, hipStream_t st) {
  Q8AttnArgs a = args;
  a.per_seq = layers * a.Hkv;
  a.heads = a.Hkv % 4 == 0 ? 2 : a.Hkv % 2 == 0 ? 1 : 0;
  a.by_heads = div_by(a.Hkv);
  a.by_rep = div_by(a.rep);
  const int64_t entries = int64_t(a.rep) * a.S;
  const bool tall = entries > kShort, tallest = has_tallest(entries, D);
  // Few units have eight waves to each: 4 x 32 of them on 32 768 keys take 173 us so and 188 with four, 512 of them on 533 keys 30 and 22.
  const bool wide = !tall && int64_t(a.per_seq) * a.B <= 256;
  a.groups = wide ? 256 : 512;
  a.above = 0;
  a.up_to = tallest ? kTall : 1 << 30;
  a.tall = kTall;
  Q8AttnArgs b = a;
  b.groups = tallest ? 256 : 0;
  b.above = kTall;
  b.up_to = 1 << 30;
  b.tall = kTallest;
  b.heads = 0;
  if (a.parts != nullptr) b.parts = a.parts + parts_bytes(D) / sizeof(float);
  if constexpr (D == 128)
    if (tallest) attn_q8_tall_kernel<D><<<b.groups, 512, 0, st>>>(b, L);
  if (tall) attn_q8_kernel<D, 4, true><<<a.groups, 256, 0, st>>>(a, L);
  else if (wide) attn_q8_kernel<D, 8, false><<<a.groups, 512, 0, st>>>(a, L);
  else attn_q8_kernel<D, 4, false><<<a.groups, 256, 0, st>>>(a, L);
  LSP_CHECK_LAUNCH("lsp_attn_step_q8: launch");
  if (a.parts != nullptr) {
    join_kernel<D><<<512, 256, 0, st>>>(a, b, L);
    LSP_CHECK_LAUNCH("lsp_attn_step_q8: launch");
  }
  return LSP_OK;
}

}  // namespace
}  // namespace lsp

namespace lsp {
namespace {
int32_t check(const char *what, const lsp_attn_desc *d, int32_t num_layers, AttnArgs &c) {
  const int32_t rc = check_q8(what, d, true, c);
  if (rc != LSP_OK) return rc;
  if (d->dtype != LSP_BF16) {
    set_error("%s: bf16 queries only", what);
    return LSP_ERR_UNSUPPORTED;
  }
  LSP_CHECK_ARG(num_layers > 0, "%s: num_layers must be positive", what);
  LSP_CHECK_ARG(c.B == 1 || c.os[0] > 0, "%s: the output must not be shared by sequences", what);
  LSP_CHECK_ARG(c.cs[1] >= c.D && c.ks[1] >= c.D, "%s: rows of keys and values must not overlap", what);
  // items, and parts of 32 entries, are counted in 32 bits
  const int64_t heads = int64_t(c.B) * c.Hkv * kMaxAttnLayers, items = (int64_t(c.S) * (c.Hq / c.Hkv) + kTall - 1) / kTall + 4;
  LSP_CHECK_ARG(heads * kXcds < int64_t(1) << 31 && items < int64_t(1) << 24 && heads * items < int64_t(1) << 28,
                "%s: B * Hkv must be < 2^23, B * S * Hq and S * Hq / Hkv < 2^30", what);
  return LSP_OK;
}
}  // namespace
}  // namespace lsp

extern "C" size_t lsp_attn_q8_workspace_bytes(const lsp_attn_desc *d, int32_t num_layers) {
  using namespace lsp;
  AttnArgs c;
  if (check("lsp_attn_q8_workspace_bytes", d, num_layers, c) != LSP_OK) return 0;
  const int64_t units = int64_t(c.B) * c.Hkv * (num_layers < kMaxAttnLayers ? num_layers : kMaxAttnLayers);
  return divides(c.C, c.S, units) ? parts_bytes(c.D) * (has_tallest(int64_t(c.S) * (c.Hq / c.Hkv), c.D) ? 2 : 1) : 0;
}

extern "C" int32_t lsp_attn_step_q8_layers(const lsp_attn_desc *d, int32_t num_layers, const void *const *q_layers, const void *const *k_suf_layers,
                                           const void *const *v_suf_layers, const void *const *k_cache_layers, const void *const *v_cache_layers,
                                           const void *const *k_scale_layers, const void *const *v_scale_layers, const int32_t *prefix_len,
                                           const int32_t *suffix_len, void *const *out_layers, void *workspace, size_t workspace_bytes,
                                           void *stream) {
  using namespace lsp;
  const char *what = "lsp_attn_step_q8";
  AttnArgs c;
  const int32_t rc = check(what, d, num_layers, c);
  if (rc != LSP_OK) return rc;
  LSP_CHECK_ARG(q_layers && k_suf_layers && v_suf_layers && k_cache_layers && v_cache_layers && k_scale_layers && v_scale_layers && out_layers &&
                    prefix_len && suffix_len,
                "%s: null pointer", what);
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
  const size_t need = lsp_attn_q8_workspace_bytes(d, num_layers);
  a.parts = need > 0 && workspace != nullptr && workspace_bytes >= need && aligned16(workspace) ? static_cast<float *>(workspace) : nullptr;
  for (int k = 0; k < 3; ++k) a.qs[k] = 2 * c.qs[k], a.ks[k] = 2 * c.ks[k], a.cs[k] = c.cs[k], a.os[k] = 2 * c.os[k];
  for (int l0 = 0; l0 < num_layers; l0 += kMaxAttnLayers) {
    const int nl = num_layers - l0 < kMaxAttnLayers ? num_layers - l0 : kMaxAttnLayers;
    Q8Layers L = {};
    for (int l = 0; l < nl; ++l) {
      L.of[l].q = static_cast<const char *>(q_layers[l0 + l]);
      L.of[l].k_suf = static_cast<const char *>(k_suf_layers[l0 + l]); L.of[l].v_suf = static_cast<const char *>(v_suf_layers[l0 + l]);
      L.of[l].k_cache = static_cast<char *>(const_cast<void *>(k_cache_layers[l0 + l])); L.of[l].v_cache = static_cast<char *>(const_cast<void *>(v_cache_layers[l0 + l]));
      L.of[l].k_scale = static_cast<uint8_t *>(const_cast<void *>(k_scale_layers[l0 + l])); L.of[l].v_scale = static_cast<uint8_t *>(const_cast<void *>(v_scale_layers[l0 + l]));
      L.of[l].out = static_cast<char *>(out_layers[l0 + l]);
    }
    const int32_t r = c.D == 64 ? launch<64>(a, L, nl, static_cast<hipStream_t>(stream)) : launch<128>(a, L, nl, static_cast<hipStream_t>(stream));
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
