// Attention over a paged cache: 16-bit or e4m3 blocks, any number of new tokens a sequence.
#pragma once
#include <type_traits>

#include "kv_common.hip.h"

namespace tutti {

constexpr uint32_t kKeyTile = 32;    // keys that a wavefront takes at a time: two halves of 16
constexpr uint32_t kMostWaves = 5;   // wavefronts of a workgroup at most
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
// A row's running maximum is raised only by steps of more than this (log2): until then nothing that has been summed has to be rescaled.
constexpr float kRaise = 8.0f;
// What a row's weights are relative to is its maximum less this (log2).  Weights that become fp16 are 2^15 at most (the largest fp16 value
// is just below 2^16), keep their 11 bits down to 2^-21 of the largest and are off by 2^-32 of it at most below: of what a million keys that
// far down add up to no more than 2^-12 is lost.  (Relative to the maximum itself it would be 2^-25 a key and 2^-5.)
template <typename P>
constexpr float kBelow = __is_same(P, Fp16) ? 7.0f : 0.0f;

struct AttendArgs {
  PoolView pool;
  BatchView batch;
  tutti_rows q, out;
  float *lse;
  uint32_t kv_heads, group, d;  // group: query heads of one KV head
  // A workgroup: `abreast` neighbouring KV heads (a divisor of kv_heads), `key_waves` wavefronts each that take its tiles in turn.
  uint32_t abreast, key_waves;
  float scale_log2;             // sm_scale * log2(e)
  uint32_t causal, window;
  // How the keys are split (make_plan): workgroups that the device holds at once, the fewest tiles of a part, and what there can be.
  uint32_t slots, min_tiles, max_units, max_parts;
  uint32_t *tiles_a_part;       // what the attention kernel has chosen, for the join
  float *part_o;                // [part][rows][dp]: sums of weighted values
  f32x2 *part_ml;               // [part][rows]: running maximum (log2) and sum of weights
  uint32_t *status;
};

// Rows of a sequence: new tokens times query heads of a KV head, in tiles of ROWS.
template <int ROWS>
__device__ __forceinline__ uint32_t row_tiles(const AttendArgs &a, const tutti_seq &s) {
  return (s.n_new * a.group + ROWS - 1) / ROWS;
}

// Key tiles that a sequence's queries see, counted from the tile of the first one.
__device__ __forceinline__ uint32_t first_key(const AttendArgs &a, const tutti_seq &s) {
  const uint32_t begin = s.n_held - s.n_new;
  return a.window && begin + 1 > a.window ? begin + 1 - a.window : 0;
}
__device__ __forceinline__ uint32_t key_tiles(const AttendArgs &a, const tutti_seq &s) {
  return (s.n_held + kKeyTile - 1) / kKeyTile - first_key(a, s) / kKeyTile;
}

// How many tiles a part of the keys has.  Every workgroup works this out from the records, which costs less than a launch before it.
struct Plan {
  uint32_t tiles_a_part;
  tutti_seq lane_seq;  // record `lane` of the first 64: read once
};

__device__ __forceinline__ uint32_t parts_of(const AttendArgs &a, const Plan &p, const tutti_seq &s) {
  const uint32_t n = (key_tiles(a, s) + p.tiles_a_part - 1) / p.tiles_a_part;
  return n ? n : 1;
}

__device__ __forceinline__ tutti_seq record(const AttendArgs &a, const Plan &p, uint32_t base, uint32_t lane) {
  return base ? load_seq(a.batch.seqs + base + lane) : p.lane_seq;
}

// A part has the tiles that make the parts fill the device's slots once or, where that goes up better, twice: with one part more than
// slots the last one has them for itself (32 sequences, 516 parts for 512 slots: 56 us, 488 parts: 42).  What is weighed is rounds times
// (tiles of a part + kUnitTiles, what a workgroup costs beside its tiles).  More than 64 sequences, or more row tiles than two
// rounds have slots for: an even share of all tiles, which leaves most sequences whole (750 MB of bf16 cache in 64 sequences 134 us, in 65
// 164, in 256 166; of e4m3 147 in 64, 210 in 512, 357 in 2,048, whose records every workgroup reads).
constexpr uint32_t kUnitTiles = 8;

template <int ROWS>
__device__ __forceinline__ Plan make_plan(const AttendArgs &a) {
  const uint32_t lane = threadIdx.x & (kLanes - 1), head_groups = a.kv_heads / a.abreast;
  Plan p{};
  if (lane < a.batch.n_seq) p.lane_seq = load_seq(a.batch.seqs + lane);
  uint64_t work = 0;
  uint32_t rows = 0, tiles = 0;  // of the lane's last sequence
  for (uint32_t base = 0; base < a.batch.n_seq; base += kLanes) {
    if (base + lane < a.batch.n_seq) {
      const tutti_seq s = record(a, p, base, lane);
      if (seq_ok(a.batch, s) && s.n_new) {
        rows = row_tiles<ROWS>(a, s) * head_groups;
        tiles = key_tiles(a, s);
        work += static_cast<uint64_t>(rows) * tiles;
      }
    }
  }
#pragma unroll
  for (int m = 1; m < static_cast<int>(kLanes); m <<= 1) work += __shfl_xor(work, m, kLanes);
  const auto share = [&](uint32_t slots) {
    const uint64_t each = (work + slots - 1) / slots;
    const uint32_t most = 0x40000000u, n = each > most ? most : static_cast<uint32_t>(each);
    return uniform(n < a.min_tiles ? a.min_tiles : n);
  };
  p.tiles_a_part = share(a.slots);
  const uint32_t row_tiles_all = a.batch.n_seq > kLanes ? ~0u : from_lane(lane_prefix_sum(rows), kLanes - 1);
  uint32_t best = ~0u;
  for (uint32_t rounds = 1; rounds <= 2; ++rounds) {
    const uint32_t limit = rounds * a.slots;
    if (row_tiles_all == 0 || row_tiles_all > limit) continue;
    uint32_t n;
    bool fits = true;
    if (a.batch.n_seq == 1) {
      const uint32_t parts = limit / row_tiles_all;
      n = uniform((from_lane(tiles, 0) + parts - 1) / parts);
      if (n < a.min_tiles) n = a.min_tiles;
    } else {
      n = share(limit);
      fits = false;
      for (int x = 0; x < 6 && !fits; ++x) {
        const uint32_t units = from_lane(lane_prefix_sum(rows * ((tiles + n - 1) / n)), kLanes - 1);
        fits = units <= limit;
        if (fits) break;
        const uint32_t more = static_cast<uint32_t>(static_cast<float>(n) * static_cast<float>(units - limit) / static_cast<float>(limit));
        n = uniform(n + (more ? more : 1));
      }
    }
    if (fits && rounds * (n + kUnitTiles) < best) {
      best = rounds * (n + kUnitTiles);
      p.tiles_a_part = n;
    }
  }
  return p;
}

// Where a unit's results go.
struct Unit {
  uint32_t seq;         // n_seq: none
  tutti_seq s;
  uint32_t row_tile, head, part, parts;  // head: the first of its heads
  uint32_t part_slot;   // of its first head's first part in the work memory, where parts > 1; the next head's are behind those
};

template <int ROWS>
__device__ __forceinline__ Unit locate(const AttendArgs &a, const Plan &p, uint32_t unit, bool first) {
  const uint32_t lane = threadIdx.x & (kLanes - 1);
  Unit u{};
  u.seq = a.batch.n_seq;
  uint32_t before = 0, slots = 0;
  bool bad = false;
  for (uint32_t base = 0; base < a.batch.n_seq; base += kLanes) {
    tutti_seq s{};
    uint32_t n = 0, split = 0, tiles = 0, parts = 0;
    if (base + lane < a.batch.n_seq) {
      s = record(a, p, base, lane);
      const bool ok = seq_ok(a.batch, s);
      bad |= !ok;
      if (ok && s.n_new) {
        tiles = row_tiles<ROWS>(a, s);
        parts = parts_of(a, p, s);
        n = tiles * (a.kv_heads / a.abreast) * parts;
        split = parts > 1 ? tiles * a.kv_heads * parts : 0;
      }
    }
    const uint32_t upto = before + lane_prefix_sum(n), split_upto = slots + lane_prefix_sum(split);
    const uint64_t behind = __ballot(n != 0 && upto > unit);
    if (behind && u.seq == a.batch.n_seq) {
      const uint32_t l = static_cast<uint32_t>(__builtin_ctzll(behind));
      const uint32_t local = unit - (from_lane(upto, l) - from_lane(n, l));
      u.seq = base + l;
      u.s = tutti_seq{from_lane(s.row0, l), from_lane(s.n_new, l), from_lane(s.n_held, l), from_lane(s.table_off, l)};
      u.parts = from_lane(parts, l);
      // heads first, then parts, then row tiles, the last ones, which see most keys, in front: neighbours read the same blocks
      const uint32_t head_groups = a.kv_heads / a.abreast;
      u.head = local % head_groups * a.abreast;
      u.part = local / head_groups % u.parts;
      u.row_tile = from_lane(tiles, l) - 1 - local / head_groups / u.parts;
      u.part_slot = from_lane(split_upto, l) - from_lane(split, l) + (u.row_tile * a.kv_heads + u.head) * u.parts;
      if (!first) return u;
    }
    before = from_lane(upto, kLanes - 1);
    slots = from_lane(split_upto, kLanes - 1);
  }
  if (first) {
    if (__ballot(bad) && lane == 0) report(a.status, TUTTI_ST_BAD_EXTENT);
    if (before > a.max_units && lane == 0) report(a.status, TUTTI_ST_BAD_EXTENT);
  }
  return u;
}

template <typename T>
__device__ __forceinline__ f32x4 product(typename T::eight a, typename T::eight b, f32x4 c) {
  if constexpr (sizeof(typename T::one) == 2 && __is_same(T, Fp16))
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// A result, rounded.  A mean of fp16 values is no larger than they are, but weights that were rounded put one beside 65504 where it would
// become an infinity: it stays 65504.  (Infinities and NaN stay what they are, and so do means of e4m3 values: `mean16` is false.)
template <typename T>
__device__ __forceinline__ typename T::one rounded(float y, bool mean16) {
  if constexpr (__is_same(T, Fp16))
    if (mean16 && fabsf(y) < __builtin_inff()) y = __builtin_amdgcn_fmed3f(y, -65504.0f, 65504.0f);
  return static_cast<typename T::one>(y);
}

// Eight e4m3 codes as 16-bit values (exact in both types).
template <typename T>
__device__ __forceinline__ typename T::eight widen(u32x2 w) {
  typename T::eight r;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    typename T::two lo, hi;
    if constexpr (__is_same(T, Fp16)) {
      lo = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[i], 1.0f, false);
      hi = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[i], 1.0f, true);
    } else {
      lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], 1.0f, false);
      hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], 1.0f, true);
    }
    r[4 * i] = lo[0];
    r[4 * i + 1] = lo[1];
    r[4 * i + 2] = hi[0];
    r[4 * i + 3] = hi[1];
  }
  return r;
}

// Takes infinities and NaN out of a word of values; true if there were any.
template <typename T, bool E4M3>
__device__ __forceinline__ bool without_not_finite(uint32_t &w) {
  const uint32_t was = w;
  if constexpr (E4M3) {
#pragma unroll
    for (int i = 0; i < 32; i += 8)
      if ((was >> i & 0x7fu) == 0x7fu) w &= ~(0xffu << i);
  } else {
    constexpr uint32_t e = __is_same(T, Fp16) ? 0x7c00u : 0x7f80u;
    if ((was & e) == e) w &= 0xffff0000u;
    if ((was >> 16 & e) == e) w &= 0xffffu;
  }
  return w != was;
}

// Value i of a row in the cache, as it lies there.
template <typename T, bool E4M3>
__device__ __forceinline__ float element(const uint8_t *row, uint32_t i) {
  if constexpr (E4M3)
    return (row[i] & 0x7fu) == 0x7fu ? __builtin_nanf("") : 0.0f;  // (all that is asked of it)
  else
    return static_cast<float>(reinterpret_cast<const typename T::one *>(row)[i]);
}

template <int N>
struct Words;
template <>
struct Words<1> { using type = uint32_t; };
template <>
struct Words<2> { using type = u32x2; };
template <>
struct Words<4> { using type = u32x4; };
template <int N>
__device__ __forceinline__ uint32_t word(const typename Words<N>::type &w, int i) {
  if constexpr (N == 1)
    return w;
  else
    return w[i];
}

template <int N>
__device__ __forceinline__ void set_word(typename Words<N>::type &w, int i, uint32_t x) {
  if constexpr (N == 1)
    w = x;
  else
    w[i] = x;
}

// ---- Few queries: a workgroup takes 16 or 32 rows of queries (RT 1 or 2), which is all that a sequence has, a group of `abreast`
// neighbouring KV heads and a part of the keys.  Its wavefronts, 3 to 5: `key_waves` for each of the heads, which take the part's tiles
// in turn.
//
// Scores are computed transposed, S^T = K Q^T, with 16x16x32 matrix instructions: lane (r = l % 16, g = l / 16) holds row r of
// the queries and keys 4g..4g+3 of each half tile, which is how O^T = V^T P^T takes P, so weights stay in the lane that
// made them.  The contraction's order is free: a lane loads 16 consecutive bytes of a key's row, and the queries are laid out to
// match.  Of the values, a lane takes DP/16 consecutive ones of its eight keys, and puts pairs of keys together by byte
// permutations; so nothing passes through LDS and no wavefront waits for another until the end, where those of a head join.
// Bound by memory: 2*e*head_dim bytes a key and KV head for 4*group*head_dim flops.  32K tokens of 8 heads x 128 (128 MiB) in 28 us of
// its own, 4.8 TB/s; 128K tokens in e4m3 (256 MiB) 52 us, 5.2 TB/s; 64 sequences in e4m3 (751 MB) 142 us, 5.3 TB/s.  The same loads
// with no arithmetic reach 5.8 TB/s (nontemporal; four heads side by side, see heads_abreast), a launch of them takes 4 us to begin
// and end: records, table, scales and first keys are four trips to memory one after the other.
template <typename T, bool E4M3, int DP, bool FULL, bool PAGED16, int RT>
__global__ __launch_bounds__(64 * kMostWaves, RT == 1 && (FULL || E4M3) ? 3 : 2) void k_kv_attend(const AttendArgs a) {
  constexpr int ROWS = RT * 16, N = DP / 16;
  constexpr int KW = E4M3 ? DP / 64 : DP / 32;       // 16-byte loads of a key a lane does
  constexpr int VW = E4M3 ? N / 4 : N / 2;           // words of a value row a lane takes
  constexpr uint32_t EB = E4M3 ? 1 : 2;
  using P = std::conditional_t<E4M3, Fp16, T>;
  using VWords = typename Words<VW>::type;
  // A weight is the sum of two numbers of its type, so that its own rounding does not add to that of the result.  Error against 64 bits
  // with one and with two: 512 tokens of heads of 64, fp16 2.2e-4 and 1.9e-4, bf16 1.85e-3 and 1.53e-3 (a plain product in 32 bits, rounded
  // once at the end: 1.9e-4 and 1.5e-3), both 11 to 12 us; 32K tokens of bf16 1.63e-3 and 1.59e-3, 34.5 and 35.0 us.  A bf16 result of e4m3
  // values, whose weights are fp16, has no need of it (1.67e-3 and 1.66e-3).
  constexpr bool TWO = __is_same(T, Fp16) || !E4M3;

  const uint32_t lane = threadIdx.x & (kLanes - 1), wave = uniform(threadIdx.x / kLanes);
  const uint32_t r = lane & 15u, g = lane >> 4;
  const bool reporter = blockIdx.x == 0 && wave == 0;
  if (blockIdx.x >= a.max_units) return;
  const Plan plan = make_plan<ROWS>(a);
  if (reporter && (threadIdx.x & (kLanes - 1)) == 0) *a.tiles_a_part = plan.tiles_a_part;
  const Unit u = locate<ROWS>(a, plan, blockIdx.x, reporter);
  if (u.seq == a.batch.n_seq) return;
  if (u.parts > 1 && u.part_slot + a.abreast * u.parts > a.max_parts) {
    if (threadIdx.x == 0) report(a.status, TUTTI_ST_BAD_EXTENT);
    return;
  }
  const tutti_seq s = u.s;
  const uint32_t begin = s.n_held - s.n_new, n_rows = s.n_new * a.group;
  const uint32_t kv_head = u.head + wave % a.abreast, turn = wave / a.abreast;

  // the keys that this lane's rows see: [lo, hi)
  uint32_t lo[RT], hi[RT];
  const uint8_t *q_at[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const uint32_t row = u.row_tile * ROWS + t * 16 + r;
    const uint32_t i = row < n_rows ? row / a.group : 0, head = kv_head * a.group + (row < n_rows ? row - i * a.group : 0);
    const uint32_t place = begin + i;
    hi[t] = a.causal ? place + 1 : s.n_held;
    lo[t] = a.window && place + 1 > a.window ? place + 1 - a.window : 0;
    q_at[t] = static_cast<const uint8_t *>(a.q.base) + static_cast<uint64_t>(s.row0 + i) * a.q.row_stride + head * a.q.head_stride;
  }
  // those that any row of the tile sees, and those that all of them see
  const uint32_t row_a = u.row_tile * ROWS, row_b = min(row_a + ROWS, n_rows) - 1;
  const uint32_t place_a = begin + row_a / a.group, place_b = begin + row_b / a.group;
  const uint32_t any_hi = uniform(a.causal ? place_b + 1 : s.n_held), all_hi = uniform(a.causal ? place_a + 1 : s.n_held);
  const uint32_t any_lo = uniform(a.window && place_a + 1 > a.window ? place_a + 1 - a.window : 0);
  const uint32_t all_lo = uniform(a.window && place_b + 1 > a.window ? place_b + 1 - a.window : 0);
  const uint32_t tile_lo = any_lo / kKeyTile, tile_hi = (any_hi + kKeyTile - 1) / kKeyTile;
  const uint32_t tiles = tile_hi - tile_lo;
  const uint32_t t0 = uniform(tile_lo + static_cast<uint32_t>(static_cast<uint64_t>(tiles) * u.part / u.parts));
  const uint32_t t1 = uniform(tile_lo + static_cast<uint32_t>(static_cast<uint64_t>(tiles) * (u.part + 1) / u.parts));

  // queries, in the order of the contraction that the keys' loads give
  typename T::eight q[RT][DP / 32];
#pragma unroll
  for (int t = 0; t < RT; ++t)
#pragma unroll
    for (int j = 0; j < DP / 32; ++j) {
      const uint32_t e = E4M3 ? (j / 2) * 64 + g * 16 + (j & 1) * 8 : j * 32 + g * 8;
      u32x4 w = {0, 0, 0, 0};
      if (FULL || e < a.d) w = *reinterpret_cast<const u32x4 *>(q_at[t] + 2 * e);
      q[t][j] = __builtin_bit_cast(typename T::eight, w);
    }

  f32x4 o[RT][N];
  float m[RT], l[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    m[t] = kLowest;
    l[t] = 0.0f;
#pragma unroll
    for (int n = 0; n < N; ++n) o[t][n] = f32x4{0, 0, 0, 0};
  }

  const uint64_t head_at = static_cast<uint64_t>(kv_head) * a.pool.head_stride;
  const uint32_t ts = a.pool.token_stride;
  // of a value's row a lane takes VW words; lanes beyond the row take its first ones (nothing is made of what they add)
  const uint32_t v_in_row = FULL || r * (VW * 4) < a.d * EB ? r * (VW * 4) : 0;
  bool skipped = false;

  // S^T of a tile
  const auto scores = [&](const u32x4 (&kw)[2][KW], f32x4 (&sc)[RT][2]) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int t = 0; t < RT; ++t) sc[t][h] = f32x4{0, 0, 0, 0};
#pragma unroll
      for (int j = 0; j < KW; ++j) {
        if constexpr (E4M3) {
          const typename T::eight k0 = widen<T>(u32x2{kw[h][j][0], kw[h][j][1]}), k1 = widen<T>(u32x2{kw[h][j][2], kw[h][j][3]});
#pragma unroll
          for (int t = 0; t < RT; ++t) {
            sc[t][h] = product<T>(k0, q[t][2 * j], sc[t][h]);
            sc[t][h] = product<T>(k1, q[t][2 * j + 1], sc[t][h]);
          }
        } else {
          const typename T::eight k0 = __builtin_bit_cast(typename T::eight, kw[h][j]);
#pragma unroll
          for (int t = 0; t < RT; ++t) sc[t][h] = product<T>(k0, q[t][j], sc[t][h]);
        }
      }
    }
  };
  // weights of a tile, from its scores: c(h, i) holds the factor of key i of a lane's four in half h, the log2 and the reciprocal
  // of its value's scale, and whether it is there
  const auto weights = [&](const f32x4 (&sc)[RT][2], uint32_t key0, bool edge, auto &&c, typename P::eight (&p)[RT],
                           typename P::eight (&low)[RT]) {
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      float x[8];
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < 4; ++i) x[4 * h + i] = E4M3 ? sc[t][h][i] * c(h, i).f + c(h, i).lg : sc[t][h][i] * a.scale_log2;
      if (edge) {
        asm volatile("" ::);  // (a branch: most tiles are whole ones)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t key = key0 + 16 * h + 4 * g + i;
            if (!c(h, i).ok || key < lo[t] || key >= hi[t]) x[4 * h + i] = -__builtin_inff();
          }
      }
      float top = x[0];
#pragma unroll
      for (int i = 1; i < 8; ++i) top = fmaxf(top, x[i]);
      top = max_over_rows(top);
      if (__ballot(top > m[t] + (kRaise + kBelow<P>))) {
        const float raised = top > m[t] + (kRaise + kBelow<P>) ? top - kBelow<P> : m[t];
        const float by = __builtin_amdgcn_exp2f(m[t] - raised);
        m[t] = raised;
        l[t] *= by;
#pragma unroll
        for (int n = 0; n < N; ++n) o[t][n] *= by;
      }
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float w = __builtin_amdgcn_exp2f(x[4 * h + i] - m[t]);
          l[t] += E4M3 ? w * c(h, i).rc : w;
          p[t][4 * h + i] = static_cast<typename P::one>(w);
          if constexpr (TWO) low[t][4 * h + i] = static_cast<typename P::one>(w - static_cast<float>(p[t][4 * h + i]));
        }
    }
  };
  // O^T += V^T P^T of a tile
  const auto values = [&](VWords (&vw)[8], uint32_t key0, bool edge, auto &&c, const typename P::eight (&p)[RT],
                          const typename P::eight (&low)[RT]) {
    bool odd = false, look = edge;
    if constexpr (TWO && !E4M3) {
      // the second number of a weight may be 0 or negative: an infinity must not meet it in tiles that all rows see either
      typename T::two none = {0, 0};  // fp16: times 0, in pairs
      float nil = 0.0f;               // bf16: the same by a product of two pairs
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int x = 0; x < VW; ++x) {
          const typename T::two v = __builtin_bit_cast(typename T::two, word<VW>(vw[i], x));
          if constexpr (__is_same(T, Fp16))
            none = __builtin_elementwise_fma(v, typename T::two{0, 0}, none);
          else
            nil = __builtin_amdgcn_fdot2_f32_bf16(v, none, nil, false);
        }
      look |= __ballot(nil != nil || none[0] != none[0] || none[1] != none[1]) != 0;
    }
    if (look) {
      asm volatile("" ::);
      // values of keys that no row sees are whatever lies there: nothing of them may reach a product, not even times 0.  An infinity
      // or NaN that some rows see and others do not stays out of the products too and is added to the rows that see it (its weight is
      // positive, so what it adds is itself).
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint32_t key = key0 + 16 * (i / 4) + 4 * g + i % 4;
        if (!c(i / 4, i % 4).ok || key < any_lo || key >= any_hi) vw[i] = VWords{};
#pragma unroll
        for (int x = 0; x < VW; ++x) {
          uint32_t w = word<VW>(vw[i], x);
          odd |= without_not_finite<T, E4M3>(w);
          set_word<VW>(vw[i], x, w);
        }
      }
      odd = __ballot(odd) != 0;
    }
    // 16 values at a time: value n of the lane's, of its eight keys
#pragma unroll
    for (int n = 0; n < N; ++n) {
      u32x4 w;
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const uint32_t even = word<VW>(vw[2 * x], E4M3 ? n / 4 : n / 2), uneven = word<VW>(vw[2 * x + 1], E4M3 ? n / 4 : n / 2);
        if constexpr (E4M3) {
          const uint32_t pair = __builtin_amdgcn_perm(uneven, even, (n & 2) ? 0x07030602u : 0x05010400u);
          const f16x2 two = (n & 1) ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(pair, 1.0f, true)
                                    : __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(pair, 1.0f, false);
          w[x] = __builtin_bit_cast(uint32_t, two);
        } else {
          w[x] = __builtin_amdgcn_perm(uneven, even, (n & 1) ? 0x07060302u : 0x05040100u);
        }
      }
      const typename P::eight v = __builtin_bit_cast(typename P::eight, w);
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        if constexpr (TWO) o[t][n] = product<P>(v, low[t], o[t][n]);
        o[t][n] = product<P>(v, p[t], o[t][n]);
      }
    }
    if (odd) {
      const uint32_t from = key0 > any_lo ? key0 : any_lo, to = key0 + kKeyTile < any_hi ? key0 + kKeyTile : any_hi;
      for (uint32_t key = from; key < to; ++key) {
        const uint32_t n = block_of(a.pool, key);
        const uint64_t at = static_cast<uint64_t>(s.table_off) + n;
        const uint32_t id = at < a.batch.table_len ? a.batch.table[at] : ~0u;
        if (id >= a.pool.num_blocks) continue;
        const uint8_t *row = a.pool.v + id * a.pool.block_stride + head_at + static_cast<uint64_t>(key - n * a.pool.block_tokens) * ts;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t d0 = (4 * g + i) * N;
          if (d0 >= a.d) continue;
#pragma unroll
          for (int e = 0; e < N; ++e) {
            const float x = element<T, E4M3>(row, d0 + e);
            if (fabsf(x) < __builtin_inff()) continue;
#pragma unroll
            for (int t = 0; t < RT; ++t)
              if (key >= lo[t] && key < hi[t]) o[t][e][i] += x;
          }
        }
      }
    }
  };
  const auto load_keys = [&](const uint8_t *at, uint32_t in, u32x4 (&kw)[KW]) {
#pragma unroll
    for (int j = 0; j < KW; ++j) {
      if (!FULL) kw[j] = u32x4{0, 0, 0, 0};
      if (FULL || j * 64 + g * 16 < a.d * EB) kw[j] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(at + in + j * 64));
    }
  };

  struct Key {
    float f, lg, rc;  // factor of the score (e4m3); log2 and reciprocal of the value's scale
    bool ok;
  };
  f32x4 sc[RT][2];
  typename P::eight p[RT], low[RT];
  if constexpr (PAGED16) {
    // A half tile lies in one block.  The halves of the wavefront's next 32 tiles are looked up at once, one to a lane, and come from
    // there as uniform values.  The keys of the next tile are asked for as soon as the scores of this one have used theirs, its values as
    // soon as the products have.  (Two tiles under way, in as many registers again: 1 to 3 % less time.)
    uint64_t off_l = 0;
    Key key_l{};
    uint64_t oks = 0;
    const uint32_t mine = t1 > t0 + turn ? (t1 - t0 - turn + a.key_waves - 1) / a.key_waves : 0;  // tiles
    const auto look_up = [&](uint32_t c) {
      const uint32_t tile = t0 + turn + (c + lane / 2) * a.key_waves, key = tile * kKeyTile + 16 * (lane & 1u);
      const uint32_t n = block_of(a.pool, key);
      const uint64_t at = static_cast<uint64_t>(s.table_off) + n;
      uint32_t id = 0;
      key_l.ok = tile < t1 && key + 16 > any_lo && key < any_hi;
      if (key_l.ok) {
        if (at < a.batch.table_len) id = a.batch.table[at];
        key_l.ok = at < a.batch.table_len && id < a.pool.num_blocks;
        if (!key_l.ok) skipped = true;
      }
      if (!key_l.ok) id = 0;
      off_l = id * a.pool.block_stride + head_at + static_cast<uint64_t>(key - n * a.pool.block_tokens) * ts;
      if constexpr (E4M3) {
        const float sv = a.pool.v_scale[id * a.pool.scale_stride + kv_head];
        key_l.f = a.scale_log2 * a.pool.k_scale[id * a.pool.scale_stride + kv_head];
        key_l.lg = __builtin_amdgcn_logf(sv);
        key_l.rc = key_l.ok ? __builtin_amdgcn_rcpf(sv) : 0.0f;
      }
      oks = __ballot(key_l.ok);
    };
    struct {
      u32x4 kw[2][KW];
      VWords vw[8];
      uint64_t off[2];
      Key key[2];
    } x;  // the tile in work, then the next
    const uint32_t k_in = r * ts + (FULL || g * 16 < a.d * EB ? g * 16 : 0);
    const auto ask_keys = [&](uint32_t c) {
      if ((c & 31u) == 0) look_up(c);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t from = (c & 31u) * 2 + h;
        x.off[h] = static_cast<uint64_t>(from_lane(static_cast<uint32_t>(off_l >> 32), from)) << 32 | from_lane(static_cast<uint32_t>(off_l), from);
        x.key[h].ok = oks >> from & 1u;
        if constexpr (E4M3) {
          x.key[h].f = __uint_as_float(from_lane(__float_as_uint(key_l.f), from));
          x.key[h].lg = __uint_as_float(from_lane(__float_as_uint(key_l.lg), from));
          x.key[h].rc = __uint_as_float(from_lane(__float_as_uint(key_l.rc), from));
        }
        load_keys(a.pool.k + x.off[h], k_in, x.kw[h]);
      }
    };
    const auto ask_values = [&]() {
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          x.vw[4 * h + i] = __builtin_nontemporal_load(reinterpret_cast<const VWords *>(a.pool.v + x.off[h] + ((4 * g + i) * ts + v_in_row)));
    };
    if (mine) {
      ask_keys(0);
      ask_values();
    }
    for (uint32_t c = 0; c < mine; ++c) {
      const uint32_t key0 = (t0 + turn + c * a.key_waves) * kKeyTile;
      const Key now[2] = {x.key[0], x.key[1]};
      const bool edge = key0 < all_lo || key0 + kKeyTile > all_hi || !now[0].ok || !now[1].ok;
      const auto at = [&](int h, int) -> const Key & { return now[h]; };
      scores(x.kw, sc);
      const bool more = c + 1 < mine;
      if (more) ask_keys(c + 1);
      weights(sc, key0, edge, at, p, low);
      values(x.vw, key0, edge, at, p, low);
      if (more) ask_values();
    }
  } else {
    for (uint32_t tile = t0 + turn; tile < t1; tile += a.key_waves) {
      const uint32_t key0 = tile * kKeyTile;
      u32x4 kw[2][KW];
      VWords vw[8];
      Key key[2][4];
      bool edge = key0 < all_lo || key0 + kKeyTile > all_hi;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        // lane r looks up key r of the half; the others' come from it
        const uint32_t k = key0 + 16 * h + r;
        const uint32_t n = block_of(a.pool, k);
        const uint64_t at = static_cast<uint64_t>(s.table_off) + n;
        uint32_t id = 0;
        bool ok = k >= any_lo && k < any_hi;
        if (ok) {
          if (at < a.batch.table_len) id = a.batch.table[at];
          ok = at < a.batch.table_len && id < a.pool.num_blocks;
          if (!ok) skipped = true;
        }
        if (__ballot(!ok)) edge = true;
        if (!ok) id = 0;
        const uint32_t slot = ok ? k - n * a.pool.block_tokens : 0;
        Key mine{0, 0, 0, ok};
        if constexpr (E4M3) {
          const float sv = a.pool.v_scale[id * a.pool.scale_stride + kv_head];
          mine.f = a.scale_log2 * a.pool.k_scale[id * a.pool.scale_stride + kv_head];
          mine.lg = __builtin_amdgcn_logf(sv);
          mine.rc = ok ? __builtin_amdgcn_rcpf(sv) : 0.0f;
        }
        load_keys(a.pool.k + id * a.pool.block_stride + head_at + static_cast<uint64_t>(slot) * ts, g * 16, kw[h]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int from = static_cast<int>(4 * g + i);
          const uint32_t id_i = __shfl(id, from, 16), slot_i = __shfl(slot, from, 16);
          vw[4 * h + i] = *reinterpret_cast<const VWords *>(a.pool.v + id_i * a.pool.block_stride + head_at +
                                                            static_cast<uint64_t>(slot_i) * ts + v_in_row);
          key[h][i] = Key{__shfl(mine.f, from, 16), __shfl(mine.lg, from, 16), __shfl(mine.rc, from, 16),
                          __shfl(static_cast<int>(ok), from, 16) != 0};
        }
      }
      const auto at = [&](int h, int i) -> const Key & { return key[h][i]; };
      scores(kw, sc);
      weights(sc, key0, edge, at, p, low);
      values(vw, key0, edge, at, p, low);
    }
  }
  if (__ballot(skipped) && lane == 0) report(a.status, TUTTI_ST_BAD_BLOCK);

  // the wavefronts' maxima, sums and rows meet in LDS, 16 rows at a time
  const auto &z = arguments_again<AttendArgs>();
  constexpr int LD = DP + 4;                        // rows apart by 4 banks
  __shared__ __attribute__((aligned(16))) float rows[kMostWaves][16][LD];
  __shared__ float ml[kMostWaves][16][2];
  constexpr uint32_t EACH = 8, SEGS = DP / EACH;    // a thread joins 8 values of a row
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const float own_sum = sum_over_rows(l[t]);
    if (t) __syncthreads();
    if (g == 0) {
      ml[wave][r][0] = m[t];
      ml[wave][r][1] = own_sum;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int n = 0; n < N; n += 4)
        *reinterpret_cast<f32x4 *>(&rows[wave][r][(4 * g + i) * N + n]) =
            f32x4{o[t][n][i], o[t][n + 1][i], o[t][n + 2][i], o[t][n + 3][i]};
    __syncthreads();
    for (uint32_t x = threadIdx.x; x < z.abreast * 16 * SEGS; x += blockDim.x) {
      const uint32_t hw = x / (16 * SEGS), row_in = x / SEGS % 16, e = (x % SEGS) * EACH, row = row_a + t * 16 + row_in;
      if (row >= n_rows || e >= z.d) continue;
      float top = kLowest;
      for (uint32_t w = hw; w < z.abreast * z.key_waves; w += z.abreast) top = fmaxf(top, ml[w][row_in][0]);
      float sum = 0.0f, y[EACH] = {};
      for (uint32_t w = hw; w < z.abreast * z.key_waves; w += z.abreast) {
        const float by = __builtin_amdgcn_exp2f(ml[w][row_in][0] - top);
        sum += by * ml[w][row_in][1];
#pragma unroll
        for (uint32_t i = 0; i < EACH; ++i) y[i] += by * rows[w][row_in][e + i];
      }
      if (u.parts > 1) {
        const uint64_t at = static_cast<uint64_t>(u.part_slot + hw * u.parts + u.part) * ROWS + t * 16 + row_in;
        float *to = z.part_o + at * DP + e;
        *reinterpret_cast<f32x4 *>(to) = f32x4{y[0], y[1], y[2], y[3]};
        *reinterpret_cast<f32x4 *>(to + 4) = f32x4{y[4], y[5], y[6], y[7]};
        if (e == 0) z.part_ml[at] = f32x2{top, sum};
        continue;
      }
      const uint32_t i = row / z.group, head = (u.head + hw) * z.group + row - i * z.group;
      const float by = sum > 0.0f || sum != sum ? 1.0f / sum : 0.0f;
      typename T::eight y16;
#pragma unroll
      for (uint32_t c = 0; c < EACH; ++c) y16[c] = rounded<T>(y[c] * by, !E4M3);
      *reinterpret_cast<u32x4 *>(static_cast<uint8_t *>(z.out.base) + static_cast<uint64_t>(s.row0 + i) * z.out.row_stride +
                                 head * z.out.head_stride + 2 * e) = __builtin_bit_cast(u32x4, y16);
      if (e == 0 && z.lse)
        z.lse[static_cast<uint64_t>(s.row0 + i) * (z.kv_heads * z.group) + head] =
            sum == 0.0f ? -__builtin_inff() : (top + __builtin_amdgcn_logf(sum)) * kLn2;
    }
  }
}

// ---- Many queries: a workgroup of four wavefronts takes 128 rows of queries, a KV head and a part of the keys, 64 at a time.
//
// A tile of keys and values lies in LDS as 16-bit rows, twice: while one is worked on the next is on its way (16-bit blocks straight
// from memory to LDS, e4m3 through registers, where it is widened).  Units of 16 bytes are swapped within a row by the row's number, so
// that neither 16 keys' rows nor the transposed reads of four values' rows meet in one of the 64 banks; the swap is made by which
// address a lane loads.  S^T = K Q^T and O^T = V^T P^T with 32x32x16 matrix instructions: lane (r = l % 32, h = l / 32) holds row r of the queries
// and keys 8i+4h..8i+4h+3 of each 32, and the weights go from one product to the other where they are; values are read
// transposed, four keys of 16 values at a time.
// Bound by what a compute unit's wavefronts can issue: 2,048 queries behind 30,000 e4m3 tokens, 1.04 TFLOP, in 1.17 to 1.21 ms,
// 0.86 to 0.89 PFLOP/s (a large library product: 1.18), where a wavefront issues half of its time, waits to issue a quarter and for LDS or
// its neighbours a quarter; the matrix units are busy 38 % of the time, LDS as much.  With all loads from one tile the time is the same.
// The same of bf16 blocks 1.04 ms.  Prompts of 8,001 tokens in bf16, 0.12 TFLOP: 0.165 ms.  32 rows a wavefront, two wavefronts a SIMD: 64
// rows need all registers of one, and nothing covers its waits (1.94 ms).
// A weight is one number of its type, unlike where queries are few.  With one and with two, on one machine: the prompts 0.176 and 0.214 ms
// (error against 64 bits 2.1e-3 and 1.6e-3, the plain product's 1.6e-3), in fp16 0.182 and 0.220 (2.6e-4 and 2.1e-4), the chunk of e4m3
// blocks 1.18 and 1.58 (1.67e-3 and 1.66e-3: its weights are fp16).
constexpr uint32_t kWideTile = 64;

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
#define TUTTI_LDS __attribute__((address_space(3)))
#define TUTTI_GLOBAL __attribute__((address_space(1)))

// What the number of a unit of a row is exclusive-ored with.  Rows of 16 units: four rows lie in four quarters of the banks, 16 rows' same
// unit in all of them; rows of 8 units: the same, two rows to a round of the banks.
template <int UNITS>
__device__ __forceinline__ uint32_t swap_of(uint32_t row) {
  return UNITS == 16 ? (row & 3u) << 2 | (row >> 2 & 3u) : (row >> 1 & 1u) << 2 | (row >> 2 & 3u);
}

// LDS by its address there.
template <typename E>
__device__ __forceinline__ TUTTI_LDS E *in_lds(uint32_t at) {
  return reinterpret_cast<TUTTI_LDS E *>(static_cast<uintptr_t>(at));
}

template <typename T>
__device__ __forceinline__ f32x16 wide_product(typename T::eight a, typename T::eight b, f32x16 c) {
  if constexpr (__is_same(T, Fp16))
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

__device__ __forceinline__ float max_of_halves(float x) {
  const uint32_t a = __float_as_uint(x);
  const auto q = __builtin_amdgcn_permlane32_swap(a, a, false, false);
  return fmaxf(__uint_as_float(q[0]), __uint_as_float(q[1]));
}
__device__ __forceinline__ float sum_of_halves(float x) {
  const uint32_t a = __float_as_uint(x);
  const auto q = __builtin_amdgcn_permlane32_swap(a, a, false, false);
  return __uint_as_float(q[0]) + __uint_as_float(q[1]);
}

// D: values of a head that it is built for; FULL: a head has so many (else fewer than 64, and D is 64).
template <typename T, bool E4M3, int D, bool FULL, bool PAGED16>
__global__ __launch_bounds__(256, 2) void k_kv_attend_wide(const AttendArgs a) {
  constexpr int DP = D <= 64 ? 64 : 128, ROWS = 128, STEPS = D / 16, DT = (D + 31) / 32;
  constexpr uint32_t UNITS = DP / 8, ROW_BYTES = DP * 2, PLANE = kWideTile * ROW_BYTES;
  constexpr uint32_t EB = E4M3 ? 1 : 2;
  using P = std::conditional_t<E4M3, Fp16, T>;
  const uint32_t d = FULL ? D : a.d;
  __shared__ __attribute__((aligned(1024))) uint8_t lds[4 * PLANE];
  __shared__ uint32_t not_finite[4];  // a wavefront has met an infinity or NaN among the values of a tile that has an edge
  __shared__ float per_key[E4M3 && !PAGED16 ? 4 : 1][3][kWideTile];

  const uint32_t lane = threadIdx.x & (kLanes - 1), wave = uniform(threadIdx.x / kLanes);
  const uint32_t r = lane & 31u, hf = lane >> 5;
  const bool reporter = blockIdx.x == 0 && wave == 0;
  if (blockIdx.x >= a.max_units) return;
  const Plan plan = make_plan<ROWS>(a);
  if (reporter && (threadIdx.x & (kLanes - 1)) == 0) *a.tiles_a_part = plan.tiles_a_part;
  const Unit u = locate<ROWS>(a, plan, blockIdx.x, reporter);
  if (u.seq == a.batch.n_seq) return;
  if (u.parts > 1 && u.part_slot + u.parts > a.max_parts) {
    if (threadIdx.x == 0) report(a.status, TUTTI_ST_BAD_EXTENT);
    return;
  }
  const tutti_seq s = u.s;
  const uint32_t begin = s.n_held - s.n_new, n_rows = s.n_new * a.group;

  // the keys that a place sees: [low(place), high(place))
  const auto high = [&](uint32_t place) { return a.causal ? place + 1 : s.n_held; };
  const auto low = [&](uint32_t place) { return a.window && place + 1 > a.window ? place + 1 - a.window : 0; };
  // those that any row, and that all rows, of the workgroup (of the wavefront) see
  const uint32_t row_a = u.row_tile * ROWS, row_b = min(row_a + ROWS, n_rows) - 1;
  const uint32_t place_a = begin + row_a / a.group, place_b = begin + row_b / a.group;
  const uint32_t any_lo = uniform(low(place_a)), any_hi = uniform(high(place_b)), all_lo = uniform(low(place_b)), all_hi = uniform(high(place_a));
  const uint32_t wave_a = row_a + wave * 32, wave_b = min(wave_a + 32, n_rows);
  const bool has_rows = wave_a < wave_b;
  const uint32_t w_place_a = has_rows ? begin + wave_a / a.group : 0, w_place_b = has_rows ? begin + (wave_b - 1) / a.group : 0;
  const uint32_t w_any_lo = uniform(low(w_place_a)), w_any_hi = has_rows ? uniform(high(w_place_b)) : 0;
  const uint32_t w_all_lo = uniform(low(w_place_b)), w_all_hi = uniform(high(w_place_a));
  const uint32_t tile_lo = any_lo / kWideTile, tiles = (any_hi + kWideTile - 1) / kWideTile - tile_lo;
  const uint32_t t0 = uniform(tile_lo + static_cast<uint32_t>(static_cast<uint64_t>(tiles) * u.part / u.parts));
  const uint32_t t1 = uniform(tile_lo + static_cast<uint32_t>(static_cast<uint64_t>(tiles) * (u.part + 1) / u.parts));

  uint32_t lo, hi;  // of the lane's row
  typename T::eight q[STEPS];
  const uint32_t flip = a.scale_log2 < 0.0f ? 0x80008000u : 0;  // scores are multiplied by a factor that is positive
  const float factor = fmaxf(fabsf(a.scale_log2), 0x1p-100f);   // (0: no score counts; times 0, a masked one would be no number)
  {
    const uint32_t row = wave_a + r;
    const bool in = row < n_rows;
    const uint32_t i = in ? row / a.group : 0, head = u.head * a.group + (in ? row - i * a.group : 0);
    hi = high(begin + i);
    lo = low(begin + i);
    const uint8_t *at = static_cast<const uint8_t *>(a.q.base) + static_cast<uint64_t>(s.row0 + i) * a.q.row_stride + head * a.q.head_stride;
#pragma unroll
    for (int j = 0; j < STEPS; ++j) {
      u32x4 x = {0, 0, 0, 0};
      if (FULL || j * 16 < static_cast<int>(d)) x = *reinterpret_cast<const u32x4 *>(at + j * 32 + hf * 16);
      x ^= u32x4{flip, flip, flip, flip};
      q[j] = __builtin_bit_cast(typename T::eight, x);
    }
  }
  f32x16 o[DT];
  float m = kLowest, l = 0.0f;
  bool large = false;  // some row's m is
#pragma unroll
  for (int n = 0; n < DT; ++n)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[n][i] = 0.0f;

  const uint64_t head_at = static_cast<uint64_t>(u.head) * a.pool.head_stride;
  const uint32_t ts = a.pool.token_stride;
  TUTTI_LDS uint8_t *const base = (TUTTI_LDS uint8_t *)lds;
  const uint32_t lds_at = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(base));
  if (threadIdx.x < 4) not_finite[threadIdx.x] = 0;
  if (!FULL || D != DP) {  // units behind the rows' ends are never written: what lies there meets weights
    for (uint32_t x = threadIdx.x * 16; x < 4 * PLANE; x += 256 * 16) *(TUTTI_LDS u32x4 *)(base + x) = u32x4{0, 0, 0, 0};
    __syncthreads();
  }

  bool skipped = false;
  struct Tile {
    uint64_t oks;      // its keys that some row sees and that are there
    uint64_t at;       // !PAGED16: where the lane's key is, from a plane's begin; e4m3: its factor of the scores, log2 and reciprocal of
    float f, lg, rc;   // the values' scale
  };
  Tile now{}, next{}, second{};  // the tile in work, the next (its values are on their way), the one after that (its keys)
  u32x4 raw_k[E4M3 ? DP / 64 : 1], raw_v[E4M3 ? DP / 64 : 1];
  constexpr uint32_t CHUNKS = kWideTile * DP * EB / 4096;   // 1 KiB each, of a plane, that a wavefront brings: 16 rows
  constexpr uint32_t LANES_A_ROW = DP * EB / 16, ROWS_A_CHUNK = kLanes / LANES_A_ROW;
  static_assert(CHUNKS * ROWS_A_CHUNK == 16);
  const auto scale_of = [&](uint32_t id, bool ok, float &f, float &lg, float &rc) {
    const float sv = a.pool.v_scale[id * a.pool.scale_stride + u.head];
    // (f not 0: times 0, a score of -infinity would be no number)
    f = ok ? fmaxf(factor * a.pool.k_scale[id * a.pool.scale_stride + u.head], 0x1p-120f) : 1.0f;
    lg = ok ? __builtin_amdgcn_logf(sv) : 0.0f;
    rc = ok ? __builtin_amdgcn_rcpf(sv) : 0.0f;
  };
  // PAGED16: 16 keys from a multiple of 16 on lie in one block.  Those of 16 tiles are looked up at once, 16 keys to a lane, and from
  // the tile in work on again when the one after the next is none of them; a tile's come from there as uniform values, and the
  // wavefront brings the 16 keys that are its own.
  struct {
    uint32_t tile;     // the first
    uint64_t oks, at;  // which lanes' keys are there; where the lane's are, from a plane's begin
    float f, lg, rc;
  } looked{};
  const auto look_up_16 = [&](uint32_t tile0) {
    looked.tile = tile0;
    const uint32_t key = tile0 * kWideTile + 16 * lane, n = block_of(a.pool, key);
    const uint64_t at = static_cast<uint64_t>(s.table_off) + n;
    bool ok = key < t1 * kWideTile && key + 16 > any_lo && key < any_hi;
    uint32_t id = 0;
    const bool asked = ok;
    if (ok) {
      if (at < a.batch.table_len) id = a.batch.table[at];
      ok = at < a.batch.table_len && id < a.pool.num_blocks;
    }
    skipped |= __ballot(asked && !ok) != 0;
    if (!ok) id = 0;
    looked.at = id * a.pool.block_stride + head_at + static_cast<uint64_t>(key - n * a.pool.block_tokens) * ts;
    if constexpr (E4M3) scale_of(id, ok, looked.f, looked.lg, looked.rc);
    looked.oks = __ballot(ok);
  };
  // brings the wavefront's 16 rows of a tile from a plane
  const auto bring = [&](const uint8_t *plane, uint32_t tile, const Tile &t, uint32_t to_at, u32x4 (&raw)[E4M3 ? DP / 64 : 1]) {
    // PAGED16: an address for all lanes, in scalar registers, and what a lane adds to it
    uintptr_t rows = reinterpret_cast<uintptr_t>(plane);
    if constexpr (PAGED16) {
      const uint32_t from = (tile - looked.tile) * 4 + wave;
      rows += static_cast<uint64_t>(from_lane(static_cast<uint32_t>(looked.at >> 32), from)) << 32 | from_lane(static_cast<uint32_t>(looked.at), from);
      asm volatile("" : "+s"(rows));
    }
    const uint32_t oks = static_cast<uint32_t>(t.oks >> (wave * 16));
    uint32_t l = lane;
    if constexpr (E4M3) asm volatile("" : "+v"(l));  // (what follows from it is worked out anew: it has no registers to wait in)
    const uint32_t place = l % LANES_A_ROW;
#pragma unroll
    for (uint32_t c = 0; c < CHUNKS; ++c) {
      const uint32_t in = c * ROWS_A_CHUNK + l / LANES_A_ROW, row = wave * 16 + in;
      if constexpr (!PAGED16)
        rows = reinterpret_cast<uintptr_t>(plane) + (static_cast<uint64_t>(__shfl(static_cast<uint32_t>(t.at >> 32), row, kLanes)) << 32 |
                                                     __shfl(static_cast<uint32_t>(t.at), row, kLanes));
      const TUTTI_GLOBAL uint8_t *from = reinterpret_cast<const TUTTI_GLOBAL uint8_t *>(rows);
      const uint32_t unit = E4M3 ? place : place ^ swap_of<UNITS>(row);
      uint32_t off = (PAGED16 ? in * ts : 0) + unit * 16;
      const bool inside = unit * 16 < d * EB;
      if constexpr (E4M3) {
        raw[c] = u32x4{0, 0, 0, 0};
        if (inside && (oks >> in & 1u)) {
          asm volatile("" : "+v"(off));  // (32 bits, to be added to the scalar address by the load)
          raw[c] = *reinterpret_cast<const TUTTI_GLOBAL u32x4 *>(from + off);
        }
      } else if (inside) {
        asm volatile("" : "+v"(off));
        __builtin_amdgcn_global_load_lds((const TUTTI_GLOBAL void *)(from + off),
                                         (TUTTI_LDS void *)(base + to_at + (wave * CHUNKS + c) * 1024), 16, 0, 0);
      }
    }
  };
  // e4m3: widens what bring() has brought
  const auto put = [&](uint32_t to_at, const u32x4 (&raw)[E4M3 ? DP / 64 : 1], auto to_type) {
    if constexpr (E4M3) {
      uint32_t l = lane;
      asm volatile("" : "+v"(l));
      const uint32_t place = l % LANES_A_ROW;
#pragma unroll
      for (uint32_t c = 0; c < CHUNKS; ++c) {
        const uint32_t row = wave * 16 + c * ROWS_A_CHUNK + l / LANES_A_ROW;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const uint32_t unit = (2 * place + x) ^ swap_of<UNITS>(row);
          *(TUTTI_LDS u32x4 *)(base + to_at + row * ROW_BYTES + unit * 16) =
              __builtin_bit_cast(u32x4, widen<decltype(to_type)>(u32x2{raw[c][2 * x], raw[c][2 * x + 1]}));
        }
      }
    }
  };
  // else: one key to a lane, the following tile's ids on their way while this one's keys are brought
  uint32_t id_next = 0;
  bool ok_next = false;
  const auto look_up_1 = [&](uint32_t tile) {
    const uint32_t key = tile * kWideTile + lane;
    const uint64_t at = static_cast<uint64_t>(s.table_off) + block_of(a.pool, key);
    ok_next = tile < t1 && key >= any_lo && key < any_hi;
    id_next = 0;
    if (ok_next) id_next = at < a.batch.table_len ? a.batch.table[at] : ~0u;
  };
  const auto find = [&](uint32_t tile, Tile &t) {
    if constexpr (PAGED16) {
      const uint32_t key0 = tile * kWideTile;
      if (tile - looked.tile >= 16) look_up_16(tile - 2);
      const uint32_t four = static_cast<uint32_t>(looked.oks >> ((tile - looked.tile) * 4));
      t.oks = 0;
#pragma unroll
      for (int x = 0; x < 4; ++x)
        if (four >> x & 1u) t.oks |= 0xffffull << (16 * x);
      if (key0 < any_lo) t.oks &= ~0ull << (any_lo - key0);
      if (key0 + kWideTile > any_hi) t.oks &= ~(~0ull << (any_hi - key0));  // (key0 < any_hi)
    } else {
      const uint32_t key = tile * kWideTile + lane;
      const bool lost = ok_next && id_next >= a.pool.num_blocks;
      skipped |= __ballot(lost) != 0;
      ok_next = ok_next && !lost;
      const uint32_t id = ok_next ? id_next : 0, slot = key - block_of(a.pool, key) * a.pool.block_tokens;
      t.at = id * a.pool.block_stride + head_at + static_cast<uint64_t>(slot) * ts;
      t.oks = __ballot(ok_next);
      if constexpr (E4M3) scale_of(id, ok_next, t.f, t.lg, t.rc);
      look_up_1(tile + 1);
    }
  };

  // where a lane reads: its key's row, from which step j is 2j units away by exclusive or; its four values' rows of 8, from which 32
  // values further on are 4 units away
  const uint32_t key_at = r * ROW_BYTES + (hf ^ swap_of<UNITS>(r)) * 16;
  uint32_t value_at[2];
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    const uint32_t j = lane & 15u, row = 8 * c + 4 * hf + j / 4, unit = 2 * (lane >> 4 & 1u) + (j & 3u) / 2;
    value_at[c] = row * ROW_BYTES + (unit ^ swap_of<UNITS>(row)) * 16 + (j & 1u) * 8;
  }
  // keys 16x.. of the tile, values 32n..: what the products take
  const auto values_of = [&](uint32_t from, int n, int x) {
    s16x4 v[2];
#pragma unroll
    for (int c = 0; c < 2; ++c)
      v[c] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(in_lds<s16x4>(((lds_at + from + value_at[c]) ^ (n << 6)) + 16 * x * ROW_BYTES));
    return __builtin_bit_cast(typename P::eight, __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7));
  };
  // which keys of a tile a lane's row sees: bit c for key c + 4*hf of it
  const auto seen_of = [&](uint32_t key0) {
    const uint32_t from = lo > key0 ? min(lo - key0, kWideTile) : 0, to = hi > key0 ? min(hi - key0, kWideTile) : 0;
    uint64_t bits = now.oks;
    bits &= from < 64 ? ~0ull << from : 0;
    bits &= to < 64 ? ~(~0ull << to) : ~0ull;
    return bits >> (4 * hf);
  };
  // Products of a tile's scores: step i of 2*STEPS is 16 values of the first or the second 32 keys, in turn.
  const auto key_of = [&](uint32_t k_at, int i) {
    return __builtin_bit_cast(typename T::eight, *in_lds<u32x4>(((lds_at + k_at + key_at) ^ (i / 2 << 5)) + i % 2 * 32 * ROW_BYTES));
  };
  // LDS: keys of even and of odd tiles, then the values
  const auto k_of = [&](uint32_t tile) { return (tile - t0 & 1u) * PLANE; };
  const auto v_of = [&](uint32_t tile) { return (2 + (tile - t0 & 1u)) * PLANE; };
  // the tiles that some row of the wavefront sees
  const uint32_t w_t0 = has_rows ? max(t0, w_any_lo / kWideTile) : t1;
  const uint32_t w_t1 = has_rows ? min(t1, (w_any_hi + kWideTile - 1) / kWideTile) : 0;

  // reads of LDS that are under way before the product that takes the first of them: of keys, of values, and of those between the
  // products of the keys already (e4m3 has fewer registers left: the rows that come in are there too)
  constexpr int AHEAD = 4, VALUES_AHEAD = DT, VALUES_EARLY = DT;
  f32x16 sc[2];
  const auto scores_alone = [&](uint32_t tile) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < 16; ++i) sc[h][i] = 0.0f;
#pragma unroll
    for (int i = 0; i < 2 * STEPS; ++i) sc[i % 2] = wide_product<T>(key_of(k_of(tile), i), q[i / 2], sc[i % 2]);
  };

  // Before tile t is worked on its scores are there, its values and the next tile's keys are in LDS; while it is worked on the next
  // tile's values and the keys of the one after that come in.
  // A plane is filled only behind a barrier that is behind the last read of it, in the first turn too: some wavefronts read the first
  // tile's keys for its scores, others, whose rows see nothing of it, go straight on to that turn, which fills the same plane.  (Turns
  // end with the barrier: where they began with it prompts of 8,001 tokens took 185 us, so 174 on the same machine.)
  if (t1 > t0) {
    if (PAGED16)
      look_up_16(t0);
    else
      look_up_1(t0);
    find(t0, now);
    bring(a.pool.k, t0, now, k_of(t0), raw_k);
    bring(a.pool.v, t0, now, v_of(t0), raw_v);
    put(k_of(t0), raw_k, T{});
    put(v_of(t0), raw_v, Fp16{});
    if (t0 + 1 < t1) {
      find(t0 + 1, next);
      bring(a.pool.k, t0 + 1, next, k_of(t0 + 1), raw_k);
      put(k_of(t0 + 1), raw_k, T{});
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (w_t0 == t0 && w_t1 > t0) scores_alone(t0);
    __syncthreads();
  }
  for (uint32_t tile = t0; tile < t1; ++tile) {
    const uint32_t key0 = tile * kWideTile, v_at = v_of(tile), k_at = k_of(tile + 1);
    const bool more = tile + 1 < t1, more_keys = tile + 2 < t1;
    if (E4M3 && !PAGED16) {
      per_key[wave][0][lane] = now.f;
      per_key[wave][1][lane] = now.lg;
      per_key[wave][2][lane] = now.rc;
    }
    if (more) bring(a.pool.v, tile + 1, next, v_of(tile + 1), raw_v);
    if (more_keys) {
      find(tile + 2, second);
      bring(a.pool.k, tile + 2, second, k_of(tile + 2), raw_k);
    }
    const bool wg_edge = key0 < all_lo || key0 + kWideTile > all_hi || now.oks != ~0ull;
    bool odd = false;
    if (wg_edge) {
      // values of keys that no row sees are whatever lies there, and an infinity or NaN that some rows see must not meet the others'
      // weights of 0: both leave the tile, the latter are added to the rows that see them further down
      constexpr uint32_t EACH = PLANE / 256 / 16;
      bool any = false;
#pragma unroll
      for (uint32_t x = 0; x < EACH; ++x) {
        const uint32_t unit = threadIdx.x * EACH + x, row = unit / UNITS;
        TUTTI_LDS u32x4 *at = (TUTTI_LDS u32x4 *)(base + v_at + unit * 16);
        u32x4 w = *at;
        if (!(now.oks >> row & 1u)) w = u32x4{0, 0, 0, 0};
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          uint32_t one = w[c];
          any |= without_not_finite<P, false>(one);
          w[c] = one;
        }
        *at = w;
      }
      if (__ballot(any) && lane == 0) not_finite[wave] = 1;
      __syncthreads();
      odd = not_finite[0] | not_finite[1] | not_finite[2] | not_finite[3];
    }
    if (tile >= w_t0 && tile < w_t1) {
      typename T::eight k[2 * STEPS];
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) k[i] = key_of(k_at, i);
      if (E4M3 && !PAGED16) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int i = 0; i < 16; i += 4) {
            const f32x4 f = *reinterpret_cast<const f32x4 *>(&per_key[wave][0][32 * h + 2 * i + 4 * hf]);
            const f32x4 lg = *reinterpret_cast<const f32x4 *>(&per_key[wave][1][32 * h + 2 * i + 4 * hf]);
#pragma unroll
            for (int x = 0; x < 4; ++x) sc[h][i + x] = sc[h][i + x] * f[x] + lg[x];
          }
      }
      if (key0 < w_all_lo || key0 + kWideTile > w_all_hi || now.oks != ~0ull) {
        asm volatile("" ::);  // (a branch: most tiles are whole ones)
        const uint64_t seen = seen_of(key0);
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (!(seen >> (32 * h + 8 * (i / 4) + i % 4) & 1u)) sc[h][i] = -__builtin_inff();
      }
      float f16[4], lg16[4], rc16[4];  // e4m3, PAGED16: of each 16 keys
      if constexpr (E4M3 && PAGED16)
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const uint32_t from = (tile - looked.tile) * 4 + x;
          f16[x] = __uint_as_float(from_lane(__float_as_uint(looked.f), from));
          lg16[x] = __uint_as_float(from_lane(__float_as_uint(looked.lg), from));
          rc16[x] = __uint_as_float(from_lane(__float_as_uint(looked.rc), from));
        }
      // the largest of each 16 keys, then with their factors of all
      float top = -__builtin_inff();
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        float most = sc[x / 2][8 * (x & 1)];
#pragma unroll
        for (int i = 1; i < 8; ++i) most = fmaxf(most, sc[x / 2][8 * (x & 1) + i]);
        if constexpr (E4M3 && PAGED16) most = __builtin_fmaf(most, f16[x], lg16[x]);
        top = fmaxf(top, most);
      }
      if (!E4M3) top *= factor;
      top = max_of_halves(top);
      // A weight is 2^(score*factor - m) with the product not rounded by itself, where m is one that was: from 2^12 on the difference, 2^-12
      // and more, would count beside 1, and from 2^27 on overflow.  There the products are rounded first, and m taken off them exactly.
      float times = factor, from_m = m;
      if (large || __ballot(top > m + (kRaise + kBelow<P>))) {
        const float raised = top > m + (kRaise + kBelow<P>) ? top - kBelow<P> : m;
        const float by = __builtin_amdgcn_exp2f(m - raised);
        m = raised;
        l *= by;
#pragma unroll
        for (int n = 0; n < DT; ++n) o[n] *= by;
        from_m = m;
        if constexpr (!E4M3 || PAGED16) {
          constexpr uint32_t kLarge = 0x45800000u, kEnd = 0x7f7fffffu;  // magnitudes of 2^12 and more, but not that of kLowest
          large = __ballot((__float_as_uint(m) & 0x7fffffffu) - kLarge < kEnd - kLarge) != 0;
          if (large) {
#pragma clang fp contract(off)
#pragma unroll
            for (int x = 0; x < 4; ++x) {
#pragma unroll
              for (int i = 0; i < 8; ++i) {
                const float s = sc[x / 2][8 * (x & 1) + i], product = E4M3 ? __builtin_fmaf(s, f16[x], lg16[x]) : s * factor;
                sc[x / 2][8 * (x & 1) + i] = product - m;
              }
              f16[x] = 1.0f;
              lg16[x] = 0.0f;
            }
            times = 1.0f;
            from_m = 0.0f;
          }
        }
      }
      // this tile's weights, two at a time, between the products of the next one's scores (of what lies there, if there is none:
      // nobody asks for them)
      typename P::eight p[4];
      f32x16 following[2];
      typename P::eight v[4 * DT];
      float sum = 0.0f;
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < 16; ++i) following[h][i] = 0.0f;
#pragma unroll
      for (int y = 0; y < 16; ++y) {
#pragma unroll
        for (int i = y * 2 * STEPS / 16; i < (y + 1) * 2 * STEPS / 16; ++i) {
          if (i + AHEAD < 2 * STEPS) k[i + AHEAD] = key_of(k_at, i + AHEAD);
          following[i % 2] = wide_product<T>(k[i], q[i / 2], following[i % 2]);
        }
        if (y >= 16 - VALUES_EARLY) v[y - (16 - VALUES_EARLY)] = values_of(v_at, y - (16 - VALUES_EARLY), 0);
        const int x = y / 4;
        const float f = E4M3 ? (PAGED16 ? f16[x] : 1.0f) : times, less = (E4M3 && PAGED16 ? lg16[x] : 0.0f) - from_m;
#pragma unroll
        for (int z = 0; z < 2; ++z) {
          const int i = (2 * y + z) % 8;
          const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[x / 2][8 * (x & 1) + i], f, less));
          if constexpr (E4M3 && !PAGED16)
            sum += w * per_key[wave][2][16 * x + 8 * (i / 4) + 4 * hf + i % 4];
          else
            sum += w;
          p[x][i] = static_cast<typename P::one>(w);
        }
        if (y % 4 == 3) {
          l += E4M3 && PAGED16 ? sum * rc16[x] : sum;
          sum = 0.0f;
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      __builtin_amdgcn_s_setprio(1);  // the other wavefront's arithmetic fits between matrix instructions, not the other way round
#pragma unroll
      for (int i = VALUES_EARLY; i < VALUES_AHEAD; ++i) v[i] = values_of(v_at, i % DT, i / DT);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < 4 * DT; ++i) {
        const int soon = i + VALUES_AHEAD;
        if (soon < 4 * DT) v[soon] = values_of(v_at, soon % DT, soon / DT);
        o[i % DT] = wide_product<P>(v[i], p[i / DT], o[i % DT]);
        __builtin_amdgcn_sched_barrier(0);
      }
      __builtin_amdgcn_s_setprio(0);
#pragma unroll
      for (int h = 0; h < 2; ++h) sc[h] = following[h];
    } else if (tile + 1 == w_t0 && more) {
      scores_alone(tile + 1);
    }
    if (odd) {
      // the infinities and NaN of the tile as numbers that say what they are, for the rows that see them: 1, 2^7 and 2^14, sums of
      // 64 of which say which there were
      __syncthreads();
      if (threadIdx.x < 4) not_finite[threadIdx.x] = 0;  // (all have read it before they met here)
#pragma unroll 1
      for (uint32_t x = threadIdx.x; x < PLANE / 16; x += 256) {
        const uint32_t row = x / UNITS, d0 = ((x % UNITS) ^ swap_of<UNITS>(row)) * 8, key = key0 + row;
        typename P::eight w = {};
        if (d0 < d && key >= any_lo && key < any_hi) {
          const uint32_t n = block_of(a.pool, key);
          const uint64_t at = static_cast<uint64_t>(s.table_off) + n;
          const uint32_t id = at < a.batch.table_len ? a.batch.table[at] : ~0u;
          if (id < a.pool.num_blocks) {
            const uint8_t *from = a.pool.v + id * a.pool.block_stride + head_at + static_cast<uint64_t>(key - n * a.pool.block_tokens) * ts;
#pragma unroll
            for (int c = 0; c < 8; ++c) {
              const float e = element<T, E4M3>(from, d0 + c);
              w[c] = static_cast<typename P::one>(e != e ? 16384.0f : e == __builtin_inff() ? 1.0f : e == -__builtin_inff() ? 128.0f : 0.0f);
            }
          }
        }
        *(TUTTI_LDS u32x4 *)(base + v_at + x * 16) = __builtin_bit_cast(u32x4, w);
      }
      __syncthreads();
      if (has_rows) {
        const uint64_t bits = seen_of(key0);
#pragma unroll
        for (int n = 0; n < DT; ++n) {
          f32x16 sums;
#pragma unroll
          for (int i = 0; i < 16; ++i) sums[i] = 0.0f;
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            const typename P::eight v = values_of(v_at, n, x);
            typename P::eight seen;
#pragma unroll
            for (int i = 0; i < 8; ++i) seen[i] = static_cast<typename P::one>(bits >> (16 * x + 8 * (i / 4) + i % 4) & 1u ? 1.0f : 0.0f);
            sums = wide_product<P>(v, seen, sums);
          }
#pragma unroll
          for (int i = 0; i < 16; ++i) {
              const uint32_t which = static_cast<uint32_t>(sums[i]);
              const bool up = which & 0x7fu, down = which >> 7 & 0x7fu, none = which >> 14;
              if (which) o[n][i] += none || (up && down) ? __builtin_nanf("") : up ? __builtin_inff() : -__builtin_inff();
            }
        }
      }
    }
    if (more) put(v_of(tile + 1), raw_v, Fp16{});
    if (more_keys) put(k_of(tile + 2), raw_k, T{});
    now = next;
    next = second;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
  }
  if (skipped && lane == 0) report(a.status, TUTTI_ST_BAD_BLOCK);
  // LDS changes hands behind the last turn's barrier: from here each wavefront has a part of it
  const auto &z = arguments_again<AttendArgs>();

  {
    const float sum = sum_of_halves(l);
    const uint32_t row_in = wave * 32 + r, row = row_a + row_in;
    if (u.parts > 1) {
      if (row < n_rows) {
        const uint64_t at = static_cast<uint64_t>(u.part_slot + u.part) * ROWS + row_in;
#pragma unroll
        for (int n = 0; n < DT; ++n)
#pragma unroll
          for (int i = 0; i < 16; i += 4)
            *reinterpret_cast<f32x4 *>(z.part_o + at * DP + 32 * n + 2 * i + 4 * hf) =
                f32x4{o[n][i], o[n][i + 1], o[n][i + 2], o[n][i + 3]};
        if (hf == 0) z.part_ml[at] = f32x2{m, sum};
      }
      return;
    }
    // through LDS, so that whole rows are stored
    constexpr uint32_t OUT_BYTES = ROW_BYTES + 16;
    TUTTI_LDS uint8_t *const mine = base + wave * 32 * OUT_BYTES;
    const float by = sum > 0.0f || sum != sum ? 1.0f / sum : 0.0f;
#pragma unroll
    for (int n = 0; n < DT; ++n)
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        typename T::two two[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          two[x][0] = rounded<T>(o[n][i + 2 * x] * by, !E4M3);
          two[x][1] = rounded<T>(o[n][i + 2 * x + 1] * by, !E4M3);
        }
        *(TUTTI_LDS u32x2 *)(mine + r * OUT_BYTES + (32 * n + 2 * i + 4 * hf) * 2) =
            u32x2{__builtin_bit_cast(uint32_t, two[0]), __builtin_bit_cast(uint32_t, two[1])};
      }
    if (row < n_rows && hf == 0 && z.lse) {
      const uint32_t i = row / z.group, head = u.head * z.group + row - i * z.group;
      z.lse[static_cast<uint64_t>(s.row0 + i) * (z.kv_heads * z.group) + head] =
          sum == 0.0f ? -__builtin_inff() : (m + __builtin_amdgcn_logf(sum)) * kLn2;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    for (uint32_t x = lane; x < 32 * UNITS; x += kLanes) {
      const uint32_t in = x / UNITS, unit = x % UNITS, out_row = wave_a + in;
      if (out_row >= n_rows || unit * 8 >= d) continue;
      const uint32_t i = out_row / z.group, head = u.head * z.group + out_row - i * z.group;
      *reinterpret_cast<u32x4 *>(static_cast<uint8_t *>(z.out.base) + static_cast<uint64_t>(s.row0 + i) * z.out.row_stride +
                                 head * z.out.head_stride + unit * 16) = *(TUTTI_LDS u32x4 *)(mine + in * OUT_BYTES + unit * 16);
    }
  }
}

// ---- Joins the parts of sequences that were split: one workgroup (WAVES 4) or one wavefront (1) a row.  DP/4 threads take a
// part, four values each; so many parts go abreast, and four times that many are under way at once.  Bound by its trips to memory:
// records and plan, maxima, sums; 4.4 us for 4 parts, 6.7 for 128.
template <typename T, int DP, int ROWS, int WAVES>
__global__ __launch_bounds__(256) void k_kv_join(const AttendArgs a) {
  constexpr uint32_t TP = DP / 4, ABREAST = WAVES * kLanes / TP, U = 4;
  const uint32_t lane = threadIdx.x & (kLanes - 1), wave = threadIdx.x / kLanes;
  const uint32_t thread = WAVES == 1 ? lane : threadIdx.x;   // among those of the row
  Plan plan{*a.tiles_a_part, {}};
  if (lane < a.batch.n_seq) plan.lane_seq = load_seq(a.batch.seqs + lane);
  // items: rows of the sequences that are split
  for (uint32_t item = WAVES == 1 ? blockIdx.x * 4 + uniform(wave) : blockIdx.x;; item += gridDim.x * (WAVES == 1 ? 4 : 1)) {
    uint32_t before = 0, slots = 0, units = 0;
    bool found = false;
    uint32_t row0 = 0, parts = 0, local = 0, first_slot = 0, units_upto_it = 0;
    for (uint32_t base = 0; base < a.batch.n_seq && !found; base += kLanes) {
      tutti_seq s{};
      uint32_t n = 0, split = 0, p = 0, all = 0;
      if (base + lane < a.batch.n_seq) {
        s = record(a, plan, base, lane);
        if (seq_ok(a.batch, s) && s.n_new) {
          p = parts_of(a, plan, s);
          all = row_tiles<ROWS>(a, s) * (a.kv_heads / a.abreast) * p;
          if (p > 1) {
            n = s.n_new * a.group * a.kv_heads;
            split = row_tiles<ROWS>(a, s) * a.kv_heads * p;
          }
        }
      }
      const uint32_t upto = before + lane_prefix_sum(n), split_upto = slots + lane_prefix_sum(split);
      const uint32_t units_upto = units + lane_prefix_sum(all);
      const uint64_t behind = __ballot(n != 0 && upto > item);
      if (behind) {
        const uint32_t l = static_cast<uint32_t>(__builtin_ctzll(behind));
        found = true;
        local = item - (from_lane(upto, l) - from_lane(n, l));
        row0 = from_lane(s.row0, l);
        parts = from_lane(p, l);
        first_slot = from_lane(split_upto, l) - from_lane(split, l);
        units_upto_it = from_lane(units_upto, l);
      }
      before = from_lane(upto, kLanes - 1);
      slots = from_lane(split_upto, kLanes - 1);
      units = from_lane(units_upto, kLanes - 1);
    }
    if (!found) return;
    const uint32_t heads = a.group * a.kv_heads, i = local / heads, head = local - i * heads;
    const uint32_t kv = head / a.group, row = i * a.group + head - kv * a.group;
    const uint32_t slot = first_slot + (row / ROWS * a.kv_heads + kv) * parts;
    // what the attention kernel did not do, a workgroup's heads together, is not joined
    if (first_slot + (row / ROWS * a.kv_heads + (kv / a.abreast + 1) * a.abreast) * parts > a.max_parts || units_upto_it > a.max_units)
      continue;
    const uint64_t at0 = static_cast<uint64_t>(slot) * ROWS + row % ROWS;

    float top = kLowest;
    for (uint32_t p = thread; p < parts; p += WAVES * kLanes) top = fmaxf(top, a.part_ml[at0 + static_cast<uint64_t>(p) * ROWS][0]);
#pragma unroll
    for (int x = 1; x < 16; x <<= 1) top = fmaxf(top, __shfl_xor(top, x, kLanes));
    top = max_over_rows(top);
    __shared__ float tops[4], sums[4 * kLanes / TP];
    __shared__ __attribute__((aligned(16))) float half[4 * kLanes / TP][DP];
    if constexpr (WAVES != 1) {
      if (lane == 0) tops[wave] = top;
      __syncthreads();
#pragma unroll
      for (int x = 0; x < WAVES; ++x) top = fmaxf(top, tops[x]);
    }
    const uint32_t e = thread % TP * 4, mine = thread / TP;
    float sum = 0.0f;
    f32x4 y = {0, 0, 0, 0};
    if (e < a.d) {
      for (uint32_t p0 = mine; p0 < parts; p0 += U * ABREAST) {
        f32x2 ml[U];
        f32x4 o[U];
#pragma unroll
        for (uint32_t u = 0; u < U; ++u)
          if (p0 + u * ABREAST < parts) {
            const uint64_t at = at0 + static_cast<uint64_t>(p0 + u * ABREAST) * ROWS;
            ml[u] = a.part_ml[at];
            o[u] = *reinterpret_cast<const f32x4 *>(a.part_o + at * DP + e);
          }
#pragma unroll
        for (uint32_t u = 0; u < U; ++u)
          if (p0 + u * ABREAST < parts) {
            const float by = __builtin_amdgcn_exp2f(ml[u][0] - top);
            sum += by * ml[u][1];
            y += by * o[u];
          }
      }
    }
    // the parts that went abreast: in LDS, a wavefront in its own rows of it
    const uint32_t first = WAVES == 1 ? uniform(wave) * ABREAST : 0;
    *reinterpret_cast<f32x4 *>(&half[first + mine][e]) = y;
    if (e == 0) sums[first + mine] = sum;
    if constexpr (WAVES != 1) {
      __syncthreads();
    } else {
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
    if (thread * 2 < a.d) {
      float total = 0.0f;
      f32x2 z = {0, 0};
#pragma unroll
      for (uint32_t w = 0; w < ABREAST; ++w) {
        total += sums[first + w];
        z += *reinterpret_cast<const f32x2 *>(&half[first + w][2 * thread]);
      }
      const float by = total > 0.0f || total != total ? 1.0f / total : 0.0f;
      uint8_t *to = static_cast<uint8_t *>(a.out.base) + static_cast<uint64_t>(row0 + i) * a.out.row_stride + head * a.out.head_stride;
      reinterpret_cast<typename T::two *>(to)[thread] =
          typename T::two{rounded<T>(z[0] * by, !a.pool.k_scale), rounded<T>(z[1] * by, !a.pool.k_scale)};
      if (thread == 0 && a.lse)
        a.lse[static_cast<uint64_t>(row0 + i) * heads + head] =
            total == 0.0f ? -__builtin_inff() : (top + __builtin_amdgcn_logf(total)) * kLn2;
    }
    if constexpr (WAVES != 1) {
      __syncthreads();  // LDS is the next row's
    } else {
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
  }
}

}  // namespace tutti
