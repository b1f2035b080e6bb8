// Appending to a paged cache: rotation of queries and keys, 16-bit or e4m3 blocks.
#pragma once
#include "kv_common.hip.h"

namespace tutti {

struct RopeView {
  const float *cos_sin;
  const uint32_t *pos;
  uint64_t pos_stride;
  uint32_t n_pos, rot, half;  // rot 0: nothing is rotated
  uint32_t interleaved;
  uint32_t end[3];            // first pair behind axis 0, 1, 2
  uint32_t axes;              // axes that have pairs: bit a
};

struct AppendArgs {
  PoolView pool;
  BatchView batch;
  RopeView rope;
  tutti_rows q, q_out, k, v;
  uint32_t q_heads, kv_heads, d;
  uint32_t heads_a_job;       // for jobs that go head by head
  uint32_t q_jobs, jobs;      // jobs of a unit: for its queries, in all
  uint32_t max_units;
  uint32_t *status;
};

// How a lane's 8 values of a row and their partners lie.
enum Turn : int {
  kNoTurn = 0,
  kHalves = 1,  // partners rot/2 values apart; rot/2 and the axes' sections are multiples of 8: whole vectors
  kPairs = 2,   // partners side by side; rot/2 and the sections are multiples of 4
  kAnyTurn = 3  // whatever else
};

template <typename T>
__device__ __forceinline__ void unpack8(u32x4 w, float (&x)[8]) {
  const typename T::eight v = __builtin_bit_cast(typename T::eight, w);
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = static_cast<float>(v[i]);
}
template <typename T>
__device__ __forceinline__ u32x4 pack8(const float (&x)[8]) {
  typename T::eight v;
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = static_cast<typename T::one>(x[i]);
  return __builtin_bit_cast(u32x4, v);
}

__device__ __forceinline__ uint32_t axis_of(const RopeView &r, uint32_t pair) {
  return (pair >= r.end[0]) + (pair >= r.end[1]) + (pair >= r.end[2]);
}

// Whether all of a token's positions are in the table of angles.
__device__ __forceinline__ bool positions_known(const RopeView &r, uint32_t row, uint32_t place) {
  if (!r.pos) return place < r.n_pos;
  bool ok = true;
#pragma unroll
  for (int a = 0; a < 4; ++a)
    if (r.axes & (1u << a)) ok &= r.pos[a * r.pos_stride + row] < r.n_pos;
  return ok;
}

// The angles of a lane's values e0..e0+7: kHalves c[8] and s[8], s with the sign that the partner's product takes; kPairs four
// pairs' c and s; kAnyTurn like kHalves, value by value.
template <int TURN>
struct Angles {
  float c[TURN == kPairs ? 4 : 8], s[TURN == kPairs ? 4 : 8];
};

// Angles of a token that positions_known() has let pass, for e0 < rot.
template <int TURN>
__device__ __forceinline__ void load_angles(const RopeView &r, uint32_t e0, uint32_t row, uint32_t place, Angles<TURN> &g) {
  if constexpr (TURN == kHalves || TURN == kPairs) {
    const bool second = TURN == kHalves && e0 >= r.half;
    const uint32_t j = TURN == kPairs ? e0 / 2 : second ? e0 - r.half : e0;
    const uint32_t pos = r.pos ? r.pos[axis_of(r, j) * r.pos_stride + row] : place;
    const float *at = r.cos_sin + static_cast<uint64_t>(pos) * r.rot + j;
#pragma unroll
    for (int i = 0; i < (TURN == kPairs ? 4 : 8); i += 4) {
      const f32x4 c = *reinterpret_cast<const f32x4 *>(at + i), s = *reinterpret_cast<const f32x4 *>(at + r.half + i);
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        g.c[i + x] = c[x];
        g.s[i + x] = TURN == kPairs || second ? s[x] : -s[x];
      }
    }
  } else if constexpr (TURN == kAnyTurn) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t e = e0 + i;
      g.c[i] = 1.0f;
      g.s[i] = 0.0f;
      if (e < r.rot) {
        const bool second = r.interleaved ? (e & 1u) : e >= r.half;
        const uint32_t j = r.interleaved ? e >> 1 : second ? e - r.half : e;
        const uint32_t pos = r.pos ? r.pos[axis_of(r, j) * r.pos_stride + row] : place;
        const float *at = r.cos_sin + static_cast<uint64_t>(pos) * r.rot + j;
        g.c[i] = at[0];
        g.s[i] = second ? at[r.half] : -at[r.half];
      }
    }
  }
}

// What a lane loads of a head for its 8 values: the values and, where they are another lane's, their partners (from memory: the
// same lines, a moment later).
template <int TURN>
struct Raw {
  u32x4 own, partner;
};
template <typename T, int TURN>
__device__ __forceinline__ void load_raw(const RopeView &r, const uint8_t *head, uint32_t e0, Raw<TURN> &w) {
  w.own = *reinterpret_cast<const u32x4 *>(head + 2 * e0);
  if constexpr (TURN == kHalves) {
    const uint32_t p0 = e0 >= r.rot ? e0 : e0 >= r.half ? e0 - r.half : e0 + r.half;
    w.partner = *reinterpret_cast<const u32x4 *>(head + 2 * p0);
  } else if constexpr (TURN == kAnyTurn) {
    typename T::eight p = {};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t e = e0 + i;
      if (e < r.rot) {
        const uint32_t from = r.interleaved ? e ^ 1u : e >= r.half ? e - r.half : e + r.half;
        p[i] = reinterpret_cast<const typename T::one *>(head)[from];
      }
    }
    w.partner = __builtin_bit_cast(u32x4, p);
  }
}

// a*c - b*s and b*c + a*s, three roundings each.  (A fused multiply-add would round twice; then this and the definition would
// not be the same to the last bit, which decides how a value at the edge between two codes is rounded.)
template <typename T, int TURN>
__device__ __forceinline__ void turned(const RopeView &r, const Raw<TURN> &w, const Angles<TURN> &g, uint32_t e0, float (&x)[8]) {
#pragma clang fp contract(off)
  unpack8<T>(w.own, x);
  if constexpr (TURN == kPairs) {
    if (e0 >= r.rot) return;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float a = x[2 * i], b = x[2 * i + 1];
      const float ac = a * g.c[i], bs = b * g.s[i], bc = b * g.c[i], as = a * g.s[i];
      x[2 * i] = ac - bs;
      x[2 * i + 1] = bc + as;
    }
  } else if constexpr (TURN != kNoTurn) {
    float y[8];
    unpack8<T>(w.partner, y);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float own = x[i] * g.c[i], other = y[i] * g.s[i];
      const bool in = e0 + (TURN == kHalves ? 0 : i) < r.rot;
      x[i] = in ? own + other : x[i];
    }
  }
}

// One token's slot in the pool; there: its block is in the table.
struct Slot {
  uint32_t block, index;
  bool there;
};
__device__ __forceinline__ Slot slot_of(const AppendArgs &a, const tutti_seq &s, uint32_t place) {
  Slot r{0, 0, false};
  const uint32_t n = block_of(a.pool, place);
  r.index = place - n * a.pool.block_tokens;
  const uint64_t at = static_cast<uint64_t>(s.table_off) + n;
  if (at < a.batch.table_len) {
    r.block = a.batch.table[at];
    r.there = r.block < a.pool.num_blocks;
  }
  return r;
}

// A job of whole rows: `heads` heads from `head0` on of tokens [i0, i0 + n) of a sequence, LPR lanes a row.  The wavefront's
// rows of lanes take tokens, or where there are fewer tokens than that, heads of one token.
// KIND 0: queries to q_out, 1: keys, 2: values to their 16-bit slots.
template <typename T, int LPR, int TURN, int KIND>
__device__ __forceinline__ void append_rows(const AppendArgs &a, const tutti_seq &s, uint32_t head0, uint32_t heads, uint32_t i0,
                                            uint32_t n) {
  constexpr uint32_t ROWS = kLanes / LPR, U = 4;
  constexpr int TURNS = KIND == 2 ? static_cast<int>(kNoTurn) : TURN;
  const uint32_t lane = threadIdx.x & (kLanes - 1), e0 = (lane % LPR) * 8, sub = lane / LPR;
  const tutti_rows &src = KIND == 0 ? a.q : KIND == 1 ? a.k : a.v;
  const uint32_t side = n == 1 ? 1 : n == 2 ? 2 : ROWS;             // tokens side by side
  const uint32_t step = ROWS / side, h_first = sub / side;          // heads side by side
  for (uint32_t i = sub % side; i < n; i += side) {
    const uint32_t row = s.row0 + i0 + i, place = s.n_held - s.n_new + i0 + i;
    bool live = e0 < a.d;
    uint8_t *to;
    uint64_t head_step;
    if constexpr (KIND == 0) {
      to = static_cast<uint8_t *>(a.q_out.base) + row * a.q_out.row_stride;
      head_step = a.q_out.head_stride;
    } else {
      const Slot slot = slot_of(a, s, place);
      if (!slot.there && e0 == 0) report(a.status, TUTTI_ST_BAD_BLOCK);
      live &= slot.there;
      to = (KIND == 1 ? a.pool.k : a.pool.v) + slot.block * a.pool.block_stride +
           slot.index * static_cast<uint64_t>(a.pool.token_stride);
      head_step = a.pool.head_stride;
    }
    if constexpr (TURN != kNoTurn) {
      const bool known = positions_known(a.rope, row, place);
      if (!known && e0 == 0) report(a.status, TUTTI_ST_BAD_POS);
      live &= known;
    }
    if (!live) continue;
    const uint8_t *from = static_cast<const uint8_t *>(src.base) + row * src.row_stride;
    Angles<TURNS> g;
    // the loads of up to four heads are under way before the first is used (q_out may be q: a head is read and written by the
    // same lanes, and all of it is read before any of it is written)
    for (uint32_t h0 = h_first; h0 < heads; h0 += U * step) {
      Raw<TURNS> w[U];
#pragma unroll
      for (uint32_t u = 0; u < U; ++u)
        if (h0 + u * step < heads) load_raw<T, TURNS>(a.rope, from + (head0 + h0 + u * step) * src.head_stride, e0, w[u]);
      if (TURNS != kNoTurn && h0 == h_first && e0 < a.rope.rot) load_angles<TURNS>(a.rope, e0, row, place, g);
#pragma unroll
      for (uint32_t u = 0; u < U; ++u)
        if (h0 + u * step < heads) {
          float x[8];
          turned<T, TURNS>(a.rope, w[u], g, e0, x);
          *reinterpret_cast<u32x4 *>(to + (head0 + h0 + u * step) * head_step + 2 * e0) = pack8<T>(x);
        }
    }
  }
}

__device__ __forceinline__ float finite_magnitude(float x) {
  const float m = fabsf(x);
  return m < __builtin_inff() ? m : 0.0f;
}

// Exponent of the smallest power of two s with m <= 448 s, at least -64: m = f 2^e with f in [0.5, 1) and 448 = 0.875 * 2^9.
__device__ __forceinline__ int scale_exponent(float m) {
  const uint32_t bits = __float_as_uint(m);
  const int e = static_cast<int>(bits >> 23) - 126 - 9 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0);
  return e < -64 ? -64 : e;
}
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float(static_cast<uint32_t>(e + 127) << 23); }

__device__ __forceinline__ float within_e4m3(float x) { return x > 448.0f ? 448.0f : x < -448.0f ? -448.0f : x; }

__device__ __forceinline__ u32x2 to_e4m3(const float (&x)[8], float by) {
  u32x2 w;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    int r = __builtin_amdgcn_cvt_pk_fp8_f32(within_e4m3(x[4 * i] * by), within_e4m3(x[4 * i + 1] * by), 0, false);
    r = __builtin_amdgcn_cvt_pk_fp8_f32(within_e4m3(x[4 * i + 2] * by), within_e4m3(x[4 * i + 3] * by), r, true);
    w[i] = static_cast<uint32_t>(r);
  }
  return w;
}
__device__ __forceinline__ void from_e4m3(u32x2 w, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(w[i]), false);
    const f32x2 hi = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(w[i]), true);
    x[4 * i] = lo[0];
    x[4 * i + 1] = lo[1];
    x[4 * i + 2] = hi[0];
    x[4 * i + 3] = hi[1];
  }
}

// One block's new tokens in one head of one plane, e4m3: tokens [i0, i0 + n) of the sequence, of which the first goes to slot
// `slot.index`.  One wavefront: the largest magnitude, the scale, the codes.  The values of the first KEPT passes over the rows
// stay in registers between the two; a block with more new tokens (T > 16, or > 32 of up to 64 values) has the rest read and
// rotated again.
template <typename T, int LPR, int TURN, bool KEY>
__device__ __forceinline__ void append_e4m3(const AppendArgs &a, const tutti_seq &s, uint32_t head, uint32_t i0, uint32_t n,
                                            const Slot &slot) {
  constexpr uint32_t ROWS = kLanes / LPR, KEPT = 4;
  constexpr int TURNS = KEY ? TURN : static_cast<int>(kNoTurn);
  const uint32_t lane = threadIdx.x & (kLanes - 1), e0 = (lane % LPR) * 8, sub = lane / LPR;
  const uint32_t first = s.n_held - s.n_new + i0;  // place of the first new token
  const bool live = e0 < a.d;
  float *scale_at = (KEY ? a.pool.k_scale : a.pool.v_scale) + slot.block * a.pool.scale_stride + head;
  uint8_t *to = (KEY ? a.pool.k : a.pool.v) + slot.block * a.pool.block_stride + head * static_cast<uint64_t>(a.pool.head_stride);
  float had = 0.0f;
  if (slot.index != 0) had = *scale_at;  // older tokens
  const tutti_rows &src = KEY ? a.k : a.v;
  const uint8_t *from = static_cast<const uint8_t *>(src.base) + head * src.head_stride;

  // one token's values; false: it is skipped
  const auto known = [&](uint32_t i) {
    if constexpr (TURN == kNoTurn) return true;
    if (positions_known(a.rope, s.row0 + i0 + i, first + i)) return true;
    if (e0 == 0) report(a.status, TUTTI_ST_BAD_POS);
    return false;
  };
  const auto values = [&](uint32_t i, const Raw<TURNS> &w, float (&x)[8]) {
    Angles<TURNS> g;
    if (TURNS != kNoTurn && e0 < a.rope.rot) load_angles<TURNS>(a.rope, e0, s.row0 + i0 + i, first + i, g);
    turned<T, TURNS>(a.rope, w, g, e0, x);
  };
  Raw<TURNS> raw[KEPT];
  bool have[KEPT];
#pragma unroll
  for (uint32_t u = 0; u < KEPT; ++u) {
    const uint32_t i = u * ROWS + sub;
    have[u] = live && i < n;
    if (have[u]) load_raw<T, TURNS>(a.rope, from + (s.row0 + i0 + i) * src.row_stride, e0, raw[u]);
  }
  float kept[KEPT][8];
  float top = 0.0f;
#pragma unroll
  for (uint32_t u = 0; u < KEPT; ++u) {
    const uint32_t i = u * ROWS + sub;
    if (have[u]) have[u] = known(i);
    if (have[u]) {
      values(i, raw[u], kept[u]);
#pragma unroll
      for (int j = 0; j < 8; ++j) top = fmaxf(top, finite_magnitude(kept[u][j]));
    }
  }
  const auto rest = [&](auto &&use) {
    for (uint32_t i = KEPT * ROWS + sub; i < n; i += ROWS) {
      if (!live || !known(i)) continue;
      Raw<TURNS> w;
      float x[8];
      load_raw<T, TURNS>(a.rope, from + (s.row0 + i0 + i) * src.row_stride, e0, w);
      values(i, w, x);
      use(i, x);
    }
  };
  rest([&](uint32_t, const float (&x)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) top = fmaxf(top, finite_magnitude(x[j]));
  });
#pragma unroll
  for (int m = 1; m < 16; m <<= 1) top = fmaxf(top, __shfl_xor(top, m, kLanes));
  top = max_over_rows(top);
  float scale = power_of_two(scale_exponent(top));
  if (slot.index != 0) {
    if (had >= scale) {
      scale = had;
    } else if (live) {
      const float by = 1.0f / scale;  // a power of two: exact
      for (uint32_t i = sub; i < slot.index; i += ROWS) {
        u32x2 *code = reinterpret_cast<u32x2 *>(to + i * static_cast<uint64_t>(a.pool.token_stride) + e0);
        float x[8];
        from_e4m3(*code, x);
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] *= had;
        *code = to_e4m3(x, by);
      }
    }
  }
  const float by = 1.0f / scale;
  if (lane == 0) *scale_at = scale;
#pragma unroll
  for (uint32_t u = 0; u < KEPT; ++u)
    if (have[u])
      *reinterpret_cast<u32x2 *>(to + (slot.index + u * ROWS + sub) * static_cast<uint64_t>(a.pool.token_stride) + e0) =
          to_e4m3(kept[u], by);
  rest([&](uint32_t i, const float (&x)[8]) {
    *reinterpret_cast<u32x2 *>(to + (slot.index + i) * static_cast<uint64_t>(a.pool.token_stride) + e0) = to_e4m3(x, by);
  });
}

// Bound by memory, and by the launch below a megabyte: one token of 40 heads x 128 3.3 to 4.1 us; 256 sequences' tokens to e4m3 blocks 6.3
// us (2.2 a launch, then four trips: record, table, angles and values, scale); 8,191 tokens to e4m3 blocks (189 MB) 46 us, 4.1 TB/s;
// 16,384 tokens with three axes to 16-bit blocks (411 MB) 82 us, 5.0 TB/s (a large copy: 5.1 to 6.15).  Each kind of rotation has
// kernels of its own: the general one needs 156 registers, which in every kernel made the first two cases 6.9 and 40 us.  By kind, those
// 16,384 tokens: halves 83 us, pairs 77; with heads of 80 (floor 42 us) halves 63, pairs 55, 40 of 80 values rotated (value by value) 189.
//
// One wavefront, one job.  A unit is some tokens of one sequence: for 16-bit pools as many as a wavefront has rows of lanes, for
// e4m3 pools those that go to one block.  Its jobs: queries, `heads_a_job` heads each, then keys and values, 16-bit as the
// queries, e4m3 one KV head and plane each.  Where no sequence has more than one new token, unit u is sequence u.
template <typename T, bool E4M3, int LPR, int TURN>
__global__ __launch_bounds__(256) void k_kv_append(const AppendArgs a) {
  const uint32_t job = blockIdx.x * 4u + uniform(threadIdx.x / kLanes);
  const uint32_t unit = job / a.jobs, part = job - unit * a.jobs;
  if (unit >= a.max_units) return;
  const uint32_t lane = threadIdx.x & (kLanes - 1);
  constexpr uint32_t ROWS = kLanes / LPR;
  tutti_seq s;
  uint32_t local = 0;
  if (a.batch.max_new == 1) {
    s = uniform_seq(a.batch.seqs + unit);
    if (!seq_ok(a.batch, s)) {
      if (part == 0 && lane == 0) report(a.status, TUTTI_ST_BAD_EXTENT);
      return;
    }
    if (s.n_new == 0) return;
  } else {
    const bool first = job == 0;
    const Found f = find_unit(a.batch, unit, first, a.status, [&](const tutti_seq &q) -> uint32_t {
      if (q.n_new == 0) return 0;
      if (!E4M3) return (q.n_new + ROWS - 1) / ROWS;
      return block_of(a.pool, q.n_held - 1) - block_of(a.pool, q.n_held - q.n_new) + 1;
    });
    if (first && f.total > a.max_units && lane == 0) report(a.status, TUTTI_ST_BAD_EXTENT);
    if (f.seq == a.batch.n_seq) return;
    s = f.s;
    local = f.local;
  }
  uint32_t i0, n;
  Slot slot{};
  if constexpr (E4M3) {
    const uint32_t block_tokens = a.pool.block_tokens, begin = s.n_held - s.n_new, block = block_of(a.pool, begin) + local;
    const uint32_t from = block * block_tokens > begin ? block * block_tokens : begin;
    const uint32_t to = s.n_held - block * block_tokens < block_tokens ? s.n_held : block * block_tokens + block_tokens;
    i0 = from - begin;
    n = to - from;
    if (part >= a.q_jobs) {
      slot = slot_of(a, s, from);
      if (!slot.there) {
        if (lane == 0) report(a.status, TUTTI_ST_BAD_BLOCK);
        return;
      }
    }
  } else {
    i0 = local * ROWS;
    n = s.n_new - i0 < ROWS ? s.n_new - i0 : ROWS;
  }
  const auto heads_from = [&](uint32_t h0, uint32_t all) { return all - h0 < a.heads_a_job ? all - h0 : a.heads_a_job; };
  if (part < a.q_jobs) {
    const uint32_t h0 = part * a.heads_a_job;
    append_rows<T, LPR, TURN, 0>(a, s, h0, heads_from(h0, a.q_heads), i0, n);
    return;
  }
  const uint32_t kv_jobs = (a.jobs - a.q_jobs) / 2, p = part - a.q_jobs;
  const bool key = p < kv_jobs;
  const uint32_t c = key ? p : p - kv_jobs;
  if constexpr (E4M3) {
    if (key)
      append_e4m3<T, LPR, TURN, true>(a, s, c, i0, n, slot);
    else
      append_e4m3<T, LPR, TURN, false>(a, s, c, i0, n, slot);
  } else {
    const uint32_t h0 = c * a.heads_a_job, heads = heads_from(h0, a.kv_heads);
    if (key)
      append_rows<T, LPR, TURN, 1>(a, s, h0, heads, i0, n);
    else
      append_rows<T, LPR, TURN, 2>(a, s, h0, heads, i0, n);
  }
}

}  // namespace tutti
