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
  uint32_t heads_a_job;       // of one token, for jobs that go head by head
  uint32_t q_jobs, jobs;      // jobs of a unit: for its queries, in all
  uint32_t max_units;
  uint32_t *status;
};

// A lane's 8 values of a row, their partners in the rotation, and the angles of both.
struct Angles {
  float c[8], s[8];  // s with the sign that the partner's product takes
  bool rotated[8];
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

// A token's positions, one for each axis that is used.  false: one of them is not in the table.
__device__ __forceinline__ bool positions(const RopeView &r, uint32_t row, uint32_t place, uint32_t (&pos)[4]) {
  bool ok = true;
#pragma unroll
  for (int a = 0; a < 4; ++a) {
    pos[a] = 0;
    if (!(r.axes & (1u << a))) continue;
    pos[a] = r.pos ? r.pos[a * r.pos_stride + row] : place;
    ok &= pos[a] < r.n_pos;
  }
  return ok;
}

// Angles of values e0..e0+7 of a head.  Sections of 8 pairs that lie in one axis come as vectors.
__device__ __forceinline__ void load_angles(const RopeView &r, uint32_t e0, const uint32_t (&pos)[4], Angles &g) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    g.c[i] = 1.0f;
    g.s[i] = 0.0f;
    g.rotated[i] = e0 + i < r.rot;
  }
  if (e0 >= r.rot) return;
  const bool whole = (r.half & 7u) == 0;  // then rot is a multiple of 16, and a lane's values are all in one half or none
  if (whole && !r.interleaved) {
    const bool second = e0 >= r.half;
    const uint32_t j = second ? e0 - r.half : e0, ax = axis_of(r, j);
    if (ax == axis_of(r, j + 7)) {
      const float *at = r.cos_sin + static_cast<uint64_t>(pos[ax]) * r.rot + j;
      const f32x4 c0 = *reinterpret_cast<const f32x4 *>(at), c1 = *reinterpret_cast<const f32x4 *>(at + 4);
      const f32x4 s0 = *reinterpret_cast<const f32x4 *>(at + r.half), s1 = *reinterpret_cast<const f32x4 *>(at + r.half + 4);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        g.c[i] = c0[i];
        g.c[4 + i] = c1[i];
        g.s[i] = second ? s0[i] : -s0[i];
        g.s[4 + i] = second ? s1[i] : -s1[i];
      }
      return;
    }
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t e = e0 + i;
    if (e < r.rot) {
      const bool second = r.interleaved ? (e & 1u) : e >= r.half;
      const uint32_t j = r.interleaved ? e >> 1 : second ? e - r.half : e;
      const float *at = r.cos_sin + static_cast<uint64_t>(pos[axis_of(r, j)]) * r.rot + j;
      g.c[i] = at[0];
      g.s[i] = second ? at[r.half] : -at[r.half];
    }
  }
}

// Values e0..e0+7 of the head at `head`, rotated.  The partners of a lane's values are another lane's; they are read from memory
// (the same lines, a moment later).
template <typename T>
__device__ __forceinline__ void load_partners(const RopeView &r, const uint8_t *head, uint32_t e0, const float (&x)[8],
                                              float (&y)[8]) {
  using one = typename T::one;
  if (r.interleaved) {
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = x[i ^ 1];
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = 0.0f;
  if (e0 >= r.rot) return;
  if ((r.half & 7u) == 0) {
    const uint32_t p0 = e0 >= r.half ? e0 - r.half : e0 + r.half;
    unpack8<T>(*reinterpret_cast<const u32x4 *>(head + 2 * p0), y);
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t e = e0 + i;
    if (e < r.rot) {
      const uint32_t p = e >= r.half ? e - r.half : e + r.half;
      y[i] = static_cast<float>(reinterpret_cast<const one *>(head)[p]);
    }
  }
}

// a*c - b*s and b*c + a*s, three roundings each (a fused multiply-add would round twice, and the two forms of the operator, this
// one and the definition, would no longer be the same to the last bit, which decides how a value at the edge of two codes
// is rounded).
__device__ __forceinline__ void rotate8(const Angles &g, const float (&partner)[8], float (&x)[8]) {
#pragma clang fp contract(off)
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float a = x[i] * g.c[i], b = partner[i] * g.s[i];
    x[i] = g.rotated[i] ? a + b : x[i];
  }
}

// One token's slot in the pool: false if its block is not in the table.
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

// A job of whole rows: `heads` heads from `head0` on of tokens [i0, i0 + rows) of a sequence, LPR lanes a row.
// KIND 0: queries to q_out, 1: keys, 2: values to their 16-bit slots.
template <typename T, int LPR>
__device__ __forceinline__ void append_rows(const AppendArgs &a, const tutti_seq &s, uint32_t kind, uint32_t head0,
                                            uint32_t heads, uint32_t i0, uint32_t n_tokens) {
  const uint32_t lane = threadIdx.x & (kLanes - 1), e0 = (lane % LPR) * 8, sub = lane / LPR;
  const tutti_rows &src = kind == 0 ? a.q : kind == 1 ? a.k : a.v;
  for (uint32_t i = sub; i < n_tokens; i += kLanes / LPR) {
    const uint32_t row = s.row0 + i0 + i, place = s.n_held - s.n_new + i0 + i;
    bool live = e0 < a.d;
    uint8_t *to;
    uint64_t step;
    if (kind == 0) {
      to = static_cast<uint8_t *>(a.q_out.base) + row * a.q_out.row_stride;
      step = a.q_out.head_stride;
    } else {
      const Slot slot = slot_of(a, s, place);
      if (!slot.there && live && e0 == 0) report(a.status, TUTTI_ST_BAD_BLOCK);
      live &= slot.there;
      to = (kind == 1 ? a.pool.k : a.pool.v) + slot.block * a.pool.block_stride + slot.index * static_cast<uint64_t>(a.pool.token_stride);
      step = a.pool.head_stride;
    }
    Angles g;
    uint32_t pos[4];
    const bool turn = a.rope.rot != 0;
    if (turn) {
      const bool known = positions(a.rope, row, place, pos);
      if (!known && live && e0 == 0) report(a.status, TUTTI_ST_BAD_POS);
      live &= known;
      if (live && kind != 2) load_angles(a.rope, e0, pos, g);
    }
    if (!live) continue;
    const uint8_t *from = static_cast<const uint8_t *>(src.base) + row * src.row_stride + head0 * src.head_stride;
    to += head0 * step;
    const bool rotates = turn && kind != 2;
    // the loads of four heads are under way before the first is used (q_out may be q: a head is read, rotated and written by
    // the same lanes, and both halves of it are read before either is written)
    constexpr uint32_t U = 4;
    for (uint32_t h0 = 0; h0 < heads; h0 += U) {
      float x[U][8], y[U][8];
#pragma unroll
      for (uint32_t u = 0; u < U; ++u) {
        if (h0 + u < heads) {
          const uint8_t *head = from + (h0 + u) * src.head_stride;
          unpack8<T>(*reinterpret_cast<const u32x4 *>(head + 2 * e0), x[u]);
          if (rotates) load_partners<T>(a.rope, head, e0, x[u], y[u]);
        }
      }
#pragma unroll
      for (uint32_t u = 0; u < U; ++u) {
        if (h0 + u < heads) {
          if (rotates) rotate8(g, y[u], x[u]);
          *reinterpret_cast<u32x4 *>(to + (h0 + u) * step + 2 * e0) = pack8<T>(x[u]);
        }
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

// Values e0..e0+7 of one new token's key (rotated) or value.  false: the token is skipped.
template <typename T>
__device__ __forceinline__ bool new_values(const AppendArgs &a, bool key, uint32_t head, uint32_t row, uint32_t place, uint32_t e0,
                                           float (&x)[8]) {
  const tutti_rows &src = key ? a.k : a.v;
  const uint8_t *at = static_cast<const uint8_t *>(src.base) + row * src.row_stride + head * src.head_stride;
  unpack8<T>(*reinterpret_cast<const u32x4 *>(at + 2 * e0), x);
  if (a.rope.rot == 0) return true;
  uint32_t pos[4];
  if (!positions(a.rope, row, place, pos)) {
    if (e0 == 0) report(a.status, TUTTI_ST_BAD_POS);
    return false;
  }
  if (!key) return true;
  Angles g;
  float y[8];
  load_angles(a.rope, e0, pos, g);
  load_partners<T>(a.rope, at, e0, x, y);
  rotate8(g, y, x);
  return true;
}

// One block's new tokens in one head of one plane, e4m3: tokens [i0, i0 + n) of the sequence, of which the first goes to slot
// `slot0`.  One wavefront: the largest magnitude, the scale, the codes.  The values of the first KEPT passes over the rows stay in
// registers between the two; a block with more new tokens (T > 16 or 32) has the rest read and rotated again.
template <typename T, int LPR>
__device__ __forceinline__ void append_e4m3(const AppendArgs &a, const tutti_seq &s, bool key, uint32_t head, uint32_t i0,
                                            uint32_t n, const Slot &slot) {
  constexpr uint32_t ROWS = kLanes / LPR, KEPT = 4;
  const uint32_t lane = threadIdx.x & (kLanes - 1), e0 = (lane % LPR) * 8, sub = lane / LPR;
  const uint32_t first = s.n_held - s.n_new + i0;  // place of the first new token
  const bool live = e0 < a.d;
  float kept[KEPT][8];
  bool have[KEPT];
  float top = 0.0f;
#pragma unroll
  for (uint32_t u = 0; u < KEPT; ++u) {
    const uint32_t i = u * ROWS + sub;
    have[u] = live && i < n;
    if (have[u]) have[u] = new_values<T>(a, key, head, s.row0 + i0 + i, first + i, e0, kept[u]);
    if (have[u])
#pragma unroll
      for (int j = 0; j < 8; ++j) top = fmaxf(top, finite_magnitude(kept[u][j]));
  }
  for (uint32_t i = KEPT * ROWS + sub; i < n; i += ROWS) {
    float x[8];
    if (live && new_values<T>(a, key, head, s.row0 + i0 + i, first + i, e0, x))
#pragma unroll
      for (int j = 0; j < 8; ++j) top = fmaxf(top, finite_magnitude(x[j]));
  }
#pragma unroll
  for (int m = 1; m < static_cast<int>(kLanes); m <<= 1) top = fmaxf(top, __shfl_xor(top, m, kLanes));
  float *scale_at = (key ? a.pool.k_scale : a.pool.v_scale) + slot.block * a.pool.scale_stride + head;
  uint8_t *to = (key ? a.pool.k : a.pool.v) + slot.block * a.pool.block_stride + head * static_cast<uint64_t>(a.pool.head_stride);
  int e = scale_exponent(top);
  float scale = power_of_two(e);
  if (slot.index != 0) {  // older tokens
    const float had = *scale_at;
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
  for (uint32_t i = KEPT * ROWS + sub; i < n; i += ROWS) {
    float x[8];
    if (live && new_values<T>(a, key, head, s.row0 + i0 + i, first + i, e0, x))
      *reinterpret_cast<u32x2 *>(to + (slot.index + i) * static_cast<uint64_t>(a.pool.token_stride) + e0) = to_e4m3(x, by);
  }
}

// One wavefront, one job.  A unit is some tokens of one sequence: for 16-bit pools as many as a wavefront has rows of lanes, for
// e4m3 pools those that go to one block.  Its jobs: queries, `heads_a_job` heads each, then keys and values, 16-bit as the
// queries, e4m3 one KV head and plane each.
template <typename T, bool E4M3, int LPR>
__global__ __launch_bounds__(256) void k_kv_append(const AppendArgs a) {
  const uint32_t job = blockIdx.x * 4u + uniform(threadIdx.x / kLanes);
  const uint32_t unit = job / a.jobs, part = job - unit * a.jobs;
  if (unit >= a.max_units) return;
  const uint32_t T_ = a.pool.block_tokens;
  constexpr uint32_t ROWS = kLanes / LPR;
  const bool first = job == 0;
  const Found f = find_unit(a.batch, unit, first, a.status, [&](const tutti_seq &s) -> uint32_t {
    if (s.n_new == 0) return 0;
    if (!E4M3) return (s.n_new + ROWS - 1) / ROWS;
    return block_of(a.pool, s.n_held - 1) - block_of(a.pool, s.n_held - s.n_new) + 1;
  });
  if (first && f.total > a.max_units && (threadIdx.x & (kLanes - 1)) == 0) report(a.status, TUTTI_ST_BAD_EXTENT);
  if (f.seq == a.batch.n_seq) return;
  uint32_t i0, n;
  Slot slot{};
  if (E4M3) {
    const uint32_t begin = f.s.n_held - f.s.n_new, block = block_of(a.pool, begin) + f.local;
    const uint32_t from = block * T_ > begin ? block * T_ : begin;
    const uint32_t to = f.s.n_held - block * T_ < T_ ? f.s.n_held : block * T_ + T_;
    i0 = from - begin;
    n = to - from;
    if (part >= a.q_jobs) {
      slot = slot_of(a, f.s, from);
      if (!slot.there) {
        if ((threadIdx.x & (kLanes - 1)) == 0) report(a.status, TUTTI_ST_BAD_BLOCK);
        return;
      }
    }
  } else {
    i0 = f.local * ROWS;
    n = f.s.n_new - i0 < ROWS ? f.s.n_new - i0 : ROWS;
  }
  if (part < a.q_jobs) {
    const uint32_t h0 = part * a.heads_a_job;
    append_rows<T, LPR>(a, f.s, 0, h0, a.q_heads - h0 < a.heads_a_job ? a.q_heads - h0 : a.heads_a_job, i0, n);
    return;
  }
  const uint32_t kv_jobs = (a.jobs - a.q_jobs) / 2, p = part - a.q_jobs;
  const bool key = p < kv_jobs;
  const uint32_t c = key ? p : p - kv_jobs;
  if (E4M3) {
    append_e4m3<T, LPR>(a, f.s, key, c, i0, n, slot);
  } else {
    const uint32_t h0 = c * a.heads_a_job;
    append_rows<T, LPR>(a, f.s, key ? 1 : 2, h0, a.kv_heads - h0 < a.heads_a_job ? a.kv_heads - h0 : a.heads_a_job, i0, n);
  }
}

}  // namespace tutti
