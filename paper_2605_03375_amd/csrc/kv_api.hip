// Host side of the calls that use a paged cache in place: tutti_kv_append, tutti_kv_attend.  As everywhere in the library a call
// checks its host arguments in O(1), enqueues a constant number of kernels on the caller's stream and returns.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "kv_append.hip.h"
#include "kv_attend.hip.h"
#include "library_state.h"
#include "tutti.h"

namespace {

using namespace tutti;

bool aligned(const void *p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

// What of a call's arguments goes by sizes and types alone: the pool's, a batch's.
int check_shape(const tutti_pool *pool, uint32_t dtype) {
  if (!pool) return TUTTI_EINVAL;
  if (dtype != TUTTI_BF16 && dtype != TUTTI_FP16) return TUTTI_EINVAL;
  if (pool->elt_bytes != 1 && pool->elt_bytes != 2) return TUTTI_EINVAL;
  if (pool->head_dim == 0 || pool->head_dim % 16 != 0 || pool->head_dim > 128) return TUTTI_EINVAL;
  if (pool->num_blocks == 0 || pool->block_tokens == 0 || pool->num_kv_heads == 0) return TUTTI_EINVAL;
  if (pool->pool_layout != TUTTI_LAYOUT_NHD && pool->pool_layout != TUTTI_LAYOUT_HND) return TUTTI_EINVAL;
  uint64_t b = static_cast<uint64_t>(pool->block_tokens) * pool->num_kv_heads;
  if (b > 0xffffffffull) return TUTTI_EINVAL;
  b *= pool->head_dim * pool->elt_bytes;  // (at most 256)
  if (b > 0xffffffffull || pool->block_stride < b || pool->block_stride % 16 != 0) return TUTTI_EINVAL;
  return TUTTI_OK;
}
int check_counts(const tutti_batch *b) {
  if (!b) return TUTTI_EINVAL;
  return b->n_seq > TUTTI_MAX_REQ || b->n_rows >= 0x80000000u ? TUTTI_ERANGE : TUTTI_OK;
}

int check_pool(const tutti_pool *pool, const tutti_scales *scales, uint32_t dtype) {
  if (const int rc = check_shape(pool, dtype)) return rc;
  if (!pool->k_base || !pool->v_base || !aligned(pool->k_base, 16) || !aligned(pool->v_base, 16)) return TUTTI_EINVAL;
  if ((pool->elt_bytes == 1) != (scales != nullptr)) return TUTTI_EINVAL;
  if (scales && (!scales->k || !scales->v || !aligned(scales->k, 4) || !aligned(scales->v, 4) ||
                 scales->stride < pool->num_kv_heads))
    return TUTTI_EINVAL;
  return TUTTI_OK;
}

int check_batch(const tutti_batch *b) {
  if (const int rc = check_counts(b)) return rc;
  if (b->n_seq == 0 || b->n_rows == 0 || b->max_new == 0) return TUTTI_OK;
  if (!b->d_seqs || !aligned(b->d_seqs, 16)) return TUTTI_EINVAL;
  if (b->table_len && (!b->d_block_table || !aligned(b->d_block_table, 4))) return TUTTI_EINVAL;
  return TUTTI_OK;
}
bool nothing_to_do(const tutti_batch *b) { return b->n_seq == 0 || b->n_rows == 0 || b->max_new == 0; }

bool good_rows(const tutti_rows *r) {
  return r && r->base && aligned(r->base, 16) && r->row_stride % 16 == 0 && r->head_stride % 16 == 0;
}

PoolView view(const tutti_pool *p, const tutti_scales *s) {
  PoolView v{};
  v.k = static_cast<uint8_t *>(p->k_base);
  v.v = static_cast<uint8_t *>(p->v_base);
  v.block_stride = p->block_stride;
  const uint32_t row = p->head_dim * p->elt_bytes;
  const bool hnd = p->pool_layout == TUTTI_LAYOUT_HND;
  v.token_stride = hnd ? row : row * p->num_kv_heads;
  v.head_stride = hnd ? row * p->block_tokens : row;
  v.num_blocks = p->num_blocks;
  v.block_tokens = p->block_tokens;
  v.shift = 255;
  for (uint32_t i = 0; i < 32; ++i)
    if (p->block_tokens == 1u << i) v.shift = i;
  if (s) {
    v.k_scale = s->k;
    v.v_scale = s->v;
    v.scale_stride = s->stride;
  }
  return v;
}

BatchView view(const tutti_batch *b) {
  return BatchView{b->d_seqs, b->d_block_table, b->n_seq, b->max_new, b->table_len, b->n_rows};
}

constexpr uint64_t kMostThreads = 0xffffffffull;  // of a launch

int launched() {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? TUTTI_OK : hip_failed(e);
}

// ---- append

template <typename T, bool E4M3, int LPR>
void launch_append(const AppendArgs &a, int turn, uint32_t grid, hipStream_t stream) {
  const dim3 g(grid), wg(256);
  if (turn == kNoTurn)
    hipLaunchKernelGGL((k_kv_append<T, E4M3, LPR, kNoTurn>), g, wg, 0, stream, a);
  else if (turn == kHalves)
    hipLaunchKernelGGL((k_kv_append<T, E4M3, LPR, kHalves>), g, wg, 0, stream, a);
  else if (turn == kPairs)
    hipLaunchKernelGGL((k_kv_append<T, E4M3, LPR, kPairs>), g, wg, 0, stream, a);
  else
    hipLaunchKernelGGL((k_kv_append<T, E4M3, LPR, kAnyTurn>), g, wg, 0, stream, a);
}
template <typename T>
void launch_append(const AppendArgs &a, bool e4m3, int turn, uint32_t grid, hipStream_t stream) {
  if (e4m3)
    a.d <= 64 ? launch_append<T, true, 8>(a, turn, grid, stream) : launch_append<T, true, 16>(a, turn, grid, stream);
  else
    a.d <= 64 ? launch_append<T, false, 8>(a, turn, grid, stream) : launch_append<T, false, 16>(a, turn, grid, stream);
}

// How the rotation's pairs lie for lanes that take 8 values each.
int turn_of(const RopeView &r) {
  if (r.rot == 0) return kNoTurn;
  const uint32_t all = r.half | r.end[0] | r.end[1] | r.end[2];
  if (!r.interleaved) return all % 8 == 0 ? kHalves : kAnyTurn;
  return all % 4 == 0 ? kPairs : kAnyTurn;
}

// ---- attend

// Rows of queries a workgroup takes: 16 or 32 where no sequence has more, else 128 (with keys and values in LDS), for all sequences of
// the call.  32 sequences of 8,000 tokens, one KV head, by 16 or 32 rows and by 128, us: bf16 blocks, 8 rows a sequence 33.4 and 38.2,
// 32 rows 39.0 and 41.4, 40 rows 56.5 and 42.8, 96 rows 81.9 and 51.2; e4m3, 32 rows 30.3 and 35.3, 64 rows 40.1 and 41.1.
uint32_t rows_a_tile(const tutti_batch *b, uint32_t group) {
  const uint64_t most = static_cast<uint64_t>(b->max_new) * group;
  return most <= 16 ? 16 : most <= 32 ? 32 : 128;
}

// Workgroups of an attention kernel that the device is taken to hold at once: two a compute unit.  (The kernels for few rows would fit
// three times; 128K tokens of one sequence: 61.7 us with 512, 66.7 with 768, whose parts take longer to join.)  The size of the work
// memory goes by it, so it does not go by the device.
constexpr uint32_t kAttendSlots = 512;

// Neighbouring KV heads that a workgroup takes side by side, so that it reads stretches of a block and not a head's rows here and
// there (128-byte rows of 8 heads: 4.7 TB/s one head a workgroup, 5.8 with four side by side, 6.0 with eight).
uint32_t heads_abreast(uint32_t kv_heads) {
  for (uint32_t n : {4u, 5u, 3u, 2u})
    if (kv_heads % n == 0) return n;
  return 1;
}

struct AttendSizes {
  uint32_t rows, dp, abreast, key_waves, slots, min_tiles, max_units, max_parts;
  uint64_t ml_bytes, bytes;
};

int attend_sizes(const tutti_pool *pool, const tutti_batch *b, const tutti_attn *attn, AttendSizes *s) {
  const uint32_t group = attn->n_q_heads / pool->num_kv_heads;
  s->rows = rows_a_tile(b, group);
  s->dp = pool->head_dim <= 64 ? 64 : 128;
  if (s->rows < 128) {
    s->abreast = heads_abreast(pool->num_kv_heads);
    s->key_waves = s->abreast == 1 ? 4 : s->abreast == 2 ? 2 : 1;
  } else {
    s->abreast = s->key_waves = 1;
  }
  s->slots = kAttendSlots;
  // fewer tiles than this a part are not worth their join (32K tokens: parts of 8 tiles 34.4 us, of 4 tiles 36.9; 512 tokens, where
  // two wavefronts share a part: of 4 tiles 11.2, of 8 tiles 12.4)
  s->min_tiles = s->key_waves == 1 ? 8 : 4;
  // Units: two rounds of the slots at most or, with an even share a part, a round of them and one more for every row tile.  Parts of
  // sequences that are split: the same two rounds; with an even share a split sequence's row tiles have more tiles than a share
  // each, so that they are no more than a round, and their parts no more than two.
  const uint64_t tiles = static_cast<uint64_t>(b->n_rows) * group / s->rows + std::min(b->n_seq, b->n_rows);
  const uint64_t units = 2 * s->slots + tiles * (pool->num_kv_heads / s->abreast);
  if (units * 64 * (s->rows < 128 ? s->abreast * s->key_waves : 4) > kMostThreads || static_cast<uint64_t>(b->n_rows) * attn->n_q_heads >= 0x80000000ull) return TUTTI_ERANGE;
  s->max_units = static_cast<uint32_t>(units);
  s->max_parts = 2 * s->slots * s->abreast;
  s->ml_bytes = static_cast<uint64_t>(s->max_parts) * s->rows * sizeof(f32x2);
  s->bytes = 16 + s->ml_bytes + static_cast<uint64_t>(s->max_parts) * s->rows * s->dp * sizeof(float);
  return TUTTI_OK;
}

int check_attn(const tutti_pool *pool, const tutti_attn *attn) {
  if (!attn || attn->n_q_heads == 0 || attn->n_q_heads % pool->num_kv_heads != 0) return TUTTI_EINVAL;
  if (!std::isfinite(attn->sm_scale) || attn->causal > 1 || (attn->window && !attn->causal)) return TUTTI_EINVAL;
  return TUTTI_OK;
}

template <typename T, bool E4M3, int DP, bool PAGED16, int RT>
void launch_attend(const AttendArgs &a, hipStream_t stream) {
  const dim3 grid(a.max_units), wg(64 * a.abreast * a.key_waves);
  if (a.d == DP)
    hipLaunchKernelGGL((k_kv_attend<T, E4M3, DP, true, PAGED16, RT>), grid, wg, 0, stream, a);
  else
    hipLaunchKernelGGL((k_kv_attend<T, E4M3, DP, false, PAGED16, RT>), grid, wg, 0, stream, a);
}
template <typename T, int DP, int ROWS>
void launch_join(const AttendArgs &a, hipStream_t stream) {
  // a sequence that is split has two parts or more to a row tile, so no more rows are to be joined than this
  const uint32_t joins = std::min(a.batch.n_rows * a.kv_heads * a.group, a.max_parts / 2 * ROWS);
  // A workgroup a row for few rows, which may have many parts (32 rows of 128 parts: one wavefront, part after part, 75 us, four
  // wavefronts 6.7, 16 wavefronts 6.2, but 1,280 rows of some parts 7.5 and 21); else a wavefront a row (1,511 queries of 20 heads in
  // two parts: 20 us, with workgroups 61), 8192 at a time (8,001 prompt tokens that are not split: 5 us, with a wavefront for each row
  // that there might be 21).
  if (joins <= 4096)
    hipLaunchKernelGGL((k_kv_join<T, DP, ROWS, 4>), dim3(joins), dim3(256), 0, stream, a);
  else
    hipLaunchKernelGGL((k_kv_join<T, DP, ROWS, 1>), dim3(2048), dim3(256), 0, stream, a);
}
template <typename T, bool E4M3, bool PAGED16>
void launch_wide(const AttendArgs &a, hipStream_t stream) {
  const dim3 grid(a.max_units), wg(256);
  if (a.d == 128)
    hipLaunchKernelGGL((k_kv_attend_wide<T, E4M3, 128, true, PAGED16>), grid, wg, 0, stream, a);
  else if (a.d == 112)
    hipLaunchKernelGGL((k_kv_attend_wide<T, E4M3, 112, true, PAGED16>), grid, wg, 0, stream, a);
  else if (a.d == 96)
    hipLaunchKernelGGL((k_kv_attend_wide<T, E4M3, 96, true, PAGED16>), grid, wg, 0, stream, a);
  else if (a.d == 80)
    hipLaunchKernelGGL((k_kv_attend_wide<T, E4M3, 80, true, PAGED16>), grid, wg, 0, stream, a);
  else if (a.d == 64)
    hipLaunchKernelGGL((k_kv_attend_wide<T, E4M3, 64, true, PAGED16>), grid, wg, 0, stream, a);
  else
    hipLaunchKernelGGL((k_kv_attend_wide<T, E4M3, 64, false, PAGED16>), grid, wg, 0, stream, a);
}
template <typename T, bool E4M3, int DP>
void launch_attend(const AttendArgs &a, uint32_t rows, hipStream_t stream) {
  if (rows == 128) {
    if (a.pool.block_tokens % 16 == 0)
      launch_wide<T, E4M3, true>(a, stream);
    else
      launch_wide<T, E4M3, false>(a, stream);
    launch_join<T, DP, 128>(a, stream);
    return;
  }
  if (a.pool.block_tokens % 16 == 0)
    rows == 16 ? launch_attend<T, E4M3, DP, true, 1>(a, stream) : launch_attend<T, E4M3, DP, true, 2>(a, stream);
  else
    rows == 16 ? launch_attend<T, E4M3, DP, false, 1>(a, stream) : launch_attend<T, E4M3, DP, false, 2>(a, stream);
  rows == 16 ? launch_join<T, DP, 16>(a, stream) : launch_join<T, DP, 32>(a, stream);
}
template <typename T>
void launch_attend(const AttendArgs &a, bool e4m3, uint32_t rows, hipStream_t stream) {
  if (e4m3)
    a.d <= 64 ? launch_attend<T, true, 64>(a, rows, stream) : launch_attend<T, true, 128>(a, rows, stream);
  else
    a.d <= 64 ? launch_attend<T, false, 64>(a, rows, stream) : launch_attend<T, false, 128>(a, rows, stream);
}

}  // namespace

extern "C" {

int tutti_kv_append(const tutti_pool *pool, const tutti_scales *scales, const tutti_batch *batch, const tutti_rope *rope,
                    const tutti_rows *q, const tutti_rows *q_out, const tutti_rows *k, const tutti_rows *v,
                    uint32_t n_q_heads, uint32_t dtype, uint32_t *d_status, void *stream) {
  int rc = check_pool(pool, scales, dtype);
  if (rc) return rc;
  if ((rc = check_batch(batch)) != TUTTI_OK) return rc;
  if (!aligned(d_status, 4)) return TUTTI_EINVAL;
  if (!good_rows(k) || !good_rows(v)) return TUTTI_EINVAL;
  if (q && (!good_rows(q) || !good_rows(q_out) || n_q_heads == 0)) return TUTTI_EINVAL;
  if (q && n_q_heads > 0xffffu) return TUTTI_ERANGE;
  AppendArgs a{};
  if (rope) {
    RopeView &r = a.rope;
    if (rope->rot_dim % 2 != 0 || rope->rot_dim == 0 || rope->rot_dim > pool->head_dim || rope->interleaved > 1) return TUTTI_EINVAL;
    if (!rope->d_cos_sin || !aligned(rope->d_cos_sin, 16) || rope->n_pos == 0 || !aligned(rope->d_pos, 4)) return TUTTI_EINVAL;
    r.cos_sin = rope->d_cos_sin;
    r.pos = rope->d_pos;
    r.pos_stride = rope->pos_stride;
    r.n_pos = rope->n_pos;
    r.rot = rope->rot_dim;
    r.half = rope->rot_dim / 2;
    r.interleaved = rope->interleaved;
    if (rope->d_pos) {
      uint64_t end = 0;
      for (int i = 0; i < 4; ++i) {
        end += rope->axis_pairs[i];
        if (i < 3) r.end[i] = static_cast<uint32_t>(std::min<uint64_t>(end, r.half));
        if (rope->axis_pairs[i]) r.axes |= 1u << i;
      }
      if (end != r.half) return TUTTI_EINVAL;
    } else {
      r.end[0] = r.end[1] = r.end[2] = r.half;
      r.axes = 1;
    }
  }
  if (nothing_to_do(batch)) return TUTTI_OK;
  a.pool = view(pool, scales);
  a.batch = view(batch);
  if (q) {
    a.q = *q;
    a.q_out = *q_out;
    a.q_heads = n_q_heads;
  }
  a.k = *k;
  a.v = *v;
  a.kv_heads = pool->num_kv_heads;
  a.d = pool->head_dim;
  a.status = d_status;
  const bool e4m3 = scales != nullptr;
  // a unit has at least one new token, and only a sequence's first and last may have fewer than a whole unit's
  const uint64_t tokens = e4m3 ? pool->block_tokens : kLanes / (a.d <= 64 ? 8 : 16);
  uint64_t units = std::min<uint64_t>(batch->n_rows, batch->n_rows / tokens + 2ull * batch->n_seq);
  if (batch->max_new == 1) units = batch->n_seq;
  a.heads_a_job = 4;
  a.q_jobs = (a.q_heads + a.heads_a_job - 1) / a.heads_a_job;
  a.jobs = a.q_jobs + 2 * (e4m3 ? a.kv_heads : (a.kv_heads + a.heads_a_job - 1) / a.heads_a_job);
  if ((units * a.jobs + 3) / 4 * 256 > kMostThreads) return TUTTI_ERANGE;
  a.max_units = static_cast<uint32_t>(units);
  const uint32_t grid = static_cast<uint32_t>((units * a.jobs + 3) / 4);
  const hipStream_t st = static_cast<hipStream_t>(stream);
  if (dtype == TUTTI_BF16)
    launch_append<Bf16>(a, e4m3, turn_of(a.rope), grid, st);
  else
    launch_append<Fp16>(a, e4m3, turn_of(a.rope), grid, st);
  return launched();
}

uint64_t tutti_kv_attend_work_bytes(const tutti_pool *pool, const tutti_batch *batch, const tutti_attn *attn) {
  AttendSizes s;
  if (!attn || check_shape(pool, attn->dtype) != TUTTI_OK || check_counts(batch) != TUTTI_OK || check_attn(pool, attn) != TUTTI_OK) return 0;
  if (attend_sizes(pool, batch, attn, &s) != TUTTI_OK) return 0;
  return s.bytes;
}

int tutti_kv_attend(const tutti_pool *pool, const tutti_scales *scales, const tutti_batch *batch, const tutti_attn *attn,
                    const tutti_rows *q, const tutti_rows *out, float *d_lse, void *d_work, uint64_t work_bytes,
                    uint32_t *d_status, void *stream) {
  if (!attn) return TUTTI_EINVAL;
  int rc = check_pool(pool, scales, attn->dtype);
  if (rc) return rc;
  if ((rc = check_batch(batch)) != TUTTI_OK) return rc;
  if ((rc = check_attn(pool, attn)) != TUTTI_OK) return rc;
  if (!good_rows(q) || !good_rows(out) || !aligned(d_lse, 4) || !aligned(d_status, 4)) return TUTTI_EINVAL;
  AttendSizes s;
  if ((rc = attend_sizes(pool, batch, attn, &s)) != TUTTI_OK) return rc;
  if (nothing_to_do(batch)) return TUTTI_OK;
  if (!d_work || !aligned(d_work, 16)) return TUTTI_EINVAL;
  if (work_bytes < s.bytes) return TUTTI_ERANGE;
  AttendArgs a{};
  a.pool = view(pool, scales);
  a.batch = view(batch);
  a.q = *q;
  a.out = *out;
  a.lse = d_lse;
  a.kv_heads = pool->num_kv_heads;
  a.group = attn->n_q_heads / pool->num_kv_heads;
  a.d = pool->head_dim;
  a.scale_log2 = attn->sm_scale * kLog2e;
  a.causal = attn->causal;
  a.window = attn->window;
  a.abreast = s.abreast;
  a.key_waves = s.key_waves;
  a.slots = s.slots;
  a.min_tiles = s.min_tiles;
  a.max_units = s.max_units;
  a.max_parts = s.max_parts;
  a.tiles_a_part = static_cast<uint32_t *>(d_work);
  a.part_ml = reinterpret_cast<f32x2 *>(static_cast<uint8_t *>(d_work) + 16);
  a.part_o = reinterpret_cast<float *>(static_cast<uint8_t *>(d_work) + 16 + s.ml_bytes);
  a.status = d_status;
  const hipStream_t st = static_cast<hipStream_t>(stream);
  if (attn->dtype == TUTTI_BF16)
    launch_attend<Bf16>(a, scales != nullptr, s.rows, st);
  else
    launch_attend<Fp16>(a, scales != nullptr, s.rows, st);
  return launched();
}

}  // extern "C"
