// Host side of the calls that use a paged cache in place: tutti_kv_append, tutti_kv_attend.  As everywhere in the library a call
// checks its host arguments in O(1), enqueues a constant number of kernels on the caller's stream and returns.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "attend_rules.h"
#include "kv_append.hip.h"
#include "kv_attend_launch.h"
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

int check_attn(const tutti_pool *pool, const tutti_attn *attn) {
  if (!attn || attn->n_q_heads == 0 || attn->n_q_heads % pool->num_kv_heads != 0) return TUTTI_EINVAL;
  if (!std::isfinite(attn->sm_scale) || attn->causal > 1 || (attn->window && !attn->causal)) return TUTTI_EINVAL;
  return TUTTI_OK;
}

template <typename T>
void launch_attend(const AttendArgs &a, bool e4m3, uint32_t rows, hipStream_t stream) {
  // kernels of their own where first keys stay visible beside a window: the others have no tiles to leap over
  if (e4m3)
    a.sinks ? launch_attend<T, true, true>(a, rows, stream) : launch_attend<T, true, false>(a, rows, stream);
  else
    a.sinks ? launch_attend<T, false, true>(a, rows, stream) : launch_attend<T, false, false>(a, rows, stream);
}

// Both calls of attention; n_sinks: of tutti_kv_attend_sinks.
int attend(const tutti_pool *pool, const tutti_scales *scales, const tutti_batch *batch, const tutti_attn *attn, uint32_t n_sinks,
           const tutti_rows *q, const tutti_rows *out, float *d_lse, void *d_work, uint64_t work_bytes, uint32_t *d_status,
           void *stream) {
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
  const bool with_sinks = attn->window && n_sinks;  // (without a window every key stays visible)
  const uint32_t group = attn->n_q_heads / pool->num_kv_heads;
  const uint32_t sinks = std::min(n_sinks, 0x7fffffffu), most = with_sinks ? most_tiles(s.rows, group, attn->window, sinks) : 0;
  if (with_sinks) sizes_of_few(pool, batch, attn, most, &s);
  AttendArgs a{};
  a.pool = view(pool, scales);
  a.batch = view(batch);
  a.q = *q;
  a.out = *out;
  a.lse = d_lse;
  a.kv_heads = pool->num_kv_heads;
  a.group = group;
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
  if (with_sinks) {
    a.sinks = sinks;
    a.most_tiles = most;
    a.unit_tiles = 2 * s.key_waves;
    a.join_tiles = 3 * s.key_waves;
    // So few that they are not split, by one sequence of 1 to 8 heads whole and in parts, us: one head 14 tiles 12.2 and 13.4, 27 tiles 16.3 and
    // 13.5; two heads side by side 10 tiles 13.7 and 13.9; eight, four abreast, 8 tiles 19.6 and 23.6, 14 tiles 32 and 24; 40 queries 8 tiles 16.6 and 16.3 to 16.8.
    a.whole_tiles = s.rows < 128 ? 6 + s.key_waves * 5 / 2 : 12;
    if (a.most_tiles <= a.whole_tiles) a.min_tiles = a.most_tiles;
  }
  const hipStream_t st = static_cast<hipStream_t>(stream);
  if (attn->dtype == TUTTI_BF16)
    launch_attend<Bf16>(a, scales != nullptr, s.rows, st);
  else
    launch_attend<Fp16>(a, scales != nullptr, s.rows, st);
  return launched();
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
  return attend(pool, scales, batch, attn, 0, q, out, d_lse, d_work, work_bytes, d_status, stream);
}

int tutti_kv_attend_sinks(const tutti_pool *pool, const tutti_scales *scales, const tutti_batch *batch, const tutti_attn *attn,
                          uint32_t n_sinks, const tutti_rows *q, const tutti_rows *out, float *d_lse, void *d_work,
                          uint64_t work_bytes, uint32_t *d_status, void *stream) {
  return attend(pool, scales, batch, attn, n_sinks, q, out, d_lse, d_work, work_bytes, d_status, stream);
}

}  // extern "C"
