// Rules that decide by sizes alone how a call of attention is run, and how much work memory it needs.  Plain C++, so that they can be
// tested without a GPU.
#pragma once

#include <stdint.h>

#include <algorithm>

#include "tutti.h"

namespace tutti {

constexpr uint32_t kKeyTile = 32;  // keys that a wavefront of the kernels for few rows takes at a time: two halves of 16
constexpr uint64_t kMostThreads = 0xffffffffull;  // of a launch

// Rows of queries a workgroup takes: 16 or 32 where no sequence has more, else 128 (with keys and values in LDS), for all sequences of
// the call.  32 sequences of 8,000 tokens, one KV head, by 16 or 32 rows and by 128, us: bf16 blocks, 8 rows a sequence 33.4 and 38.2,
// 32 rows 39.0 and 41.4, 40 rows 56.5 and 42.8, 96 rows 81.9 and 51.2; e4m3, 32 rows 30.3 and 35.3, 64 rows 40.1 and 41.1.
inline uint32_t rows_a_tile(const tutti_batch *b, uint32_t group) {
  const uint64_t most = static_cast<uint64_t>(b->max_new) * group;
  return most <= 16 ? 16 : most <= 32 ? 32 : 128;
}

// Workgroups of an attention kernel that the device is taken to hold at once: two a compute unit.  (The kernels for few rows would fit
// three times; 128K tokens of one sequence: 61.7 us with 512, 66.7 with 768, whose parts take longer to join.)  The size of the work
// memory goes by it, so it does not go by the device.
constexpr uint32_t kAttendSlots = 512;

// Neighbouring KV heads that a workgroup takes side by side, so that it reads stretches of a block and not a head's rows here and
// there (128-byte rows of 8 heads: 4.7 TB/s one head a workgroup, 5.8 with four side by side, 6.0 with eight).
inline uint32_t heads_abreast(uint32_t kv_heads) {
  for (uint32_t n : {4u, 5u, 3u, 2u})
    if (kv_heads % n == 0) return n;
  return 1;
}

struct AttendSizes {
  uint32_t rows, dp, abreast, key_waves, slots, min_tiles, max_units, max_parts;
  uint64_t ml_bytes, bytes;
};

// abreast: KV heads of a workgroup, 0 for as many as go with the pool
inline int attend_sizes(const tutti_pool *pool, const tutti_batch *b, const tutti_attn *attn, AttendSizes *s, uint32_t abreast = 0) {
  const uint32_t group = attn->n_q_heads / pool->num_kv_heads;
  s->rows = rows_a_tile(b, group);
  s->dp = pool->head_dim <= 64 ? 64 : 128;
  if (s->rows < 128) {
    s->abreast = abreast ? abreast : heads_abreast(pool->num_kv_heads);
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
  s->ml_bytes = static_cast<uint64_t>(s->max_parts) * s->rows * 2 * sizeof(float);
  s->bytes = 16 + s->ml_bytes + static_cast<uint64_t>(s->max_parts) * s->rows * s->dp * sizeof(float);
  return TUTTI_OK;
}

// Key tiles that a tile of `rows` rows sees at most: the windows of its places, which follow each other, wherever they begin, and the
// first keys.
inline uint32_t most_tiles(uint32_t rows, uint32_t group, uint32_t window, uint32_t sinks) {
  const uint64_t places = (rows + group - 2) / group + 1, keys = window + places - 1;
  const uint64_t n = (keys + kKeyTile - 2) / kKeyTile + 1 + (static_cast<uint64_t>(sinks) + kKeyTile - 1) / kKeyTile;
  return static_cast<uint32_t>(std::min<uint64_t>(n, 0x7fffffffu));
}

// With first tokens: KV heads of a workgroup where what all windows hold is so little that the time is that of a workgroup's tiles one after the
// other.  Then four wavefronts share a head's tiles, as long as there is a workgroup a slot at most.  One token each, four, two and one
// heads abreast, us: e4m3, 8 heads, windows of 1,000 keys, one sequence 20.2, 14.4, 13.5, 32 sequences 30.0, 26.0, 24.2, 64 37.3, 37.5,
// 39.0; windows of 200 keys, 32 sequences 23.0, 14.2, 11.8, 128 28.0, 20.9, 28.1 (two rounds of the slots); five heads and one, windows of
// 4,096 keys, 32 sequences 52.4 and 42.3, 64 84.4 and 90.7.
inline uint32_t heads_abreast_of_few(const tutti_pool *pool, const AttendSizes &s, uint64_t row_tiles, uint32_t tiles) {
  const uint32_t heads = pool->num_kv_heads;
  if (row_tiles * heads * tiles > static_cast<uint64_t>(s.slots) * (s.key_waves == 1 && s.abreast != 4 ? 48 : 24)) return s.abreast;
  for (const uint32_t n : {1u, 2u})
    if (n < s.abreast && heads % n == 0 && row_tiles * (heads / n) <= s.slots) return n;
  return s.abreast == 4 || row_tiles * heads > 4 * s.slots ? s.abreast : 1;
}

// `s` with as many heads a workgroup as go with what the windows hold, in calls with first tokens.  It never needs more work memory.
inline void sizes_of_few(const tutti_pool *pool, const tutti_batch *batch, const tutti_attn *attn, uint32_t most, AttendSizes *s) {
  if (s->rows >= 128) return;
  const uint32_t abreast = heads_abreast_of_few(pool, *s, std::min(batch->n_seq, batch->n_rows), most);  // (a row tile a sequence)
  AttendSizes few;  // (more workgroups: rows that no sequence has may make them too many for a launch)
  if (abreast != s->abreast && attend_sizes(pool, batch, attn, &few, abreast) == TUTTI_OK) *s = few;
}

}  // namespace tutti
