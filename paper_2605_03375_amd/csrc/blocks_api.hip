// Host side of the calls that share, copy, give back and move blocks: tutti_blocks_*.  As everywhere in the library a call checks its host
// arguments in O(1), enqueues a constant number of kernels on the caller's stream and returns.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "blocks.hip.h"
#include "library_state.h"
#include "tutti.h"

namespace {

using namespace tutti;

bool aligned(const void *p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

int launched() {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? TUTTI_OK : hip_failed(e);
}

constexpr uint32_t kMostThings = 0x80000000u;          // blocks, or entries of a record, are fewer
constexpr uint64_t kMostGroups = 0xffffffffull / 256;  // workgroups of 256 threads of a launch

// Spans of whole chunks, at most kMostSpans of them.
uint32_t span_size(uint32_t num_blocks) {
  const uint32_t chunks = num_blocks / kChunk + (num_blocks % kChunk != 0);
  return (chunks + kMostSpans - 1) / kMostSpans * kChunk;
}
Spans spans_of(uint32_t *uses, uint32_t num_blocks, uint32_t *counts) {
  const uint32_t size = span_size(num_blocks);
  return Spans{uses, num_blocks, size, num_blocks / size + (num_blocks % size != 0), counts};
}

int check_table(const uint32_t *uses, uint32_t num_blocks, const uint32_t *table, uint32_t table_len, const uint32_t *status) {
  if (!uses || !aligned(uses, 16) || num_blocks == 0) return TUTTI_EINVAL;
  if (num_blocks >= kMostThings) return TUTTI_ERANGE;
  if (table_len && (!table || !aligned(table, 4))) return TUTTI_EINVAL;
  return aligned(status, 4) ? TUTTI_OK : TUTTI_EINVAL;
}

uint64_t list_bytes(uint32_t num_blocks) { return (static_cast<uint64_t>(num_blocks) * 4 + 15) / 16 * 16; }
uint64_t bits_bytes(uint32_t num_blocks) { return (static_cast<uint64_t>(num_blocks) + 127) / 128 * 16; }

}  // namespace

extern "C" {

uint64_t tutti_blocks_fork_work_bytes(uint32_t num_blocks, uint32_t n_forks) {
  if (num_blocks == 0 || num_blocks >= kMostThings || n_forks > TUTTI_MAX_REQ) return 0;
  return kMostSpans * 4 + static_cast<uint64_t>(n_forks) * sizeof(u32x2) + 16 + list_bytes(num_blocks) + bits_bytes(num_blocks);
}

int tutti_blocks_fork(uint32_t *d_uses, uint32_t num_blocks, uint32_t *d_block_table, uint32_t table_len, const tutti_fork *d_forks,
                      uint32_t n_forks, uint32_t max_entries, tutti_block_pair *d_pairs, uint32_t *d_n_pairs, uint32_t max_pairs,
                      void *d_work, uint64_t work_bytes, uint32_t *d_status, void *stream) {
  if (const int rc = check_table(d_uses, num_blocks, d_block_table, table_len, d_status)) return rc;
  if (n_forks > TUTTI_MAX_REQ || max_entries >= kMostThings) return TUTTI_ERANGE;
  if (n_forks && (!d_forks || !aligned(d_forks, 16))) return TUTTI_EINVAL;
  if (max_pairs == TUTTI_NO_BLOCK) return TUTTI_ERANGE;
  if (max_pairs && (!d_pairs || !aligned(d_pairs, 8))) return TUTTI_EINVAL;
  if (!aligned(d_n_pairs, 4) || !d_work || !aligned(d_work, 16)) return TUTTI_EINVAL;
  if (work_bytes < tutti_blocks_fork_work_bytes(num_blocks, n_forks)) return TUTTI_ERANGE;
  ForkArgs a{};
  a.chunks = max_entries / kEntries + (max_entries % kEntries != 0);
  const uint32_t groups = (n_forks + kGroup - 1) / kGroup;
  if (static_cast<uint64_t>(a.chunks) * groups > kMostGroups) return TUTTI_ERANGE;
  uint8_t *const work = static_cast<uint8_t *>(d_work);
  a.spans = spans_of(d_uses, num_blocks, reinterpret_cast<uint32_t *>(work));
  a.first = reinterpret_cast<u32x2 *>(work + kMostSpans * 4);
  a.list = reinterpret_cast<uint32_t *>(work + kMostSpans * 4 + (static_cast<uint64_t>(n_forks) * sizeof(u32x2) + 15) / 16 * 16);
  a.free = a.list + list_bytes(num_blocks) / 4;
  a.uses = d_uses;
  a.table = d_block_table;
  a.table_len = table_len;
  a.forks = d_forks;
  a.n_forks = n_forks;
  a.max_entries = max_entries;
  a.pairs = d_pairs;
  a.n_pairs = d_n_pairs;
  a.max_pairs = max_pairs;
  a.status = d_status;
  const hipStream_t st = static_cast<hipStream_t>(stream);
  if (num_blocks <= kSmallBlocks && n_forks <= kSmallRecords && static_cast<uint64_t>(n_forks) * max_entries <= kSmallEntries) {
    hipLaunchKernelGGL(k_blocks_fork_small, dim3(1), dim3(1024), 0, st, a);
    return launched();
  }
  const bool entries = n_forks && max_entries;
  if (!entries) a.spans.n = 0;  // (records to be counted, or none: nothing is taken)
  hipLaunchKernelGGL(k_blocks_list_free, dim3(a.spans.n + 1), dim3(256), 0, st, a);
  if (entries) hipLaunchKernelGGL(k_blocks_fork, dim3(a.chunks * groups), dim3(256), 0, st, a);
  return launched();
}

int tutti_blocks_free(uint32_t *d_uses, uint32_t num_blocks, uint32_t *d_block_table, uint32_t table_len,
                      const tutti_block_range *d_ranges, uint32_t n_ranges, uint32_t max_entries, uint32_t *d_status, void *stream) {
  if (const int rc = check_table(d_uses, num_blocks, d_block_table, table_len, d_status)) return rc;
  if (n_ranges > TUTTI_MAX_REQ || max_entries >= kMostThings) return TUTTI_ERANGE;
  if (n_ranges && (!d_ranges || !aligned(d_ranges, 8))) return TUTTI_EINVAL;
  if (n_ranges == 0) return TUTTI_OK;
  FreeArgs a{};
  a.chunks = std::max(1u, max_entries / kEntries + (max_entries % kEntries != 0));
  // Ranges of a few entries go one by one: 256 of one entry 2.5 us, eight to a workgroup 3.9.
  const uint32_t each = max_entries > 32 ? kGroup : 1, groups = (n_ranges + each - 1) / each;
  if (static_cast<uint64_t>(a.chunks) * groups > kMostGroups) return TUTTI_ERANGE;
  a.uses = d_uses;
  a.table = d_block_table;
  a.num_blocks = num_blocks;
  a.table_len = table_len;
  a.ranges = d_ranges;
  a.n_ranges = n_ranges;
  a.max_entries = max_entries;
  a.status = d_status;
  const hipStream_t st = static_cast<hipStream_t>(stream);
  if (each == 1)
    hipLaunchKernelGGL((k_blocks_free<1>), dim3(a.chunks * groups), dim3(256), 0, st, a);
  else
    hipLaunchKernelGGL((k_blocks_free<kGroup>), dim3(a.chunks * groups), dim3(256), 0, st, a);
  return launched();
}

uint64_t tutti_blocks_compact_work_bytes(uint32_t num_blocks) {
  if (num_blocks == 0 || num_blocks >= kMostThings) return 0;
  return kMostSpans * 4 + 16 + 2 * list_bytes(num_blocks) + bits_bytes(num_blocks);
}

int tutti_blocks_compact(uint32_t *d_uses, uint32_t num_blocks, uint32_t *d_block_table, uint32_t table_len,
                         tutti_block_pair *d_pairs, uint32_t *d_totals, uint32_t max_pairs, void *d_work, uint64_t work_bytes,
                         uint32_t *d_status, void *stream) {
  if (const int rc = check_table(d_uses, num_blocks, d_block_table, table_len, d_status)) return rc;
  if (max_pairs && (!d_pairs || !aligned(d_pairs, 8))) return TUTTI_EINVAL;
  if (!d_totals || !aligned(d_totals, 4) || !d_work || !aligned(d_work, 16)) return TUTTI_EINVAL;
  if (work_bytes < tutti_blocks_compact_work_bytes(num_blocks)) return TUTTI_ERANGE;
  CompactArgs a{};
  uint8_t *const work = static_cast<uint8_t *>(d_work);
  a.spans = spans_of(d_uses, num_blocks, reinterpret_cast<uint32_t *>(work));
  a.found = reinterpret_cast<uint32_t *>(work + kMostSpans * 4);
  a.holes = reinterpret_cast<uint32_t *>(work + kMostSpans * 4 + 16);
  a.rank = reinterpret_cast<uint32_t *>(work + kMostSpans * 4 + 16 + list_bytes(num_blocks));
  a.used_at = static_cast<uint32_t>(list_bytes(num_blocks) / 4);
  a.used = a.rank + a.used_at;
  a.uses = d_uses;
  a.table = d_block_table;
  a.table_len = table_len;
  a.pairs = d_pairs;
  a.totals = d_totals;
  a.max_pairs = max_pairs;
  a.status = d_status;
  const hipStream_t st = static_cast<hipStream_t>(stream);
  // what the device holds at once: 2,048 workgroups, four things a thread
  const auto groups = [](uint32_t things, uint32_t most) { return std::min(most, things / 256 + (things % 256 != 0)); };
  a.table_groups = groups(table_len, 1536);
  hipLaunchKernelGGL(k_blocks_count_used, dim3(a.spans.n), dim3(256), 0, st, a);
  hipLaunchKernelGGL(k_blocks_rank, dim3(a.spans.n), dim3(256), 0, st, a);
  hipLaunchKernelGGL(k_blocks_move, dim3(a.table_groups + groups(num_blocks, 512)), dim3(256), 0, st, a);
  return launched();
}

int tutti_blocks_copy(const tutti_pool *pool, const tutti_scales *scales, const tutti_block_pair *d_pairs, const uint32_t *d_n_pairs,
                      uint32_t max_pairs, uint32_t *d_status, void *stream) {
  if (!pool || !pool->k_base || !pool->v_base || !aligned(pool->k_base, 16) || !aligned(pool->v_base, 16)) return TUTTI_EINVAL;
  if (pool->num_blocks == 0 || pool->block_tokens == 0 || pool->num_kv_heads == 0 || pool->head_dim == 0 || pool->elt_bytes == 0)
    return TUTTI_EINVAL;
  if (pool->pool_layout != TUTTI_LAYOUT_NHD && pool->pool_layout != TUTTI_LAYOUT_HND) return TUTTI_EINVAL;
  uint64_t bytes = 1;
  for (const uint32_t n : {pool->block_tokens, pool->num_kv_heads, pool->head_dim, pool->elt_bytes}) {
    bytes *= n;
    if (bytes > 0xffffffffull) return TUTTI_EINVAL;
  }
  if (bytes % 16 != 0 || pool->block_stride % 16 != 0 || pool->block_stride < bytes) return TUTTI_EINVAL;
  if (scales && (!scales->k || !scales->v || !aligned(scales->k, 4) || !aligned(scales->v, 4) || scales->stride < pool->num_kv_heads))
    return TUTTI_EINVAL;
  if (!aligned(d_n_pairs, 4) || !aligned(d_status, 4)) return TUTTI_EINVAL;
  if (max_pairs == 0) return TUTTI_OK;
  if (!d_pairs || !aligned(d_pairs, 8)) return TUTTI_EINVAL;
  CopyArgs a{};
  a.planes[0] = static_cast<uint8_t *>(pool->k_base);
  a.planes[1] = static_cast<uint8_t *>(pool->v_base);
  if (scales) {
    a.scales[0] = scales->k;
    a.scales[1] = scales->v;
    a.scale_stride = scales->stride;
  }
  a.block_stride = pool->block_stride;
  a.units = static_cast<uint32_t>(bytes / 16);
  a.pieces = (a.units + kPiece - 1) / kPiece;
  a.kv_heads = pool->num_kv_heads;
  a.num_blocks = pool->num_blocks;
  a.pairs = d_pairs;
  a.n_pairs = d_n_pairs;
  a.max_pairs = max_pairs;
  a.status = d_status;
  const uint64_t jobs = static_cast<uint64_t>(max_pairs) * 2 * a.pieces;
  // A wavefront a piece where the number of pairs is known (6,001 pairs of 32 KiB, 787 MB: 155 us, 158 with 2,048 workgroups); where
  // there may be few of max_pairs, workgroups without a piece would cost more than their order gains.
  const uint64_t most = d_n_pairs ? 2048 : 1u << 20;
  const uint32_t grid = static_cast<uint32_t>(std::min<uint64_t>(most, (jobs + 3) / 4));
  a.step_rows = grid * 4 / a.pieces;
  a.step_pieces = grid * 4 % a.pieces;
  hipLaunchKernelGGL(k_blocks_copy, dim3(grid), dim3(256), 0, static_cast<hipStream_t>(stream), a);
  return launched();
}

}  // extern "C"
