// Blocks of a paged cache shared, copied, given back and moved together: counts of uses, tables, and one layer's data.
#pragma once
#include "kv_common.hip.h"

namespace tutti {

constexpr uint32_t kNoBlock = TUTTI_NO_BLOCK;
constexpr uint32_t kChunk = 1024;    // counts or table entries that a workgroup of 256 takes at a time
constexpr uint32_t kMostSpans = 1024;

// The pool's counts in spans of whole chunks, one to a workgroup; at most kMostSpans of them, so that whoever needs the number of
// (free, used) blocks in front of a span adds them up by itself, in one pass of a workgroup, instead of a launch that does.
struct Spans {
  const uint32_t *uses;
  uint32_t num_blocks, size, n;
  uint32_t *counts;  // of each span
};

// Sum over the workgroup's threads of what lies in front of a thread's, and of all.  `sums`: 4 words of LDS; behind a barrier.
__device__ __forceinline__ uint32_t sum_in_front(uint32_t mine, uint32_t *sums, uint32_t &all) {
  const uint32_t lane = threadIdx.x & (kLanes - 1), wave = threadIdx.x / kLanes, upto = lane_prefix_sum(mine);
  if (lane == kLanes - 1) sums[wave] = upto;
  __syncthreads();
  uint32_t before = 0;
  all = 0;
#pragma unroll
  for (uint32_t w = 0; w < 4; ++w) {
    if (w < wave) before += sums[w];
    all += sums[w];
  }
  __syncthreads();
  return before + upto - mine;
}

// Four counts from a multiple of 4 on; those behind the pool's end are `beyond`.
__device__ __forceinline__ u32x4 four_uses(const Spans &s, uint32_t id, uint32_t beyond) {
  if (id < s.num_blocks && s.num_blocks - id >= 4) return *reinterpret_cast<const u32x4 *>(s.uses + id);
  u32x4 u = {beyond, beyond, beyond, beyond};
#pragma unroll
  for (uint32_t i = 0; i < 3; ++i)
    if (id < s.num_blocks && i < s.num_blocks - id) u[i] = s.uses[id + i];
  return u;
}

// counts_before[i] <- counts of the spans in front of span i (LDS, kMostSpans words); returns the sum of all.
__device__ __forceinline__ uint32_t add_up(const Spans &s, uint32_t *counts_before, uint32_t *sums) {
  uint32_t c[4], mine = 0, all;
#pragma unroll
  for (uint32_t i = 0; i < 4; ++i) {
    const uint32_t at = threadIdx.x * 4 + i;
    c[i] = at < s.n ? s.counts[at] : 0;
    mine += c[i];
  }
  uint32_t before = sum_in_front(mine, sums, all);
#pragma unroll
  for (uint32_t i = 0; i < 4; ++i) {
    counts_before[threadIdx.x * 4 + i] = before;
    before += c[i];
  }
  __syncthreads();
  return all;
}

// ---- fork

struct ForkArgs {
  Spans spans;
  uint32_t *uses, *table;
  uint32_t table_len;
  const tutti_fork *forks;
  uint32_t n_forks, max_entries, chunks;  // chunks: of max_entries
  tutti_block_pair *pairs;
  uint32_t *n_pairs;
  uint32_t max_pairs;
  uint32_t *list;      // free blocks: those of span i from i * size on
  u32x2 *first;        // of each record: numbers of its first new block and its first pair; kNoBlock: the record is skipped
  uint32_t *status;
};

struct Fork {
  uint32_t src, dst, shared, copied, fresh;  // fresh: copied and new ones
};
__device__ __forceinline__ Fork load_fork(const tutti_fork *f) {
  const u32x4 w = *reinterpret_cast<const u32x4 *>(f);
  const uint32_t n_new = f->n_new;
  return Fork{w[0], w[1], w[2], w[3], w[3] + n_new};
}
__device__ __forceinline__ bool fork_ok(const ForkArgs &a, const tutti_fork *f) {
  const u32x4 w = *reinterpret_cast<const u32x4 *>(f);
  const uint64_t old = static_cast<uint64_t>(w[2]) + w[3], all = old + f->n_new;
  return all <= a.max_entries && w[1] + all <= a.table_len && (old == 0 || w[0] + old <= a.table_len);
}

// The first of two launches: workgroup i lists the free blocks of span i in order; one more numbers the records' new blocks and pairs.
// Bound by its trips to memory (counts, then sums in LDS).
__global__ __launch_bounds__(256) void k_blocks_list_free(const ForkArgs a) {
  __shared__ uint32_t sums[4];
  const Spans &s = a.spans;
  if (blockIdx.x < s.n) {
    uint32_t n = 0;
    const uint32_t begin = blockIdx.x * s.size;
    for (uint32_t in = 0; in < s.size && in < s.num_blocks - begin; in += kChunk) {
      const uint32_t id = begin + in + threadIdx.x * 4;
      const u32x4 u = four_uses(s, id, 1);
      const uint32_t mine = (u[0] == 0) + (u[1] == 0) + (u[2] == 0) + (u[3] == 0);
      uint32_t all, at = n + sum_in_front(mine, sums, all);
#pragma unroll
      for (uint32_t i = 0; i < 4; ++i)
        if (u[i] == 0) a.list[begin + at++] = id + i;
      n += all;
    }
    if (threadIdx.x == 0) s.counts[blockIdx.x] = n;
    return;
  }
  // records: at most TUTTI_MAX_REQ, 8 a thread
  constexpr uint32_t EACH = TUTTI_MAX_REQ / 256;
  __shared__ uint64_t wide[2][4];
  __shared__ uint32_t most;
  const uint32_t lane = threadIdx.x & (kLanes - 1), wave = threadIdx.x / kLanes;
  if (threadIdx.x == 0) most = 0;
  uint64_t sum[2] = {0, 0};
  uint32_t fresh[EACH], copied[EACH];
  bool ok[EACH], bad = false;
#pragma unroll
  for (uint32_t i = 0; i < EACH; ++i) {
    const uint32_t r = threadIdx.x * EACH + i;
    ok[i] = r < a.n_forks && fork_ok(a, a.forks + r);
    bad |= r < a.n_forks && !ok[i];
    const Fork f = ok[i] ? load_fork(a.forks + r) : Fork{};
    fresh[i] = f.fresh;
    copied[i] = f.copied;
    sum[0] += f.fresh;
    sum[1] += f.copied;
  }
  // 64-bit sums in front of the thread's
  uint64_t upto[2] = {sum[0], sum[1]};
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    for (uint32_t m = 1; m < kLanes; m <<= 1) {
      const uint64_t left = __shfl_up(upto[x], m, kLanes);
      if (lane >= m) upto[x] += left;
    }
    if (lane == kLanes - 1) wide[x][wave] = upto[x];
  }
  __syncthreads();
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    upto[x] -= sum[x];
    for (uint32_t w = 0; w < wave; ++w) upto[x] += wide[x][w];
  }
  uint32_t pairs = 0;
#pragma unroll
  for (uint32_t i = 0; i < EACH; ++i) {
    const uint32_t r = threadIdx.x * EACH + i;
    const bool fits = upto[1] + copied[i] <= a.max_pairs;
    if (r < a.n_forks) {
      bad |= ok[i] && !fits;
      // (a number that 32 bits do not hold is one that no free block has)
      a.first[r] = u32x2{upto[0] < kNoBlock ? static_cast<uint32_t>(upto[0]) : kNoBlock,
                         ok[i] && fits ? static_cast<uint32_t>(upto[1]) : kNoBlock};
      if (ok[i] && fits) pairs = static_cast<uint32_t>(upto[1] + copied[i]);
    }
    upto[0] += fresh[i];
    upto[1] += copied[i];
  }
  if (pairs) atomicMax(&most, pairs);
  if (bad) report(a.status, TUTTI_ST_BAD_EXTENT);
  __syncthreads();
  if (threadIdx.x == 0 && a.n_pairs) *a.n_pairs = most;
}

// The second: a chunk of a record's entries to a workgroup.  New block number k lies in the span whose free blocks are numbered around
// it: a search in LDS over the sums of the spans' counts.
__global__ __launch_bounds__(256) void k_blocks_fork(const ForkArgs a) {
  __shared__ uint32_t before[kMostSpans], sums[4];
  const uint32_t r = blockIdx.x / a.chunks, chunk = blockIdx.x - r * a.chunks;
  const u32x2 first = a.first[r];
  if (first[1] == kNoBlock) return;
  const Fork f = load_fork(a.forks + r);
  const uint32_t n = f.shared + f.fresh, begin = chunk * kChunk;
  if (begin >= n) return;
  uint32_t n_free = 0;
  if (f.fresh && (begin >= f.shared || f.shared - begin < kChunk)) n_free = add_up(a.spans, before, sums);
  uint32_t bad = 0;
#pragma unroll
  for (uint32_t i = 0; i < kChunk / 256; ++i) {
    const uint32_t e = begin + i * 256 + threadIdx.x;
    if (e >= n) break;
    const bool has_source = e < f.shared + f.copied, shared = e < f.shared;
    uint32_t id = kNoBlock, old = kNoBlock;
    if (has_source) {
      old = a.table[f.src + e];
      if (old >= a.spans.num_blocks) {
        if (old != kNoBlock) bad |= TUTTI_ST_BAD_BLOCK;
        old = kNoBlock;
      }
    }
    if (shared) {
      id = old;
    } else if (!has_source || old != kNoBlock) {
      const uint64_t number = static_cast<uint64_t>(first[0]) + (e - f.shared);
      if (number < n_free) {
        const uint32_t k = static_cast<uint32_t>(number);
        uint32_t lo = 0, hi = a.spans.n;  // the last span with before <= k
        while (hi - lo > 1) {
          const uint32_t mid = (lo + hi) / 2;
          if (before[mid] <= k)
            lo = mid;
          else
            hi = mid;
        }
        id = a.list[lo * a.spans.size + (k - before[lo])];
      } else {
        bad |= TUTTI_ST_NO_FREE;
      }
    }
    if (has_source && !shared)
      a.pairs[first[1] + (e - f.shared)] = id == kNoBlock ? tutti_block_pair{kNoBlock, kNoBlock} : tutti_block_pair{old, id};
    a.table[f.dst + e] = id;
    if (id != kNoBlock) atomicAdd(a.uses + id, 1u);
  }
  if (bad) report(a.status, bad);
}

// ---- free

struct FreeArgs {
  uint32_t *uses, *table;
  uint32_t num_blocks, table_len;
  const tutti_block_range *ranges;
  uint32_t n_ranges, max_entries, chunks;
  uint32_t *status;
};

// An entry is taken out of the table by an exchange, so that two ranges that both have it release its block once.
__global__ __launch_bounds__(256) void k_blocks_free(const FreeArgs a) {
  const uint32_t r = blockIdx.x / a.chunks, chunk = blockIdx.x - r * a.chunks;
  const u32x2 w = *reinterpret_cast<const u32x2 *>(a.ranges + r);
  const uint32_t n = w[1];
  if (n > a.max_entries || static_cast<uint64_t>(w[0]) + n > a.table_len) {
    if (chunk == 0 && threadIdx.x == 0) report(a.status, TUTTI_ST_BAD_EXTENT);
    return;
  }
  uint32_t bad = 0;
  uint32_t id[kChunk / 256], had[kChunk / 256];
#pragma unroll
  for (uint32_t i = 0; i < kChunk / 256; ++i) {
    const uint32_t e = chunk * kChunk + i * 256 + threadIdx.x;
    id[i] = e < n ? atomicExch(a.table + (w[0] + e), kNoBlock) : kNoBlock;
  }
#pragma unroll
  for (uint32_t i = 0; i < kChunk / 256; ++i) {
    had[i] = 1;
    if (id[i] < a.num_blocks)
      had[i] = atomicSub(a.uses + id[i], 1u);
    else if (id[i] != kNoBlock)
      bad |= TUTTI_ST_BAD_BLOCK;
  }
#pragma unroll
  for (uint32_t i = 0; i < kChunk / 256; ++i)
    if (static_cast<int32_t>(had[i]) <= 0) {
      // nothing was left to release: whoever finds that puts back what it took.  As many releases as there were uses find one, whatever
      // the order: the first that does not comes after all of them.
      atomicAdd(a.uses + id[i], 1u);
      bad |= TUTTI_ST_BAD_USES;
    }
  if (bad) report(a.status, bad);
}

// ---- compact

struct CompactArgs {
  Spans spans;
  uint32_t *uses, *table;
  uint32_t table_len;
  tutti_block_pair *pairs;
  uint32_t *totals;
  uint32_t max_pairs;
  uint32_t *holes;   // free blocks in front of the end, in order
  uint32_t *rank;    // of a used block behind the end: how many used ones are behind it; kNoBlock for free ones
  uint32_t *found;   // holes, used blocks
  uint32_t id_groups;
  uint32_t *status;
};

// Three launches: how many blocks of each span are used; where the used ones will end, the free blocks in front of that and
// the used ones behind; moves and tables.  The k-th used block from the back goes to the k-th free one from the front: either number
// follows from the sums of the spans in front, and a call that makes a few moves alone takes the last blocks first.
__global__ __launch_bounds__(256) void k_blocks_count_used(const CompactArgs a) {
  __shared__ uint32_t sums[4];
  const Spans &s = a.spans;
  const uint32_t begin = blockIdx.x * s.size;
  uint32_t mine = 0, all;
  for (uint32_t in = 0; in < s.size && in < s.num_blocks - begin; in += kChunk) {
    const u32x4 u = four_uses(s, begin + in + threadIdx.x * 4, 0);
    mine += (u[0] != 0) + (u[1] != 0) + (u[2] != 0) + (u[3] != 0);
  }
  sum_in_front(mine, sums, all);
  if (threadIdx.x == 0) s.counts[blockIdx.x] = all;
}

__global__ __launch_bounds__(256) void k_blocks_rank(const CompactArgs a) {
  __shared__ uint32_t before[kMostSpans], sums[4];
  const Spans &s = a.spans;
  const uint32_t end = add_up(s, before, sums), begin = blockIdx.x * s.size;
  uint32_t used = before[blockIdx.x];  // in front of the chunk
  if (blockIdx.x == 0 && threadIdx.x == 0 && end == 0) {
    a.found[0] = a.found[1] = 0;
    a.totals[0] = a.totals[1] = 0;
  }
  for (uint32_t in = 0; in < s.size && in < s.num_blocks - begin; in += kChunk) {
    const uint32_t id = begin + in + threadIdx.x * 4;
    const u32x4 u = four_uses(s, id, 0);
    const uint32_t mine = (u[0] != 0) + (u[1] != 0) + (u[2] != 0) + (u[3] != 0);
    uint32_t all, upto = used + sum_in_front(mine, sums, all);
    used += all;
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) {
      const uint32_t b = id + i;
      if (id >= s.num_blocks || i >= s.num_blocks - id) break;
      const bool is_used = u[i] != 0;
      if (b < end) {
        if (!is_used) a.holes[b - upto] = b;
      }
      upto += is_used;
      if (b >= end) a.rank[b] = is_used ? end - upto : kNoBlock;
      if (b + 1 == end) {  // the last place that will be used: the holes are all in front of it
        a.found[0] = end - upto;
        a.found[1] = end;
        a.totals[0] = min(end - upto, a.max_pairs);
        a.totals[1] = end;
      }
    }
  }
}

__global__ __launch_bounds__(256) void k_blocks_move(const CompactArgs a) {
  const uint32_t moves = min(a.found[0], a.max_pairs), end = a.found[1];
  if (blockIdx.x < a.id_groups) {
    // used blocks behind the end
    for (uint64_t at = static_cast<uint64_t>(blockIdx.x) * 256 + threadIdx.x + end; at < a.spans.num_blocks;
         at += static_cast<uint64_t>(a.id_groups) * 256) {
      const uint32_t b = static_cast<uint32_t>(at), r = a.rank[b];
      if (r >= moves) continue;
      const uint32_t to = a.holes[r];
      a.pairs[r] = tutti_block_pair{b, to};
      a.uses[to] = a.uses[b];
      a.uses[b] = 0;
    }
    return;
  }
  bool bad = false;
  const uint64_t groups = gridDim.x - a.id_groups;
  for (uint64_t e = static_cast<uint64_t>(blockIdx.x - a.id_groups) * 256 + threadIdx.x; e < a.table_len; e += groups * 256) {
    const uint32_t b = a.table[e];
    if (b >= a.spans.num_blocks) {
      bad |= b != kNoBlock;
    } else if (b >= end) {
      const uint32_t r = a.rank[b];
      if (r < moves) a.table[e] = a.holes[r];
    }
  }
  if (bad) report(a.status, TUTTI_ST_BAD_BLOCK);
}

// ---- copy

struct CopyArgs {
  uint8_t *planes[2];
  float *scales[2];
  uint64_t block_stride, scale_stride;
  uint32_t units, pieces;   // 16-byte units of a block; pieces of kPiece units
  uint32_t kv_heads, num_blocks;
  const tutti_block_pair *pairs;
  const uint32_t *n_pairs;
  uint32_t max_pairs;
  uint32_t *status;
};
constexpr uint32_t kPieceLoads = 4, kPiece = kPieceLoads * kLanes;

// A wavefront copies a piece of 4 KiB of one plane's block; neighbours have neighbouring pieces.
__global__ __launch_bounds__(256) void k_blocks_copy(const CopyArgs a) {
  const uint32_t lane = threadIdx.x & (kLanes - 1);
  const uint32_t n = a.n_pairs ? min(*constant(a.n_pairs), a.max_pairs) : a.max_pairs;
  const uint64_t jobs = static_cast<uint64_t>(n) * 2 * a.pieces;
  for (uint64_t job = static_cast<uint64_t>(blockIdx.x) * 4 + uniform(threadIdx.x / kLanes); job < jobs;
       job += static_cast<uint64_t>(gridDim.x) * 4) {
    const uint64_t row = job / a.pieces;
    const uint32_t piece = static_cast<uint32_t>(job - row * a.pieces), kind = row & 1u;
    const u32x2 pair = *constant(reinterpret_cast<const u32x2 *>(a.pairs + (row >> 1)));
    if (pair[0] >= a.num_blocks || pair[1] >= a.num_blocks) {
      if ((pair[0] & pair[1]) != kNoBlock && piece == 0 && lane == 0) report(a.status, TUTTI_ST_BAD_BLOCK);
      continue;
    }
    const uint8_t *from = a.planes[kind] + pair[0] * a.block_stride;
    uint8_t *to = a.planes[kind] + pair[1] * a.block_stride;
    u32x4 x[kPieceLoads];
#pragma unroll
    for (uint32_t i = 0; i < kPieceLoads; ++i) {
      const uint32_t unit = piece * kPiece + i * kLanes + lane;
      if (unit < a.units) x[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(from + static_cast<uint64_t>(unit) * 16));
    }
#pragma unroll
    for (uint32_t i = 0; i < kPieceLoads; ++i) {
      const uint32_t unit = piece * kPiece + i * kLanes + lane;
      if (unit < a.units) __builtin_nontemporal_store(x[i], reinterpret_cast<u32x4 *>(to + static_cast<uint64_t>(unit) * 16));
    }
    if (piece == 0 && a.scales[kind])
      for (uint32_t h = lane; h < a.kv_heads; h += kLanes)
        a.scales[kind][pair[1] * a.scale_stride + h] = a.scales[kind][pair[0] * a.scale_stride + h];
  }
}

}  // namespace tutti
