// Blocks of a paged cache shared, copied, given back and moved together: counts of uses, tables, and one layer's data.
#pragma once
#include "kv_common.hip.h"

namespace tutti {

constexpr uint32_t kNoBlock = TUTTI_NO_BLOCK;
constexpr uint32_t kChunk = 1024;    // counts that a workgroup of 256 takes at a time
constexpr uint32_t kEntries = 256;   // table entries of a record that a workgroup takes
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

// Which of a chunk's counts are 0 (or, `used`, not 0): 16 stretches of 64 blocks, of which wavefront w has 4, w and every fourth from there.
// A lane's bit of each, and how many come in front of it in the chunk; `stretches`: 16 words of LDS.  Behind the pool's end: none.
struct Marked {
  uint32_t bits, before[4], all;
  uint64_t found[4];  // the wavefront's stretches
};
struct Four {
  uint32_t x[4];
};
__device__ __forceinline__ Four chunk_uses(const Spans &s, uint32_t begin) {
  Four u;
#pragma unroll
  for (uint32_t i = 0; i < 4; ++i) {
    const uint32_t id = begin + i * 256 + threadIdx.x;
    u.x[i] = s.uses[min(id, s.num_blocks - 1)];
  }
  return u;
}
__device__ __forceinline__ Marked mark(const Spans &s, uint32_t begin, const Four &u, bool used, uint32_t *stretches) {
  const uint32_t lane = threadIdx.x & (kLanes - 1), wave = threadIdx.x / kLanes;
  Marked m{};
#pragma unroll
  for (uint32_t i = 0; i < 4; ++i) {
    const uint32_t id = begin + i * 256 + threadIdx.x;
    const bool is = id < s.num_blocks && (u.x[i] != 0) == used;
    m.found[i] = __ballot(is);
    m.bits |= static_cast<uint32_t>(is) << i;
  }
#pragma unroll
  for (uint32_t i = 0; i < 4; ++i) {
    m.before[i] = __builtin_amdgcn_mbcnt_hi(static_cast<uint32_t>(m.found[i] >> 32), __builtin_amdgcn_mbcnt_lo(static_cast<uint32_t>(m.found[i]), 0));
    if (lane == 0) stretches[i * 4 + wave] = static_cast<uint32_t>(__popcll(m.found[i]));
  }
  __syncthreads();
#pragma unroll
  for (uint32_t i = 0; i < 4; ++i) {
#pragma unroll
    for (uint32_t w = 0; w < 4; ++w) {
      if (w == wave) m.before[i] += m.all;
      m.all += stretches[i * 4 + w];
    }
  }
  __syncthreads();
  return m;
}

// A bit for each block of the chunk that was found: a stretch's are a word.
__device__ __forceinline__ void keep_bits(const Spans &s, uint32_t begin, const Marked &m, uint32_t *bits) {
  if (threadIdx.x & (kLanes - 1)) return;
#pragma unroll
  for (uint32_t i = 0; i < 4; ++i) {
    const uint32_t id = begin + i * 256 + threadIdx.x;
    if (id < s.num_blocks) *reinterpret_cast<uint64_t *>(bits + id / 32) = m.found[i];
  }
}

__device__ __forceinline__ bool bit_of(const uint32_t *bits, uint32_t id) { return bits[id / 32] >> (id % 32) & 1u; }

// counts_before[i] <- counts of the spans in front of span i (LDS, kMostSpans words); returns the sum of all.
__device__ __forceinline__ uint32_t add_up(const Spans &s, uint32_t *counts_before, uint32_t *sums) {
  // (there is room for kMostSpans counts; those behind the last span's are garbage)
  u32x4 c = *reinterpret_cast<const u32x4 *>(s.counts + threadIdx.x * 4);
  uint32_t mine = 0, all;
#pragma unroll
  for (uint32_t i = 0; i < 4; ++i) {
    if (threadIdx.x * 4 + i >= s.n) c[i] = 0;
    mine += c[i];
  }
  const uint32_t before = sum_in_front(mine, sums, all);
  *reinterpret_cast<u32x4 *>(counts_before + threadIdx.x * 4) = u32x4{before, before + c[0], before + c[0] + c[1], before + c[0] + c[1] + c[2]};
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
  uint32_t *free;      // a bit for each block: it is free when the call begins
  u32x2 *first;        // of each record: numbers of its first new block and its first pair; kNoBlock: the record is skipped
  uint32_t *status;
};

struct Fork {
  uint32_t src, dst, shared, copied, fresh;  // fresh: copied and new ones
};
// A record; false: one that cannot be honoured (n_pairs apart).
__device__ __forceinline__ bool make_fork(const ForkArgs &a, u32x4 w, uint32_t n_new, Fork &f) {
  const uint64_t old = static_cast<uint64_t>(w[2]) + w[3], all = old + n_new;
  f = Fork{w[0], w[1], w[2], w[3], w[3] + n_new};
  return all <= a.max_entries && w[1] + all <= a.table_len && (old == 0 || w[0] + old <= a.table_len);
}

// The first of two launches: workgroup i + 1 lists the free blocks of span i in order; the first numbers the records' new blocks and pairs.
// Bound by its trips to memory (counts, then sums in LDS).
__global__ __launch_bounds__(256) void k_blocks_list_free(const ForkArgs a) {
  const Spans &s = a.spans;
  if (blockIdx.x) {
    __shared__ uint32_t stretches[16];
    uint32_t n = 0;
    const uint32_t begin = (blockIdx.x - 1) * s.size;
    for (uint32_t in = 0; in < s.size && in < s.num_blocks - begin; in += kChunk) {
      const Marked m = mark(s, begin + in, chunk_uses(s, begin + in), false, stretches);
#pragma unroll
      for (uint32_t i = 0; i < 4; ++i)
        if (m.bits >> i & 1u) a.list[begin + n + m.before[i]] = begin + in + i * 256 + threadIdx.x;
      keep_bits(s, begin + in, m, a.free);
      n += m.all;
    }
    if (threadIdx.x == 0) s.counts[blockIdx.x - 1] = n;
    return;
  }
  // records, 256 neighbours at a time.  Sums of up to 2048 numbers below 2^31, in halves of 16 bits, whose sums 32 bits hold.
  constexpr uint32_t EACH = TUTTI_MAX_REQ / 256;
  __shared__ uint32_t halves[4][4];
  const uint32_t lane = threadIdx.x & (kLanes - 1), wave = threadIdx.x / kLanes;
  uint32_t fresh[EACH], copied[EACH], n_new[EACH];
  u32x4 w[EACH];
  bool ok[EACH], bad = false;
#pragma unroll
  for (uint32_t i = 0; i < EACH; ++i) {
    if (i * 256 >= a.n_forks) break;
    const tutti_fork *f = a.forks + min(i * 256 + threadIdx.x, a.n_forks - 1);
    w[i] = *reinterpret_cast<const u32x4 *>(f);
    n_new[i] = f->n_new;
  }
#pragma unroll
  for (uint32_t i = 0; i < EACH; ++i) {
    const uint32_t r = i * 256 + threadIdx.x;
    if (i * 256 >= a.n_forks) break;
    Fork f;
    ok[i] = make_fork(a, w[i], n_new[i], f) && r < a.n_forks;
    bad |= r < a.n_forks && !ok[i];
    fresh[i] = ok[i] ? f.fresh : 0;
    copied[i] = ok[i] ? f.copied : 0;
  }
  uint64_t before[2] = {0, 0};  // of the records of earlier turns
  uint32_t pairs = 0;
#pragma unroll
  for (uint32_t i = 0; i < EACH; ++i) {
    const uint32_t r = i * 256 + threadIdx.x;
    if (i * 256 >= a.n_forks) break;
    const uint32_t x[4] = {fresh[i] & 0xffffu, fresh[i] >> 16, copied[i] & 0xffffu, copied[i] >> 16};
    uint32_t upto[4];
#pragma unroll
    for (int h = 0; h < 4; ++h) {
      upto[h] = lane_prefix_sum(x[h]);
      if (lane == kLanes - 1) halves[h][wave] = upto[h];
    }
    __syncthreads();
    uint32_t all[4] = {0, 0, 0, 0};
#pragma unroll
    for (int h = 0; h < 4; ++h) {
      upto[h] -= x[h];
#pragma unroll
      for (uint32_t w = 0; w < 4; ++w) {
        if (w < wave) upto[h] += halves[h][w];
        all[h] += halves[h][w];
      }
    }
    __syncthreads();
    const uint64_t number = before[0] + (static_cast<uint64_t>(upto[1]) << 16) + upto[0];
    const uint64_t pair = before[1] + (static_cast<uint64_t>(upto[3]) << 16) + upto[2];
    const bool fits = pair + copied[i] <= a.max_pairs;
    if (r < a.n_forks) {
      bad |= ok[i] && !fits;
      // (a number that 32 bits do not hold is one that no free block has)
      a.first[r] = u32x2{number < kNoBlock ? static_cast<uint32_t>(number) : kNoBlock,
                         ok[i] && fits ? static_cast<uint32_t>(pair) : kNoBlock};
      if (ok[i] && fits) pairs = static_cast<uint32_t>(pair + copied[i]);
    }
    before[0] += (static_cast<uint64_t>(all[1]) << 16) + all[0];
    before[1] += (static_cast<uint64_t>(all[3]) << 16) + all[2];
  }
  if (bad) report(a.status, TUTTI_ST_BAD_EXTENT);
  // as many pairs as the last record that fits has behind it
#pragma unroll
  for (int m = 1; m < static_cast<int>(kLanes); m <<= 1) pairs = max(pairs, static_cast<uint32_t>(__shfl_xor(static_cast<int>(pairs), m, kLanes)));
  if (lane == 0) halves[0][wave] = pairs;
  __syncthreads();
  if (threadIdx.x == 0 && a.n_pairs) *a.n_pairs = max(max(halves[0][0], halves[0][1]), max(halves[0][2], halves[0][3]));
}

// Uses that a thread adds to (takes from) a block: those of neighbouring records that name the same block at the same place, as samples of
// one prompt do, go together.  Blocks' counts lie all over memory, and the device makes 27 such additions a nanosecond: 1,024 sequences of
// 515,000 entries, groups of 8 that share their prompts, 24.4 us one by one, 10.0 so (and 0.5 for the bits of free blocks, which came
// later); 384 sequences given back, 32.7 and 11.8.
struct Run {
  uint32_t id, n;
};

// What an entry of a record needs: the source's block (kNoBlock: none), and the number of a new block.
struct Entry {
  uint32_t old, bad;
  bool takes;       // a new block, if there is one
  uint64_t number;
};
// A source's entry that names a free block is taken as one that names none: the call may give that block to another sequence.
__device__ __forceinline__ uint32_t leave_out(uint32_t &old, uint32_t &id) {
  old = id = kNoBlock;
  return TUTTI_ST_BAD_USES;
}
__device__ __forceinline__ Entry entry_of(const ForkArgs &a, const Fork &f, u32x2 first, uint32_t e, uint32_t old) {
  const bool has_source = e < f.shared + f.copied;
  Entry x{has_source ? old : kNoBlock, 0, false, 0};
  if (x.old >= a.spans.num_blocks) {
    if (x.old != kNoBlock) x.bad = TUTTI_ST_BAD_BLOCK;
    x.old = kNoBlock;
  }
  x.takes = e >= f.shared && e < f.shared + f.fresh && (!has_source || x.old != kNoBlock);
  x.number = static_cast<uint64_t>(first[0]) + (e - f.shared);
  return x;
}
// Writes the entry, and the pair of one that is copied; `id`: the new block.  Returns the entry's block.
__device__ __forceinline__ uint32_t put_entry(const ForkArgs &a, const Fork &f, u32x2 first, uint32_t e, uint32_t old, uint32_t id) {
  if (e < f.shared) id = old;
  if (e >= f.shared && e < f.shared + f.copied)
    a.pairs[first[1] + (e - f.shared)] = id == kNoBlock ? tutti_block_pair{kNoBlock, kNoBlock} : tutti_block_pair{old, id};
  a.table[f.dst + e] = id;
  return id;
}

// The second: the same chunk of entries of kGroup neighbouring records to a workgroup.  New block number k lies in the span whose free
// blocks are numbered around it: a search in LDS over the sums of the spans' counts.
constexpr uint32_t kGroup = 4;   // (the 1,024 sequences, without the bits: 4 together 10.0 us, 8 11.5, 16 18.8)
__global__ __launch_bounds__(256) void k_blocks_fork(const ForkArgs a) {
  __shared__ __attribute__((aligned(16))) uint32_t before[kMostSpans];
  __shared__ uint32_t sums[4];
  const uint32_t group = blockIdx.x / a.chunks, chunk = blockIdx.x - group * a.chunks, begin = chunk * kEntries, e = begin + threadIdx.x;
  Fork f[kGroup];
  u32x2 first[kGroup];
  uint32_t old[kGroup];
  bool counts = false;  // a record has new blocks in this chunk
#pragma unroll
  for (uint32_t g = 0; g < kGroup; ++g) {
    const uint32_t r = min(group * kGroup + g, a.n_forks - 1);
    const u32x4 w = *constant(reinterpret_cast<const u32x4 *>(a.forks + r));
    f[g] = Fork{w[0], w[1], w[2], w[3], w[3] + constant(a.forks + r)->n_new};
    first[g] = *constant(a.first + r);
  }
#pragma unroll
  for (uint32_t g = 0; g < kGroup; ++g) {
    if (group * kGroup + g >= a.n_forks || first[g][1] == kNoBlock) f[g] = Fork{};
    old[g] = kNoBlock;
    if (e < f[g].shared + f[g].copied) old[g] = a.table[f[g].src + e];
    counts |= begin < f[g].shared + f[g].fresh && (begin >= f[g].shared || f[g].shared - begin < kEntries) && f[g].fresh != 0;
  }
  uint32_t n_free = 0, bad = 0, id[kGroup];
  if (counts) n_free = add_up(a.spans, before, sums);
  uint32_t number[kGroup], span[kGroup];  // of the new block; where it is listed
  bool takes[kGroup], is_free[kGroup];
#pragma unroll
  for (uint32_t g = 0; g < kGroup; ++g) {
    const Entry x = entry_of(a, f[g], first[g], e, old[g]);
    old[g] = x.old;
    bad |= x.bad;
    number[g] = x.takes && x.number < n_free ? static_cast<uint32_t>(x.number) : kNoBlock;
    takes[g] = x.takes;
    span[g] = 0;
  }
  if (counts) {
    // the last span with before <= number, for all at once (behind the spans lies the sum of all, which no number reaches)
    for (uint32_t step = kMostSpans / 2; step; step >>= 1) {
      if (step >= a.spans.n) continue;
      uint32_t there[kGroup];
#pragma unroll
      for (uint32_t g = 0; g < kGroup; ++g) there[g] = before[span[g] + step];
#pragma unroll
      for (uint32_t g = 0; g < kGroup; ++g) span[g] += there[g] <= number[g] ? step : 0;
    }
  }
#pragma unroll
  for (uint32_t g = 0; g < kGroup; ++g) {
    id[g] = kNoBlock;
    // (the counts grow while this runs.  Loads beside those of the list: no trip to memory more)
    is_free[g] = bit_of(a.free, min(old[g], a.spans.num_blocks - 1)) && old[g] != kNoBlock;
    if (number[g] != kNoBlock) id[g] = a.list[span[g] * a.spans.size + (number[g] - before[span[g]])];
  }
  Run run{kNoBlock, 0};
#pragma unroll
  for (uint32_t g = 0; g < kGroup; ++g) {
    if (e >= f[g].shared + f[g].fresh) continue;
    if (is_free[g])
      bad |= leave_out(old[g], id[g]);
    else if (takes[g] && id[g] == kNoBlock)
      bad |= TUTTI_ST_NO_FREE;
    id[g] = put_entry(a, f[g], first[g], e, old[g], id[g]);
    if (id[g] != run.id) {
      if (run.id != kNoBlock) atomicAdd(a.uses + run.id, run.n);
      run = Run{id[g], 0};
    }
    ++run.n;
  }
  if (run.id != kNoBlock) atomicAdd(a.uses + run.id, run.n);
  if (bad) report(a.status, bad);
}

// Both in one workgroup, for the few entries of a step in which sequences begin blocks or beams change places: no second launch.  Counts are
// read until there are enough free blocks, 16,384 at a time, so the pool's size matters where the free ones lie at its end.  4 records of
// 64 entries, with the copy of the state in front of it, in one launch and in two, us: free blocks everywhere, pools of 32,768 and 65,536
// blocks 8.4 and 9.9, of 131,072 8.2 and 10.1, of a million 8.4 and 12.2; free blocks at the end alone, 32,768 10.3 and 9.7, 65,536 15.3
// and 10.2, 131,072 26 and 10.1, a million 170 and 11.8.  So up to 65,536, where a pool that is all but full loses 5 and any other gains
// 1.6.  Bound by its trips to memory: records and counts, tables, whether the sources' blocks have uses, and what is written.
constexpr uint32_t kSmallEntries = 4096, kSmallRecords = 1024, kSmallBlocks = 65536;
__global__ __launch_bounds__(1024) void k_blocks_fork_small(const ForkArgs a) {
  __shared__ Fork records[kSmallRecords];
  __shared__ u32x2 firsts[kSmallRecords];
  __shared__ uint32_t list[kSmallEntries], sums[4][16], most[16];
  const uint32_t lane = threadIdx.x & (kLanes - 1), wave = threadIdx.x / kLanes;
  u32x4 u[4];
#pragma unroll
  for (uint32_t i = 0; i < 4; ++i) u[i] = four_uses(a.spans, i * 4096 + threadIdx.x * 4, 1);
  Fork f{};
  bool ok = false;
  if (threadIdx.x < a.n_forks) {
    ok = make_fork(a, *reinterpret_cast<const u32x4 *>(a.forks + threadIdx.x), a.forks[threadIdx.x].n_new, f);
    if (!ok) f = Fork{};
  }
  // (entries are kSmallEntries at most, and so are the sums)
  uint32_t upto[2] = {lane_prefix_sum(f.fresh), lane_prefix_sum(f.copied)}, wanted = 0;
  if (lane == kLanes - 1) {
    sums[0][wave] = upto[0];
    sums[1][wave] = upto[1];
  }
  __syncthreads();
#pragma unroll
  for (uint32_t w = 0; w < 16; ++w) {
    if (w < wave) {
      upto[0] += sums[0][w];
      upto[1] += sums[1][w];
    }
    wanted += sums[0][w];
  }
  const bool fits = ok && upto[1] <= a.max_pairs;
  uint32_t bad = threadIdx.x < a.n_forks && !fits ? TUTTI_ST_BAD_EXTENT : 0;
  records[threadIdx.x] = f;
  firsts[threadIdx.x] = u32x2{upto[0] - f.fresh, fits ? upto[1] - f.copied : kNoBlock};
  const uint64_t some = __ballot(fits);  // as many pairs as the last record that fits has behind it
  if (lane == 0) most[wave] = some ? from_lane(upto[1], 63 - static_cast<uint32_t>(__builtin_clzll(some))) : 0;
  __syncthreads();
  // what the sources name, under the search for free blocks
  constexpr uint32_t ITEMS = kSmallEntries / 1024;
  uint32_t old[ITEMS], of[ITEMS];
  bool is_free[ITEMS];
#pragma unroll
  for (uint32_t i = 0; i < ITEMS; ++i) {
    const uint32_t x = i * 1024 + threadIdx.x;
    old[i] = of[i] = kNoBlock;
    if (x >= a.n_forks * a.max_entries) continue;
    const uint32_t r = x / a.max_entries, e = x - r * a.max_entries;
    if (firsts[r][1] == kNoBlock || e >= records[r].shared + records[r].fresh) continue;
    of[i] = r;
    if (e < records[r].shared + records[r].copied) old[i] = a.table[records[r].src + e];
  }
  uint32_t n_free = 0;
  for (uint32_t begin = 0; begin < a.spans.num_blocks && n_free < wanted; begin += 4 * 4096) {
    uint32_t mine[4], at[4];
    if (begin) {
#pragma unroll
      for (uint32_t i = 0; i < 4; ++i) u[i] = four_uses(a.spans, begin + i * 4096 + threadIdx.x * 4, 1);
      __syncthreads();  // (what was in `sums` has been read)
    }
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) {
      mine[i] = (u[i][0] == 0) + (u[i][1] == 0) + (u[i][2] == 0) + (u[i][3] == 0);
      at[i] = lane_prefix_sum(mine[i]);
      if (lane == kLanes - 1) sums[i][wave] = at[i];
    }
    __syncthreads();
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) {
      at[i] += n_free - mine[i];
#pragma unroll
      for (uint32_t w = 0; w < 16; ++w) {
        if (w < wave) at[i] += sums[i][w];
        n_free += sums[i][w];
      }
#pragma unroll
      for (uint32_t x = 0; x < 4; ++x)
        if (u[i][x] == 0) {
          if (at[i] < wanted) list[at[i]] = begin + i * 4096 + threadIdx.x * 4 + x;
          ++at[i];
        }
    }
  }
  // (before anybody's count grows; here the tables' entries have come under the search: 0.3 us less than in front of it)
#pragma unroll
  for (uint32_t i = 0; i < ITEMS; ++i) is_free[i] = a.uses[min(old[i], a.spans.num_blocks - 1)] == 0 && old[i] < a.spans.num_blocks;
  __syncthreads();
  if (threadIdx.x == 0 && a.n_pairs) {
    uint32_t n = 0;
#pragma unroll
    for (uint32_t w = 0; w < 16; ++w) n = max(n, most[w]);
    *a.n_pairs = n;
  }
#pragma unroll
  for (uint32_t i = 0; i < ITEMS; ++i) {
    const uint32_t r = of[i];
    if (r == kNoBlock) continue;
    const uint32_t e = i * 1024 + threadIdx.x - r * a.max_entries;
    Entry x = entry_of(a, records[r], firsts[r], e, old[i]);
    bad |= x.bad;
    uint32_t id = x.takes && x.number < n_free ? list[x.number] : kNoBlock;
    if (is_free[i])
      bad |= leave_out(x.old, id);
    else if (x.takes && id == kNoBlock)
      bad |= TUTTI_ST_NO_FREE;
    id = put_entry(a, records[r], firsts[r], e, x.old, id);
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

// An entry is taken out of the table by an exchange, so that two ranges that both have it release its block once (96 x 4 sequences, 747,000
// entries, each block released by itself: 32.7 us, with loads and stores 31.5).  Neighbouring ranges to a workgroup: see Run.
template <uint32_t kGroup>
__global__ __launch_bounds__(256) void k_blocks_free(const FreeArgs a) {
  const uint32_t group = blockIdx.x / a.chunks, e = (blockIdx.x - group * a.chunks) * kEntries + threadIdx.x;
  uint32_t bad = 0, id[kGroup];
  u32x2 w[kGroup];
#pragma unroll
  for (uint32_t g = 0; g < kGroup; ++g)
    w[g] = *constant(reinterpret_cast<const u32x2 *>(a.ranges + min(group * kGroup + g, a.n_ranges - 1)));
#pragma unroll
  for (uint32_t g = 0; g < kGroup; ++g) {
    id[g] = kNoBlock;
    if (group * kGroup + g >= a.n_ranges) continue;
    if (w[g][1] > a.max_entries || static_cast<uint64_t>(w[g][0]) + w[g][1] > a.table_len)
      bad |= TUTTI_ST_BAD_EXTENT;
    else if (e < w[g][1])
      id[g] = atomicExch(a.table + (w[g][0] + e), kNoBlock);
  }
  Run run[kGroup];  // run[g].n > 0: a run ends with range g
#pragma unroll
  for (uint32_t g = 0; g < kGroup; ++g) {
    if (id[g] >= a.num_blocks && id[g] != kNoBlock) {
      bad |= TUTTI_ST_BAD_BLOCK;
      id[g] = kNoBlock;
    }
    run[g] = Run{id[g], id[g] != kNoBlock};
    if (g && id[g] == id[g - 1]) {
      run[g].n += run[g - 1].n;
      run[g - 1].n = 0;
    }
  }
  uint32_t had[kGroup];
#pragma unroll
  for (uint32_t g = 0; g < kGroup; ++g) had[g] = run[g].n ? atomicSub(a.uses + run[g].id, run[g].n) : 0;
#pragma unroll
  for (uint32_t g = 0; g < kGroup; ++g) {
    const int32_t left = static_cast<int32_t>(had[g]), n = static_cast<int32_t>(run[g].n);
    if (left < n) {
      // More was taken than there was: whoever finds that puts the rest back.  The first who does has taken the last use, so that nobody
      // after that finds any: what is released in all, and whether it is too much, does not go by the order.
      atomicAdd(a.uses + run[g].id, static_cast<uint32_t>(n - max(left, 0)));
      bad |= TUTTI_ST_BAD_USES;
    }
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
  uint32_t *used;    // a bit for each block; behind `rank`, `used_at` words from there
  uint32_t used_at;
  uint32_t *found;   // holes, used blocks
  uint32_t table_groups;
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
  __shared__ __attribute__((aligned(16))) uint32_t before[kMostSpans];
  __shared__ uint32_t sums[4];
  const Spans &s = a.spans;
  const uint32_t begin = blockIdx.x * s.size;
  Four u = chunk_uses(s, begin);
  const uint32_t end = add_up(s, before, sums);
  __shared__ uint32_t stretches[16];
  uint32_t used = before[blockIdx.x];  // in front of the chunk
  if (blockIdx.x == 0 && threadIdx.x == 0 && end == 0) {
    a.found[0] = a.found[1] = 0;
    a.totals[0] = a.totals[1] = 0;
  }
  for (uint32_t in = 0; in < s.size && in < s.num_blocks - begin; in += kChunk) {
    if (in) u = chunk_uses(s, begin + in);
    const Marked m = mark(s, begin + in, u, true, stretches);
    keep_bits(s, begin + in, m, a.used);
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) {
      const uint32_t b = begin + in + i * 256 + threadIdx.x;
      if (b >= s.num_blocks) break;
      const bool is_used = m.bits >> i & 1u;
      const uint32_t upto = used + m.before[i] + is_used;
      if (b >= end)
        a.rank[b] = is_used ? end - upto : kNoBlock;
      else if (!is_used)
        a.holes[b - upto] = b;
      if (b + 1 == end) {  // the last place that will be used: the holes are all in front of it
        a.found[0] = end - upto;
        a.found[1] = end;
        a.totals[0] = min(end - upto, a.max_pairs);
        a.totals[1] = end;
      }
    }
    used += m.all;
  }
}

__global__ __launch_bounds__(256) void k_blocks_move(const CompactArgs a) {
  const uint32_t moves = min(a.found[0], a.max_pairs), end = a.found[1];
  // Four things a thread at a time, apart by the grid's width: what an entry names, where that is listed and where it goes are trips to
  // memory one after the other.
  if (blockIdx.x < a.table_groups) {
    uint32_t bad = 0;
    const uint64_t step = static_cast<uint64_t>(a.table_groups) * 256;
    for (uint64_t from = static_cast<uint64_t>(blockIdx.x) * 256 + threadIdx.x; from < a.table_len; from += 4 * step) {
      uint32_t b[4], r[4];
#pragma unroll
      for (uint32_t i = 0; i < 4; ++i) b[i] = from + i * step < a.table_len ? a.table[from + i * step] : kNoBlock;
#pragma unroll
      for (uint32_t i = 0; i < 4; ++i) {
        if (b[i] >= a.spans.num_blocks && b[i] != kNoBlock) bad |= TUTTI_ST_BAD_BLOCK;
        // a block's rank or its word of bits: one load.  (The words of those in front of the end: 1.2 us of the pass over a million blocks.)
        r[i] = b[i] < a.spans.num_blocks ? a.rank[b[i] >= end ? b[i] : a.used_at + b[i] / 32] : kNoBlock;
      }
#pragma unroll
      for (uint32_t i = 0; i < 4; ++i) {
        if (b[i] < end) {
          // an entry that names a hole must not name what moves there
          if (!(r[i] >> (b[i] % 32) & 1u)) {
            a.table[from + i * step] = kNoBlock;
            bad |= TUTTI_ST_BAD_USES;
          }
        } else if (r[i] < moves) {
          a.table[from + i * step] = a.holes[r[i]];
        }
      }
    }
    if (bad) report(a.status, bad);
    return;
  }
  // used blocks behind the end
  const uint64_t step = static_cast<uint64_t>(gridDim.x - a.table_groups) * 256;
  for (uint64_t from = static_cast<uint64_t>(blockIdx.x - a.table_groups) * 256 + threadIdx.x + end; from < a.spans.num_blocks; from += 4 * step) {
    uint32_t r[4], to[4], n[4];
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) r[i] = from + i * step < a.spans.num_blocks ? a.rank[from + i * step] : kNoBlock;
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i)
      if (r[i] < moves) {
        to[i] = a.holes[r[i]];
        n[i] = a.uses[from + i * step];
      }
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i)
      if (r[i] < moves) {
        const uint32_t b = static_cast<uint32_t>(from + i * step);
        a.pairs[r[i]] = tutti_block_pair{b, to[i]};
        a.uses[to[i]] = n[i];
        a.uses[b] = 0;
      }
  }
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
  uint32_t step_rows, step_pieces;   // the grid's wavefronts: so many rows and pieces
  uint32_t *status;
};
constexpr uint32_t kPieceLoads = 4, kPiece = kPieceLoads * kLanes;

// A wavefront copies a piece of 4 KiB of one plane's block; neighbours have neighbouring pieces.  Bound by memory: 6,001 blocks of 32 KiB a
// plane, 787 MB read and written, in 157 us, 5.0 TB/s (a contiguous copy of 1 GiB by PyTorch: 5.14).  72 registers: seven workgroups a
// compute unit at once.
__global__ __launch_bounds__(256) void k_blocks_copy(const CopyArgs a) {
  const uint32_t lane = threadIdx.x & (kLanes - 1);
  const uint32_t n = a.n_pairs ? min(*constant(a.n_pairs), a.max_pairs) : a.max_pairs;
  const uint32_t wave = blockIdx.x * 4 + uniform(threadIdx.x / kLanes);
  // row of pair and plane, piece of it: the first, then as many further on as there are wavefronts
  uint64_t row = wave / a.pieces;
  uint32_t piece = wave - static_cast<uint32_t>(row) * a.pieces;
  for (; row < 2ull * n; row += a.step_rows, piece += a.step_pieces) {
    if (piece >= a.pieces) {
      piece -= a.pieces;
      if (++row >= 2ull * n) break;
    }
    const uint32_t kind = row & 1u;
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
