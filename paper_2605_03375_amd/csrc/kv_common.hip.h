// What the kernels that use a paged cache in place share: records, 16-bit and e4m3 types, and how a wavefront finds its work
// among the sequences of a step.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "tutti.h"

namespace tutti {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr uint32_t kLanes = 64;
// Stands for "nothing seen yet" in running maxima: finite, so that differences stay numbers, and no score that is finite is below it.
constexpr float kLowest = -__FLT_MAX__;

struct Fp16 {
  using one = _Float16;
  using two = f16x2;
  using eight = f16x8;
};
struct Bf16 {
  using one = __bf16;
  using two = bf16x2;
  using eight = bf16x8;
};

// Where the elements of a pool are.  Byte strides; shift: log2 of block_tokens, or 255 where that is no power of two.
struct PoolView {
  uint8_t *k, *v;
  uint64_t block_stride;
  uint32_t token_stride, head_stride;
  uint32_t num_blocks, block_tokens, shift;
  float *k_scale, *v_scale;
  uint64_t scale_stride;
};

struct BatchView {
  const tutti_seq *seqs;
  const uint32_t *table;
  uint32_t n_seq, max_new, table_len, n_rows;
};

// Memory that nobody writes while the kernel runs: a word of it at a wavefront's own address comes by the scalar path.
template <typename E>
__device__ __forceinline__ const __attribute__((address_space(4))) E *constant(const E *p) {
  return reinterpret_cast<const __attribute__((address_space(4))) E *>(reinterpret_cast<uintptr_t>(p));
}

// The kernel's arguments (its only one, a record) read from memory again: behind a long loop that is cheaper than scalar registers
// that hold them all the while, which the compiler would put away in vector registers.
template <typename Args>
__device__ __forceinline__ const __attribute__((address_space(4))) Args &arguments_again() {
  auto at = reinterpret_cast<uintptr_t>(__builtin_amdgcn_kernarg_segment_ptr());
  asm volatile("" : "+s"(at));
  return *reinterpret_cast<const __attribute__((address_space(4))) Args *>(at);
}

__device__ __forceinline__ void report(uint32_t *status, uint32_t bits) {
  if (status) atomicOr(status, bits);
}

__device__ __forceinline__ uint32_t block_of(const PoolView &p, uint32_t token) {
  return p.shift < 32 ? token >> p.shift : token / p.block_tokens;
}

__device__ __forceinline__ tutti_seq load_seq(const tutti_seq *s) {
  const u32x4 w = *reinterpret_cast<const u32x4 *>(s);
  return tutti_seq{w[0], w[1], w[2], w[3]};
}

__device__ __forceinline__ bool seq_ok(const BatchView &b, const tutti_seq &s) {
  return s.n_new <= b.max_new && s.n_new <= s.n_held && s.row0 <= b.n_rows && s.n_new <= b.n_rows - s.row0 &&
         s.n_held < 0x80000000u;
}

// The record at a wavefront's own address, by the scalar path.
__device__ __forceinline__ tutti_seq uniform_seq(const tutti_seq *s) {
  const u32x4 w = *constant(reinterpret_cast<const u32x4 *>(s));
  return tutti_seq{w[0], w[1], w[2], w[3]};
}

// Inclusive sum over the wavefront's lanes: data-parallel moves inside rows of 16 lanes, then across them.
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t moved_or_0(uint32_t v) {
  return static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), CTRL, ROWS, 0xf, false));
}
__device__ __forceinline__ uint32_t lane_prefix_sum(uint32_t v) {
  v += moved_or_0<0x111, 0xf>(v);
  v += moved_or_0<0x112, 0xf>(v);
  v += moved_or_0<0x114, 0xf>(v);
  v += moved_or_0<0x118, 0xf>(v);
  v += moved_or_0<0x142, 0xa>(v);
  v += moved_or_0<0x143, 0xc>(v);
  return v;
}
__device__ __forceinline__ uint32_t from_lane(uint32_t v, uint32_t lane) {
  return static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(v), static_cast<int>(lane)));
}
__device__ __forceinline__ uint32_t uniform(uint32_t v) {
  return static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(v)));
}

// Largest value over the lanes l, l^16, l^32, l^48: two register swaps, no trip through LDS.
__device__ __forceinline__ float max_over_rows(float x) {
  const uint32_t a = __float_as_uint(x);
  const auto p = __builtin_amdgcn_permlane16_swap(a, a, false, false);
  const uint32_t b = __float_as_uint(fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1])));
  const auto q = __builtin_amdgcn_permlane32_swap(b, b, false, false);
  return fmaxf(__uint_as_float(q[0]), __uint_as_float(q[1]));
}
__device__ __forceinline__ float sum_over_rows(float x) {
  const uint32_t a = __float_as_uint(x);
  const auto p = __builtin_amdgcn_permlane16_swap(a, a, false, false);
  const uint32_t b = __float_as_uint(__uint_as_float(p[0]) + __uint_as_float(p[1]));
  const auto q = __builtin_amdgcn_permlane32_swap(b, b, false, false);
  return __uint_as_float(q[0]) + __uint_as_float(q[1]);
}

struct Found {
  uint32_t seq;    // index, n_seq if there is no such unit
  uint32_t local;  // the unit's number within its sequence
  uint32_t total;  // units of all sequences (where asked for)
  tutti_seq s;
};

// The sequence that unit `unit` belongs to, if sequence s has count(s) units and they are numbered sequence by sequence.  Every
// lane of the wavefront has the same answer.  64 records are read and summed at a time; to_the_end: all of them, for the total
// and for the report of records that cannot be honoured.
template <typename Count>
__device__ __forceinline__ Found find_unit(const BatchView &b, uint32_t unit, bool to_the_end, uint32_t *status, Count count) {
  const uint32_t lane = threadIdx.x & (kLanes - 1);
  Found f{b.n_seq, 0, 0, {}};
  uint32_t before = 0;
  bool bad = false;
  for (uint32_t base = 0; base < b.n_seq; base += kLanes) {
    tutti_seq s{};
    uint32_t n = 0;
    if (base + lane < b.n_seq) {
      s = load_seq(b.seqs + base + lane);
      const bool ok = seq_ok(b, s);
      n = ok ? count(s) : 0;
      bad |= !ok;
    }
    const uint32_t upto = before + lane_prefix_sum(n);
    const uint64_t behind = __ballot(n != 0 && upto > unit);
    if (behind && f.seq == b.n_seq) {
      const uint32_t l = static_cast<uint32_t>(__builtin_ctzll(behind));
      f.seq = base + l;
      f.local = unit - (from_lane(upto, l) - from_lane(n, l));
      f.s = tutti_seq{from_lane(s.row0, l), from_lane(s.n_new, l), from_lane(s.n_held, l), from_lane(s.table_off, l)};
      if (!to_the_end) return f;
    }
    before = from_lane(upto, kLanes - 1);
  }
  f.total = before;
  if (to_the_end && __ballot(bad) && lane == 0) report(status, TUTTI_ST_BAD_EXTENT);
  return f;
}

}  // namespace tutti
