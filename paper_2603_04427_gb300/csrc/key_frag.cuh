// Cached keys as operands of mma.sync.m16n8k16, straight from global memory, and
// where a token's slot is.  Shared by the operators over a long context.
#pragma once

#include "common.cuh"
#include "longctx.h"
#include "widen.cuh"

namespace tk {

// Row of token t of (sequence b, kv head g); t is within SlotMap::limit.  A page
// id out of range is recorded and read as page 0.
__device__ __forceinline__ long long slot_row(const SlotMap& m, int b, int g, int t) {
  if (m.page_size == 0) return (static_cast<long long>(b) * m.Hkv + g) * m.capacity + t;
  int page = m.page_table[static_cast<long long>(b) * m.max_pages + (t >> m.page_shift)];
  if (page < 0 || page >= m.num_pages) {
    record_error(m.err, TK_DEVERR_INDEX);
    page = 0;
  }
  return (static_cast<long long>(page) * m.Hkv + g) * m.page_size + (t & (m.page_size - 1));
}

// The same for a row that is written, with the table's entry in hand: -1 for a bad page.
__device__ __forceinline__ long long slot_of_page(const SlotMap& m, int b, int g, int page, int t) {
  if (m.page_size == 0) return (static_cast<long long>(b) * m.Hkv + g) * m.capacity + t;
  if (page < 0 || page >= m.num_pages) {
    record_error(m.err, TK_DEVERR_INDEX);
    return -1;
  }
  return (static_cast<long long>(page) * m.Hkv + g) * m.page_size + (t & (m.page_size - 1));
}

__device__ __forceinline__ long long slot_row_or_none(const SlotMap& m, int b, int g, int t) {
  const int page = m.page_size == 0 ? 0 : m.page_table[static_cast<long long>(b) * m.max_pages + (t >> m.page_shift)];
  return slot_of_page(m, b, g, page, t);
}

// A context length, clamped into what the cache can hold.
__device__ __forceinline__ int checked_len(int L, const SlotMap& m) {
  if (L >= 0 && L <= m.limit) return L;
  record_error(m.err, TK_DEVERR_INDEX);
  return L < 0 ? 0 : m.limit;
}

__device__ __forceinline__ void mma_bf16(float* d, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                         uint32_t b0, uint32_t b1) {
  asm(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, "
      "{%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// The same onto zeros.
__device__ __forceinline__ void mma_bf16_first(float* d, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                               uint32_t b0, uint32_t b1) {
  asm(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, "
      "{%8,%9}, {%10,%10,%10,%10};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}

// One row's share of lane t (of the four that hold a row): with k in an order
// of our own, elements 8 c .. 8 c + 7 of every 32 (c = t) are the k indices 2t,
// 2t+1, 2t+8, 2t+9 of two consecutive steps of 16, so a lane's elements are
// contiguous: 16 bytes of bf16, 8 of int8 or 4 of int4 for 32 elements.  r = 16 is
// one step: elements 4t .. 4t+3.  The other operand uses the same order.
template <int R, int KF>
struct KeyRow {
  static constexpr int STEPS = R / 16;
  static constexpr int BYTES = KF == 0 ? 2 * R : (KF == 1 ? R : R / 2);   // of a row
  static constexpr int WORDS = BYTES / 16;    // 32-bit words of a lane (4 lanes a row)
  static constexpr int GROUPS = R >= 32 ? R / 32 : 1;
  uint32_t w[WORDS];

  // From a row that is in shared memory.
  __device__ __forceinline__ void load(const unsigned char* row, int t) {
    constexpr int PER = WORDS / GROUPS;       // words of a lane in a group of 32 (16 for r = 16)
#pragma unroll
    for (int j = 0; j < GROUPS; ++j) {
      const unsigned char* s = row + j * (BYTES / GROUPS) + t * PER * 4;
      if constexpr (PER == 4) {
        const uint4 x = *reinterpret_cast<const uint4*>(s);
        w[4 * j] = x.x; w[4 * j + 1] = x.y; w[4 * j + 2] = x.z; w[4 * j + 3] = x.w;
      } else if constexpr (PER == 2) {
        const uint2 x = *reinterpret_cast<const uint2*>(s);
        w[2 * j] = x.x; w[2 * j + 1] = x.y;
      } else {
        w[j] = *reinterpret_cast<const uint32_t*>(s);
      }
    }
  }

  // bf16 pairs of step s: (k 2t, 2t+1) and (k 2t+8, 2t+9); codes are widened exactly.
  __device__ __forceinline__ void steps(uint32_t (&lo)[STEPS], uint32_t (&hi)[STEPS]) const {
    if constexpr (KF == 0) {
#pragma unroll
      for (int s = 0; s < STEPS; ++s) lo[s] = w[2 * s], hi[s] = w[2 * s + 1];
    } else if constexpr (KF == 1) {
#pragma unroll
      for (int s = 0; s < STEPS; ++s) i8x4_to_bf16(w[s], lo[s], hi[s]);
    } else {
#pragma unroll
      for (int j = 0; j < STEPS / 2; ++j) i4x8_to_bf16(w[j], lo[2 * j], hi[2 * j], lo[2 * j + 1], hi[2 * j + 1]);
    }
  }
};

// First element of lane t's four of step s, in the order of KeyRow.
template <int R>
__device__ __forceinline__ int step_element(int s, int t) {
  return R >= 32 ? (s >> 1) * 32 + 8 * t + (s & 1) * 4 : 4 * t;
}

}  // namespace tk
