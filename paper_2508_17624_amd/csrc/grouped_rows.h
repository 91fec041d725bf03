// Rows sorted by slot, as the permutation leaves them: finding a workgroup's share of them on the device.
//
// The host knows only the number of rows and slots, so a launch over row chunks has as many workgroups as there can be chunks
// and each finds its own: no plan in memory, no launch before the first product, nothing that two calls could share.
#pragma once
#include "ew_internal.h"

namespace ew {

struct GroupedRows {
  const int32_t* counts;   // [P] rows per slot
  const int32_t* offsets;  // [P+1]
  const int32_t* por;      // row -> pair, or NULL: row r is pair r
  int P, rows, k;          // rows: room for sorted rows; offsets[P] of them exist
};

struct RowChunk {
  int slot, first, rows;   // slot < 0: there is no such chunk
};

// Most row chunks of at most B rows that `rows` rows in P slots can make.
inline long long max_chunks(long long rows, long long P, int B) {
  const long long used = P < rows ? P : rows;
  return (rows - used) / B + used;
}

// Rows per chunk of a slot with c rows where a chunk may have B: the least number of chunks, of about equal size, multiples of A.
template <int B, int A>
__device__ __forceinline__ int chunk_rows(int c) {
  const int n = (c + B - 1) / B;
  return n <= 1 ? B : ((c + n - 1) / n + A - 1) / A * A;
}

// Chunks of all slots.  Every lane gets the answer.
template <int B>
__device__ __forceinline__ int count_chunks(const GroupedRows& g) {
  int sum = 0;
  for (int s = threadIdx.x & 63; s < g.P; s += 64) sum += (g.counts[s] + B - 1) / B;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
  return __builtin_amdgcn_readfirstlane(sum);
}

// Workgroups go round the eight XCDs, each with an L2 of its own: unit `i` of `n` for this one so that an XCD works on one run of
// neighbouring units (which share weights and rows).  Returns n where there is none left.
__device__ __forceinline__ int unit_of_block(int n) {
  const int per = (n + 7) / 8, i = (int)blockIdx.x >> 3, x = (int)blockIdx.x & 7;
  return i < per ? min(n, x * per + i) : n;
}

// The chunk number `want` of all slots' chunks in slot order.  Every lane of the wave gets the same answer.  A lane looks at 8 slots,
// the lanes' sums meet in one scan: two dependent round trips to L2 for up to 512 slots (about 1.5 us), the same for every chunk.
template <int B, int A>
__device__ __forceinline__ RowChunk find_chunk(const GroupedRows& g, int want) {
  const int lane = threadIdx.x & 63;
  for (int base = 0; base < g.P; base += 512) {
    int c[8], sum = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int s = base + 8 * lane + i;
      c[i] = s < g.P ? g.counts[s] : 0;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) sum += (c[i] + B - 1) / B;
    int incl = sum;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int v = __shfl_up(incl, o, 64);
      if (lane >= o) incl += v;
    }
    const int total = __builtin_amdgcn_readlane(incl, 63);
    if (want < total) {
      const int l = __ffsll((long long)__ballot(want < incl)) - 1;
      int left = want - (incl - sum), at = 0, cnt = c[0];
      bool found = false;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int n = (c[i] + B - 1) / B;
        if (!found && left < n) { found = true; at = i; cnt = c[i]; }
        if (!found) left -= n;
      }
      const int slot = __builtin_amdgcn_readfirstlane(base + 8 * l + __shfl(at, l, 64));
      const int j = __builtin_amdgcn_readfirstlane(__shfl(left, l, 64)), count = __builtin_amdgcn_readfirstlane(__shfl(cnt, l, 64));
      const int step = chunk_rows<B, A>(count), first = j * step;
      if (first >= count) return {-1, 0, 0};  // rounding the rows up may leave the last chunk empty
      const int off = g.offsets[slot], rows = min(step, count - first);
      // (never beyond the room that the caller stated, whatever the counts say)
      return {slot, off + first, max(0, min(rows, g.rows - off - first))};
    }
    want -= total;
  }
  return {-1, 0, 0};
}

__device__ __forceinline__ int source_row(const GroupedRows& g, int r) { return (int)((uint32_t)(g.por ? g.por[r] : r) / (uint32_t)g.k); }

}  // namespace ew
