// What the products grouped by expert share: their three directions and the arguments of one of them.
#pragma once
#include "grouped_rows.h"

namespace ew {

enum { kFwd = 0,     // out[r][n] = sum_k x[src(r)][k] * w[slot][n][k]
       kDgrad = 1,   // out[r][n] = sum_k x[src(r)][k] * w[slot][k][n]
       kWgrad = 2 }; // out[slot][n][k] = sum_r dy[r][n] * x[src(r)][k]
enum { kWF32 = 0, kWBf16 = 1, kW4 = 2 };  // how weights (kWgrad: rows) are held

struct GemmArgs {
  GroupedRows g;
  const void* x;      // token rows
  const void* w;      // weights of slot 0; kWgrad: dy
  void* out;
  size_t slot_bytes;  // of a slot's weights
  int K, N;           // kWgrad: K is x's width, N is dy's
  int first_slot, num_slots, accumulate;  // kWgrad
};

// Bytes of an expert's [N, K] weights in 4 bits: codes [N, K/2], then scales [N, K/32].
inline size_t w4_bytes(long long N, long long K) { return (size_t)(N * (K / 2) + N * (K / 32)); }
__host__ __device__ __forceinline__ size_t w4_scales_at(int N, int K) { return (size_t)N * (K / 2); }

// grouped_gemm.hip: any sizes and alignments.
int launch_gemm_any(int way, int weights, bool bf16_rows, bool out_f32, const GemmArgs& a, hipStream_t st);
// grouped_gemm.hip: the kernel for these arguments.
int launch_gemm(int way, int weights, bool bf16_rows, bool out_f32, const GemmArgs& a, hipStream_t st);

// Checks what every call over sorted rows needs; 0 or an error.
int check_rows(const char* who, int num_rows, int k, int P, const void* counts, const void* offsets);

}  // namespace ew
