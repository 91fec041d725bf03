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
  const void* x;      // token rows, x_rows of them
  const void* w;      // weights of slot 0; kWgrad: dy
  void* out;
  size_t slot_bytes;  // of a slot's weights
  const float* da;    // kEpBack: [rows, N] gradient of the activation
  void* dh;           // kEpBack: [rows, 2N], in the rows' type
  int K, N;           // kWgrad: K is x's width, N is dy's
  int x_rows;
  int first_slot, num_slots, accumulate;  // kWgrad
};

// What becomes of a product's sums.
enum { kEpBf16 = 0, kEpF32 = 1,
       kEpSwiglu = 2,   // out[r][n] = silu(g) u, weights [2N, K]: gate rows, then up rows
       kEpBack = 3 };   // the same out, and dh[r] = [dg, du] from da (grouped_backward.hip)

// Bytes of an expert's [N, K] weights in 4 bits: codes [N, K/2], then scales [N, K/32].
inline size_t w4_bytes(long long N, long long K) { return (size_t)(N * (K / 2) + N * (K / 32)); }
__host__ __device__ __forceinline__ size_t w4_scales_at(int N, int K) { return (size_t)N * (K / 2); }

// grouped_gemm.hip: any sizes and alignments.  bf16: rows and results (but for kEpF32's).
int launch_gemm_any(int way, int weights, int epilogue, bool bf16, const GemmArgs& a, hipStream_t st);
// grouped_stream.hip: few rows per slot, bf16 or 4-bit weights; whether it takes these arguments.
bool stream_takes(int way, int weights, int epilogue, const GemmArgs& a);
int launch_stream(int way, int weights, int epilogue, const GemmArgs& a, hipStream_t st);
// grouped_tile.hip: bf16 matrix cores; whether it takes these arguments.
bool tile_takes(int way, int weights, int epilogue, const GemmArgs& a);
int launch_tile(int way, int weights, int epilogue, const GemmArgs& a, hipStream_t st);
// grouped_gemm.hip: by the kernel for these arguments.
int launch_gemm(int way, int weights, int epilogue, bool bf16, const GemmArgs& a, hipStream_t st);

// a = silu(g) u, and from da the gradients of g and u (kEpBack).
// The relative error of __expf grows with its argument, to 7e-6 at 80.  That is nothing beside the rounding to bf16 that follows (4e-3);
// results in fp32 take expf, as the forward pass in fp32 does.
struct SwigluBack { float a, dg, du; };
template <bool F32>
__device__ __forceinline__ SwigluBack swiglu_back(float g, float u, float da) {
  const float s = 1.f / (1.f + (F32 ? expf(-g) : __expf(-g))), gs = g * s;
  return {gs * u, da * u * (s + gs * (1.f - s)), da * gs};
}
// (for results in bf16)
__device__ __forceinline__ float swiglu(float g, float u) { return g / (1.f + __expf(-g)) * u; }

// Loops and tile borders count in 32 bits and reach a little past the ends: sizes and rows stay this far below 2^31.
constexpr int kMostSize = (int)((1u << 31) - 1024);
inline int check_size(const char* who, const char* what, long long v) {
  return v <= kMostSize ? EW_OK : fail(EW_ERR_UNSUPPORTED, "%s: %s=%lld is too many (at most 2^31 - 1024)", who, what, v);
}

// A launch has fewer than 2^32 threads.
inline int check_grid(long long workgroups, int threads) {
  return workgroups * threads < (1ll << 32) ? EW_OK : fail(EW_ERR_UNSUPPORTED, "grouped product: %lld output tiles are too many for one launch", workgroups);
}

// Checks what every call over sorted rows needs; 0 or an error.
int check_sizes(const char* who, const char* a, long long na, const char* b, long long nb);
int check_rows(const char* who, int num_tokens, int num_rows, int k, int P, const void* counts, const void* offsets, const void* pair_of_row);

}  // namespace ew
