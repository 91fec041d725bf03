// Gradients of the grouped SwiGLU expert FFN and of the weighted combine.
//
// FFN, for the rows of one slot (g = W1g x, u = W1u x, s = sigmoid(g), a = g s u, y = W2 a):
//     da  = W2^T dy                     dW2  = sum_r dy a^T
//     dg  = da u s (1 + g (1 - s))      du   = da g s
//     dx  = W1g^T dg + W1u^T du         dW13 = sum_r [dg; du] x^T
// g and u are computed again: kept from the forward pass they would be 2 I values a row for as long as the layers behind this one run.
// da comes first, in fp32; the product that makes g and u then forms dg, du and a in its epilogue, where a lane holds both of a feature.  Of what
// lies between the products only dg, du and a are rounded to bf16, as operands of the matrix cores: the gradients are 2.3e-3 from 64 bits in bf16, where
// the rounding of the results alone is 1.7e-3.  (With g, u and da in bf16 too 3.5e-3.)
// fp32: 8 slots of 512 rows, 2048 x 1408, 1884 us (100 TFLOP/s of the 140 that a large library product reaches); configuration 0's layer, 16 slots of 8
// rows, 256 x 128, 44 us, five launches one after the other.
#include "grouped_gemm.h"

namespace ew {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

template <typename T>
struct Vec;
template <>
struct Vec<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void load(const float* p, float* v) {
    const f32x4 a = *(const f32x4*)p;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = a[i];
  }
  static __device__ __forceinline__ void store(float* p, const float* v) {
    f32x4 a;
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] = v[i];
    *(f32x4*)p = a;
  }
  static __device__ __forceinline__ float get(float v) { return v; }
  static __device__ __forceinline__ float put(float v) { return v; }
};
template <>
struct Vec<uint16_t> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void load(const uint16_t* p, float* v) {
    const u32x4 a = *(const u32x4*)p;
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(a[i] << 16); v[2 * i + 1] = __uint_as_float(a[i] & 0xFFFF0000u); }
  }
  static __device__ __forceinline__ uint16_t put(float v) { return __builtin_bit_cast(uint16_t, (__bf16)v); }
  static __device__ __forceinline__ float get(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }
  static __device__ __forceinline__ void store(uint16_t* p, const float* v) {
    u32x4 a;
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] = (uint32_t)put(v[2 * i]) | (uint32_t)put(v[2 * i + 1]) << 16;
    *(u32x4*)p = a;
  }
};

// dy[row_of_pair[p]] = w[p] dout[t], dw[p] = <dout[t], y[row_of_pair[p]]>, p = t k + j.  One wave per pair; a token's waves are
// neighbours, so its row of dout comes from L2 after the first.
template <typename T, bool V>
__global__ __launch_bounds__(256) void k_unpermute_back(const T* __restrict__ dout, const T* __restrict__ y, const int32_t* __restrict__ rop,
                                                        const float* __restrict__ w, long long pairs, int k, int H, T* __restrict__ dy,
                                                        float* __restrict__ dw) {
  constexpr int W = V ? Vec<T>::N : 1;
  const int lane = threadIdx.x & 63;
  for (long long p = (long long)blockIdx.x * 4 + (threadIdx.x >> 6); p < pairs; p += (long long)gridDim.x * 4) {
    const T* d = dout + (size_t)(p / k) * H;
    const size_t row = (size_t)rop[p] * H;
    const float wp = w[p];
    float sum = 0.f;
    for (int h = lane * W; h < H; h += 64 * W) {
      float v[W], o[W], f[W];
      if constexpr (V) Vec<T>::load(d + h, v); else v[0] = Vec<T>::get(d[h]);
      if (y) {
        if constexpr (V) Vec<T>::load(y + row + h, f); else f[0] = Vec<T>::get(y[row + h]);
#pragma unroll
        for (int j = 0; j < W; ++j) sum = fmaf(v[j], f[j], sum);
      }
#pragma unroll
      for (int j = 0; j < W; ++j) o[j] = wp * v[j];
      if constexpr (V) Vec<T>::store(dy + row + h, o); else dy[row + h] = Vec<T>::put(o[0]);
    }
    if (!y) continue;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
    if (lane == 0) dw[p] = sum;
  }
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

template <typename T>
int unpermute_back(const T* dout, const T* y, const int32_t* rop, const float* w, long long pairs, int k, int H, T* dy, float* dw, hipStream_t st) {
  const dim3 grid((unsigned)((pairs + 3) / 4 < 1 << 22 ? (pairs + 3) / 4 : 1 << 22));  // (a launch has fewer than 2^32 threads)
  if (H % Vec<T>::N == 0 && aligned16(dout) && aligned16(y) && aligned16(dy))
    hipLaunchKernelGGL((k_unpermute_back<T, true>), grid, dim3(256), 0, st, dout, y, rop, w, pairs, k, H, dy, dw);
  else
    hipLaunchKernelGGL((k_unpermute_back<T, false>), grid, dim3(256), 0, st, dout, y, rop, w, pairs, k, H, dy, dw);
  EW_LAUNCH_CHECK("k_unpermute_back");
  return EW_OK;
}

// Workspace: da [rows, I] fp32, dg and du [rows, 2I], a [rows, I].
struct BackScratch { size_t dh, act, all; };
BackScratch back_scratch(int num_rows, int I, int dtype) {
  const size_t el = dtype == EW_BF16 ? 2 : 4, n = (size_t)num_rows * I;
  const size_t dh = align_up(n * 4, 256), act = dh + align_up(n * 2 * el, 256);
  return {dh, act, act + align_up(n * el, 256)};
}

}  // namespace

}  // namespace ew

extern "C" size_t moe_grouped_ffn_backward_workspace_bytes(int num_rows, int I, int dtype) {
  if (num_rows < 1 || I < 1 || (dtype != EW_F32 && dtype != EW_BF16)) return 0;
  return ew::back_scratch(num_rows, I, dtype).all;
}

extern "C" int moe_grouped_ffn_backward(const void* x, const void* dy, int dtype, int num_tokens, int num_rows, int k, int H, int I, int P, const int32_t* counts,
                                        const int32_t* offsets, const int32_t* pair_of_row, const void* w13_base, const void* w2_base,
                                        void* dx_sorted, int first_slot, int num_slots, int dw_dtype, int accumulate, void* dw13, void* dw2,
                                        void* ws, size_t ws_bytes, void* stream) {
  using ew::fail;
  const char* who = "moe_grouped_ffn_backward";
  if (H < 1 || I < 1 || I >= (1 << 30)) return fail(EW_ERR_INVALID_ARG, "%s: need H>=1, 1<=I<2^30 (got %d, %d)", who, H, I);
  if (const int rc = ew::check_sizes(who, "H", H, "2 I", 2ll * I)) return rc;
  if (dtype != EW_F32 && dtype != EW_BF16) return fail(EW_ERR_INVALID_ARG, "%s: unknown dtype %d", who, dtype);
  if (dw_dtype != EW_F32 && !(dw_dtype == EW_BF16 && dtype == EW_BF16))
    return fail(EW_ERR_INVALID_ARG, "%s: weight gradients are float32, or bfloat16 for bfloat16 rows (dw_dtype=%d)", who, dw_dtype);
  if (accumulate && dw_dtype != EW_F32) return fail(EW_ERR_UNSUPPORTED, "%s: only float32 gradients accumulate", who);
  if (const int rc = ew::check_rows(who, num_tokens, num_rows, k, P, counts, offsets, pair_of_row)) return rc;
  if (first_slot < 0 || num_slots < 0 || first_slot > P - num_slots)
    return fail(EW_ERR_INVALID_ARG, "%s: slots [%d, %d + %d) outside 0..P=%d", who, first_slot, first_slot, num_slots, P);
  const bool want_w = num_slots > 0 && (dw13 || dw2);
  if (num_rows > 0) {
    if (!x || !dy || !w13_base || !w2_base) return fail(EW_ERR_INVALID_ARG, "%s: NULL device pointer", who);
    const size_t need = moe_grouped_ffn_backward_workspace_bytes(num_rows, I, dtype);
    if (!ws || ((uintptr_t)ws & 255) || ws_bytes < need)
      return fail(EW_ERR_WORKSPACE, "%s: workspace needs %zu bytes aligned to 256 (got %zu at %p)", who, need, ws_bytes, ws);
  }
  if (!dx_sorted && !want_w) return EW_OK;
  const hipStream_t st = (hipStream_t)stream;
  const bool bf16 = dtype == EW_BF16;
  const int wt = bf16 ? ew::kWBf16 : ew::kWF32;
  const size_t el = bf16 ? 2 : 4;
  const ew::BackScratch at = ew::back_scratch(num_rows, I, dtype);
  void *dh = (char*)ws + at.dh, *act = (char*)ws + at.act;
  const ew::GroupedRows mapped{counts, offsets, pair_of_row, P, num_rows, k}, sorted{counts, offsets, nullptr, P, num_rows, 1};
  const int ep = bf16 ? ew::kEpBf16 : ew::kEpF32;
  ew::GemmArgs a{};
  int rc;
  if (num_rows > 0) {
    a.g = sorted; a.x = dy; a.x_rows = num_rows; a.w = w2_base; a.out = ws; a.K = H; a.N = I; a.slot_bytes = (size_t)I * H * el;
    if ((rc = ew::launch_gemm(ew::kDgrad, wt, ew::kEpF32, bf16, a, st))) return rc;
    a.g = mapped; a.x = x; a.x_rows = num_tokens; a.w = w13_base; a.out = act; a.da = (const float*)ws; a.dh = dh;
    a.slot_bytes = (size_t)2 * I * H * el;
    if ((rc = ew::launch_gemm(ew::kFwd, wt, ew::kEpBack, bf16, a, st))) return rc;
    if (dx_sorted) {
      a.g = sorted; a.x = dh; a.x_rows = num_rows; a.out = dx_sorted; a.K = 2 * I; a.N = H;
      if ((rc = ew::launch_gemm(ew::kDgrad, wt, ep, bf16, a, st))) return rc;
    }
  }
  if (!want_w) return EW_OK;
  const int dw_ep = dw_dtype == EW_F32 ? ew::kEpF32 : ew::kEpBf16;
  a.first_slot = first_slot; a.num_slots = num_slots; a.accumulate = accumulate != 0;
  if (dw13) {
    a.g = mapped; a.x = x; a.x_rows = num_tokens; a.w = dh; a.out = dw13; a.K = H; a.N = 2 * I;
    if ((rc = ew::launch_gemm(ew::kWgrad, wt, dw_ep, bf16, a, st))) return rc;
  }
  if (dw2) {
    a.g = sorted; a.x = act; a.x_rows = num_rows; a.w = dy; a.out = dw2; a.K = I; a.N = H;
    if ((rc = ew::launch_gemm(ew::kWgrad, wt, dw_ep, bf16, a, st))) return rc;
  }
  return EW_OK;
}

extern "C" int moe_unpermute_backward(const void* dout, const void* y_sorted, const int32_t* row_of_pair, const float* topk_w, int T, int k, int H,
                                      int dtype, void* dy_sorted, float* dw, void* stream) {
  using ew::fail;
  const char* who = "moe_unpermute_backward";
  if (T < 0 || k < 1 || H < 1) return fail(EW_ERR_INVALID_ARG, "%s: need T>=0, k>=1, H>=1 (got %d, %d, %d)", who, T, k, H);
  if (const int rc = ew::check_size(who, "H", H)) return rc;
  if (dtype != EW_F32 && dtype != EW_BF16) return fail(EW_ERR_INVALID_ARG, "%s: unknown dtype %d", who, dtype);
  if ((long long)T * k >= (1ll << 31)) return fail(EW_ERR_UNSUPPORTED, "%s: the row count must be below 2^31", who);
  if (T == 0) return EW_OK;
  if (!dout || !row_of_pair || !topk_w || !dy_sorted || !y_sorted != !dw)
    return fail(EW_ERR_INVALID_ARG, "%s: NULL device pointer (y_sorted and dw: both or neither)", who);
  const long long pairs = (long long)T * k;
  const hipStream_t st = (hipStream_t)stream;
  if (dtype == EW_BF16)
    return ew::unpermute_back((const uint16_t*)dout, (const uint16_t*)y_sorted, row_of_pair, topk_w, pairs, k, H, (uint16_t*)dy_sorted, dw, st);
  return ew::unpermute_back((const float*)dout, (const float*)y_sorted, row_of_pair, topk_w, pairs, k, H, (float*)dy_sorted, dw, st);
}
