// Experts held in 4 bits: E2M1 values (0, 1/2, 1, 3/2, 2, 3, 4, 6 and their negatives), 32 of them along K sharing a power of two
// (E8M0: 2^(byte - 127), 255 = NaN), the OCP Microscaling format for 4 bits.  An expert's [N, K] weights are one run of bytes:
// codes [N, K/2] (even elements in the low half of a byte), then scales [N, K/32].
#include "grouped_gemm.h"

namespace ew {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ void load8(const float* p, float (&v)[8]) {
  const f32x4 a = *(const f32x4*)p, b = *(const f32x4*)(p + 4);
#pragma unroll
  for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[4 + i] = b[i]; }
}
__device__ __forceinline__ void load8(const uint16_t* p, float (&v)[8]) {
  const u32x4 a = *(const u32x4*)p;
#pragma unroll
  for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(a[i] << 16); v[2 * i + 1] = __uint_as_float(a[i] & 0xFFFF0000u); }
}

// A lane has 8 neighbours, four lanes a group of 32.  The scale is 2^(floor(log2 of the largest)) / 4: it brings the largest of the
// group into [4, 8), and what lies above 6 becomes 6.  A group with an infinity or a NaN becomes NaN.  Rounding to the nearest value,
// halves to the even code, is the conversion instruction's; its scale operand is used by its exponent alone.
// Bytes bound it: it reads 16 or 32 and writes 4 a lane.
template <typename T>
__global__ __launch_bounds__(256) void k_quantize_w4(const T* __restrict__ w, long long eights, long long per_expert,
                                                     unsigned char* __restrict__ out) {
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < eights; i += (long long)gridDim.x * 256) {  // (K % 32 == 0: whole groups)
    float v[8];
    load8(w + 8 * i, v);
    uint32_t most = 0;  // bits of magnitudes: ordered as the magnitudes are
#pragma unroll
    for (int j = 0; j < 8; ++j) most = max(most, __float_as_uint(v[j]) & 0x7FFFFFFFu);
    most = max(most, (uint32_t)__shfl_xor((int)most, 1, 64));
    most = max(most, (uint32_t)__shfl_xor((int)most, 2, 64));
    const uint32_t e = most >> 23, byte = e == 255 ? 255 : e < 2 ? 0 : e - 2;  // (below 2^-124 the scale stays at its least, 2^-127)
    const float scale = __uint_as_float(byte << 23);
    uint32_t code = 0;
    code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[0], v[1], scale, 0);
    code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[2], v[3], scale, 1);
    code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[4], v[5], scale, 2);
    code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[6], v[7], scale, 3);
    const long long expert = i / per_expert, at = i - expert * per_expert;
    unsigned char* p = out + (size_t)expert * ((size_t)per_expert * 4 + (size_t)per_expert / 4);
    *(uint32_t*)(p + 4 * at) = byte == 255 ? 0u : code;
    if ((threadIdx.x & 3) == 0) p[4 * per_expert + at / 4] = (unsigned char)byte;
  }
}

// The values that the codes stand for, exactly: bf16 has room for all of them, down to 2^-128; with scales of 253 and 254 the larger
// codes are beyond both types' range and become infinities.
template <typename T>
__global__ __launch_bounds__(256) void k_dequantize_w4(const unsigned char* __restrict__ in, long long eights, long long per_expert,
                                                       T* __restrict__ w) {
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < eights; i += (long long)gridDim.x * 256) {
    const long long expert = i / per_expert, at = i - expert * per_expert;
    const unsigned char* p = in + (size_t)expert * ((size_t)per_expert * 4 + (size_t)per_expert / 4);
    const uint32_t code = *(const uint32_t*)(p + 4 * at), byte = p[4 * per_expert + at / 4];
    const float scale = __uint_as_float(byte << 23);
    if constexpr (sizeof(T) == 2) {
      u32x4 o;
      o[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 0));
      o[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 1));
      o[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 2));
      o[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 3));
      *(u32x4*)(w + 8 * i) = o;
    } else {
      f32x4 lo, hi;
      auto a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, scale, 1);
      auto c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, scale, 3);
      lo[0] = a[0]; lo[1] = a[1]; lo[2] = b[0]; lo[3] = b[1];
      hi[0] = c[0]; hi[1] = c[1]; hi[2] = d[0]; hi[3] = d[1];
      *(f32x4*)(w + 8 * i) = lo;
      *(f32x4*)(w + 8 * i + 4) = hi;
    }
  }
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

// Common checks of packing and reading back; what both kernels step through, or 0 where there is nothing to do.
int check_pack(const char* who, const void* a, const void* b, int dtype, int num_experts, int N, int K, long long* eights) {
  if (dtype != EW_F32 && dtype != EW_BF16) return fail(EW_ERR_INVALID_ARG, "%s: unknown dtype %d", who, dtype);
  if (num_experts < 0 || N < 1 || K < 1) return fail(EW_ERR_INVALID_ARG, "%s: need num_experts>=0, N>=1, K>=1 (got %d, %d, %d)", who, num_experts, N, K);
  if (!moe_w4_expert_bytes(N, K)) return fail(EW_ERR_UNSUPPORTED, "%s: K must be a multiple of 32 and N*K of 512 (N=%d K=%d)", who, N, K);
  *eights = (long long)num_experts * N * K / 8;
  if (*eights == 0) return EW_OK;
  if (!a || !b) return fail(EW_ERR_INVALID_ARG, "%s: NULL device pointer", who);
  if (!aligned16(a) || !aligned16(b)) return fail(EW_ERR_INVALID_ARG, "%s: pointers must be aligned to 16 bytes", who);
  return EW_OK;
}
unsigned pack_grid(long long eights) { return (unsigned)(eights + 255 < 256ll * 16384 ? (eights + 255) / 256 : 16384); }

}  // namespace

}  // namespace ew

extern "C" size_t moe_w4_expert_bytes(int N, int K) {
  if (N < 1 || K < 1 || K % 32 || ((long long)N * K) % 512) return 0;
  return ew::w4_bytes(N, K);
}

extern "C" int moe_quantize_w4(const void* w, int dtype, int num_experts, int N, int K, void* out, void* stream) {
  long long eights = 0;
  if (const int rc = ew::check_pack("moe_quantize_w4", w, out, dtype, num_experts, N, K, &eights)) return rc;
  if (!eights) return EW_OK;
  const dim3 grid(ew::pack_grid(eights));
  const long long per = (long long)N * K / 8;
  if (dtype == EW_BF16)
    hipLaunchKernelGGL((ew::k_quantize_w4<uint16_t>), grid, dim3(256), 0, (hipStream_t)stream, (const uint16_t*)w, eights, per, (unsigned char*)out);
  else
    hipLaunchKernelGGL((ew::k_quantize_w4<float>), grid, dim3(256), 0, (hipStream_t)stream, (const float*)w, eights, per, (unsigned char*)out);
  EW_LAUNCH_CHECK("k_quantize_w4");
  return EW_OK;
}

extern "C" int moe_dequantize_w4(const void* w4, int dtype, int num_experts, int N, int K, void* w, void* stream) {
  long long eights = 0;
  if (const int rc = ew::check_pack("moe_dequantize_w4", w4, w, dtype, num_experts, N, K, &eights)) return rc;
  if (!eights) return EW_OK;
  const dim3 grid(ew::pack_grid(eights));
  const long long per = (long long)N * K / 8;
  if (dtype == EW_BF16)
    hipLaunchKernelGGL((ew::k_dequantize_w4<uint16_t>), grid, dim3(256), 0, (hipStream_t)stream, (const unsigned char*)w4, eights, per, (uint16_t*)w);
  else
    hipLaunchKernelGGL((ew::k_dequantize_w4<float>), grid, dim3(256), 0, (hipStream_t)stream, (const unsigned char*)w4, eights, per, (float*)w);
  EW_LAUNCH_CHECK("k_dequantize_w4");
  return EW_OK;
}

namespace {

ew::GemmArgs w4_args(const int32_t* counts, const int32_t* offsets, const int32_t* por, int P, int num_rows, int k, const void* x, int x_rows, const void* w,
                     void* out, int K, int N, size_t slot_bytes) {
  ew::GemmArgs a{};
  a.g = {counts, offsets, por, P, num_rows, k};
  a.x = x; a.x_rows = x_rows; a.w = w; a.out = out; a.K = K; a.N = N;
  a.slot_bytes = slot_bytes;
  return a;
}

}  // namespace

extern "C" int moe_grouped_gemm_w4(const void* x, int num_tokens, int num_rows, int k, int K, int N, int P, const int32_t* counts, const int32_t* offsets,
                                   const int32_t* pair_of_row, const void* w4_base, void* y, void* stream) {
  using ew::fail;
  const char* who = "moe_grouped_gemm_w4";
  if (K < 1 || N < 1) return fail(EW_ERR_INVALID_ARG, "%s: need K>=1, N>=1 (got %d, %d)", who, K, N);
  if (const int rc = ew::check_sizes(who, "K", K, "N", N)) return rc;
  if (!moe_w4_expert_bytes(N, K)) return fail(EW_ERR_UNSUPPORTED, "%s: K must be a multiple of 32 and N*K of 512 (N=%d K=%d)", who, N, K);
  if (num_rows == 0 && k >= 1 && P >= 1) return EW_OK;
  if (const int rc = ew::check_rows(who, num_tokens, num_rows, k, P, counts, offsets, pair_of_row)) return rc;
  if (!x || !w4_base || !y) return fail(EW_ERR_INVALID_ARG, "%s: NULL device pointer", who);
  return ew::launch_gemm(ew::kFwd, ew::kW4, ew::kEpBf16, true,
                         w4_args(counts, offsets, pair_of_row, P, num_rows, k, x, num_tokens, w4_base, y, K, N, moe_w4_expert_bytes(N, K)), (hipStream_t)stream);
}

extern "C" size_t moe_grouped_ffn_w4_workspace_bytes(int num_rows, int I) {
  if (num_rows < 1 || I < 1) return 0;
  return ew::align_up((size_t)num_rows * I * 2, 256);
}

extern "C" int moe_grouped_ffn_w4(const void* x, int num_tokens, int num_rows, int k, int H, int I, int P, const int32_t* counts, const int32_t* offsets,
                                  const int32_t* pair_of_row, const void* w13_base, const void* w2_base, void* y_sorted, void* ws,
                                  size_t ws_bytes, void* stream) {
  using ew::fail;
  const char* who = "moe_grouped_ffn_w4";
  if (H < 1 || I < 1 || I >= (1 << 30)) return fail(EW_ERR_INVALID_ARG, "%s: need H>=1, 1<=I<2^30 (got %d, %d)", who, H, I);
  if (const int rc = ew::check_sizes(who, "H", H, "2 I", 2ll * I)) return rc;
  if (!moe_w4_expert_bytes(2 * I, H) || !moe_w4_expert_bytes(H, I))
    return fail(EW_ERR_UNSUPPORTED, "%s: H and I must be multiples of 32 and H*I of 512 (H=%d I=%d)", who, H, I);
  if (num_rows == 0 && k >= 1 && P >= 1) return EW_OK;
  if (const int rc = ew::check_rows(who, num_tokens, num_rows, k, P, counts, offsets, pair_of_row)) return rc;
  if (!x || !w13_base || !w2_base || !y_sorted) return fail(EW_ERR_INVALID_ARG, "%s: NULL device pointer", who);
  const size_t need = moe_grouped_ffn_w4_workspace_bytes(num_rows, I);
  if (!ws || ((uintptr_t)ws & 255) || ws_bytes < need)
    return fail(EW_ERR_WORKSPACE, "%s: workspace needs %zu bytes aligned to 256 (got %zu at %p)", who, need, ws_bytes, ws);
  // The activation is bf16 between the products, as in moe_grouped_ffn: it is the second one's operand on the bf16 matrix cores.  (2.3e-3 from 64 bits;
  // an activation in fp32 would leave the rounding of y, 1.7e-3.)
  const hipStream_t st = (hipStream_t)stream;
  const int rc = ew::launch_gemm(ew::kFwd, ew::kW4, ew::kEpSwiglu, true,
                                 w4_args(counts, offsets, pair_of_row, P, num_rows, k, x, num_tokens, w13_base, ws, H, I, moe_w4_expert_bytes(2 * I, H)), st);
  if (rc) return rc;
  return ew::launch_gemm(ew::kFwd, ew::kW4, ew::kEpBf16, true,
                         w4_args(counts, offsets, nullptr, P, num_rows, 1, ws, num_rows, w2_base, y_sorted, I, H, moe_w4_expert_bytes(H, I)), st);
}
