// Matrix products grouped by expert over ragged rows, in three directions (forward, input gradient, weight gradient).
//
// k_gemm_any is the kernel for fp32, and for bf16 and 4-bit sizes that the matrix-core kernels do not take: plain fp32 products
// and sums on v_mfma_f32_32x32x2_f32 whatever the inputs' type, any sizes, any alignment.  A workgroup makes 64 x 64 outputs, its four
// waves 32 x 32 each; 32 contraction steps at a time reach LDS contraction-major, so that both operands are read without bank
// conflicts whichever way they lie in memory, and the next 32 are loaded meanwhile.  Outputs of a lane are four neighbours along the contiguous axis.
// Small calls are bound by the latency of those rounds, large ones by the matrix cores' fp32 rate: 4 slots of 2048 rows, 2048 x 2048, takes 620 to 665 us
// (103 to 111 TFLOP/s; a large library product reaches 140), and an input gradient 256 x 512 of 128 rows 17 us.  With single loads, 16 steps at a time and
// nothing loaded ahead the same calls took 1120 to 1830 and 27 us.
#include "grouped_gemm.h"

namespace ew {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

__device__ __forceinline__ float as_f32(float v) { return v; }
__device__ __forceinline__ float as_f32(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }
__device__ __forceinline__ void put(float* p, float v) { *p = v; }
__device__ __forceinline__ void put(uint16_t* p, float v) { *p = __builtin_bit_cast(uint16_t, (__bf16)v); }

// E2M1 value times 2^(scale - 127); scale 255 means NaN.
__device__ __forceinline__ float w4_value(uint32_t code, uint32_t scale) {
  const uint32_t e = code >> 1 & 3, m = code & 1;
  const float mag = e ? __uint_as_float((126 + e) << 23 | m << 22) : 0.5f * (float)m;
  const float v = ldexpf(code & 8 ? -mag : mag, (int)scale - 127);
  return scale == 255 ? __uint_as_float(0x7FC00000u) : v;
}

constexpr int kTile = 64, kStep = 32, kPitch = kTile + 4;

// TW: type of the weights' elements (kWgrad: dy's); float, uint16_t (bf16), or uint8_t for a 4-bit expert's bytes.  VEC: 16-byte loads of floats.
template <int WAY, typename TX, typename TW, int EP, bool VEC>
__global__ __launch_bounds__(256) void k_gemm_any(GemmArgs a, int tiles_n) {
  constexpr bool GATED = EP == kEpSwiglu || EP == kEpBack;  // 32 features: tile index 16 q + 8 s + r is feature 8 q + r of the gate (s = 0) or up rows
  __shared__ float s_a[2][kStep][kPitch], s_b[2][kStep][kPitch];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int tile = blockIdx.x % tiles_n, unit = blockIdx.x / tiles_n;
  const int K = a.K, N = a.N;
  RowChunk ch;
  int na, nb, a0, b0, len;  // extents and start of the output tile along A (contiguous) and B, length of the contraction
  if constexpr (WAY == kWgrad) {
    const int slot = a.first_slot + unit;
    const int off = a.g.offsets[slot];
    ch = {slot, off, max(0, min(a.g.counts[slot], a.g.rows - off))};
    const int tk = (K + kTile - 1) / kTile;
    a0 = tile % tk * kTile; b0 = tile / tk * kTile;
    na = K; nb = N; len = ch.rows;
    if (len == 0 && a.accumulate) return;
  } else {
    ch = find_chunk<kTile, 1>(a.g, unit);
    if (ch.slot < 0) return;
    a0 = tile * (GATED ? kTile / 2 : kTile); b0 = 0;
    na = N; nb = ch.rows; len = K;
  }
  const TX* x = (const TX*)a.x;
  const unsigned char* ws = (const unsigned char*)a.w + (WAY == kWgrad ? 0 : (size_t)ch.slot * a.slot_bytes);
  // operand A: weights, or x of the weight gradient; operand B: token rows, or dy.  Where element (o, kk), o < na or nb and kk < len, lies:
  auto a_at = [&](int o, int kk) -> size_t {
    if constexpr (WAY == kWgrad) return (size_t)source_row(a.g, ch.first + kk) * K + o;
    else return WAY == kFwd ? (size_t)o * K + kk : (size_t)kk * N + o;
  };
  auto a_value = [&](int o, int kk) -> float {
    if constexpr (WAY == kWgrad) return as_f32(x[a_at(o, kk)]);
    else if constexpr (sizeof(TW) == 1) {
      const uint32_t two = ws[(size_t)o * (K / 2) + kk / 2];
      return w4_value(kk & 1 ? two >> 4 : two & 15, ws[w4_scales_at(GATED ? 2 * N : N, K) + (size_t)o * (K / 32) + kk / 32]);
    } else return as_f32(((const TW*)ws)[a_at(o, kk)]);
  };
  const int row_k = tid >> 2, k_k = (tid & 3) * 4;   // a thread's four elements along the contraction
  const int k_o = tid >> 4, row_o = (tid & 15) * 4;  // and across it
  int src = 0;
  if constexpr (WAY != kWgrad) src = row_k < nb ? source_row(a.g, ch.first + row_k) : 0;
  constexpr int J = kStep / 16;
  float va[J][4], vb[J][4];
  auto fetch = [&](int k0) {
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const int ka = k0 + 16 * j + k_k, kc = k0 + 16 * j + k_o;  // along, across
      const int f = a0 + (GATED ? 8 * (row_k >> 4) + (row_k & 7) : row_k), ff = GATED && (row_k & 8) ? f + N : f;
      if constexpr (VEC) {
        const float *w = (const float*)ws, *xf = (const float*)x;
        const f32x4 zero = {};
        f32x4 p, q;
        if constexpr (WAY == kFwd) p = f < na && ka < len ? *(const f32x4*)(w + a_at(ff, ka)) : zero;
        else p = a0 + row_o < na && kc < len ? *(const f32x4*)((WAY == kWgrad ? xf : w) + a_at(a0 + row_o, kc)) : zero;
        if constexpr (WAY == kWgrad) q = b0 + row_o < nb && kc < len ? *(const f32x4*)(w + (size_t)(ch.first + kc) * N + b0 + row_o) : zero;
        else q = row_k < nb && ka < len ? *(const f32x4*)(xf + (size_t)src * K + ka) : zero;
#pragma unroll
        for (int i = 0; i < 4; ++i) { va[j][i] = p[i]; vb[j][i] = q[i]; }
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if constexpr (WAY == kFwd) va[j][i] = f < na && ka + i < len ? a_value(ff, ka + i) : 0.f;
          else va[j][i] = a0 + row_o + i < na && kc < len ? a_value(a0 + row_o + i, kc) : 0.f;
          if constexpr (WAY == kWgrad) vb[j][i] = b0 + row_o + i < nb && kc < len ? as_f32(((const TW*)ws)[(size_t)(ch.first + kc) * N + b0 + row_o + i]) : 0.f;
          else vb[j][i] = row_k < nb && ka + i < len ? as_f32(x[(size_t)src * K + ka + i]) : 0.f;
        }
      }
    }
  };
  f32x16 acc = {};
  fetch(0);
  for (int k0 = 0, buf = 0; k0 < len; k0 += kStep, buf ^= 1) {
#pragma unroll
    for (int j = 0; j < J; ++j) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (WAY == kFwd) s_a[buf][16 * j + k_k + i][row_k] = va[j][i]; else s_a[buf][16 * j + k_o][row_o + i] = va[j][i];
        if constexpr (WAY == kWgrad) s_b[buf][16 * j + k_o][row_o + i] = vb[j][i]; else s_b[buf][16 * j + k_k + i][row_k] = vb[j][i];
      }
    }
    __syncthreads();  // (one a step: whoever writes a buffer again has met, at the barrier between, all that read it)
    fetch(k0 + kStep);
#pragma unroll
    for (int j = 0; j < kStep; j += 2)
      acc = __builtin_amdgcn_mfma_f32_32x32x2f32(s_a[buf][j + (lane >> 5)][(wave & 1) * 32 + (lane & 31)],
                                                 s_b[buf][j + (lane >> 5)][(wave >> 1) * 32 + (lane & 31)], acc, 0, 0, 0);
  }
  // lane l: B element l % 32, A elements 8 (i / 4) + 4 (l / 32) + i % 4
  const int b = b0 + (wave >> 1) * 32 + (lane & 31);
  if (b >= nb) return;
  const size_t row = WAY == kWgrad ? (size_t)unit * N + b : (size_t)(ch.first + b);
  if constexpr (GATED) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int o = a0 + (wave & 1) * 16 + 8 * (i >> 2) + 4 * (lane >> 5) + (i & 3);
      if (o >= na) continue;
      const float g = acc[8 * (i >> 2) + (i & 3)], u = acc[8 * (i >> 2) + 4 + (i & 3)];
      if constexpr (EP == kEpBack) {
        const SwigluBack v = swiglu_back<sizeof(TX) == 4>(g, u, a.da[row * N + o]);
        put((TX*)a.out + row * N + o, v.a);
        put((TX*)a.dh + row * 2 * N + o, v.dg);
        put((TX*)a.dh + row * 2 * N + N + o, v.du);
      } else {
        put((TX*)a.out + row * N + o, swiglu(g, u));
      }
    }
    return;
  }
  const size_t at = row * (WAY == kWgrad ? K : N);
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int o = a0 + (wave & 1) * 32 + 8 * (i >> 2) + 4 * (lane >> 5) + (i & 3);
    if (o >= na) continue;
    if constexpr (EP == kEpF32) {
      float* p = (float*)a.out + at + o;
      *p = WAY == kWgrad && a.accumulate ? *p + acc[i] : acc[i];
    } else {
      put((uint16_t*)a.out + at + o, acc[i]);
    }
  }
}

template <int WAY, typename TX, typename TW, int EP>
int launch_any(const GemmArgs& a, hipStream_t st) {
  long long units, tiles;
  if (WAY == kWgrad) {
    units = a.num_slots;
    tiles = (long long)ceil_div(a.K, kTile) * ceil_div(a.N, kTile);
  } else {
    units = max_chunks(a.g.rows, a.g.P, kTile);
    tiles = ceil_div(a.N, EP == kEpSwiglu || EP == kEpBack ? kTile / 2 : kTile);
  }
  if (const int rc = check_grid(units * tiles, 256)) return rc;
  if (units * tiles == 0) return EW_OK;
  const bool vec = sizeof(TX) == 4 && a.K % 4 == 0 && a.N % 4 == 0 && (((uintptr_t)a.x | (uintptr_t)a.w) & 15) == 0;
  if (vec) hipLaunchKernelGGL((k_gemm_any<WAY, TX, TW, EP, sizeof(TX) == 4>), dim3((unsigned)(units * tiles)), dim3(256), 0, st, a, (int)tiles);
  else hipLaunchKernelGGL((k_gemm_any<WAY, TX, TW, EP, false>), dim3((unsigned)(units * tiles)), dim3(256), 0, st, a, (int)tiles);
  EW_LAUNCH_CHECK("k_gemm_any");
  return EW_OK;
}

// In the rows' type, or fp32.
template <int WAY, typename TW>
int launch_any_bf16(int epilogue, const GemmArgs& a, hipStream_t st) {
  return epilogue == kEpF32 ? launch_any<WAY, uint16_t, TW, kEpF32>(a, st) : launch_any<WAY, uint16_t, TW, kEpBf16>(a, st);
}

}  // namespace

int launch_gemm_any(int way, int weights, int epilogue, bool bf16, const GemmArgs& a, hipStream_t st) {
  if (weights == kW4) return epilogue == kEpSwiglu ? launch_any<kFwd, uint16_t, uint8_t, kEpSwiglu>(a, st) : launch_any<kFwd, uint16_t, uint8_t, kEpBf16>(a, st);
  if (epilogue == kEpBack) return bf16 ? launch_any<kFwd, uint16_t, uint16_t, kEpBack>(a, st) : launch_any<kFwd, float, float, kEpBack>(a, st);
  if (bf16) {
    if (way == kFwd) return launch_any<kFwd, uint16_t, uint16_t, kEpBf16>(a, st);
    if (way == kDgrad) return launch_any_bf16<kDgrad, uint16_t>(epilogue, a, st);
    return launch_any_bf16<kWgrad, uint16_t>(epilogue, a, st);
  }
  if (way == kFwd) return launch_any<kFwd, float, float, kEpF32>(a, st);
  if (way == kDgrad) return launch_any<kDgrad, float, float, kEpF32>(a, st);
  return launch_any<kWgrad, float, float, kEpF32>(a, st);
}

int launch_gemm(int way, int weights, int epilogue, bool bf16, const GemmArgs& a, hipStream_t st) {
  if (stream_takes(way, weights, epilogue, a)) return launch_stream(way, weights, epilogue, a, st);
  if (tile_takes(way, weights, epilogue, a)) return launch_tile(way, weights, epilogue, a, st);
  return launch_gemm_any(way, weights, epilogue, bf16, a, st);
}

int check_rows(const char* who, int num_tokens, int num_rows, int k, int P, const void* counts, const void* offsets, const void* pair_of_row) {
  if (num_tokens < 0 || num_rows < 0 || k < 1 || P < 1)
    return fail(EW_ERR_INVALID_ARG, "%s: need num_tokens>=0, num_rows>=0, k>=1, P>=1 (got %d, %d, %d, %d)", who, num_tokens, num_rows, k, P);
  if (!counts || !offsets) return fail(EW_ERR_INVALID_ARG, "%s: NULL device pointer", who);
  if (const int rc = check_size(who, "num_rows", num_rows)) return rc;
  if (!pair_of_row && num_rows > (long long)num_tokens * k)
    return fail(EW_ERR_INVALID_ARG, "%s: without pair_of_row there are no more rows than pairs (num_rows=%d, num_tokens=%d, k=%d)", who, num_rows, num_tokens, k);
  return EW_OK;
}

int check_sizes(const char* who, const char* a, long long na, const char* b, long long nb) {
  const int rc = check_size(who, a, na);
  return rc ? rc : check_size(who, b, nb);
}

}  // namespace ew

extern "C" int moe_grouped_gemm(const void* x, int dtype, int num_tokens, int num_rows, int k, int K, int N, int P, int transposed,
                                const int32_t* counts, const int32_t* offsets, const int32_t* pair_of_row, const void* w_base, void* y,
                                void* stream) {
  using ew::fail;
  const char* who = "moe_grouped_gemm";
  if (K < 1 || N < 1) return fail(EW_ERR_INVALID_ARG, "%s: need K>=1, N>=1 (got %d, %d)", who, K, N);
  if (const int rc = ew::check_sizes(who, "K", K, "N", N)) return rc;
  if (dtype != EW_F32 && dtype != EW_BF16) return fail(EW_ERR_INVALID_ARG, "%s: unknown dtype %d", who, dtype);
  if (num_rows == 0 && k >= 1 && P >= 1) return EW_OK;
  if (const int rc = ew::check_rows(who, num_tokens, num_rows, k, P, counts, offsets, pair_of_row)) return rc;
  if (!x || !w_base || !y) return fail(EW_ERR_INVALID_ARG, "%s: NULL device pointer", who);
  ew::GemmArgs a{};
  a.g = {counts, offsets, pair_of_row, P, num_rows, k};
  a.x = x; a.w = w_base; a.out = y; a.K = K; a.N = N; a.x_rows = num_tokens;
  a.slot_bytes = (size_t)N * K * (dtype == EW_BF16 ? 2 : 4);
  return ew::launch_gemm(transposed ? ew::kDgrad : ew::kFwd, dtype == EW_BF16 ? ew::kWBf16 : ew::kWF32,
                         dtype == EW_BF16 ? ew::kEpBf16 : ew::kEpF32, dtype == EW_BF16, a, (hipStream_t)stream);
}

extern "C" int moe_grouped_gemm_wgrad(const void* dy, const void* x, int dtype, int num_tokens, int num_rows, int k, int K, int N, int P,
                                      const int32_t* counts, const int32_t* offsets, const int32_t* pair_of_row, int first_slot,
                                      int num_slots, int dw_dtype, int accumulate, void* dw, void* stream) {
  using ew::fail;
  const char* who = "moe_grouped_gemm_wgrad";
  if (K < 1 || N < 1) return fail(EW_ERR_INVALID_ARG, "%s: need K>=1, N>=1 (got %d, %d)", who, K, N);
  if (const int rc = ew::check_sizes(who, "K", K, "N", N)) return rc;
  if (dtype != EW_F32 && dtype != EW_BF16) return fail(EW_ERR_INVALID_ARG, "%s: unknown dtype %d", who, dtype);
  if (dw_dtype != EW_F32 && !(dw_dtype == EW_BF16 && dtype == EW_BF16))
    return fail(EW_ERR_INVALID_ARG, "%s: dw is float32, or bfloat16 for bfloat16 rows (dw_dtype=%d)", who, dw_dtype);
  if (accumulate && dw_dtype != EW_F32) return fail(EW_ERR_UNSUPPORTED, "%s: only float32 gradients accumulate", who);
  if (const int rc = ew::check_rows(who, num_tokens, num_rows, k, P, counts, offsets, pair_of_row)) return rc;
  if (first_slot < 0 || num_slots < 0 || first_slot > P - num_slots)
    return fail(EW_ERR_INVALID_ARG, "%s: slots [%d, %d + %d) outside 0..P=%d", who, first_slot, first_slot, num_slots, P);
  if (num_slots == 0) return EW_OK;
  if (!dw || (num_rows > 0 && (!dy || !x))) return fail(EW_ERR_INVALID_ARG, "%s: NULL device pointer", who);
  ew::GemmArgs a{};
  a.g = {counts, offsets, pair_of_row, P, num_rows, k};
  a.x = x; a.w = dy; a.out = dw; a.K = K; a.N = N; a.x_rows = num_tokens;
  a.first_slot = first_slot; a.num_slots = num_slots; a.accumulate = accumulate != 0;
  return ew::launch_gemm(ew::kWgrad, dtype == EW_BF16 ? ew::kWBf16 : ew::kWF32, dw_dtype == EW_F32 ? ew::kEpF32 : ew::kEpBf16, dtype == EW_BF16, a,
                         (hipStream_t)stream);
}
