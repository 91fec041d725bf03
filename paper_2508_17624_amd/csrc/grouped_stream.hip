// Matrix products grouped by expert with few rows per slot: a stream of weights, in bf16 or in 4 bits, straight into registers.
//
// With a handful of rows per slot every weight is used once or a few times, so what counts is bytes in flight and how few instructions
// load them.  The waves of a workgroup split the contraction, up to four blocks of 128 elements each; a wave keeps its part of up to 16 TL rows of x in
// registers and streams strip after strip of 16 features past it with v_mfma_f32_16x16x32_bf16: a lane's 16-byte load of weights is its
// operand, neither LDS nor barrier stands between a load and its use.  Every R strips the waves' partial sums meet in LDS.
// A lane (feature l % 16, quarter q = l / 16) holds of a block of 128 contraction elements
//   bf16:   elements 32 j + 8 q .. + 7 for MFMA j = 0 .. 3, one load each
//   4 bits: elements 32 q .. + 31 in one load, MFMA j takes elements 8 j .. + 7 of them: a lane's load is exactly one group, with one scale,
//           and v_cvt_scalef32_pk_bf16_fp4 makes two bf16 values of them at a time, exactly, scale included; a row's scales of all
//           four blocks are one load
// and x is loaded to match (any order of the contraction will do as long as both operands have the same).
// Both products of the FFN in 4 bits take 68 + 42 us at 64 tokens on 20 adapters of 2048 x 1408 (501 MB, 4.5 TB/s); the first product in bf16, four
// adapters, 165 (933 MB, 5.6 TB/s).  What keeps the 4-bit stream from the other's rate is in part the loads of scales, one load in five, of which
// the four lanes of a feature fetch the same 16 bytes: without them 64 + 36; without the conversion it takes as long as with it.  (Waves that walked
// over the whole contraction, loading x and scales block by block, three loads per strip and block instead of 1.25, took 163 for both.)
#include "grouped_gemm.h"

#include <type_traits>

namespace ew {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kBlock = 128;                 // contraction elements of a step
constexpr uint32_t kNowhere = 0xFFFFFF00u;  // an offset past every descriptor's end: reads as zero

using Rsrc = __amdgpu_buffer_rsrc_t;
__device__ __forceinline__ Rsrc resource(const void* p, uint32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), (short)0, (int)bytes, 0x00027000);
}
__device__ __forceinline__ u32x4 load16(Rsrc r, uint32_t off, uint32_t uniform_off) {
  return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, (int)off, (int)uniform_off, 0));
}

// A strip's weights of one block in registers.
template <int WT>
struct Strip;
template <>
struct Strip<kWBf16> {
  u32x4 w[4];
  __device__ __forceinline__ bf16x8 get(int j, int) const { return __builtin_bit_cast(bf16x8, w[j]); }
};
template <>
struct Strip<kW4> {
  u32x4 codes;
  uint32_t scales;  // of the row's four groups
  __device__ __forceinline__ bf16x8 get(int j, int q) const {
    const float scale = __uint_as_float((scales >> (8 * q) & 255u) << 23);
    u32x4 v;
    v[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes[j], scale, 0));
    v[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes[j], scale, 1));
    v[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes[j], scale, 2));
    v[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes[j], scale, 3));
    return __builtin_bit_cast(bf16x8, v);
  }
};

__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {
  return (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)a) | (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)b) << 16;
}

// NW: waves of a workgroup; TL: row tiles; R: strips of a round; D: strips in flight; WPE: waves per SIMD.
template <int WT_, int NW_, int TL_, int EP_, int R_, int D_, int WPE_>
struct Cfg {
  static constexpr int WT = WT_, NW = NW_, TL = TL_, EP = EP_, R = R_, D = D_, WPE = WPE_;
  // Blocks of the contraction that a wave holds of x: 64 registers a row tile, beside as many of a bf16 strip.  For bf16 that ends at K = 2048 with four
  // waves; eight are slower than the tiles (64 slots of 2816 features, 1 to 6 rows, eight waves / tiles, us: K = 2560 196 to 202 / 164 to 165, 4096 265
  // to 271 / 252 to 256; at 2048, four waves: 128 to 135 / 142 to 143).
  static constexpr int XB = 4;
  static constexpr bool GATED = EP == kEpSwiglu;  // strips come in pairs, gate and up
};
template <int WT>
struct StripRun;
template <>
struct StripRun<kW4> {
  u32x4 codes[4], scales;  // a row's four groups of a block per word
  __device__ __forceinline__ Strip<kW4> block(int b) const { return {codes[b], scales[b]}; }
};
template <>
struct StripRun<kWBf16> {
  Strip<kWBf16> blocks[4];
  __device__ __forceinline__ Strip<kWBf16> block(int b) const { return blocks[b]; }
};

template <typename C, int TL>
__device__ __forceinline__ void body(const GemmArgs& a, const RowChunk& ch, int s0, int strips, f32x4* parts) {
  const int lane = threadIdx.x & 63, m = lane & 15, q = lane >> 4, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), K = a.K, N = a.N;
  const bool mapped = a.g.por != nullptr || a.g.k > 1;
  const int nkb = (K + kBlock - 1) / kBlock, kb0 = wave * nkb / C::NW, n_kb = (wave + 1) * nkb / C::NW - kb0;
  const Rsrc rw = resource((const unsigned char*)a.w + (size_t)ch.slot * a.slot_bytes, (uint32_t)a.slot_bytes);
  const Rsrc rx = mapped ? resource(a.x, (uint32_t)a.x_rows * (uint32_t)K * 2u)
                         : resource((const unsigned char*)a.x + (size_t)ch.first * K * 2, (uint32_t)ch.rows * (uint32_t)K * 2u);
  const uint32_t scales_at = (uint32_t)w4_scales_at(C::GATED ? 2 * N : N, K);
  // Uniform offsets stay within the row, and so within their descriptor, also where the lanes' say that there is nothing to load.
  auto uniform_at = [&](int b, int byte) {
    const int at = (kb0 + b) * (kBlock * 2) + byte;
    return b < n_kb && at < 2 * K ? (uint32_t)at : 0u;
  };
  StripRun<C::WT> w[C::D];
  auto load = [&](int d, int s) {  // strip s of this workgroup; none: zeros, without memory traffic
    const int f = 16 * (s0 + (C::GATED ? s >> 1 : s)) + m;
    const uint32_t row = (uint32_t)(C::GATED && (s & 1) ? f + N : f);
    const bool there = s < strips;
    if constexpr (C::WT == kW4) {
      const uint32_t at = there ? row * (uint32_t)(K / 2) + 16 * q : kNowhere;
#pragma unroll
      for (int b = 0; b < C::XB; ++b) w[d].codes[b] = load16(rw, b < n_kb ? at : kNowhere, b < n_kb ? (uint32_t)(kb0 + b) * (kBlock / 2) : 0u);
      w[d].scales = load16(rw, there ? scales_at + row * (uint32_t)(K / 32) : kNowhere, (uint32_t)kb0 * (kBlock / 32));
    } else {
      const uint32_t at = there && f < N ? (row * (uint32_t)K + 8 * q) * 2 : kNowhere;
#pragma unroll
      for (int b = 0; b < C::XB; ++b)
#pragma unroll
        for (int jj = 0; jj < 4; ++jj)
          w[d].blocks[b].w[jj] = load16(rw, b < n_kb && (kb0 + b) * kBlock + 32 * jj + 8 * q < K ? at : kNowhere, uniform_at(b, 64 * jj));
    }
  };
#pragma unroll
  for (int d = 0; d < C::D; ++d) load(d, d);
  u32x4 x[TL][C::XB][4];
#pragma unroll
  for (int t = 0; t < TL; ++t) {
    const int r = 16 * t + m;
    uint32_t src = (uint32_t)r;
    if (mapped) src = r < ch.rows ? (uint32_t)source_row(a.g, ch.first + r) : 0u;
    const uint32_t at = r < ch.rows ? (src * (uint32_t)K + (C::WT == kW4 ? 32 * q : 8 * q)) * 2 : kNowhere;
#pragma unroll
    for (int b = 0; b < C::XB; ++b)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const bool there = b < n_kb && (C::WT == kW4 || (kb0 + b) * kBlock + 32 * j + 8 * q < K);
        x[t][b][j] = load16(rx, there ? at : kNowhere, uniform_at(b, (C::WT == kW4 ? 16 : 64) * j));
      }
  }
  for (int s = 0; s < strips; s += C::R) {
    f32x4 acc[C::R][TL] = {};
#pragma unroll
    for (int r = 0; r < C::R; ++r) {
      const int d = r % C::D;
      static_assert(C::R % C::D == 0, "a strip's registers are known when compiled");
#pragma unroll
      for (int b = 0; b < C::XB; ++b) {
        if (b >= n_kb) continue;  // (uniform; the scales behind the row's last are another row's)
        const Strip<C::WT> block = w[d].block(b);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const bf16x8 f = block.get(j, q);
#pragma unroll
          for (int t = 0; t < TL; ++t) acc[r][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, __builtin_bit_cast(bf16x8, x[t][b][j]), acc[r][t], 0, 0, 0);
        }
      }
      load(d, s + r + C::D);
    }
    // (two buffers: whoever writes one again has met, at the barrier between, all that read it)
    f32x4* part = parts + (s / C::R & 1) * C::NW * C::R * C::TL * 64;
#pragma unroll
    for (int r = 0; r < C::R; ++r)
#pragma unroll
      for (int t = 0; t < TL; ++t) part[(wave * C::R * TL + r * TL + t) * 64 + lane] = acc[r][t];
    __syncthreads();
    auto sum = [&](int r, int t) {
      f32x4 v = part[(r * TL + t) * 64 + lane];
#pragma unroll(C::NW <= 8 ? C::NW : 3)  // (16 partial sums of two strips at once do not fit beside x)
      for (int p = 1; p < C::NW; ++p) v += part[(p * C::R * TL + r * TL + t) * 64 + lane];
      return v;
    };
    constexpr int OUT = C::GATED ? C::R / 2 : C::R;  // results of a round, dealt to the waves
#pragma unroll
    for (int o = 0; o < (OUT * TL + C::NW - 1) / C::NW; ++o) {
      const int i = o * C::NW + wave, strip = i / TL, t = i - strip * TL, row = 16 * t + m;
      const int f = 16 * (s0 + (C::GATED ? s >> 1 : s) + strip) + 4 * q;
      if (strip >= OUT || s + (C::GATED ? 2 : 1) * strip >= strips || row >= ch.rows || f >= N) continue;
      f32x4 v;
      if constexpr (C::GATED) {
        const f32x4 g = sum(2 * strip, t), u = sum(2 * strip + 1, t);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = swiglu(g[e], u[e]);
      } else {
        v = sum(strip, t);
      }
      *(u32x2*)((uint16_t*)a.out + (size_t)(ch.first + row) * N + f) = (u32x2){bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3])};
    }
  }
}

template <typename C>
__global__ __launch_bounds__(64 * C::NW, C::WPE) void k_stream(GemmArgs a, int groups, int per_group) {
  __shared__ f32x4 s_part[2 * C::NW * C::R * C::TL * 64];
  const int c = blockIdx.x / groups, g = blockIdx.x - c * groups;
  const RowChunk ch = find_chunk<16 * C::TL, 16>(a.g, c);
  if (ch.slot < 0 || ch.rows == 0) return;
  const int s0 = g * per_group, n = min(per_group, (a.N + 15) / 16 - s0), strips = C::GATED ? 2 * n : n;  // in strips of results
  if (C::TL == 1 || ch.rows <= 16) body<C, 1>(a, ch, s0, strips, s_part);
  else body<C, C::TL>(a, ch, s0, strips, s_part);
}

template <int WT, int NW, int TL, int EP, int R, int D, int WPE>
int launch_cfg(const GemmArgs& a, int per_group, hipStream_t st) {
  using C = Cfg<WT, NW, TL, EP, R, D, WPE>;
  const int groups = ceil_div(ceil_div(a.N, 16), per_group);
  const long long units = max_chunks(a.g.rows, a.g.P, 16 * TL) * groups;
  if (const int rc = check_grid(units, 64 * NW)) return rc;
  hipLaunchKernelGGL((k_stream<C>), dim3((unsigned)units), dim3(64 * NW), 0, st, a, groups, per_group);
  EW_LAUNCH_CHECK("k_stream");
  return EW_OK;
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

// Strips for a workgroup: 16, or as many fewer as it takes to have four workgroups a CU, but 4 at least; 2 where even those make no more than
// one a CU and nothing is left but latency.  (us, 2048 x 1408, one row on so many slots, 4 / 2 strips: 4 bits, both products: 1 12.1 / 10.0,
// 2 12.2 / 10.0, 12 20.8 / 22.6; bf16, first product: 1 11.8 / 8.1.)
int strips_per_group(const GemmArgs& a, int strips, int most) {
  const long long used = a.g.P < a.g.rows ? a.g.P : a.g.rows;
  while (most > 4 && used * strips < 1024ll * most) most /= 2;
  return used * strips <= 2 * 256 ? 2 : most;
}

template <int NW, int EP>
int launch_w4(const GemmArgs& a, hipStream_t st) {
  constexpr int PAIR = EP == kEpSwiglu ? 2 : 1, WPE = NW == 4 ? 3 : NW / 4;
  const long long used = a.g.P < a.g.rows ? a.g.P : a.g.rows;
  const int strips = PAIR * a.N / 16;
  if (NW == 16 || a.g.rows <= 16 * used)
    return launch_cfg<kW4, NW, 1, EP, 2, NW == 16 ? 1 : 2, WPE>(a, strips_per_group(a, strips, 16) / PAIR, st);
  constexpr int NW2 = NW == 16 ? 8 : NW;  // (never 16 here)
  return launch_cfg<kW4, NW2, 2, EP, 2, 2, 2>(a, strips_per_group(a, strips, 16) / PAIR, st);
}
template <int EP>
int launch_w4_waves(const GemmArgs& a, hipStream_t st) {
  if (a.K <= 16 * kBlock) return launch_w4<4, EP>(a, st);
  if (a.K <= 32 * kBlock) return launch_w4<8, EP>(a, st);
  return launch_w4<16, EP>(a, st);
}

}  // namespace

bool stream_takes(int way, int weights, int epilogue, const GemmArgs& a) {
  const unsigned long long lim = (1ull << 32) - 65536;
  if (way != kFwd || !(weights == kW4 ? epilogue == kEpBf16 || epilogue == kEpSwiglu : weights == kWBf16 && epilogue == kEpBf16)) return false;
  if (!aligned16(a.x) || !aligned16(a.w) || !aligned16(a.out) || a.N % 8) return false;
  if (weights == kW4 ? a.K % kBlock || a.N % 16 : a.K % 8) return false;
  const bool mapped = a.g.por != nullptr || a.g.k > 1;
  if (mapped && (unsigned long long)a.x_rows * a.K * 2 >= lim) return false;
  if (a.slot_bytes >= lim) return false;
  // What the waves of a workgroup can hold of x, and where it is faster than the tiles: us, 64 slots of 2048 x 1408 with so many rows, this kernel / tiles:
  // 4 bits, both products: 16 81 / 129, 32 105 / 132, 48 161 / 145; bf16, first product: 4 134 / 141, 12 142 / 143, 24 155 / 146 (weights of
  // 16 slots, which the memory-side cache holds: 4 33 / 30).
  // The host knows the average over all slots, and these lines hold where all are in use.  Slots without rows move them: the same 64 slots of base experts in a
  // pool of 384 take the stream up to six times as many rows per slot in use.  This kernel / tiles there, us: 4 bits 24 116 / 148, 48 167 / 161, 94 296 /
  // 182, 188 382 / 318 (a pool of 64: 100, 150, 169, 241); bf16 6 163 / 152, 24 159 / 155 (130, 148).  Counts are on the device, where nothing
  // chooses between kernels.
  const long long used = a.g.P < a.g.rows ? a.g.P : a.g.rows;
  // Beyond K = 4096 one tile of 16 rows is all that fits beside the partial sums, and 32 rows would read the weights twice: 8192 x 1024, 64
  // slots: 16 rows 93 / 106, 32 rows 169 / 110 (both products with a hidden size of 8192: 222 / 333 at 16 rows).
  if (weights == kW4) return a.K <= 64 * kBlock && a.g.rows <= (a.K <= 32 * kBlock ? 32 : 16) * used;
  return a.K <= 16 * kBlock && a.g.rows <= 6 * used;
}

int launch_stream(int way, int weights, int epilogue, const GemmArgs& a, hipStream_t st) {
  (void)way;
  if (weights == kW4) return epilogue == kEpSwiglu ? launch_w4_waves<kEpSwiglu>(a, st) : launch_w4_waves<kEpBf16>(a, st);
  // Two row tiles where a slot can have many rows: slots of 17 to 32 read their weights once (64 slots in use of 384, 24 rows each: one tile 262 us, two 159).
  // Spread evenly, up to 6 rows a slot, one tile is up to 4 % faster (2048 x 2816, us: 128 slots 226 rows 219 / 218, 506 246 / 256, 773 283 / 288; 384 slots
  // 1572 rows 716 / 727; with fewer tokens 0 to 9 %).
  const int tokens = a.g.por || a.g.k > 1 ? a.x_rows : a.g.rows, strips = ceil_div(a.N, 16);
  if (tokens <= 64) return launch_cfg<kWBf16, 4, 1, kEpBf16, 2, 1, 3>(a, strips_per_group(a, strips, 4), st);
  return launch_cfg<kWBf16, 4, 2, kEpBf16, 2, 1, 2>(a, strips_per_group(a, strips, 16), st);
}

}  // namespace ew
