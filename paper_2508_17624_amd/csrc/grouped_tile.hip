// Matrix products grouped by expert on the bf16 matrix cores, many rows per slot: forward, input gradient, weight gradient.
//
// A workgroup makes one tile of TA outputs along the contiguous axis of the result ("features", operand A) times up to TB along the
// other ("rows", operand B) with v_mfma_f32_32x32x16_bf16, four waves of half of the features x half of the rows: at 256 x 256 a wave's 128 x 128
// sums fill half of its registers and 8 operand reads feed 16 MFMAs (eight waves of 64 x 128: 6 for 8, 2 to 5 % slower).
// The contraction comes in slabs of 64 through an LDS ring, filled by LDS-direct loads while earlier slabs are multiplied.
//
// An operand lies in memory along the contraction (x, and w of the forward product) or across it (w of the input gradient, both
// operands of the weight gradient).  The first kind is staged as [rows][64] and read 16 bytes a lane; the second as [64][outputs] and read by
// ds_read_b64_tr_b16, which transposes 4 x 16 elements over 16 lanes on the way: no transposed copy is made in memory.  Both kinds of
// LDS rows are XOR-swizzled so that the reads of a wave cover all banks.
// MFMA row m = 8 a + 4 h + b of a feature fragment is feature 16 h + 4 a + b: a lane's 16 sums are neighbours.
//
// The operands are loaded through buffer descriptors: rows and contraction steps past the end read as zeros (a slot's sums never see what
// lies behind it, NaN or not), and no looked-up row, however wrong, is read outside x.  Counts and offsets are taken as they are but for the
// room of the row arrays, and so is pair_of_row where it is read.
#include "grouped_gemm.h"

#include <type_traits>

namespace ew {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kSlab = 64;                     // contraction elements
constexpr uint32_t kNowhere = 0xFFFFFF00u;    // an offset past every descriptor's end

// LDS rows along the contraction: 128 bytes in 8 pieces of 16, piece p of row r at p ^ swz(r).  Features are read in the order of the
// fragment (rows 0-7 and 16-23 together), rows in their own: 16 neighbouring lanes meet all 16 piece positions of two rows.
template <bool FEATURES>
__device__ __forceinline__ int swz(int r) { return FEATURES ? (r >> 1 & 3) | (r >> 4 & 1) << 2 : r >> 1 & 7; }

template <int OFF>
__device__ __forceinline__ void read_16(uint32_t at, u32x4& v) { asm volatile("ds_read_b128 %0, %1 offset:%2" : "=&v"(v) : "v"(at), "n"(OFF)); }
template <int OFF>
__device__ __forceinline__ void read_tr(uint32_t at, u32x2& v) { asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=&v"(v) : "v"(at), "n"(OFF)); }
__device__ __forceinline__ void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
template <int N>
__device__ __forceinline__ void wait_mem() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }  // all but the last N loads
__device__ __forceinline__ void in_order() { asm volatile("" ::: "memory"); }

// One operand's fragment of a k-step in registers.  The reads are issued without waiting; landed() is called behind the wait and
// names the registers, so that nothing uses them earlier.
template <bool ACROSS>
struct Frag;
template <>
struct Frag<false> {
  u32x4 v;
  template <int OFF> __device__ __forceinline__ void read(uint32_t at) { read_16<OFF>(at, v); }
  __device__ __forceinline__ void landed() { asm volatile("" : "+v"(v)); }
  __device__ __forceinline__ bf16x8 get() const { return __builtin_bit_cast(bf16x8, v); }
};
template <>
struct Frag<true> {
  u32x2 lo, hi;
  template <int OFF, int ROW> __device__ __forceinline__ void read(uint32_t at) { read_tr<OFF>(at, lo); read_tr<OFF + 4 * ROW>(at, hi); }
  __device__ __forceinline__ void landed() { asm volatile("" : "+v"(lo), "+v"(hi)); }
  __device__ __forceinline__ bf16x8 get() const { return __builtin_bit_cast(bf16x8, (u32x4){lo[0], lo[1], hi[0], hi[1]}); }
};

template <int WAY_, int TA_, int TB_, int EP_, bool MAPPED_, bool W4_>
struct Cfg {
  static constexpr int WAY = WAY_, TA = TA_, TB = TB_, EP = EP_;
  static constexpr bool MAPPED = MAPPED_;                            // rows of x are looked up
  static constexpr bool W4 = W4_;                                    // weights in 4 bits
  static constexpr bool A_ACROSS = WAY != kFwd, B_ACROSS = WAY == kWgrad;
  static constexpr bool GATED = EP == kEpSwiglu || EP == kEpBack;    // weights [2N, K]: a lane holds g and u of a feature
  static constexpr int WAVES = 4, THREADS = 64 * WAVES;        // two halves of the features x two halves of the rows
  static constexpr int MA = TA / 64, MB = TB / 64;                         // a wave's fragments; row fragment f of half b is rows 32 (b + 2 f) ..
  static constexpr int UNIT = TA * kSlab * 2, RING = 5, LDS = RING * UNIT;
  static constexpr int NL = UNIT / 1024 / WAVES;                     // load instructions of a wave for one operand's slab
  static constexpr int ROW = TA * 2;                                 // bytes of an LDS row across the contraction
  static constexpr int PPR = TA / 8, RPI = 64 / PPR;                 // its pieces of 16 bytes; rows of a load instruction
  static constexpr int WPE = TA == 256 ? 1 : 2;                      // waves per SIMD: what LDS has room for
  static_assert(TA == TB && LDS * WPE <= 160 * 1024, "LDS budget of a CU");
  static constexpr int RW = TA / 64;                                 // W4: features of a thread
  // Results of a wave and row fragment in LDS, on their way out: 32 rows.  (16 bytes more than a row: rows begin at different banks.)
  static constexpr int OUT_EL = EP == kEpF32 ? 4 : 2, OUT_ROW = (GATED ? MA / 2 : MA) * 32 * OUT_EL, OUT_PITCH = OUT_ROW + 16, OUT_WAVE = 32 * OUT_PITCH;
  static_assert(WAVES * OUT_WAVE <= LDS, "what the ring leaves when it is done");
  // first LDS row, along the contraction, of feature fragment i of half a
  static constexpr int feature_row(int a, int i) { return GATED ? (i < MA / 2 ? 0 : TA / 2) + a * (MA / 2) * 32 + i % (MA / 2) * 32 : (a * MA + i) * 32; }
};

__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {
  return (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)a) | (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)b) << 16;
}

using Rsrc = __amdgpu_buffer_rsrc_t;
__device__ __forceinline__ Rsrc resource(const void* p, uint32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), (short)0, (int)bytes, 0x00027000);
}
typedef __attribute__((address_space(3))) unsigned char lds_byte;
__device__ __forceinline__ void load_lds(Rsrc r, lds_byte* to, uint32_t off, uint32_t uniform_off) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void*)to, 16, (int)off, (int)uniform_off, 0, 0);
}

// LDS offsets of a slab's operands.
struct Slab { uint32_t a, b; };

// The K loop of a wave with NBF live row fragments.  step(kt): meets the others, says where slab kt lies; load(q): load instruction q of
// the 2 NL that belong to a slab.  They are spread over the MFMAs: a load stalls its wave while the CU's queue of outstanding lines is
// full, and all of a slab's loads in a row left the matrix cores without work for as long as they took (8192 x 8192 x 8192: 1201 us, with the
// loads alone 727 and everything but the loads 696).
template <typename C, int NBF, typename Step, typename Load>
__device__ __forceinline__ void multiply(int nk, const uint32_t (&fa)[C::MA], const uint32_t (&fb)[2], f32x16 (&acc)[C::MA][NBF], Step step, Load load) {
  Frag<C::A_ACROSS> a[2][C::MA];
  Frag<C::B_ACROSS> b[2][NBF];
  Slab at{};
  auto read = [&](auto c_tag, auto ks_tag) {
    constexpr int c = decltype(c_tag)::value, ks = decltype(ks_tag)::value;
    auto read_a = [&](auto i_tag) {
      constexpr int i = decltype(i_tag)::value;
      if constexpr (i < C::MA) {
        if constexpr (C::A_ACROSS) a[c][i].template read<ks * 16 * C::ROW, C::ROW>(at.a + fa[i]);
        else a[c][i].template read<(C::feature_row(0, i) - C::feature_row(0, 0)) * 128>((at.a + fa[0]) ^ (uint32_t)(32 * ks));
      }
    };
    auto read_b = [&](auto f_tag) {
      constexpr int f = decltype(f_tag)::value;
      if constexpr (f < NBF) {
        if constexpr (C::B_ACROSS) b[c][f].template read<ks * 16 * C::ROW + (f >> 1) * 256, C::ROW>(at.b + fb[f & 1]);
        else b[c][f].template read<f * 64 * 128>((at.b + fb[0]) ^ (uint32_t)(32 * ks));
      }
    };
    read_a(std::integral_constant<int, 0>{}); read_b(std::integral_constant<int, 0>{});
    read_a(std::integral_constant<int, 1>{}); read_b(std::integral_constant<int, 1>{});
    read_a(std::integral_constant<int, 2>{}); read_b(std::integral_constant<int, 2>{});
    read_a(std::integral_constant<int, 3>{}); read_b(std::integral_constant<int, 3>{});
  };
  auto landed = [&](auto c_tag) {
    constexpr int c = decltype(c_tag)::value;
    wait_lds();
#pragma unroll
    for (int i = 0; i < C::MA; ++i) a[c][i].landed();
#pragma unroll
    for (int f = 0; f < NBF; ++f) b[c][f].landed();
  };
  constexpr int PER = 2 * C::NL / 4;  // loads of a k-step, behind groups of MFMAs
  auto mul = [&](auto c_tag, auto part_tag, auto odd_tag) {
    constexpr int c = decltype(c_tag)::value, part = decltype(part_tag)::value;
#pragma unroll
    for (int f = 0; f < NBF; ++f) {
#pragma unroll
      for (int i = 0; i < C::MA; ++i) acc[i][f] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[c][i].get(), b[c][f].get(), acc[i][f], 0, 0, 0);
      if constexpr (part >= 0) {
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int q = 0; q < PER; ++q)
          if (q * NBF / PER == f) load(part * PER + q, odd_tag);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  };
  const std::integral_constant<int, 0> _0{};
  const std::integral_constant<int, 1> _1{};
  const std::integral_constant<int, 2> _2{};
  const std::integral_constant<int, 3> _3{};
  // Reads run a k-step ahead of the products, across slabs too: what is multiplied first are zeros.
#pragma unroll
  for (int i = 0; i < C::MA; ++i) a[1][i] = {};
#pragma unroll
  for (int f = 0; f < NBF; ++f) b[1][f] = {};
  auto slab = [&](int kt, auto odd) {
    at = step(kt);
    read(_0, _0); mul(_1, _0, odd); landed(_0);
    read(_1, _1); mul(_0, _1, odd); landed(_1);
    read(_0, _2); mul(_1, _2, odd); landed(_0);
    read(_1, _3); mul(_0, _3, odd); landed(_1);
  };
  if constexpr (C::W4) {
    for (int kt = 0; kt < nk; kt += 2) {  // (an even number: K % 128 == 0)
      slab(kt, _0);
      slab(kt + 1, _1);
    }
  } else {
    for (int kt = 0; kt < nk; ++kt) slab(kt, _0);
  }
  mul(_1, std::integral_constant<int, -1>{}, _0);
}
template <typename C, typename Step, typename Load>
__device__ __forceinline__ void idle(int nk, Step step, Load load) {  // a wave without rows keeps loading
  auto slab = [&](int kt, auto odd) {
    step(kt);
#pragma unroll
    for (int q = 0; q < 2 * C::NL; ++q) load(q, odd);
    wait_lds();
  };
  for (int kt = 0; kt < nk; kt += C::W4 ? 2 : 1) {
    slab(kt, std::integral_constant<int, 0>{});
    if constexpr (C::W4) slab(kt + 1, std::integral_constant<int, 1>{});
  }
}

template <typename C>
__global__ __launch_bounds__(C::THREADS) __attribute__((amdgpu_waves_per_eu(C::WPE, C::WPE))) void k_tile(GemmArgs a, int tiles_a, int units, uint32_t by_k) {
  __shared__ __attribute__((aligned(1024))) unsigned char s_lds[C::LDS];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int K = a.K, N = a.N;
  // ---- which tile
  RowChunk ch;
  int a0, b0, na, nb, len, unit;
  if constexpr (C::WAY == kWgrad) {
    unit = unit_of_block(units);
    if (unit >= units) return;
    const int tiles = units / a.num_slots, slot = unit / tiles, t = unit - slot * tiles;
    const int s = a.first_slot + slot, off = a.g.offsets[s];
    ch = {s, off, max(0, min(a.g.counts[s], a.g.rows - off))};
    a0 = t % tiles_a * C::TA; b0 = t / tiles_a * C::TB;
    na = K; nb = N; len = ch.rows;
    unit = slot;
    if (len == 0 && a.accumulate) return;
  } else {
    const int n = count_chunks<C::TB>(a.g) * tiles_a;
    unit = unit_of_block(n);
    if (unit >= n) return;
    const int c = unit / tiles_a;
    ch = find_chunk<C::TB, 32>(a.g, c);
    if (ch.slot < 0 || ch.rows == 0) return;
    a0 = (unit - c * tiles_a) * (C::GATED ? C::TA / 2 : C::TA); b0 = 0;
    na = N; nb = ch.rows; len = K;
  }
  const int nk = (len + kSlab - 1) / kSlab;
  const int live_b = min(C::TB, nb - b0);
  // ---- staging: load instruction n of this wave fills 1 KB of an operand's LDS rows
  const unsigned char *pa, *pb;                           // what the operands' descriptors begin with, and their bytes
  uint32_t na_bytes, nb_bytes;
  uint32_t oa[C::NL], ob[C::NL], sa, sb;                  // byte offsets of a lane; bytes a slab further
  const unsigned char *wp = (const unsigned char*)a.w, *xp = (const unsigned char*)a.x;
  const uint32_t x_bytes = (uint32_t)a.x_rows * (uint32_t)K * 2u;
  auto across_row = [&](int n) { return (wave * C::NL + n) * C::RPI + lane / C::PPR; };  // along the contraction
  auto along_row = [&](int n) { return (wave * C::NL + n) * 8 + (lane >> 3); };
  if constexpr (C::A_ACROSS) {
    constexpr bool looked_up = C::WAY == kWgrad && C::MAPPED;
#pragma unroll
    for (int n = 0; n < C::NL; ++n) {
      const int kr = across_row(n), piece = lane % C::PPR ^ (kr & 3) << 2;
      oa[n] = ((looked_up ? 0u : (uint32_t)kr * (uint32_t)na) + a0 + piece * 8) * 2;
    }
    sa = looked_up ? 0u : kSlab * (uint32_t)na * 2;
    if constexpr (C::WAY == kDgrad) { pa = wp + (size_t)ch.slot * a.slot_bytes; na_bytes = (uint32_t)a.slot_bytes; }
    else if constexpr (looked_up) { pa = xp; na_bytes = x_bytes; }
    else { pa = xp + (size_t)ch.first * K * 2; na_bytes = (uint32_t)len * (uint32_t)K * 2u; }
  } else {
#pragma unroll
    for (int n = 0; n < C::NL; ++n) {
      const int r = along_row(n), piece = (lane & 7) ^ swz<true>(r);
      const int f = a0 + (C::GATED && r >= C::TA / 2 ? r - C::TA / 2 : r);
      oa[n] = f < N ? ((uint32_t)(C::GATED && r >= C::TA / 2 ? f + N : f) * (uint32_t)K + piece * 8) * 2 : kNowhere;
    }
    sa = kSlab * 2;
    pa = wp + (size_t)ch.slot * a.slot_bytes;
    na_bytes = (uint32_t)a.slot_bytes;
  }
  if constexpr (C::B_ACROSS) {
#pragma unroll
    for (int n = 0; n < C::NL; ++n) {
      const int kr = across_row(n), piece = lane % C::PPR ^ (kr & 3) << 2;
      ob[n] = ((uint32_t)kr * (uint32_t)N + b0 + piece * 8) * 2;
    }
    sb = kSlab * (uint32_t)N * 2;
    pb = wp + (size_t)ch.first * N * 2;
    nb_bytes = (uint32_t)len * (uint32_t)N * 2u;
  } else {
#pragma unroll
    for (int n = 0; n < C::NL; ++n) {
      const int r = along_row(n), piece = (lane & 7) ^ swz<false>(r);
      uint32_t src = (uint32_t)r;
      if constexpr (C::MAPPED) src = r < ch.rows ? (uint32_t)source_row(a.g, ch.first + r) : 0u;
      ob[n] = r < ch.rows ? (src * (uint32_t)K + (C::W4 ? (piece >> 1) * 32 + (piece & 1) * 8 : piece * 8)) * 2 : kNowhere;
    }
    sb = kSlab * 2;
    pb = C::MAPPED ? xp : xp + (size_t)ch.first * K * 2;
    nb_bytes = C::MAPPED ? x_bytes : (uint32_t)ch.rows * (uint32_t)K * 2u;
  }
  auto lds_at = [&](int unit, int n) { return (lds_byte*)s_lds + (unit * C::UNIT + (wave * C::NL + n) * 1024); };
  // The K loop's loads take no branches.  A slab that does not exist is loaded through a descriptor of no bytes (the uniform
  // offsets stay within their descriptors), rows that do not exist from kNowhere: neither costs memory traffic, and the number of loads in
  // flight is always the same.
  // Rows of the weight gradient's x are looked up a slab ahead of their loads: a wave's 16 rows of a slab in one load, handed to the lanes
  // that need them.  (Every lane loading its own rows is half as many load instructions again: 49152 rows, 2816 x 2048: 769 us instead of 680.)
  constexpr bool LOOK_UP = C::WAY == kWgrad && C::MAPPED;
  uint32_t row_next = 0, step_a[LOOK_UP ? C::NL : 1] = {};  // token rows on their way; byte offsets of the present ones
  auto look_up = [&](int kt) {                               // slab kt's rows; those asked for before become offsets
    if constexpr (LOOK_UP) {
      static_assert(C::NL * C::RPI == 16, "a wave's rows of a slab");
      const int r = kt * kSlab + wave * 16 + (lane & 15);
      const uint32_t token = by_k ? __umulhi(row_next, by_k) : row_next, at = r - kSlab < len ? token * ((uint32_t)K * 2) : 0xFFFF0000u;  // (past the end with the offset in the row, which is below 2^16)
#pragma unroll
      for (int n = 0; n < C::NL; ++n) step_a[n] = oa[n] + (uint32_t)__shfl((int)at, n * C::RPI + lane / C::PPR, 64);
      row_next = r < len ? (uint32_t)(a.g.por ? a.g.por[ch.first + r] : ch.first + r) : 0u;
    }
  };
  // The last slab of a contraction that 64 does not divide: pieces past its end (rows across it end by their descriptor).
  auto cut_tail = [&](uint32_t (&off)[C::NL], int kt, auto features) {
    if (kt * kSlab + kSlab <= K) return;
#pragma unroll
    for (int n = 0; n < C::NL; ++n)
      if (kt * kSlab + ((lane & 7) ^ swz<decltype(features)::value>(along_row(n))) * 8 >= K) off[n] = kNowhere;
  };
  // W4: codes come two slabs at a time, 64 bytes of a feature by four neighbouring lanes, a lane's 16 bytes being one group of 32 with one
  // scale.  The even slab of the two takes the first half of every group, the odd one the second (x is loaded to match), so all lanes turn
  // half of what they hold into bf16 in LDS, a slab ahead of its use.  (A lane with 32 bytes of a feature of its own instead, a slab's worth,
  // touches 64 lines per load instruction: 64 slots of 16 rows, both products of the FFN, 161 us instead of 147.)
  // Codes are asked for two to four slabs before their use but are only one slab in flight: outstanding loads are counted in order, and the wait for the
  // rows of a slab is a wait for the codes before them.  What the 4-bit form costs, 3999 tokens on 20 adapters of 2048 x 1408, both kernels: 513 + 278 us,
  // without the conversion 496 + 267, without the LDS writes of its results either 451 + 248 (a quarter of the LDS cycles are bank conflicts there).
  u32x4 codes[C::RW], codes_next[C::RW];
  uint32_t scales[C::RW] = {}, scales_next[C::RW] = {}, w4_codes[C::RW], w4_scales[C::RW];
  if constexpr (C::W4) {
#pragma unroll
    for (int i = 0; i < C::RW; ++i) {
      const int r = wave * (C::TA / 4) + 16 * i + (lane >> 2), f = a0 + (C::GATED && r >= C::TA / 2 ? r - C::TA / 2 : r);
      const uint32_t row = (uint32_t)(C::GATED && r >= C::TA / 2 ? f + N : f);
      w4_codes[i] = f < N ? row * (uint32_t)(K / 2) + 16 * (lane & 3) : kNowhere;
      w4_scales[i] = f < N ? (uint32_t)w4_scales_at(C::GATED ? 2 * N : N, K) + row * (uint32_t)(K / 32) + (lane & 3) : kNowhere;
    }
  }
  auto fetch_codes = [&](int two) {
    if constexpr (C::W4) {
      const Rsrc r = resource(pa, 2 * two < nk ? na_bytes : 0u);
      if (2 * two >= nk) two = 0;
#pragma unroll
      for (int i = 0; i < C::RW; ++i) codes_next[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, (int)w4_codes[i], two * kSlab, 0));
    }
  };
  auto fetch_scales = [&](int two) {
    if constexpr (C::W4) {
      const Rsrc r = resource(pa, 2 * two < nk ? na_bytes : 0u);
      if (2 * two >= nk) two = 0;
#pragma unroll
      for (int i = 0; i < C::RW; ++i) scales_next[i] = __builtin_amdgcn_raw_buffer_load_b8(r, (int)w4_scales[i], two * (kSlab / 16), 0);
    }
  };
  auto fetched = [&] {
#pragma unroll
    for (int i = 0; i < C::RW; ++i) {
      codes[i] = codes_next[i];
      scales[i] = scales_next[i];
    }
  };
  auto stage = [&](int unit, int n, auto half_tag) {  // 16 bytes in LDS: word n & 1 of half a group of feature n / 2
    if constexpr (C::W4) {
      constexpr int half = decltype(half_tag)::value;
      const int r = wave * (C::TA / 4) + 16 * (n >> 1) + (lane >> 2);
      const float scale = __uint_as_float(scales[n >> 1] << 23);
      const uint32_t word = codes[n >> 1][2 * half + (n & 1)];
      u32x4 v;
      v[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, 0));
      v[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, 1));
      v[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, 2));
      v[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, 3));
      const uint32_t at = (uint32_t)(uintptr_t)(lds_byte*)s_lds + unit * C::UNIT + r * 128 + ((2 * (lane & 3) + (n & 1)) ^ swz<true>(r)) * 16;
      asm volatile("ds_write_b128 %0, %1" ::"v"(at), "v"(v));
    }
  };
  auto load_a = [&](int kt, int unit, int n) {
    load_lds(resource(pa, kt < nk ? na_bytes : 0u), lds_at(unit, n), LOOK_UP ? step_a[LOOK_UP ? n : 0] : oa[n], kt < nk ? (uint32_t)kt * sa : 0u);
  };
  auto load_b = [&](int kt, int unit, int n) {
    const uint32_t at = C::W4 ? (uint32_t)(kt >> 1) * 256 + (kt & 1) * 32 : (uint32_t)kt * sb;
    load_lds(resource(pb, kt < nk ? nb_bytes : 0u), lds_at(unit, n), ob[n], kt < nk ? at : 0u);
  };
  // ---- reading
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_byte*)s_lds;
  const int wa = wave >> 1, wb = wave & 1, h = lane >> 5;
  uint32_t fa[C::MA], fb[2];
  const int g = lane >> 4, c4 = lane & 3, kr = (g >> 1) * 8 + (lane & 15) / 4;  // across the contraction: a lane's row, and its four outputs
#pragma unroll
  for (int i = 0; i < C::MA; ++i) {
    if constexpr (C::A_ACROSS) {
      fa[i] = lds0 + kr * C::ROW + ((wa * C::MA + i) ^ (kr & 3)) * 64 + (16 * (c4 & 1) + 8 * (g & 1) + 4 * (c4 >> 1)) * 2;
    } else {
      const int m = lane & 31, r = C::feature_row(wa, 0) + 16 * (m >> 2 & 1) + 4 * (m >> 3) + (m & 3);
      fa[i] = lds0 + r * 128 + ((h ^ swz<true>(r)) << 4);
    }
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if constexpr (C::B_ACROSS) {
      fb[i] = lds0 + kr * C::ROW + ((wb + 2 * i) ^ (kr & 3)) * 64 + (16 * (g & 1) + 4 * c4) * 2;
    } else {
      const int r = wb * 32 + (lane & 31);
      fb[i] = lds0 + r * 128 + ((h ^ swz<false>(r)) << 4);
    }
  }

  // The ring holds five operand slabs in the order A0 B0 A1 B1 ..: while slab kt is multiplied, A and B of kt + 1 and A of kt + 2
  // are on their way (weights come from farther than rows).
  int slab = 0, now = 0;  // unit of slab `now`'s A
  auto unit_of = [&](int ahead) { return slab + ahead >= C::RING ? slab + ahead - C::RING : slab + ahead; };
  if constexpr (C::W4) {
    fetch_codes(0);
    fetch_scales(0);
    in_order();
  }
  look_up(0);
  look_up(1);
  if constexpr (!C::A_ACROSS) cut_tail(oa, 0, std::true_type{});
  if constexpr (!C::B_ACROSS) cut_tail(ob, 0, std::false_type{});
  in_order();
  if constexpr (!C::W4) {
#pragma unroll
    for (int n = 0; n < C::NL; ++n) load_a(0, 0, n);
  }
#pragma unroll
  for (int n = 0; n < C::NL; ++n) load_b(0, 1, n);
  in_order();
  look_up(2);
  if constexpr (!C::A_ACROSS) cut_tail(oa, 1, std::true_type{});
  in_order();
  if constexpr (C::W4) {
    fetched();
    fetch_codes(1);
    fetch_scales(1);
    in_order();
#pragma unroll
    for (int n = 0; n < C::NL; ++n) stage(0, n, std::integral_constant<int, 0>{});
    wait_lds();
  } else {
#pragma unroll
    for (int n = 0; n < C::NL; ++n) load_a(1, 2, n);
    in_order();
  }
  auto step = [&](int kt) -> Slab {
    wait_mem<C::W4 ? C::RW : C::NL>();  // all but A of slab kt + 1
    __builtin_amdgcn_s_barrier();
    if (kt) slab = unit_of(2);
    now = kt;
    if constexpr (!C::A_ACROSS) cut_tail(oa, kt + 2, std::true_type{});
    if constexpr (!C::B_ACROSS) cut_tail(ob, kt + 1, std::false_type{});
    return {(uint32_t)(slab * C::UNIT), (uint32_t)(unit_of(1) * C::UNIT)};
  };
  auto load = [&](int q, auto odd_tag) {  // B of the next slab, then A of the one behind it (W4: A of the next slab into LDS, and codes two to four slabs ahead)
    if constexpr (C::W4) {
      constexpr int odd = decltype(odd_tag)::value;
      static_assert(C::NL == 2 * C::RW, "a piece for each of the second half of the instructions");
      if (q < C::NL) {
        load_b(now + 1, unit_of(3), q);
        if (q == C::NL - 1) in_order();
      } else {
        stage(unit_of(2), q - C::NL, std::integral_constant<int, 1 - odd>{});
        if (q == 2 * C::NL - 1) {
          in_order();
          if constexpr (odd == 0) {
            fetched();
            fetch_codes(now / 2 + 2);
          } else {
            fetch_scales(now / 2 + 2);
          }
          in_order();
        }
      }
    } else if (q < C::NL) {
      load_b(now + 1, unit_of(3), q);
    } else {
      if (q == C::NL) {
        in_order();
        look_up(now + 3);
        in_order();
      }
      load_a(now + 2, unit_of(4), q - C::NL);
    }
  };
  // Results pass through LDS so that whole lines are stored: a lane has 16 neighbours of one row, and stored as they lie every 16 bytes of a wave
  // are a request of their own (weight gradient of 128 slots of 1536 x 640 in fp32, 125 rows each on average: 198 us instead of 128; a batch
  // of 8192 x 6 rows through the FFN's backward: 2622 instead of 2482).  A wave uses its own part of what was the ring, one row fragment at a time.
  const size_t first_row = C::WAY == kWgrad ? (size_t)unit * N : (size_t)ch.first;
  int el = lane;
  auto put = [&](int at, u32x4 v) { *(u32x4*)(s_lds + wave * C::OUT_WAVE + (el & 31) * C::OUT_PITCH + at) = v; };  // at: bytes into the row
  auto store = [&](int f, void* out, size_t row_len, auto add_tag) {  // rows of fragment f; row_len in elements
    constexpr bool add = decltype(add_tag)::value;
    constexpr int lanes = C::OUT_ROW / 16, rows = 64 / lanes;
    // Lanes read what others wrote.  A wave's LDS accesses happen in order, so all it takes is that the compiler keeps theirs: it must not know
    // that a lane reads elsewhere than it wrote.  (A full barrier for the compiler also holds back the loads of da: 690 -> 707 us for one adapter.)
    int reader = el;
    asm volatile("" : "+v"(reader));
#pragma unroll 8
    for (int t = 0; t < 32 / rows; ++t) {
      const int r = t * rows + reader / lanes, piece = reader % lanes, b = b0 + 32 * (wb + 2 * f) + r;
      const int o = a0 + C::feature_row(wa, 0) + piece * (16 / C::OUT_EL);
      u32x4 v = *(const u32x4*)(s_lds + wave * C::OUT_WAVE + r * C::OUT_PITCH + piece * 16);
      if (b >= nb || o >= na) continue;
      unsigned char* p = (unsigned char*)out + ((first_row + b) * row_len + o) * C::OUT_EL;
      if constexpr (add) v = __builtin_bit_cast(u32x4, __builtin_bit_cast(f32x4, v) + *(const f32x4*)p);
      *(u32x4*)p = v;
    }
  };
  auto body = [&](auto nbf_tag) {  // with this many live row fragments
    constexpr int NBF = decltype(nbf_tag)::value;
    f32x16 acc[C::MA][NBF] = {};
    multiply<C, NBF>(nk, fa, fb, acc, step, load);
    wait_mem<0>();  // (of slabs that do not exist: nothing may reach LDS once the ring is used otherwise)
    __builtin_amdgcn_s_barrier();
    // sums e = 0 .. 15 of a fragment are features 16 h + e
    asm volatile("" : "+v"(el));  // addresses of results are not made ahead of the loop, where there is no room for them
    const int eh = el >> 5;
#pragma unroll
    for (int f = 0; f < NBF; ++f) {
      __builtin_amdgcn_sched_barrier(0);  // one fragment's addresses at a time: all of them at once do not fit beside the sums
      if constexpr (C::EP == kEpBack) {
        const int b = b0 + 32 * (wb + 2 * f) + (el & 31);
        u32x4 vg[C::MA / 2][2], vu[C::MA / 2][2];
#pragma unroll
        for (int i = 0; i < C::MA / 2; ++i)
#pragma unroll
          for (int p = 0; p < 2; ++p) {
            const int o = a0 + C::feature_row(wa, i) + 16 * eh + 8 * p;
            f32x4 d[2] = {};
            if (b < nb && o < na) {
              const f32x4* dp = (const f32x4*)(a.da + (first_row + b) * N + o);
              d[0] = dp[0]; d[1] = dp[1];
            }
            const f32x16 &g = acc[i][f], &u = acc[C::MA / 2 + i][f];
            u32x4 va;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              const SwigluBack x = swiglu_back<false>(g[8 * p + 2 * q], u[8 * p + 2 * q], d[q >> 1][2 * (q & 1)]);
              const SwigluBack y = swiglu_back<false>(g[8 * p + 2 * q + 1], u[8 * p + 2 * q + 1], d[q >> 1][2 * (q & 1) + 1]);
              va[q] = bf16_pair(x.a, y.a); vg[i][p][q] = bf16_pair(x.dg, y.dg); vu[i][p][q] = bf16_pair(x.du, y.du);
            }
            put(i * 64 + eh * 32 + p * 16, va);
          }
        auto put_all = [&](const u32x4 (&v)[C::MA / 2][2]) {
#pragma unroll
          for (int i = 0; i < C::MA / 2; ++i)
#pragma unroll
            for (int p = 0; p < 2; ++p) put(i * 64 + eh * 32 + p * 16, v[i][p]);
        };
        store(f, a.out, N, std::false_type{});
        put_all(vg);
        store(f, a.dh, 2 * (size_t)N, std::false_type{});
        put_all(vu);
        store(f, (uint16_t*)a.dh + N, 2 * (size_t)N, std::false_type{});
      } else if constexpr (C::EP == kEpSwiglu) {
#pragma unroll
        for (int i = 0; i < C::MA / 2; ++i)
#pragma unroll
          for (int p = 0; p < 2; ++p) {
            const f32x16 &g = acc[i][f], &u = acc[C::MA / 2 + i][f];
            u32x4 v;
#pragma unroll
            for (int q = 0; q < 4; ++q)
              v[q] = bf16_pair(swiglu(g[8 * p + 2 * q], u[8 * p + 2 * q]), swiglu(g[8 * p + 2 * q + 1], u[8 * p + 2 * q + 1]));
            put(i * 64 + eh * 32 + p * 16, v);
          }
        store(f, a.out, N, std::false_type{});
      } else if constexpr (C::EP == kEpF32) {
#pragma unroll
        for (int i = 0; i < C::MA; ++i)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const f32x16& e = acc[i][f];
            const f32x4 v = {e[4 * q], e[4 * q + 1], e[4 * q + 2], e[4 * q + 3]};
            put(i * 128 + eh * 64 + q * 16, __builtin_bit_cast(u32x4, v));
          }
        if (C::WAY == kWgrad && a.accumulate) store(f, a.out, K, std::true_type{});
        else store(f, a.out, C::WAY == kWgrad ? K : N, std::false_type{});
      } else {
#pragma unroll
        for (int i = 0; i < C::MA; ++i)
#pragma unroll
          for (int p = 0; p < 2; ++p) {
            u32x4 v;
#pragma unroll
            for (int q = 0; q < 4; ++q) v[q] = bf16_pair(acc[i][f][8 * p + 2 * q], acc[i][f][8 * p + 2 * q + 1]);
            put(i * 64 + eh * 32 + p * 16, v);
          }
        store(f, a.out, C::WAY == kWgrad ? K : N, std::false_type{});
      }
    }
  };
  const int frags = (live_b + 31) / 32 - wb;           // live row fragments of both waves of a pair: this one has every other
  const int mine = __builtin_amdgcn_readfirstlane(frags <= 0 ? 0 : (frags + 1) / 2);
  if (mine == 0) {
    idle<C>(nk, step, load);
    wait_mem<0>();
    __builtin_amdgcn_s_barrier();
  } else if (mine == 1) {
    body(std::integral_constant<int, 1>{});
  } else if (C::MB < 3 || mine == 2) {
    body(std::integral_constant<int, 2>{});
  } else if constexpr (C::MB > 2) {
    if (mine == 3) body(std::integral_constant<int, 3>{});
    else body(std::integral_constant<int, 4>{});
  }
}

template <int WAY, int TA, int TB, int EP, bool MAPPED, bool W4 = false>
int launch_cfg(const GemmArgs& a, hipStream_t st) {
  using C = Cfg<WAY, TA, TB, EP, MAPPED, W4>;
  long long units;
  int tiles_a;
  if (WAY == kWgrad) {
    tiles_a = ceil_div(a.K, TA);
    units = (long long)tiles_a * ceil_div(a.N, TB) * a.num_slots;
  } else {
    tiles_a = ceil_div(a.N, C::GATED ? TA / 2 : TA);
    units = max_chunks(a.g.rows, a.g.P, TB) * tiles_a;
  }
  if (const int rc = check_grid(units + 7, C::THREADS)) return rc;
  if (units == 0) return EW_OK;
  const uint32_t by_k = a.g.k > 1 ? (uint32_t)(((1ull << 32) + a.g.k - 1) / a.g.k) : 0u;  // n / k = n * by_k >> 32 for n * k < 2^32 (tile_takes)
  hipLaunchKernelGGL((k_tile<C>), dim3((unsigned)((units + 7) / 8 * 8)), dim3(C::THREADS), 0, st, a, tiles_a, (int)units, by_k);
  EW_LAUNCH_CHECK("k_tile");
  return EW_OK;
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

// The larger tile where a slot has many rows on average (the weight gradient: wherever the outputs fill it).  Both sides, us, 64 slots of 2048 x
// 1408 with so many rows, small / large tile: bf16, first product: 48 154 / 154, 96 171 / 166, 192 237 / 188; 4 bits, both products: 64 146 / 165,
// 128 188 / 203, 192 297 / 240.  The average is over all slots, those without rows too: 64 slots of 188 rows each get the small tile in a pool of 384 (bf16
// 246 instead of 190, 4 bits 318 instead of 241).
// Weight gradient in fp32 (bf16), 64 slots, small / large, at 32, 125 and 768 rows a slot: 512 x 512 16 / 15, 18 / 17, 40 / 39; 640 x 640 23 / 25, 26 / 30,
// 62 / 66 (17 / 22, 19 / 26, 50 / 63); 1024 x 512 26 / 28, 29 / 31, 83 / 68; 1536 x 640 51 / 48, 60 / 59, 155 / 138 (30 / 34, 34 / 39, 131 / 120); 2048 x 1408
// 141 / 131, 186 / 171, 439 / 350: between 512 x 512 and 1024 x 640 few rows would rather have the small one.
template <int WAY, int EP, bool MAPPED, bool W4>
int launch_sized(const GemmArgs& a, hipStream_t st) {
  const long long used = a.g.P < a.g.rows ? a.g.P : a.g.rows;
  const bool large = WAY == kWgrad ? (long long)a.K * a.N > 512 * 512 : a.g.rows > (W4 ? 128 : 64) * used && a.N > 128;
  return large ? launch_cfg<WAY, 256, 256, EP, MAPPED, W4>(a, st) : launch_cfg<WAY, 128, 128, EP, MAPPED, W4>(a, st);
}
template <int WAY, int EP, bool W4 = false>
int launch_mapped(const GemmArgs& a, hipStream_t st) {
  return a.g.por || a.g.k > 1 ? launch_sized<WAY, EP, true, W4>(a, st) : launch_sized<WAY, EP, false, W4>(a, st);
}

}  // namespace

bool tile_takes(int way, int weights, int epilogue, const GemmArgs& a) {
  const unsigned long long lim = 1ull << 32;
  if (weights == kW4 ? way != kFwd || a.K % 128 || a.N % 16 : weights != kWBf16 || a.K % 8 || a.N % 8) return false;
  if (epilogue == kEpSwiglu && weights != kW4) return false;
  if (epilogue == kEpBack && (weights == kW4 || way != kFwd)) return false;
  const bool mapped = a.g.por != nullptr || a.g.k > 1;
  if (epilogue == kEpF32 && (way == kFwd || (way == kDgrad && mapped))) return false;  // (nobody asks for these)
  if (!aligned16(a.x) || !aligned16(a.w) || !aligned16(a.out)) return false;
  if (epilogue == kEpBack && (!aligned16(a.da) || !aligned16(a.dh))) return false;
  // byte offsets are 32 bits wide: into a slot's weights and the looked-up rows, and into one slot's rows where they are the contraction
  const unsigned long long x_bytes = (unsigned long long)a.x_rows * a.K * 2, row_bytes = (unsigned long long)a.g.rows * (a.N > a.K ? a.N : a.K) * 2;
  if (mapped && x_bytes >= lim - 65536) return false;
  if (way == kWgrad) return row_bytes < lim - (unsigned long long)65536 * 64 && (!mapped || (a.K <= 32000 && (unsigned long long)a.x_rows * a.g.k * a.g.k < lim));
  return (unsigned long long)a.slot_bytes + 64ull * a.N * 2 < lim - 65536 && 256ull * a.K * 2 < lim - 65536;
}

int launch_tile(int way, int weights, int epilogue, const GemmArgs& a, hipStream_t st) {
  if (weights == kW4) return epilogue == kEpSwiglu ? launch_mapped<kFwd, kEpSwiglu, true>(a, st) : launch_mapped<kFwd, kEpBf16, true>(a, st);
  if (way == kDgrad) {
    if (epilogue == kEpF32) return launch_sized<kDgrad, kEpF32, false, false>(a, st);
    return launch_mapped<kDgrad, kEpBf16>(a, st);
  }
  if (way == kWgrad) return epilogue == kEpF32 ? launch_mapped<kWgrad, kEpF32>(a, st) : launch_mapped<kWgrad, kEpBf16>(a, st);
  if (epilogue == kEpBack) return launch_mapped<kFwd, kEpBack>(a, st);
  return launch_mapped<kFwd, kEpBf16>(a, st);
}

}  // namespace ew
