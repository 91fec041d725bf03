// Matrix products grouped by expert on the bf16 matrix cores, many rows per slot: forward, input gradient, weight gradient.
//
// A workgroup makes one tile of TA outputs along the contiguous axis of the result ("features", operand A) times up to TB along the
// other ("rows", operand B) with v_mfma_f32_32x32x16_bf16, eight waves (four at the smaller tile) of 64 features x half of the rows.
// The contraction comes in slabs of 64 through two LDS buffers, filled by LDS-direct loads while the slab before is multiplied.
//
// An operand lies in memory along the contraction (x, and w of the forward product) or across it (w of the input gradient, both
// operands of the weight gradient).  The first kind is staged as [rows][64] and read 16 bytes a lane; the second as [64][outputs] and read by
// ds_read_b64_tr_b16, which transposes 4 x 16 elements over 16 lanes on the way: no transposed copy is made in memory.  Both kinds of
// LDS rows are XOR-swizzled so that the reads of a wave cover all banks.
// MFMA row m = 8 a + 4 h + b of a feature fragment is feature 16 h + 4 a + b: a lane's 16 sums are neighbours, stored 16 bytes at a time.
//
// Loads go through buffer descriptors: rows and contraction steps past the end read as zeros (a slot's sums never see what lies behind
// it, NaN or not), and no index, however wrong, reaches memory outside the tensors.
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
__device__ __forceinline__ void wait_mem() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

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

template <int WAY_, int TA_, int TB_, int EP_>
struct Cfg {
  static constexpr int WAY = WAY_, TA = TA_, TB = TB_, EP = EP_;
  static constexpr bool A_ACROSS = WAY != kFwd, B_ACROSS = WAY == kWgrad;
  static constexpr bool GATED = EP == kEpSwiglu;
  static constexpr int WAVES_A = TA / 64, WAVES = 2 * WAVES_A, THREADS = 64 * WAVES;
  static constexpr int MAXB = TB / 64;                               // row fragments of a wave: fragment f of wave half b is rows 32 (b + 2 f) ..
  static constexpr int A_BYTES = TA * kSlab * 2, B_BYTES = TB * kSlab * 2, STAGE = A_BYTES + B_BYTES, LDS = 2 * STAGE;
  static constexpr int NA = A_BYTES / 1024 / WAVES, NB = B_BYTES / 1024 / WAVES;   // load instructions of a wave and slab
  static constexpr int AR = TA * 2, BR = TB * 2;                     // bytes of an LDS row across the contraction
  static constexpr int A_FRAG = GATED ? TA / 2 : 32;                 // features between a wave's two feature fragments
};

__device__ __forceinline__ float bf16_up(uint32_t bits16) { return __uint_as_float(bits16 << 16); }
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

template <typename C>
struct Tile {
  // a wave's part of staging and reading; everything here is per lane unless it says uniform
  Rsrc ra, rb;                                  // uniform
  uint32_t oa[C::NA], ob[C::NB];                // byte offsets of the load instructions
  uint32_t sa, sb;                              // uniform: bytes a slab further
  uint32_t fa[2], fb[2];                        // LDS addresses of the feature fragments, of row fragments 0 and 1
};

// The K loop of a wave with NBF live row fragments.  step(kt): meets the others, starts the loads of slab kt + 1, returns the LDS
// offset of slab kt's buffer.
template <typename C, int NBF, typename Step>
__device__ __forceinline__ void multiply(int nk, const uint32_t (&fa)[2], const uint32_t (&fb)[2], f32x16 (&acc)[2][C::MAXB], Step step) {
  Frag<C::A_ACROSS> a[2][2];
  Frag<C::B_ACROSS> b[2][NBF];
  uint32_t buf = 0;
  auto read = [&](auto c_tag, auto ks_tag) {
    constexpr int c = decltype(c_tag)::value, ks = decltype(ks_tag)::value;
    if constexpr (C::A_ACROSS) {
#pragma unroll
      for (int i = 0; i < 2; ++i) a[c][i].template read<ks * 16 * C::AR, C::AR>(buf + fa[i]);
    } else {
#pragma unroll
      for (int i = 0; i < 2; ++i) a[c][i].template read<0>((buf + fa[i]) ^ (uint32_t)(32 * ks));
    }
    auto read_b = [&](auto f_tag) {
      constexpr int f = decltype(f_tag)::value;
      if constexpr (f < NBF) {
        if constexpr (C::B_ACROSS) b[c][f].template read<ks * 16 * C::BR + (f >> 1) * 256, C::BR>(buf + fb[f & 1]);
        else b[c][f].template read<f * 64 * 128>((buf + fb[0]) ^ (uint32_t)(32 * ks));
      }
    };
    read_b(std::integral_constant<int, 0>{});
    read_b(std::integral_constant<int, 1>{});
    read_b(std::integral_constant<int, 2>{});
    read_b(std::integral_constant<int, 3>{});
  };
  auto landed = [&](auto c_tag) {
    constexpr int c = decltype(c_tag)::value;
    wait_lds();
    a[c][0].landed();
    a[c][1].landed();
#pragma unroll
    for (int f = 0; f < NBF; ++f) b[c][f].landed();
  };
  auto mul = [&](auto c_tag) {
    constexpr int c = decltype(c_tag)::value;
#pragma unroll
    for (int f = 0; f < NBF; ++f)
#pragma unroll
      for (int i = 0; i < 2; ++i) acc[i][f] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[c][i].get(), b[c][f].get(), acc[i][f], 0, 0, 0);
  };
  const std::integral_constant<int, 0> _0{};
  const std::integral_constant<int, 1> _1{};
  const std::integral_constant<int, 2> _2{};
  const std::integral_constant<int, 3> _3{};
  // reads run a k-step ahead of the products, across slabs too
  for (int kt = 0; kt < nk; ++kt) {
    buf = step(kt);
    read(_0, _0);
    if (kt) mul(_1);
    landed(_0);
    read(_1, _1); mul(_0); landed(_1);
    read(_0, _2); mul(_1); landed(_0);
    read(_1, _3); mul(_0); landed(_1);
  }
  if (nk) mul(_1);
}
template <typename C, typename Step>
__device__ __forceinline__ void idle(int nk, Step step) {  // a wave without rows keeps loading
  for (int kt = 0; kt < nk; ++kt) step(kt);
}

template <typename C>
__global__ __launch_bounds__(C::THREADS) __attribute__((amdgpu_waves_per_eu(2, 2))) void k_tile(GemmArgs a, int tiles_a, int units, int mapped) {
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
  // ---- staging
  Tile<C> t;
  const unsigned char *wp = (const unsigned char*)a.w, *xp = (const unsigned char*)a.x;
  const bool rows_mapped = mapped;  // uniform: rows of x are looked up
  const uint32_t x_bytes = (uint32_t)a.x_rows * (uint32_t)K * 2u;
  if constexpr (C::A_ACROSS) {
    // instruction n of this wave: LDS rows (contraction) first + n * rpi + lane / ppr
    constexpr int PPR = C::TA / 8, RPI = 64 / PPR;  // pieces per row, rows per instruction
    const int pos = lane % PPR;
#pragma unroll
    for (int n = 0; n < C::NA; ++n) {
      const int kr = (wave * C::NA + n) * RPI + lane / PPR, piece = pos ^ (kr & 3) << 2;
      if constexpr (C::WAY == kDgrad) t.oa[n] = ((uint32_t)kr * (uint32_t)N + a0 + piece * 8) * 2;
      else t.oa[n] = ((uint32_t)(rows_mapped ? 0 : kr) * (uint32_t)K + a0 + piece * 8) * 2;
    }
    if constexpr (C::WAY == kDgrad) {
      t.ra = resource(wp + (size_t)ch.slot * a.slot_bytes, (uint32_t)a.slot_bytes);
      t.sa = kSlab * (uint32_t)N * 2;
    } else if (rows_mapped) {
      t.ra = resource(xp, x_bytes);
      t.sa = 0;
    } else {
      t.ra = resource(xp + (size_t)ch.first * K * 2, (uint32_t)len * (uint32_t)K * 2u);
      t.sa = kSlab * (uint32_t)K * 2;
    }
  } else {
#pragma unroll
    for (int n = 0; n < C::NA; ++n) {
      const int r = (wave * C::NA + n) * 8 + (lane >> 3), piece = (lane & 7) ^ swz<true>(r);
      int f = a0 + r;
      if constexpr (C::GATED) f = a0 + (r < C::TA / 2 ? r : r - C::TA / 2 + N);
      const bool there = C::GATED ? a0 + (r < C::TA / 2 ? r : r - C::TA / 2) < N : f < N;
      t.oa[n] = there ? ((uint32_t)f * (uint32_t)K + piece * 8) * 2 : kNowhere;
    }
    t.ra = resource(wp + (size_t)ch.slot * a.slot_bytes, (uint32_t)a.slot_bytes);
    t.sa = kSlab * 2;
  }
  if constexpr (C::B_ACROSS) {
    constexpr int PPR = C::TB / 8, RPI = 64 / PPR;
    const int pos = lane % PPR;
#pragma unroll
    for (int n = 0; n < C::NB; ++n) {
      const int kr = (wave * C::NB + n) * RPI + lane / PPR, piece = pos ^ (kr & 3) << 2;
      t.ob[n] = ((uint32_t)kr * (uint32_t)N + b0 + piece * 8) * 2;
    }
    t.rb = resource(wp + (size_t)ch.first * N * 2, (uint32_t)len * (uint32_t)N * 2u);
    t.sb = kSlab * (uint32_t)N * 2;
  } else {
#pragma unroll
    for (int n = 0; n < C::NB; ++n) {
      const int r = (wave * C::NB + n) * 8 + (lane >> 3), piece = (lane & 7) ^ swz<false>(r);
      const uint32_t src = r < ch.rows ? (rows_mapped ? (uint32_t)source_row(a.g, ch.first + r) : (uint32_t)r) : 0u;
      t.ob[n] = r < ch.rows ? (src * (uint32_t)K + piece * 8) * 2 : kNowhere;
    }
    t.rb = rows_mapped ? resource(xp, x_bytes) : resource(xp + (size_t)ch.first * K * 2, (uint32_t)ch.rows * (uint32_t)K * 2u);
    t.sb = kSlab * 2;
  }
  // rows of the weight gradient's x are looked up a slab ahead of their loads
  uint32_t next_row[C::WAY == kWgrad ? C::NA : 1];
  auto look_up = [&](int kt) {
    if constexpr (C::WAY == kWgrad) {
      constexpr int PPR = C::TA / 8, RPI = 64 / PPR;
#pragma unroll
      for (int n = 0; n < C::NA; ++n) {
        const int r = kt * kSlab + (wave * C::NA + n) * RPI + lane / PPR;
        next_row[n] = r < len ? (uint32_t)(a.g.por ? a.g.por[ch.first + r] : ch.first + r) : 0u;
      }
    }
  };
  auto lds_at = [&](uint32_t off) { return (lds_byte*)s_lds + off; };
  const bool tail = !C::B_ACROSS && K % kSlab;  // the last slab has less than 64 of the contraction (rows across it end by their descriptor)
  auto load = [&](int kt) {
    const uint32_t to = (uint32_t)(kt & 1) * C::STAGE;
    const bool last = tail && kt == nk - 1;
#pragma unroll
    for (int n = 0; n < C::NA; ++n) {
      uint32_t off = t.oa[n];
      if constexpr (C::WAY == kWgrad) {
        if (rows_mapped) {
          constexpr int PPR = C::TA / 8, RPI = 64 / PPR;
          const int r = kt * kSlab + (wave * C::NA + n) * RPI + lane / PPR;
          off = r < len ? off + next_row[n] / (uint32_t)a.g.k * ((uint32_t)K * 2) : kNowhere;
        }
      } else if constexpr (!C::A_ACROSS) {
        if (last && kt * kSlab + (int)(((lane & 7) ^ swz<true>((wave * C::NA + n) * 8 + (lane >> 3))) * 8) >= K) off = kNowhere;
      }
      load_lds(t.ra, lds_at(to + (wave * C::NA + n) * 1024), off, (uint32_t)kt * t.sa);
    }
#pragma unroll
    for (int n = 0; n < C::NB; ++n) {
      uint32_t off = t.ob[n];
      if constexpr (!C::B_ACROSS) {
        if ((wave * C::NB + n) * 8 >= (live_b + 31) / 32 * 32) continue;  // (uniform) a fragment without rows
        if (last && kt * kSlab + (int)(((lane & 7) ^ swz<false>((wave * C::NB + n) * 8 + (lane >> 3))) * 8) >= K) off = kNowhere;
      }
      load_lds(t.rb, lds_at(to + C::A_BYTES + (wave * C::NB + n) * 1024), off, (uint32_t)kt * t.sb);
    }
  };
  // ---- reading
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_byte*)s_lds;
  const int wa = wave >> 1, wb = wave & 1, h = lane >> 5;
  if constexpr (C::A_ACROSS) {
    const int g = lane >> 4, c = lane & 3, kr = (g >> 1) * 8 + (lane & 15) / 4;
    const int feat = 16 * (c & 1) + 8 * (g & 1) + 4 * (c >> 1);
#pragma unroll
    for (int i = 0; i < 2; ++i) t.fa[i] = lds0 + kr * C::AR + (((wa * 2 + i) ^ (kr & 3)) * 64) + feat * 2;
  } else {
    const int m = lane & 31, r = wa * (C::GATED ? 32 : 64) + 16 * (m >> 2 & 1) + 4 * (m >> 3) + (m & 3);
    t.fa[0] = lds0 + r * 128 + ((h ^ swz<true>(r)) << 4);
    t.fa[1] = t.fa[0] + C::A_FRAG * 128;
  }
  if constexpr (C::B_ACROSS) {
    const int g = lane >> 4, c = lane & 3, kr = (g >> 1) * 8 + (lane & 15) / 4;
#pragma unroll
    for (int i = 0; i < 2; ++i) t.fb[i] = lds0 + C::A_BYTES + kr * C::BR + (((wb + 2 * i) ^ (kr & 3)) * 64) + (16 * (g & 1) + 4 * c) * 2;
  } else {
    const int r = wb * 32 + (lane & 31);
    t.fb[0] = t.fb[1] = lds0 + C::A_BYTES + r * 128 + ((h ^ swz<false>(r)) << 4);
  }

  f32x16 acc[2][C::MAXB] = {};
  if (nk) {
    look_up(0);
    load(0);
    if (nk > 1) look_up(1);
  }
  auto step = [&](int kt) -> uint32_t {
    wait_mem();
    __builtin_amdgcn_s_barrier();
    if (kt + 1 < nk) {
      load(kt + 1);
      if (kt + 2 < nk) look_up(kt + 2);
    }
    return (uint32_t)(kt & 1) * C::STAGE;
  };
  const int frags = (live_b + 31) / 32 - wb;           // live row fragments of both waves of a pair: this one has every other
  const int mine = __builtin_amdgcn_readfirstlane(frags <= 0 ? 0 : (frags + 1) / 2);
  if (mine == 0) idle<C>(nk, step);
  else if (mine == 1) multiply<C, 1>(nk, t.fa, t.fb, acc, step);
  else if (C::MAXB < 3 || mine == 2) multiply<C, 2>(nk, t.fa, t.fb, acc, step);
  else if (mine == 3) multiply<C, C::MAXB < 3 ? 2 : 3>(nk, t.fa, t.fb, acc, step);
  else multiply<C, C::MAXB < 3 ? 2 : 4>(nk, t.fa, t.fb, acc, step);

  // ---- results: sums e = 0 .. 15 of a fragment are features 16 h + e
  const size_t row_len = C::WAY == kWgrad ? K : N;
#pragma unroll
  for (int f = 0; f < C::MAXB; ++f) {
    if (f >= mine) continue;
    const int b = b0 + 32 * (wb + 2 * f) + (lane & 31);
    if (b >= nb) continue;
    const size_t row = C::WAY == kWgrad ? (size_t)unit * N + b : (size_t)(ch.first + b);
    if constexpr (C::EP == kEpSwiglu) {
      const int o = a0 + wa * 32 + 16 * h;
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        if (o + 8 * p >= na) continue;
        u32x4 v;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          float r[2];
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            r[j] = swiglu(acc[0][f][8 * p + 2 * q + j], acc[1][f][8 * p + 2 * q + j]);
          }
          v[q] = bf16_pair(r[0], r[1]);
        }
        *(u32x4*)((uint16_t*)a.out + row * row_len + o + 8 * p) = v;
      }
      continue;
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int o = a0 + wa * 64 + i * 32 + 16 * h;
      if constexpr (C::EP == kEpF32) {
        float* p = (float*)a.out + row * row_len + o;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          if (o + 4 * q >= na) continue;
          f32x4 v;
#pragma unroll
          for (int j = 0; j < 4; ++j) v[j] = acc[i][f][4 * q + j];
          if (C::WAY == kWgrad && a.accumulate) v += *(const f32x4*)(p + 4 * q);
          *(f32x4*)(p + 4 * q) = v;
        }
      } else if constexpr (C::EP == kEpBf16) {
#pragma unroll
        for (int p = 0; p < 2; ++p) {
          if (o + 8 * p >= na) continue;
          u32x4 v;
#pragma unroll
          for (int q = 0; q < 4; ++q) v[q] = bf16_pair(acc[i][f][8 * p + 2 * q], acc[i][f][8 * p + 2 * q + 1]);
          *(u32x4*)((uint16_t*)a.out + row * row_len + o + 8 * p) = v;
        }
      } else if constexpr (C::EP == kEpBack) {
#pragma unroll
        for (int p = 0; p < 2; ++p) {
          if (o + 8 * p >= na) continue;
          const float* hp = a.h + row * 2 * N + o + 8 * p;
          u32x4 va, vg, vu;
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            float ra[2], rg[2], ru[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              const SwigluBack v = swiglu_back(hp[2 * q + j], hp[N + 2 * q + j], acc[i][f][8 * p + 2 * q + j]);
              ra[j] = v.a; rg[j] = v.dg; ru[j] = v.du;
            }
            va[q] = bf16_pair(ra[0], ra[1]); vg[q] = bf16_pair(rg[0], rg[1]); vu[q] = bf16_pair(ru[0], ru[1]);
          }
          *(u32x4*)((uint16_t*)a.out + row * N + o + 8 * p) = va;
          *(u32x4*)((uint16_t*)a.dh + row * 2 * N + o + 8 * p) = vg;
          *(u32x4*)((uint16_t*)a.dh + row * 2 * N + N + o + 8 * p) = vu;
        }
      }
    }
  }
}

template <int WAY, int TA, int TB, int EP>
int launch_cfg(const GemmArgs& a, hipStream_t st) {
  using C = Cfg<WAY, TA, TB, EP>;
  long long units;
  int tiles_a;
  if (WAY == kWgrad) {
    tiles_a = ceil_div(a.K, TA);
    units = (long long)tiles_a * ceil_div(a.N, TB) * a.num_slots;
  } else {
    tiles_a = ceil_div(a.N, C::GATED ? TA / 2 : TA);
    units = max_chunks(a.g.rows, a.g.P, TB) * tiles_a;
  }
  if (units >= (1ll << 31) - 8) return fail(EW_ERR_UNSUPPORTED, "grouped product: too many output tiles for one launch");
  if (units == 0) return EW_OK;
  static_assert(C::LDS <= 160 * 1024, "LDS budget of a CU");
  const int mapped = a.g.por != nullptr || a.g.k > 1;
  hipLaunchKernelGGL((k_tile<C>), dim3((unsigned)((units + 7) / 8 * 8)), dim3(C::THREADS), 0, st, a, tiles_a, (int)units, mapped);
  EW_LAUNCH_CHECK("k_tile");
  return EW_OK;
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

// The larger tile where a slot has more than 128 rows on average (the weight gradient: wherever the outputs fill it).
template <int WAY, int EP>
int launch_sized(const GemmArgs& a, hipStream_t st) {
  const long long used = a.g.P < a.g.rows ? a.g.P : a.g.rows;
  const bool large = WAY == kWgrad ? (long long)a.K * a.N > 512 * 512 : a.g.rows > 64 * used && a.N > 128;
  return large ? launch_cfg<WAY, 256, 256, EP>(a, st) : launch_cfg<WAY, 128, 128, EP>(a, st);
}

}  // namespace

bool tile_takes(int way, int weights, int epilogue, const GemmArgs& a) {
  const unsigned long long lim = 1ull << 32;
  if (weights != kWBf16 || a.K % 8 || a.N % 8 || !aligned16(a.x) || !aligned16(a.w) || !aligned16(a.out)) return false;
  if (epilogue == kEpBack && (!aligned16(a.h) || !aligned16(a.dh))) return false;
  const bool mapped = a.g.por != nullptr || a.g.k > 1;
  // byte offsets are 32 bits wide: into a slot's weights and the looked-up rows, and into one slot's rows where they are the contraction
  const unsigned long long x_bytes = (unsigned long long)a.x_rows * a.K * 2, row_bytes = (unsigned long long)a.g.rows * (a.N > a.K ? a.N : a.K) * 2;
  if (mapped && x_bytes >= lim - 65536) return false;
  if (way == kWgrad) return row_bytes < lim - (unsigned long long)65536 * 64;
  return (unsigned long long)a.slot_bytes + 64ull * a.N * 2 < lim - 65536 && 256ull * a.K * 2 < lim - 65536;
}

int launch_tile(int way, int weights, int epilogue, const GemmArgs& a, hipStream_t st) {
  (void)weights;
  if (way == kDgrad) {
    if (epilogue == kEpBack) return launch_sized<kDgrad, kEpBack>(a, st);
    return launch_sized<kDgrad, kEpBf16>(a, st);
  }
  if (way == kWgrad) return epilogue == kEpF32 ? launch_sized<kWgrad, kEpF32>(a, st) : launch_sized<kWgrad, kEpBf16>(a, st);
  if (epilogue == kEpF32) return launch_sized<kFwd, kEpF32>(a, st);
  return launch_sized<kFwd, kEpBf16>(a, st);
}

}  // namespace ew
