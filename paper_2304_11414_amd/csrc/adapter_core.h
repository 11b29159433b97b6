// Low-rank adapters beside a grouped product: what the matrix kernels add to their accumulators before they store them.
//
//   C[r, n] += sum_j low[r, j] * up[a][i][n, j],   a the adapter of packed row r (none: nothing), i the expert, j < rank
//
// low [rows, 2 rank] 16-bit: each row's factor, scaled already, as two summands (the kernels of few rows read the float32 that they stand
// for), up [n_adapters, n_exp, Nout, rank] 16-bit.  rank is a multiple of 8, so an adapter is rank / 8 pieces of 16 bytes per row of `up`, twice as
// many per row of `low`: what a lane holds of a matrix instruction's operand.  Both summands meet the same pieces of `up`.  A
// wavefront goes through the adapters that its rows have, in ascending order; a row's operand is zero where it has another
// one.  Both operands come straight from memory: it is a step or two per tile where the rows are whole requests, next to the 32 of a
// contraction of 1024.
//
// 0 * infinity would carry an adapter's infinities and NaNs to other requests' rows.  They are looked for in the operand,
// replaced by zeros where there are any, and their columns become infinite in that adapter's own rows.
#pragma once

#include <type_traits>

#include "gemm_core.h"

namespace ppmoe {

template <int DT>
struct NonFinite {   // marks (in bits 15 and 31) the elements of a word whose exponent is all ones
  static constexpr uint32_t kExponent = DT == MOE_F16 ? 0x7c007c00u : 0x7f807f80u, kOne = DT == MOE_F16 ? 0x04000400u : 0x00800080u;
  static __device__ __forceinline__ uint32_t marks(uint32_t w) { return ((w & kExponent) + kOne) & 0x80008000u; }
  static __device__ __forceinline__ uint32_t cleared(uint32_t w) { return w & ~((marks(w) >> 15) * 0xffffu); }
};

// An operand (of a bf16 product, whatever the other types) of the largest numbers, or of zeros: a product of two such is infinite
// where both have the numbers, and nothing elsewhere.
__device__ __forceinline__ bf16x8 overflowing(bool is) {
  const uint32_t w = is ? 0x7f7f7f7fu : 0u;
  return __builtin_bit_cast(bf16x8, u32x4{w, w, w, w});
}

constexpr int kNone = 0x7fffffff;   // after the last adapter

// fp16: a row's `low` is its factor divided by a power of two, so that it is within the type's range and its small values keep their bits;
// the row's accumulators are divided by it before the low-rank part is added and multiplied by it afterwards (add_low_rank32; the persistent
// kernel, whose accumulators take all registers, adds such rows in its epilogue, in float32 as the kernels of few rows do).  Rows whose largest
// factor is at least 2^-4 and below 2^15 have the power 0 (the second summand is then off by 2^-21 of that factor at most), others are
// brought to 2^13.
// A word of of_row: -1, or the adapter with the power in bits 16 to 23.  (bf16 has float32's range: the power is 0.)
constexpr int kMostPower = 64, kLeastPower = -32;   // (factors up to 2^77; below 2^-19 steps of 2^-56 are finer than any result's)
__device__ __forceinline__ int row_word(int adapter, int power) { return adapter < 0 ? -1 : adapter | (power & 0xff) << 16; }
__device__ __forceinline__ int adapter_of(int word) { return word < 0 ? -1 : word & 0xffff; }
__device__ __forceinline__ int power_of(int word) { return word < 0 ? 0 : static_cast<int>(static_cast<uint32_t>(word) << 8) >> 24; }
__device__ __forceinline__ bool has_adapter(int word, int adapter) { return (word & static_cast<int>(0x8000ffffu)) == adapter; }
__device__ __forceinline__ float two_to(int power) { return __uint_as_float(static_cast<uint32_t>(127 + power) << 23); }
// top: the bits of the row's largest finite factor
__device__ __forceinline__ int power_for(uint32_t top) {
  const int e = static_cast<int>(top >> 23) - 127;
  return top == 0 || (e >= -4 && e < 15) ? 0 : min(max(e - 13, kLeastPower), kMostPower);
}

// The least adapter above a among this lane's rows and those of the 15 lanes beside it.
template <int MI>
__device__ __forceinline__ int least_above(const int (&mine)[MI], int a) {
  int least = kNone;
#pragma unroll
  for (int mi = 0; mi < MI; ++mi) least = mine[mi] > a && mine[mi] < least ? mine[mi] : least;
  least = min(least, __builtin_amdgcn_update_dpp(0, least, 0x128, 0xf, 0xf, true));   // row_ror:8, 4, 2, 1
  least = min(least, __builtin_amdgcn_update_dpp(0, least, 0x124, 0xf, 0xf, true));
  least = min(least, __builtin_amdgcn_update_dpp(0, least, 0x122, 0xf, 0xf, true));
  return min(least, __builtin_amdgcn_update_dpp(0, least, 0x121, 0xf, 0xf, true));
}

// The kernels of few rows: four columns from `col` on of packed row `row`, which has adapter a >= 0.  In float32 from the float32
// factor: the products are not the matrix instruction's.
template <int DT>
__device__ __forceinline__ f32x4 low_rank_of_four(const AdapterRows& ad, int row, int a, int expert, int col, int Nout) {
  const f32x4* wide = reinterpret_cast<const f32x4*>(ad.wide + static_cast<int64_t>(row) * ad.rank);
  const u32x4* up = reinterpret_cast<const u32x4*>(ad.up + ((static_cast<int64_t>(a) * ad.n_exp + expert) * Nout + col) * ad.rank);
  const int pieces = ad.rank >> 3;
  f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma clang loop unroll(disable)
  for (int p = 0; p < pieces; ++p) {
    const f32x4 w[2] = {wide[2 * p], wide[2 * p + 1]};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const u32x4 u = up[i * pieces + p];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        float u0, u1;
        Elem16<DT>::widen2(u[q], u0, u1);
        sum[i] = fmaf(w[q >> 1][(q & 1) * 2 + 1], u1, fmaf(w[q >> 1][(q & 1) * 2], u0, sum[i]));
      }
    }
  }
  return ad.scale != nullptr ? sum * ad.scale[a] : sum;
}

// The kernels of 32x32x16 instructions: a k-step has two pieces, which may be two adapters' (rank 8).  acc[mi][ni] += the block of
// rows row0 + 32 mi .. and columns col0 + 32 ni .. of this wavefront; rows from `nrow` on are not looked at, columns past the
// last one read the last one (neither is stored).  Accumulator layout: row lane % 32, columns by register.
template <int DT, int MI, int NI>
__device__ __forceinline__ void add_low_rank32(f32x16 (&acc)[MI][NI], const AdapterRows& ad, int expert, int row0, int nrow, int col0, int Nout) {
  typedef typename Elem16<DT>::vec8 vec8;
  constexpr int R = 32, kSlots = 2;
  const u32x4 zero = u32x4{0u, 0u, 0u, 0u};
  const int lane = threadIdx.x & 63;
  const int fr = lane & (R - 1), fq = lane / R;
  int mine[MI], power[MI], any_power = 0;
#pragma unroll
  for (int mi = 0; mi < MI; ++mi) {
    const int r = mi * R + fr;
    const int word = r < nrow ? ad.of_row[row0 + r] : -1;
    mine[mi] = adapter_of(word);
    power[mi] = power_of(word);
    any_power |= power[mi];
  }
  const bool scaled = DT == MOE_F16 && __ballot(any_power != 0) != 0;
  auto times = [&](int sign) __attribute__((always_inline)) {
    if (!scaled) return;
#pragma unroll
    for (int mi = 0; mi < MI; ++mi)
#pragma unroll
      for (int ni = 0; ni < NI; ++ni) acc[mi][ni] *= two_to(sign * power[mi]);
  };
  auto next_after = [&](int a) __attribute__((always_inline)) -> int {
    return __builtin_amdgcn_readfirstlane(min(least_above(mine, a), __shfl_xor(least_above(mine, a), 16, 64)));
  };
  const int pieces = ad.rank >> 3;
  int at = next_after(-1), piece = 0;
  times(-1);
#pragma clang loop unroll(disable)
  while (at != kNone) {
    int my_a = -1, my_p = 0;   // of this lane's slot
#pragma unroll
    for (int s = 0; s < kSlots; ++s) {
      if (at == kNone) break;
      if (fq == s) {
        my_a = at;
        my_p = piece;
      }
      if (++piece == pieces) {
        piece = 0;
        at = next_after(at);
      }
    }
    u32x4 up[NI], low[2][MI];
    const bf16_t* base = ad.up + (static_cast<int64_t>(max(my_a, 0)) * ad.n_exp + expert) * Nout * ad.rank + my_p * 8;
#pragma unroll
    for (int ni = 0; ni < NI; ++ni)
      up[ni] = my_a >= 0 ? *reinterpret_cast<const u32x4*>(base + static_cast<int64_t>(min(col0 + ni * R + fr, Nout - 1)) * ad.rank) : zero;
#pragma unroll
    for (int part = 0; part < 2; ++part)
#pragma unroll
      for (int mi = 0; mi < MI; ++mi)
        low[part][mi] =
            my_a >= 0 && mine[mi] == my_a
                ? *reinterpret_cast<const u32x4*>(ad.low + (static_cast<int64_t>(row0 + mi * R + fr) * 2 + part) * ad.rank + my_p * 8)
                : zero;
    uint32_t marks = 0;
#pragma unroll
    for (int ni = 0; ni < NI; ++ni)
#pragma unroll
      for (int q = 0; q < 4; ++q) marks |= NonFinite<DT>::marks(up[ni][q]);
    uint64_t bad[NI] = {};   // by column block: the lanes (slot and column) with such an element
    const bool any = __ballot(marks != 0) != 0;
    if (any) {
#pragma unroll
      for (int ni = 0; ni < NI; ++ni) {
        uint32_t m = 0;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          m |= NonFinite<DT>::marks(up[ni][q]);
          up[ni][q] = NonFinite<DT>::cleared(up[ni][q]);
        }
        bad[ni] = __ballot(m != 0);
      }
    }
#pragma unroll
    for (int mi = 0; mi < MI; ++mi)
#pragma unroll
      for (int ni = 0; ni < NI; ++ni) {
        const vec8 u = __builtin_bit_cast(vec8, up[ni]);
        acc[mi][ni] = Elem16<DT>::mfma32(u, __builtin_bit_cast(vec8, low[0][mi]), acc[mi][ni]);
        acc[mi][ni] = Elem16<DT>::mfma32(u, __builtin_bit_cast(vec8, low[1][mi]), acc[mi][ni]);
      }
    if (any) {
#pragma unroll
      for (int ni = 0; ni < NI; ++ni) {
        if (bad[ni] == 0) continue;
        const bf16x8 u = overflowing((bad[ni] >> lane) & 1);
#pragma unroll
        for (int mi = 0; mi < MI; ++mi)
          acc[mi][ni] = Elem16<MOE_BF16>::mfma32(u, overflowing(my_a >= 0 && mine[mi] == my_a), acc[mi][ni]);
      }
    }
  }
  times(1);
}

// Names accumulators as accumulator registers at this point of the program (left to itself the
// register allocator moves some of them to vector registers and spills).
template <int MI, int NI, typename ACC>
__device__ __forceinline__ void hold(ACC& acc) {
#pragma unroll
  for (int mi = 0; mi < MI; ++mi)
#pragma unroll
    for (int ni = 0; ni < NI; ++ni) asm volatile("" : "+a"(acc[mi][ni]));
}

// The persistent kernel's wavefront: 8 x NI blocks of 16x16x32 instructions, mine[mi] the adapter of row 16 mi + lane % 16 (-1: none,
// or not a row of the tile), row0 and col0 its first row and column.  A step is up to 32 of one adapter's rank, with both summands
// (up to rank 16 in one operand); blocks of 16 rows of which none has the adapter are passed over (8192 rows of 24 requests over 8
// experts: four adapters per wavefront, each in a third of its rows), so a step is little work and what it costs is the latency of
// its operands.
template <int DT, int NI>
__device__ __forceinline__ void add_low_rank16(f32x4 (&acc)[8][NI], const AdapterRows& ad, const int (&mine)[8], int expert, int row0,
                                               int col0, int Nout) {
  typedef typename Elem16<DT>::vec8 vec8;
  constexpr int MI = 8;
  int at = __builtin_amdgcn_readfirstlane(least_above(mine, -1)), piece0 = 0;
  const int ncol = Nout - col0;
  if (at == kNone || ncol <= 0) return;
  int lane = threadIdx.x & 63;
  asm volatile("" : "+v"(lane));   // (what follows is computed here, not kept across the K loop)
  const int fr = lane & 15, fq = lane >> 4;
  const int pieces = ad.rank >> 3, row_bytes = ad.rank * 2;   // of up; twice as many of low
  constexpr uint32_t kOutside = 0x80000000u;   // no descriptor covers it: the lane gets zeros
  const __amdgpu_buffer_rsrc_t low_rsrc = __builtin_amdgcn_make_buffer_rsrc(
      const_cast<bf16_t*>(ad.low + static_cast<int64_t>(row0) * 2 * ad.rank), 0, 0x7fffffff, 0x00020000);
  // Half of the columns at a time: while one half's operand is multiplied the other half's, or the next step's, is on its
  // way, and a row block's takes the next step's place as soon as both halves have used it (96 registers; the next step's in flight as well
  // spill, and cost more than they hide).  The second summands as steps of their own, with 64 registers, cost 20 us more where 8192 rows of 24
  // requests, rank 32, 2048 to 8192 take 313; the first summands alone 10 less.
  constexpr int H = NI / 2;
  const bool split = pieces > 2;
  u32x4 up[2][H], low[2][MI];
  auto fetch_up = [&](u32x4 (&u)[H], int first) __attribute__((always_inline)) {
    const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<bf16_t*>(ad.up + ((static_cast<int64_t>(at) * ad.n_exp + expert) * Nout + col0) * ad.rank), 0, 0x7fffffff, 0x00020000);
    const int p = split || fq < pieces ? piece0 + fq : fq - pieces;
#pragma unroll
    for (int ni = 0; ni < H; ++ni) {
      const uint32_t off = min((first + ni) * 16 + fr, ncol - 1) * row_bytes + p * 16;
      u[ni] = __builtin_amdgcn_raw_buffer_load_b128(rsrc, p < pieces ? off : kOutside, 0, 0);
    }
  };
  auto fetch_low = [&](int mi) __attribute__((always_inline)) {
    const bool is = mine[mi] == at;
    if (__ballot(is) != 0) {
      const uint32_t off = is && piece0 + fq < (split ? pieces : 2 * pieces) ? (mi * 16 + fr) * 2 * row_bytes + fq * 16 : kOutside;
      low[0][mi] = __builtin_amdgcn_raw_buffer_load_b128(low_rsrc, off, piece0 * 16, 0);
      if (split) low[1][mi] = __builtin_amdgcn_raw_buffer_load_b128(low_rsrc, off, (pieces + piece0) * 16, 0);
    }
  };
  auto clean = [&](u32x4 (&u)[H], auto first_c, int now) __attribute__((always_inline)) {
    constexpr int first = decltype(first_c)::value;
    uint32_t marks = 0;
#pragma unroll
    for (int ni = 0; ni < H; ++ni)
#pragma unroll
      for (int q = 0; q < 4; ++q) marks |= NonFinite<DT>::marks(u[ni][q]);
    if (__builtin_expect(__ballot(marks != 0) == 0, 1)) return;
#pragma unroll
    for (int ni = 0; ni < H; ++ni) {
      uint32_t m = 0;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        m |= NonFinite<DT>::marks(u[ni][q]);
        u[ni][q] = NonFinite<DT>::cleared(u[ni][q]);
      }
      if (__ballot(m != 0) != 0) {
        const bf16x8 column = overflowing(m != 0);
#pragma unroll
        for (int mi = 0; mi < MI; ++mi)
          acc[mi][first + ni] = Elem16<MOE_BF16>::mfma16(column, overflowing(mine[mi] == now), acc[mi][first + ni]);
      }
    }
    hold<MI, NI>(acc);
  };
  auto multiply = [&](u32x4 (&u)[H], auto first_c, int now, bool more) __attribute__((always_inline)) {
    constexpr int first = decltype(first_c)::value;
    clean(u, first_c, now);
#pragma unroll
    for (int mi = 0; mi < MI; ++mi) {
      if (__ballot(mine[mi] == now) != 0) {
#pragma unroll
        for (int ni = 0; ni < H; ++ni)
          acc[mi][first + ni] = Elem16<DT>::mfma16(__builtin_bit_cast(vec8, u[ni]), __builtin_bit_cast(vec8, low[0][mi]), acc[mi][first + ni]);
        if (split) {
#pragma unroll
          for (int ni = 0; ni < H; ++ni)
            acc[mi][first + ni] = Elem16<DT>::mfma16(__builtin_bit_cast(vec8, u[ni]), __builtin_bit_cast(vec8, low[1][mi]), acc[mi][first + ni]);
        }
      }
      if (first > 0 && more) fetch_low(mi);
    }
    hold<MI, NI>(acc);
  };
  fetch_up(up[0], 0);
#pragma unroll
  for (int mi = 0; mi < MI; ++mi) fetch_low(mi);
#pragma clang loop unroll(disable)
  while (true) {
    fetch_up(up[1], H);
    const int now = at;
    multiply(up[0], std::integral_constant<int, 0>{}, now, false);
    piece0 += 4;
    if (piece0 >= pieces) {
      piece0 = 0;
      at = __builtin_amdgcn_readfirstlane(least_above(mine, at));
    }
    const bool more = at != kNone;
    if (more) fetch_up(up[0], 0);
    multiply(up[1], std::integral_constant<int, H>{}, now, more);
    if (!more) break;
  }
}

}  // namespace ppmoe
