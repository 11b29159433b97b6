// Low-rank adapters beside a grouped product: what the matrix kernels add to their accumulators before they store them.
//
//   C[r, n] += sum_j low[r, j] * up[a][i][n, j],   a the adapter of packed row r (none: nothing), i the expert, j < rank
//
// low [rows, rank] 16-bit (scaled already), up [n_adapters, n_exp, Nout, rank] 16-bit.  rank is a multiple of 8, so an adapter is
// rank / 8 pieces of 16 bytes per row of either matrix: what a lane holds of a matrix instruction's operand.  A
// wavefront goes through the adapters that its rows have, in ascending order, and packs their pieces into k-steps one behind the
// other (two adapters of rank 16 share a step of 32): a row's operand is zero at other adapters' pieces.  Both operands
// come straight from memory: it is a step or two per tile where the rows are whole requests, next to the 32 of a contraction of 1024.
//
// 0 * infinity would carry an adapter's infinities and NaNs to other requests' rows.  They are looked for in the operand,
// replaced by zeros where there are any, and the blocks of R columns they are in become NaN in that adapter's own rows.
#pragma once

#include "common.h"

namespace ppmoe {

template <int DT>
struct NonFinite {   // marks (in bits 15 and 31) the elements of a word whose exponent is all ones
  static constexpr uint32_t kExponent = DT == MOE_F16 ? 0x7c007c00u : 0x7f807f80u, kOne = DT == MOE_F16 ? 0x04000400u : 0x00800080u;
  static __device__ __forceinline__ uint32_t marks(uint32_t w) { return ((w & kExponent) + kOne) & 0x80008000u; }
  static __device__ __forceinline__ uint32_t cleared(uint32_t w) { return w & ~((marks(w) >> 15) * 0xffffu); }
};

// Names accumulators as accumulator registers at this point of the program (R = 16: the persistent kernel's 256; left to
// itself the register allocator moves some of them to vector registers and spills).
template <int MI, int NI, typename ACC>
__device__ __forceinline__ void hold(ACC& acc) {
#pragma unroll
  for (int mi = 0; mi < MI; ++mi)
#pragma unroll
    for (int ni = 0; ni < NI; ++ni) asm volatile("" : "+a"(acc[mi][ni]));
}

// R: 16 or 32, rows and columns of a matrix instruction (16x16x32, 32x32x16): a k-step has 64 / R pieces.  acc[mi][ni] += the block of
// rows row0 + mi R .. and columns col0 + ni R .. of this wavefront; rows from `nrow` on are not looked at, columns past the
// last one read the last one (neither is stored).  Accumulator layout: row lane % R, columns by register.
template <int DT, int R, int MI, int NI, typename ACC>
__device__ __forceinline__ void add_low_rank(ACC& acc, const AdapterRows& ad, int expert, int row0, int nrow, int col0, int Nout) {
  typedef typename Elem16<DT>::vec8 vec8;
  constexpr int kSlots = 64 / R;
  constexpr int kNone = 0x7fffffff;
  const u32x4 zero = u32x4{0u, 0u, 0u, 0u};
  int lane = threadIdx.x & 63;
  asm volatile("" : "+v"(lane));   // (what follows is computed here, not kept across the caller's K loop)
  const int fr = lane & (R - 1), fq = lane / R;
  int mine[MI];
#pragma unroll
  for (int mi = 0; mi < MI; ++mi) {
    const int r = mi * R + fr;
    mine[mi] = r < nrow ? ad.of_row[row0 + r] : -1;
  }
  auto next_after = [&](int a) __attribute__((always_inline)) -> int {   // the least adapter above a among the rows
    int least = kNone;
#pragma unroll
    for (int mi = 0; mi < MI; ++mi) least = mine[mi] > a && mine[mi] < least ? mine[mi] : least;
#pragma unroll
    for (int off = R / 2; off >= 1; off >>= 1) least = min(least, __shfl_xor(least, off, 64));
    return __builtin_amdgcn_readfirstlane(least);
  };
  const int pieces = ad.rank >> 3;
  int at = next_after(-1), piece = 0;
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
    u32x4 up[NI], low[MI];
    const bf16_t* base = ad.up + (static_cast<int64_t>(max(my_a, 0)) * ad.n_exp + expert) * Nout * ad.rank + my_p * 8;
#pragma unroll
    for (int ni = 0; ni < NI; ++ni)
      up[ni] = my_a >= 0 ? *reinterpret_cast<const u32x4*>(base + static_cast<int64_t>(min(col0 + ni * R + fr, Nout - 1)) * ad.rank) : zero;
#pragma unroll
    for (int mi = 0; mi < MI; ++mi)
      low[mi] = my_a >= 0 && mine[mi] == my_a
                    ? *reinterpret_cast<const u32x4*>(ad.low + static_cast<int64_t>(row0 + mi * R + fr) * ad.rank + my_p * 8)
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
        const vec8 u = __builtin_bit_cast(vec8, up[ni]), l = __builtin_bit_cast(vec8, low[mi]);
        if constexpr (R == 16) acc[mi][ni] = Elem16<DT>::mfma16(u, l, acc[mi][ni]);
        else acc[mi][ni] = Elem16<DT>::mfma32(u, l, acc[mi][ni]);
      }
    if constexpr (R == 16) hold<MI, NI>(acc);
    if (any) {
      // (as products: accumulators that a branch changed element by element would all pass through vector registers)
#pragma unroll
      for (int ni = 0; ni < NI; ++ni) {
        if (bad[ni] == 0) continue;
        const bool slot = ((bad[ni] >> (fq * R)) & ((uint64_t(1) << R) - 1)) != 0;
        const vec8 u = __builtin_bit_cast(vec8, up[ni]);
#pragma unroll
        for (int mi = 0; mi < MI; ++mi) {
          const uint32_t w = slot && my_a >= 0 && mine[mi] == my_a ? 0x7fff7fffu : 0u;
          const vec8 l = __builtin_bit_cast(vec8, u32x4{w, w, w, w});
          if constexpr (R == 16) acc[mi][ni] = Elem16<DT>::mfma16(u, l, acc[mi][ni]);
          else acc[mi][ni] = Elem16<DT>::mfma32(u, l, acc[mi][ni]);
        }
        if constexpr (R == 16) hold<MI, NI>(acc);
      }
    }
  }
}

}  // namespace ppmoe
