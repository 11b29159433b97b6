// Low-rank adapters of many requests beside the experts' projections (Section 3.3.2: the local experts' matrices; rows packed
// by expert as the dispatch leaves them), forward and backward:
//
//   v[r, :] = A[a][i] x[r, :],   u[r, :] = W[i] x[r, :] + scale[a] B[a][i] v[r, :],   y = u or GeLU(u)
//   t[r, :] = scale[a] B[a][i]^T dy[r, :],   dx[r, :] = W[i]^T dy[r, :] + A[a][i]^T t[r, :]
//   dA[a][i] = sum_r t[r, :] x[r, :]^T,      dB[a][i] = sum_r dy[r, :] (scale[a] v[r, :])^T
//
// for packed row r of expert i whose token has adapter a.  The product with W is the grouped product of the layer; the matrix
// kernels add the low-rank part to their accumulators (adapter_core.h), so y and dx are rounded once.  Here are the
// products that are narrow in one direction: they read x or dy once and are bound by that.

#include <atomic>
#include <cmath>

#include "adapter_core.h"

namespace ppmoe {
namespace adapter {

constexpr int kMaxRank = 128;
constexpr int kMaxPairs = 1 << 16;   // adapters x experts
constexpr int kMaxColumns = 1 << 20;
constexpr int kMaxRows = (1 << 28) - 256;   // 32 rows a block of 512 threads: below the 2^32 threads that a launch may have

// ---- x A^T: [rows, K] with a matrix [rank, K] of each row's own ------------------------------------------
//
// A block has up to 16 G packed rows, its wavefronts split the contraction, fetch both operands of the matrix instruction
// from memory and meet in LDS, where the partial sums are added in wavefront order.  Within a stretch of the contraction it goes through the
// distinct (adapter, expert) pairs of its rows; a product is kept for the rows of its pair (a row of the operand never meets another
// one's).  Consecutive blocks' rows mostly have the same pairs: an XCD takes a run of them, so that its L2 holds their matrices.
//
// What bounds it is what a CU fetches, x and the pairs' matrices: (16 G + rank) K elements per block of one pair.  Ranks
// above 32 take 64 rows a block, and where that leaves CUs without one the contraction is cut between blocks as well, whose partial sums
// another launch adds (combine_kernel).  Measured: 8192 rows of 2048, 24 requests over 8 experts, rank 32 22 us (34 MB of x, 17 of A: 2.3 TB/s;
// 30 with operands fetched by half lines; 8 of them without any adapter; a step per pair and stretch, each a fetch); 8192 rows of 2048,
// rank 16 14; 4096 rows of 8192, rank 64, cut in four 22 and 6 (3 TB/s); one row of 2048 5.
struct ShrinkArgs {
  const bf16_t* x;        // [rows, K]
  const bf16_t* m;        // [n_adapters, n_exp, rank, K]
  const int32_t *offsets, *adapter, *perm;
  const float* scale;     // [n_adapters] or NULL
  int32_t* of_row;        // out: a word per packed row (adapter_of)
  float* wide;            // out [rows, rank]
  bf16_t* low;            // out [rows, 2 rank]: scaled, as two 16-bit summands
  int n_exp, n_adapters, top_k, K, rank, tile_rows;
  bool scale_wide;        // wide is scaled as well
  int32_t* ticket;        // of count_kernel, set to 0; or NULL
  float* partial;         // [cuts, rows, rank] or NULL
  int cuts, rows;
};

// (low: an operand of the matrix instruction that adds the low-rank part, as two summands, the rounding to 16 bits and that of what it
// leaves, a row's first ones before its second ones: together 16 bits (bf16) or 22, so that the result is as good as rounded once.)
// `power`: of two, that the row's summands are divided by.
template <int DT>
__device__ __forceinline__ void store_low_rank(const ShrinkArgs& a, int64_t row, int j, f32x4 v, float scale, int power) {
  const f32x4 scaled = v * scale;
  *reinterpret_cast<f32x4*>(a.wide + row * a.rank + j) = a.scale_wide ? scaled : v;
  f32x4 rest = DT == MOE_F16 ? scaled * two_to(-power) : scaled;
#pragma unroll
  for (int part = 0; part < 2; ++part) {
    const u32x2 o = {Elem16<DT>::pack2(rest[0], rest[1]), Elem16<DT>::pack2(rest[2], rest[3])};
    *reinterpret_cast<u32x2*>(a.low + (row * 2 + part) * a.rank + j) = o;
    float h[4];
    Elem16<DT>::widen2(o[0], h[0], h[1]);
    Elem16<DT>::widen2(o[1], h[2], h[3]);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      rest[e] -= h[e];
      if (!(fabsf(rest[e]) < 3.0e38f)) rest[e] = 0.f;   // (an infinity or a NaN is in the first summand whole)
    }
  }
}

__host__ __device__ inline int lanes_of_row(int rank) { return rank <= 64 ? 16 : 32; }

// The bits of the largest finite magnitude of v * scale.
__device__ __forceinline__ uint32_t largest_finite(f32x4 v, float scale) {
  uint32_t top = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const uint32_t bits = __float_as_uint(v[e] * scale) & 0x7fffffffu;
    top = bits < 0x7f800000u ? max(top, bits) : top;
  }
  return top;
}

template <int MR, int WAVES, int G>
constexpr int kPartBytes = sizeof(float) * WAVES * 16 * G * (16 * MR + 4);

// MR: blocks of 16 of the rank; J: k-steps of 32 fetched at a time
template <int DT, int MR, int WAVES, int G, int J>
__global__ __launch_bounds__(64 * WAVES) void shrink_kernel(ShrinkArgs a) {
  typedef typename Elem16<DT>::vec8 vec8;
  extern __shared__ __attribute__((aligned(16))) float shrink_lds[];
  auto part = reinterpret_cast<float(*)[16 * G][16 * MR + 4]>(shrink_lds);   // [WAVES]
  __shared__ float row_scale[16 * G];
  __shared__ int row_pair[16 * G];
  __shared__ uint32_t row_top[DT == MOE_F16 ? 16 * G : 1];   // (fp16: of a row's factors)
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int fr = lane & 15, fq = lane >> 4;
  if (a.ticket != nullptr && blockIdx.x == 0 && threadIdx.x == 0) *a.ticket = 0;
  const int lo = a.offsets[0], rows = a.offsets[a.n_exp] - lo;
  const int per = gridDim.x >> 3, nth = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
  const int tile = nth / a.cuts, cut = nth - tile * a.cuts;
  const int row0 = tile * a.tile_rows;
  const int count = min(a.tile_rows, rows - row0);
  if (count <= 0) return;
  // the contraction's share of this block, in whole stretches of all its wavefronts
  constexpr int kStretch = WAVES * 32 * J;
  const int stretches = (a.K + kStretch - 1) / kStretch;
  const int k_end = min(a.K, (cut + 1) * stretches / a.cuts * kStretch), k_begin = cut * stretches / a.cuts * kStretch;
  // Two k-steps of 16 rows are fetched as eight rows of 128 bytes each, whole lines (rows may be a power of two apart, and then one line of each
  // of 16 rows is more than their set of the cache holds until its other half is asked for), and change places in LDS of the
  // wavefront's own.
  static_assert(J % 2 == 0, "k-steps come in pairs");
  unsigned char* own = reinterpret_cast<unsigned char*>(shrink_lds) + kPartBytes<MR, WAVES, G> + wave * 2048;
  auto row_at = [&](int j) __attribute__((always_inline)) -> int { return (j & 1) * 8 + (lane >> 3); };   // of 16
  auto k_at = [&](int j) __attribute__((always_inline)) -> int { return (j >> 1) * 64 + (lane & 7) * 8; };
  auto settle = [&](auto& v) __attribute__((always_inline)) {
    constexpr int N = sizeof(v[0]) / sizeof(u32x4);
#pragma unroll
    for (int j = 0; j < J; j += 2)
#pragma unroll
      for (int n = 0; n < N; ++n) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int row = row_at(h);
          *reinterpret_cast<u32x4*>(own + row * 128 + (((lane & 7) ^ (row & 7)) << 4)) = v[j + h][n];
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) v[j + h][n] = *reinterpret_cast<const u32x4*>(own + fr * 128 + (((h * 4 + fq) ^ (fr & 7)) << 4));
      }
  };
  const u32x4 zero = u32x4{0u, 0u, 0u, 0u};
  u32x4 x[J][G];
  auto load_x = [&](int k0) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
      for (int g = 0; g < G; ++g) {
        const int row = lo + row0 + min(g * 16 + row_at(j), count - 1);
        x[j][g] = k0 + k_at(j) < k_end ? *reinterpret_cast<const u32x4*>(a.x + static_cast<int64_t>(row) * a.K + k0 + k_at(j)) : zero;
      }
  };
  int k0 = k_begin + wave * 32 * J;
  load_x(k0);   // (on their way while the pairs are looked up)
  if (wave == 0 && lane < 16 * G) {
    const bool is = lane < count;
    const int row = lo + row0 + min(lane, count - 1);
    int id = a.adapter[a.perm != nullptr ? a.perm[row] / a.top_k : row];
    if (id < 0 || id >= a.n_adapters) id = -1;
    int expert = 0;   // how many experts' rows end at or before this one
    for (int i = 1; i < a.n_exp; ++i) expert += a.offsets[i] <= row;
    if (DT == MOE_F16) row_top[lane] = 0;
    if (is && cut == 0 && (DT != MOE_F16 || a.cuts > 1)) a.of_row[row] = id;   // (else with its power, below)
    row_scale[lane] = id >= 0 && a.scale != nullptr ? a.scale[id] : 1.f;
    row_pair[lane] = id >= 0 && is ? id * a.n_exp + expert : -1;
  }
  __syncthreads();
  int mine[G];
#pragma unroll
  for (int g = 0; g < G; ++g) mine[g] = row_pair[g * 16 + fr];

  f32x4 acc[G][MR];
#pragma unroll
  for (int g = 0; g < G; ++g)
#pragma unroll
    for (int mr = 0; mr < MR; ++mr) acc[g][mr] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int first = __builtin_amdgcn_readfirstlane(least_above(mine, -1));
  // (the next pair's, or stretch's, operand is on its way while this one's is multiplied)
  auto load_w = [&](u32x4 (&w)[J][MR], int pair, int k) __attribute__((always_inline)) {
    const bf16_t* m = a.m + static_cast<int64_t>(pair) * a.rank * a.K + k;
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
      for (int mr = 0; mr < MR; ++mr)   // (rows past the rank re-read the last one; their sums are not stored)
        w[j][mr] = k + k_at(j) < k_end
                       ? *reinterpret_cast<const u32x4*>(m + static_cast<int64_t>(min(mr * 16 + row_at(j), a.rank - 1)) * a.K + k_at(j))
                       : zero;
  };
  auto multiply = [&](const u32x4 (&w)[J][MR], int pair) __attribute__((always_inline)) {
#pragma unroll
    for (int g = 0; g < G; ++g) {
      f32x4 sum[MR];
#pragma unroll
      for (int mr = 0; mr < MR; ++mr) sum[mr] = acc[g][mr];
#pragma unroll
      for (int j = 0; j < J; ++j)
#pragma unroll
        for (int mr = 0; mr < MR; ++mr)
          sum[mr] = Elem16<DT>::mfma16(__builtin_bit_cast(vec8, w[j][mr]), __builtin_bit_cast(vec8, x[j][g]), sum[mr]);
      // D: lane row fr, rank index mr * 16 + fq * 4 + v
#pragma unroll
      for (int mr = 0; mr < MR; ++mr)
        if (mine[g] == pair) acc[g][mr] = sum[mr];
    }
  };
  if (first != kNone && k0 < k_end) {
    u32x4 w0[J][MR], w1[J][MR];
    int pair = first, now;
    bool fresh = true;   // x has been asked for
    load_w(w0, pair, k0);
    // what follows (pair, k0): the next pair of the same stretch, or the first one of the next
    auto turn = [&](u32x4 (&w)[J][MR], u32x4 (&other)[J][MR]) __attribute__((always_inline)) -> bool {
      now = pair;
      pair = __builtin_amdgcn_readfirstlane(least_above(mine, pair));
      const bool same = pair != kNone;
      if (!same) {
        pair = first;
        k0 += kStretch;
      }
      const bool more = k0 < k_end;
      if (more) load_w(other, pair, k0);
      __builtin_amdgcn_sched_barrier(0);
      if (fresh) settle(x);
      settle(w);
      multiply(w, now);
      fresh = more && !same;
      if (fresh) load_x(k0);
      return more;
    };
    while (turn(w0, w1) && turn(w1, w0)) {
    }
  }
#pragma unroll
  for (int g = 0; g < G; ++g)
#pragma unroll
    for (int mr = 0; mr < MR; ++mr) *reinterpret_cast<f32x4*>(&part[wave][g * 16 + fr][mr * 16 + fq * 4]) = acc[g][mr];
  __syncthreads();
  for (int p = threadIdx.x; p < count * (a.rank / 4); p += 64 * WAVES) {
    const int q = p / (a.rank / 4), j = (p - q * (a.rank / 4)) * 4;
    f32x4 v = *reinterpret_cast<const f32x4*>(&part[0][q][j]);
#pragma unroll
    for (int w = 1; w < WAVES; ++w) v += *reinterpret_cast<const f32x4*>(&part[w][q][j]);
    const int64_t row = lo + row0 + q;
    if (a.cuts > 1) {
      *reinterpret_cast<f32x4*>(a.partial + (cut * static_cast<int64_t>(a.rows) + row) * a.rank + j) = v;
    } else if (DT == MOE_F16) {
      *reinterpret_cast<f32x4*>(&part[0][q][j]) = v;
      atomicMax(&row_top[q], largest_finite(v, row_scale[q]));   // (the largest, in whatever order)
    } else {
      store_low_rank<DT>(a, row, j, v, row_scale[q], 0);
    }
  }
  if (DT != MOE_F16 || a.cuts > 1) return;
  __syncthreads();
  for (int p = threadIdx.x; p < count * (a.rank / 4); p += 64 * WAVES) {   // (each thread what it has left there)
    const int q = p / (a.rank / 4), j = (p - q * (a.rank / 4)) * 4;
    const int power = power_for(row_top[q]);
    const int64_t row = lo + row0 + q;
    store_low_rank<DT>(a, row, j, *reinterpret_cast<const f32x4*>(&part[0][q][j]), row_scale[q], power);
    if (j == 0) a.of_row[row] = row_word(row_pair[q] < 0 ? -1 : row_pair[q] / a.n_exp, power);
  }
}

// The shares of a cut contraction, added in order; 16 or 32 lanes have a row, four columns each (ranks up to 64, up to 128).
template <int DT>
__global__ __launch_bounds__(256) void combine_kernel(ShrinkArgs a) {
  const int lo = a.offsets[0], lanes = lanes_of_row(a.rank);
  const int64_t total = static_cast<int64_t>(a.offsets[a.n_exp] - lo) * lanes;
  for (int64_t p = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; p < total; p += static_cast<int64_t>(gridDim.x) * 256) {
    const int64_t row = lo + p / lanes;
    const int j = static_cast<int>(p % lanes) * 4;
    const bool is = j < a.rank;
    const int64_t at = row * a.rank + min(j, a.rank - 4);
    f32x4 v = *reinterpret_cast<const f32x4*>(a.partial + at);
    for (int cut = 1; cut < a.cuts; ++cut) v += *reinterpret_cast<const f32x4*>(a.partial + cut * static_cast<int64_t>(a.rows) * a.rank + at);
    const int id = a.of_row[row];
    const float scale = id >= 0 && a.scale != nullptr ? a.scale[id] : 1.f;
    int power = 0;
    if (DT == MOE_F16) {
      uint32_t top = largest_finite(v, scale);
      for (int off = lanes / 2; off >= 1; off >>= 1) top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), off, 64)));
      power = power_for(top);
      if (j == 0) a.of_row[row] = row_word(id, power);   // (the row's lanes, one wavefront's, have read it)
    }
    if (is) store_low_rank<DT>(a, row, j, v, scale, power);
  }
}

// ---- [batch, R, C] -> [batch, C, R], 16-bit, both multiples of 8; two such tensors in one launch ---------------------
//
// A thread turns 8 x 8 elements in its registers: eight pieces of 16 bytes in, eight out.  Neighbouring threads are neighbours along the
// shorter side (the rank), then along the other: what a wavefront reads, or writes, are runs of rank elements and more.
// Bound by memory: 42 MB turned in 21 us (4.0 TB/s; 26 us through LDS in tiles of 64 x 64, which a rank of 16 fills to a quarter).
struct Transpose {
  const bf16_t* in;
  bf16_t* out;
  int R, C;
  int64_t units;   // of 8 x 8
};
__global__ __launch_bounds__(256) void transpose_kernel(Transpose t0, Transpose t1, unsigned blocks0) {
  const bool first = blockIdx.x < blocks0;
  const Transpose a = first ? t0 : t1;
  const int64_t unit = static_cast<int64_t>(first ? blockIdx.x : blockIdx.x - blocks0) * 256 + threadIdx.x;
  if (unit >= a.units) return;
  const uint32_t r8 = a.R >> 3, c8 = a.C >> 3, per = r8 * c8, low = min(r8, c8);
  const uint32_t batch = static_cast<uint32_t>(unit / per), u = static_cast<uint32_t>(unit - static_cast<int64_t>(batch) * per);
  const uint32_t outer = u / low, inner = u - outer * low;
  const uint32_t r = (r8 <= c8 ? inner : outer) * 8, c = (r8 <= c8 ? outer : inner) * 8;
  const int64_t base = static_cast<int64_t>(batch) * a.R * a.C;
  const bf16_t* src = a.in + base + static_cast<int64_t>(r) * a.C + c;
  bf16_t* dst = a.out + base + static_cast<int64_t>(c) * a.R + r;
  u32x4 v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = *reinterpret_cast<const u32x4*>(src + static_cast<int64_t>(i) * a.C);
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    u32x4 o;
#pragma unroll
    for (int q = 0; q < 4; ++q)   // columns j of rows 2 q and 2 q + 1
      o[q] = __builtin_amdgcn_perm(v[2 * q + 1][j >> 1], v[2 * q][j >> 1], j & 1 ? 0x07060302u : 0x05040100u);
    *reinterpret_cast<u32x4*>(dst + static_cast<int64_t>(j) * a.R) = o;
  }
}

// ---- the rows of each (adapter, expert) pair -----------------------------------------------------------
//
// list: the packed rows ordered by pair (adapter-major, as dA and dB are), ascending inside it; begin[pair] where they start.
// A pair's rows are cut into pieces of at most `most` for a gradient (one table for dA, one for dB); a pair of several pieces
// has a slot of partial sums for each.  Counted, scanned, filled: the same order on every run.
struct Pieces {
  int32_t *begin;   // [pairs + 1] first piece of a pair
  int32_t *slot;    // [pairs + 1] its first slot
  int32_t *pair;    // [most pieces] a piece's pair
  int most;
};
struct Groups {
  int32_t *begin;   // [pairs + 1]
  int32_t *list;    // [rows]
  int32_t *ticket;  // blocks of count_kernel that are done
  Pieces pieces[2];
};

__device__ __forceinline__ int sum_of_block(int v, int* lds) {   // 256 threads
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) v += __shfl_xor(v, off, 64);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  return lds[0] + lds[1] + lds[2] + lds[3];
}

// A block counts a pair's rows; the one that comes last adds them up (the ticket: which one that is does not show in what it writes).
__global__ __launch_bounds__(256) void count_kernel(const int32_t* __restrict__ of_row, const int32_t* __restrict__ offsets, int n_exp, Groups g,
                                                    int pairs) {
  __shared__ int lds[4];
  __shared__ int last;
  __shared__ int sums[5][4];
  {
    const int id = blockIdx.x / n_exp, expert = blockIdx.x - id * n_exp;
    int n = 0;
    const int end = offsets[expert + 1];
    for (int r = offsets[expert] + threadIdx.x; r < end; r += 4 * 256) {   // (four loads under way)
      int v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = of_row[min(r + i * 256, end - 1)];
#pragma unroll
      for (int i = 0; i < 4; ++i) n += r + i * 256 < end && has_adapter(v[i], id);
    }
    n = sum_of_block(n, lds);
    if (threadIdx.x == 0) {
      __hip_atomic_store(g.begin + blockIdx.x, n, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      last = __hip_atomic_fetch_add(g.ticket, 1, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == pairs - 1;
    }
  }
  __syncthreads();
  if (!last) return;
  int before[5] = {0, 0, 0, 0, 0};
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int p0 = 0; p0 < pairs; p0 += 256) {
    const int p = p0 + threadIdx.x;
    const int n = p < pairs ? __hip_atomic_load(g.begin + p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0;
    const int p_a = (n + g.pieces[0].most - 1) / g.pieces[0].most, p_b = (n + g.pieces[1].most - 1) / g.pieces[1].most;
    int own[5] = {n, p_a, p_a > 1 ? p_a : 0, p_b, p_b > 1 ? p_b : 0}, up_to[5];
#pragma unroll
    for (int q = 0; q < 5; ++q) {
      int v = own[q];
#pragma unroll
      for (int off = 1; off < 64; off <<= 1) {
        const int o = __shfl_up(v, off, 64);
        if (lane >= off) v += o;
      }
      up_to[q] = v;
      if (lane == 63) sums[q][wave] = v;
    }
    __syncthreads();
    int total[5];
#pragma unroll
    for (int q = 0; q < 5; ++q) {
      int base = 0;
      total[q] = 0;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        if (w < wave) base += sums[q][w];
        total[q] += sums[q][w];
      }
      up_to[q] += base + before[q] - own[q];
    }
    if (p < pairs) {
      g.begin[p] = up_to[0];
      g.pieces[0].begin[p] = up_to[1];
      g.pieces[0].slot[p] = up_to[2];
      g.pieces[1].begin[p] = up_to[3];
      g.pieces[1].slot[p] = up_to[4];
    }
#pragma unroll
    for (int q = 0; q < 5; ++q) before[q] += total[q];
    __syncthreads();
  }
  if (threadIdx.x == 0) {
    g.begin[pairs] = before[0];
    g.pieces[0].begin[pairs] = before[1];
    g.pieces[0].slot[pairs] = before[2];
    g.pieces[1].begin[pairs] = before[3];
    g.pieces[1].slot[pairs] = before[4];
  }
}

__global__ __launch_bounds__(256) void fill_kernel(const int32_t* __restrict__ of_row, const int32_t* __restrict__ offsets, int n_exp, Groups g) {
  __shared__ int lds[4];
  const int pair = blockIdx.x, id = pair / n_exp, expert = pair - id * n_exp;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int at = g.begin[pair];
  if (at == g.begin[pair + 1]) return;
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const int p0 = g.pieces[t].begin[pair], p1 = g.pieces[t].begin[pair + 1];
    for (int p = p0 + threadIdx.x; p < p1; p += 256) g.pieces[t].pair[p] = pair;
  }
  // A thread has four neighbouring rows of 1024.
  const int end = offsets[expert + 1];
  for (int r0 = offsets[expert]; r0 < end; r0 += 1024) {
    const int r = r0 + threadIdx.x * 4;
    int v[4], mine = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = of_row[min(r + i, end - 1)];
#pragma unroll
    for (int i = 0; i < 4; ++i) mine += r + i < end && has_adapter(v[i], id);
    int before = mine;   // of the wavefront's lanes up to this one
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
      const int o = __shfl_up(before, off, 64);
      if (lane >= off) before += o;
    }
    __syncthreads();
    if (lane == 63) lds[wave] = before;
    __syncthreads();
    int to = at + before - mine;
    for (int w = 0; w < wave; ++w) to += lds[w];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (r + i < end && has_adapter(v[i], id)) g.list[to++] = r + i;
    at += lds[0] + lds[1] + lds[2] + lds[3];
  }
}

// ---- G[pair][j, c] = sum over the pair's rows of s u[r, j] z[r, c] ------------------------------------------
//
// u [rows, rank] float32 (t, or v), z [rows, C] 16-bit (x, or dy).  dA is stored [rank, C], dB [C, rank] (BY_COLUMN).
// A block takes one piece of a pair's rows and 128 columns, 64 rows at a time: both as they are into LDS and from there
// across their rows into operands (transposing read), u as 16-bit summands, each the rounding of what those before it leave: three for
// bf16, two for fp16 (24 and 22 bits together), so that the result has float32's accuracy.  fp16: u is first brought
// to a largest value of 2^13 by a power of two, exactly, as its small values have no 22 bits.
// Bound by memory where the pairs are many (8192 rows, x of 8192 and dy of 2048, 128 pairs of rank 16: 251 MB in 48 us, 5.2 TB/s), by staging u
// at larger ranks (4096 rows, 2048 and 8192, rank 64: 84 MB and 40 MB of partial sums in 42 us; u turned by 2-byte stores into LDS: 75).
constexpr int kGradColumns = 128, kGradThreads = 256, kGradRows = 64;

struct GradArgs {
  const float* u;
  const float* scale;           // by adapter, or NULL
  const bf16_t* z;
  float *out, *partial;         // [pairs, rank * C], [slots, rank * C]
  Pieces pieces;
  int C;
};
struct BothGrads {
  GradArgs of[2];               // dA, dB
  Groups g;
  int pairs, n_exp, rank, blocks_a;
};

template <int DT, int MR, bool BY_COLUMN>
__device__ __forceinline__ void gradient_piece(const BothGrads& b, const GradArgs& a, int block, unsigned char* z_lds, unsigned char* u_lds,
                                               int (*ids)[kGradRows], float* wave_top) {
  typedef typename Elem16<DT>::vec8 vec8;
  constexpr int P = DT == MOE_F16 ? 2 : 3;   // summands
  const int col_blocks = (a.C + kGradColumns - 1) / kGradColumns;
  const int piece = block / col_blocks, col0 = (block - piece * col_blocks) * kGradColumns;
  if (piece >= a.pieces.begin[b.pairs]) return;
  const int pair = a.pieces.pair[piece];
  const int nth = piece - a.pieces.begin[pair], pieces = a.pieces.begin[pair + 1] - a.pieces.begin[pair];
  const int first = b.g.begin[pair] + nth * a.pieces.most, count = min(a.pieces.most, b.g.begin[pair + 1] - first);
  const int32_t* list = b.g.list + first;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int fr = lane & 15, fq = lane >> 4;
  const float s = a.scale != nullptr ? a.scale[pair / b.n_exp] : 1.f;
  const int rank = b.rank, quads = rank / 4;   // of a row of u

  float up = 1.f, down = 1.f;
  if (DT == MOE_F16) {
    float top = 0.f;
    for (int p = tid; p < count * quads; p += kGradThreads) {
      const int q = p / quads;
      const f32x4 v = *reinterpret_cast<const f32x4*>(a.u + static_cast<int64_t>(list[q]) * rank + (p - q * quads) * 4);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float m = fabsf(v[e] * s);
        top = m < __builtin_inff() ? fmaxf(top, m) : top;   // (infinities and NaNs stay what they are at any scale)
      }
    }
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) top = fmaxf(top, __shfl_xor(top, off, 64));
    if (lane == 0) wave_top[wave] = top;
    __syncthreads();
    top = fmaxf(fmaxf(wave_top[0], wave_top[1]), fmaxf(wave_top[2], wave_top[3]));
    const int e = static_cast<int>(__float_as_uint(top) >> 23) - 127;
    if (e > -110) {   // (zeros, and what is beyond any use, as they are)
      up = __uint_as_float(static_cast<uint32_t>(127 + 13 - e) << 23);
      down = __uint_as_float(static_cast<uint32_t>(127 - 13 + e) << 23);
    }
  }

  // The rows' numbers are in LDS a stage ahead of their data: a load then waits for nothing.
  auto number = [&](int k) __attribute__((always_inline)) -> int { return list[min(k, count - 1)]; };   // (threads of the first wavefront)
  int upcoming = 0, now = 0;
  if (tid < kGradRows) {
    ids[0][tid] = number(tid);
    upcoming = number(kGradRows + tid);
  }
  __syncthreads();
  // staging: z in 1024 pieces of 16 bytes, four per thread (row p / 16, piece p % 16); u in quads
  u32x4 zv[4];
  constexpr int kQuads = 16 * MR * kGradRows / 4 / kGradThreads;
  f32x4 uv[kQuads];
  auto load = [&](int k0) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int p = tid + i * kGradThreads, row = k0 + (p >> 4), c = col0 + (p & 15) * 8;
      zv[i] = row < count && c < a.C ? *reinterpret_cast<const u32x4*>(a.z + static_cast<int64_t>(ids[now][p >> 4]) * a.C + c) : u32x4{0u, 0u, 0u, 0u};
    }
#pragma unroll
    for (int i = 0; i < kQuads; ++i) {
      const int p = tid + i * kGradThreads, q = p / (4 * MR), j = (p % (4 * MR)) * 4, row = k0 + q;
      uv[i] = row < count && j < rank ? *reinterpret_cast<const f32x4*>(a.u + static_cast<int64_t>(ids[now][q]) * rank + j) : f32x4{0.f, 0.f, 0.f, 0.f};
    }
  };
  // 32-byte block b of row k of z at b ^ ((k & 3) + 4 ((k >> 3) & 1)): what 32 lanes of a transposing read touch falls on all banks; u's
  // rows of 32 MR bytes the same way as far as they have blocks
  auto u_swizzle = [](int k) __attribute__((always_inline)) -> int {
    return (MR == 8 ? (k & 3) + 4 * ((k >> 3) & 1) : (k & 3) ^ ((k >> 3) & 1)) & (MR - 1);
  };
  auto store = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int p = tid + i * kGradThreads, k = p >> 4, c = p & 15;
      const int blk = (c >> 1) ^ ((k & 3) + 4 * ((k >> 3) & 1));
      *reinterpret_cast<u32x4*>(z_lds + k * (kGradColumns * 2) + blk * 32 + (c & 1) * 16) = zv[i];
    }
#pragma unroll
    for (int i = 0; i < kQuads; ++i) {
      const int p = tid + i * kGradThreads, q = p / (4 * MR), j = p % (4 * MR);
      unsigned char* at = u_lds + q * (32 * MR) + ((j >> 2) ^ u_swizzle(q)) * 32 + (j & 3) * 8;
      f32x4 rest = uv[i] * (s * up);
#pragma unroll
      for (int part = 0; part < P; ++part) {
        const u32x2 o = {Elem16<DT>::pack2(rest[0], rest[1]), Elem16<DT>::pack2(rest[2], rest[3])};
        *reinterpret_cast<u32x2*>(at + part * (kGradRows * 32 * MR)) = o;
        float h[4];
        Elem16<DT>::widen2(o[0], h[0], h[1]);
        Elem16<DT>::widen2(o[1], h[2], h[3]);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          rest[e] -= h[e];
          if (!(fabsf(rest[e]) < 3.0e38f)) rest[e] = 0.f;   // (an infinity or a NaN is in the first summand whole)
        }
      }
    }
  };

  f32x4 acc[MR][2];
#pragma unroll
  for (int mr = 0; mr < MR; ++mr)
#pragma unroll
    for (int ni = 0; ni < 2; ++ni) acc[mr][ni] = f32x4{0.f, 0.f, 0.f, 0.f};
  const uint32_t z0 = core::lds_address(z_lds), u0 = core::lds_address(u_lds);
  load(0);
  for (int k0 = 0; k0 < count; k0 += kGradRows) {
    __syncthreads();
    store();
    now ^= 1;
    if (tid < kGradRows) ids[now][tid] = upcoming;
    __syncthreads();
    if (k0 + kGradRows < count) {
      load(k0 + kGradRows);
      if (tid < kGradRows) upcoming = number(k0 + 2 * kGradRows + tid);
    }
    const int j = (lane >> 2) & 3;
#pragma unroll
    for (int ks = 0; ks < kGradRows / 32; ++ks) {
      u32x2 zt[2][2];
#pragma unroll
      for (int ni = 0; ni < 2; ++ni) {
        const uint32_t at = z0 + (ks * 32 + fq * 8 + j) * (kGradColumns * 2) + (((wave * 2 + ni) ^ (j + 4 * (fq & 1))) << 5) + (lane & 3) * 8;
        asm volatile("ds_read_b64_tr_b16 %0, %2\n\tds_read_b64_tr_b16 %1, %2 offset:1024"
                     : "=&v"(zt[ni][0]), "=&v"(zt[ni][1]) : "v"(at) : "memory");
      }
      u32x2 ut[P][MR][2];
      core::each<P * MR>([&](auto i) __attribute__((always_inline)) {
        constexpr int part = i.value / MR, mr = i.value % MR;
        const uint32_t at = u0 + (ks * 32 + fq * 8 + j) * (32 * MR) + ((mr ^ u_swizzle(fq * 8 + j)) << 5) + (lane & 3) * 8;
        core::lds_read_transposed<part * (kGradRows * 32 * MR)>(ut[part][mr][0], at);
        core::lds_read_transposed<part * (kGradRows * 32 * MR) + 4 * 32 * MR>(ut[part][mr][1], at);
      });
      asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(zt[0][0]), "+v"(zt[0][1]), "+v"(zt[1][0]), "+v"(zt[1][1]) : : "memory");
      vec8 u[P][MR];
#pragma unroll
      for (int part = 0; part < P; ++part)
#pragma unroll
        for (int mr = 0; mr < MR; ++mr) {
          asm volatile("" : "+v"(ut[part][mr][0]), "+v"(ut[part][mr][1]) : : "memory");
          u[part][mr] = __builtin_bit_cast(vec8, __builtin_shufflevector(ut[part][mr][0], ut[part][mr][1], 0, 1, 2, 3));
        }
#pragma unroll
      for (int ni = 0; ni < 2; ++ni) {
        const vec8 z = __builtin_bit_cast(vec8, __builtin_shufflevector(zt[ni][0], zt[ni][1], 0, 1, 2, 3));
#pragma unroll
        for (int mr = 0; mr < MR; ++mr)
#pragma unroll
          for (int part = P - 1; part >= 0; --part)   // D: lane: index of the second operand, registers: 4 (lane / 16) + v of the first
            acc[mr][ni] = BY_COLUMN ? Elem16<DT>::mfma16(u[part][mr], z, acc[mr][ni]) : Elem16<DT>::mfma16(z, u[part][mr], acc[mr][ni]);
      }
    }
  }
  const int64_t size = static_cast<int64_t>(rank) * a.C;
  float* out = pieces > 1 ? a.partial + (a.pieces.slot[pair] + nth) * size : a.out + pair * size;
#pragma unroll
  for (int ni = 0; ni < 2; ++ni)
#pragma unroll
    for (int mr = 0; mr < MR; ++mr) {
      const int c = col0 + wave * 32 + ni * 16 + (BY_COLUMN ? fr : fq * 4), jj = mr * 16 + (BY_COLUMN ? fq * 4 : fr);
      if (c < a.C && jj < rank)
        *reinterpret_cast<f32x4*>(out + (BY_COLUMN ? static_cast<int64_t>(c) * rank + jj : static_cast<int64_t>(jj) * a.C + c)) =
            acc[mr][ni] * down;
    }
}

// Both gradients in one launch: the first blocks_a blocks dA's, the others dB's.
template <int DT, int MR>
__global__ __launch_bounds__(kGradThreads) void gradient_kernel(BothGrads b) {
  constexpr int P = DT == MOE_F16 ? 2 : 3;
  __shared__ __attribute__((aligned(16))) unsigned char z_lds[kGradRows * kGradColumns * 2];
  __shared__ __attribute__((aligned(16))) unsigned char u_lds[P * kGradRows * 32 * MR];
  __shared__ float wave_top[4];
  __shared__ int ids[2][kGradRows];
  if (static_cast<int>(blockIdx.x) < b.blocks_a) gradient_piece<DT, MR, false>(b, b.of[0], blockIdx.x, z_lds, u_lds, ids, wave_top);
  else gradient_piece<DT, MR, true>(b, b.of[1], blockIdx.x - b.blocks_a, z_lds, u_lds, ids, wave_top);
}

// Pairs without rows: zeros; of several pieces: the partial sums in order.  per_pair[t] blocks per pair for gradient t.
struct FinishArgs {
  BothGrads b;
  int per_pair[2];
  bool no_rows;     // nothing was counted: zeros everywhere
};
__global__ __launch_bounds__(256) void finish_kernel(FinishArgs f) {
  const int t = static_cast<int>(blockIdx.x) < f.b.pairs * f.per_pair[0] ? 0 : 1;
  const GradArgs& a = f.b.of[t];
  const int block = blockIdx.x - t * f.b.pairs * f.per_pair[0];
  const int pair = block / f.per_pair[t], part = block - pair * f.per_pair[t];
  int slot = 0, slots = 0;
  if (!f.no_rows) {
    slot = a.pieces.slot[pair];
    slots = a.pieces.slot[pair + 1] - slot;
    if (slots == 0 && f.b.g.begin[pair + 1] > f.b.g.begin[pair]) return;   // written already
  }
  const int64_t quads = static_cast<int64_t>(f.b.rank) * a.C / 4;
  f32x4* out = reinterpret_cast<f32x4*>(a.out) + pair * quads;
  const f32x4* in = reinterpret_cast<const f32x4*>(a.partial) + slot * quads;
  for (int64_t q = static_cast<int64_t>(part) * 256 + threadIdx.x; q < quads; q += static_cast<int64_t>(f.per_pair[t]) * 256) {
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    for (int k = 0; k < slots; k += 4) {
      f32x4 p[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) p[i] = in[min(k + i, slots - 1) * quads + q];
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (k + i < slots) v += p[i];
    }
    out[q] = v;
  }
}

// ---- host ----------------------------------------------------------------------------------------

inline size_t align_up(size_t v) { return (v + 255) / 256 * 256; }
inline bool misaligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }

int check_config(const moe_adapter_config* c) {
  if (c == nullptr) return MOE_ERR_NULL;
  if (c->rows < 0 || c->rows > kMaxRows) return MOE_ERR_SHAPE;
  if (c->K <= 0 || c->N <= 0 || (c->K & 7) || (c->N & 7) || c->K > kMaxColumns || c->N > kMaxColumns) return MOE_ERR_SHAPE;
  if (c->n_exp < 1 || c->n_exp > kMaxExperts || c->n_adapters < 1 || c->n_adapters > kMaxPairs / c->n_exp) return MOE_ERR_SHAPE;
  if (c->rank < 8 || c->rank > kMaxRank || (c->rank & 7) || c->top_k < 1 || c->top_k > kMaxTopK) return MOE_ERR_SHAPE;
  if (!is_16bit(c->dtype)) return MOE_ERR_DTYPE;
  if (c->activation != MOE_ACT_NONE && c->activation != MOE_ACT_GELU) return MOE_ERR_SHAPE;
  return MOE_OK;
}

// Rows of a piece of a gradient of C columns: so many pieces that there are some 256 blocks, one per CU, if one pair has all the
// rows; 256 at least (fewer would write and read more partial sums than they read of z: rank * C floats per piece).  Half as many rows, against these:
// the backward of 4096 rows of 2048 from 8192, rank 64: 224 and 218 us; of 1024 from 1024, 8 adapters: 61 and 58.
int rows_of_piece(const moe_adapter_config& c, int C) {
  const int64_t col_blocks = (C + kGradColumns - 1) / kGradColumns;
  int64_t n = (c.rows * col_blocks + 255) / 256;
  if (n > c.rows) n = c.rows;   // (more than 256 blocks side by side already)
  return static_cast<int>(n < 256 ? 256 : (n + kGradRows - 1) / kGradRows * kGradRows);
}
int64_t most_pieces(const moe_adapter_config& c, int C) {
  const int64_t pairs = static_cast<int64_t>(c.n_exp) * c.n_adapters;
  return c.rows / rows_of_piece(c, C) + 1 + (pairs < c.rows ? pairs : c.rows);
}
// A pair of several pieces has more rows than one piece: at most two slots per full piece.
int64_t most_slots(const moe_adapter_config& c, int C) { return 2 * (static_cast<int64_t>(c.rows) / rows_of_piece(c, C)) + 1; }

// Rows of a block and cuts of the contraction.  Ranks above 32 with more than 512 rows: 64 rows, as the matrices weigh as much as the rows,
// and the contraction cut, down to a stretch of the block's wavefronts, while that leaves CUs without a block (1000 rows of 2048 to 8192, rank
// 128, whole forward: 93 us with shares of 1024 and more, 83 with these).  Otherwise 32 rows, and fewer while that leaves CUs without a block, down
// to one: a row's own adapter is a block's whole work then (300 rows of 1024, rank 64: 45 us the forward, 48 with 64 rows a block).
void shape_of_shrink(int64_t rows, int rank, int K, int* tile_rows, int* cuts) {
  *cuts = 1;
  if (rank > 32 && rows > 512) {
    const int64_t tiles = (rows + 63) / 64;
    const int stretch = rank > 64 ? 256 : 512;
    *tile_rows = 64;
    while (*cuts < 8 && tiles * *cuts * 2 <= 256 && K / (*cuts * 2) >= stretch) *cuts *= 2;
    return;
  }
  int t = 32;
  while (t > 1 && (rows + t / 2 - 1) / (t / 2) <= 256) t /= 2;
  *tile_rows = t;
}

struct Layout {
  size_t of_row, low, gemm, cut, total;                                                   // forward and backward
  size_t t, At, Bt, begin, list, ticket, piece_begin[2], slot[2], piece_pair[2], partial[2];   // backward
};

Layout layout_of(const moe_adapter_config& c, bool backward) {
  Layout L = {};
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t at = off;
    off = align_up(off + bytes);
    return at;
  };
  const size_t rows = c.rows, pairs = static_cast<size_t>(c.n_exp) * c.n_adapters;
  L.of_row = take(rows * 4);
  L.low = take(rows * c.rank * 4);
  L.gemm = take(grouped_gemm_workspace_bytes());
  int tile_rows = 0, cuts = 1;
  shape_of_shrink(c.rows, c.rank, backward ? c.N : c.K, &tile_rows, &cuts);
  L.cut = take(cuts > 1 ? cuts * rows * c.rank * 4 : 0);
  if (backward) {
    L.t = take(rows * c.rank * 4);
    L.At = take(pairs * c.rank * c.K * 2);
    L.Bt = take(pairs * c.rank * c.N * 2);
    L.begin = take((pairs + 1) * 4);
    L.list = take(rows * 4);
    L.ticket = take(4);
    for (int t = 0; t < 2; ++t) {
      const int C = t == 0 ? c.K : c.N;
      L.piece_begin[t] = take((pairs + 1) * 4);
      L.slot[t] = take((pairs + 1) * 4);
      L.piece_pair[t] = take(most_pieces(c, C) * 4);
      L.partial[t] = take(most_slots(c, C) * c.rank * C * 4);
    }
  }
  L.total = off;
  return L;
}

// The backward's launches over pairs and columns stay within what a grid may have.
int check_backward(const moe_adapter_config* c) {
  const int st = check_config(c);
  if (st != MOE_OK) return st;
  if (c->activation != MOE_ACT_NONE) return MOE_ERR_SHAPE;
  return (static_cast<int64_t>(c->K) + c->N) * c->n_exp * c->n_adapters > (int64_t(1) << 28) ? MOE_ERR_SHAPE : MOE_OK;
}

struct Memory {
  const void* at;   // or NULL
  size_t bytes;
};
// Does one of the first `written` overlap another?
template <int N>
bool overlapping(const Memory (&m)[N], int written) {
  for (int i = 0; i < written; ++i)
    for (int j = i + 1; j < N; ++j) {
      const uintptr_t a = reinterpret_cast<uintptr_t>(m[i].at), b = reinterpret_cast<uintptr_t>(m[j].at);
      if (a != 0 && b != 0 && a < b + m[j].bytes && b < a + m[i].bytes) return true;
    }
  return false;
}

// What the call knows of the size of `adapter`: a token per row without perm, else at least one.
size_t bytes_of_adapter(const moe_adapter_config& c, const int32_t* perm) {
  return c.rows == 0 ? 0 : perm == nullptr ? static_cast<size_t>(c.rows) * 4 : 4;
}

template <int DT>
hipError_t launch_shrink_of(const ShrinkArgs& a, int64_t rows, hipStream_t s) {
  const int64_t tiles = (rows + a.tile_rows - 1) / a.tile_rows * a.cuts;
  const unsigned grid = static_cast<unsigned>((tiles + 7) / 8 * 8);   // (every XCD the same run of tiles)
#define PPMOE_SHRINK(MR, WAVES, G, J)                                                                      \
  do {                                                                                                     \
    constexpr int kLds = kPartBytes<MR, WAVES, G> + WAVES * 2048;                                          \
    if (kLds > 65536) {                                                                                    \
      static std::atomic<uint64_t> done{0};                                                                \
      const hipError_t e = once_per_device(done, [] {                                                      \
        return hipFuncSetAttribute(reinterpret_cast<const void*>(shrink_kernel<DT, MR, WAVES, G, J>),      \
                                   hipFuncAttributeMaxDynamicSharedMemorySize, kLds);                      \
      });                                                                                                  \
      if (e != hipSuccess) return e;                                                                       \
    }                                                                                                      \
    shrink_kernel<DT, MR, WAVES, G, J><<<grid, 64 * WAVES, kLds, s>>>(a);                                  \
  } while (0)
  if (a.tile_rows > 32) {
    if (a.rank <= 64) PPMOE_SHRINK(4, 8, 4, 2);
    else PPMOE_SHRINK(8, 4, 4, 2);
  } else if (a.tile_rows > 16) {   // (ranks up to 32 alone: shape_of_shrink)
    if (a.rank <= 16) PPMOE_SHRINK(1, 8, 2, 4);
    else PPMOE_SHRINK(2, 8, 2, 4);
  } else if (a.rank <= 16) PPMOE_SHRINK(1, 8, 1, 8);
  else if (a.rank <= 32) PPMOE_SHRINK(2, 8, 1, 4);
  else if (a.rank <= 64) PPMOE_SHRINK(4, 8, 1, 4);
  else PPMOE_SHRINK(8, 8, 1, 2);
#undef PPMOE_SHRINK
  if (a.cuts > 1) {
    const int64_t blocks = (rows * lanes_of_row(a.rank) + 255) / 256;
    combine_kernel<DT><<<static_cast<unsigned>(blocks < 4096 ? blocks : 4096), 256, 0, s>>>(a);
  }
  return hipGetLastError();
}
hipError_t launch_shrink(int dtype, ShrinkArgs a, int64_t rows, hipStream_t s) {
  shape_of_shrink(rows, a.rank, a.K, &a.tile_rows, &a.cuts);
  a.rows = static_cast<int>(rows);
  return dtype == MOE_F16 ? launch_shrink_of<MOE_F16>(a, rows, s) : launch_shrink_of<MOE_BF16>(a, rows, s);
}

Transpose transpose_of(const void* in, void* out, int R, int C, int64_t batch) {
  return {static_cast<const bf16_t*>(in), static_cast<bf16_t*>(out), R, C, batch * (R / 8) * (C / 8)};
}
unsigned blocks_of(const Transpose& t) { return static_cast<unsigned>((t.units + 255) / 256); }

template <int DT>
hipError_t launch_gradients_of(const BothGrads& b, int64_t blocks, hipStream_t s) {
  const unsigned grid = static_cast<unsigned>(blocks);
  if (b.rank <= 16) gradient_kernel<DT, 1><<<grid, kGradThreads, 0, s>>>(b);
  else if (b.rank <= 32) gradient_kernel<DT, 2><<<grid, kGradThreads, 0, s>>>(b);
  else if (b.rank <= 64) gradient_kernel<DT, 4><<<grid, kGradThreads, 0, s>>>(b);
  else gradient_kernel<DT, 8><<<grid, kGradThreads, 0, s>>>(b);
  return hipGetLastError();
}

}  // namespace adapter
}  // namespace ppmoe

using namespace ppmoe;

extern "C" {

size_t moe_adapter_workspace_bytes(const moe_adapter_config* cfg) {
  return adapter::check_config(cfg) == MOE_OK ? adapter::layout_of(*cfg, false).total : 0;
}

size_t moe_adapter_backward_workspace_bytes(const moe_adapter_config* cfg) {
  return adapter::check_backward(cfg) == MOE_OK ? adapter::layout_of(*cfg, true).total : 0;
}

int moe_adapter_forward(const moe_adapter_config* cfg, const void* x, const int32_t* offsets, const void* W, const void* A,
                        const void* B, const float* scale, const int32_t* adapter, const int32_t* perm, void* y, float* v,
                        void* workspace, size_t workspace_bytes, void* stream) {
  const int st = adapter::check_config(cfg);
  if (st != MOE_OK) return st;
  if (cfg->rows == 0) return MOE_OK;   // (empty arrays may be NULL)
  if (x == nullptr || offsets == nullptr || W == nullptr || A == nullptr || B == nullptr || adapter == nullptr || y == nullptr ||
      v == nullptr || workspace == nullptr)
    return MOE_ERR_NULL;
  for (const void* p : {x, static_cast<const void*>(offsets), W, A, B, static_cast<const void*>(scale), static_cast<const void*>(adapter),
                        static_cast<const void*>(perm), static_cast<const void*>(y), static_cast<const void*>(v),
                        static_cast<const void*>(workspace)})
    if (adapter::misaligned(p)) return MOE_ERR_ALIGN;
  const adapter::Layout L = adapter::layout_of(*cfg, false);
  if (workspace_bytes < L.total) return MOE_ERR_WORKSPACE;
  const size_t n_rows = cfg->rows, pairs = static_cast<size_t>(cfg->n_exp) * cfg->n_adapters, k = cfg->K, n = cfg->N, r = cfg->rank;
  const adapter::Memory memory[] = {{y, n_rows * n * 2}, {v, n_rows * r * 4}, {workspace, L.total}, {x, n_rows * k * 2},
                                    {offsets, (cfg->n_exp + 1) * size_t(4)}, {W, cfg->n_exp * n * k * 2}, {A, pairs * r * k * 2},
                                    {B, pairs * n * r * 2}, {scale, cfg->n_adapters * size_t(4)},
                                    {adapter, adapter::bytes_of_adapter(*cfg, perm)}, {perm, n_rows * 4}};
  if (adapter::overlapping(memory, 3)) return MOE_ERR_OVERLAP;
  hipStream_t s = static_cast<hipStream_t>(stream);
  unsigned char* ws = static_cast<unsigned char*>(workspace);
  int32_t* of_row = reinterpret_cast<int32_t*>(ws + L.of_row);
  bf16_t* low = reinterpret_cast<bf16_t*>(ws + L.low);
  adapter::ShrinkArgs a = {static_cast<const bf16_t*>(x), static_cast<const bf16_t*>(A), offsets, adapter, perm, scale, of_row, v, low,
                           cfg->n_exp, cfg->n_adapters, cfg->top_k, cfg->K, cfg->rank, 0, false, nullptr, reinterpret_cast<float*>(ws + L.cut), 1, 0};
  hipError_t e = adapter::launch_shrink(cfg->dtype, a, cfg->rows, s);
  if (e != hipSuccess) return MOE_ERR_HIP;
  const AdapterRows rows = {of_row, low, v, scale, static_cast<const bf16_t*>(B), cfg->n_exp, cfg->rank};
  e = launch_grouped_gemm(cfg->dtype, cfg->activation == MOE_ACT_GELU, x, W, y, offsets, cfg->n_exp, cfg->rows, cfg->N, cfg->K,
                          ws + L.gemm, s, 0, nullptr, nullptr, 1, nullptr, nullptr, &rows);
  return e == hipSuccess ? MOE_OK : MOE_ERR_HIP;
}

int moe_adapter_backward(const moe_adapter_config* cfg, const void* x, const int32_t* offsets, const void* W, const void* A,
                         const void* B, const float* scale, const int32_t* adapter, const int32_t* perm, const void* dy,
                         const float* v, void* dx, float* dA, float* dB, void* workspace, size_t workspace_bytes, void* stream) {
  const int st = adapter::check_backward(cfg);
  if (st != MOE_OK) return st;
  if (offsets == nullptr || dA == nullptr || dB == nullptr || workspace == nullptr) return MOE_ERR_NULL;
  if (cfg->rows > 0 && (x == nullptr || W == nullptr || A == nullptr || B == nullptr || adapter == nullptr || dy == nullptr || v == nullptr))
    return MOE_ERR_NULL;
  for (const void* p : {x, static_cast<const void*>(offsets), W, A, B, static_cast<const void*>(scale), static_cast<const void*>(adapter),
                        static_cast<const void*>(perm), dy, static_cast<const void*>(v), static_cast<const void*>(dx),
                        static_cast<const void*>(dA), static_cast<const void*>(dB), static_cast<const void*>(workspace)})
    if (adapter::misaligned(p)) return MOE_ERR_ALIGN;
  const adapter::Layout L = adapter::layout_of(*cfg, true);
  if (workspace_bytes < L.total) return MOE_ERR_WORKSPACE;
  hipStream_t s = static_cast<hipStream_t>(stream);
  unsigned char* ws = static_cast<unsigned char*>(workspace);
  const int n_exp = cfg->n_exp, rank = cfg->rank, K = cfg->K, N = cfg->N;
  const int64_t pairs = static_cast<int64_t>(n_exp) * cfg->n_adapters;
  {
    const size_t n_rows = cfg->rows, k = K, n = N, a = pairs * rank * k, b = pairs * rank * n;
    const adapter::Memory memory[] = {{dx, n_rows * k * 2}, {dA, a * 4}, {dB, b * 4}, {workspace, L.total}, {x, n_rows * k * 2},
                                      {offsets, (n_exp + 1) * size_t(4)}, {W, n_exp * n * k * 2}, {A, a * 2}, {B, b * 2},
                                      {scale, cfg->n_adapters * size_t(4)}, {adapter, adapter::bytes_of_adapter(*cfg, perm)}, {perm, n_rows * 4},
                                      {dy, n_rows * n * 2}, {v, n_rows * rank * 4}};
    if (adapter::overlapping(memory, 4)) return MOE_ERR_OVERLAP;
  }
  int32_t* of_row = reinterpret_cast<int32_t*>(ws + L.of_row);
  bf16_t* low = reinterpret_cast<bf16_t*>(ws + L.low);
  float* t = reinterpret_cast<float*>(ws + L.t);
  bf16_t *At = reinterpret_cast<bf16_t*>(ws + L.At), *Bt = reinterpret_cast<bf16_t*>(ws + L.Bt);
  hipError_t e = hipSuccess;
  if (cfg->rows > 0) {
    // The contractions over what A and B have as their rows: t, and the low-rank part of dx.
    const adapter::Transpose tb = adapter::transpose_of(B, Bt, N, rank, pairs), ta = adapter::transpose_of(A, At, rank, K, pairs);
    const unsigned blocks_b = adapter::blocks_of(tb), blocks_a = dx != nullptr ? adapter::blocks_of(ta) : 0;
    adapter::transpose_kernel<<<blocks_b + blocks_a, 256, 0, s>>>(tb, ta, blocks_b);
    adapter::ShrinkArgs a = {static_cast<const bf16_t*>(dy), Bt, offsets, adapter, perm, scale, of_row, t, low,
                             n_exp, cfg->n_adapters, cfg->top_k, N, rank, 0, true, reinterpret_cast<int32_t*>(ws + L.ticket), reinterpret_cast<float*>(ws + L.cut), 1, 0};
    e = adapter::launch_shrink(cfg->dtype, a, cfg->rows, s);
    if (e != hipSuccess) return MOE_ERR_HIP;
    if (dx != nullptr) {
      const AdapterRows rows = {of_row, low, t, nullptr, At, n_exp, rank};
      e = launch_data_gradient(cfg->dtype, static_cast<const bf16_t*>(dy), static_cast<const bf16_t*>(W), static_cast<bf16_t*>(dx),
                               offsets, n_exp, cfg->rows, cfg->rows, K, N, ws + L.gemm, s, &rows);
      if (e != hipSuccess) return MOE_ERR_HIP;
    }
  }
  auto words = [&](size_t off) { return reinterpret_cast<int32_t*>(ws + off); };
  adapter::FinishArgs f = {};
  f.no_rows = cfg->rows == 0;
  adapter::BothGrads& b = f.b;
  b.g.begin = words(L.begin);
  b.g.list = words(L.list);
  b.g.ticket = words(L.ticket);
  b.pairs = static_cast<int>(pairs);
  b.n_exp = n_exp;
  b.rank = rank;
  int64_t blocks[2];
  for (int i = 0; i < 2; ++i) {
    const int C = i == 0 ? K : N;
    b.g.pieces[i] = {words(L.piece_begin[i]), words(L.slot[i]), words(L.piece_pair[i]), adapter::rows_of_piece(*cfg, C)};
    b.of[i] = {i == 0 ? t : v, i == 0 ? nullptr : scale, static_cast<const bf16_t*>(i == 0 ? x : dy), i == 0 ? dA : dB,
               reinterpret_cast<float*>(ws + L.partial[i]), b.g.pieces[i], C};
    blocks[i] = adapter::most_pieces(*cfg, C) * ((C + adapter::kGradColumns - 1) / adapter::kGradColumns);
    const int64_t quads = static_cast<int64_t>(rank) * C / 4;
    f.per_pair[i] = static_cast<int>(quads < 2048 ? 1 : quads / 1024 < 128 ? quads / 1024 : 128);
  }
  const unsigned n_pairs = static_cast<unsigned>(pairs);
  if (cfg->rows > 0) {
    b.blocks_a = static_cast<int>(blocks[0]);
    adapter::count_kernel<<<n_pairs, 256, 0, s>>>(of_row, offsets, n_exp, b.g, b.pairs);
    adapter::fill_kernel<<<n_pairs, 256, 0, s>>>(of_row, offsets, n_exp, b.g);
    e = cfg->dtype == MOE_F16 ? adapter::launch_gradients_of<MOE_F16>(b, blocks[0] + blocks[1], s)
                              : adapter::launch_gradients_of<MOE_BF16>(b, blocks[0] + blocks[1], s);
    if (e != hipSuccess) return MOE_ERR_HIP;
  }
  adapter::finish_kernel<<<n_pairs * (f.per_pair[0] + f.per_pair[1]), 256, 0, s>>>(f);
  return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_HIP;
}

}  // extern "C"
