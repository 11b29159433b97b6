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

#include <cmath>

#include "adapter_core.h"

namespace ppmoe {
namespace adapter {

constexpr int kMaxRank = 128;
constexpr int kMaxPairs = 1 << 16;   // adapters x experts
constexpr int kMaxColumns = 1 << 20;

// ---- x A^T: [rows, K] with a matrix [rank, K] of each row's own ------------------------------------------
//
// A block has up to 16 packed rows, its wavefronts split the contraction, fetch both operands of the matrix instruction
// from memory and meet in LDS, where the partial sums are added in wavefront order.  It goes through the distinct
// (adapter, expert) pairs of its rows; each takes the whole contraction and is kept for the rows it belongs to (a row of the
// operand never meets another one's).

struct ShrinkArgs {
  const bf16_t* x;        // [rows, K]
  const bf16_t* m;        // [n_adapters, n_exp, rank, K]
  const int32_t *offsets, *adapter, *perm;
  const float* scale;     // [n_adapters] or NULL
  int32_t* of_row;        // out: the adapter of each packed row, or -1
  float* wide;            // out [rows, rank]
  bf16_t* low;            // out [rows, rank]: scaled, in 16 bits
  int n_exp, n_adapters, top_k, K, rank, tile_rows;
  bool scale_wide;        // wide is scaled as well
};

template <int DT, int MR, int WAVES>   // MR: blocks of 16 of the rank
__global__ __launch_bounds__(64 * WAVES) void shrink_kernel(ShrinkArgs a) {
  typedef typename Elem16<DT>::vec8 vec8;
  __shared__ __attribute__((aligned(16))) float part[WAVES][16][16 * MR + 4];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int fr = lane & 15, fq = lane >> 4;
  const int lo = a.offsets[0], rows = a.offsets[a.n_exp] - lo;
  const int row0 = blockIdx.x * a.tile_rows;
  const int count = min(a.tile_rows, rows - row0);
  if (count <= 0) return;
  // this lane's row: its expert (the experts whose rows end at or before it), its adapter
  const int r = lo + row0 + min(fr, count - 1);
  int expert = 0;
  for (int i0 = 0; i0 < a.n_exp; i0 += 64) {
    const int end = a.offsets[min(i0 + lane, a.n_exp - 1) + 1];
    for (int q = 0; q < 16; ++q) {
      const int n = __popcll(__ballot(i0 + lane < a.n_exp && end <= __builtin_amdgcn_readlane(r, q)));
      if (fr == q) expert += n;
    }
  }
  int id = a.adapter[a.perm != nullptr ? a.perm[r] / a.top_k : r];
  if (id < 0 || id >= a.n_adapters) id = -1;
  if (wave == 0 && lane < count) a.of_row[r] = id;
  const int mine = id >= 0 && fr < count ? id * a.n_exp + expert : -1;

  const u32x4 zero = u32x4{0u, 0u, 0u, 0u};
  f32x4 kept[MR];
#pragma unroll
  for (int mr = 0; mr < MR; ++mr) kept[mr] = f32x4{0.f, 0.f, 0.f, 0.f};
  const bf16_t* xr = a.x + static_cast<int64_t>(r) * a.K + fq * 8;
  int pair = -1;
  while (true) {
    int least = mine > pair ? mine : 0x7fffffff;
#pragma unroll
    for (int off = 8; off >= 1; off >>= 1) least = min(least, __shfl_xor(least, off, 64));
    pair = __builtin_amdgcn_readfirstlane(least);
    if (pair == 0x7fffffff) break;
    const bf16_t* m = a.m + static_cast<int64_t>(pair) * a.rank * a.K + fq * 8;
    f32x4 acc[MR];
#pragma unroll
    for (int mr = 0; mr < MR; ++mr) acc[mr] = f32x4{0.f, 0.f, 0.f, 0.f};
    constexpr int J = MR <= 2 ? 4 : 2;   // k-steps of 32 fetched at a time
    for (int k0 = wave * 32 * J; k0 < a.K; k0 += WAVES * 32 * J) {
      u32x4 x[J], w[J][MR];
#pragma unroll
      for (int j = 0; j < J; ++j) {
        const int k = k0 + 32 * j;
        const bool ok = k + fq * 8 < a.K;
        x[j] = ok ? *reinterpret_cast<const u32x4*>(xr + k) : zero;
#pragma unroll
        for (int mr = 0; mr < MR; ++mr)   // (rows past the rank re-read the last one; their sums are not stored)
          w[j][mr] = ok ? *reinterpret_cast<const u32x4*>(m + static_cast<int64_t>(min(mr * 16 + fr, a.rank - 1)) * a.K + k) : zero;
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int j = 0; j < J; ++j)
#pragma unroll
        for (int mr = 0; mr < MR; ++mr)
          acc[mr] = Elem16<DT>::mfma16(__builtin_bit_cast(vec8, w[j][mr]), __builtin_bit_cast(vec8, x[j]), acc[mr]);
    }
    // D: lane row fr, rank index mr * 16 + fq * 4 + v
#pragma unroll
    for (int mr = 0; mr < MR; ++mr)
      if (mine == pair) kept[mr] = acc[mr];
  }
#pragma unroll
  for (int mr = 0; mr < MR; ++mr) *reinterpret_cast<f32x4*>(&part[wave][fr][mr * 16 + fq * 4]) = kept[mr];
  __syncthreads();
  for (int p = threadIdx.x; p < count * (a.rank / 4); p += 64 * WAVES) {
    const int q = p / (a.rank / 4), j = (p - q * (a.rank / 4)) * 4;
    f32x4 v = *reinterpret_cast<const f32x4*>(&part[0][q][j]);
#pragma unroll
    for (int w = 1; w < WAVES; ++w) v += *reinterpret_cast<const f32x4*>(&part[w][q][j]);
    const int row = lo + row0 + q;
    int whose = a.adapter[a.perm != nullptr ? a.perm[row] / a.top_k : row];
    if (whose < 0 || whose >= a.n_adapters) whose = -1;
    const float s = whose < 0 || a.scale == nullptr ? 1.f : a.scale[whose];
    const f32x4 scaled = v * s;
    *reinterpret_cast<f32x4*>(a.wide + static_cast<int64_t>(row) * a.rank + j) = a.scale_wide ? scaled : v;
    // (16 bits: an operand of the matrix instruction that adds the low-rank part.  A rounding of each of `rank` terms, as
    // far off as the one rounding of the result is, and only of the low-rank part.)
    const u32x2 o = {Elem16<DT>::pack2(scaled[0], scaled[1]), Elem16<DT>::pack2(scaled[2], scaled[3])};
    *reinterpret_cast<u32x2*>(a.low + static_cast<int64_t>(row) * a.rank + j) = o;
  }
}

// ---- [batch, R, C] -> [batch, C, R], 16-bit, both multiples of 8 ----------------------------------------
__global__ __launch_bounds__(256) void transpose_kernel(const bf16_t* __restrict__ in, bf16_t* __restrict__ out, int R, int C,
                                                        int r_tiles, int c_tiles) {
  __shared__ uint16_t tile[64][66];
  const int64_t per = static_cast<int64_t>(r_tiles) * c_tiles, batch = blockIdx.x / per;
  const int t = static_cast<int>(blockIdx.x - batch * per);
  const int r0 = (t / c_tiles) * 64, c0 = (t % c_tiles) * 64;
  const bf16_t* src = in + batch * R * C;
  bf16_t* dst = out + batch * R * C;
  for (int p = threadIdx.x; p < 64 * 8; p += 256) {
    const int r = p >> 3, c = (p & 7) * 8;
    if (r0 + r < R && c0 + c < C) {
      const u32x4 v = *reinterpret_cast<const u32x4*>(src + static_cast<int64_t>(r0 + r) * C + c0 + c);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        tile[r][c + 2 * q] = static_cast<uint16_t>(v[q]);
        tile[r][c + 2 * q + 1] = static_cast<uint16_t>(v[q] >> 16);
      }
    }
  }
  __syncthreads();
  for (int p = threadIdx.x; p < 64 * 8; p += 256) {
    const int c = p >> 3, r = (p & 7) * 8;
    if (c0 + c < C && r0 + r < R) {
      u32x4 v;
#pragma unroll
      for (int q = 0; q < 4; ++q) v[q] = tile[r + 2 * q][c] | (static_cast<uint32_t>(tile[r + 2 * q + 1][c]) << 16);
      *reinterpret_cast<u32x4*>(dst + static_cast<int64_t>(c0 + c) * R + r0 + r) = v;
    }
  }
}

// ---- the rows of each (adapter, expert) pair -----------------------------------------------------------
//
// list: the packed rows ordered by pair (adapter-major, as dA and dB are), ascending inside it; begin[pair] where they start.
// A pair's rows are cut into pieces of at most `most` for the gradients; a pair of several pieces has a slot of partial sums
// for each.  Counted, scanned, filled: no atomics, the same order on every run.
struct Groups {
  int32_t *begin;         // [pairs + 1]
  int32_t *piece_begin;   // [pairs + 1]
  int32_t *slot_begin;    // [pairs + 1]
  int32_t *piece_pair;    // [most pieces]
  int32_t *list;          // [rows]
};

__device__ __forceinline__ int sum_of_block(int v, int* lds) {   // 256 threads
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) v += __shfl_xor(v, off, 64);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  return lds[0] + lds[1] + lds[2] + lds[3];
}

__global__ __launch_bounds__(256) void count_kernel(const int32_t* __restrict__ of_row, const int32_t* __restrict__ offsets, int n_exp,
                                                    int32_t* __restrict__ count) {
  __shared__ int lds[4];
  const int id = blockIdx.x / n_exp, expert = blockIdx.x - id * n_exp;
  int n = 0;
  for (int r = offsets[expert] + threadIdx.x; r < offsets[expert + 1]; r += 256) n += of_row[r] == id;
  n = sum_of_block(n, lds);
  if (threadIdx.x == 0) count[blockIdx.x] = n;
}

// One block of 1024 threads; count[] is begin[] (overwritten).
__global__ __launch_bounds__(1024) void scan_kernel(Groups g, int pairs, int most) {
  __shared__ int sums[3][16];
  int before[3] = {0, 0, 0};
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int p0 = 0; p0 < pairs; p0 += 1024) {
    const int p = p0 + threadIdx.x;
    const int n = p < pairs ? g.begin[p] : 0;
    const int pieces = (n + most - 1) / most;
    int own[3] = {n, pieces, pieces > 1 ? pieces : 0}, up_to[3];
#pragma unroll
    for (int q = 0; q < 3; ++q) {
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
    int total[3];
#pragma unroll
    for (int q = 0; q < 3; ++q) {
      int base = 0;
      total[q] = 0;
      for (int w = 0; w < 16; ++w) {
        if (w < wave) base += sums[q][w];
        total[q] += sums[q][w];
      }
      up_to[q] += base + before[q] - own[q];
    }
    if (p < pairs) {
      g.begin[p] = up_to[0];
      g.piece_begin[p] = up_to[1];
      g.slot_begin[p] = up_to[2];
    }
#pragma unroll
    for (int q = 0; q < 3; ++q) before[q] += total[q];
    __syncthreads();
  }
  if (threadIdx.x == 0) {
    g.begin[pairs] = before[0];
    g.piece_begin[pairs] = before[1];
    g.slot_begin[pairs] = before[2];
  }
}

__global__ __launch_bounds__(256) void fill_kernel(const int32_t* __restrict__ of_row, const int32_t* __restrict__ offsets, int n_exp, Groups g) {
  __shared__ int lds[4];
  const int pair = blockIdx.x, id = pair / n_exp, expert = pair - id * n_exp;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int at = g.begin[pair];
  if (at == g.begin[pair + 1]) return;
  const int p0 = g.piece_begin[pair], p1 = g.piece_begin[pair + 1];
  for (int p = p0 + threadIdx.x; p < p1; p += 256) g.piece_pair[p] = pair;
  const int end = offsets[expert + 1];
  for (int r0 = offsets[expert]; r0 < end; r0 += 256) {
    const int r = r0 + threadIdx.x;
    const bool is = r < end && of_row[r] == id;
    const uint64_t lanes = __ballot(is);
    __syncthreads();
    if (lane == 0) lds[wave] = __popcll(lanes);
    __syncthreads();
    int base = at;
    for (int w = 0; w < wave; ++w) base += lds[w];
    if (is) g.list[base + __popcll(lanes & ((uint64_t(1) << lane) - 1))] = r;
    at += lds[0] + lds[1] + lds[2] + lds[3];
  }
}

// ---- G[pair][j, c] = sum over the pair's rows of s u[r, j] z[r, c] ------------------------------------------
//
// u [rows, rank] float32 (t, or v), z [rows, C] 16-bit (x, or dy).  BY_COLUMN: stored [C, rank] (dB), else [rank, C] (dA).
// A block takes one piece of a pair's rows and 256 columns, 32 rows at a time: z as it is into LDS and from there
// across its rows into operands (transposing read), u as two 16-bit summands (what the first one's rounding leaves, rounded
// again: 16 or 22 bits together), so that the products keep float32's accuracy as far as the result shows it.  fp16: u is first brought
// to a largest value of 2^13 by a power of two, exactly, as its small values have no 22 bits.
constexpr int kGradColumns = 256, kGradThreads = 256, kGradRows = 32;
constexpr int kLowStride = kGradRows * 2 + 16;   // bytes of a row of u's halves in LDS

struct GradArgs {
  const float* u;
  const float* scale;           // by adapter, or NULL
  const bf16_t* z;
  float *out, *partial;         // [pairs, rank * C], [slots, rank * C]
  Groups g;
  int pairs, n_exp, rank, C, most;
};

template <int DT, int MR, bool BY_COLUMN>
__global__ __launch_bounds__(kGradThreads) void gradient_kernel(GradArgs a) {
  typedef typename Elem16<DT>::vec8 vec8;
  __shared__ __attribute__((aligned(16))) unsigned char z_lds[kGradRows * kGradColumns * 2];
  __shared__ __attribute__((aligned(16))) unsigned char u_lds[2][16 * MR * kLowStride];
  __shared__ float wave_top[4];
  const int col_blocks = (a.C + kGradColumns - 1) / kGradColumns;
  const int piece = blockIdx.x / col_blocks, col0 = (blockIdx.x - piece * col_blocks) * kGradColumns;
  if (piece >= a.g.piece_begin[a.pairs]) return;
  const int pair = a.g.piece_pair[piece];
  const int nth = piece - a.g.piece_begin[pair], pieces = a.g.piece_begin[pair + 1] - a.g.piece_begin[pair];
  const int first = a.g.begin[pair] + nth * a.most, count = min(a.most, a.g.begin[pair + 1] - first);
  const int32_t* list = a.g.list + first;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int fr = lane & 15, fq = lane >> 4;
  const float s = a.scale != nullptr ? a.scale[pair / a.n_exp] : 1.f;
  const int quads = a.rank / 4;   // of a row of u

  float up = 1.f, down = 1.f;
  if (DT == MOE_F16) {
    float top = 0.f;
    for (int p = tid; p < count * quads; p += kGradThreads) {
      const int q = p / quads;
      const f32x4 v = *reinterpret_cast<const f32x4*>(a.u + static_cast<int64_t>(list[q]) * a.rank + (p - q * quads) * 4);
#pragma unroll
      for (int e = 0; e < 4; ++e) top = fmaxf(top, fabsf(v[e] * s));
    }
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) top = fmaxf(top, __shfl_xor(top, off, 64));
    if (lane == 0) wave_top[wave] = top;
    __syncthreads();
    top = fmaxf(fmaxf(wave_top[0], wave_top[1]), fmaxf(wave_top[2], wave_top[3]));
    const int e = static_cast<int>(__float_as_uint(top) >> 23) - 127;
    if (e > -110 && e < 128) {   // (zeros, and what is beyond any use, as they are; infinities too)
      up = __uint_as_float(static_cast<uint32_t>(127 + 13 - e) << 23);
      down = __uint_as_float(static_cast<uint32_t>(127 - 13 + e) << 23);
    }
  }

  // staging: z in 1024 pieces of 16 bytes, four per thread (row p / 32, piece p % 32); u in quads
  u32x4 zv[4];
  constexpr int kQuads = (16 * MR * kGradRows / 4 + kGradThreads - 1) / kGradThreads;
  f32x4 uv[kQuads];
  auto load = [&](int k0) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int p = tid + i * kGradThreads, row = k0 + (p >> 5), c = col0 + (p & 31) * 8;
      zv[i] = row < count && c < a.C ? *reinterpret_cast<const u32x4*>(a.z + static_cast<int64_t>(list[row]) * a.C + c) : u32x4{0u, 0u, 0u, 0u};
    }
#pragma unroll
    for (int i = 0; i < kQuads; ++i) {
      const int p = tid + i * kGradThreads, q = p & (kGradRows - 1), j = (p / kGradRows) * 4, row = k0 + q;
      uv[i] = row < count && j < a.rank ? *reinterpret_cast<const f32x4*>(a.u + static_cast<int64_t>(list[row]) * a.rank + j) : f32x4{0.f, 0.f, 0.f, 0.f};
    }
  };
  // 32-byte block b of row k at b ^ ((k & 3) + 4 ((k >> 3) & 1)): what 32 lanes of a transposing read touch falls on all banks
  auto store = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int p = tid + i * kGradThreads, k = p >> 5, c = p & 31;
      const int block = (c >> 1) ^ ((k & 3) + 4 * ((k >> 3) & 1));
      *reinterpret_cast<u32x4*>(z_lds + k * (kGradColumns * 2) + block * 32 + (c & 1) * 16) = zv[i];
    }
#pragma unroll
    for (int i = 0; i < kQuads; ++i) {
      const int p = tid + i * kGradThreads, q = p & (kGradRows - 1), j = (p / kGradRows) * 4;
      if (j < 16 * MR) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float v = uv[i][e] * s * up;
          const uint16_t hi = static_cast<uint16_t>(Elem16<DT>::pack2(v, 0.f));
          const float rest = v - Elem16<DT>::widen(hi);
          // (an infinite or NaN v: the rest is NaN or 0 * ..., and the sum is what it has to be with the rest left out)
          const uint16_t lo = static_cast<uint16_t>(Elem16<DT>::pack2(fabsf(rest) < 3.0e38f ? rest : 0.f, 0.f));
          *reinterpret_cast<uint16_t*>(u_lds[0] + (j + e) * kLowStride + q * 2) = hi;
          *reinterpret_cast<uint16_t*>(u_lds[1] + (j + e) * kLowStride + q * 2) = lo;
        }
      }
    }
  };

  f32x4 acc[MR][4];
#pragma unroll
  for (int mr = 0; mr < MR; ++mr)
#pragma unroll
    for (int ni = 0; ni < 4; ++ni) acc[mr][ni] = f32x4{0.f, 0.f, 0.f, 0.f};
  const uint32_t z0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((const __attribute__((address_space(3))) unsigned char*)z_lds));
  load(0);
  for (int k0 = 0; k0 < count; k0 += kGradRows) {
    __syncthreads();
    store();
    __syncthreads();
    if (k0 + kGradRows < count) load(k0 + kGradRows);
    u32x2 zt[4][2];
    const int j = (lane >> 2) & 3;
#pragma unroll
    for (int ni = 0; ni < 4; ++ni) {
      const uint32_t at = z0 + (fq * 8 + j) * (kGradColumns * 2) + (((wave * 4 + ni) ^ (j + 4 * (fq & 1))) << 5) + (lane & 3) * 8;
      asm volatile("ds_read_b64_tr_b16 %0, %2\n\tds_read_b64_tr_b16 %1, %2 offset:2048"
                   : "=&v"(zt[ni][0]), "=&v"(zt[ni][1]) : "v"(at) : "memory");
    }
    vec8 uh[MR], ul[MR];
#pragma unroll
    for (int mr = 0; mr < MR; ++mr) {
      uh[mr] = *reinterpret_cast<const vec8*>(u_lds[0] + (mr * 16 + fr) * kLowStride + fq * 16);
      ul[mr] = *reinterpret_cast<const vec8*>(u_lds[1] + (mr * 16 + fr) * kLowStride + fq * 16);
    }
    asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(zt[0][0]), "+v"(zt[0][1]), "+v"(zt[1][0]), "+v"(zt[1][1]), "+v"(zt[2][0]), "+v"(zt[2][1]),
                 "+v"(zt[3][0]), "+v"(zt[3][1]) : : "memory");
#pragma unroll
    for (int ni = 0; ni < 4; ++ni) {
      const vec8 z = __builtin_bit_cast(vec8, __builtin_shufflevector(zt[ni][0], zt[ni][1], 0, 1, 2, 3));
#pragma unroll
      for (int mr = 0; mr < MR; ++mr) {
        // D: lane: index of the second operand, registers: 4 (lane / 16) + v of the first
        if (BY_COLUMN) {
          acc[mr][ni] = Elem16<DT>::mfma16(uh[mr], z, acc[mr][ni]);
          acc[mr][ni] = Elem16<DT>::mfma16(ul[mr], z, acc[mr][ni]);
        } else {
          acc[mr][ni] = Elem16<DT>::mfma16(z, uh[mr], acc[mr][ni]);
          acc[mr][ni] = Elem16<DT>::mfma16(z, ul[mr], acc[mr][ni]);
        }
      }
    }
  }
  const int64_t size = static_cast<int64_t>(a.rank) * a.C;
  float* out = pieces > 1 ? a.partial + (a.g.slot_begin[pair] + nth) * size : a.out + pair * size;
#pragma unroll
  for (int ni = 0; ni < 4; ++ni)
#pragma unroll
    for (int mr = 0; mr < MR; ++mr) {
      const int c = col0 + wave * 64 + ni * 16 + (BY_COLUMN ? fr : fq * 4), jj = mr * 16 + (BY_COLUMN ? fq * 4 : fr);
      if (c < a.C && jj < a.rank)
        *reinterpret_cast<f32x4*>(out + (BY_COLUMN ? static_cast<int64_t>(c) * a.rank + jj : static_cast<int64_t>(jj) * a.C + c)) =
            acc[mr][ni] * down;
    }
}

// Pairs without rows: zeros; of several pieces: the partial sums in order.
__global__ __launch_bounds__(256) void finish_kernel(GradArgs a, int per_pair) {
  const int pair = blockIdx.x / per_pair, part = blockIdx.x - pair * per_pair;
  const int slot = a.g.slot_begin[pair], slots = a.g.slot_begin[pair + 1] - slot;
  if (slots == 0 && a.g.begin[pair + 1] > a.g.begin[pair]) return;   // written already
  const int64_t quads = static_cast<int64_t>(a.rank) * a.C / 4;
  f32x4* out = reinterpret_cast<f32x4*>(a.out) + pair * quads;
  const f32x4* in = reinterpret_cast<const f32x4*>(a.partial) + slot * quads;
  for (int64_t q = static_cast<int64_t>(part) * 256 + threadIdx.x; q < quads; q += static_cast<int64_t>(per_pair) * 256) {
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    for (int k = 0; k < slots; ++k) v += in[k * quads + q];
    out[q] = v;
  }
}

// ---- host ----------------------------------------------------------------------------------------

inline size_t align_up(size_t v) { return (v + 255) / 256 * 256; }
inline bool misaligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }

int check_config(const moe_adapter_config* c) {
  if (c == nullptr) return MOE_ERR_NULL;
  if (c->rows < 0 || c->K <= 0 || c->N <= 0 || (c->K & 7) || (c->N & 7) || c->K > kMaxColumns || c->N > kMaxColumns) return MOE_ERR_SHAPE;
  if (c->n_exp < 1 || c->n_exp > kMaxExperts || c->n_adapters < 1 || c->n_adapters > kMaxPairs / c->n_exp) return MOE_ERR_SHAPE;
  if (c->rank < 8 || c->rank > kMaxRank || (c->rank & 7) || c->top_k < 1 || c->top_k > kMaxTopK) return MOE_ERR_SHAPE;
  if (!is_16bit(c->dtype)) return MOE_ERR_DTYPE;
  if (c->activation != MOE_ACT_NONE && c->activation != MOE_ACT_GELU) return MOE_ERR_SHAPE;
  return MOE_OK;
}

// Rows of a piece of the gradients: at least 256, so that a launch has some 32 pieces at most per pair that has all the rows.
int rows_of_piece(const moe_adapter_config& c) {
  const int64_t n = ((static_cast<int64_t>(c.rows) + 31) / 32 + kGradRows - 1) / kGradRows * kGradRows;
  return static_cast<int>(n < 256 ? 256 : n);
}
int64_t most_pieces(const moe_adapter_config& c) {
  const int64_t pairs = static_cast<int64_t>(c.n_exp) * c.n_adapters;
  return c.rows / rows_of_piece(c) + 1 + (pairs < c.rows ? pairs : c.rows);
}
// A pair of several pieces has more rows than one piece: at most two slots per full piece.
int64_t most_slots(const moe_adapter_config& c) { return 2 * (static_cast<int64_t>(c.rows) / rows_of_piece(c)) + 1; }

struct Layout {
  size_t of_row, low, gemm, total;                                                        // forward and backward
  size_t t, At, Bt, begin, piece_begin, slot_begin, piece_pair, list, partial_a, partial_b;   // backward
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
  L.low = take(rows * c.rank * 2);
  L.gemm = take(grouped_gemm_workspace_bytes());
  if (backward) {
    L.t = take(rows * c.rank * 4);
    L.At = take(pairs * c.rank * c.K * 2);
    L.Bt = take(pairs * c.rank * c.N * 2);
    L.begin = take((pairs + 1) * 4);
    L.piece_begin = take((pairs + 1) * 4);
    L.slot_begin = take((pairs + 1) * 4);
    L.piece_pair = take(most_pieces(c) * 4);
    L.list = take(rows * 4);
    L.partial_a = take(most_slots(c) * c.rank * c.K * 4);
    L.partial_b = take(most_slots(c) * c.rank * c.N * 4);
  }
  L.total = off;
  return L;
}

template <int DT>
hipError_t launch_shrink_of(const ShrinkArgs& a, int64_t rows, hipStream_t s) {
  const unsigned grid = static_cast<unsigned>((rows + a.tile_rows - 1) / a.tile_rows);
  if (a.rank <= 16) shrink_kernel<DT, 1, 8><<<grid, 512, 0, s>>>(a);
  else if (a.rank <= 32) shrink_kernel<DT, 2, 8><<<grid, 512, 0, s>>>(a);
  else if (a.rank <= 64) shrink_kernel<DT, 4, 8><<<grid, 512, 0, s>>>(a);
  else shrink_kernel<DT, 8, 4><<<grid, 256, 0, s>>>(a);   // (the partial sums' place in LDS)
  return hipGetLastError();
}
// Blocks of 16 rows, or of fewer while that leaves CUs without one (a row's own adapter is a block's whole work then).
hipError_t launch_shrink(int dtype, ShrinkArgs a, int64_t rows, hipStream_t s) {
  a.tile_rows = 16;
  while (a.tile_rows > 1 && (rows + a.tile_rows / 2 - 1) / (a.tile_rows / 2) <= 256) a.tile_rows /= 2;
  return dtype == MOE_F16 ? launch_shrink_of<MOE_F16>(a, rows, s) : launch_shrink_of<MOE_BF16>(a, rows, s);
}

hipError_t launch_transpose(const void* in, void* out, int64_t batch, int R, int C, hipStream_t s) {
  const int rt = (R + 63) / 64, ct = (C + 63) / 64;
  transpose_kernel<<<static_cast<unsigned>(batch * rt * ct), 256, 0, s>>>(static_cast<const bf16_t*>(in), static_cast<bf16_t*>(out), R, C, rt, ct);
  return hipGetLastError();
}

template <int DT, bool BY_COLUMN>
hipError_t launch_gradient_of(const GradArgs& a, int64_t pieces, int64_t pairs, hipStream_t s) {
  const unsigned grid = static_cast<unsigned>(pieces * ((a.C + kGradColumns - 1) / kGradColumns));
  if (a.rank <= 16) gradient_kernel<DT, 1, BY_COLUMN><<<grid, kGradThreads, 0, s>>>(a);
  else if (a.rank <= 32) gradient_kernel<DT, 2, BY_COLUMN><<<grid, kGradThreads, 0, s>>>(a);
  else if (a.rank <= 64) gradient_kernel<DT, 4, BY_COLUMN><<<grid, kGradThreads, 0, s>>>(a);
  else gradient_kernel<DT, 8, BY_COLUMN><<<grid, kGradThreads, 0, s>>>(a);
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
  return adapter::check_config(cfg) == MOE_OK && cfg->activation == MOE_ACT_NONE ? adapter::layout_of(*cfg, true).total : 0;
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
  hipStream_t s = static_cast<hipStream_t>(stream);
  unsigned char* ws = static_cast<unsigned char*>(workspace);
  int32_t* of_row = reinterpret_cast<int32_t*>(ws + L.of_row);
  bf16_t* low = reinterpret_cast<bf16_t*>(ws + L.low);
  adapter::ShrinkArgs a = {static_cast<const bf16_t*>(x), static_cast<const bf16_t*>(A), offsets, adapter, perm, scale, of_row, v, low,
                           cfg->n_exp, cfg->n_adapters, cfg->top_k, cfg->K, cfg->rank, 0, false};
  hipError_t e = adapter::launch_shrink(cfg->dtype, a, cfg->rows, s);
  if (e != hipSuccess) return MOE_ERR_HIP;
  const AdapterRows rows = {of_row, low, static_cast<const bf16_t*>(B), cfg->n_exp, cfg->rank};
  e = launch_grouped_gemm(cfg->dtype, cfg->activation == MOE_ACT_GELU, x, W, y, offsets, cfg->n_exp, cfg->rows, cfg->N, cfg->K,
                          ws + L.gemm, s, 0, nullptr, nullptr, 1, nullptr, nullptr, &rows);
  return e == hipSuccess ? MOE_OK : MOE_ERR_HIP;
}

int moe_adapter_backward(const moe_adapter_config* cfg, const void* x, const int32_t* offsets, const void* W, const void* A,
                         const void* B, const float* scale, const int32_t* adapter, const int32_t* perm, const void* dy,
                         const float* v, void* dx, float* dA, float* dB, void* workspace, size_t workspace_bytes, void* stream) {
  const int st = adapter::check_config(cfg);
  if (st != MOE_OK) return st;
  if (cfg->activation != MOE_ACT_NONE) return MOE_ERR_SHAPE;
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
  int32_t* of_row = reinterpret_cast<int32_t*>(ws + L.of_row);
  bf16_t* low = reinterpret_cast<bf16_t*>(ws + L.low);
  float* t = reinterpret_cast<float*>(ws + L.t);
  bf16_t *At = reinterpret_cast<bf16_t*>(ws + L.At), *Bt = reinterpret_cast<bf16_t*>(ws + L.Bt);
  hipError_t e = hipSuccess;
  if (cfg->rows > 0) {
    // t, of the contraction over N that B has as its rows
    e = adapter::launch_transpose(B, Bt, pairs, N, rank, s);
    if (e != hipSuccess) return MOE_ERR_HIP;
    adapter::ShrinkArgs a = {static_cast<const bf16_t*>(dy), Bt, offsets, adapter, perm, scale, of_row, t, low,
                             n_exp, cfg->n_adapters, cfg->top_k, N, rank, 0, true};
    e = adapter::launch_shrink(cfg->dtype, a, cfg->rows, s);
    if (e != hipSuccess) return MOE_ERR_HIP;
    if (dx != nullptr) {
      e = adapter::launch_transpose(A, At, pairs, rank, K, s);
      if (e != hipSuccess) return MOE_ERR_HIP;
      const AdapterRows rows = {of_row, low, At, n_exp, rank};
      e = launch_data_gradient(cfg->dtype, static_cast<const bf16_t*>(dy), static_cast<const bf16_t*>(W), static_cast<bf16_t*>(dx),
                               offsets, n_exp, cfg->rows, cfg->rows, K, N, ws + L.gemm, s, &rows);
      if (e != hipSuccess) return MOE_ERR_HIP;
    }
  }
  adapter::Groups g = {reinterpret_cast<int32_t*>(ws + L.begin), reinterpret_cast<int32_t*>(ws + L.piece_begin),
                       reinterpret_cast<int32_t*>(ws + L.slot_begin), reinterpret_cast<int32_t*>(ws + L.piece_pair),
                       reinterpret_cast<int32_t*>(ws + L.list)};
  const int most = adapter::rows_of_piece(*cfg);
  const unsigned n_pairs = static_cast<unsigned>(pairs);
  adapter::count_kernel<<<n_pairs, 256, 0, s>>>(of_row, offsets, n_exp, g.begin);
  adapter::scan_kernel<<<1, 1024, 0, s>>>(g, static_cast<int>(pairs), most);
  adapter::fill_kernel<<<n_pairs, 256, 0, s>>>(of_row, offsets, n_exp, g);
  adapter::GradArgs ga = {t, nullptr, static_cast<const bf16_t*>(x), dA, reinterpret_cast<float*>(ws + L.partial_a), g,
                          static_cast<int>(pairs), n_exp, rank, K, most};
  adapter::GradArgs gb = {v, scale, static_cast<const bf16_t*>(dy), dB, reinterpret_cast<float*>(ws + L.partial_b), g,
                          static_cast<int>(pairs), n_exp, rank, N, most};
  if (cfg->rows > 0) {
    const int64_t pieces = adapter::most_pieces(*cfg);
    if (cfg->dtype == MOE_F16) {
      e = adapter::launch_gradient_of<MOE_F16, false>(ga, pieces, pairs, s);
      if (e == hipSuccess) e = adapter::launch_gradient_of<MOE_F16, true>(gb, pieces, pairs, s);
    } else {
      e = adapter::launch_gradient_of<MOE_BF16, false>(ga, pieces, pairs, s);
      if (e == hipSuccess) e = adapter::launch_gradient_of<MOE_BF16, true>(gb, pieces, pairs, s);
    }
    if (e != hipSuccess) return MOE_ERR_HIP;
  }
  for (const adapter::GradArgs& q : {ga, gb}) {
    const int64_t quads = static_cast<int64_t>(rank) * q.C / 4;
    const int per_pair = static_cast<int>(quads < 1024 ? 1 : quads / 1024 < 64 ? quads / 1024 : 64);
    adapter::finish_kernel<<<n_pairs * per_pair, 256, 0, s>>>(q, per_pair);
  }
  return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_HIP;
}

}  // extern "C"
