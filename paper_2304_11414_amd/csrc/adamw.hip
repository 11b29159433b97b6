// One AdamW step over many tensors (the paper trains with Adam, float32 master weights and moments, Section 4.1):
//
//   g = grad * grad_scale,   m' = b1 m + (1 - b1) g,   v' = b2 v + (1 - b2) g^2,
//   p' = p (1 - lr wd) - lr / (1 - b1^t) * m' / (sqrt(v') / sqrt(1 - b2^t) + eps),   half = p' in 16 bits.
//
// Every element is read once and written once, so the memory bounds it: 30 bytes per element with float32 moments, 18.1 with
// 8-bit ones.  All tensors are one launch: a block takes one chunk of kChunk elements of one tensor, and the plan tells which.  A
// thread's loads all go out before its first product (16 of 16 bytes; with 8-bit moments 8 of 16, 4 of 8 and 4 of one).  Measured: two tensors of
// 127 million elements together 712 us (5.4 TB/s; a copy of 4.3 GB reaches 4.8) and 427 us (5.4 TB/s) with 8-bit moments; 96 tensors of 1000 to
// 300 000, 5 million elements, 29 and 24 us.
//
// 8-bit moments.  32 consecutive elements of a tensor share a power of two, each is an e4m3 code (the OCP microscaling
// format): m as it is, v as its square root, which halves the range of exponents to cover and is what the update divides by.
// Rounding to nearest would freeze v: with b2 = 0.999 a step moves the root by 0.05 %, neighbouring codes are 6 to 12 % apart.  So a
// value is rounded up when the part of a code step it exceeds the lower code by and a phase in [0, 1) add up to one, the
// phase advancing by the golden ratio from step to step (a Weyl sequence, evenly spread over any run of steps) from a start that
// differs by element: the mean over the steps is right, the error at any one of them below one code step.  A value on a
// code stays there.  No root is rounded to zero (its element's next update would divide by eps alone).
//
// The arithmetic is float32, in the order written above, without contraction to fused multiply-adds: a program that follows it operation by
// operation gets the same bits, codes included.

#include <algorithm>
#include <cmath>
#include <cstring>
#include <vector>

#include "common.h"

#pragma clang fp contract(off)

namespace ppmoe {
namespace adamw {

constexpr int kThreads = 256;
constexpr int kChunk = 4096;      // elements of a block
constexpr int kBlock = 32;        // elements that share a power of two
constexpr int kLowestPower = -100;

// What the plan holds per tensor, and behind the tensors one tensor index per chunk.
struct Entry {
  float* p;
  const float* g;
  void *m, *v;
  uint8_t *m_power, *v_power;   // NULL with float32 moments
  uint16_t* half;
  int64_t n;
  int32_t first_chunk, half_dtype;
  float lr_scale, weight_decay;
};
static_assert(sizeof(Entry) == 80, "the plan's layout");

struct Hyper {
  double beta1, beta2;
  float eps;
};

// b^n, n >= 0
__device__ __forceinline__ double int_power(double b, uint32_t n) {
  double r = 1.0;
  for (; n != 0; n >>= 1) {
    if (n & 1) r *= b;
    b *= b;
  }
  return r;
}

// What is the same for all elements of a tensor.
struct Step {
  float b1, omb1, b2, omb2, grad_scale, decay, size, root_scale, eps;
  uint32_t phase;
};
__device__ __forceinline__ Step step_of(const Hyper& h, const moe_adamw_values& s, const Entry& e) {
  const uint32_t t = s.step < 1 ? 1 : s.step;
  const double lr = static_cast<double>(s.lr) * e.lr_scale;
  Step st;
  st.b1 = static_cast<float>(h.beta1);
  st.omb1 = static_cast<float>(1.0 - h.beta1);
  st.b2 = static_cast<float>(h.beta2);
  st.omb2 = static_cast<float>(1.0 - h.beta2);
  st.grad_scale = s.grad_scale;
  st.decay = static_cast<float>(1.0 - lr * e.weight_decay);
  st.size = static_cast<float>(lr / (1.0 - int_power(h.beta1, t)));
  st.root_scale = static_cast<float>(1.0 / sqrt(1.0 - int_power(h.beta2, t)));
  st.eps = h.eps;
  st.phase = t * 0x9E3779B9u;
  return st;
}

__device__ __forceinline__ float updated(const Step& st, float p, float m, float root) {
  const float denominator = root * st.root_scale + st.eps;
  return p * st.decay - st.size * m / denominator;
}

__device__ __forceinline__ uint32_t pack_half(int dtype, float lo, float hi) {
  return dtype == MOE_F16 ? Elem16<MOE_F16>::pack2(lo, hi) : Elem16<MOE_BF16>::pack2(lo, hi);
}

// Four elements from element i on; elements at or beyond n read zero and are not written.
__device__ __forceinline__ f32x4 load4(const float* a, int64_t i, int64_t n) {
  if (i + 4 <= n) return *reinterpret_cast<const f32x4*>(a + i);
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (i + j < n) v[j] = a[i + j];
  return v;
}
__device__ __forceinline__ void store4(float* a, int64_t i, int64_t n, f32x4 v) {
  if (i + 4 <= n) {
    *reinterpret_cast<f32x4*>(a + i) = v;
    return;
  }
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (i + j < n) a[i + j] = v[j];
}
__device__ __forceinline__ void store_half4(uint16_t* a, int dtype, int64_t i, int64_t n, f32x4 v) {
  const u32x2 w = {pack_half(dtype, v[0], v[1]), pack_half(dtype, v[2], v[3])};
  if (i + 4 <= n) {
    *reinterpret_cast<u32x2*>(a + i) = w;
    return;
  }
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (i + j < n) a[i + j] = static_cast<uint16_t>(w[j >> 1] >> (16 * (j & 1)));
}

__global__ __launch_bounds__(kThreads) void adamw_f32_kernel(const Entry* __restrict__ entries, const int32_t* __restrict__ of_chunk,
                                                             const moe_adamw_values* __restrict__ values, Hyper h) {
  const moe_adamw_values s = *values;
  if (s.skip != 0) return;
  const Entry e = entries[of_chunk[blockIdx.x]];
  if (e.m_power != nullptr) return;   // (a plan of 8-bit moments)
  const Step st = step_of(h, s, e);
  const int64_t begin = static_cast<int64_t>(blockIdx.x - e.first_chunk) * kChunk + threadIdx.x * 4;
  constexpr int kTurns = kChunk / (4 * kThreads);
  f32x4 p[kTurns], g[kTurns], m[kTurns], v[kTurns];
#pragma unroll
  for (int k = 0; k < kTurns; ++k) {
    const int64_t i = begin + k * (4 * kThreads);
    p[k] = load4(e.p, i, e.n);
    g[k] = load4(e.g, i, e.n);
    m[k] = load4(static_cast<const float*>(e.m), i, e.n);
    v[k] = load4(static_cast<const float*>(e.v), i, e.n);
  }
#pragma unroll
  for (int k = 0; k < kTurns; ++k) {
    const int64_t i = begin + k * (4 * kThreads);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float gj = g[k][j] * st.grad_scale;
      m[k][j] = st.b1 * m[k][j] + st.omb1 * gj;
      v[k][j] = st.b2 * v[k][j] + st.omb2 * (gj * gj);
      p[k][j] = updated(st, p[k][j], m[k][j], sqrtf(v[k][j]));
    }
    store4(e.p, i, e.n, p[k]);
    store4(static_cast<float*>(e.m), i, e.n, m[k]);
    store4(static_cast<float*>(e.v), i, e.n, v[k]);
    if (e.half != nullptr) store_half4(e.half, e.half_dtype, i, e.n, p[k]);
  }
}

// ---- 8-bit moments: a thread holds eight elements, four threads a block of 32 --------------------------

__device__ __forceinline__ u32x2 load_codes(const void* a, int64_t i, int64_t n) {
  const uint8_t* c = static_cast<const uint8_t*>(a);
  if (i + 8 <= n) return *reinterpret_cast<const u32x2*>(c + i);
  u32x2 w = {0u, 0u};
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (i + j < n) w[j >> 2] |= static_cast<uint32_t>(c[i + j]) << (8 * (j & 3));
  return w;
}
__device__ __forceinline__ void store_codes(void* a, int64_t i, int64_t n, u32x2 w) {
  uint8_t* c = static_cast<uint8_t*>(a);
  if (i + 8 <= n) {
    *reinterpret_cast<u32x2*>(c + i) = w;
    return;
  }
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (i + j < n) c[i + j] = static_cast<uint8_t>(w[j >> 2] >> (8 * (j & 3)));
}

// 2^(power - 127); 255 is NaN
__device__ __forceinline__ float power_of_two(uint32_t power) {
  return __uint_as_float(power == 0 ? 0x00400000u : power == 255 ? 0x7fc00000u : power << 23);
}

__device__ __forceinline__ void widen(u32x2 codes, float scale, float (&v)[8]) {
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    const f32x2_t lo = __builtin_amdgcn_cvt_pk_f32_fp8(codes[q], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(codes[q], true);
    v[4 * q + 0] = lo.x * scale;
    v[4 * q + 1] = lo.y * scale;
    v[4 * q + 2] = hi.x * scale;
    v[4 * q + 3] = hi.y * scale;
  }
}

// The largest of four neighbouring lanes' values (as bits: of non-negative floats in their order, NaN above all).
__device__ __forceinline__ uint32_t largest_of_four(uint32_t v) {
  v = max(v, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), 0xB1, 0xf, 0xf, true)));   // lane ^ 1
  return max(v, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), 0x4E, 0xf, 0xf, true)));   // lane ^ 2
}

// Codes of eight values; `power` is the block's.  phase[j]: 20 bits.
template <bool POSITIVE>
__device__ __forceinline__ u32x2 narrow(const float (&v)[8], const uint32_t (&phase)[8], uint32_t& power) {
  uint32_t top = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(v[j]) & 0x7fffffffu);
  top = largest_of_four(top);
  if (top >= 0x7f800000u) {   // (the whole block: what it stands for is lost)
    power = 255;
    return u32x2{0x7f7f7f7fu, 0x7f7f7f7fu};
  }
  // the least power of two with `top` at most 448 of it
  const int e = max(static_cast<int>(top >> 23) - 127 - 8 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0), kLowestPower);
  power = e + 127;
  const float inverse = __uint_as_float(static_cast<uint32_t>(127 - e) << 23);
  u32x2 w = {0u, 0u};
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float y = fabsf(v[j]) * inverse;
    const uint32_t normal = ((__float_as_uint(y) + phase[j]) >> 20) - 960u;         // exponent bias 127 -> 7
    const uint32_t small = (static_cast<uint32_t>(y * 536870912.0f) + phase[j]) >> 20;   // steps of 2^-9
    uint32_t code = min(y >= 0.015625f ? normal : small, 126u);
    if (POSITIVE) code = v[j] > 0.f ? max(code, 1u) : code;
    else code |= v[j] < 0.f ? 128u : 0u;
    w[j >> 2] |= code << (8 * (j & 3));
  }
  return w;
}

__global__ __launch_bounds__(kThreads) void adamw_8bit_kernel(const Entry* __restrict__ entries, const int32_t* __restrict__ of_chunk,
                                                              const moe_adamw_values* __restrict__ values, Hyper h) {
  const moe_adamw_values s = *values;
  if (s.skip != 0) return;
  const Entry e = entries[of_chunk[blockIdx.x]];
  if (e.m_power == nullptr) return;   // (a plan of float32 moments)
  const Step st = step_of(h, s, e);
  const int64_t begin = static_cast<int64_t>(blockIdx.x - e.first_chunk) * kChunk + threadIdx.x * 8;
  constexpr int kTurns = kChunk / (8 * kThreads);
  f32x4 p[kTurns][2], g[kTurns][2];
  u32x2 mc[kTurns], rc[kTurns];
  uint32_t mp[kTurns], rp[kTurns];
#pragma unroll
  for (int k = 0; k < kTurns; ++k) {
    const int64_t i = begin + k * (8 * kThreads);
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      p[k][q] = load4(e.p, i + 4 * q, e.n);
      g[k][q] = load4(e.g, i + 4 * q, e.n);
    }
    mc[k] = load_codes(e.m, i, e.n);
    rc[k] = load_codes(e.v, i, e.n);
    mp[k] = i < e.n ? e.m_power[i / kBlock] : 0;
    rp[k] = i < e.n ? e.v_power[i / kBlock] : 0;
  }
#pragma unroll
  for (int k = 0; k < kTurns; ++k) {
    const int64_t i = begin + k * (8 * kThreads);
    float m[8], root[8];
    widen(mc[k], power_of_two(mp[k]), m);
    widen(rc[k], power_of_two(rp[k]), root);
    uint32_t phase[8], other[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float gj = g[k][j >> 2][j & 3] * st.grad_scale;
      m[j] = st.b1 * m[j] + st.omb1 * gj;
      root[j] = sqrtf(st.b2 * (root[j] * root[j]) + st.omb2 * (gj * gj));
      p[k][j >> 2][j & 3] = updated(st, p[k][j >> 2][j & 3], m[j], root[j]);
      phase[j] = (((static_cast<uint32_t>(i) + j) & 511u) * 0x85EBCA6Bu + st.phase) >> 12;
      other[j] = phase[j] ^ 0x80000u;   // (the roots' are half a turn away)
    }
    // (elements past the end hold zeros: g and the codes read zero)
    mc[k] = narrow<false>(m, phase, mp[k]);
    rc[k] = narrow<true>(root, other, rp[k]);
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      store4(e.p, i + 4 * q, e.n, p[k][q]);
      if (e.half != nullptr) store_half4(e.half, e.half_dtype, i + 4 * q, e.n, p[k][q]);
    }
    store_codes(e.m, i, e.n, mc[k]);
    store_codes(e.v, i, e.n, rc[k]);
    if ((threadIdx.x & 3) == 0 && i < e.n) {
      e.m_power[i / kBlock] = static_cast<uint8_t>(mp[k]);
      e.v_power[i / kBlock] = static_cast<uint8_t>(rp[k]);
    }
  }
}

// ---- host ----------------------------------------------------------------------------------------

int check_config(const moe_adamw_config* c) {
  if (c == nullptr) return MOE_ERR_NULL;
  if (!(c->beta1 >= 0.0 && c->beta1 < 1.0) || !(c->beta2 >= 0.0 && c->beta2 < 1.0)) return MOE_ERR_SHAPE;
  if (!(static_cast<float>(c->eps) > 0.f) || std::isinf(c->eps)) return MOE_ERR_SHAPE;
  if (c->moment_bits != 32 && c->moment_bits != 8) return MOE_ERR_DTYPE;
  return MOE_OK;
}

constexpr int64_t kMostChunks = (int64_t(1) << 31) - 1;

// Chunks of all tensors; -1: a size is negative or there are too many.
int64_t chunks_of(const moe_adamw_tensor* t, int n) {
  int64_t total = 0;
  for (int i = 0; i < n; ++i) {
    if (t[i].n < 0 || t[i].n > kMostChunks * kChunk) return -1;
    total += (t[i].n + kChunk - 1) / kChunk;
    if (total > kMostChunks) return -1;
  }
  return total;
}

int check_tensor(const moe_adamw_config& c, const moe_adamw_tensor& t) {
  if (t.n == 0) return MOE_OK;
  const void* ptr[7] = {t.p, t.g, t.m, t.v, t.m_power, t.v_power, t.half};
  for (int i = 0; i < 6; ++i)
    if (ptr[i] == nullptr && (i < 4 || c.moment_bits == 8)) return MOE_ERR_NULL;
  for (const void* a : ptr)
    if (reinterpret_cast<uintptr_t>(a) & 15u) return MOE_ERR_ALIGN;
  if (t.half != nullptr && !is_16bit(t.half_dtype)) return MOE_ERR_DTYPE;
  if (!std::isfinite(t.lr_scale) || !std::isfinite(t.weight_decay)) return MOE_ERR_SHAPE;
  return MOE_OK;
}

// Does memory that one tensor of the plan writes belong to another one, or twice to the same?
bool overlapping(const moe_adamw_config& c, const moe_adamw_tensor* t, int n) {
  struct Range {
    uintptr_t at, end;
    bool written;
  };
  std::vector<Range> all;
  auto add = [&](const void* a, int64_t bytes, bool written) {
    if (a != nullptr && bytes > 0) all.push_back({reinterpret_cast<uintptr_t>(a), reinterpret_cast<uintptr_t>(a) + bytes, written});
  };
  for (int i = 0; i < n; ++i) {
    const int64_t moment = c.moment_bits == 8 ? t[i].n : 4 * t[i].n, powers = c.moment_bits == 8 ? (t[i].n + kBlock - 1) / kBlock : 0;
    add(t[i].p, 4 * t[i].n, true);
    add(t[i].g, 4 * t[i].n, false);
    add(t[i].m, moment, true);
    add(t[i].v, moment, true);
    add(t[i].m_power, powers, true);
    add(t[i].v_power, powers, true);
    add(t[i].half, 2 * t[i].n, true);
  }
  std::sort(all.begin(), all.end(), [](const Range& a, const Range& b) { return a.at < b.at; });
  uintptr_t end_any = 0, end_written = 0;
  for (const Range& r : all) {
    if (r.at < (r.written ? end_any : end_written)) return true;
    end_any = std::max(end_any, r.end);
    if (r.written) end_written = std::max(end_written, r.end);
  }
  return false;
}

}  // namespace adamw
}  // namespace ppmoe

using namespace ppmoe;

extern "C" {

size_t moe_adamw_plan_bytes(const moe_adamw_config* cfg, const moe_adamw_tensor* tensors, int32_t n_tensors) {
  if (adamw::check_config(cfg) != MOE_OK || n_tensors < 0 || (n_tensors > 0 && tensors == nullptr)) return 0;
  const int64_t chunks = adamw::chunks_of(tensors, n_tensors);
  if (chunks < 0) return 0;
  const size_t bytes = n_tensors * sizeof(adamw::Entry) + static_cast<size_t>(chunks) * sizeof(int32_t);
  return (bytes + 15) / 16 * 16 + 16;   // (never 0 for what is allowed)
}

int moe_adamw_plan(const moe_adamw_config* cfg, const moe_adamw_tensor* tensors, int32_t n_tensors, void* plan, size_t plan_bytes,
                   int64_t* n_chunks) {
  int st = adamw::check_config(cfg);
  if (st != MOE_OK) return st;
  if (plan == nullptr || n_chunks == nullptr || (n_tensors > 0 && tensors == nullptr)) return MOE_ERR_NULL;
  if (n_tensors < 0 || adamw::chunks_of(tensors, n_tensors) < 0) return MOE_ERR_SHAPE;
  for (int i = 0; i < n_tensors; ++i) {
    st = adamw::check_tensor(*cfg, tensors[i]);
    if (st != MOE_OK) return st;
  }
  if (plan_bytes < moe_adamw_plan_bytes(cfg, tensors, n_tensors)) return MOE_ERR_WORKSPACE;
  try {
    if (adamw::overlapping(*cfg, tensors, n_tensors)) return MOE_ERR_OVERLAP;
  } catch (...) {
    return MOE_ERR_WORKSPACE;   // (no host memory for the check)
  }
  unsigned char* at = static_cast<unsigned char*>(plan);
  int32_t chunk = 0;
  for (int i = 0; i < n_tensors; ++i) {
    const moe_adamw_tensor& t = tensors[i];
    const bool codes = cfg->moment_bits == 8;
    const adamw::Entry e = {t.p, t.g, t.m, t.v, codes ? t.m_power : nullptr, codes ? t.v_power : nullptr, static_cast<uint16_t*>(t.half), t.n, chunk, t.half_dtype,
                            t.lr_scale, t.weight_decay};
    memcpy(at + i * sizeof(e), &e, sizeof(e));
    for (int64_t left = t.n; left > 0; left -= adamw::kChunk, ++chunk)
      memcpy(at + n_tensors * sizeof(e) + static_cast<size_t>(chunk) * sizeof(int32_t), &i, sizeof(int32_t));
  }
  *n_chunks = chunk;
  return MOE_OK;
}

int moe_adamw_step(const moe_adamw_config* cfg, const void* plan, int32_t n_tensors, int64_t n_chunks, const moe_adamw_values* values,
                   void* stream) {
  const int st = adamw::check_config(cfg);
  if (st != MOE_OK) return st;
  if (plan == nullptr || values == nullptr) return MOE_ERR_NULL;
  if (n_tensors < 0 || n_chunks < 0 || n_chunks > adamw::kMostChunks || (n_tensors == 0 && n_chunks > 0)) return MOE_ERR_SHAPE;
  if ((reinterpret_cast<uintptr_t>(plan) & 15u) || (reinterpret_cast<uintptr_t>(values) & 15u)) return MOE_ERR_ALIGN;
  if (n_chunks == 0) return MOE_OK;
  const adamw::Entry* entries = static_cast<const adamw::Entry*>(plan);
  const int32_t* of_chunk = reinterpret_cast<const int32_t*>(entries + n_tensors);
  const adamw::Hyper h = {cfg->beta1, cfg->beta2, static_cast<float>(cfg->eps)};
  hipStream_t s = static_cast<hipStream_t>(stream);
  const unsigned grid = static_cast<unsigned>(n_chunks);
  if (cfg->moment_bits == 8) adamw::adamw_8bit_kernel<<<grid, adamw::kThreads, 0, s>>>(entries, of_chunk, values, h);
  else adamw::adamw_f32_kernel<<<grid, adamw::kThreads, 0, s>>>(entries, of_chunk, values, h);
  return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_HIP;
}

}  // extern "C"
