// Set-up and launches of the persistent grouped GEMM (gemm_fast.h).

#include <atomic>
#include <mutex>

#include "gemm_fast.h"

namespace ppmoe {

namespace fast {

// Set-up check of the placement rule the hand-over of partial sums relies on (block b runs on XCD
// b mod 8, so blocks b and b' with b = b' mod 8 share an L2): every block reports where it ran.
__device__ uint32_t g_xcc_of_block[kMaxPersistentBlocks];   // (each device holds its own copy)
__global__ __launch_bounds__(kThreads) void xcc_probe_kernel() {
  if (threadIdx.x == 0) g_xcc_of_block[blockIdx.x] = xcc_id();
}

}  // namespace fast

hipError_t read_gemm_error_word(const void* workspace, uint32_t* word, hipStream_t s) {
  const float* slots = static_cast<const float*>(workspace);
  const uint32_t* flags = reinterpret_cast<const uint32_t*>(
      slots + static_cast<size_t>(fast::kSlotsPerBlock) * kMaxPersistentBlocks * fast::kSlotFloats);
  hipError_t e = hipMemcpyAsync(word, flags + kMaxPersistentBlocks, sizeof(uint32_t),
                                hipMemcpyDeviceToHost, s);
  if (e != hipSuccess) return e;
  e = hipStreamSynchronize(s);
  if (e != hipSuccess) return e;
  if ((*word & 0xffffff00u) == kGemmErrorMagic) {   // reported once: lower it again
    static const uint32_t zero = 0;
    e = hipMemcpyAsync(const_cast<uint32_t*>(flags) + kMaxPersistentBlocks, &zero, sizeof(uint32_t),
                       hipMemcpyHostToDevice, s);
    if (e != hipSuccess) return e;
    e = hipStreamSynchronize(s);
  }
  return e;
}

unsigned long long* gemm_clock_words(void* workspace) {
  uint32_t* flags = reinterpret_cast<uint32_t*>(
      static_cast<float*>(workspace) +
      static_cast<size_t>(fast::kSlotsPerBlock) * kMaxPersistentBlocks * fast::kSlotFloats);
  return reinterpret_cast<unsigned long long*>(flags + fast::kClockWord);
}

// Shader-clock and wall-clock ticks a block of the last fast-path launch on this workspace counted
// between its start and its end.  Synchronises the stream.
hipError_t read_gemm_clock_words(const void* workspace, uint64_t* shader_ticks, uint64_t* wall_ticks,
                                 hipStream_t s) {
  const float* slots = static_cast<const float*>(workspace);
  const uint32_t* flags = reinterpret_cast<const uint32_t*>(
      slots + static_cast<size_t>(fast::kSlotsPerBlock) * kMaxPersistentBlocks * fast::kSlotFloats);
  uint64_t w[4] = {0, 0, 0, 0};
  hipError_t e = hipMemcpyAsync(w, flags + fast::kClockWord, sizeof(w), hipMemcpyDeviceToHost, s);
  if (e != hipSuccess) return e;
  e = hipStreamSynchronize(s);
  if (e != hipSuccess) return e;
  *shader_ticks = w[2] - w[0];
  *wall_ticks = w[3] - w[1];
  return hipSuccess;
}

size_t grouped_gemm_fast_workspace_bytes() {
  // slots, flags (+1 word: the error word), and inside the padding the four clock words
  return static_cast<size_t>(fast::kSlotsPerBlock) * kMaxPersistentBlocks * fast::kSlotFloats * sizeof(float) +
         (2 * kMaxPersistentBlocks + 1) * sizeof(uint32_t) + 256;
}

// ---- per-device set-up --------------------------------------------------------------------------
// Once per device: the dynamic-LDS attribute of the kernels, the number of persistent blocks, and the
// placement check (do blocks b and b + 8 share an XCD, as the workgroup-scope hand-over assumes?).
// The check launches a probe and waits for it, so it is the one thing here that synchronises; it
// runs from moe_init, or from the first launch on a device that finds it not done -- unless that
// launch is being captured into a graph, in which case the launch uses device-scope fences and
// leaves the check for later.
namespace {

constexpr int kMaxDevices = 64;
struct FastSetup {
  bool attrs = false;   // kernel attributes set, `blocks` valid
  bool probed = false;  // same_l2 valid
  int blocks = 0;
  int same_l2 = 0;
};
FastSetup g_setup[kMaxDevices];
std::mutex g_setup_mutex;
std::atomic<int> g_force_device_scope{0};
std::atomic<int> g_spin_limit{fast::kDefaultSpinLimit};

hipError_t setup_attrs(FastSetup& st, int dev) {
  using namespace fast;
  if (st.attrs) return hipSuccess;
#define PPMOE_KERNELS(DT, R)                                                               \
  reinterpret_cast<const void*>(grouped_gemm_fast_kernel<1, 0, DT, R, false>),          \
      reinterpret_cast<const void*>(grouped_gemm_fast_kernel<0, 0, DT, R, false>),     \
      reinterpret_cast<const void*>(grouped_gemm_fast_kernel<1, 1, DT, R, false>),      \
      reinterpret_cast<const void*>(grouped_gemm_fast_kernel<0, 2, DT, R, false>)
  const void* kernels[] = {PPMOE_KERNELS(MOE_BF16, false), PPMOE_KERNELS(MOE_BF16, true),
                           PPMOE_KERNELS(MOE_F16, false), PPMOE_KERNELS(MOE_F16, true),
                           reinterpret_cast<const void*>(grouped_gemm_fast_kernel<2, 0, MOE_BF16, false, false>),
                           reinterpret_cast<const void*>(grouped_gemm_fast_kernel<2, 0, MOE_F16, false, false>),
                           reinterpret_cast<const void*>(grouped_gemm_fast_kernel<0, 0, MOE_BF16, false, true>),
                           reinterpret_cast<const void*>(grouped_gemm_fast_kernel<0, 0, MOE_F16, false, true>)};
#undef PPMOE_KERNELS
  for (const void* k : kernels) {
    hipError_t e = hipFuncSetAttribute(k, hipFuncAttributeMaxDynamicSharedMemorySize, kLdsBytes);
    if (e != hipSuccess) return e;
  }
  for (int k = 0; k < 16; ++k) {   // (the bits of k are the variant)
    const FastKernel kernel = fast_kernel_with_adapters((k & 8) ? MOE_F16 : MOE_BF16, (k & 1) != 0, (k & 2) != 0, (k & 4) != 0);
    if (kernel == nullptr) continue;
    hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, kLdsBytes);
    if (e != hipSuccess) return e;
  }
  int cus = 0;
  hipError_t e = hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev);
  if (e != hipSuccess) return e;
  if (cus > kMaxPersistentBlocks) cus = kMaxPersistentBlocks;
  st.blocks = cus & ~7;   // one block per CU, the same number on each of the 8 XCDs
  if (st.blocks < 8) return hipErrorInvalidConfiguration;
  st.attrs = true;
  return hipSuccess;
}

// Launches the placement probe on `s` and waits for it.  Must not be called while `s` is capturing.
hipError_t setup_probe(FastSetup& st, hipStream_t s) {
  if (st.probed) return hipSuccess;
  uint32_t host[kMaxPersistentBlocks];
  fast::xcc_probe_kernel<<<st.blocks, fast::kThreads, 0, s>>>();
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  e = hipMemcpyFromSymbolAsync(host, HIP_SYMBOL(fast::g_xcc_of_block), st.blocks * sizeof(uint32_t), 0,
                               hipMemcpyDeviceToHost, s);
  if (e != hipSuccess) return e;
  e = hipStreamSynchronize(s);
  if (e != hipSuccess) return e;
  st.same_l2 = 1;
  for (int b = 8; b < st.blocks; ++b)
    if (host[b] != host[b & 7]) st.same_l2 = 0;
  st.probed = true;
  return hipSuccess;
}

}  // namespace

// The set-up as a launch on `s` finds it or, outside a capture, makes it.
static hipError_t set_up_for_launch(hipStream_t s, int* blocks, int* same_l2) {
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  if (dev < 0 || dev >= kMaxDevices) return hipErrorInvalidDevice;
  std::lock_guard<std::mutex> lock(g_setup_mutex);
  FastSetup& st = g_setup[dev];
  e = setup_attrs(st, dev);
  if (e != hipSuccess) return e;
  if (!st.probed) {
    hipStreamCaptureStatus cap = hipStreamCaptureStatusNone;
    e = hipStreamIsCapturing(s, &cap);
    if (e != hipSuccess) return e;
    if (cap == hipStreamCaptureStatusNone) {
      e = setup_probe(st, s);
      if (e != hipSuccess) return e;
    }
  }
  *blocks = st.blocks;
  *same_l2 = st.probed ? st.same_l2 : 0;   // unknown placement: device-scope fences are always right
  return hipSuccess;
}

hipError_t grouped_gemm_set_up(hipStream_t s) {
  int blocks = 0, same_l2 = 0;
  return set_up_for_launch(s, &blocks, &same_l2);
}

hipError_t grouped_gemm_fast_init(hipStream_t s) {
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  if (dev < 0 || dev >= kMaxDevices) return hipErrorInvalidDevice;
  std::lock_guard<std::mutex> lock(g_setup_mutex);
  e = setup_attrs(g_setup[dev], dev);
  if (e != hipSuccess) return e;
  return setup_probe(g_setup[dev], s);
}

void grouped_gemm_fast_set_handover(int force_device_scope, int spin_limit) {
  if (force_device_scope >= 0) g_force_device_scope = force_device_scope ? 1 : 0;
  if (spin_limit >= 0) g_spin_limit = spin_limit;
}

hipError_t launch_grouped_gemm_fast(int in_dtype, bool gelu, const bf16_t* A, const bf16_t* B, bf16_t* C,
                                    const int32_t* offsets, int n_exp, int few_most, int Nout,
                                    int K, void* workspace, hipStream_t s, int fuse,
                                    const int32_t* aux_rows, const float* aux_w, int aux_div,
                                    const int32_t* aux_inv, bf16_t* C2, bool b_by_rows, int pick_cus,
                                    const AdapterRows* adapters) {
  using namespace fast;
  int blocks = 0, same_l2 = 0;
  hipError_t e = set_up_for_launch(s, &blocks, &same_l2);
  if (e != hipSuccess) return e;
  if (g_force_device_scope.load()) same_l2 = 0;
  const int spin_limit = g_spin_limit.load();
  static std::atomic<uint32_t> launches{0};
  // 28 bits (the flag word also carries the XCD id), spread over the word so that small integers
  // left in a recycled workspace do not look like an epoch; 0 means "flag down".
  uint32_t epoch = (++launches * 0x9E3779B1u) >> 4;
  if (epoch == 0) epoch = (++launches * 0x9E3779B1u) >> 4;
  float* slots = static_cast<float*>(workspace);
  uint32_t* flags = reinterpret_cast<uint32_t*>(
      slots + static_cast<size_t>(kSlotsPerBlock) * kMaxPersistentBlocks * kSlotFloats);
  const bool ragged = K % BK != 0;
  // fuse: 0 none; 1 rows of A through aux_rows (first GEMM only); 2 rows of the result placed through
  // aux_rows (second GEMM only; with aux_div > 1 it needs the inverse permutation and a place for
  // the rows it cannot place)
  if ((fuse == 1 && !gelu) || (fuse == 2 && gelu) || fuse < 0 || fuse > 2 ||
      (fuse != 0 && aux_rows == nullptr) || (fuse == 2 && aux_w == nullptr) || aux_div < 1 ||
      (fuse == 2 && aux_div != 1 && (aux_inv == nullptr || C2 == nullptr)) ||
      (adapters != nullptr && (fuse != 0 || C2 != nullptr)))
    return hipErrorInvalidValue;
  const AdapterRows rows = adapters != nullptr ? *adapters : AdapterRows{};
#define PPMOE_LAUNCH_KERNEL(...)                                                      \
  __VA_ARGS__<<<blocks, kThreads, kLdsBytes, s>>>(     \
      A, B, C, offsets, n_exp, few_most, Nout, K, slots, flags, epoch, same_l2, spin_limit, aux_rows, aux_w, aux_div, \
      aux_inv, C2, pick_cus, rows)
#define PPMOE_LAUNCH_DT(G, F, DT, R) PPMOE_LAUNCH_KERNEL(grouped_gemm_fast_kernel<G, F, DT, R, false>)
#define PPMOE_LAUNCH(G, F)                            \
  do {                                                \
    if (in_dtype == MOE_F16 && ragged) PPMOE_LAUNCH_DT(G, F, MOE_F16, true); \
    else if (in_dtype == MOE_F16) PPMOE_LAUNCH_DT(G, F, MOE_F16, false);     \
    else if (ragged) PPMOE_LAUNCH_DT(G, F, MOE_BF16, true);                  \
    else PPMOE_LAUNCH_DT(G, F, MOE_BF16, false);                             \
  } while (0)
  if (b_by_rows && (gelu || fuse != 0 || ragged)) return hipErrorInvalidValue;
  if (adapters != nullptr) {
    const FastKernel kernel = fast_kernel_with_adapters(in_dtype, gelu, ragged, b_by_rows);
    if (kernel == nullptr) return hipErrorInvalidValue;
    PPMOE_LAUNCH_KERNEL(kernel);
  } else if (b_by_rows) {
    if (in_dtype == MOE_F16) PPMOE_LAUNCH_KERNEL(grouped_gemm_fast_kernel<0, 0, MOE_F16, false, true>);
    else PPMOE_LAUNCH_KERNEL(grouped_gemm_fast_kernel<0, 0, MOE_BF16, false, true>);
  } else if (fuse == 1) PPMOE_LAUNCH(1, 1);
  else if (fuse == 2) PPMOE_LAUNCH(0, 2);
  else if (gelu && C2 != nullptr) {   // (the pre-activations as well)
    if (ragged) return hipErrorInvalidValue;
    if (in_dtype == MOE_F16) PPMOE_LAUNCH_KERNEL(grouped_gemm_fast_kernel<2, 0, MOE_F16, false, false>);
    else PPMOE_LAUNCH_KERNEL(grouped_gemm_fast_kernel<2, 0, MOE_BF16, false, false>);
  } else if (gelu) PPMOE_LAUNCH(1, 0);
  else PPMOE_LAUNCH(0, 0);
#undef PPMOE_LAUNCH_DT
#undef PPMOE_LAUNCH_KERNEL
#undef PPMOE_LAUNCH
  return hipGetLastError();
}

}  // namespace ppmoe
