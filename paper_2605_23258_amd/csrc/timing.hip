// Optional per-kernel timing with HIP events on the launch stream, for benchmarks.
// Off by default; when off a launch costs one predictable branch.  Not thread-safe:
// enable, run and read from one host thread.
#include <vector>

#include "../../include/vector.h"
#include "launch.hpp"

namespace vec {

namespace {
struct Span { hipEvent_t start, stop; };
struct Slot {
  std::vector<Span> spans;     // recorded since the last read
  std::vector<Span> free_list; // events ready for reuse
};
bool g_enabled = false;
Slot g_slots[K_COUNT];
const char* const kNames[K_COUNT] = {"score_stats", "stats_combine", "mass_residual", "pool_scores",
                                     "route", "gather_rows", "decode_split", "decode_combine", "fp4_rows", "block_tables"};
}  // namespace

bool timing_enabled() { return g_enabled; }

void timing_begin(int id, hipStream_t stream) {
  Slot& s = g_slots[id];
  Span sp;
  if (!s.free_list.empty()) {
    sp = s.free_list.back();
    s.free_list.pop_back();
  } else {
    if (hipEventCreate(&sp.start) != hipSuccess || hipEventCreate(&sp.stop) != hipSuccess) return;
  }
  hipEventRecord(sp.start, stream);
  s.spans.push_back(sp);
}

void timing_end(int id, hipStream_t stream) {
  Slot& s = g_slots[id];
  if (!s.spans.empty()) hipEventRecord(s.spans.back().stop, stream);
}

}  // namespace vec

extern "C" {

int vector_timing_enable(int on) {
  vec::g_enabled = on != 0;
  return VECTOR_OK;
}

int vector_timing_kernels(void) { return vec::K_COUNT; }

const char* vector_timing_name(int kernel_id) {
  return (kernel_id >= 0 && kernel_id < vec::K_COUNT) ? vec::kNames[kernel_id] : "";
}

int vector_timing_read(int kernel_id, double* total_ms, int64_t* launches) {
  if (kernel_id < 0 || kernel_id >= vec::K_COUNT || !total_ms || !launches) return VECTOR_ERR_ARG;
  vec::Slot& s = vec::g_slots[kernel_id];
  double sum = 0.0;
  int64_t count = 0;
  for (vec::Span& sp : s.spans) {
    if (hipEventSynchronize(sp.stop) != hipSuccess) return VECTOR_ERR_HIP;
    float ms = 0.f;
    if (hipEventElapsedTime(&ms, sp.start, sp.stop) != hipSuccess) return VECTOR_ERR_HIP;
    sum += ms;
    ++count;
    s.free_list.push_back(sp);
  }
  s.spans.clear();
  *total_ms = sum;
  *launches = count;
  return VECTOR_OK;
}

}  // extern "C"

// ---------------------------------------------------------------------------
// Measured matrix-core ceiling: every wave runs `iters` rounds of four independent
// v_mfma_f32_32x32x16_bf16 on operands in registers (no memory traffic in the loop).
// 256 workgroups of 1024 threads: four waves per SIMD on every CU.
// ---------------------------------------------------------------------------
namespace vec {
namespace {
typedef __attribute__((ext_vector_type(8))) __bf16 probe_bf16x8;
typedef __attribute__((ext_vector_type(16))) float probe_f32x16;
constexpr int kMfmaProbeGrid = 256, kMfmaProbeThreads = 1024;

__global__ __launch_bounds__(kMfmaProbeThreads) void mfma_loop_kernel(float* out, int iters) {
  probe_f32x16 a0 = {0}, a1 = {0}, a2 = {0}, a3 = {0};
  probe_bf16x8 a, b;
#pragma unroll
  for (int i = 0; i < 8; ++i) { a[i] = (__bf16)(float)(threadIdx.x & 3); b[i] = (__bf16)1.0f; }
  for (int it = 0; it < iters; ++it) {
    a0 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, a0, 0, 0, 0);
    a1 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, a1, 0, 0, 0);
    a2 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, a2, 0, 0, 0);
    a3 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, a3, 0, 0, 0);
  }
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) s += a0[i] + a1[i] + a2[i] + a3[i];
  out[(size_t)blockIdx.x * kMfmaProbeThreads + threadIdx.x] = s;
}

// Read-only stream: every workgroup takes a contiguous slice with 16-byte loads, eight in flight per
// thread; the xor of what was read reaches memory only for one impossible value.
constexpr int kReadProbeThreads = 512, kReadProbeLoads = 8;
__global__ __launch_bounds__(kReadProbeThreads) void read_stream_kernel(const uint4* __restrict__ src, size_t per_wg, float* out) {
  const uint4* p = src + (size_t)blockIdx.x * per_wg;
  unsigned acc = 0;
  for (size_t i = threadIdx.x; i + (kReadProbeLoads - 1) * kReadProbeThreads < per_wg; i += (size_t)kReadProbeLoads * kReadProbeThreads) {
    uint4 v[kReadProbeLoads];
#pragma unroll
    for (int u = 0; u < kReadProbeLoads; ++u) v[u] = p[i + (size_t)u * kReadProbeThreads];
#pragma unroll
    for (int u = 0; u < kReadProbeLoads; ++u) acc += v[u].x ^ v[u].y ^ v[u].z ^ v[u].w;
  }
  if (acc == 0x9e3779b9u && out) out[blockIdx.x] = 1.f;
}
}  // namespace
}  // namespace vec

extern "C" {

int vector_probe_read_stream(const void* src, size_t bytes, float* out, int64_t* bytes_read, void* stream) {
  constexpr size_t kGrid = 1024, kSlice = (size_t)vec::kReadProbeThreads * vec::kReadProbeLoads * 16;
  if (!src || !out || !bytes_read || (reinterpret_cast<uintptr_t>(src) & 15u)) return VECTOR_ERR_ARG;
  const size_t per_wg_bytes = bytes / kGrid / kSlice * kSlice;      // whole rounds of loads only: nothing beyond `bytes` is read
  if (per_wg_bytes == 0) return VECTOR_ERR_ARG;
  hipLaunchKernelGGL(vec::read_stream_kernel, dim3((unsigned)kGrid), dim3(vec::kReadProbeThreads), 0, (hipStream_t)stream,
                     static_cast<const uint4*>(src), per_wg_bytes / 16, out);
  if (hipGetLastError() != hipSuccess) return VECTOR_ERR_HIP;
  *bytes_read = (int64_t)(per_wg_bytes * kGrid);
  return VECTOR_OK;
}

int vector_probe_mfma_loop(float* out, int32_t iters, int64_t* flops, void* stream) {
  if (!out || iters < 1 || !flops) return VECTOR_ERR_ARG;
  hipLaunchKernelGGL(vec::mfma_loop_kernel, dim3(vec::kMfmaProbeGrid), dim3(vec::kMfmaProbeThreads), 0, (hipStream_t)stream, out, iters);
  if (hipGetLastError() != hipSuccess) return VECTOR_ERR_HIP;
  *flops = (int64_t)vec::kMfmaProbeGrid * (vec::kMfmaProbeThreads / 64) * iters * 4 * (2LL * 32 * 32 * 16);
  return VECTOR_OK;
}

}  // extern "C"
