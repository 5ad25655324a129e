// Key and value rows into 4 bits and back: vector_compact_fp4, vector_store_fp4, vector_load_fp4.
//
// What bounds them is memory: a bf16 row of 128 elements is 256 bytes, in 4 bits 68.  Eight elements go to a lane (16 or 32 bytes
// in, four bytes of codes out), so D / 8 adjacent lanes hold a row, every load of a wave covers whole rows, and the four lanes of a
// block find its largest magnitude by two exchanges inside the group of four.  Rows in 16 and 32 bits are read and written past the caches
// (non-temporal), which are left to the codes: eight prompts of 2048 to 8192 tokens, 8 KV heads, 229 MB, stored in 58.5 us without and 39.6 with (5.8 TB/s),
// read back (101 MB) in 19.6 and 18.2.  Four rows a thread instead of two: 42.8.
// By the routing's lists (a layer of 32768 tokens, 8 KV heads, a tenth of them retained and a tenth approximated, 25.7 MB) 7.8 us, 3.3 TB/s: one chain of
// list, row and store, which all workgroups go through at once.
#include "fp4.hpp"
#include "launch.hpp"

namespace vec {

namespace {

constexpr int kThreads = 256;

struct StoreParams {
  const void *k, *v;
  int64_t k_sh, k_st, v_sh, v_st;          // element strides
  const int32_t *idx_a, *idx_b;            // lists of rows [heads, n_a], [heads, n_b]; null with slots
  const int64_t* slots;                    // [heads, n_a]: where a row goes, or null
  int64_t pool_rows;
  uint8_t *ka, *ka_scale, *va, *va_scale, *kb, *kb_scale;
  int n_tokens, n_a, n_b, cap;
  int parts_a;                             // workgroups along the first rows, the second ones' follow
};

// A workgroup takes kRows rows of a head: keys and values of the first kind of rows, keys of the second.  What a thread loads of its
// kUnroll rows is on its way before the first is rounded; by slots the rows do not wait for these.
template <typename T, int D> struct StoreShape {
  static constexpr int kLanes = D / 8;                       // of a row
  static constexpr int kAtOnce = kThreads / kLanes;          // rows
  static constexpr int kUnroll = 2;
  static constexpr int kRows = kAtOnce * kUnroll;
};

// eight elements as they lie in memory; the bits of the largest magnitude, as a float's; their codes
template <typename T> struct Eight;
template <> struct Eight<bf16_t> {
  u32x4 x;
  __device__ __forceinline__ void load(const bf16_t* at) { x = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(at)); }
  __device__ __forceinline__ uint32_t top() const {
    typedef __attribute__((ext_vector_type(2))) uint16_t u16x2;
    u16x2 most = __builtin_bit_cast(u16x2, x[0] & 0x7fff7fffu);
#pragma unroll
    for (int i = 1; i < 4; ++i) most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, x[i] & 0x7fff7fffu));
    return (uint32_t)max(most[0], most[1]) << 16;
  }
  __device__ __forceinline__ uint32_t codes(uint32_t byte) const {
    if (byte == 255u) return 0u;
    const float unit = fp4_unit(byte);
    const uint32_t w[4] = {x[0], x[1], x[2], x[3]};          // (a bit cast of a vector's element takes the first one)
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, w[0]), unit, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, w[1]), unit, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, w[2]), unit, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, w[3]), unit, 3);
    return c;
  }
};
template <> struct Eight<float> {
  float x[8];
  __device__ __forceinline__ void load(const float* at) { load8(at, x); }
  __device__ __forceinline__ uint32_t top() const { return top_bits8(x); }
  __device__ __forceinline__ uint32_t codes(uint32_t byte) const { return fp4_codes(x, byte); }
};

template <typename T, int D, bool SLOTS>
__global__ __launch_bounds__(kThreads) void store_fp4_kernel(StoreParams p) {
  using S = StoreShape<T, D>;
  const int lane_in_row = threadIdx.x % S::kLanes, row_in = threadIdx.x / S::kLanes, h = blockIdx.y;
  const bool second = !SLOTS && (int)blockIdx.x >= p.parts_a;
  const int first = (second ? (int)blockIdx.x - p.parts_a : (int)blockIdx.x) * S::kRows, n = second ? p.n_b : p.n_a;
  const int32_t* idx = second ? p.idx_b : p.idx_a;
  const bool values = !second && p.v;
  int64_t to[S::kUnroll];
  Eight<T> x[S::kUnroll], y[S::kUnroll];
  const T* k = reinterpret_cast<const T*>(p.k) + h * p.k_sh + lane_in_row * 8;
  const T* v = reinterpret_cast<const T*>(p.v) + h * p.v_sh + lane_in_row * 8;
  if constexpr (SLOTS) {
    // the rows lie one after the other: one product for a thread
    const int64_t k_at = (first + row_in) * p.k_st, v_at = (first + row_in) * p.v_st;
#pragma unroll
    for (int u = 0; u < S::kUnroll; ++u) {
      to[u] = -1;
      if (first + row_in + u * S::kAtOnce < n) {
        to[u] = p.slots[(int64_t)h * n + first + row_in + u * S::kAtOnce];
        x[u].load(k + (k_at + u * S::kAtOnce * p.k_st));
        if (values) y[u].load(v + (v_at + u * S::kAtOnce * p.v_st));
      }
      if (to[u] >= p.pool_rows) to[u] = -1;
    }
  } else {
    int from[S::kUnroll];
#pragma unroll
    for (int u = 0; u < S::kUnroll; ++u) {
      const int r = first + u * S::kAtOnce + row_in;
      from[u] = idx[(int64_t)h * n + min(r, n - 1)];
      to[u] = r < n ? (int64_t)h * (second ? p.n_b : p.cap) + r : -1;
    }
#pragma unroll
    for (int u = 0; u < S::kUnroll; ++u) {
      if ((uint32_t)from[u] >= (uint32_t)p.n_tokens) { from[u] = 0; to[u] = -1; }       // no token: nothing is stored
      x[u].load(k + from[u] * p.k_st);
      if (values) y[u].load(v + from[u] * p.v_st);
    }
  }
  // the scales of a row go out as one word, by its first lane
  auto store = [&](const Eight<T>& e, int64_t at, uint8_t* codes, uint8_t* scales) VEC_INLINE {
    if (at < 0) return;                                // the same for the lanes of a row
    const uint32_t byte = fp4_scale_byte(quad_max(e.top()));
    *reinterpret_cast<uint32_t*>(codes + at * fp4_code_bytes(D) + lane_in_row * 4) = e.codes(byte);
    uint32_t word = byte << lane_in_row / 4 * 8;
    if constexpr (D == 128) {
      word |= (uint32_t)__builtin_amdgcn_update_dpp(0, (int)word, 0x124, 0xf, 0xf, false);           // row_ror:4, row_ror:8
      word |= (uint32_t)__builtin_amdgcn_update_dpp(0, (int)word, 0x128, 0xf, 0xf, false);
      if (lane_in_row == 0) *reinterpret_cast<uint32_t*>(scales + at * 4) = word;
    } else {
      word |= (uint32_t)__builtin_amdgcn_update_dpp(0, (int)word, 0x141, 0xf, 0xf, false);           // the other half of eight lanes
      if (lane_in_row == 0) *reinterpret_cast<uint16_t*>(scales + at * 2) = (uint16_t)word;
    }
  };
#pragma unroll
  for (int u = 0; u < S::kUnroll; ++u) {
    store(x[u], to[u], second ? p.kb : p.ka, second ? p.kb_scale : p.ka_scale);
    if (values) store(y[u], to[u], p.va, p.va_scale);
  }
}

struct LoadParams {
  const uint8_t *codes, *scales;
  const int64_t* slots;
  int64_t n_rows, pool_rows;
  void* out;
};

constexpr int kLoadUnroll = 4;

template <typename T, int D>
__global__ __launch_bounds__(kThreads) void load_fp4_kernel(LoadParams p) {
  constexpr int kLanes = D / 8, kAtOnce = kThreads / kLanes;
  const int lane_in_row = threadIdx.x % kLanes;
  const int64_t first = (int64_t)blockIdx.x * kAtOnce * kLoadUnroll + threadIdx.x / kLanes;
  int64_t from[kLoadUnroll];
  uint32_t codes[kLoadUnroll], byte[kLoadUnroll];
#pragma unroll
  for (int u = 0; u < kLoadUnroll; ++u) {
    const int64_t r = min(first + u * kAtOnce, p.n_rows - 1);
    from[u] = p.slots ? p.slots[r] : r;
  }
#pragma unroll
  for (int u = 0; u < kLoadUnroll; ++u) {
    codes[u] = byte[u] = 0;                  // no row: zeros
    if (from[u] >= 0 && from[u] < p.pool_rows) {
      codes[u] = *reinterpret_cast<const uint32_t*>(p.codes + from[u] * fp4_code_bytes(D) + lane_in_row * 4);
      byte[u] = p.scales[from[u] * fp4_scale_bytes(D) + lane_in_row / 4];
    }
  }
#pragma unroll
  for (int u = 0; u < kLoadUnroll; ++u) {
    const int64_t r = first + u * kAtOnce;
    if (r >= p.n_rows) return;
    const float unit = fp4_unit(byte[u]);
    T* out = reinterpret_cast<T*>(p.out) + r * D + lane_in_row * 8;
    if constexpr (sizeof(T) == 2) {
      u32x4 x;
      for_each_constant<4>([&](auto i) VEC_INLINE { x[(int)i] = fp4_pair_bf16<decltype(i)::value>(codes[u], unit); });
      __builtin_nontemporal_store(x, reinterpret_cast<u32x4*>(out));
    } else {
      float x[8];
      for_each_constant<4>([&](auto i) VEC_INLINE {
        const f32x2 two = fp4_pair_f32<decltype(i)::value>(codes[u], unit);
        x[2 * i] = two[0];
        x[2 * i + 1] = two[1];
      });
      __builtin_nontemporal_store(f32x4{x[0], x[1], x[2], x[3]}, reinterpret_cast<f32x4*>(out));
      __builtin_nontemporal_store(f32x4{x[4], x[5], x[6], x[7]}, reinterpret_cast<f32x4*>(out + 4));
    }
  }
}

template <typename T, int D> int run_store(StoreParams p, int heads, hipStream_t stream) {
  constexpr int rows = StoreShape<T, D>::kRows;
  p.parts_a = (int)(((int64_t)p.n_a + rows - 1) / rows);
  const int64_t parts = p.parts_a + ((int64_t)p.n_b + rows - 1) / rows;
  if (parts == 0) return VECTOR_OK;
  if (p.slots) VEC_LAUNCH(K_FP4_ROWS, (store_fp4_kernel<T, D, true>), dim3((unsigned)parts, heads), dim3(kThreads), 0, stream, p);
  else VEC_LAUNCH(K_FP4_ROWS, (store_fp4_kernel<T, D, false>), dim3((unsigned)parts, heads), dim3(kThreads), 0, stream, p);
  VEC_HIP(hipGetLastError());
  return VECTOR_OK;
}

template <typename T, int D> int run_load(const LoadParams& p, hipStream_t stream) {
  constexpr int rows = kThreads / (D / 8) * kLoadUnroll;
  const int64_t grid = (p.n_rows + rows - 1) / rows;
  VEC_LAUNCH(K_FP4_ROWS, (load_fp4_kernel<T, D>), dim3((unsigned)grid), dim3(kThreads), 0, stream, p);
  VEC_HIP(hipGetLastError());
  return VECTOR_OK;
}

}  // namespace

int launch_store_fp4(const vector_shape& s, const Fp4Rows& r, hipStream_t stream) {
  StoreParams p = {};
  p.k = r.k; p.v = r.v;
  p.k_st = s.k_stride_tok ? s.k_stride_tok : s.head_dim;
  p.k_sh = s.k_stride_head ? s.k_stride_head : p.k_st * s.seq_len;
  p.v_st = s.v_stride_tok ? s.v_stride_tok : s.head_dim;
  p.v_sh = s.v_stride_head ? s.v_stride_head : p.v_st * s.seq_len;
  p.idx_a = r.idx_retain; p.idx_b = r.idx_approx; p.slots = r.slots;
  p.pool_rows = r.slots ? r.pool_rows : INT64_MAX;
  p.ka = r.k_ret; p.ka_scale = r.k_ret_scale; p.va = r.v_ret; p.va_scale = r.v_ret_scale; p.kb = r.k_apx; p.kb_scale = r.k_apx_scale;
  p.n_tokens = s.seq_len; p.n_a = r.n_retain; p.n_b = r.n_approx; p.cap = r.cap_retain;
  if (s.dtype == VECTOR_BF16) return s.head_dim == 128 ? run_store<bf16_t, 128>(p, s.n_kv_heads, stream) : run_store<bf16_t, 64>(p, s.n_kv_heads, stream);
  return s.head_dim == 128 ? run_store<float, 128>(p, s.n_kv_heads, stream) : run_store<float, 64>(p, s.n_kv_heads, stream);
}

int launch_load_fp4(int64_t n_rows, int head_dim, int dtype, const uint8_t* codes, const uint8_t* scales, int64_t pool_rows, const int64_t* slots,
                    void* out, hipStream_t stream) {
  const LoadParams p = {codes, scales, slots, n_rows, pool_rows, out};
  if (dtype == VECTOR_BF16) return head_dim == 128 ? run_load<bf16_t, 128>(p, stream) : run_load<bf16_t, 64>(p, stream);
  return head_dim == 128 ? run_load<float, 128>(p, stream) : run_load<float, 64>(p, stream);
}

}  // namespace vec
