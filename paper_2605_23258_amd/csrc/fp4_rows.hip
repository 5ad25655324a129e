// Key and value rows into 4 bits and back: vector_compact_fp4, vector_store_fp4, vector_load_fp4.
//
// What bounds them is memory: a bf16 row of 128 elements is 256 bytes, in 4 bits 68.  Eight elements go to a lane (16 or 32 bytes
// in, four bytes of codes out), so D / 8 adjacent lanes hold a row, every load of a wave covers whole rows, and the four lanes of a
// block find its largest magnitude by two exchanges inside the group of four.
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

// A workgroup takes kRows rows of a head: keys and values of the first kind of rows, keys of the second.
template <typename T, int D> struct StoreShape {
  static constexpr int kLanes = D / 8;                       // of a row
  static constexpr int kAtOnce = kThreads / kLanes;          // rows
  static constexpr int kUnroll = 2;
  static constexpr int kRows = kAtOnce * kUnroll;
};

template <typename T, int D>
__global__ __launch_bounds__(kThreads) void store_fp4_kernel(StoreParams p) {
  using S = StoreShape<T, D>;
  const int lane_in_row = threadIdx.x % S::kLanes, row_in = threadIdx.x / S::kLanes, h = blockIdx.y;
  const bool second = (int)blockIdx.x >= p.parts_a;
  const int first = (second ? (int)blockIdx.x - p.parts_a : (int)blockIdx.x) * S::kRows, n = second ? p.n_b : p.n_a;
  const int32_t* idx = second ? p.idx_b : p.idx_a;
  const bool values = !second && p.v;
  int64_t to[S::kUnroll];
  float x[2][S::kUnroll][8];
#pragma unroll
  for (int u = 0; u < S::kUnroll; ++u) {
    const int r = first + u * S::kAtOnce + row_in;
    to[u] = -1;
    int from = r;
    if (r < n) {
      if (idx) from = idx[(int64_t)h * n + r];
      to[u] = p.slots ? p.slots[(int64_t)h * n + r] : (int64_t)h * (second ? p.n_b : p.cap) + r;
      if ((uint32_t)from >= (uint32_t)p.n_tokens || to[u] >= p.pool_rows) to[u] = -1;
    }
    if (to[u] >= 0) {
      load8(reinterpret_cast<const T*>(p.k) + h * p.k_sh + from * p.k_st + lane_in_row * 8, x[0][u]);
      if (values) load8(reinterpret_cast<const T*>(p.v) + h * p.v_sh + from * p.v_st + lane_in_row * 8, x[1][u]);
    }
  }
#pragma unroll
  for (int u = 0; u < S::kUnroll; ++u) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      if ((t == 1 && !values) || to[u] < 0) continue;          // the same for the lanes of a row
      const uint32_t byte = fp4_scale_byte(quad_max(top_bits8(x[t][u])));
      uint8_t* codes = t ? p.va : second ? p.kb : p.ka;
      uint8_t* scales = t ? p.va_scale : second ? p.kb_scale : p.ka_scale;
      *reinterpret_cast<uint32_t*>(codes + to[u] * fp4_code_bytes(D) + lane_in_row * 4) = fp4_codes(x[t][u], byte);
      if (lane_in_row % 4 == 0) scales[to[u] * fp4_scale_bytes(D) + lane_in_row / 4] = (uint8_t)byte;
    }
  }
}

struct LoadParams {
  const uint8_t *codes, *scales;
  const int64_t* slots;
  int64_t n_rows, pool_rows;
  void* out;
};

template <typename T, int D>
__global__ __launch_bounds__(kThreads) void load_fp4_kernel(LoadParams p) {
  constexpr int kLanes = D / 8, kAtOnce = kThreads / kLanes;
  const int lane_in_row = threadIdx.x % kLanes;
  const int64_t r = (int64_t)blockIdx.x * kAtOnce + threadIdx.x / kLanes;
  if (r >= p.n_rows) return;
  const int64_t from = p.slots ? p.slots[r] : r;
  float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  if (from >= 0 && from < p.pool_rows) {
    const uint32_t codes = *reinterpret_cast<const uint32_t*>(p.codes + from * fp4_code_bytes(D) + lane_in_row * 4);
    const float unit = fp4_unit(p.scales[from * fp4_scale_bytes(D) + lane_in_row / 4]);
    for_each_constant<4>([&](auto i) VEC_INLINE {
      const f32x2 two = fp4_pair_f32<decltype(i)::value>(codes, unit);
      x[2 * i] = two[0];
      x[2 * i + 1] = two[1];
    });
  }
  T* out = reinterpret_cast<T*>(p.out) + r * D + lane_in_row * 8;
  if constexpr (sizeof(T) == 2) {
    *reinterpret_cast<uint4*>(out) = make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
  } else {
    *reinterpret_cast<f32x4*>(out) = f32x4{x[0], x[1], x[2], x[3]};
    *reinterpret_cast<f32x4*>(out + 4) = f32x4{x[4], x[5], x[6], x[7]};
  }
}

template <typename T, int D> int run_store(StoreParams p, int heads, hipStream_t stream) {
  constexpr int rows = StoreShape<T, D>::kRows;
  p.parts_a = (int)(((int64_t)p.n_a + rows - 1) / rows);
  const int64_t parts = p.parts_a + ((int64_t)p.n_b + rows - 1) / rows;
  if (parts == 0) return VECTOR_OK;
  VEC_LAUNCH(K_FP4_ROWS, (store_fp4_kernel<T, D>), dim3((unsigned)parts, heads), dim3(kThreads), 0, stream, p);
  VEC_HIP(hipGetLastError());
  return VECTOR_OK;
}

template <typename T, int D> int run_load(const LoadParams& p, hipStream_t stream) {
  constexpr int rows = kThreads / (D / 8);
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
