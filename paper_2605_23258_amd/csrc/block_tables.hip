// Blocks of a paged cache for the requests of a batch, and the slots of their tokens, from lengths on the GPU (vector_block_tables).
//
// Which blocks a request gets follows from the requests before it: one running sum over the batch of the blocks they need
// and one of their tokens.  There is one launch, without workspace: every workgroup makes both sums for itself (a batch of up to kMaxRequests lengths,
// which lie in the L2 after the first workgroup's read) and then writes its part of the slots or of the table.  A second launch that
// only read the sums would cost more than they do.  Small batches are a chain of two trips to memory (lengths; block ids); large ones are
// bound by the writes, 8 bytes per token and KV head: two tokens a thread, 16 bytes a store.
#include "common.hpp"
#include "launch.hpp"

namespace vec {

namespace {

constexpr int kThreads = 256, kWaves = kThreads / kWave;
constexpr int kTokensPerGroup = 512;         // slots a workgroup writes for every KV head
constexpr int kHeadsAtOnce = 4;
constexpr int kPairsPerGroup = 8;            // (request, KV head) rows of the table a workgroup writes

struct TableParams {
  const int32_t *held, *len, *free_blocks, *used;
  int32_t *table, *live, *counts;
  int64_t* slots;
  int B, H, shift, per_seq, n_free, n_slots;
  int slot_groups;                           // workgroups that write slots, those that write the table follow
};

// A request's lengths as they count: none below zero, and none below what it holds
struct Request { int held, len; };
__device__ __forceinline__ Request request(const TableParams& p, int b) {
  const int held = p.held ? max(p.held[b], 0) : 0;
  return {held, max(p.len[b], held)};
}
__device__ __forceinline__ int blocks_of(int rows, int shift) { return (int)(((int64_t)rows + (1 << shift) - 1) >> shift); }
// blocks it asks for, for one KV head; a request longer than a row of the table asks for none, and is not admitted
__device__ __forceinline__ bool too_long(const TableParams& p, const Request& r) { return blocks_of(r.len, p.shift) > p.per_seq; }
__device__ __forceinline__ int wanted(const TableParams& p, const Request& r) {
  return too_long(p, r) ? 0 : blocks_of(r.len, p.shift) - blocks_of(r.held, p.shift);
}
// blocks, tokens: of the requests up to this one
__device__ __forceinline__ bool admitted(const TableParams& p, const Request& r, int blocks, int tokens) {
  if (too_long(p, r)) return false;
  return (wanted(p, r) == 0 || blocks <= p.n_free) && (!p.slots || r.len == r.held || tokens <= p.n_slots);
}

// running sum over the lanes that stops at 2^32 - 1 (of numbers below 2^31)
template <int CTRL, int ROW_MASK> __device__ __forceinline__ uint32_t add_upto(uint32_t v) {
  return __builtin_elementwise_add_sat(v, (uint32_t)dpp_take<CTRL, ROW_MASK>((int)v));
}
__device__ __forceinline__ uint32_t wave_incl_scan_upto(uint32_t v) {
  v = add_upto<0x111, 0xf>(v);
  v = add_upto<0x112, 0xf>(v);
  v = add_upto<0x114, 0xf>(v);
  v = add_upto<0x118, 0xf>(v);
  v = add_upto<0x142, 0xa>(v);
  return add_upto<0x143, 0xc>(v);
}

__global__ __launch_bounds__(kThreads) void block_tables_kernel(TableParams p) {
  // of request b - 1: blocks up to it, of all KV heads; tokens up to it; and its lengths
  extern __shared__ __align__(16) int lds[];
  __shared__ int wave_blocks[kWaves];
  __shared__ uint32_t wave_tokens[kWaves];
  int *blocks = lds, *tokens = lds + p.B + 1;
  Request* requests = reinterpret_cast<Request*>(lds + 2 * (p.B + 1));
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  // the list without what calls before have taken from its front; without a list, the first of the ids
  const int first_id = p.used ? min(max(*p.used, 0), p.n_free) : 0;
  p.n_free -= first_id;
  if (p.free_blocks) p.free_blocks += first_id;
  int base_blocks = 0;                       // at most B * H * per_seq, which the host has checked
  uint32_t base_tokens = 0;
  if (tid == 0) blocks[0] = tokens[0] = 0;
  for (int b0 = 0; b0 < p.B; b0 += kThreads) {
    const int b = b0 + tid;
    const Request r = b < p.B ? request(p, b) : Request{0, 0};
    int nb = wave_incl_scan_dpp(wanted(p, r) * p.H);
    uint32_t nt = wave_incl_scan_upto((uint32_t)(r.len - r.held));
    if (b0 > 0) __syncthreads();             // the waves' sums of the round before have been read
    if (lane == 63) { wave_blocks[wave] = nb; wave_tokens[wave] = nt; }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      if (w < wave) { nb += wave_blocks[w]; nt = __builtin_elementwise_add_sat(nt, wave_tokens[w]); }
    }
    nb += base_blocks;
    nt = __builtin_elementwise_add_sat(nt, base_tokens);
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      base_blocks += wave_blocks[w];
      base_tokens = __builtin_elementwise_add_sat(base_tokens, wave_tokens[w]);
    }
    if (b < p.B) {
      blocks[b + 1] = nb;
      tokens[b + 1] = (int)min(nt, (uint32_t)INT32_MAX);        // slots end before that
      requests[b] = r;
    }
  }
  __syncthreads();

  if ((int)blockIdx.x < p.slot_groups) {
    // slots: a thread takes two tokens for all KV heads; neighbours are tokens of one request, mostly
    static_assert(kTokensPerGroup == 2 * kThreads, "one pair a thread");
    const int t = (int)blockIdx.x * kTokensPerGroup + 2 * tid;         // below 2^31: n_slots is, and of no more groups than it takes
    if (t < p.n_slots) {
      // the request b with tokens[b] <= t < tokens[b + 1]
      int lo = 0, hi = p.B;                  // tokens[lo] <= t; hi == B or t < tokens[hi]
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (tokens[mid] <= t) lo = mid; else hi = mid;
      }
      // where a token's block id lies: in the free list, or (a block that the request holds, which this launch does not write) in the
      // table, and how far the next KV head's lies behind it
      const int32_t* at[2];
      int step[2], row[2], id[2];
      bool ok[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        if (i == 1) {
          while (lo + 1 < p.B && tokens[lo + 1] <= t + 1) ++lo;
        }
        const Request r = requests[lo];
        ok[i] = t + i < tokens[lo + 1] && admitted(p, r, blocks[lo + 1], tokens[lo + 1]);      // behind the last token there are none
        const int pos = r.held + (t + i - tokens[lo]), before = blocks_of(r.held, p.shift), n = wanted(p, r), block = pos >> p.shift;
        row[i] = pos & ((1 << p.shift) - 1);
        const bool fresh = block >= before;
        id[i] = blocks[lo] + block - before;
        step[i] = fresh ? n : p.per_seq;
        at[i] = fresh ? (p.free_blocks ? p.free_blocks + id[i] : nullptr) : p.table + (int64_t)lo * p.H * p.per_seq + block;
      }
      int64_t* to = p.slots + t;
      const bool both = t + 1 < p.n_slots;
      for (int h0 = 0; h0 < p.H; h0 += kHeadsAtOnce) {
        int64_t slot[kHeadsAtOnce][2];
#pragma unroll
        for (int u = 0; u < kHeadsAtOnce; ++u)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const int h = min(h0 + u, p.H - 1);
            int block = first_id + id[i] + h * step[i];
            if (ok[i] && at[i]) block = at[i][(int64_t)h * step[i]];
            slot[u][i] = ok[i] ? ((int64_t)block << p.shift) + row[i] : -1;
          }
#pragma unroll
        for (int u = 0; u < kHeadsAtOnce; ++u) {
          if (h0 + u >= p.H) break;
          int64_t* out = to + (int64_t)(h0 + u) * p.n_slots;
          if (both) {
            typedef __attribute__((ext_vector_type(2), aligned(8))) int64_t i64x2;
            *reinterpret_cast<i64x2*>(out) = i64x2{slot[u][0], slot[u][1]};
          } else {
            *out = slot[u][0];
          }
        }
      }
    }
    return;
  }
  const int group = blockIdx.x - p.slot_groups;
  if (group == 0) {
    for (int b = tid; b < p.B; b += kThreads) {
      const Request r = requests[b];
      p.live[b] = admitted(p, r, blocks[b + 1], tokens[b + 1]) ? r.len : r.held;
    }
  }
  if (group == 0 && wave == 0) {
    // blocks taken: those of the admitted requests, which are the first ones that ask for any
    int taken = 0;
    for (int b = lane; b < p.B; b += kWave) {
      const Request r = requests[b];
      if (wanted(p, r) > 0 && admitted(p, r, blocks[b + 1], tokens[b + 1])) taken = max(taken, blocks[b + 1]);
    }
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) taken = max(taken, __shfl_xor(taken, o, kWave));
    if (lane == 0) {
      p.counts[0] = taken;
      p.counts[1] = blocks[p.B];
      p.counts[2] = tokens[p.B];
    }
  }
  const int pairs = p.B * p.H;
  for (int pair = group * kPairsPerGroup + wave; pair < min((group + 1) * kPairsPerGroup, pairs); pair += kWaves) {
    const int b = pair / p.H, h = pair % p.H;
    const Request r = requests[b];
    const bool ok = admitted(p, r, blocks[b + 1], tokens[b + 1]);
    const int before = blocks_of(r.held, p.shift), n = ok ? wanted(p, r) : 0, first = blocks[b] + h * n;
    int32_t* row = p.table + (int64_t)pair * p.per_seq;
    const int from = p.held ? before : 0, to = p.held ? before + n : p.per_seq;      // a new table is written whole
    for (int c = from + lane; c < to; c += kWave) {
      int id = 0;
      if (c - before < n) id = p.free_blocks ? p.free_blocks[first + c - before] : first_id + first + c - before;
      row[c] = id;
    }
  }
}

}  // namespace

int launch_block_tables(const vector_blocks& v, int32_t* table, int32_t* live, int64_t* slots, int64_t n_slots, int32_t* counts, hipStream_t stream) {
  TableParams p = {};
  p.held = v.len_held; p.len = v.len; p.free_blocks = v.free_blocks; p.used = v.n_used;
  p.table = table; p.live = live; p.counts = counts; p.slots = n_slots > 0 ? slots : nullptr;
  p.B = v.batch; p.H = v.n_kv_heads; p.per_seq = v.blocks_per_seq; p.n_free = v.n_free; p.n_slots = (int)n_slots;
  while ((1 << p.shift) < v.block_rows) ++p.shift;
  p.slot_groups = (int)((n_slots + kTokensPerGroup - 1) / kTokensPerGroup);
  const int table_groups = (p.B * p.H + kPairsPerGroup - 1) / kPairsPerGroup;
  const size_t lds = 2 * (p.B + 1) * sizeof(int) + p.B * sizeof(Request);
  VEC_HIP(set_max_lds(reinterpret_cast<const void*>(block_tables_kernel), lds));
  VEC_LAUNCH(K_BLOCK_TABLES, block_tables_kernel, dim3(p.slot_groups + table_groups), dim3(kThreads), lds, stream, p);
  VEC_HIP(hipGetLastError());
  return VECTOR_OK;
}

}  // namespace vec
