// What the decode kernels share: where a sequence's rows lie, which of them a workgroup takes, and the merge of the
// workgroups' partial results.
#pragma once
#include "common.hpp"
#include "decode_rows.hpp"
#include "launch.hpp"

namespace vec {

struct DecodeParams {
  const void* q; const void* k_ret; const void* v_ret; const void* k_apx; const void* W;
  const int32_t* len_retain;
  // per-sequence capacities and first rows of the sequences' blocks (all null: uniform blocks)
  const int32_t* cap_retain_seq; const int32_t* n_approx_seq;
  const int64_t* ret_row_start; const int64_t* apx_row_start;
  // the step's own token (null: none): exact key and value [B, Hkv, D]; it is attended as row
  // len_retain[b] of the retained segment and stored there when the block has room
  const void* k_new; const void* v_new;
  // paged retained segments (null: contiguous): block ids [B, Hkv, blocks_per_seq]; a block is
  // 1 << block_shift rows of the k_ret / v_ret pools
  const int32_t* block_table;
  int block_shift, blocks_per_seq;
  void* out;
  float* part;            // [B, Hkv, S, 2*G + G*D] floats: (m, l)[G], acc[G][D]
  int B, Hq, Hkv, cap_retain, n_approx;
  int splits_ret, splits_apx;   // workgroups per (sequence, head) on each segment
  int by_kind;                  // the grid is (KV head, sequence, split) and not (split, KV head, sequence)
  // Sequences of different lengths (see PlannedSplits): [B, Hkv, 2] (first partial, number of partials) of either segment; and what
  // a step of approximated rows counts in steps of retained ones
  int2* plan;
  float plan_apx;
  int plan_most_retained;       // workgroups
  int64_t w_sh;           // element stride between per-head W
  float c2;               // scale * log2(e)
  int literal;            // approximated rows: rebuild v_hat = k W per row instead of (sum p k) W
  int only_values;        // the partials of approximated rows are values already: W is not the merge's
  int out_f32;            // store the result as fp32 whatever the cache dtype
};

// Where the rows of one (sequence, KV head) lie: row offsets into k_ret / v_ret and into k_apx,
// the live length of the retained segment and the length of the approximated one.
struct SegmentRows {
  size_t ret_row0, apx_row0;
  int len_retain, n_approx, new_row, cap;
  const int32_t* blocks;      // paged: this (sequence, head)'s block ids; ret_row0 is then 0
  int block_shift;
};
// row r of the retained segment as a row of the k_ret / v_ret arrays.  PAGED is a template
// argument of the kernels: the lookups cost registers that the contiguous layout should not pay.
template <bool PAGED>
__device__ __forceinline__ size_t retained_row(const SegmentRows& s, int r) {
  if (PAGED) return ((size_t)s.blocks[r >> s.block_shift] << s.block_shift) + (size_t)(r & ((1 << s.block_shift) - 1));
  return s.ret_row0 + (size_t)r;
}
// of a sequence with the capacity, approximated rows, live retained rows and first rows given
__device__ __forceinline__ SegmentRows sequence_rows(const DecodeParams& p, int b, int h, int cap, int n_approx, int live, int64_t ret0, int64_t apx0) {
  SegmentRows s;
  s.n_approx = n_approx;
  s.ret_row0 = (size_t)ret0 + (size_t)h * cap;
  s.apx_row0 = (size_t)apx0 + (size_t)h * n_approx;
  s.blocks = nullptr;
  s.block_shift = 0;
  if (p.block_table) {
    s.blocks = p.block_table + ((size_t)b * p.Hkv + h) * p.blocks_per_seq;
    s.block_shift = p.block_shift;
    s.ret_row0 = 0;
  }
  s.len_retain = live;
  s.cap = cap;
  s.new_row = -1;
  if (p.k_new) { s.new_row = s.len_retain; s.len_retain += 1; }      // the new token is the last live row
  return s;
}
__device__ __forceinline__ SegmentRows segment_rows(const DecodeParams& p, int b, int h) {
  int cap = p.cap_retain, n_approx = p.n_approx;
  int64_t ret0 = (int64_t)b * p.Hkv * cap, apx0 = (int64_t)b * p.Hkv * n_approx;
  if (p.cap_retain_seq) {
    cap = max(p.cap_retain_seq[b], 0);
    n_approx = max(p.n_approx_seq[b], 0);
    ret0 = p.ret_row_start[b];
    apx0 = p.apx_row_start[b];
  }
  return sequence_rows(p, b, h, cap, n_approx, min(max(p.len_retain[b], 0), cap), ret0, apx0);
}

constexpr int DT_ = 256;          // threads per workgroup
constexpr int DW = DT_ / kWave;   // waves

// Rows of one segment of one (sequence, KV head) that a workgroup takes
struct SplitRows {
  int b, h;
  bool is_apx;
  int begin, end;
  size_t slot;                    // of the partial
  SegmentRows seg;
};
// One range per workgroup, the grid says which: as many splits for every sequence.  Ranges are multiples of STEP rows, so
// that loads stay aligned to it.
template <int STEP> __device__ __forceinline__ SplitRows grid_split(const DecodeParams& p) {
  SplitRows r;
  const int split = p.by_kind ? blockIdx.z : blockIdx.x;
  r.h = p.by_kind ? blockIdx.x : blockIdx.y;
  r.b = p.by_kind ? blockIdx.y : blockIdx.z;
  r.seg = segment_rows(p, r.b, r.h);
  r.is_apx = split >= p.splits_ret;
  const int len = r.is_apx ? r.seg.n_approx : r.seg.len_retain;
  const int n_sp = r.is_apx ? p.splits_apx : p.splits_ret, sp = r.is_apx ? split - p.splits_ret : split;
  const int steps = (len + STEP - 1) / STEP;
  r.begin = (int)((int64_t)steps * sp / n_sp) * STEP;
  r.end = min(len, (int)((int64_t)steps * (sp + 1) / n_sp) * STEP);
  r.slot = ((size_t)r.b * p.Hkv + r.h) * (p.splits_ret + p.splits_apx) + split;
  return r;
}

// Sequences of different lengths: the same share of the work for every workgroup, wherever one sequence's rows end and
// the next one's begin.  With as many splits for every sequence the longest are waited for.  The host does not know the live lengths;
// every workgroup adds the work up itself, lane b that of sequence b.  The retained rows are one line, sequence after
// sequence, head after head, and the approximated rows another; the first workgroups share the first, the others the second, so
// that a CU, which gets two workgroups half a grid apart, has one of each (all of both lines in one, 32 sequences of up to
// 32768 tokens 89 us, now 86; 16 of them 52.5, 48.6).  A workgroup takes the granules that begin in its share; the arithmetic is in
// decode_rows.hpp.  The workgroup with a segment's first granule says in `plan` where its partials begin and how many there are.
//   A step, us, as many splits for every sequence / this: 24 sequences of 4000 to 16000 tokens on rotated keys 51.5 / 44.6, plain 43.1 /
//   40.4; 16 of 8192 to 32768 62.2 / 52.2, plain 55.2 / 48.6.
struct PlannedSequence { int cap, n_approx, live; long long ret0, apx0; };
struct PlannedSplits {
  const DecodeParams& p;
  int id, share, lo, hi, log_rows;           // a granule is 1 << log_rows rows
  int b, h, at;                              // the segment at hand begins at `at`
  bool is_apx, done;
  PlannedSequence s;                         // sequence b
  // Scalars are kept scalar: the compiler would keep in vector registers what follows from a float or from memory.
  static __device__ __forceinline__ int same(int x) { return __builtin_amdgcn_readfirstlane(x); }
  static __device__ __forceinline__ long long same(long long x) { return ((long long)same((int)(x >> 32)) << 32) | (uint32_t)same((int)x); }
  __device__ __forceinline__ int granules(int len) const { return plan_granules(len, log_rows); }
  // of a sequence with nothing cached an empty granule, whose workgroup writes the empty partial
  __device__ __forceinline__ int granules_ret(const PlannedSequence& x) const {
    const int n = granules(x.live + (p.k_new ? 1 : 0));
    return x.n_approx == 0 ? max(n, 1) : n;
  }
  static __device__ __forceinline__ PlannedSequence sequence(const DecodeParams& p, int i) {
    const int cap = planned_rows(p.cap_retain, p.cap_retain_seq[i]);
    return {cap, planned_rows(p.n_approx, p.n_approx_seq[i]), min(max(p.len_retain[i], 0), cap), p.ret_row_start[i], p.apx_row_start[i]};
  }
  __device__ __forceinline__ explicit PlannedSplits(const DecodeParams& p_) : p(p_) {
    const int lane = threadIdx.x & 63;
    const PlannedSequence x = sequence(p, min(lane, p.B - 1));
    // granules so long that a line stays shorter than kMaxPlanUnits: 32 rows unless the cache were larger than the memory
    log_rows = kLogGranule;
    int len_r = plan_length(granules_ret(x)), len_a = plan_length(granules(x.n_approx));
    float top_r = wave_max_dpp((float)len_r), top_a = wave_max_dpp((float)len_a);
    while (__builtin_expect(plan_too_long(fmaxf(top_r, top_a), p.B, p.Hkv, log_rows), 0)) {
      log_rows = same(log_rows + 1);
      len_r = plan_length(granules_ret(x));
      len_a = plan_length(granules(x.n_approx));
      top_r = wave_max_dpp((float)len_r);
      top_a = wave_max_dpp((float)len_a);
    }
    const int seq_r = lane < p.B ? len_r * p.Hkv : 0, seq_a = lane < p.B ? len_a * p.Hkv : 0;
    const int upto_r = wave_incl_scan_dpp(seq_r), upto_a = wave_incl_scan_dpp(seq_a);
    const int total_r = __builtin_amdgcn_readlane(upto_r, 63), total_a = __builtin_amdgcn_readlane(upto_a, 63), wgs = gridDim.x;
    const int wgs_r = same(plan_retained(wgs, p.plan_most_retained, total_r, total_a, __builtin_amdgcn_rcpf((float)total_r + (float)total_a * p.plan_apx)));
    id = blockIdx.x;
    is_apx = id >= wgs_r;
    const int mine = is_apx ? id - wgs_r : id, total = is_apx ? total_a : total_r;
    share = same(plan_share(total, is_apx ? top_a : top_r, __builtin_amdgcn_rcpf((float)(is_apx ? wgs - wgs_r : wgs_r))));
    lo = mine * share;
    hi = lo + share;
    done = lo >= total;                      // of small caches fewer workgroups than the grid has
    b = h = at = 0;
    s = PlannedSequence{};
    if (done) return;
    const int upto = is_apx ? upto_a : upto_r, of_sequence = is_apx ? seq_a : seq_r;
    b = __popcll(__ballot(upto <= lo));
    at = __builtin_amdgcn_readlane(upto - of_sequence, b);
    const int head = __builtin_amdgcn_readlane(is_apx ? len_a : len_r, b);
    h = same(plan_head(lo - at, head, __builtin_amdgcn_rcpf((float)head)));
    at += h * head;
    auto of_b = [&](int v) VEC_INLINE { return __builtin_amdgcn_readlane(v, b); };
    auto of_b64 = [&](long long v) VEC_INLINE { return ((long long)of_b((int)(v >> 32)) << 32) | (uint32_t)of_b((int)v); };
    s = {of_b(x.cap), of_b(x.n_approx), of_b(x.live), of_b64(x.ret0), of_b64(x.apx0)};
  }
  // the next rows of this workgroup; false: there are none
  __device__ __forceinline__ bool next(SplitRows& r) {
    while (!done) {
      const int n_r = granules_ret(s), n_a = granules(s.n_approx), n = is_apx ? n_a : n_r;
      const PlanPiece piece = plan_piece(at, n, lo, share);
      const int pair = b * p.Hkv + h, place = plan_place(id, pair, is_apx, p.B * p.Hkv);
      const bool any = piece.first < piece.last;
      if (any) {
        r.b = b; r.h = h; r.is_apx = is_apx;
        r.seg = sequence_rows(p, b, h, s.cap, s.n_approx, s.live, s.ret0, s.apx0);
        r.begin = piece.first << log_rows;
        r.end = (int)min((int64_t)(is_apx ? r.seg.n_approx : r.seg.len_retain), (int64_t)piece.last << log_rows);
        r.slot = (size_t)place;
        if (piece.first == 0 && threadIdx.x == 0) {
          p.plan[2 * pair + (is_apx ? 1 : 0)] = make_int2(place, plan_partials(at, n, lo, share));
          if ((is_apx ? n_r : n_a) == 0) p.plan[2 * pair + (is_apx ? 0 : 1)] = make_int2(0, 0);
        }
      }
      at += plan_length(n);
      done = at >= hi;
      if (++h == p.Hkv) {
        h = 0;
        if (++b == p.B) done = true;
        if (!done) {
          const PlannedSequence x = sequence(p, b);
          s = {same(x.cap), same(x.n_approx), same(x.live), same(x.ret0), same(x.apx0)};
        }
      }
      if (any) return true;
    }
    return false;
  }
};

// what a workgroup of a split launch does
template <int STEP, bool PLANNED, typename F> __device__ __forceinline__ void for_split_rows(const DecodeParams& p, F attend) {
  if constexpr (PLANNED) {
    static_assert(STEP == kStepGranules << kLogGranule, "a step of the bf16 kernel");
    PlannedSplits splits(p);
    SplitRows r;
    while (splits.next(r)) {
      int tid = threadIdx.x;
      asm volatile("" : "+v"(tid));                  // what is made of it would be kept in registers from range to range
      attend(r, tid);
      __syncthreads();                               // LDS may be written again
    }
  } else {
    attend(grid_split<STEP>(p), (int)threadIdx.x);
  }
}

// The merge of a split launch's partials (decode_attn.hip): weights the splits, applies W to the sums of approximated keys, divides, stores, and
// makes a step's own token a live row.  dtype: of W and out
int launch_decode_merge(const DecodeParams& p, int dtype, int head_dim, hipStream_t stream);

}  // namespace vec
