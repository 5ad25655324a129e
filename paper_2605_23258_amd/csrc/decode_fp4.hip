// Decode attention over caches held in 4 bits (vector_decode_attn_fp4, vector_decode_step_fp4): the same sum as over caches in 16 or 32 bits
// (decode_attn.hip), one softmax over the live retained rows and the approximated ones, z = sum p k over the latter, the same
// partial results and the same merge.
//
// What bounds it is memory, 136 bytes for the key and the value of a token at 128 dims, against 512 in bf16; but a quarter of the bytes
// leaves a quarter of the time for a row's arithmetic, which comes close behind it.  Both products run on the matrix cores with fp32 sums.
// An element in 4 bits times its scale has two significant bits and is a bf16 number exactly; the weights go in as parts of eight bits each.
//
// A wave takes 32 rows at a time and waits for no other before the end.  Their codes and scales go from memory straight into a ring of its
// own in LDS (Fp4Stage), past the caches (16 whole caches of 32768 tokens 105 us with them, 90 without: 6.3 TB/s), so that what is on its way
// takes no registers, and are read back in the matrix cores' order:
//   scores   S[t][g] = sum_e K[t][e] q[g][e]      A = K: lane (m, quarter) holds D / 4 consecutive elements of a row, which is one read and
//                                                  one scale.  128 dims: as they are, in 4 bits with their scales, against query rows in
//                                                  two fp8 parts (kMx); 64 dims and fp32: converted to bf16
//   output   O[j][g] += sum_t R[t][j] P[t][g]     A = R^T: lane (m, quarter) holds dims D / 16 m .. of eight rows, 8 quarter ..; the conversion
//                                                  hands out two neighbouring dims of one row
// Row 4 a + i of score tile u is token 8 a + 4 u + i, so that the eight weights that a lane gets from both score tiles are those
// of the eight rows that it holds of R.  R is the values, or for approximated rows the keys, read a second time in the other order;
// under ROPE these are turned back by their positions first.
//
// Sixteen columns, COLS of them for different query rows:
//   4   columns 4 and 12 on take what the weights' leading bits leave.  The contraction runs over (row, even or odd dim), as the conversion hands
//       them out; the weights of columns below 8 are zero at odd dims, those from 8 on at even ones, so that a product gives both dims,
//       each in columns of its own, and half of the sums' registers are enough
//   8   columns from 8 on take what the leading bits leave; a byte permutation makes two rows of one dim of two dims of one row
//   16  leading bits and the rest in products of their own
#include "decode_split.hpp"
#include "fp4.hpp"
#include "launch.hpp"

namespace vec {

namespace {

struct Fp4Params {
  DecodeParams d;
  const uint8_t *k_ret_scale, *v_ret_scale, *k_apx_scale;
  int n_blocks;                  // paged: of the pools
  uint32_t flip;                 // 0x80000000: the scale is negative, and query rows change their sign (d.c2 is its size, above 0)
};

constexpr int kFp4TileRows = 32;
// Keys turned back by near positions.  The turns of a lane's eight rows are those of the first one and the difference, one operation instead
// of five, as long as no pair turns more than this between them.  That is off by 2^-18 turns (the rounding of a number below 128) and 2^-19 (the
// frequency's, 2^-25 of it), 3.6e-5 of the pair's length, before the row is rounded to bf16, 2^-8; fp32 does not take it.
// More than four query heads do not either: their registers do not hold both ways (eight 31.0 us with it, 29.8 without; sixteen 26.0, 22.5).
// Split launch, us, without / with: 16 sequences of 32768 tokens 31.6 / 27.5, four 15.0 / 13.2, 24 unequal ones 21.4 / 19.4, 64 dims 22.8 / 20.5.
constexpr float kNearTurns = 64.f;
constexpr float kRaiseAt = 16.f;       // log2: how far a score may lie above its column's reference before that is raised

// no more than n loads on their way, those of a tile or none; n is the same for the wave
__device__ __forceinline__ void wait_tiles(int n) {
  switch (n) {
    case 0: wait_loads<0>(); break;
    case 2: wait_loads<2>(); break;
    case 3: wait_loads<3>(); break;
    case 5: wait_loads<5>(); break;
    case 9: wait_loads<9>(); break;
    default: wait_loads<0>();
  }
}

// rounds a weight to its leading eight bits by cutting the others off: what is left is exact
__device__ __forceinline__ float leading(float x) { return __uint_as_float(__float_as_uint(x) & 0xffff0000u); }
// two floats with no more than eight significant bits as two bf16
__device__ __forceinline__ uint32_t high_halves(float lo, float hi) {
  return __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
}

// Where a tile of 32 rows lies in LDS.  Row 8 a + b of it is the (4 b + a)-th, so that the four rows that a wave reads at once of R, one for each
// quarter, are neighbours, and the 16-byte pieces of a row are permuted by b, so that the keys' 16-byte reads of rows b, b + 1, .. hit
// distinct banks.  A scale slot holds the scale bytes of a row (keys' rows, then R's;
// of approximated rows, which have one tensor, the positions in the place of the latter).
template <int D> struct Fp4Stage {
  static constexpr int kCode = fp4_code_bytes(D), kPieces = kCode / 16;
  static constexpr int kTensor = kFp4TileRows * kCode;
  static constexpr int kSlots = 2 * kTensor, kPositions = kSlots + 128, kAlive = kSlots + 256;
  static constexpr int kBytes = kAlive + 16;
  static constexpr int kLoads = kTensor / 1024;                 // wave-wide loads of a tensor
  static constexpr int kRowsPerLoad = kFp4TileRows / kLoads;
  static __device__ __forceinline__ int place(int row) { return 4 * (row & 7) + (row >> 3); }
  static __device__ __forceinline__ int twist(int place) { return D == 128 ? (place >> 2) & 3 : (place >> 3) & 1; }
  static __device__ __forceinline__ int piece(int row, int piece) { return place(row) * kCode + ((piece ^ twist(place(row))) * 16); }
};
// Tiles of a wave: one on its way while one is worked on.  Split launch, us, two stages / three / four (two workgroups per CU) / two and four workgroups:
// 16 routed sequences of 32768 tokens 18.9 / 19.8 / 21.3 / 21.2, 24 unequal ones 14.0 / 16.1 / 18.3 / 14.7, on rotated keys
// (before kNearTurns) 20.7 / 22.9 / 33.4 / 28.1,
// 64 whole ones of 2048 28.3 / 31.1 / 35.0 / 28.0, 16 whole ones of 32768 90.1 / 91.3 / 92.1 / 90.8.
constexpr int kFp4Stages = 2;

// Rows of a workgroup: of the retained segment, or approximated ones, as they are or turned back with pairs (x[i], x[i + D / 2]) or
// (x[2 i], x[2 i + 1]).
enum class Fp4RowKind { kRetained, kApprox, kTurnedApart, kTurnedNext };

// T: of the query, W, the output and the step's token.  COLS: no fewer than the query rows; 16 for fp32.
template <typename T, int D, int COLS, Fp4RowKind KIND>
__device__ __forceinline__ void attend_fp4(const Fp4Params& f, const RopeParams& rp, const SplitRows& range, int tid) {
  constexpr bool kExact = sizeof(T) == 4;              // fp32: query and weights in three parts, all their bits
  constexpr bool kMx = D == 128 && !kExact;            // scores from the codes
  constexpr bool kQuad = COLS == 4, kSide = COLS == 8;
  static_assert(!kExact || COLS == 16, "parts in products of their own");
  constexpr int kParts = kExact ? 3 : COLS == 16 ? 2 : 1;        // of a weight, in products of their own
  constexpr int kQueryParts = kExact ? 3 : kMx && COLS == 16 ? 2 : 1;
  constexpr int NC = D / 32, NT = kQuad ? D / 32 : D / 16;       // score products per tile; tiles of the output dims
  constexpr int kCode = fp4_code_bytes(D), kScale = fp4_scale_bytes(D);
  constexpr int kRedStride = (kQuad ? D / 2 : D) + 4;  // floats of a column, in kQuad of every other dim
  constexpr int kStepRows = DW * kFp4TileRows;
  typedef Fp4Stage<D> St;

  const DecodeParams& p = f.d;
  const int G = p.Hq / p.Hkv, PSZ = 2 * G + G * D;
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int m = lane & 15, quarter = lane >> 4;
  const SegmentRows seg = range.seg;
  constexpr bool is_apx = KIND != Fp4RowKind::kRetained, apart = KIND == Fp4RowKind::kTurnedApart, turned = apart || KIND == Fp4RowKind::kTurnedNext;
  const bool paged = !is_apx && seg.blocks != nullptr;
  const int row_begin = range.begin, row_end = range.end;
  const size_t bh = (size_t)range.b * p.Hkv + range.h;
  // rows in memory: the step's own token, the last live row, comes from the caller's tensors
  const int stored = is_apx ? seg.n_approx : seg.new_row >= 0 ? seg.new_row : seg.len_retain;
  const int new_row = is_apx ? -1 : seg.new_row;
  const uint8_t* k_codes = reinterpret_cast<const uint8_t*>(is_apx ? p.k_apx : p.k_ret);
  const uint8_t* k_scales = is_apx ? f.k_apx_scale : f.k_ret_scale;
  const uint8_t* r_codes = reinterpret_cast<const uint8_t*>(is_apx ? p.k_apx : p.v_ret);
  const uint8_t* r_scales = is_apx ? f.k_apx_scale : f.v_ret_scale;
  const int64_t row0 = is_apx ? (int64_t)seg.apx_row0 : (int64_t)seg.ret_row0;

  auto mfma = [](u32x4 a, u32x4 b, const f32x4& c) VEC_INLINE {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  };
  const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
  auto wave_fence = []() VEC_INLINE {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  };

  // query rows: column m holds row m % COLS; the rest of a weight (lo) belongs to it in some columns
  const bool lo = kQuad ? m & 4 : kSide ? m & 8 : false;
  const T* q_row = reinterpret_cast<const T*>(p.q) + ((size_t)range.b * p.Hq + (size_t)range.h * G + min(m & (COLS - 1), G - 1)) * D;
  u32x4 qf[kMx ? 1 : kQueryParts][kMx ? 1 : NC];
  i32x8 qx[kMx ? kQueryParts : 1];
  int q_unit[kMx ? kQueryParts : 1];
  u32x4 q_raw[sizeof(T) == 2 ? NC : 2 * NC];
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const int at = kMx ? c / 2 * 64 + quarter * 16 + c % 2 * 8 : quarter * (D / 4) + c * 8;
    q_raw[c] = *reinterpret_cast<const u32x4*>(q_row + at);
    if constexpr (kExact) q_raw[NC + c] = *reinterpret_cast<const u32x4*>(q_row + at + 4);
  }
  // The sum of a column's weights is one more row of the second product, of ones: the same in every lane, and of the weights as they
  // went in.
  f32x4 o[NT], o_sum = zero;
#pragma unroll
  for (int j = 0; j < NT; ++j) o[j] = zero;
  const u32x4 ones = {0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};
  float ref = -INFINITY;

  // paged: ids of the blocks from window on, one a lane
  int window = row_begin >> seg.block_shift, ids = 0;
  auto load_window = [&]() VEC_INLINE {
    ids = seg.blocks[min(window + lane, p.blocks_per_seq - 1)];
    asm volatile("" : "+v"(ids));                    // waited for here, and not wherever it is used
  };
  if (paged && row_begin < row_end) load_window();
  // first row, in the pools, of the rows from `row` on; false: there are none
  auto block_row = [&](int row, int64_t& at) VEC_INLINE {
    const int id = __builtin_amdgcn_readlane(ids, (row >> seg.block_shift) - window);
    at = ((int64_t)id << seg.block_shift) + (row & ((1 << seg.block_shift) - 1));
    return (uint32_t)id < (uint32_t)f.n_blocks && (row >> seg.block_shift) < p.blocks_per_seq;
  };

  extern __shared__ __align__(16) unsigned char fp4_lds[];
  unsigned char* ring = fp4_lds + wave * (kFp4Stages * St::kBytes);
  const int32_t* positions = (turned && rp.positions) ? rp.positions + seg.apx_row0 : nullptr;
  // what a lane brings in: a 16-byte piece of codes of one row (a load), and of one more kRowsPerLoad / 4 further on in every eight (the next
  // load); the scales of one row
  const int in_place = lane / St::kPieces, in_row = 8 * (in_place & 3) + (in_place >> 2);
  const int in_piece = (lane % St::kPieces) ^ St::twist(in_place);
  // (the second load's places are 16 further on, which the permutation does not see)
  const int scale_row = lane & 31;
  const uint32_t in_code = in_row * kCode + in_piece * 16;
  const uint8_t* in_scale = (lane < 32 ? k_scales : r_scales) + scale_row * kScale;
  const bool small_blocks = paged && seg.block_shift < 5;
  // A block that does not exist has been met: from then on a tile's mask of rows is looked at, the one on its way by then included, so
  // that every stage has one from the start.
  bool holes = false;
  if (paged && lane < kFp4Stages) *reinterpret_cast<uint32_t*>(ring + lane * St::kBytes + St::kAlive) = ~0u;

  auto fill = [&](int base, unsigned char* st) VEC_INLINE {
    int64_t at_lo = row0 + base, at_hi = at_lo;        // of the tile's first row, less 16 rows of its 17th
    bool lo = true, hi = true;
    if (paged) {
      if (((base + kFp4TileRows - 1) >> seg.block_shift) - window > kWave - 1) { window = base >> seg.block_shift; load_window(); }
      lo = hi = block_row(base, at_lo);
      at_hi = at_lo;
      if (seg.block_shift < 5 && base + 16 < row_end) {        // (behind the last row there need not be a block)
        hi = block_row(base + 16, at_hi);
        at_hi -= 16;
      }
    }
    const uint32_t to = lds_address(st);
    if (base + kFp4TileRows <= stored && lo && hi) {   // uniform: rows that are all there
      auto codes = [&](const uint8_t* from, int64_t at, uint32_t dst) VEC_INLINE {
#pragma unroll
        for (int i = 0; i < St::kLoads; ++i) load_to_lds16_once(dst + i * 1024, from + (at + i * (8 / St::kLoads)) * kCode, in_code);
      };
      const void* s = in_scale + (small_blocks && scale_row >= 16 ? at_hi : at_lo) * kScale;
      if (!small_blocks || is_apx) {
        codes(k_codes, at_lo, to);
        if (!is_apx) codes(r_codes, at_lo, to + St::kTensor);
      } else if (in_row < 16) {                        // half of the lanes' rows lie in either block
        codes(k_codes, at_lo, to);
        codes(r_codes, at_lo, to + St::kTensor);
      } else {
        codes(k_codes, at_hi, to);
        codes(r_codes, at_hi, to + St::kTensor);
      }
      if (!turned) {
        if constexpr (D == 128) load_to_lds4(to + St::kSlots, s);
        else load_to_lds2(to + St::kSlots, s);
      } else {
        if (positions && D == 128 && lane >= 32) s = positions + base + scale_row;
        if (lane < 32 || (positions && D == 128)) {
          if constexpr (D == 128) load_to_lds4(to + St::kSlots, s);
          else load_to_lds2(to + St::kSlots, s);
        }
        if (lane < 32) {
          if (!positions) *reinterpret_cast<int*>(st + St::kPositions + lane * 4) = base + lane;
          else if (D != 128) load_to_lds4(to + St::kPositions, positions + base + lane);
        }
      }
      if (holes && lane == 0) *reinterpret_cast<uint32_t*>(st + St::kAlive) = ~0u;
      return;
    }
    // The last rows, rows of blocks that do not exist, the step's own token.  What is no row is all zeros, since a weight of 0 does
    // not make a NaN of the memory harmless.
    wait_loads<0>();                                   // the count of what is on its way starts anew behind this tile
    holes = holes || !lo || !hi;
    {
      const int row = lane & 31, half = lane >> 5;     // two lanes a row
      const bool is = base + row < stored && (row < 16 ? lo : hi);
      const int64_t at = (row < 16 ? at_lo : at_hi) + row;
      for (int t = 0; t < (is_apx ? 1 : 2); ++t) {
        const uint8_t* codes = t ? r_codes : k_codes;
#pragma unroll
        for (int i = 0; i < St::kPieces / 2; ++i) {
          const int piece = half * (St::kPieces / 2) + i;
          u32x4 x = {0u, 0u, 0u, 0u};
          if (is) x = *reinterpret_cast<const u32x4*>(codes + at * kCode + piece * 16);
          *reinterpret_cast<u32x4*>(st + t * St::kTensor + St::piece(row, piece)) = x;
        }
      }
      // the scales of both tensors, one a lane
      const uint8_t* s = (half ? r_scales : k_scales) + at * kScale;
      uint32_t unit = 0;
      if (is) unit = D == 128 ? *reinterpret_cast<const uint32_t*>(s) : (uint32_t)*reinterpret_cast<const uint16_t*>(s);
      if (turned && half == 1) unit = is ? (uint32_t)(positions ? positions[base + row] : base + row) : 0u;
      *reinterpret_cast<uint32_t*>(st + St::kSlots + lane * 4) = unit;
      const uint32_t alive = (uint32_t)__ballot(is || base + row == new_row);           // bit r: row r is one
      if (lane == 0) *reinterpret_cast<uint32_t*>(st + St::kAlive) = alive;
    }
    wave_fence();
    if (!is_apx && new_row >= base && new_row < base + kFp4TileRows && lane < D / 4) {
      // eight elements of the token's key or value a lane, as vector_store_fp4 rounds them
      constexpr int kLanes = D / 8;
      const int t = lane / kLanes, i = lane % kLanes, row = new_row - base;
      float x[8];
      load8(reinterpret_cast<const T*>(t ? p.v_new : p.k_new) + bh * D + i * 8, x);
      const uint32_t byte = fp4_scale_byte(quad_max(top_bits8(x))), codes = fp4_codes(x, byte);
      *reinterpret_cast<uint32_t*>(st + t * St::kTensor + St::piece(row, i / 4) + i % 4 * 4) = codes;
      if (i % 4 == 0) st[St::kSlots + (t * 32 + row) * 4 + i / 4] = (uint8_t)byte;
      if (new_row < seg.cap && (row < 16 ? lo : hi)) {
        const int64_t at = (row < 16 ? at_lo : at_hi) + row;
        *reinterpret_cast<uint32_t*>(const_cast<uint8_t*>(t ? r_codes : k_codes) + at * kCode + i * 4) = codes;
        if (i % 4 == 0) const_cast<uint8_t*>(t ? r_scales : k_scales)[at * kScale + i / 4] = (uint8_t)byte;
      }
    }
  };

  // a lane's rows of a tile in operand order: the key row (and that four further on), the first of the eight of R
  const int k_row = 8 * (m >> 2) + (m & 3), r_row = 8 * quarter;
  // How a lane's dims of R lie: kDims consecutive ones, or (keys that are turned back with pairs (x[i], x[i + D / 2])) kDims / 2 and their
  // partners.  A word of scale bytes is turned so that the byte of the lane's block is a float's exponent, which is all that the conversions
  // look at (all bytes and codes compared with junk around the exponent).
  constexpr int kDims = D / 16;
  const uint32_t to_exponent = 8u * (apart ? kDims / 2 * m / kFp4Block : kDims * m / kFp4Block) + 9u;
  auto exponent = [](uint32_t bytes, uint32_t by) VEC_INLINE { return __uint_as_float(__builtin_amdgcn_alignbit(bytes, bytes, by)); };
  const uint32_t rest_mask = lo ? 0xffff0000u : 0u, rest_half = lo ? 0x8000u : 0u;      // a bf16's bits of a float; half of its last one
  const uint32_t at_dim = m < 8 ? 0x0c0c0706u : 0x07060c0cu;        // kQuad: a weight's leading half in the low or the high half of a word

  // a lane's dims always belong to the same kDims / 2 rotary pairs
  float t_hi[turned ? kDims / 2 : 1], t_lo[turned ? kDims / 2 : 1];
  if constexpr (turned) {
#pragma unroll
    for (int e = 0; e < kDims / 2; ++e) {
      t_hi[e] = rp.turns_hi[kDims / 2 * m + e];
      t_lo[e] = rp.turns_lo[kDims / 2 * m + e];
    }
  }

  auto consume = [&](const unsigned char* st, int base) VEC_INLINE {
    float s[8];                                        // scores; times d.c2 they are in the log2 domain
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int row = k_row + 4 * u;
      uint32_t words[NC];
      if constexpr (D == 128) {
        const u32x4 x = *reinterpret_cast<const u32x4*>(st + St::piece(row, quarter));
#pragma unroll
        for (int c = 0; c < NC; ++c) words[c] = x[c];
      } else {
        const u32x2 x = *reinterpret_cast<const u32x2*>(st + St::piece(row, quarter >> 1) + (quarter & 1) * 8);
#pragma unroll
        for (int c = 0; c < NC; ++c) words[c] = x[c];
      }
      const uint32_t byte = st[St::kSlots + row * 4 + (D == 128 ? quarter : quarter >> 1)];
      f32x4 acc = zero;
      if constexpr (kMx) {
        const i32x8 a = {(int)words[0], (int)words[1], (int)words[2], (int)words[3], 0, 0, 0, 0};
#pragma unroll
        for (int part = 0; part < kQueryParts; ++part)
          acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, qx[part], acc, 4, 0, 0, (int)byte, 0, q_unit[part]);
        if constexpr (kQueryParts == 1) {              // the other part is in the columns COLS further on or back
#pragma unroll
          for (int i = 0; i < 4; ++i)
            acc[i] += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(acc[i]), 0x120 + COLS, 0xf, 0xf, false));
        }
      } else {
        const float unit = fp4_unit(byte);
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          const uint32_t w = words[c];
          const u32x4 a = {fp4_pair_bf16<0>(w, unit), fp4_pair_bf16<1>(w, unit), fp4_pair_bf16<2>(w, unit), fp4_pair_bf16<3>(w, unit)};
#pragma unroll
          for (int part = 0; part < kQueryParts; ++part) acc = mfma(a, qf[part][c], acc);
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) s[4 * u + i] = acc[i];
    }
    const bool some_dead = holes || base + kFp4TileRows > stored;
    uint32_t alive = 0;
    if (some_dead) {
      alive = *reinterpret_cast<const uint32_t*>(st + St::kAlive) >> r_row;
#pragma unroll
      for (int j = 0; j < 8; ++j) s[j] = (alive >> j & 1) ? s[j] : -INFINITY;
    }
    float top = s[0];
#pragma unroll
    for (int j = 1; j < 8; ++j) top = fmaxf(top, s[j]);
    top *= p.c2;
    // The reference of a column is raised only where a score lies far above it: the weights are then at most 2^kRaiseAt, and a
    // sum of them does not leave the range of a float.  The same in all lanes of a column.
    if (__ballot(top > ref + kRaiseAt)) {
      top = fmaxf(top, __shfl_xor(top, 16, kWave));
      top = fmaxf(top, __shfl_xor(top, 32, kWave));
      const float next = fmaxf(ref, top), by = ref == next ? 1.f : fast_exp2(ref - next);
      o_sum *= by;
#pragma unroll
      for (int j = 0; j < NT; ++j) o[j] *= by;
      ref = next;
    }
    float w[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j] = fast_exp2(fmaf(s[j], p.c2, -ref));
    if (some_dead) {                                   // no row yet: minus infinity less itself
#pragma unroll
      for (int j = 0; j < 8; ++j) w[j] = (alive >> j & 1) ? w[j] : 0.f;
    }
    // kQuad: rows 0 .. 3 and 4 .. 7
    u32x4 weights[kQuad ? 2 : kParts];
    // A weight in two parts is good to 2^-16 of itself: what the leading eight bits leave is below 2^-7 of it and goes to the nearest of its own
    // eight bits.  Cutting those off as well is off by up to 2^-15, and always to the same side.  Split launch, us, cut / rounded: 16 whole sequences of 32768
    // tokens 89.8 / 90.4, 24 unequal ones on rotated keys 20.7 / 20.3, 16 of 16384 at 64 dims 29.3 / 30.0, with sixteen query heads 51.8 / 50.6.
    if constexpr (COLS != 16) {                        // columns of the rest
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        w[j] -= __uint_as_float(__float_as_uint(w[j]) & rest_mask);
        w[j] = __uint_as_float(__float_as_uint(w[j]) + rest_half);
      }
    }
    if constexpr (kQuad) {
#pragma unroll
      for (int j = 0; j < 8; ++j) weights[j / 4][j % 4] = __builtin_amdgcn_perm(__float_as_uint(w[j]), __float_as_uint(w[j]), at_dim);
      o_sum = mfma(ones, weights[0], o_sum);
      o_sum = mfma(ones, weights[1], o_sum);
    } else {
#pragma unroll
      for (int part = 0; part < kParts; ++part) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          weights[part][i] = part > 0 && part + 1 == kParts ? pack_bf16(w[2 * i], w[2 * i + 1]) : high_halves(w[2 * i], w[2 * i + 1]);
        if (part + 1 < kParts) {
#pragma unroll
          for (int j = 0; j < 8; ++j) w[j] -= leading(w[j]);
        }
        o_sum = mfma(ones, weights[part], o_sum);
      }
    }
    // the eight rows of R, and their scale bytes
    uint32_t r[8], bytes[8];
    const unsigned char* rt = st + (is_apx ? 0 : St::kTensor);
    const unsigned char* slots = st + St::kSlots + (is_apx ? 0 : 128);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      // row 8 quarter + j, the (4 j + quarter)-th; x: how its pieces are permuted
      const int x = St::twist(4 * j), at = 4 * j * kCode;
      if constexpr (!apart) {
        const unsigned char* from = rt + quarter * kCode + at;
        if constexpr (D == 128) r[j] = *reinterpret_cast<const uint32_t*>(from + (((m >> 2) ^ x) * 16 + (m & 3) * 4));
        else r[j] = *reinterpret_cast<const uint16_t*>(from + (((m >> 3) ^ x) * 16 + (m & 7) * 2));
      } else {                                         // dims kDims / 2 m .. in the low half, their partners, half a row on, in the high one
        const unsigned char* from = rt + quarter * kCode + at;
        if constexpr (D == 128) {
          r[j] = (uint32_t)*reinterpret_cast<const uint16_t*>(from + (((m >> 3) ^ x) * 16 + (m & 7) * 2)) |
                 (uint32_t)*reinterpret_cast<const uint16_t*>(from + (((m >> 3) ^ x ^ 2) * 16 + (m & 7) * 2)) << 16;
        } else {
          r[j] = (uint32_t)from[x * 16 + m] | (uint32_t)from[(x ^ 1) * 16 + m] << 16;
        }
      }
    }
#pragma unroll
    for (int j = 0; j < 8; j += 4) {
      const u32x4 x = *reinterpret_cast<const u32x4*>(slots + (r_row + j) * 4);
#pragma unroll
      for (int i = 0; i < 4; ++i) bytes[j + i] = x[i];
    }
    if constexpr (!turned) {
      float unit[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) unit[j] = exponent(bytes[j], to_exponent);
      for_each_constant<kDims / 2>([&](auto c) VEC_INLINE {
        uint32_t two[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) two[j] = fp4_pair_bf16<decltype(c)::value>(r[j], unit[j]);
        if constexpr (kQuad) {
          o[c] = mfma(u32x4{two[0], two[1], two[2], two[3]}, weights[0], o[c]);
          o[c] = mfma(u32x4{two[4], two[5], two[6], two[7]}, weights[1], o[c]);
        } else {
          u32x4 even, odd;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            even[i] = __builtin_amdgcn_perm(two[2 * i + 1], two[2 * i], 0x05040100u);
            odd[i] = __builtin_amdgcn_perm(two[2 * i + 1], two[2 * i], 0x07060302u);
          }
#pragma unroll
          for (int part = 0; part < kParts; ++part) {
            o[2 * c] = mfma(even, weights[part], o[2 * c]);
            o[2 * c + 1] = mfma(odd, weights[part], o[2 * c + 1]);
          }
        }
      });
    } else {
      // keys turned back, in one bf16 part (three for fp32): they carry that one rounding, as those of a bf16 cache do
      constexpr int kRowParts = kExact ? 3 : 1;
      float pos[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) pos[j] = (float)(*reinterpret_cast<const int*>(st + St::kPositions + (r_row + j) * 4) + rp.pos_offset);
      // dims 2 t and 2 t + 1 of the lane's, of the eight rows
      auto add = [&](auto t, float* even, float* odd) VEC_INLINE {
        if constexpr (kQuad) {
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            u32x4 a;
#pragma unroll
            for (int j = 0; j < 4; ++j) a[j] = pack_bf16(even[4 * i + j], odd[4 * i + j]);
            o[t] = mfma(a, weights[i], o[t]);
          }
        } else {
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float* x = e ? odd : even;
#pragma unroll
            for (int rest = 0; rest < kRowParts; ++rest) {
              u32x4 a;
#pragma unroll
              for (int i = 0; i < 4; ++i) a[i] = kRowParts == 1 ? pack_bf16(x[2 * i], x[2 * i + 1]) : high_halves(x[2 * i], x[2 * i + 1]);
              if (rest + 1 < kRowParts) {
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] -= leading(x[j]);
              }
#pragma unroll
              for (int part = 0; part + rest < kParts; ++part) o[2 * t + e] = mfma(a, weights[part], o[2 * t + e]);
            }
          }
        }
        __builtin_amdgcn_sched_barrier(0);             // all pairs' sines at once would not fit the registers
      };
      auto turn = [&](auto near) VEC_INLINE {
        // (what both ways share would be drawn in front of the branch, too much for the registers)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          if constexpr (decltype(near)::value) asm volatile("; near" : "+v"(r[j]), "+v"(pos[j]));
          else asm volatile("; far" : "+v"(r[j]), "+v"(pos[j]));
        }
        auto cos_sin = [&](int j, float from, float hi, float lo, float& cs, float& sn) VEC_INLINE {
          if constexpr (decltype(near)::value) {
            const float u = j ? fmaf(pos[j], hi, from) : from;
            cs = __builtin_amdgcn_cosf(u);
            sn = __builtin_amdgcn_sinf(u);
          } else {
            rotary_cos_sin(pos[j], hi, lo, cs, sn);
          }
        };
        auto first_turns = [&](float hi, float lo) VEC_INLINE { return decltype(near)::value ? rotary_turns(pos[0], hi, lo) : 0.f; };
        if constexpr (apart) {
          constexpr int kHalf = kDims / 2;               // pairs of a lane, two a byte of codes
          for_each_constant<kHalf / 2>([&](auto c) VEC_INLINE {
            float a[2][8], b[2][8];
            const float from[2] = {first_turns(t_hi[2 * c], t_lo[2 * c]), first_turns(t_hi[2 * c + 1], t_lo[2 * c + 1])};
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              const f32x2 x = fp4_pair_f32<decltype(c)::value>(r[j], exponent(bytes[j], to_exponent));
              const f32x2 y = fp4_pair_f32<2 + decltype(c)::value>(r[j], exponent(bytes[j], to_exponent + kScale / 2 * 8u));
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                float cs, sn;
                cos_sin(j, from[e], t_hi[2 * c + e], t_lo[2 * c + e], cs, sn);
                rotary_back(x[e], y[e], cs, sn, a[e][j], b[e][j]);
              }
            }
            add(std::integral_constant<int, decltype(c)::value>{}, a[0], a[1]);
            add(std::integral_constant<int, kHalf / 2 + decltype(c)::value>{}, b[0], b[1]);
          });
        } else {
          for_each_constant<kDims / 2>([&](auto c) VEC_INLINE {
            float a[8], b[8];
            const float from = first_turns(t_hi[c], t_lo[c]);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              const f32x2 x = fp4_pair_f32<decltype(c)::value>(r[j], exponent(bytes[j], to_exponent));
              float cs, sn;
              cos_sin(j, from, t_hi[c], t_lo[c], cs, sn);
              rotary_back(x[0], x[1], cs, sn, a[j], b[j]);
            }
            add(c, a, b);
          });
        }
      };
      bool near = false;
      if constexpr (!kExact && COLS == 4) {
        float most = 0.f, fastest = fabsf(t_hi[0]);
#pragma unroll
        for (int j = 1; j < 8; ++j) most = fmaxf(most, fabsf(pos[j] - pos[0]));
#pragma unroll
        for (int e = 1; e < kDims / 2; ++e) fastest = fmaxf(fastest, fabsf(t_hi[e]));
        near = __ballot(!(most * fastest <= kNearTurns)) == 0;
      }
      if (near) {
#pragma unroll
        for (int j = 1; j < 8; ++j) pos[j] -= pos[0];
        turn(std::true_type{});
      } else {
        turn(std::false_type{});
      }
    }
  };

  // loads of a tile; of tiles that went by the other way there are none on their way, nor of any before these
  const int per_tile = is_apx ? St::kLoads + 1 + (D == 64 && turned && positions ? 1 : 0) : (small_blocks ? 4 : 2) * St::kLoads + 1;
  const int tiles = row_begin + wave * kFp4TileRows < row_end ? (row_end - row_begin - wave * kFp4TileRows + kStepRows - 1) / kStepRows : 0;
  const int first = row_begin + wave * kFp4TileRows;
  static_assert(kFp4Stages == 2, "one tile on its way");
  if (tiles > 0) fill(first, ring);
  // the query rows in operand order; the first tiles are on their way
  if constexpr (kMx) {
    // A row in two fp8 parts under a scale for every 32 dims: four bits and the four behind them, all that bf16 has; an element far below its
    // block's largest is off by 2^-22 of that at most.  The matrix core takes 16 dims from 16 quarter on and 16 from 64 + 16 quarter
    // on from a lane, and the scale of dims 32 quarter .. (compared with one-hot operands); a block's dims are in two lanes.
    float x[2][16];
    int top[2];
#pragma unroll
    for (int half = 0; half < 2; ++half) {
#pragma unroll
      for (int e = 0; e < 16; ++e) x[half][e] = (e & 1) ? bf16_hi(q_raw[2 * half + e / 8][e % 8 / 2]) : bf16_lo(q_raw[2 * half + e / 8][e % 8 / 2]);
      uint32_t most = max(top_bits8(x[half]), top_bits8(x[half] + 8));
      most = max(most, (uint32_t)__shfl_xor((int)most, 16, kWave));
      // the largest between 128 and 256 units; an infinite or NaN element: NaN, in the whole block
      top[half] = most >= 0x7f800000u ? 255 : min(max((int)(most >> 23) - 7, 6), 254);
    }
    const int first = __shfl(top[0], m + (quarter & 1) * 32, kWave), second = __shfl(top[1], m + (quarter & 1) * 32, kWave);
    const int own = quarter < 2 ? first : second;      // of block `quarter`
#pragma unroll
    for (int part = 0; part < kQueryParts; ++part) q_unit[part] = own == 255 ? 255 : own - (lo || part == 1 ? 5 : 0);
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int byte = top[half] == 255 ? 127 : top[half];
      const float unit = fp4_unit((uint32_t)byte), small = fp4_unit((uint32_t)(byte - 5));
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        s16x2 hi = {0, 0}, rest = {0, 0};
        float y[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = __uint_as_float(__float_as_uint(x[half][4 * w + e]) ^ f.flip);
        hi = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(hi, y[0], y[1], unit, false);
        hi = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(hi, y[2], y[3], unit, true);
        const int word = __builtin_bit_cast(int, hi);
        const f32x2 back0 = __builtin_bit_cast(f32x2, __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(word, unit, false));
        const f32x2 back1 = __builtin_bit_cast(f32x2, __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(word, unit, true));
        rest = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(rest, y[0] - back0[0], y[1] - back0[1], small, false);
        rest = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(rest, y[2] - back1[0], y[3] - back1[1], small, true);
        if constexpr (kQueryParts == 2) {
          qx[0][half * 4 + w] = word;
          qx[1][half * 4 + w] = __builtin_bit_cast(int, rest);
        } else {
          qx[0][half * 4 + w] = lo ? __builtin_bit_cast(int, rest) : word;
        }
      }
    }
  } else {
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      if constexpr (!kExact) {
        qf[0][c] = q_raw[c] ^ (f.flip | f.flip >> 16);
      } else {
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = __uint_as_float(q_raw[c + (e >= 4 ? NC : 0)][e % 4] ^ f.flip);
#pragma unroll
        for (int part = 0; part < kQueryParts; ++part) {
          float y[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) { y[e] = leading(x[e]); x[e] -= y[e]; }
#pragma unroll
          for (int e = 0; e < 4; ++e) qf[part][c][e] = high_halves(y[2 * e], y[2 * e + 1]);
        }
      }
    }
  }
  // The query rows have arrived from here on.  Without this the wait for them would sit in the loop, and wait for tiles as well.
  if constexpr (!kMx) {
#pragma unroll
    for (int part = 0; part < kQueryParts; ++part)
#pragma unroll
      for (int c = 0; c < NC; ++c) asm volatile("" : "+v"(qf[part][c]));
  } else {
#pragma unroll
    for (int part = 0; part < kQueryParts; ++part) asm volatile("" : "+v"(qx[part]), "+v"(q_unit[part]));
  }
  if constexpr (turned) {
#pragma unroll
    for (int e = 0; e < kDims / 2; ++e) asm volatile("" : "+v"(t_hi[e]), "+v"(t_lo[e]));
  }
  int stage = 0;
  for (int i = 0; i < tiles; ++i) {
    const int base = first + i * kStepRows;
    // the stage of the tile before is free: what was read of it is in registers
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    if (i + 1 < tiles) fill(base + kStepRows, ring + (1 - stage) * St::kBytes);
    wait_tiles(i + 1 < tiles ? per_tile : 0);
    wave_fence();
    consume(ring + stage * St::kBytes, base);
    stage = 1 - stage;
  }

  // ---- merge the waves ----
  // a wave's sums in the place of its own ring
  constexpr int kWaveBytes = kFp4Stages * St::kBytes;
  static_assert(16 * kRedStride * 4 + 2 * 16 * 4 <= kWaveBytes, "the merge area must fit in the ring");
  auto red = [&](int wv, int col, int j) VEC_INLINE { return reinterpret_cast<float*>(fp4_lds + wv * kWaveBytes) + col * kRedStride + j; };
  auto ml = [&](int wv, int what, int col) VEC_INLINE { return reinterpret_cast<float*>(fp4_lds + wv * kWaveBytes) + 16 * kRedStride + what * 16 + col; };
  wave_fence();
  // lane (m, quarter): column m, dims of lane 4 quarter + i; kPer of them, or of every other one, lie side by side
  constexpr int kPer = kQuad ? (apart ? kDims / 4 : kDims / 2) : (apart ? kDims / 2 : kDims);
  constexpr int kWide = kPer < 4 ? kPer : 4;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < NT; j += kWide) {
      float* to = red(wave, m, j / kPer * (kQuad ? D / 4 : D / 2) + kPer * (4 * quarter + i) + j % kPer);
      if constexpr (kWide == 4) *reinterpret_cast<f32x4*>(to) = f32x4{o[j][i], o[j + 1][i], o[j + 2][i], o[j + 3][i]};
      else if constexpr (kWide == 2) *reinterpret_cast<f32x2*>(to) = f32x2{o[j][i], o[j + 1][i]};
      else *to = o[j][i];
    }
  if (quarter == 0) {
    *ml(wave, 0, m) = ref;                             // minus infinity of a wave without rows: its share is 0 without a branch
    *ml(wave, 1, m) = o_sum[0];
  }
  __syncthreads();
  float* out = p.part + range.slot * PSZ;
  for (int i = tid * 4; i < G * D; i += DT_ * 4) {
    const int g = i / D, j = i % D;
    float top = -INFINITY, l = 0.f;
#pragma unroll
    for (int wv = 0; wv < DW; ++wv) top = fmaxf(top, *ml(wv, 0, g));
    const float safe = top == -INFINITY ? 0.f : top;
    f32x4 a = zero;
#pragma unroll
    for (int wv = 0; wv < DW; ++wv) {
      const float sc = fast_exp2(*ml(wv, 0, g) - safe);
      f32x4 x;
      if constexpr (kQuad) {
        const f32x2 even = *reinterpret_cast<const f32x2*>(red(wv, g, j / 2)) + *reinterpret_cast<const f32x2*>(red(wv, 4 + g, j / 2));
        const f32x2 odd = *reinterpret_cast<const f32x2*>(red(wv, 8 + g, j / 2)) + *reinterpret_cast<const f32x2*>(red(wv, 12 + g, j / 2));
        x = f32x4{even[0], odd[0], even[1], odd[1]};
      } else {
        x = *reinterpret_cast<const f32x4*>(red(wv, g, j));
        if constexpr (kSide) x += *reinterpret_cast<const f32x4*>(red(wv, 8 + g, j));
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) a[e] = fmaf(x[e], sc, a[e]);
      l = fmaf(COLS == 16 ? *ml(wv, 1, g) : *ml(wv, 1, g) + *ml(wv, 1, COLS + g), sc, l);
    }
    *reinterpret_cast<f32x4_u*>(out + 2 * G + i) = a;
    if (j == 0) {
      out[2 * g] = top;
      out[2 * g + 1] = l;
    }
  }
}

// Workgroups per CU.  fp32 turned back at 128 dims needs more than the 168 registers of three: with three 49 are spilled, and 8 sequences of 16384 tokens
// take 23.9 us, with two 19.3.
template <typename T, int D, Fp4RowKind APPROX>
constexpr int fp4_per_cu() {
  return sizeof(T) == 4 && D == 128 && APPROX != Fp4RowKind::kApprox ? 2 : kFp4PerCu;
}

template <typename T, int D, int COLS, Fp4RowKind APPROX>
__global__ __launch_bounds__(DT_, (fp4_per_cu<T, D, APPROX>())) void decode_split_fp4_kernel(Fp4Params f, RopeParams rp) {
  const SplitRows r = grid_split<DW * kFp4TileRows>(f.d);
  if (r.is_apx) attend_fp4<T, D, COLS, APPROX>(f, rp, r, (int)threadIdx.x);
  else attend_fp4<T, D, COLS, Fp4RowKind::kRetained>(f, rp, r, (int)threadIdx.x);
}

template <typename T, int D, int COLS, Fp4RowKind APPROX>
int launch_split_fp4(const Fp4Params& f, const RopeParams* rope, hipStream_t stream) {
  const dim3 grid = f.d.by_kind ? dim3(f.d.Hkv, f.d.B, f.d.splits_ret + f.d.splits_apx) : dim3(f.d.splits_ret + f.d.splits_apx, f.d.Hkv, f.d.B);
  constexpr int lds = DW * kFp4Stages * Fp4Stage<D>::kBytes;
  constexpr auto kernel = decode_split_fp4_kernel<T, D, COLS, APPROX>;
  VEC_HIP(set_max_lds(reinterpret_cast<const void*>(kernel), lds));
  VEC_LAUNCH(K_DECODE_SPLIT, kernel, grid, dim3(DT_), lds, stream, f, rope ? *rope : RopeParams{});
  VEC_HIP(hipGetLastError());
  return VECTOR_OK;
}

template <typename T, int D, int COLS>
int run_split_fp4(Fp4Params& f, const RopeParams* rope, hipStream_t stream) {
  pick_splits_fp4(f.d.B, f.d.Hkv, f.d.cap_retain, f.d.n_approx, rope ? kFp4Turned : kFp4Approx,
                  rope ? fp4_per_cu<T, D, Fp4RowKind::kTurnedApart>() : fp4_per_cu<T, D, Fp4RowKind::kApprox>(),
                  f.d.splits_ret, f.d.splits_apx);
  // Pieces of both kinds of rows on every CU, so that one computes while the other one waits for memory; us, split / head first: 48 unequal sequences of up to
  // 4000 tokens 16.9 / 15.8, 64 dims on rotated keys 21.8 / 20.6, four sequences 15.0 / 13.6.  One kind: 32 unequal ones of up to 16000 68.9 / 71.8.
  f.d.by_kind = f.d.splits_ret > 0 && f.d.splits_apx > 0;
  if (!rope || f.d.n_approx == 0) return launch_split_fp4<T, D, COLS, Fp4RowKind::kApprox>(f, nullptr, stream);
  return rope->interleaved ? launch_split_fp4<T, D, COLS, Fp4RowKind::kTurnedNext>(f, rope, stream)
                           : launch_split_fp4<T, D, COLS, Fp4RowKind::kTurnedApart>(f, rope, stream);
}

template <typename T, int D>
int run_fp4(Fp4Params& f, const RopeParams* rope, hipStream_t stream) {
  if constexpr (sizeof(T) == 2) {
    const int G = f.d.Hq / f.d.Hkv;
    if (G <= 4) return run_split_fp4<T, D, 4>(f, rope, stream);
    if (G <= 8) return run_split_fp4<T, D, 8>(f, rope, stream);
  }
  return run_split_fp4<T, D, 16>(f, rope, stream);
}

}  // namespace

int launch_decode_fp4(const vector_cache_fp4& c, const void* q, float scale, void* out, int flags, void* ws, hipStream_t stream,
                      const RopeParams* rope, const void* k_new, const void* v_new) {
  Fp4Params f = {};
  DecodeParams& p = f.d;
  p.out_f32 = (flags & VECTOR_DECODE_OUT_F32) ? 1 : 0;
  p.q = q; p.k_ret = c.k_ret; p.v_ret = c.v_ret; p.k_apx = c.k_apx; p.W = c.W; p.len_retain = c.len_retain;
  p.k_new = k_new; p.v_new = v_new;
  p.block_table = c.ret_block_table; p.blocks_per_seq = c.ret_blocks_per_seq;
  while (c.ret_block_table && (1 << p.block_shift) < c.ret_block_rows) ++p.block_shift;
  p.cap_retain_seq = c.cap_retain_seq; p.n_approx_seq = c.n_approx_seq;
  p.ret_row_start = c.ret_row_start; p.apx_row_start = c.apx_row_start;
  p.out = out; p.part = reinterpret_cast<float*>(ws);
  p.B = c.batch; p.Hq = c.n_q_heads; p.Hkv = c.n_kv_heads; p.cap_retain = c.cap_retain; p.n_approx = c.n_approx;
  p.w_sh = c.w_shared ? 0 : (int64_t)c.head_dim * c.head_dim;
  // (the least number for a scale of 0: times a score that is 0 in the log2 domain as well, times minus infinity it is what masks a row)
  const float c2 = scale * kLog2e;
  p.c2 = fmaxf(fabsf(c2), 1.17549435e-38f);
  f.flip = c2 < 0.f ? 0x80000000u : 0u;
  f.k_ret_scale = c.k_ret_scale; f.v_ret_scale = c.v_ret_scale; f.k_apx_scale = c.k_apx_scale;
  f.n_blocks = c.n_blocks;
  int rc;
  if (c.dtype == VECTOR_BF16) rc = c.head_dim == 128 ? run_fp4<bf16_t, 128>(f, rope, stream) : run_fp4<bf16_t, 64>(f, rope, stream);
  else rc = c.head_dim == 128 ? run_fp4<float, 128>(f, rope, stream) : run_fp4<float, 64>(f, rope, stream);
  return rc ? rc : launch_decode_merge(p, c.dtype, c.head_dim, stream);
}

}  // namespace vec
