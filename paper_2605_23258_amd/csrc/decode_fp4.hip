// Decode attention over caches held in 4 bits (vector_decode_attn_fp4, vector_decode_step_fp4): the same sum as over caches in 16 or 32 bits
// (decode_attn.hip), one softmax over the live retained rows and the approximated ones, z = sum p k over the latter, the same
// partial results and the same merge.
//
// What bounds it is memory, 136 bytes for the key and the value of a token at 128 dims, against 512 in bf16; but a quarter of the bytes
// leaves a quarter of the time for a row's arithmetic.  Both products run on the matrix cores in bf16 with fp32 sums:
// an element in 4 bits times its scale has two significant bits and is a bf16 number exactly, so the only
// roundings are those of the weights, which go in as parts of eight bits each (kParts).
//
// A wave takes 32 rows at a time and waits for no other before the end.  Their codes and scales go from memory straight into a ring of its
// own in LDS (Fp4Stage), so that what is on its way takes no registers, and are read back in the matrix cores' order:
//   scores   S[t][g] = sum_e K[t][e] q[g][e]      A = K: lane (m, quarter) holds D / 4 consecutive elements of a row, which is one read and
//                                                  one scale; B = the query rows in the same order of e
//   output   O[j][g] += sum_t R[t][j] P[t][g]     A = R^T: lane (m, quarter) holds dims D / 16 m .. of eight rows, 8 quarter ..; the conversion
//                                                  hands out two neighbouring dims of one row, and a byte permutation makes
//                                                  two rows of one dim of them
// Row 4 a + i of score tile u is token 8 a + 4 u + i, so that the eight weights that a lane gets from both score tiles are those
// of the eight rows that it holds of R.  R is the values, or for approximated rows the keys, read a second time in the other order;
// under ROPE these are turned back by their positions first.
//
// Sixteen columns hold up to 16 query rows.  Up to eight (SIDE): columns g take the weights' leading bits and columns 8 + g what these leave,
// with one product for both.
#include "decode_split.hpp"
#include "fp4.hpp"
#include "launch.hpp"

namespace vec {

namespace {

struct Fp4Params {
  DecodeParams d;
  const uint8_t *k_ret_scale, *v_ret_scale, *k_apx_scale;
  int n_blocks;                  // paged: of the pools
};

constexpr int kFp4TileRows = 32;
constexpr float kRaiseAt = 16.f;       // log2: how far a score may lie above its column's reference before that is raised

// no more than n loads on their way; n is the same for the wave
__device__ __forceinline__ void wait_tiles(int n) {
  switch (n) {
    case 0: wait_loads<0>(); break;
    case 2: wait_loads<2>(); break;
    case 3: wait_loads<3>(); break;
    case 4: wait_loads<4>(); break;
    case 5: wait_loads<5>(); break;
    case 6: wait_loads<6>(); break;
    case 10: wait_loads<10>(); break;
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
constexpr int kFp4Stages = 3;

// T: of the query, W, the output and the step's token.  SIDE: no more than eight query rows, T bf16.
template <typename T, int D, bool SIDE, bool ROPE>
__device__ __forceinline__ void attend_fp4(const Fp4Params& f, const RopeParams& rp, const SplitRows& range, int tid) {
  constexpr bool kExact = sizeof(T) == 4;              // fp32: query and weights in three parts, all their bits
  constexpr int kParts = kExact ? 3 : SIDE ? 1 : 2;    // of a weight, in products of their own
  constexpr int kQueryParts = kExact ? 3 : 1;
  constexpr int NC = D / 32, NT = D / 16;              // score products per tile; tiles of the output dims
  constexpr int kCode = fp4_code_bytes(D), kScale = fp4_scale_bytes(D);
  constexpr int kRedStride = D + 4;
  constexpr float kNegBig = -1.0e30f;                  // reference before any row: finite, so differences stay finite
  constexpr int kStepRows = DW * kFp4TileRows;
  typedef Fp4Stage<D> St;

  const DecodeParams& p = f.d;
  const int G = p.Hq / p.Hkv, PSZ = 2 * G + G * D;
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int m = lane & 15, quarter = lane >> 4;
  const SegmentRows seg = range.seg;
  const bool is_apx = range.is_apx, paged = !is_apx && seg.blocks != nullptr;
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

  // query rows: column m holds row m, or m % 8
  u32x4 qf[kQueryParts][NC];
  {
    const int g = min(SIDE ? m & 7 : m, G - 1);
    const T* q = reinterpret_cast<const T*>(p.q) + ((size_t)range.b * p.Hq + (size_t)range.h * G + g) * D + quarter * (D / 4);
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      if constexpr (!kExact) {
        qf[0][c] = *reinterpret_cast<const u32x4*>(q + c * 8);
      } else {
        float x[8];
        load8(q + c * 8, x);
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

  f32x4 o[NT];
#pragma unroll
  for (int j = 0; j < NT; ++j) o[j] = zero;
  float ref = kNegBig, l_run = 0.f;

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
  const int32_t* positions = (ROPE && is_apx && rp.positions) ? rp.positions + seg.apx_row0 : nullptr;
  const bool turned = ROPE && is_apx;
  // what a lane brings in: a 16-byte piece of codes of one row (a load), and of one more kRowsPerLoad / 4 further on in every eight (the next
  // load); the scales of one row
  const int in_place = lane / St::kPieces, in_row = 8 * (in_place & 3) + (in_place >> 2);
  const int in_piece = (lane % St::kPieces) ^ St::twist(in_place);
  // (the second load's places are 16 further on, which the permutation does not see)
  const int scale_row = lane & 31;
  bool holes = false;                                  // a block that does not exist has been met

  auto fill = [&](int base, unsigned char* st) VEC_INLINE {
    int64_t at_lo = row0 + base, at_hi = at_lo;        // of the tile's first row, less 16 rows of its 17th
    bool lo = true, hi = true;
    if (paged) {
      if (((base + kFp4TileRows - 1) >> seg.block_shift) - window > kWave - 1) { window = base >> seg.block_shift; load_window(); }
      lo = hi = block_row(base, at_lo);
      at_hi = at_lo;
      if (seg.block_shift < 5) {
        hi = block_row(base + 16, at_hi);
        at_hi -= 16;
      }
    }
    const uint32_t to = lds_address(st);
    if (base + kFp4TileRows <= stored && lo && hi) {   // uniform: rows that are all there
      const int64_t row = (in_row < 16 ? at_lo : at_hi) + in_row;
      const uint8_t* k = k_codes + row * kCode + in_piece * 16;
#pragma unroll
      for (int i = 0; i < St::kLoads; ++i) load_to_lds16(to + i * 1024, k + i * (8 / St::kLoads) * kCode);
      if (!is_apx) {
        const uint8_t* r = r_codes + row * kCode + in_piece * 16;
#pragma unroll
        for (int i = 0; i < St::kLoads; ++i) load_to_lds16(to + St::kTensor + i * 1024, r + i * (8 / St::kLoads) * kCode);
      }
      const void* s = (lane < 32 ? k_scales : r_scales) + ((scale_row < 16 ? at_lo : at_hi) + scale_row) * kScale;
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
    if (new_row >= base && new_row < base + kFp4TileRows && lane < D / 4) {
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
  const int my_block = m / (16 / kScale);

  // under ROPE a lane's dims always belong to the same rotary pairs
  constexpr int kDims = D / 16;
  float t_hi[ROPE ? kDims : 1], t_lo[ROPE ? kDims : 1];
  if constexpr (ROPE) {
    if (is_apx) {
#pragma unroll
      for (int e = 0; e < kDims; ++e) {
        const int dim = kDims * m + e, i = rp.interleaved ? dim / 2 : dim % (D / 2);
        t_hi[e] = rp.turns_hi[i];
        t_lo[e] = rp.turns_lo[i];
      }
    }
  }
  auto consume = [&](const unsigned char* st, int base) VEC_INLINE {
    // scores, in the log2 domain
    float s[8];
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
      const float unit = fp4_unit(st[St::kSlots + row * 4 + (D == 128 ? quarter : quarter >> 1)]);
      f32x4 acc = zero;
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const uint32_t w = words[c];
        const u32x4 a = {fp4_pair_bf16<0>(w, unit), fp4_pair_bf16<1>(w, unit), fp4_pair_bf16<2>(w, unit), fp4_pair_bf16<3>(w, unit)};
#pragma unroll
        for (int part = 0; part < kQueryParts; ++part) acc = mfma(a, qf[part][c], acc);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) s[4 * u + i] = acc[i] * p.c2;
    }
    if (holes || base + kFp4TileRows > stored) {
      const uint32_t alive = *reinterpret_cast<const uint32_t*>(st + St::kAlive) >> r_row;
#pragma unroll
      for (int j = 0; j < 8; ++j) s[j] = (alive >> j & 1) ? s[j] : -INFINITY;
    }
    float top = s[0];
#pragma unroll
    for (int j = 1; j < 8; ++j) top = fmaxf(top, s[j]);
    // The reference of a column is raised only where a score lies far above it: the weights are then at most 2^kRaiseAt, and a
    // sum of them does not leave the range of a float.  The same in all lanes of a column.
    if (__ballot(top > ref + kRaiseAt)) {
      top = fmaxf(top, __shfl_xor(top, 16, kWave));
      top = fmaxf(top, __shfl_xor(top, 32, kWave));
      const float next = fmaxf(ref, top), by = fast_exp2(ref - next);
      l_run *= by;
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[j][i] *= by;
      ref = next;
    }
    float w[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      w[j] = fast_exp2(s[j] - ref);
      l_run += w[j];
    }
    u32x4 weights[kParts];
#pragma unroll
    for (int part = 0; part < kParts; ++part) {
      float y[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        y[j] = leading(w[j]);
        if constexpr (SIDE) { if (m >= 8) y[j] = w[j] - y[j]; }
        else w[j] -= y[j];
      }
      // what SIDE leaves has up to 16 bits and is rounded to the nearest eight; the others are cut exactly
#pragma unroll
      for (int i = 0; i < 4; ++i) weights[part][i] = SIDE ? pack_bf16(y[2 * i], y[2 * i + 1]) : high_halves(y[2 * i], y[2 * i + 1]);
    }
    // the eight rows of R, and their scales for the lane's dims
    uint32_t r[8];
    float unit[8];
    const unsigned char* rt = st + (is_apx ? 0 : St::kTensor);
    const unsigned char* slots = st + St::kSlots + (is_apx ? 0 : 128);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int at = St::piece(r_row + j, D == 128 ? m >> 2 : m >> 3);
      if constexpr (D == 128) r[j] = *reinterpret_cast<const uint32_t*>(rt + at + (m & 3) * 4);
      else r[j] = *reinterpret_cast<const uint16_t*>(rt + at + (m & 7) * 2);
    }
#pragma unroll
    for (int j = 0; j < 8; j += 4) {
      const u32x4 x = *reinterpret_cast<const u32x4*>(slots + (r_row + j) * 4);
#pragma unroll
      for (int i = 0; i < 4; ++i) unit[j + i] = fp4_unit(x[i] >> 8 * my_block & 0xffu);
    }
    if (!ROPE || !is_apx) {
      for_each_constant<kDims / 2>([&](auto c) VEC_INLINE {
        uint32_t two[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) two[j] = fp4_pair_bf16<decltype(c)::value>(r[j], unit[j]);
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
      });
      return;
    }
    if constexpr (ROPE) {
      // keys turned back, in one bf16 part (three for fp32): they carry that one rounding, as those of a bf16 cache do
      constexpr int kRowParts = kExact ? 3 : 1;
      float pos[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) pos[j] = (float)(*reinterpret_cast<const int*>(st + St::kPositions + (r_row + j) * 4) + rp.pos_offset);
      for_each_constant<kDims / 2>([&](auto c) VEC_INLINE {
        f32x2 two[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          f32x2 x = fp4_pair_f32<decltype(c)::value>(r[j], unit[j]);
          if (rp.interleaved) {
            float cs, sn;
            rotary_cos_sin(pos[j], t_hi[2 * c], t_lo[2 * c], cs, sn);
            float a, b;
            rotary_back(x[0], x[1], cs, sn, a, b);
            x[0] = a;
            x[1] = b;
          } else {
            // pairs (x[i], x[i + D / 2]): the other member is in the lane eight further on or back
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              float cs, sn;
              rotary_cos_sin(pos[j], t_hi[2 * c + e], t_lo[2 * c + e], cs, sn);
              const float other = __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x[e]), 0x128, 0xf, 0xf, false));   // row_ror:8
              x[e] = m < 8 ? fmaf(x[e], cs, other * sn) : fmaf(x[e], cs, -(other * sn));
            }
          }
          two[j] = x;
        }
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
          for (int rest = 0; rest < kRowParts; ++rest) {
            u32x4 a;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              if constexpr (kRowParts == 1) {
                a[i] = pack_bf16(two[2 * i][e], two[2 * i + 1][e]);
              } else {
                a[i] = high_halves(two[2 * i][e], two[2 * i + 1][e]);
                two[2 * i][e] -= leading(two[2 * i][e]);
                two[2 * i + 1][e] -= leading(two[2 * i + 1][e]);
              }
            }
#pragma unroll
            for (int part = 0; part + rest < kParts; ++part) o[2 * c + e] = mfma(a, weights[part], o[2 * c + e]);
          }
      });
    }
  };

  // loads of a tile; of tiles that went by the other way there are none on their way, nor of any before these
  const int per_tile = is_apx ? St::kLoads + 1 + (D == 64 && turned && positions ? 1 : 0) : 2 * St::kLoads + 1;
  static_assert(kFp4Stages == 3, "two tiles on their way while one is worked on");
  const int tiles = row_begin + wave * kFp4TileRows < row_end ? (row_end - row_begin - wave * kFp4TileRows + kStepRows - 1) / kStepRows : 0;
  const int first = row_begin + wave * kFp4TileRows;
  if (tiles > 0) fill(first, ring);
  if (tiles > 1) fill(first + kStepRows, ring + St::kBytes);
  // The query rows have arrived from here on.  Without this the wait for them would sit in the loop, and wait for tiles as well.
#pragma unroll
  for (int part = 0; part < kQueryParts; ++part)
#pragma unroll
    for (int c = 0; c < NC; ++c) asm volatile("" : "+v"(qf[part][c]));
  int stage = 0;
  for (int i = 0; i < tiles; ++i) {
    const int base = first + i * kStepRows;
    // the stage of the tile before is free: what was read of it is in registers
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    if (i + 2 < tiles) fill(base + 2 * kStepRows, ring + (stage == 0 ? 2 : stage - 1) * St::kBytes);
    wait_tiles(per_tile * min(2, tiles - 1 - i));
    wave_fence();
    consume(ring + stage * St::kBytes, base);
    stage = stage == 2 ? 0 : stage + 1;
  }

  // ---- merge the waves ----
  // a wave's sums in the place of its own ring
  constexpr int kWaveBytes = kFp4Stages * St::kBytes;
  static_assert(16 * kRedStride * 4 + 2 * 16 * 4 <= kWaveBytes, "the merge area must fit in the ring");
  auto red = [&](int wv, int col, int j) VEC_INLINE { return reinterpret_cast<float*>(fp4_lds + wv * kWaveBytes) + col * kRedStride + j; };
  auto ml = [&](int wv, int what, int col) VEC_INLINE { return reinterpret_cast<float*>(fp4_lds + wv * kWaveBytes) + 16 * kRedStride + what * 16 + col; };
  wave_fence();
  float l_tot = l_run + __shfl_xor(l_run, 16, kWave);
  l_tot += __shfl_xor(l_tot, 32, kWave);
  // lane (m, quarter): column m, dims kDims * (4 quarter + i) + j
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < NT; j += 4)
      *reinterpret_cast<f32x4*>(red(wave, m, kDims * (4 * quarter + i) + j)) = f32x4{o[j][i], o[j + 1][i], o[j + 2][i], o[j + 3][i]};
  if (quarter == 0) {
    *ml(wave, 0, m) = l_tot > 0.f ? ref : -INFINITY;    // a wave without rows: its share is 0 without a branch
    *ml(wave, 1, m) = l_tot;
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
      f32x4 x = *reinterpret_cast<const f32x4*>(red(wv, g, j));
      if constexpr (SIDE) x += *reinterpret_cast<const f32x4*>(red(wv, 8 + g, j));
#pragma unroll
      for (int e = 0; e < 4; ++e) a[e] = fmaf(x[e], sc, a[e]);
      l = fmaf(*ml(wv, 1, g), sc, l);
    }
    *reinterpret_cast<f32x4_u*>(out + 2 * G + i) = a;
    if (j == 0) {
      out[2 * g] = top;
      out[2 * g + 1] = l;
    }
  }
}

template <typename T, int D, bool SIDE, bool ROPE>
__global__ __launch_bounds__(DT_, 3) void decode_split_fp4_kernel(Fp4Params f, RopeParams rp) {
  attend_fp4<T, D, SIDE, ROPE>(f, rp, grid_split<DW * kFp4TileRows>(f.d), (int)threadIdx.x);
}

template <typename T, int D, bool SIDE, bool ROPE>
int launch_split_fp4(const Fp4Params& f, const RopeParams* rope, hipStream_t stream) {
  const dim3 grid(f.d.splits_ret + f.d.splits_apx, f.d.Hkv, f.d.B);
  constexpr int lds = DW * kFp4Stages * Fp4Stage<D>::kBytes;
  VEC_HIP(set_max_lds(reinterpret_cast<const void*>(decode_split_fp4_kernel<T, D, SIDE, ROPE>), lds));
  VEC_LAUNCH(K_DECODE_SPLIT, (decode_split_fp4_kernel<T, D, SIDE, ROPE>), grid, dim3(DT_), lds, stream, f, rope ? *rope : RopeParams{});
  VEC_HIP(hipGetLastError());
  return VECTOR_OK;
}

template <typename T, int D>
int run_split_fp4(Fp4Params& f, const RopeParams* rope, hipStream_t stream) {
  pick_splits_fp4(f.d.B, f.d.Hkv, f.d.cap_retain, f.d.n_approx, f.d.splits_ret, f.d.splits_apx);
  const bool turned = rope && f.d.n_approx > 0;
  if constexpr (sizeof(T) == 2) {
    if (f.d.Hq / f.d.Hkv <= 8)
      return turned ? launch_split_fp4<T, D, true, true>(f, rope, stream) : launch_split_fp4<T, D, true, false>(f, rope, stream);
  }
  return turned ? launch_split_fp4<T, D, false, true>(f, rope, stream) : launch_split_fp4<T, D, false, false>(f, rope, stream);
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
  p.c2 = scale * kLog2e;
  f.k_ret_scale = c.k_ret_scale; f.v_ret_scale = c.v_ret_scale; f.k_apx_scale = c.k_apx_scale;
  f.n_blocks = c.n_blocks;
  int rc;
  if (c.dtype == VECTOR_BF16) rc = c.head_dim == 128 ? run_split_fp4<bf16_t, 128>(f, rope, stream) : run_split_fp4<bf16_t, 64>(f, rope, stream);
  else rc = c.head_dim == 128 ? run_split_fp4<float, 128>(f, rope, stream) : run_split_fp4<float, 64>(f, rope, stream);
  return rc ? rc : launch_decode_merge(p, c.dtype, c.head_dim, stream);
}

}  // namespace vec
