// Decode attention over caches held in 4 bits (vector_decode_attn_fp4, vector_decode_step_fp4): the same sum as over caches in 16 or 32 bits
// (decode_attn.hip), one softmax over the live retained rows and the approximated ones, z = sum p k over the latter, the same
// partial results and the same merge.
//
// What bounds it is memory, 136 bytes for the key and the value of a token at 128 dims, against 512 in bf16; but a quarter of the bytes
// leaves a quarter of the time for a row's arithmetic.  Both products run on the matrix cores in bf16 with fp32 sums:
// an element in 4 bits times its scale has two significant bits and is a bf16 number exactly, so the only
// roundings are those of the weights, which go in as parts of eight bits each (kParts).
//
// Nothing passes through LDS before the end and no wave waits for another: a wave takes 32 rows at a time, and both operands come
// straight from memory in the matrix cores' order.
//   scores   S[t][g] = sum_e K[t][e] q[g][e]      A = K: lane (m, quarter) holds D / 4 consecutive elements of a row, which is one load and
//                                                  one scale; B = the query rows in the same order of e
//   output   O[j][g] += sum_t R[t][j] P[t][g]     A = R^T: lane (m, quarter) holds dims D / 16 m .. of eight rows, 8 quarter ..; the conversion
//                                                  hands out two neighbouring dims of one row, and a byte permutation makes
//                                                  two rows of one dim of them
// Row 4 a + i of score tile u is token 8 a + 4 u + i, so that the eight weights that a lane gets from both score tiles are those
// of the eight rows that it holds of R.  R is the values, or for approximated rows the keys, loaded a second time in the other order
// (from the caches); under ROPE these are turned back by their positions first.
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

// rounds a weight to its leading eight bits by cutting the others off: what is left is exact
__device__ __forceinline__ float leading(float x) { return __uint_as_float(__float_as_uint(x) & 0xffff0000u); }
// two floats with no more than eight significant bits as two bf16
__device__ __forceinline__ uint32_t high_halves(float lo, float hi) {
  return __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
}

template <int D> struct Fp4Tile {
  static constexpr int kWords = D / 32;      // of a lane's part of a key row
  uint32_t k[2][kWords], k_unit[2];          // scales as they are, a byte
  uint32_t r[8];                             // codes of D / 16 dims of eight rows
  u32x4 r_unit[D / 64];                      // scale bytes of these rows, D / 32 a row
  uint32_t dead;                             // bit j: row j of the eight is none
};

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
  const int live = is_apx ? seg.n_approx : seg.len_retain;
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
  auto load_window = [&]() VEC_INLINE { ids = seg.blocks[min(window + lane, p.blocks_per_seq - 1)]; };
  if (paged) load_window();
  // first row, in the pools, of the tile's 16 rows from `row` on; false: there are none
  auto block_row = [&](int row, int64_t& at) VEC_INLINE {
    const int id = __builtin_amdgcn_readlane(ids, (row >> seg.block_shift) - window);
    at = ((int64_t)id << seg.block_shift) + (row & ((1 << seg.block_shift) - 1));
    return (uint32_t)id < (uint32_t)f.n_blocks && (row >> seg.block_shift) < p.blocks_per_seq;
  };

  // rows of a lane inside a tile: of the key tiles (+ 4 for the second one), the first of the eight of R
  const int k_row = 8 * (m >> 2) + (m & 3), r_row = 8 * quarter;
  auto load_key = [&](Fp4Tile<D>& t, int u, int64_t row) VEC_INLINE {
    if constexpr (D == 128) {
      const u32x4 x = *reinterpret_cast<const u32x4*>(k_codes + row * kCode + quarter * 16);
#pragma unroll
      for (int i = 0; i < 4; ++i) t.k[u][i] = x[i];
      t.k_unit[u] = k_scales[row * kScale + quarter];
    } else {
      const u32x2 x = *reinterpret_cast<const u32x2*>(k_codes + row * kCode + quarter * 8);
      t.k[u][0] = x[0];
      t.k[u][1] = x[1];
      t.k_unit[u] = k_scales[row * kScale + (quarter >> 1)];
    }
  };
  auto load_r = [&](int64_t row) VEC_INLINE {
    if constexpr (D == 128) return *reinterpret_cast<const uint32_t*>(r_codes + row * kCode + m * 4);
    else return (uint32_t)*reinterpret_cast<const uint16_t*>(r_codes + row * kCode + m * 2);
  };
  // codes and scale of a block of the step's token, elements first .. first + 7 of it
  auto new_codes = [&](const void* token, int block, int first, uint32_t& byte) VEC_INLINE {
    const T* x = reinterpret_cast<const T*>(token) + bh * D + block * kFp4Block;
    uint32_t top = 0;
    float y[8];
#pragma unroll
    for (int i = 0; i < kFp4Block; i += 8) { load8(x + i, y); top = max(top, top_bits8(y)); }
    byte = fp4_scale_byte(top);
    load8(x + first, y);
    return fp4_codes(y, byte);
  };

  auto fetch = [&](Fp4Tile<D>& t, int base) VEC_INLINE {
    int64_t k_at = row0 + base, r_at = row0 + base;         // of the tile's first row, or (blocks of 16 rows) of the lane's half
    bool there = true, k_there = true, r_there = true;
    if (paged) {
      if (((base + kFp4TileRows - 1) >> seg.block_shift) - window > kWave - 1) { window = base >> seg.block_shift; load_window(); }
      int64_t at[2];
      bool ok[2];
      ok[0] = block_row(base, at[0]);
      if (seg.block_shift >= 5) {
        k_at = r_at = at[0];
        there = k_there = r_there = ok[0];
      } else {
        ok[1] = block_row(base + 16, at[1]);
        at[1] -= 16;
        there = ok[0] && ok[1];
        k_at = (m >> 3) ? at[1] : at[0];
        r_at = (quarter >> 1) ? at[1] : at[0];
        k_there = (m >> 3) ? ok[1] : ok[0];
        r_there = (quarter >> 1) ? ok[1] : ok[0];
      }
    }
    t.dead = 0;
    if (base + kFp4TileRows <= stored && there) {           // uniform: rows that are all there
#pragma unroll
      for (int u = 0; u < 2; ++u) load_key(t, u, k_at + k_row + 4 * u);
#pragma unroll
      for (int j = 0; j < 8; ++j) t.r[j] = load_r(r_at + r_row + j);
      const uint8_t* s = r_scales + (r_at + r_row) * kScale;
      if constexpr (D == 128) {
        t.r_unit[0] = *reinterpret_cast<const u32x4_a4*>(s);
        t.r_unit[1] = *reinterpret_cast<const u32x4_a4*>(s + 16);
      } else {
        t.r_unit[0] = *reinterpret_cast<const u32x4_a2*>(s);
      }
      return;
    }
    // The last rows, rows of blocks that do not exist, the step's own token: row by row.  What is no row is all zeros, since a
    // weight of 0 does not make a NaN of the memory harmless.
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int row = base + k_row + 4 * u;
      t.k_unit[u] = 0;
#pragma unroll
      for (int i = 0; i < Fp4Tile<D>::kWords; ++i) t.k[u][i] = 0;
      if (row < stored && k_there) load_key(t, u, k_at + k_row + 4 * u);
      if (row == new_row) {
        constexpr int kBlockOf = D == 128 ? 1 : 2;           // lanes of a block
        const int block = quarter / kBlockOf, inside = quarter % kBlockOf * 16;
        uint32_t byte = 0;
#pragma unroll
        for (int i = 0; i < Fp4Tile<D>::kWords; ++i) t.k[u][i] = new_codes(p.k_new, block, inside + 8 * i, byte);
        t.k_unit[u] = byte;
        if (new_row < seg.cap && k_there) {
          const int64_t at = k_at + k_row + 4 * u;
          uint8_t* codes = const_cast<uint8_t*>(k_codes) + at * kCode + quarter * (D / 8);
#pragma unroll
          for (int i = 0; i < Fp4Tile<D>::kWords; ++i) reinterpret_cast<uint32_t*>(codes)[i] = t.k[u][i];
          if (quarter % kBlockOf == 0) const_cast<uint8_t*>(k_scales)[at * kScale + block] = (uint8_t)byte;
        }
      }
    }
    uint32_t unit[D == 128 ? 8 : 4];
#pragma unroll
    for (int j = 0; j < (D == 128 ? 8 : 4); ++j) unit[j] = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int row = base + r_row + j;
      uint32_t scales = 0;                                    // the row's, of all blocks
      t.r[j] = 0;
      if (row < stored && r_there) {
        t.r[j] = load_r(r_at + r_row + j);
        const uint8_t* s = r_scales + (r_at + r_row + j) * kScale;
        if constexpr (D == 128) scales = *reinterpret_cast<const uint32_t*>(s);
        else scales = *reinterpret_cast<const uint16_t*>(s);
      } else if (row != new_row) {
        t.dead |= 1u << j;
      }
      if (row == new_row) {
        const int block = m / (16 / kScale), inside = m % (16 / kScale) * (D / 16);
        uint32_t byte = 0, codes = new_codes(p.v_new, block, inside & ~7, byte);
        if constexpr (D == 64) codes = codes >> (m & 1) * 16 & 0xffffu;
        t.r[j] = codes;
        scales = byte << 8 * block;
        if (new_row < seg.cap && r_there) {
          const int64_t at = r_at + r_row + j;
          uint8_t* to = const_cast<uint8_t*>(r_codes) + at * kCode + m * (D / 32);
          if constexpr (D == 128) *reinterpret_cast<uint32_t*>(to) = codes;
          else *reinterpret_cast<uint16_t*>(to) = (uint16_t)codes;
          if (inside == 0) const_cast<uint8_t*>(r_scales)[at * kScale + block] = (uint8_t)byte;
        }
      }
      if constexpr (D == 128) unit[j] = scales;
      else unit[j / 2] |= scales << (j & 1) * 16;
    }
#pragma unroll
    for (int j = 0; j < (D == 128 ? 8 : 4); ++j) t.r_unit[j / 4][j % 4] = unit[j];
  };

  // the scale of row j of the eight, for the lane's dims
  const int my_block = m / (16 / kScale);
  auto row_unit = [&](const Fp4Tile<D>& t, int j) VEC_INLINE {
    const uint32_t word = D == 128 ? t.r_unit[j / 4][j % 4] : t.r_unit[0][j / 2] >> (j & 1) * 16;
    return fp4_unit(word >> 8 * my_block & 0xffu);
  };

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
  const int32_t* positions = (ROPE && is_apx && rp.positions) ? rp.positions + seg.apx_row0 : nullptr;

  auto consume = [&](const Fp4Tile<D>& t, int base) VEC_INLINE {
    // scores, in the log2 domain
    float s[8];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const float unit = fp4_unit(t.k_unit[u]);
      f32x4 acc = zero;
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const uint32_t w = t.k[u][c];
        const u32x4 a = {fp4_pair_bf16<0>(w, unit), fp4_pair_bf16<1>(w, unit), fp4_pair_bf16<2>(w, unit), fp4_pair_bf16<3>(w, unit)};
#pragma unroll
        for (int part = 0; part < kQueryParts; ++part) acc = mfma(a, qf[part][c], acc);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) s[4 * u + i] = acc[i] * p.c2;
    }
    if (__ballot(t.dead != 0)) {
#pragma unroll
      for (int j = 0; j < 8; ++j) s[j] = (t.dead >> j & 1) ? -INFINITY : s[j];
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
    float unit[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) unit[j] = row_unit(t, j);
    if (!ROPE || !is_apx) {
      for_each_constant<kDims / 2>([&](auto c) VEC_INLINE {
        uint32_t two[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) two[j] = fp4_pair_bf16<decltype(c)::value>(t.r[j], unit[j]);
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
      for (int j = 0; j < 8; ++j) {
        const int row = min(base + r_row + j, live - 1);
        pos[j] = (float)((positions ? positions[row] : row) + rp.pos_offset);
      }
      for_each_constant<kDims / 2>([&](auto c) VEC_INLINE {
        f32x2 two[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          f32x2 x = fp4_pair_f32<decltype(c)::value>(t.r[j], unit[j]);
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

  int base = row_begin + wave * kFp4TileRows;
  Fp4Tile<D> next;
  if (base < row_end) fetch(next, base);
  while (base < row_end) {
    const Fp4Tile<D> tile = next;
    const int then = base + kStepRows;
    if (then < row_end) fetch(next, then);           // in flight while this tile is consumed
    consume(tile, base);
    base = then;
  }

  // ---- merge the waves ----
  __shared__ float red[DW][16][kRedStride];
  __shared__ float ml[DW][2][16];
  float l_tot = l_run + __shfl_xor(l_run, 16, kWave);
  l_tot += __shfl_xor(l_tot, 32, kWave);
  // lane (m, quarter): column m, dims kDims * (4 quarter + i) + j
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < NT; j += 4)
      *reinterpret_cast<f32x4*>(&red[wave][m][kDims * (4 * quarter + i) + j]) = f32x4{o[j][i], o[j + 1][i], o[j + 2][i], o[j + 3][i]};
  if (quarter == 0) {
    ml[wave][0][m] = l_tot > 0.f ? ref : -INFINITY;    // a wave without rows: its share is 0 without a branch
    ml[wave][1][m] = l_tot;
  }
  __syncthreads();
  float* out = p.part + range.slot * PSZ;
  for (int i = tid * 4; i < G * D; i += DT_ * 4) {
    const int g = i / D, j = i % D;
    float top = -INFINITY, l = 0.f;
#pragma unroll
    for (int wv = 0; wv < DW; ++wv) top = fmaxf(top, ml[wv][0][g]);
    const float safe = top == -INFINITY ? 0.f : top;
    f32x4 a = zero;
#pragma unroll
    for (int wv = 0; wv < DW; ++wv) {
      const float sc = fast_exp2(ml[wv][0][g] - safe);
      f32x4 x = *reinterpret_cast<const f32x4*>(&red[wv][g][j]);
      if constexpr (SIDE) x += *reinterpret_cast<const f32x4*>(&red[wv][8 + g][j]);
#pragma unroll
      for (int e = 0; e < 4; ++e) a[e] = fmaf(x[e], sc, a[e]);
      l = fmaf(ml[wv][1][g], sc, l);
    }
    *reinterpret_cast<f32x4_u*>(out + 2 * G + i) = a;
    if (j == 0) {
      out[2 * g] = top;
      out[2 * g + 1] = l;
    }
  }
}

template <typename T, int D, bool SIDE, bool ROPE>
__global__ __launch_bounds__(DT_, 2) void decode_split_fp4_kernel(Fp4Params f, RopeParams rp) {
  attend_fp4<T, D, SIDE, ROPE>(f, rp, grid_split<DW * kFp4TileRows>(f.d), (int)threadIdx.x);
}

template <typename T, int D, bool SIDE, bool ROPE>
int launch_split_fp4(const Fp4Params& f, const RopeParams* rope, hipStream_t stream) {
  const dim3 grid(f.d.splits_ret + f.d.splits_apx, f.d.Hkv, f.d.B);
  VEC_LAUNCH(K_DECODE_SPLIT, (decode_split_fp4_kernel<T, D, SIDE, ROPE>), grid, dim3(DT_), 0, stream, f, rope ? *rope : RopeParams{});
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
