// Device code of the decode over an 8-bit cache (decode_q8.hip): one step of a wave
// over a pair of 16-slot blocks of one (row, KV head) segment.
//
// As in the 16-bit decode, the G query heads of a KV head form a dense product per
// block, and the softmax weights never move between lanes. Lane l = 16 grp + col:
//   S^T[slot][head] = K[slot][:] . q[head][:]         mfma 16x16x32, four a block
//   O^T[dim][head] += V^T[dim][slot] P^T[slot][head]  mfma 16x16x32, eight a pair
// In the C layout of the first product lane l holds the scores of four K rows for head
// col, and which slots these are is free (slot_of): those whose V rows the lane has.
// The 32 slots of a pair are ordered so that the four of the first block and the four of
// the second are the eight the second product wants in that lane.
//
// Codes become bf16 values in registers, two per instruction (exact; V's scale is
// applied on the way, K's to the scores, a power of two either way), so what follows
// is the 16-bit decode of the values the cache stands for.
//
// What bounds a step is how the memory system takes its reads. 288 rows of 256 to 16384
// tokens, 64 / 8 heads, take 820 us, 6.0 TB/s; before V's loads were joined as below it was
// 834, and 852 with all arithmetic taken out. Fewer load instructions and reads that
// lie together help:
//   K: the lane reads row slot_of(col / 4, col % 4), dims 16 grp .. + 15 and 64 + 16 grp ..
//      + 15 (the contraction's order of dims is free, q uses the same).
//   V: an instruction reads eight rows of a block, 1 KiB: lane (grp, col) reads 16 codes,
//      chunk col % 8, of rows 2 grp + col / 8 and 8 + 2 grp + col / 8; lanes col and col + 8
//      then swap halves, so that both have 8 codes of the four rows, dims 16 (col % 8) +
//      8 (col / 8) .. + 7. Output row m of product t is that of lane col = m, plus t, so lane
//      l ends up with dims run_dim(grp) + 16 r + t of head col.
//   Scales: one instruction for both blocks' K and V.
#pragma once

#include "decode_device.h"
#include "q8_device.h"

namespace bros {
namespace dq {

using dm::bf16x8_t;
using dm::floatx4_t;
using dm::load_uniform;
using q8::v2u_t;

constexpr int kPairSlots = 2 * kBlockSize;           // slots of a step
constexpr int kTileBytes = kBlockSize * kHeadDim;    // codes of one (block, KV head), K or V
constexpr int kScaleBytes = 2 * kBlockSize;          // its scales, K then V

// What a wave has read of a pair.
struct KRegs {
  v4u_t lo[2], hi[2];   // per block, row col: dims 16 grp .., 64 + 16 grp ..
};
struct VRegs {
  v4u_t row[2][2];      // per block, rows 8 i + 2 grp + col / 8: dims 16 (col % 8) ..
  uint32_t scales;      // lane col % 8 = 4 x + 2 w + i: block x's scale bytes of slots 8 i + 2 grp, + 1, K (w = 0) or V
};

// Slot of the r-th score of a lane of group grp.
__device__ __forceinline__ int slot_of(int grp, int r) { return 8 * (r >> 1) + 2 * grp + (r & 1); }

// First of the four runs of 8 dims a lane holds of the output, 16 apart.
__device__ __forceinline__ int run_dim(int grp) { return 64 * (grp & 1) + 8 * (grp >> 1); }

__device__ __forceinline__ v4u_t load16(const uint8_t* p) { return __builtin_nontemporal_load(reinterpret_cast<const v4u_t*>(p)); }

// tile0, tile1: the (block, KV head) rows of the pair's two blocks, uniform.
__device__ __forceinline__ void issue_k(const Q8Pool& p, size_t tile0, size_t tile1, int grp, int col, KRegs& k) {
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    const uint8_t* b = p.k + (x ? tile1 : tile0) * kTileBytes + (uint32_t)(slot_of(col >> 2, col & 3) * kHeadDim + 16 * grp);
    k.lo[x] = load16(b);
    k.hi[x] = load16(b + 64);
  }
}
__device__ __forceinline__ void issue_v(const Q8Pool& p, size_t tile0, size_t tile1, int grp, int col, VRegs& v) {
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    const uint8_t* b = p.v + (x ? tile1 : tile0) * kTileBytes + (uint32_t)((2 * grp + (col >> 3)) * kHeadDim + 16 * (col & 7));
    v.row[x][0] = load16(b);
    v.row[x][1] = load16(b + 8 * kHeadDim);
  }
  // (32 bytes of scales for 4 KiB of codes: their offsets stay below 4 GiB on any card)
  const uint32_t t = (uint32_t)((col & 4) ? tile1 : tile0);
  v.scales = *reinterpret_cast<const uint16_t*>(p.scales + (t * kScaleBytes + (uint32_t)(8 * (col & 3) + 2 * grp)));
}

// The lane's column of the query, in the order of K's dims: row `head` of q.
__device__ __forceinline__ void load_q_row(const void* q, size_t head, int grp, v4u_t (&qf)[4]) {
  const uint16_t* p = static_cast<const uint16_t*>(q) + head * kHeadDim + 16 * grp;
#pragma unroll
  for (int c = 0; c < 4; ++c) qf[c] = *reinterpret_cast<const v4u_t*>(p + 64 * (c >> 1) + 8 * (c & 1));
}
// A segment's (padding columns repeat a head).
template <int G>
__device__ __forceinline__ void load_q(const void* q, size_t first_head, int grp, int col, v4u_t (&qf)[4]) {
  load_q_row(q, first_head + min(col, G - 1), grp, qf);
}

// Products of a block's codes with the query: slots slot_of(grp, r) of head col, without K's scale.
__device__ __forceinline__ floatx4_t block_products(const v4u_t& lo, const v4u_t& hi, const v4u_t (&qf)[4]) {
  floatx4_t sc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    const v4u_t& w = c < 2 ? lo : hi;
    const uint32_t w0 = w[2 * (c & 1)], w1 = w[2 * (c & 1) + 1];
    const v4u_t kv = {q8::values2_bf16<false>(w0, 1.0f), q8::values2_bf16<true>(w0, 1.0f), q8::values2_bf16<false>(w1, 1.0f),
                      q8::values2_bf16<true>(w1, 1.0f)};
    sc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, kv), __builtin_bit_cast(bf16x8_t, qf[c]), sc, 0, 0, 0);
  }
  return sc;
}

// The scale bytes of a pair as words of four slots (slot_of), in every lane: block x's K
// (w = 0) or V. From the two-byte pieces of lanes 4 x + 2 w and the next of each 16.
struct PairScales {
  uint32_t w[2][2];
};
template <int LANE>
__device__ __forceinline__ uint32_t of_row(uint32_t w) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)w, 0x150 + LANE, 0xf, 0xf, true);   // row_newbcast
}
__device__ __forceinline__ PairScales pair_scales(uint32_t two) {
  const uint32_t next = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)two, 0xb1, 0xf, 0xf, true);   // quad_perm: the neighbour's
  const uint32_t four = two | (next << 16);   // (as wanted in the even lanes)
  return PairScales{{{of_row<0>(four), of_row<2>(four)}, {of_row<4>(four), of_row<6>(four)}}};
}
__device__ __forceinline__ float byte_scale(uint32_t w, int j) { return q8::scale_of((w >> (8 * j)) & 0xffu); }

// Scores of a pair in log2 units, slots slot_of(grp, r) of the first block, then of the second.
__device__ __forceinline__ void pair_scores(const KRegs& k, const v4u_t (&qf)[4], const PairScales& ps, float scale_log2, float (&s)[8]) {
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    const floatx4_t sc = block_products(k.lo[x], k.hi[x], qf);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      // (byte 255, the scale of no number, is infinite here: added to the score it makes NaN of what would else be
      // an infinity, and a key without weight where it is negative)
      const float f = byte_scale(ps.w[x][0], r);
      s[4 * x + r] = fmaf(sc[r] * scale_log2, f, f - f);
    }
  }
}

// The V rows of a pair as the second product takes them: row slot_of(grp, j) of block x,
// the lane's eight dims, and the rows' scale bytes.
struct VRows {
  v2u_t row[2][4];
  uint32_t scales[2];
};
__device__ __forceinline__ VRows exchange(const VRegs& v, const PairScales& ps) {
  constexpr int kShl8 = 0x108, kShr8 = 0x118;   // row_shl:8, row_shr:8: from lane + 8, from lane - 8 of 16
  VRows o;
#pragma unroll
  for (int x = 0; x < 2; ++x) {
#pragma unroll
    for (int n = 0; n < 2; ++n) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int low = (int)v.row[x][n][i], high = (int)v.row[x][n][2 + i];
        // the even row: lanes 0..7 have it and keep its low half, lanes 8..15 get its high half
        o.row[x][2 * n][i] = (uint32_t)__builtin_amdgcn_update_dpp(low, high, kShr8, 0xf, 0xc, false);
        // the odd row: lanes 8..15 have it and keep its high half, lanes 0..7 get its low half
        o.row[x][2 * n + 1][i] = (uint32_t)__builtin_amdgcn_update_dpp(high, low, kShl8, 0xf, 0x3, false);
      }
    }
    o.scales[x] = ps.w[x][1];
  }
  return o;
}

// A wave's running result over its part of a segment, per head col.
struct Running {
  floatx4_t acc[8];   // acc[t][r]: dim run_dim(grp) + 16 r + t
  float m_ref, l_part;

  __device__ __forceinline__ void clear() {
    m_ref = kNoMax;
    l_part = 0.0f;
#pragma unroll
    for (int t = 0; t < 8; ++t) acc[t] = floatx4_t{0.0f, 0.0f, 0.0f, 0.0f};
  }

  // Folds a pair in: s its scores (-inf where masked), v its V rows. kTwoParts: the weights as
  // two bf16 values instead of one.
  template <bool kTwoParts>
  __device__ __forceinline__ void fold(const float (&s)[8], const VRows& v, bool head_lane) {
    float mx = fmaxf(fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3])), fmaxf(fmaxf(s[4], s[5]), fmaxf(s[6], s[7])));
    if (__builtin_amdgcn_ballot_w64(head_lane && mx > m_ref + kRescaleSlack) != 0) {
      // rare: move each head's reference max to the max over the pair's slots
      mx = fmaxf(mx, __shfl_xor(mx, 16));
      mx = fmaxf(mx, __shfl_xor(mx, 32));
      const float m_new = fmaxf(m_ref, mx);
      const float alpha = fast_exp2(m_ref - m_new);
      m_ref = m_new;
      l_part *= alpha;
#pragma unroll
      for (int t = 0; t < 8; ++t) {
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[t][r] *= alpha;
      }
    }
    float p[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) p[i] = fast_exp2(s[i] - m_ref);
    // The weights as a bf16 and the bf16 of what it leaves: 8 bits more for eight
    // products a pair, which cost the decode nothing measurable. The total is that of the weights
    // which the products apply: what many alike keys lose in rounding it loses too. (Of two parts
    // it takes the fp32 weights: they differ by 2^-16 of them.)
    const v4u_t hi4 = {q8::pack2_bf16(p[0], p[1]), q8::pack2_bf16(p[2], p[3]), q8::pack2_bf16(p[4], p[5]), q8::pack2_bf16(p[6], p[7])};
    v4u_t lo4 = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int i = 0; kTwoParts && i < 4; ++i) lo4[i] = q8::pack2_bf16(p[2 * i] - bf16_lo(hi4[i]), p[2 * i + 1] - bf16_hi(hi4[i]));
    if constexpr (kTwoParts) {
      l_part += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t two = hi4[i];   // (a bit cast of the vector's element itself reads its first)
        l_part = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(q8::bf16x2_t, two), q8::bf16x2_t{(__bf16)1.0f, (__bf16)1.0f}, l_part, false);
      }
    }
    const bf16x8_t ph = __builtin_bit_cast(bf16x8_t, hi4), pl = __builtin_bit_cast(bf16x8_t, lo4);
    float sc[2][4];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
#pragma unroll
      for (int j = 0; j < 4; ++j) sc[x][j] = byte_scale(v.scales[x], j);
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {   // dims 2 u and 2 u + 1 of the lane's eight
      uint32_t w[2][4];
#pragma unroll
      for (int x = 0; x < 2; ++x) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          w[x][j] = (u & 1) ? q8::values2_bf16<true>(v.row[x][j][u >> 1], sc[x][j]) : q8::values2_bf16<false>(v.row[x][j][u >> 1], sc[x][j]);
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t sel = h ? 0x07060302u : 0x05040100u;
        const v4u_t vt = {__builtin_amdgcn_perm(w[0][1], w[0][0], sel), __builtin_amdgcn_perm(w[0][3], w[0][2], sel),
                          __builtin_amdgcn_perm(w[1][1], w[1][0], sel), __builtin_amdgcn_perm(w[1][3], w[1][2], sel)};
        const bf16x8_t va = __builtin_bit_cast(bf16x8_t, vt);
        const int t = 2 * u + h;
        acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, ph, acc[t], 0, 0, 0);
        if constexpr (kTwoParts) acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, pl, acc[t], 0, 0, 0);
      }
    }
  }

  // NaN where the lane's column sees a marked value: `marks` holds a byte that is not zero
  // in its place, `seen` a bf16 one for each slot that the column sees.
  __device__ __forceinline__ void spoil(const VRows& marks, const uint32_t (&seen)[4]) {
    const bf16x8_t p = __builtin_bit_cast(bf16x8_t, v4u_t{seen[0], seen[1], seen[2], seen[3]});
#pragma unroll
    for (int t = 0; t < 8; ++t) {
      uint32_t w[2][4];
#pragma unroll
      for (int x = 0; x < 2; ++x) {
#pragma unroll
        for (int j = 0; j < 4; ++j) w[x][j] = (marks.row[x][j][t >> 2] >> (8 * (t & 3))) & 0xffu ? 0x3f80u : 0u;
      }
      const v4u_t vt = {w[0][0] | w[0][1] << 16, w[0][2] | w[0][3] << 16, w[1][0] | w[1][1] << 16, w[1][2] | w[1][3] << 16};
      const floatx4_t hit = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, vt), p, floatx4_t{0.0f, 0.0f, 0.0f, 0.0f}, 0, 0, 0);
#pragma unroll
      for (int r = 0; r < 4; ++r) acc[t][r] = hit[r] > 0.0f ? __uint_as_float(0x7fc00000u) : acc[t][r];
    }
  }

  // The weights' total of head col, in every lane of the head.
  __device__ __forceinline__ float total() const {
    float l = l_part;
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    return l;
  }

  // The lane's dims of head col as fp32 / as bf16 times inv, at `o` (the head's dim 0).
  __device__ __forceinline__ void store(float* o, int grp) const {
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      float* d = o + run_dim(grp) + 16 * r;
      *reinterpret_cast<floatx4_t*>(d) = floatx4_t{acc[0][r], acc[1][r], acc[2][r], acc[3][r]};
      *reinterpret_cast<floatx4_t*>(d + 4) = floatx4_t{acc[4][r], acc[5][r], acc[6][r], acc[7][r]};
    }
  }
  __device__ __forceinline__ void store_bf16(uint16_t* o, int grp, float inv) const {
#pragma unroll
    for (int r = 0; r < 4; ++r)
      *reinterpret_cast<v4u_t*>(o + run_dim(grp) + 16 * r) =
          v4u_t{q8::pack2_bf16(acc[0][r] * inv, acc[1][r] * inv), q8::pack2_bf16(acc[2][r] * inv, acc[3][r] * inv),
                q8::pack2_bf16(acc[4][r] * inv, acc[5][r] * inv), q8::pack2_bf16(acc[6][r] * inv, acc[7][r] * inv)};
  }
};

// Removes what a pair's blocks do not hold of the context: block b0 + x is `ok`, or
// an entry outside the pool (or a block past the context); slots from ctx on belong
// to nobody or to a peer. By selection, so that no value there leaks.
__device__ __forceinline__ void mask_pair(const DecodeArgs& a, int row, int ctx, int b0, const bool (&ok)[2], int grp,
                                          float (&s)[8], VRows& v) {
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    const int b = b0 + x;
    if (ok[x] && (b + 1) * kBlockSize <= ctx) continue;
    const int dir = ok[x] ? entry_direction(a.dir, a.cls, a.dir_per_entry, a.max_blocks_per_seq, row, b) : 1;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      if (!ok[x] || b * kBlockSize + slot_of_offset(slot_of(grp, r), dir) >= ctx) {
        s[4 * x + r] = -INFINITY;
        v.row[x][r] = v2u_t{0u, 0u};
        v.scales[x] &= ~(0xffu << (8 * r));   // (0 times 2^-127)
      }
    }
  }
}

// Folds pairs first, first + STRIDE, ... of blocks below b1 of sequence `seq`, KV head g, into
// `run`. `head` is the lane's row of q; pairs that end above position `plain`, or have a block
// outside the pool, go through mask(first block, ok, scores, V rows).
template <int STRIDE, bool kTwoParts, class Args, class Mask>
__device__ __forceinline__ void fold_pairs(const Args& a, const Q8Pool& pool, int seq, int g, size_t head, int first, int b1,
                                           int plain, bool head_lane, Running& run, Mask mask) {
  const int lane = threadIdx.x & (kWave - 1);
  const int grp = lane >> 4;
  const int col = lane & 15;
  const int nkv = a.num_kv_heads;
  const int n = b1 > first ? (b1 - first + STRIDE - 1) / STRIDE : 0;
  if (n == 0) return;
  v4u_t qf[4];
  KRegs k;
  VRegs v;

  // Pool tile of the x-th block of the wave's i-th pair: tile 0 of the head in place
  // of an entry outside the pool or past the piece (masked whole), so that the loads
  // need no branch. (The table is not read past the piece.)
  auto entry = [&](int i, int x, bool& ok) -> size_t {
    const int b = first + STRIDE * i + x;
    const int e = load_uniform(a.block_tables, (size_t)seq * a.max_blocks_per_seq + min(b, b1 - 1));
    ok = b < b1 && e >= 0 && e < a.num_blocks;
    return (size_t)(ok ? e : 0) * nkv + g;
  };

  bool ok[2];
  size_t tile[2];
#pragma unroll
  for (int x = 0; x < 2; ++x) tile[x] = entry(0, x, ok[x]);
  issue_k(pool, tile[0], tile[1], grp, col, k);
  load_q_row(a.q, head, grp, qf);
  issue_v(pool, tile[0], tile[1], grp, col, v);
#pragma clang loop unroll(disable)
  for (int i = 0; i < n; ++i) {
    const int b = first + STRIDE * i;
    bool next_ok[2];
#pragma unroll
    for (int x = 0; x < 2; ++x) tile[x] = entry(i + 1, x, next_ok[x]);
    float s[8];
    const PairScales ps = pair_scales(v.scales);
    pair_scores(k, qf, ps, a.scale_log2, s);
    issue_k(pool, tile[0], tile[1], grp, col, k);   // the K registers are free
    VRows rows = exchange(v, ps);
    issue_v(pool, tile[0], tile[1], grp, col, v);   // and V's
    if (!ok[0] || !ok[1] || (b + 2) * kBlockSize > plain) mask(b, ok, s, rows);
    run.fold<kTwoParts>(s, rows, head_lane);
    ok[0] = next_ok[0];
    ok[1] = next_ok[1];
  }
}

}  // namespace dq
}  // namespace bros
