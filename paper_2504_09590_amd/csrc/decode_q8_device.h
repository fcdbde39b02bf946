// Device code of the decode over an 8-bit cache (decode_q8.hip): one step of a wave
// over a pair of 16-slot blocks of one (row, KV head) segment.
//
// As in the 16-bit decode, the G query heads of a KV head form a dense product per
// block, and the softmax weights never move between lanes. Lane l = 16 grp + col:
//   S^T[slot][head] = K[slot][:] . q[head][:]         mfma 16x16x32, four a block
//   O^T[dim][head] += V^T[dim][slot] P^T[slot][head]  mfma 16x16x32, eight a pair
// In the C layout of the first product lane l holds the scores of slots 4 grp ..
// 4 grp + 3 of head col; the 32 slots of a pair are ordered so that the four of the
// first block and the four of the second are the eight the second product wants in
// that lane. K: the lane reads row col, dims 16 grp .. + 15 and 64 + 16 grp .. + 15 (the
// contraction's order of dims is free, q uses the same). V: rows 4 grp + j, dims
// 8 col .. + 7, and output row m of product t is dim 8 m + t, so lane l ends up with
// dims 32 grp .. 32 grp + 31 of head col.
//
// Codes become bf16 values in registers, two per instruction, which multiplies by
// the row's scale on the way: exact, so what follows is the 16-bit decode of the
// values the cache stands for. A pair costs a wave 64 such conversions and 32 byte
// permutations for 8 KiB of codes; at the rate HBM delivers them a SIMD has about
// 2900 cycles for a pair, and all of a step's instructions take about a third of that.
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

// The registers of one block of a step.
struct KRegs {
  v4u_t lo, hi;    // row col: dims 16 grp .., 64 + 16 grp ..
  uint32_t scale;  // the row's scale byte
};
struct VRegs {
  v2u_t row[4];    // rows 4 grp + j: dims 8 col ..
  uint32_t scale;  // their scale bytes
};

__device__ __forceinline__ v4u_t load16(const uint8_t* p) { return __builtin_nontemporal_load(reinterpret_cast<const v4u_t*>(p)); }
__device__ __forceinline__ v2u_t load8(const uint8_t* p) { return __builtin_nontemporal_load(reinterpret_cast<const v2u_t*>(p)); }

__device__ __forceinline__ void issue_k(const Q8Pool& p, size_t tile, int grp, int col, KRegs& k) {
  const uint8_t* b = p.k + tile * kTileBytes + (uint32_t)(col * kHeadDim + 16 * grp);
  k.lo = load16(b);
  k.hi = load16(b + 64);
  k.scale = p.scales[tile * kScaleBytes + (uint32_t)col];
}
__device__ __forceinline__ void issue_v(const Q8Pool& p, size_t tile, int grp, int col, VRegs& v) {
  const uint8_t* b = p.v + tile * kTileBytes + (uint32_t)(4 * grp * kHeadDim + 8 * col);
#pragma unroll
  for (int j = 0; j < 4; ++j) v.row[j] = load8(b + j * kHeadDim);
  v.scale = *reinterpret_cast<const uint32_t*>(p.scales + tile * kScaleBytes + (uint32_t)(kBlockSize + 4 * grp));
}

// The query of a segment, in the order of K's dims (padding columns repeat a head).
template <int G>
__device__ __forceinline__ void load_q(const void* q, size_t first_head, int grp, int col, v4u_t (&qf)[4]) {
  const uint16_t* p = static_cast<const uint16_t*>(q) + (first_head + min(col, G - 1)) * kHeadDim + 16 * grp;
#pragma unroll
  for (int c = 0; c < 4; ++c) qf[c] = *reinterpret_cast<const v4u_t*>(p + 64 * (c >> 1) + 8 * (c & 1));
}

// Raw scores of a block: slots 4 grp + r of head col.
__device__ __forceinline__ floatx4_t block_scores(const KRegs& k, const v4u_t (&qf)[4]) {
  const float s = q8::scale_of(k.scale);
  floatx4_t sc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    const v4u_t& w = c < 2 ? k.lo : k.hi;
    const uint32_t w0 = w[2 * (c & 1)], w1 = w[2 * (c & 1) + 1];
    const v4u_t kv = {q8::values2_bf16<false>(w0, s), q8::values2_bf16<true>(w0, s), q8::values2_bf16<false>(w1, s),
                      q8::values2_bf16<true>(w1, s)};
    sc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, kv), __builtin_bit_cast(bf16x8_t, qf[c]), sc, 0, 0, 0);
  }
  return sc;
}

// A wave's running result over its part of a segment, per head col.
struct Running {
  floatx4_t acc[8];   // acc[t][r]: dim 32 grp + 8 r + t
  float m_ref, l_part;

  __device__ __forceinline__ void clear() {
    m_ref = kNoMax;
    l_part = 0.0f;
#pragma unroll
    for (int t = 0; t < 8; ++t) acc[t] = floatx4_t{0.0f, 0.0f, 0.0f, 0.0f};
  }

  // Folds a pair in: s its eight scores in log2 units (slots 4 grp + r of the first
  // block, then of the second; -inf where masked), v its V rows.
  __device__ __forceinline__ void fold(const float (&s)[8], const VRegs (&v)[2], bool head_lane) {
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
    l_part += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
    // The weights as a bf16 and the bf16 of what it leaves: 8 bits more for eight
    // products a pair, which the matrix cores have time for.
    const v4u_t hi4 = {q8::pack2_bf16(p[0], p[1]), q8::pack2_bf16(p[2], p[3]), q8::pack2_bf16(p[4], p[5]), q8::pack2_bf16(p[6], p[7])};
    v4u_t lo4;
#pragma unroll
    for (int i = 0; i < 4; ++i) lo4[i] = q8::pack2_bf16(p[2 * i] - bf16_lo(hi4[i]), p[2 * i + 1] - bf16_hi(hi4[i]));
    const bf16x8_t ph = __builtin_bit_cast(bf16x8_t, hi4), pl = __builtin_bit_cast(bf16x8_t, lo4);
    float sc[2][4];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
#pragma unroll
      for (int j = 0; j < 4; ++j) sc[x][j] = q8::scale_of((v[x].scale >> (8 * j)) & 0xffu);
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {   // dims 2 u and 2 u + 1 of the lane's eight
      uint32_t w[2][4];
#pragma unroll
      for (int x = 0; x < 2; ++x) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          w[x][j] = (u & 1) ? q8::values2_bf16<true>(v[x].row[j][u >> 1], sc[x][j]) : q8::values2_bf16<false>(v[x].row[j][u >> 1], sc[x][j]);
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t sel = h ? 0x07060302u : 0x05040100u;
        const v4u_t vt = {__builtin_amdgcn_perm(w[0][1], w[0][0], sel), __builtin_amdgcn_perm(w[0][3], w[0][2], sel),
                          __builtin_amdgcn_perm(w[1][1], w[1][0], sel), __builtin_amdgcn_perm(w[1][3], w[1][2], sel)};
        const bf16x8_t va = __builtin_bit_cast(bf16x8_t, vt);
        const int t = 2 * u + h;
        acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, ph, acc[t], 0, 0, 0);
        acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, pl, acc[t], 0, 0, 0);
      }
    }
  }

  // The weights' total of head col, in every lane of the head.
  __device__ __forceinline__ float total() const {
    float l = l_part;
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    return l;
  }
};

// Removes what a pair's blocks do not hold of the context: block b0 + x is `ok`, or
// an entry outside the pool (or a block past the context); slots from ctx on belong
// to nobody or to a peer. By selection, so that no value there leaks.
__device__ __forceinline__ void mask_pair(const DecodeArgs& a, int row, int ctx, int b0, const bool (&ok)[2], int grp,
                                          float (&s)[8], VRegs (&v)[2]) {
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    const int b = b0 + x;
    if (ok[x] && (b + 1) * kBlockSize <= ctx) continue;
    const int dir = ok[x] ? entry_direction(a.dir, a.cls, a.dir_per_entry, a.max_blocks_per_seq, row, b) : 1;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      if (!ok[x] || b * kBlockSize + slot_of_offset(4 * grp + r, dir) >= ctx) {
        s[4 * x + r] = -INFINITY;
        v[x].row[r] = v2u_t{0u, 0u};
        v[x].scale &= ~(0xffu << (8 * r));   // (0 times 2^-127)
      }
    }
  }
}

}  // namespace dq
}  // namespace bros
