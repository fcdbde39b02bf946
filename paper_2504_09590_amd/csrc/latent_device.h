// Absorbed attention over a latent pool (latent.hip): rows_device.h's units, steps, shares and
// masks, with a loop for rows of 576 dims that are key and value at once.
//
// A step is 32 keys, 36 KiB of LDS, read twice (scores, values). A wave has 32 columns and one of H
// parts of the dims: 576 / H of the score products, whose partial sums the H waves exchange in
// LDS, and 512 / H of the values. (All dims in one wave are 400 registers of queries and
// sums; the compiler then spills, and its waits for spilled values drain the loads in flight.)
//
// Two phases a step, each ended by a barrier: S, the score products and their exchange; P, the
// softmax and the value products. With two column groups one is a phase behind the other, so that
// each SIMD, which holds a wave of both, has one wave's matrix products beside the other's softmax.
// Rows are requested two steps ahead; each wave waits for those it requested itself, and puts in
// order what it finds there (rows that are no context, values that are not finite),
// before the barrier that publishes them.
#pragma once

#include "rows_device.h"

namespace bros {
namespace ra {

template <int NCW, int H>
struct LatentShape {
  using P = LatentPool;
  static constexpr int kWaves = NCW * H, kThreads = kWaves * kWave;
  static constexpr int kGroups = NCW > 1 ? 2 : 1, kGroupWaves = kWaves / kGroups, kGroupCols = NCW / kGroups;
  static constexpr int CT = 32 * NCW, KS = kKeys, SLOTS = 3;
  static constexpr int kDims = 512, kDt = 16;               // of all parts
  static constexpr int kRotAt = kKeys * P::kMain, kTile = kRotAt + kKeys * P::kRot;
  static constexpr int kRows = kKeys / kWaves;              // rows of a step that a wave requests
  static constexpr int kLoads = kRows + (kRows + 7) / 8;
  static constexpr int kSlotFloats = CT * kDims;
  static_assert(kRows == 4 || kRows == 8, "a wave's rows lie in one block");
};

template <int NCW, int H, int OCC>
__global__ __launch_bounds__(64 * NCW * H, OCC) void latent_kernel(RowsArgs a) {
  using P = LatentPool;
  using S = LatentShape<NCW, H>;
  constexpr int kDt = S::kDt / H;                            // of this wave: 32-dim pieces of values,
  constexpr int kMainSteps = 32 / H, kRotSteps = 4 / H;      // 16-dim steps of score products
  constexpr int kRow = P::kMain + P::kRot;
  __shared__ __attribute__((aligned(1024))) uint8_t s_ring[S::SLOTS * S::kTile];
  __shared__ __attribute__((aligned(16))) float s_x[S::kWaves * 1024];
  __shared__ int32_t s_tab[S::kWaves][kTable];
  __shared__ uint32_t s_bad[S::SLOTS][S::kWaves];            // of each row that a wave requested: something is not finite
  __shared__ int64_t s_scan[2 * S::kWaves];
  __shared__ Place s_place;

  const int lane = threadIdx.x & (kWave - 1), wave = wave_id_uniform();
  const int group = wave / S::kGroupWaves, cw = group * S::kGroupCols + wave % S::kGroupCols;
  const int hp = wave % S::kGroupWaves / S::kGroupCols;
  const bool late = S::kGroups > 1 && group == 1;
  const int half = lane >> 5, col = lane & 31;
  const int G = a.num_q_heads;
  const int nb = gridDim.x;   // neighbouring shares to one die
  const int me = nb % pf::kXcds == 0 ? (blockIdx.x % pf::kXcds) * (nb / pf::kXcds) + blockIdx.x / pf::kXcds : blockIdx.x;

  Place at = find_place<P, S::CT, S::KS, S::kThreads>(
      a, G, [&](int64_t total) -> int64_t {
        const int n = sharers(a, total);
        return me < n ? share_begin(total, me, n) : -1;
      }, s_scan, &s_place);
  if (at.s < 0) return;   // (uniform: no step left for this workgroup)
  const int nshare = sharers(a, at.total);
  int64_t x = share_begin(at.total, me, nshare);
  const int64_t x_end = share_begin(at.total, me + 1, nshare);

  int32_t* tab = s_tab[wave];
  const float sl2 = a.scale_log2;
  const bf16x2_t one2 = {(__bf16)1.0f, (__bf16)1.0f};
  // Operand reads: lane addresses of a tile at 0. A chunk's low four bits are those of the
  // row's permutation, so that other chunks are a xor and a constant away.
  const uint32_t k_lane = col * P::kMain + hp * (P::kMain / H) + ((half ^ swz(col)) << 4);
  const uint32_t r_lane = S::kRotAt + (col >> 1) * 256 + ((col & 1) << 7) + (((half + 2 * kRotSteps * hp) ^ ((col >> 1) & 7)) << 4);
  const int v_key = 4 * half + ((lane >> 2) & 3);
  const uint32_t v_lane = v_key * P::kMain + hp * (kDt * 64) + (((2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ swz(v_key)) << 4) + (lane & 1) * 8;
  const uint32_t ring0 = lds_address(s_ring);

  while (x < x_end) {
    // ---- The segment: steps [first, last) of unit (s, t).
    const int s = at.s, t = at.t;
    const Seq q = seq_of(a, s);
    const Steps<P, S::CT, S::KS> st(a, q, G);
    const int usteps = __builtin_amdgcn_readfirstlane(st.of(t));
    const int first = at.step;
    const int cnt = (int)min((int64_t)(usteps - first), x_end - x);
    const int last = first + cnt;
    const bool whole = cnt == usteps;
    const int ctx = q.ctx, n = q.n;
    const int nblk = (ctx + kBlockSize - 1) / kBlockSize;
    const int c = t * S::CT + 32 * cw + col;        // the lane's column
    const int j = c / G;                            // its row
    const bool valid = j < n;
    const size_t orow = (size_t)(q.q0 + min(j, n - 1)) * G + (c - j * G);
    // keys below this position are seen by every row of the unit
    const int full_below = a.mask != nullptr ? min(ctx, q.c0) : min(ctx, q.c0 + t * S::CT / G + 1);
    const int32_t* tbl = a.block_tables + (size_t)s * a.max_blocks_per_seq;

    bf16x8_t qf[kMainSteps + kRotSteps];
    {
      // (columns behind the last row take that row's values: nothing is made of them)
      const uint16_t* qp = static_cast<const uint16_t*>(a.q) + orow * (kRow / 2) + 8 * half;
#pragma unroll
      for (int i = 0; i < kMainSteps; ++i) qf[i] = as_bf16x8(*reinterpret_cast<const v4u_t*>(qp + 16 * (hp * kMainSteps + i)));
#pragma unroll
      for (int i = 0; i < kRotSteps; ++i)
        qf[kMainSteps + i] = as_bf16x8(*reinterpret_cast<const v4u_t*>(qp + P::kMain / 2 + 16 * (hp * kRotSteps + i)));
    }

    auto load_window = [&](int e0) __attribute__((always_inline)) {   // table entries e0 .. + 63
      load_word_to_lds(tbl, 4u * (uint32_t)max(0, min(e0 + lane, nblk - 1)), tab + (e0 & (kTable - 1)));
    };
    auto entry = [&](int e) __attribute__((always_inline)) -> int {   // -1: none
      const int v = __builtin_amdgcn_readfirstlane(lds_word(tab + (e & (kTable - 1))));
      return (e < nblk && v >= 0 && v < a.num_blocks) ? v : -1;
    };
    uint32_t holes = 0;   // bit step % 32: a block of that step is missing
    // Requests the wave's rows of a step.
    auto request = [&](int step) __attribute__((always_inline)) {
      const int e = 2 * step;
      if ((e & 63) == 0 && step > first) load_window(e + 64);
      const int b0 = entry(e), b1 = entry(e + 1);
      const int row0 = S::kRows * wave, b = row0 >= kBlockSize ? b1 : b0;
      const uint8_t* src = static_cast<const uint8_t*>(a.k_pool) + ((size_t)max(b, 0) * kBlockSize + (row0 & 15)) * kRow;
      uint8_t* dst = s_ring + (step % S::SLOTS) * S::kTile;
#pragma unroll
      for (int i = 0; i < S::kRows; ++i)
        load_to_lds(src + i * kRow, (uint32_t)((lane ^ swz(row0 + i)) << 4), dst + (row0 + i) * P::kMain);
      const int r = row0 + (lane >> 3);
      if (S::kRows == 8 || lane < 8 * S::kRows)
        load_to_lds(src + P::kMain, (uint32_t)((lane >> 3) * kRow + (((lane & 7) ^ ((r >> 1) & 7)) << 4)), dst + S::kRotAt + row0 * P::kRot);
      holes = (holes & ~(1u << (step & 31))) | ((b0 < 0 || b1 < 0 ? 1u : 0u) << (step & 31));
    };
    auto masked = [&](int step) -> bool { return ((holes >> (step & 31)) & 1) || (step + 1) * kKeys > full_below; };
    auto blocks_of = [&](int step) -> TileBlocks {
      const int e = 2 * step, em = max(nblk - 1, 0);
      const int v0 = tbl[min(e, em)], v1 = tbl[min(e + 1, em)];
      return TileBlocks{e < nblk && v0 >= 0 && v0 < a.num_blocks, e + 1 < nblk && v1 >= 0 && v1 < a.num_blocks,
                        entry_direction(a.dir, a.cls, a.dir_per_entry, a.max_blocks_per_seq, s, min(e, em)),
                        entry_direction(a.dir, a.cls, a.dir_per_entry, a.max_blocks_per_seq, s, min(e + 1, em))};
    };
    // Waits for the wave's rows of a step (requests of `later` steps may be in flight) and, where the step
    // is masked, puts them in order: zeros for rows that are no context and for values that are not
    // finite, which it notes (a row that sees such a key becomes NaN). Then the barrier.
    auto publish = [&](int step, bool later) __attribute__((always_inline)) {
      if (step < last) {
        if (later) wait_vmem<S::kLoads>();
        else wait_vmem<0>();
        if (masked(step)) {
          const TileBlocks tb = blocks_of(step);
          uint8_t* tile = s_ring + (step % S::SLOTS) * S::kTile;
          uint32_t noted = 0;
#pragma unroll 1
          for (int i = 0; i < S::kRows; ++i) {
            const int r = S::kRows * wave + i;
            const int pos = step * kKeys + (r & 16) + slot_of_offset(r & 15, r < 16 ? tb.dir0 : tb.dir1);
            const bool there = (r < 16 ? tb.ok0 : tb.ok1) && pos < ctx;
            v4u_t* v = reinterpret_cast<v4u_t*>(tile + r * P::kMain) + lane;
            v4u_t w = there ? *v : v4u_t{0, 0, 0, 0};
            uint32_t any = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const uint32_t bad = not_finite(w[e]);
              any |= bad;
              w[e] &= ~((bad >> 15) * 0xffffu);
            }
            *v = w;
            noted |= (__builtin_amdgcn_ballot_w64(any != 0) != 0 ? 1u : 0u) << i;
          }
          if (lane == 0) s_bad[step % S::SLOTS][wave] = noted;
        }
      }
      lds_barrier();
    };

    floatx16 o[kDt];
#pragma unroll
    for (int i = 0; i < kDt; ++i) o[i] = floatx16{};
    float m_run = kNoMax, l0 = 0.0f, l1 = 0.0f;

    // ---- Start: the first windows of the table, the first two steps' rows.
    __syncthreads();   // (the ring's last use: the segment before this one)
    load_window((2 * first) & ~63);
    load_window(((2 * first) & ~63) + 64);
    __builtin_amdgcn_s_waitcnt(0x0F70);   // vmcnt(0): a wait the compiler sees, q's included
    asm volatile("" ::: "memory");
    request(first);
    if (first + 1 < last) request(first + 1);
    publish(first, first + 1 < last);
    if (late) lds_barrier();

    int slot = first % S::SLOTS;
#pragma unroll 1
    for (int step = first; step < last; ++step) {
      const uint32_t tile = ring0 + slot * S::kTile;
      // ---- S: the wave's part of the scores, to its partners.
      if (late && step + 2 < last) request(step + 2);
      floatx16 cur;
      {
        const uint32_t k = tile + k_lane, r = tile + r_lane;
#pragma unroll
        for (int i = 0; i < kMainSteps; ++i)
          cur = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(lds_read((k ^ ((i & 7) << 5)) + (i >> 3) * 256)), qf[i],
                                                        i == 0 ? floatx16{} : cur, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < kRotSteps; ++i)
          cur = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(lds_read(r ^ (i << 5))), qf[kMainSteps + i], cur, 0, 0, 0);
      }
      {
        float4* mine = reinterpret_cast<float4*>(s_x) + wave * 4 * kWave + lane;
#pragma unroll
        for (int i = 0; i < 4; ++i) mine[i * kWave] = make_float4(cur[4 * i], cur[4 * i + 1], cur[4 * i + 2], cur[4 * i + 3]);
      }
      if (late) publish(step + 1, step + 2 < last);
      else lds_barrier();

      // ---- P: the scores' sums ((0 + 1) + (2 + 3), whichever part adds: the waves of a
      // column must hold the same), softmax, values.
      if (!late && step + 2 < last) request(step + 2);
      {
        const auto part = [&](int k, int i) {
          return (reinterpret_cast<const float4*>(s_x) + (group * S::kGroupWaves + (hp ^ k) * S::kGroupCols + wave % S::kGroupCols) * 4 * kWave + lane)[i * kWave];
        };
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float4 y = part(1, i);
          float4 z = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
          if constexpr (H == 4) {
            const float4 u = part(2, i), v = part(3, i);
            z = make_float4(u.x + v.x, u.y + v.y, u.z + v.z, u.w + v.w);
          }
          cur[4 * i] = (cur[4 * i] + y.x) + z.x;
          cur[4 * i + 1] = (cur[4 * i + 1] + y.y) + z.y;
          cur[4 * i + 2] = (cur[4 * i + 2] + y.z) + z.z;
          cur[4 * i + 3] = (cur[4 * i + 3] + y.w) + z.w;
        }
      }
      if (masked(step)) {
        const TileBlocks tb = blocks_of(step);
        const uint32_t win = row_window(a, q, ctx, j, valid, step * kKeys);
        uint32_t bad = 0;
#pragma unroll
        for (int w = 0; w < S::kWaves; ++w) bad |= s_bad[slot][w] << (S::kRows * w);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int k = 8 * (i >> 2) + 4 * half + (i & 3);
          const int off = (k & 16) + slot_of_offset(k & 15, (i >> 3) ? tb.dir1 : tb.dir0);
          const bool sees = ((i >> 3) ? tb.ok1 : tb.ok0) && ((win >> off) & 1u);
          cur[i] = !sees ? -INFINITY : (bad >> k) & 1u ? __uint_as_float(0x7fc00000u) : cur[i];
        }
      }
      // running maximum (moved lazily) and weights, rounded to bf16 for the second product; the totals
      // add the rounded weights
      float mr = -INFINITY;
#pragma unroll
      for (int i = 0; i < 16; ++i) mr = fmaxf(mr, cur[i]);
      const float mx = pair_max(mr) * sl2;
      const float m_new = mx > m_run + kRescaleSlack ? mx : m_run;
      if (__builtin_amdgcn_ballot_w64(m_new != m_run) != 0) {
        const float alpha = fast_exp2(m_run - m_new);
#pragma unroll
        for (int i = 0; i < kDt; ++i) o[i] *= alpha;
        l0 *= alpha;
        l1 *= alpha;
        m_run = m_new;
      }
      bf16x8_t pfr[2];
#pragma unroll
      for (int c2 = 0; c2 < 2; ++c2) {
        bf16x2_t pw[4];
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const float2_t pp = {fast_exp2(fmaf(cur[8 * c2 + 2 * w], sl2, -m_run)),
                               fast_exp2(fmaf(cur[8 * c2 + 2 * w + 1], sl2, -m_run))};
          pw[w] = __builtin_convertvector(pp, bf16x2_t);
          if (w & 1) l1 = __builtin_amdgcn_fdot2_f32_bf16(pw[w], one2, l1, false);
          else l0 = __builtin_amdgcn_fdot2_f32_bf16(pw[w], one2, l0, false);
        }
        const v4u_t pk = {__builtin_bit_cast(uint32_t, pw[0]), __builtin_bit_cast(uint32_t, pw[1]),
                          __builtin_bit_cast(uint32_t, pw[2]), __builtin_bit_cast(uint32_t, pw[3])};
        pfr[c2] = as_bf16x8(pk);
      }
      {
        const uint32_t v = tile + v_lane;
#pragma unroll
        for (int c2 = 0; c2 < 2; ++c2) {
#pragma unroll
          for (int dt = 0; dt < kDt; ++dt) {
            // (keys 8 on: another bit of the row's permutation)
            const uint32_t at_v = (v ^ ((dt & 3) << 6)) + (dt >> 2) * 256 + 16 * c2 * P::kMain;
            const uint2 x0 = lds_read_turned(at_v), x1 = lds_read_turned((at_v ^ 16) + 8 * P::kMain);
            o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(v4u_t{x0.x, x0.y, x1.x, x1.y}), pfr[c2], o[dt], 0, 0, 0);
          }
        }
      }
      if (!late) publish(step + 1, step + 2 < last);
      else lds_barrier();
      slot = slot + 1 == S::SLOTS ? 0 : slot + 1;
    }
    if (S::kGroups > 1 && !late) lds_barrier();

    // ---- The end of the segment.
    const float l = pair_sum(l0 + l1);
    if (whole) {
      const float inv = l > 0.0f ? 1.0f / l : l == 0.0f ? 0.0f : l;   // (NaN stays)
      if (valid) write_columns<kDt>(static_cast<uint16_t*>(a.out) + orow * S::kDims, hp * kDt, o, inv, half);
    } else {
      // the accumulators as they lie: every store of the wave is 1 KiB contiguous
      const size_t ws = 2 * (size_t)me + (first == 0 ? 1 : 0);
      float4* po = reinterpret_cast<float4*>(a.ws_o + ws * S::kSlotFloats) + (cw * S::kDt + hp * kDt) * 4 * kWave + lane;
#pragma unroll
      for (int i = 0; i < kDt; ++i) {
#pragma unroll
        for (int jq = 0; jq < 4; ++jq)
          po[(4 * i + jq) * kWave] = make_float4(o[i][4 * jq], o[i][4 * jq + 1], o[i][4 * jq + 2], o[i][4 * jq + 3]);
      }
      if (half == 0 && hp == 0) {
        float* ml = a.ws_ml + (ws * S::CT + 32 * cw + col) * 2;
        ml[0] = m_run;
        ml[1] = l;
      }
    }

    // ---- The next unit.
    x += cnt;
    at.step = 0;
    if (x < x_end && ++at.t >= st.tiles) {
      at.t = 0;
      do ++at.s;
      while (seq_of(a, at.s).n <= 0);   // (steps are left, so a sequence with rows follows)
    }
  }
}

}  // namespace ra
}  // namespace bros
