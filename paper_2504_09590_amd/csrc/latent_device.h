// Absorbed attention over a latent pool (latent.hip): rows_device.h's units, steps, shares and
// masks, with a loop for rows of 576 dims that are key and value at once.
//
// A step is 32 keys, 36 KiB of LDS, read twice (scores, values). A wave has 16 columns, with 16x16x32
// matrix instructions: its queries (72 registers) and its sums in fp32 (128) fit the 256 of a
// wave, two to a SIMD, and no wave needs another's scores. Up to 128 columns are eight such waves; with
// fewer columns HV waves share a column group, each computing all its scores and a part of
// the value dims. The price is LDS: every operand of 1 KiB serves 16 columns, 544 KiB a step and
// compute unit with 128 columns, twice what the products take; and the rows' permutation (swz, made for 32-row operands)
// leaves the reads of the keys' 512 dims two-way bank conflicts: the lanes that are served together are of two quarters, and rows 4 to 7 of
// one meet rows 12 to 15 of the other. They are 32 % of the LDS's active cycles with 128 columns, 37 with 32 and 41 with 16
// (SQ_LDS_BANK_CONFLICT; the values' reads and the rotated dims' have none). Tried instead, and slower over 96 contexts up to 16384
// with 128 heads (302 us then, 293 with shares that count starts): 32 columns to a wave and the dims in two halves whose score sums waves exchange, 336 KiB but two
// barriers a step, 370; four waves of 32 columns and 512 registers, one block of the step's keys each, that exchange
// weights, 136 KiB for 64 columns, 387, and two such workgroups on the same keys 350: LDS no longer binds, but nothing runs
// beside one wave's softmax and barrier.
//
// Rows are requested three steps ahead; each wave waits for those it requested itself, and puts in
// order what it finds there (rows that are no context, values that are not finite),
// before the barrier that publishes them, the only one of a step.
//
// Measured, kernel and merge: 16 heads, 64 contexts up to 8192, 65 + 5 us, 289 MB, bound by memory; 128 heads, 96 contexts up to 16384,
// 315 + 19 us (410 + 22 in the middle of the first twelve calls), 790 TFLOP/s, bound by LDS; five sequences of five to eight drafts, 32 heads, on up to 4000, 32 + 6 us.
#pragma once

#include "rows_device.h"

namespace bros {
namespace ra {

typedef __attribute__((__vector_size__(4 * sizeof(float)))) float floatx4;

// Maximum and sum over the lanes of a column (l, l ^ 16, l ^ 32, l ^ 48).
__device__ __forceinline__ float column_max(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return pair_max(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
__device__ __forceinline__ float column_sum(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return pair_sum(__uint_as_float(r[0]) + __uint_as_float(r[1]));
}

// NCW column groups of 16, HV waves to each.
template <int NCW, int HV>
struct LatentShape {
  using P = LatentPool;
  static constexpr int kWaves = NCW * HV, kThreads = kWaves * kWave;
  static constexpr int CT = 16 * NCW, KS = kKeys, SLOTS = 4;
  static constexpr int kLaneCols = 16;                      // columns of a wave
  static constexpr int kDims = 512, kDt = 32;               // 16-dim pieces of a value
  static constexpr int kRotAt = kKeys * P::kMain, kTile = kRotAt + kKeys * P::kRot;
  static constexpr int kRows = kKeys / kWaves;              // rows of a step that a wave requests
  static constexpr int kLoads = kRows + (kRows + 7) / 8;
  static constexpr int kSlotFloats = CT * kDims;
  static constexpr int kChunks = kDt;                       // of a wave's partial, 1 KiB each
  // first of the four dims that a lane has in chunk i
  static __device__ __forceinline__ int dim_of(int i, int lane) { return 16 * i + 4 * (lane >> 4); }
  static_assert(kRows == 4 || kRows == 8, "a wave's rows lie in one block");
};

// Writes a wave's normalised columns: lane l holds column l % 16, and of o[i] the dims 16 (dt0 + i) + 4 (l / 16) .. + 3.
template <int N>
__device__ __forceinline__ void write_columns16(uint16_t* row, int dt0, const floatx4 (&o)[N], float inv, int quarter) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    uint2 w;
    w.x = pack2_bf16(o[i][0] * inv, o[i][1] * inv);
    w.y = pack2_bf16(o[i][2] * inv, o[i][3] * inv);
    *reinterpret_cast<uint2*>(row + 16 * (dt0 + i) + 4 * quarter) = w;
  }
}

template <int NCW, int HV, int OCC>
__global__ __launch_bounds__(64 * NCW * HV, OCC) void latent_kernel(RowsArgs a) {
  using P = LatentPool;
  using S = LatentShape<NCW, HV>;
  constexpr int kDt = S::kDt / HV;                           // of this wave: 16-dim pieces of values
  constexpr int kQSteps = 18, kMainSteps = 16;               // 32-dim steps of score products
  constexpr int kAhead = HV == 1 ? 4 : 8;                    // operands read before the first product (as registers allow)
  constexpr int kRow = P::kMain + P::kRot;
  __shared__ __attribute__((aligned(1024))) uint8_t s_ring[S::SLOTS * S::kTile];
  __shared__ int32_t s_tab[S::kWaves][kTable];
  __shared__ uint64_t s_word[S::kWaves][16];                 // the first mask word of each of a wave's columns
  __shared__ uint32_t s_bad[S::SLOTS][S::kWaves];            // of each row that a wave requested: something is not finite
  __shared__ int64_t s_scan[2 * S::kWaves];
  __shared__ Place s_place;

  const int lane = threadIdx.x & (kWave - 1), wave = wave_id_uniform();
  const int cw = wave % NCW, hv = wave / NCW;
  const int quarter = lane >> 4, col = lane & 15;
  const int G = a.num_q_heads;
  const int nb = gridDim.x;   // neighbouring shares to one die
  const int me = nb % pf::kXcds == 0 ? (blockIdx.x % pf::kXcds) * (nb / pf::kXcds) + blockIdx.x / pf::kXcds : blockIdx.x;

  Cut* cut = reinterpret_cast<Cut*>(a.ws_cut) + me;
  if (threadIdx.x == 0) cut->last = -1;

  Place at = find_place<P, S::CT, S::KS, S::kThreads>(
      a, G, [&](int64_t total) -> int64_t {
        const Shares sh(a, total);
        return me < sh.n ? sh.begin(me) : -1;
      }, s_scan, &s_place);
  if (at.s < 0) return;   // (uniform: no step left for this workgroup)
  const Shares shares(a, at.total);
  int64_t x = shares.begin(me);
  const int64_t x_end = shares.begin(me + 1);

  const float sl2 = a.scale_log2;
  const bf16x2_t one2 = {(__bf16)1.0f, (__bf16)1.0f};
  // Operand reads: lane addresses of a tile at 0. A chunk's low four bits are those of the
  // row's permutation, so that other chunks are a xor and a constant away.
  const uint32_t k_lane = col * P::kMain + ((quarter ^ swz(col)) << 4);
  const uint32_t r_lane = S::kRotAt + (col >> 1) * 256 + ((col & 1) << 7) + ((quarter ^ ((col >> 1) & 7)) << 4);
  const int v_key = 4 * quarter + ((lane >> 2) & 3);
  const uint32_t v_lane = v_key * P::kMain + hv * (kDt * 32) + ((((lane & 3) >> 1) ^ swz(v_key)) << 4) + (lane & 1) * 8;
  const uint32_t ring0 = lds_address(s_ring);

  while (x < x_end) {
    // ---- The segment: steps [first, last) of unit (s, t).
    const Segment<P, S::CT, S::KS, 1> seg(a, at, G, 0, x, x_end);
    const int s = at.s, t = seg.t, first = seg.first, last = seg.last;
    const Seq q = seg.q;
    const bool whole = seg.whole;
    x = seg.next;
    if (seg.count > 0) {   // (a share may end within a unit's start)
    const int ctx = q.ctx, n = q.n;
    // The lane's column: its row, whether there is one, and the place of both in q and out. (Formed anew at
    // each use: the loop needs the registers.)
    struct Column {
      int j;
      bool valid;
      size_t orow;
    };
    auto column = [&]() __attribute__((always_inline)) -> Column {
      const int c = t * S::CT + 16 * cw + (lane_here() & 15), j = c / G;
      return Column{j, j < n, (size_t)(q.q0 + min(j, n - 1)) * G + (c - j * G)};
    };
    // keys below this position are seen by every row of the unit
    const int full_below = a.mask != nullptr ? min(ctx, q.c0) : min(ctx, q.c0 + t * S::CT / G + 1);
    const Table table{a.block_tables + (size_t)s * a.max_blocks_per_seq, s_tab[wave], (ctx + kBlockSize - 1) / kBlockSize, a.num_blocks};

    // ---- Start: the first windows of the table, then queries and masks.
    __syncthreads();   // (the ring's last use: the segment before this one)
    const int e_first = (2 * first) & ~63;
    const int32_t win0 = table.get(e_first), win1 = table.get(e_first + 64);
    const int dir_all = seq_direction(a.dir, a.cls, s);   // (read where entries have no directions of their own)
    bf16x8_t qf[kQSteps];
    {
      // (columns behind the last row take that row's values: nothing is made of them)
      const Column my = column();
      if (a.mask != nullptr && quarter == 0) s_word[wave][col] = first_word(a, q, my.j);
      const uint16_t* qp = static_cast<const uint16_t*>(a.q) + my.orow * (kRow / 2) + 8 * quarter;
#pragma unroll
      for (int i = 0; i < kQSteps; ++i) qf[i] = as_bf16x8(*reinterpret_cast<const v4u_t*>(qp + 32 * i));
    }

    uint32_t holes = 0;               // bit step % 32: a block of that step is missing
    int32_t word_a = 0, word_b = 0;   // the next request's entries
    auto ask = [&](int step) __attribute__((always_inline)) {
      word_a = table.word(2 * step);
      word_b = table.word(2 * step + 1);
    };
    // Requests the wave's rows of a step.
    auto request = [&](int step) __attribute__((always_inline)) {
      const int e = 2 * step;
      const int b0 = table.entry(e, word_a), b1 = table.entry(e + 1, word_b);
      if ((e & 63) == 2 * Table::kLag) table.load((e & ~63) + 64);
      ask(step + 1);
      const int row0 = S::kRows * wave, b = row0 >= kBlockSize ? b1 : b0;
      const uint8_t* src = static_cast<const uint8_t*>(a.k_pool) + ((size_t)max(b, 0) * kBlockSize + (row0 & 15)) * kRow;
      uint8_t* dst = s_ring + (step % S::SLOTS) * S::kTile;
      const int ln = lane_here();
#pragma unroll
      for (int i = 0; i < S::kRows; ++i)
        load_to_lds(src + i * kRow, (uint32_t)((ln ^ swz(row0 + i)) << 4), dst + (row0 + i) * P::kMain);
      const int r = row0 + (ln >> 3);
      if (S::kRows == 8 || ln < 8 * S::kRows)
        load_to_lds(src + P::kMain, (uint32_t)((ln >> 3) * kRow + (((ln & 7) ^ ((r >> 1) & 7)) << 4)), dst + S::kRotAt + row0 * P::kRot);
      holes = (holes & ~(1u << (step & 31))) | ((b0 < 0 || b1 < 0 ? 1u : 0u) << (step & 31));
    };
    auto masked = [&](int step) -> bool { return ((holes >> (step & 31)) & 1) || (step + 1) * kKeys > full_below; };
    auto blocks_of = [&](int step) __attribute__((always_inline)) -> TileBlocks {   // (of a step whose entries are still in LDS)
      const int e = 2 * step;
      TileBlocks tb;
      tb.ok0 = table.entry(e, table.word(e)) >= 0;
      tb.ok1 = table.entry(e + 1, table.word(e + 1)) >= 0;
      directions(a, s, e, dir_all, tb);
      return tb;
    };
    // Waits for the wave's rows of a step (those of the next SLOTS - 2 may be in flight) and, where the step
    // is masked, puts them in order: zeros for rows that are no context and for values that are not
    // finite, which it notes (a row that sees such a key becomes NaN). Then the barrier.
    auto publish = [&](int step) __attribute__((always_inline)) {
      if (step < last) {
        const int later = min(S::SLOTS - 2, last - 1 - step);
        if (later == 2) wait_vmem<2 * S::kLoads>();
        else if (later == 1) wait_vmem<S::kLoads>();
        else wait_vmem<0>();
        if (masked(step)) {
          const TileBlocks tb = blocks_of(step);
          uint8_t* tile = s_ring + (step % S::SLOTS) * S::kTile;
          uint32_t noted = 0;
          v4u_t w[S::kRows];
#pragma unroll
          for (int i = 0; i < S::kRows; ++i) w[i] = reinterpret_cast<const v4u_t*>(tile + (S::kRows * wave + i) * P::kMain)[lane];
#pragma unroll
          for (int i = 0; i < S::kRows; ++i) {
            const int r = S::kRows * wave + i;
            const int pos = step * kKeys + (r & 16) + slot_of_offset(r & 15, r < 16 ? tb.dir0 : tb.dir1);
            const bool there = (r < 16 ? tb.ok0 : tb.ok1) && pos < ctx;   // (uniform)
            uint32_t any = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const uint32_t bad = not_finite(w[i][e]);
              any |= bad;
              w[i][e] = there ? w[i][e] & ~((bad >> 15) * 0xffffu) : 0;
            }
            const bool odd = there && __builtin_amdgcn_ballot_w64(any != 0) != 0;
            if (!there || odd) reinterpret_cast<v4u_t*>(tile + r * P::kMain)[lane] = w[i];
            noted |= (odd ? 1u : 0u) << i;
          }
          if (lane == 0) s_bad[step % S::SLOTS][wave] = noted;
        }
      }
      lds_barrier();
    };

    floatx4 o[kDt];
#pragma unroll
    for (int i = 0; i < kDt; ++i) o[i] = floatx4{};
    float m_run = kNoMax, l0 = 0.0f, l1 = 0.0f;

    // ---- The first step's rows as soon as the windows are there; the next ones' behind a wait that the compiler
    // sees: it then knows that the queries have come, and adds no waits for them among the steps.
    table.put(e_first, win0);
    table.put(e_first + 64, win1);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    ask(first);
    request(first);
    __builtin_amdgcn_s_waitcnt(0x0F70);   // vmcnt(0)
    asm volatile("" ::: "memory");
#pragma unroll
    for (int i = 1; i < S::SLOTS - 1; ++i)
      if (first + i < last) request(first + i);
    publish(first);

    int slot = first % S::SLOTS;
#pragma unroll 1
    for (int step = first; step < last; ++step) {
      const uint32_t tile = ring0 + slot * S::kTile;
      // (every wave is past the step before: its slot is free)
      if (step + S::SLOTS - 1 < last) request(step + S::SLOTS - 1);
      // ---- Scores: keys 0 .. 15 and 16 .. 31 of the step.
      floatx4 cur[2];
      {
        const uint32_t k = tile + k_lane, r = tile + r_lane;
        pipelined<2 * kQSteps, kAhead>(
            [&](int i) __attribute__((always_inline)) {
              const int c = i >> 1, h = i & 1;   // (the two chains in turn)
              return c < kMainSteps ? lds_read((k ^ ((c & 3) << 6)) + (c >> 2) * 256 + h * 16 * P::kMain)
                                    : lds_read((r ^ ((c - kMainSteps) << 6)) + h * 16 * P::kRot);
            },
            [&](int i, v4u_t x) __attribute__((always_inline)) {
              const int c = i >> 1, h = i & 1;
              cur[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(x), qf[c], c == 0 ? floatx4{} : cur[h], 0, 0, 0);
            });
      }
      if (masked(step)) {
        const TileBlocks tb = blocks_of(step);
        const Column my = column();
        const uint32_t win = row_window(a, q, ctx, my.j, my.valid, step * kKeys, s_word[wave][col]);
        uint32_t bad = 0;
#pragma unroll
        for (int w = 0; w < S::kWaves; ++w) bad |= s_bad[slot][w] << (S::kRows * w);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int kk = 4 * quarter + (i & 3), k = 16 * (i >> 2) + kk;
          const int off = (k & 16) + slot_of_offset(kk, (i >> 2) ? tb.dir1 : tb.dir0);
          const bool sees = ((i >> 2) ? tb.ok1 : tb.ok0) && ((win >> off) & 1u);
          cur[i >> 2][i & 3] = !sees ? -INFINITY : (bad >> k) & 1u ? __uint_as_float(0x7fc00000u) : cur[i >> 2][i & 3];
        }
      }
      // ---- Running maximum (moved lazily) and weights, rounded to bf16 for the second product; the totals
      // add the rounded weights.
      float mr = -INFINITY;
#pragma unroll
      for (int i = 0; i < 8; ++i) mr = fmaxf(mr, cur[i >> 2][i & 3]);
      const float mx = column_max(mr) * sl2;
      const float m_new = mx > m_run + kRescaleSlack ? mx : m_run;
      if (__builtin_amdgcn_ballot_w64(m_new != m_run) != 0) {
        const float alpha = fast_exp2(m_run - m_new);
#pragma unroll
        for (int i = 0; i < kDt; ++i) o[i] *= alpha;
        l0 *= alpha;
        l1 *= alpha;
        m_run = m_new;
      }
      bf16x2_t pw[4];
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const float2_t pp = {fast_exp2(fmaf(cur[w >> 1][2 * (w & 1)], sl2, -m_run)), fast_exp2(fmaf(cur[w >> 1][2 * (w & 1) + 1], sl2, -m_run))};
        pw[w] = __builtin_convertvector(pp, bf16x2_t);
        if (w & 1) l1 = __builtin_amdgcn_fdot2_f32_bf16(pw[w], one2, l1, false);
        else l0 = __builtin_amdgcn_fdot2_f32_bf16(pw[w], one2, l0, false);
      }
      // (a lane's weights are those of keys 4 quarter .. + 3 and 16 on: the value operand's keys come in that order)
      const bf16x8_t pf8 = as_bf16x8(v4u_t{__builtin_bit_cast(uint32_t, pw[0]), __builtin_bit_cast(uint32_t, pw[1]),
                                           __builtin_bit_cast(uint32_t, pw[2]), __builtin_bit_cast(uint32_t, pw[3])});
      // ---- Values.
      {
        const uint32_t v = tile + v_lane;
        pipelined<kDt, kAhead>(
            [&](int i) __attribute__((always_inline)) {
              const uint32_t at_v = (v ^ ((i & 7) << 5)) + (i >> 3) * 256;
              const uint2 x0 = lds_read_turned(at_v), x1 = lds_read_turned(at_v + 16 * P::kMain);
              return v4u_t{x0.x, x0.y, x1.x, x1.y};
            },
            [&](int i, v4u_t x) __attribute__((always_inline)) {
              o[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(x), pf8, o[i], 0, 0, 0);
            });
      }
      publish(step + 1);
      slot = (slot + 1) % S::SLOTS;
    }

    // ---- The end of the segment.
    const float l = column_sum(l0 + l1);
    if (whole) {
      const float inv = l > 0.0f ? 1.0f / l : l == 0.0f ? 0.0f : l;   // (NaN stays)
      const Column my = column();
      if (my.valid) write_columns16<kDt>(static_cast<uint16_t*>(a.out) + my.orow * S::kDims, hv * kDt, o, inv, quarter);
    } else {
      // the sums as they lie: every store of the wave is 1 KiB contiguous
      const size_t ws = 2 * (size_t)me + (first == 0 ? 1 : 0);
      float4* po = reinterpret_cast<float4*>(a.ws_o + ws * S::kSlotFloats) + (cw * S::kDt + hv * kDt) * kWave + lane;
#pragma unroll
      for (int i = 0; i < kDt; ++i) po[i * kWave] = make_float4(o[i][0], o[i][1], o[i][2], o[i][3]);
      if (quarter == 0 && hv == 0) {
        float* ml = a.ws_ml + (ws * S::CT + 16 * cw + col) * 2;
        ml[0] = m_run;
        ml[1] = l;
      }
      if (threadIdx.x == 0 && first == 0) *cut = Cut{s, 0, t, seg.last_share(shares)};
    }
    }

    // ---- The next unit.
    at.step = 0;
    if (x < x_end) next_unit<P>(a, at, seg.tiles);
  }
}

}  // namespace ra
}  // namespace bros
