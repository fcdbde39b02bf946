// Attention of a few new rows of each sequence over its paged cache: drafted tokens over a
// K/V pool, queries in the latent space over a pool of latent rows, and causal chunks over
// keys and values expanded from latents. Shared by tree.hip and latent.hip.
//
// Columns. The G query heads that read one key make a column each of every new row, so a
// sequence has n G columns per KV head (a latent row is the key of all heads: n Hq
// columns). A unit is a (sequence, KV head, tile of columns); its keys come in steps of
// 32 NKW. A workgroup of NCW NKW waves takes a step: wave (cw, kg) the columns 32 cw .. + 31
// against the keys 32 kg .. + 31.
//
// Products, transposed: S^T[key][column] = K Q^T and O^T[dim][column] += V^T P^T, both with
// 32x32x16 matrix instructions, so that a lane owns one column (lane % 32), the softmax needs
// one exchange between the two half-waves, and P goes from the score accumulators straight
// into the second product's operand (keys are permuted alike in P and V^T). K^T operands are
// 16-byte reads of LDS rows, V^T operands transposing reads; the chunks of a row are permuted
// (swz) so that neither meets a bank conflict. Rows reach LDS without registers; each wave waits
// for those it requested itself, and puts in order what it finds there, before the barrier
// that publishes them.
//
// Work (rows_units.h). The steps of all units, each with some for its start (offsets, table, queries, first rows), are laid end to end and
// cut into equal shares, one per workgroup, whatever the sequences' lengths; a unit cut between workgroups leaves partial
// sums (fp32, with their maximum and total) that a merge folds. Where no unit is long,
// whole units are shared out instead, and nothing is merged.
//
// Teams. Where a sequence has several tiles of columns, TEAM workgroups of a die take them side by side, step by step: the
// shares are those of teams, and the keys come from memory once (drafts of four tiles read 1.6 GB where the pool's rows
// are 0.44, at the rate that binds). Expanded keys are read again all the same where a (sequence, head) has more tiles than its team:
// the team comes back to them for each pair, while the other teams of the die pass through other heads' (four
// chunks of 601 to 1400 rows behind up to 6000, 64 heads: 1.97 GB read, where the dense rows are 0.28).
//
// Masks. A row sees the keys before the drafts, and of those the ones its bits name (or the
// causal ones). Only steps that reach the drafts, the context's end or an invalid table
// entry look at masks: a row's 32 bits of the tile's positions. In such tiles a value that is
// not finite enters the product as zero (whatever a slot holds that some row does not see), and
// where it is seen, it is added to the finished rows that see it (rare).
#pragma once

#include "bros_device.h"
#include "bros_kernels.h"
#include "rows_units.h"
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Wunneeded-internal-declaration"   // (its planning is not used here)
#include "prefill_device.h"
#pragma clang diagnostic pop

#include <math.h>

namespace bros {
namespace ra {

using pf::as_bf16x8;
using pf::bf16x2_t;
using pf::bf16x8_t;
using pf::float2_t;
using pf::floatx16;
using pf::lds_barrier;
using pf::lds_read_tr;
using pf::load_to_lds;
using pf::load_word_to_lds;
using pf::pack2_bf16;
using pf::pair_max;
using pf::pair_sum;
using pf::swz;
using pf::v4u_t;
using pf::wait_vmem;

constexpr float kRescaleSlack = 8.0f;    // log2 units: weights stay <= 2^8
constexpr float kNoMax = -1.0e30f;       // finite "no score yet" reference
constexpr int kTable = 128;              // staged table entries of a wave: two windows of 64
constexpr int kNoExponent = -128;        // of a value row of zeros (a row that is not zeros has -120 .. 120)

typedef const v4u_t __attribute__((address_space(3)))* lds_v4u_ptr;
typedef short v4s_t __attribute__((ext_vector_type(4)));
typedef v4s_t __attribute__((address_space(3)))* lds_v4s_ptr;
__device__ __forceinline__ uint32_t lds_address(const void* p) { return (uint32_t)(uintptr_t)p; }   // (the aperture is 4 GiB aligned)
__device__ __forceinline__ v4u_t lds_read(uint32_t at) { return *(lds_v4u_ptr)(uintptr_t)at; }
__device__ __forceinline__ uint2 lds_read_turned(uint32_t at) {
  return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s_ptr)(uintptr_t)at));
}
// Lane id that is computed where it is used (values made of it are not held in registers over a loop).
__device__ __forceinline__ int lane_here() {
  int l;
  asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=v"(l));
  return l;
}
// A word that a load into LDS may have written. (As LDS memory: a generic read would also wait for every load in flight.)
__device__ __forceinline__ int32_t lds_word(const int32_t* p) {
  return *(const volatile int32_t __attribute__((address_space(3)))*)(uintptr_t)lds_address(p);
}

// The two blocks of a tile: whether their entries are valid, and their directions.
struct TileBlocks {
  bool ok0, ok1;
  int dir0, dir1;
};
// Bits 15 and 31: the halves that are infinite or NaN, as bf16 or (HALF) fp16.
template <bool HALF = false>
__device__ __forceinline__ uint32_t not_finite(uint32_t w) {
  return HALF ? ((w & 0x7c007c00u) + 0x04000400u) & 0x80008000u : ((w & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
}
typedef __attribute__((__vector_size__(2 * sizeof(_Float16)))) _Float16 half2_t;
typedef __attribute__((__vector_size__(8 * sizeof(_Float16)))) _Float16 half8_t;
// The two values of a word, as bf16 or fp16.
template <bool HALF>
__device__ __forceinline__ float2_t two_values(uint32_t w) {
  if constexpr (HALF) {
    const half2_t h = __builtin_bit_cast(half2_t, w);
    return float2_t{(float)h[0], (float)h[1]};
  }
  return float2_t{bf16_lo(w), bf16_hi(w)};
}

// The first word of row j's mask (of one that is not there: of the last).
__device__ __forceinline__ uint64_t first_word(const RowsArgs& a, const Seq& q, int j) {
  return a.mask == nullptr ? 0 : a.mask[(size_t)(q.q0 + min(j, q.n - 1)) * a.mask_words];
}
// Bits of the positions pos0 .. + 31 that row j of a sequence sees, of a context of ctx. word0: its mask's first.
__device__ __forceinline__ uint32_t row_window(const RowsArgs& a, const Seq& q, int ctx, int j, bool valid, int pos0, uint64_t word0) {
  const auto below = [](int k) -> uint32_t { return k >= 32 ? 0xffffffffu : k <= 0 ? 0u : (1u << k) - 1u; };
  uint32_t win;
  if (a.mask != nullptr) {
    const int i0 = pos0 - q.c0;   // draft of position pos0 (negative: before the drafts)
    win = below(-i0);
    // the 64 bits from draft max(i0, 0) on
    const int f = max(i0, 0), wd = f >> 6, sh = f & 63;
    uint64_t b = wd == 0 ? word0 >> sh : 0;
    if (a.mask_words > 1) {
      const uint64_t* bits = a.mask + (size_t)(q.q0 + min(j, q.n - 1)) * a.mask_words;
      if (wd > 0 && wd < a.mask_words) b = bits[wd] >> sh;
      if (sh != 0 && wd + 1 < a.mask_words) b |= bits[wd + 1] << (64 - sh);
    }
    if (q.n - f < 64) b &= q.n - f <= 0 ? 0 : (1ull << (q.n - f)) - 1;
    if (i0 > -32) win |= i0 < 0 ? (uint32_t)b << -i0 : (uint32_t)b;
  } else {
    win = below(q.c0 + j + 1 - pos0);
  }
  return valid ? win & below(ctx - pos0) : 0u;
}

__device__ __forceinline__ int64_t wave_scan64(int64_t v, int lane) {
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) {
    const int64_t u = __shfl_up(v, o);
    if (lane >= o) v += u;
  }
  return v;
}

// The steps of all units, and the unit and step of number `at(total)` (at: a function of the
// total, the same for every thread; -1: no place wanted). All THREADS threads call it; `scratch` is 2 x (waves + 1) numbers of
// LDS and s_place a Place.
template <class P, int CT, int KS, int THREADS, class At>
__device__ __forceinline__ Place find_place(const RowsArgs& a, int group, At at, int64_t* scratch, Place* s_place) {
  constexpr int kW = THREADS / kWave;
  const int tid = threadIdx.x, lane = tid & (kWave - 1), w = tid / kWave;
  const Run run(a.num_seqs, THREADS, tid);
  int64_t mine, rows;
  count_run<P, CT, KS>(a, group, run, mine, rows);
  const int64_t inc = wave_scan64(mine, lane);
  int64_t rinc = 0;
  if constexpr (!P::kPaged) rinc = wave_scan64(rows, lane);
  if (lane == kWave - 1) {
    scratch[w] = inc;
    scratch[kW + w] = rinc;
  }
  if (tid == 0) s_place->s = -1;
  __syncthreads();
  int64_t first = inc - mine, rfirst = rinc - rows, total = 0;
#pragma unroll
  for (int i = 0; i < kW; ++i) {
    first += i < w ? scratch[i] : 0;
    if constexpr (!P::kPaged) rfirst += i < w ? scratch[kW + i] : 0;
    total += scratch[i];
  }
  const int64_t x = at(total);
  if (x >= first && x < first + mine) place_in_run<P, CT, KS>(a, group, run, x - first, rfirst, total, s_place);
  __syncthreads();
  Place p = *s_place;
  p.s = __builtin_amdgcn_readfirstlane(p.s);
  p.g = __builtin_amdgcn_readfirstlane(p.g);
  p.t = __builtin_amdgcn_readfirstlane(p.t);
  p.step = __builtin_amdgcn_readfirstlane(p.step);
  p.total = total;
  return p;
}

// Writes a wave's normalised columns: lane l holds column l % 32, accumulators 4 jq .. + 3 of o[i] are dims
// 32 (dt0 + i) + 8 jq + 4 (l / 32) .. + 3.
template <int N>
__device__ __forceinline__ void write_columns(uint16_t* row, int dt0, const floatx16 (&o)[N], float inv, int half) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
#pragma unroll
    for (int jq = 0; jq < 4; ++jq) {
      uint2 w;
      w.x = pack2_bf16(o[i][4 * jq + 0] * inv, o[i][4 * jq + 1] * inv);
      w.y = pack2_bf16(o[i][4 * jq + 2] * inv, o[i][4 * jq + 3] * inv);
      *reinterpret_cast<uint2*>(row + 32 * (dt0 + i) + 8 * jq + 4 * half) = w;
    }
  }
}

// N products, product(i, operand(i)), with the operands of the next DEPTH on their way: the order stands
// as written. (Left alone the compiler reads an operand, waits and multiplies, in turn.)
template <int N, int DEPTH, class Operand, class Product>
__device__ __forceinline__ void pipelined(Operand operand, Product product) {
  v4u_t x[DEPTH];
#pragma unroll
  for (int i = 0; i < DEPTH; ++i) x[i] = operand(i);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    __builtin_amdgcn_sched_barrier(0);
    product(i, x[i % DEPTH]);
    if (i + DEPTH < N) x[i % DEPTH] = operand(i + DEPTH);
  }
  __builtin_amdgcn_sched_barrier(0);
}

// The table entries of a sequence as a wave keeps them: two windows of 64 in LDS. The next window is requested
// kLag steps after the requests of rows have entered the one before it: until then steps may still look at
// entries of the window that it replaces.
struct Table {
  static constexpr int kLag = 4;   // more than the steps between a step's request and its masks
  const int32_t* tbl;
  int32_t* lds;      // [kTable]
  int nblk, num_blocks;
  __device__ __forceinline__ int32_t get(int e0) const { return tbl[max(0, min(e0 + lane_here(), nblk - 1))]; }
  __device__ __forceinline__ void put(int e0, int32_t v) const { lds[(e0 & (kTable - 1)) + lane_here()] = v; }
  __device__ __forceinline__ void load(int e0) const {   // entries e0 .. + 63
    load_word_to_lds(tbl, 4u * (uint32_t)max(0, min(e0 + lane_here(), nblk - 1)), lds + (e0 & (kTable - 1)));
  }
  // A word of LDS that holds entry e (asked for before it is needed), and the entry that it is, -1: none.
  __device__ __forceinline__ int32_t word(int e) const { return lds_word(lds + (e & (kTable - 1))); }
  __device__ __forceinline__ int entry(int e, int32_t word) const {
    const int v = __builtin_amdgcn_readfirstlane(word);
    return (e < nblk && v >= 0 && v < num_blocks) ? v : -1;
  }
};
// Direction of entries e and e + 1 of sequence s; `all`: that of a sequence whose entries have none of their own.
__device__ __forceinline__ void directions(const RowsArgs& a, int s, int e, int all, TileBlocks& tb) {
  tb.dir0 = tb.dir1 = all;
  if (a.dir != nullptr && a.dir_per_entry) {
    const int8_t* d = a.dir + (size_t)s * a.max_blocks_per_seq;
    tb.dir0 = d[min(e, a.max_blocks_per_seq - 1)] < 0 ? -1 : 1;
    tb.dir1 = d[min(e + 1, a.max_blocks_per_seq - 1)] < 0 ? -1 : 1;
  }
}

// A unit cut between shares, as its first share notes it for the merge: its last share (-1: none).
struct Cut {
  int32_t s, g, t, last;
};

template <class P, int NCW, int NKW, int SLOTS_>
struct Shape {
  static constexpr int SLOTS = SLOTS_;
  static constexpr int kWaves = NCW * NKW, kThreads = kWaves * kWave;
  static constexpr int CT = 32 * NCW, KS = kKeys * NKW;
  static constexpr int kLaneCols = 32;                              // columns of a wave
  static constexpr int kDims = P::kVal / 2, kDt = kDims / 32;       // 32-dim pieces of a value
  static constexpr int kQDims = (P::kMain + P::kRot) / 2;
  static constexpr int kRotAt = kKeys * P::kMain;                   // LDS of a tile: first parts, second parts, values
  static constexpr int kValAt = kRotAt + kKeys * P::kRot;
  static constexpr int kTile = kValAt + kKeys * P::kVal;
  static constexpr int kRing = NKW * SLOTS * kTile;
  static constexpr int kRows = kKeys / NCW;                         // rows of a tile that a wave requests
  static constexpr int kLoads = 2 * kRows / 4 + (P::kRot ? (kRows + 7) / 8 : 0);   // of 1 KiB
  static constexpr int kSlotFloats = CT * kDims;                    // a partial's sums
  static constexpr int kChunks = kDims / 8;                         // of a wave's partial, 1 KiB each
  // first of the four dims that a lane has in chunk i
  static __device__ __forceinline__ int dim_of(int i, int lane) { return 8 * i + 4 * (lane >> 5); }
  static_assert(P::kMain == 256 && (P::kRot == 0 || P::kRot == 128), "");
  static_assert(kRows % 4 == 0, "a load takes four rows of 256 bytes");
  static_assert((NKW - 1) * NCW * 32 * kDims * 4 <= kRing, "the key groups' sums meet in the ring");
};

template <class P, int NCW, int NKW, int SLOTS, int OCC, int TEAM>
__global__ __launch_bounds__(64 * NCW * NKW, OCC) void rows_kernel(RowsArgs a) {
  using S = Shape<P, NCW, NKW, SLOTS>;
  constexpr int kDt = S::kDt, kMainSteps = P::kMain / 32, kQSteps = S::kQDims / 16, kR = S::kRows;
  constexpr int kAhead = 6;   // operands read before the first product
  // With three steps' rows in LDS or more, the scores of a step are formed beside the softmax of the one before it,
  // whose values follow: the matrix cores and the vector units then work at the same time.
  constexpr bool kOverlap = SLOTS >= 3;
  __shared__ __attribute__((aligned(1024))) uint8_t s_ring[S::kRing];
  __shared__ int32_t s_tab[S::kWaves][kTable];
  __shared__ int64_t s_scan[2 * S::kWaves];
  __shared__ Place s_place;
  __shared__ __attribute__((aligned(4))) uint8_t s_odd[4];   // of each wave: it left out a value that is not finite
  static_assert(S::kWaves <= 4, "their notes are read as one word");

  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = wave_id_uniform();
  const int cw = wave % NCW, kg = wave / NCW;
  const int half = lane >> 5, col = lane & 31;
  const int Hkv = a.num_kv_heads, G = P::kPaged ? a.num_q_heads / Hkv : 1;   // (expanded: heads of their own)
  // neighbouring shares to one die
  const int nb = gridDim.x;
  const int me = nb % pf::kXcds == 0 ? (blockIdx.x % pf::kXcds) * (nb / pf::kXcds) + blockIdx.x / pf::kXcds : blockIdx.x;
  const int team = me / TEAM, member = me % TEAM;
  Cut* cut = reinterpret_cast<Cut*>(a.ws_cut) + me;
  if (tid == 0) cut->last = -1;

  Place at = find_place<P, S::CT * TEAM, S::KS, S::kThreads>(
      a, G, [&](int64_t total) -> int64_t {
        const Shares sh(a, total);
        return team < sh.n ? sh.begin(team) : -1;
      }, s_scan, &s_place);
  if (at.s < 0) return;   // (uniform: no step left for this workgroup)
  const Shares shares(a, at.total);
  int64_t x = shares.begin(team);
  const int64_t x_end = shares.begin(team + 1);

  const float sl2 = a.scale_log2;
  const bf16x2_t one2 = {(__bf16)1.0f, (__bf16)1.0f};
  // Operand reads: lane addresses of a tile at 0. A chunk's low four bits are those of the
  // row's permutation, so that other chunks are a xor and a constant away.
  const uint32_t k_lane = col * P::kMain + ((half ^ swz(col)) << 4);
  const uint32_t r_lane = S::kRotAt + (col >> 1) * 256 + ((col & 1) << 7) + ((half ^ ((col >> 1) & 7)) << 4);
  const int v_key = 4 * half + ((lane >> 2) & 3);
  const uint32_t v_lane = S::kValAt + v_key * P::kVal + (((2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ swz(v_key)) << 4) + (lane & 1) * 8;
  // Requests: a lane's byte of four rows of 256, and of eight of 128. The first row's other bits of the
  // permutation are the same for every lane: a xor.
  const uint32_t main_off = (uint32_t)((lane >> 4) * 256 + (((lane & 15) ^ ((lane >> 4) << 2)) << 4));
  const uint32_t rot_off = (uint32_t)((lane >> 3) * 128 + (((lane & 7) ^ (lane >> 4)) << 4));
  // The lane where it is seldom needed: with expanded keys the usual loop needs the registers that places made of it would
  // hold (42 of them went to scratch memory, and chunks took 790 us instead of 710).
  const auto lane_again = [&]() __attribute__((always_inline)) -> int { return P::kHalf ? lane_here() : lane; };
  uint8_t* const ring = s_ring + kg * SLOTS * S::kTile;
  const uint32_t ring0 = lds_address(ring);

  while (x < x_end) {
    // ---- The segment: steps [first, last) of unit (s, g, t).
    const Segment<P, S::CT, S::KS, TEAM> seg(a, at, G, member, x, x_end);
    const int s = at.s, g = at.g, t = seg.t, first = seg.first, last = seg.last, cnt = seg.count;
    const Seq q = seg.q;
    const bool whole = seg.whole;
    x = seg.next;
    if (cnt > 0) {
    // (dense keys that do not fit their buffer: the sequence's rows see nothing)
    const bool fits = P::kPaged || at.row0 + dense_rows(q.ctx) <= a.dense_rows;
    const int ctx = fits ? q.ctx : 0, n = q.n;
    const int c = t * S::CT + 32 * cw + col;        // the lane's column
    const int j = c / G;                            // its row
    const bool valid = j < n;
    const size_t orow = (size_t)(q.q0 + min(j, n - 1)) * a.num_q_heads + a.head0 + g * G + (c - j * G);
    // keys below this position are seen by every row of the unit
    const int full_below = a.mask != nullptr ? min(ctx, q.c0) : min(ctx, q.c0 + t * S::CT / G + 1);
    const Table table{a.block_tables + (size_t)s * a.max_blocks_per_seq, s_tab[wave], (ctx + kBlockSize - 1) / kBlockSize, a.num_blocks};

    // ---- Start: the first windows of the table, then queries and masks.
    __syncthreads();   // (the ring's last use: the segment before this one)
    const int e_first = 2 * (first * NKW + kg) & ~63;
    const int32_t win0 = table.get(e_first), win1 = table.get(e_first + 64);
    const int dir_all = P::kPaged ? seq_direction(a.dir, a.cls, s) : 1;   // (read where entries have no directions of their own)
    const uint64_t word0 = first_word(a, q, j);
    bf16x8_t qf[kQSteps];
    {
      // (columns behind the last row take that row's values: nothing is made of them)
      const uint16_t* qp = static_cast<const uint16_t*>(a.q) + orow * S::kQDims + 8 * half;
#pragma unroll
      for (int i = 0; i < kQSteps; ++i) qf[i] = as_bf16x8(*reinterpret_cast<const v4u_t*>(qp + 16 * i));
    }

    uint32_t holes = 0;         // bit step % 32: a block of that step's tile is missing
    int32_t word_a = 0, word_b = 0;   // the next request's entries
    auto ask = [&](int step) __attribute__((always_inline)) {
      const int e = 2 * (step * NKW + kg);
      word_a = table.word(e);
      word_b = table.word(e + 1);
    };
    // Requests the wave's part of the rows of a step.
    auto request = [&](int step) __attribute__((always_inline)) {
      const int e = 2 * (step * NKW + kg);
      const int b0 = table.entry(e, word_a), b1 = table.entry(e + 1, word_b);
      if ((e & 63) / (2 * NKW) == Table::kLag) table.load((e & ~63) + 64);
      ask(step + 1);
      holes = (holes & ~(1u << (step & 31))) | ((b0 < 0 || b1 < 0 ? 1u : 0u) << (step & 31));
      uint8_t* dst = ring + (step % SLOTS) * S::kTile;
      // (dense rows: of the tile, whose place is known; of one behind the context, which nothing is made of, within the buffer)
      const size_t row0 = P::kPaged || !fits ? 0 : (size_t)min(at.row0 + (int64_t)step * S::KS + kKeys * kg, a.dense_rows - kKeys);
#pragma unroll
      for (int i = 0; i < kR / 4; ++i) {
        const int row = kR * cw + 4 * i;   // the first of four
        size_t src;
        if constexpr (P::kPaged) src = ((size_t)max((row >> 4) ? b1 : b0, 0) * Hkv + g) * (kBlockSize * P::kMain) + (row & 15) * P::kMain;
        else src = ((size_t)g * a.dense_rows + row0 + row) * P::kMain;
        const uint32_t off = main_off ^ ((((row >> 2) & 1) << 1 | ((row >> 3) & 1)) << 4);
        load_to_lds(static_cast<const uint8_t*>(a.k_pool) + src, off, dst + row * P::kMain);
        load_to_lds(static_cast<const uint8_t*>(a.v_pool) + src, off, dst + S::kValAt + row * P::kVal);
      }
      if constexpr (P::kRot != 0) {
#pragma unroll
        for (int i = 0; i < kR / 8; ++i) {
          const int row = kR * cw + 8 * i;
          load_to_lds(static_cast<const uint8_t*>(a.rot_rows) + (row0 + row) * P::kRot, rot_off ^ (((row >> 3) & 1) << 6),
                      dst + S::kRotAt + row * P::kRot);
        }
      }
    };
    // The first position of the wave's tile in a step; whether the step needs masks there.
    auto pos_of = [&](int step) -> int { return step * S::KS + kKeys * kg; };
    auto masked = [&](int step) -> bool { return ((holes >> (step & 31)) & 1) || pos_of(step) + kKeys > full_below; };
    auto blocks_of = [&](int pos0) __attribute__((always_inline)) -> TileBlocks {   // (of a step whose entries are still in LDS)
      const int e = pos0 / kBlockSize;
      TileBlocks tb;
      tb.ok0 = table.entry(e, table.word(e)) >= 0;
      tb.ok1 = table.entry(e + 1, table.word(e + 1)) >= 0;
      if constexpr (P::kPaged) directions(a, s, e, dir_all, tb);
      else tb.dir0 = tb.dir1 = 1;   // (dense rows lie in the order of their positions)
      return tb;
    };

    floatx16 o[kDt];
#pragma unroll
    for (int i = 0; i < kDt; ++i) o[i] = floatx16{};
    float m_run = kNoMax, l0 = 0.0f, l1 = 0.0f;
    // Values that stand behind exponents e of their rows (nearly never any). An fp16 weight must not take them up: it has no
    // room below 2^-24 for a tile of small values, nor may a row that a column does not see set what is lost in it. So a tile's products are
    // made of weights 2^(score + e - r), r being the column's largest score + e in this tile, and are added to the sums in fp32, which
    // stand in units of 2^r_run, with the largest r so far. A loop of its own, without overlap: a call that is all of such values takes 1.39
    // times as long (four chunks of 700 to 1400 rows behind up to 5000, 64 heads, 1030 and 1430 us).
    // (Places are formed anew at each use: the usual loop needs the registers.)
    const auto scaled_tile = [&](int tile) __attribute__((always_inline)) -> int32_t { return a.scaled[((size_t)g * a.dense_rows + at.row0) / kKeys + tile]; };
    const auto exps_of = [&](int pos) __attribute__((always_inline)) -> uint32_t {   // of four positions
      return *reinterpret_cast<const uint32_t*>(a.exps + (size_t)g * a.dense_rows + at.row0 + pos);
    };
    uint32_t odd = 0;   // a value that is not finite was left out of a product

    // Waits for the wave's rows of a step (those of the next `most` may be in flight) and, where the step is
    // masked, puts its values in order: zeros where no context is, and for values that are not finite. Then
    // the waves that share a tile meet.
    auto publish = [&](int step, int most) __attribute__((always_inline)) {
      if (step < last) {
        const int later = min(most, last - 1 - step);
        if (later >= 2) wait_vmem<2 * S::kLoads>();
        else if (later == 1) wait_vmem<S::kLoads>();
        else wait_vmem<0>();
        // (a wave alone on its tile passes over one without context, unless the loop takes every tile)
        if (masked(step) && (NCW > 1 || kOverlap || pos_of(step) < ctx)) {
          const int pos0 = pos_of(step);
          const TileBlocks tb = blocks_of(pos0);
          const int ln = lane_again();
          uint8_t* vt = ring + (step % SLOTS) * S::kTile + S::kValAt;
          constexpr int kMine = kR * (P::kVal / 16) / kWave;   // 16-byte chunks of a lane
          v4u_t w[kMine];
#pragma unroll
          for (int i = 0; i < kMine; ++i) w[i] = reinterpret_cast<const v4u_t*>(vt + kR * cw * P::kVal)[i * kWave + ln];
#pragma unroll
          for (int i = 0; i < kMine; ++i) {
            const int r = kR * cw + (i * kWave + ln) / (P::kVal / 16);
            const int pos = pos0 + (r & 16) + slot_of_offset(r & 15, r < 16 ? tb.dir0 : tb.dir1);
            const bool there = (r < 16 ? tb.ok0 : tb.ok1) && pos < ctx;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const uint32_t bad = there ? not_finite<P::kHalf>(w[i][e]) : 0;
              odd |= bad;
              w[i][e] = there ? w[i][e] & ~((bad >> 15) * 0xffffu) : 0;
            }
            reinterpret_cast<v4u_t*>(vt + kR * cw * P::kVal)[i * kWave + ln] = w[i];
          }
        }
      }
      if constexpr (NCW > 1) lds_barrier();
      else asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // (a wave's own rows: what was read is read, what was written is there)
    };

    // ---- The first step's rows as soon as the windows are there; the next ones' behind a wait that the compiler
    // sees: it then knows that queries and masks have come, and adds no waits for them among the steps.
    table.put(e_first, win0);
    table.put(e_first + 64, win1);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    ask(first);
    request(first);
    bool scaled = false;   // any of the segment's tiles is
    if constexpr (P::kHalf) {
      int any = 0;
      const int tiles = min(last * NKW, (ctx + kKeys - 1) / kKeys);
      for (int i = first * NKW + lane_here(); i < tiles; i += kWave) any |= scaled_tile(i);
      scaled = __builtin_amdgcn_ballot_w64(any != 0) != 0;
    }
    __builtin_amdgcn_s_waitcnt(0x0F70);   // vmcnt(0)
    asm volatile("" ::: "memory");
#pragma unroll
    for (int i = 1; i < SLOTS - 1; ++i)
      if (first + i < last) request(first + i);
    publish(first, SLOTS - 2);

    const auto slot_of = [&](int step) -> uint32_t { return ring0 + (step % SLOTS) * S::kTile; };
    // The steps; kScaled: with exponents of values. (Two loops, so that the usual one has no branches for them.)
    float m_prev = kNoMax;
    auto steps = [&](auto scaledc) __attribute__((always_inline)) {
      constexpr bool kScaled = decltype(scaledc)::value;
      // Masks a tile's scores and moves the running maximum (lazily); gives the factor that the sums take for it.
      auto mask_max = [&](floatx16& cur, int step) __attribute__((always_inline)) {
        if (masked(step)) {
          const int pos0 = pos_of(step);
          const TileBlocks tb = blocks_of(pos0);
          const uint32_t win = row_window(a, q, ctx, j, valid, pos0, word0);
          const int half_here = lane_again() >> 5;
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int k = 8 * (i >> 2) + 4 * half_here + (i & 3);
            const int off = (k & 16) + slot_of_offset(k & 15, (i >> 3) ? tb.dir1 : tb.dir0);
            cur[i] = ((i >> 3) ? tb.ok1 : tb.ok0) && ((win >> off) & 1u) ? cur[i] : -INFINITY;
          }
        }
        float mr = -INFINITY;
#pragma unroll
        for (int i = 0; i < 16; ++i) mr = fmaxf(mr, cur[i]);
        const float mx = pair_max(mr) * sl2;
        m_prev = m_run;
        m_run = mx > m_run + kRescaleSlack ? mx : m_run;
      };
      auto rescale = [&]() __attribute__((always_inline)) {
        if (__builtin_amdgcn_ballot_w64(m_run != m_prev) != 0) {
          const float alpha = fast_exp2(m_prev - m_run);
          if constexpr (!kScaled) {
#pragma unroll
            for (int i = 0; i < kDt; ++i) o[i] *= alpha;
          }
          l0 *= alpha;
          l1 *= alpha;
        }
      };
      // Weights, rounded to 16 bits (bf16, or fp16 where the values are) for the second product; the totals add the
      // rounded weights.
      auto weights = [&](const floatx16& cur, bf16x8_t (&pfr)[2]) __attribute__((always_inline)) {
        if constexpr (P::kHalf) {
          const half2_t ones = {(_Float16)1.0f, (_Float16)1.0f};
#pragma unroll
          for (int c2 = 0; c2 < 2; ++c2) {
            half2_t pw[4];
#pragma unroll
            for (int w = 0; w < 4; ++w) {
              const float2_t pp = {fast_exp2(fmaf(cur[8 * c2 + 2 * w], sl2, -m_run)), fast_exp2(fmaf(cur[8 * c2 + 2 * w + 1], sl2, -m_run))};
              pw[w] = __builtin_convertvector(pp, half2_t);
              if (w & 1) l1 = __builtin_amdgcn_fdot2(pw[w], ones, l1, false);
              else l0 = __builtin_amdgcn_fdot2(pw[w], ones, l0, false);
            }
            const v4u_t pk = {__builtin_bit_cast(uint32_t, pw[0]), __builtin_bit_cast(uint32_t, pw[1]),
                              __builtin_bit_cast(uint32_t, pw[2]), __builtin_bit_cast(uint32_t, pw[3])};
            pfr[c2] = as_bf16x8(pk);
          }
          return;
        }
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
      };
      const auto key_operand = [&](uint32_t tile, int i) __attribute__((always_inline)) {
        return i < kMainSteps ? lds_read((tile + k_lane) ^ (i << 5)) : lds_read((tile + r_lane) ^ ((i - kMainSteps) << 5));
      };
      const auto value_operand = [&](uint32_t tile, int i) __attribute__((always_inline)) {
        const uint32_t at_v = ((tile + v_lane) ^ ((i % kDt) << 6)) + 16 * (i / kDt) * P::kVal;
        // (keys 8 on: another bit of the row's permutation)
        const uint2 x0 = lds_read_turned(at_v), x1 = lds_read_turned((at_v ^ 16) + 8 * P::kVal);
        return v4u_t{x0.x, x0.y, x1.x, x1.y};
      };
      const auto score = [&](floatx16& cur, int i, v4u_t x) __attribute__((always_inline)) {
        cur = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(x), qf[i], i == 0 ? floatx16{} : cur, 0, 0, 0);
      };
      const auto value = [&](const bf16x8_t (&pfr)[2], int i, v4u_t x) __attribute__((always_inline)) {
        if constexpr (P::kHalf)
          o[i % kDt] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8_t, x), __builtin_bit_cast(half8_t, pfr[i / kDt]), o[i % kDt], 0, 0, 0);
        else
          o[i % kDt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(x), pfr[i / kDt], o[i % kDt], 0, 0, 0);
      };

      // A tile's values behind exponents (the totals count a weight whatever its exponent).
      float r_run = kNoMax;
      const auto scaled_values = [&](floatx16& cur, int step, uint32_t tile) __attribute__((always_inline)) {
        const int pos0 = pos_of(step), half_here = lane_here() >> 5;
        const bool is = pos0 < ctx && __builtin_amdgcn_readfirstlane(scaled_tile(pos0 / kKeys)) != 0;
#pragma unroll
        for (int c = 0; c < 4; ++c) {   // keys 8 c + 4 half .. + 3
          const uint32_t e4 = is ? exps_of(pos0 + 8 * c + 4 * half_here) : 0;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            l0 += fast_exp2(fmaf(cur[4 * c + i], sl2, -m_run));
            cur[4 * c + i] = fmaf(cur[4 * c + i], sl2, (float)(int8_t)(e4 >> (8 * i)));
          }
        }
        float r = kNoMax;   // (nothing seen: weights of 0)
#pragma unroll
        for (int i = 0; i < 16; ++i) r = fmaxf(r, cur[i]);
        r = pair_max(r);
        const float r_new = fmaxf(r_run, r), f_run = fast_exp2(r_run - r_new), f = fast_exp2(r - r_new);
        r_run = r_new;
        v4u_t pw[2];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float2_t pp = {fast_exp2(cur[2 * i] - r), fast_exp2(cur[2 * i + 1] - r)};
          pw[i >> 2][i & 3] = __builtin_bit_cast(uint32_t, __builtin_convertvector(pp, half2_t));
        }
#pragma unroll
        for (int i = 0; i < kDt; ++i) {
          floatx16 y{};
#pragma unroll
          for (int c2 = 0; c2 < 2; ++c2)
            y = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8_t, value_operand(tile, kDt * c2 + i)), __builtin_bit_cast(half8_t, pw[c2]), y, 0, 0, 0);
          o[i] = o[i] * f_run + y * f;
        }
      };

      if constexpr (kOverlap && !kScaled) {
        // Step i: the scores of step i + 1 (from `in`'s successor's rows) while the vector units turn those of
        // step i into weights, then its values. The compiler interleaves them.
        auto turn = [&](int step, const floatx16& in, floatx16& next) __attribute__((always_inline)) {
          publish(step + 1, SLOTS - 3);
          if (step + SLOTS - 1 < last) request(step + SLOTS - 1);
          const uint32_t tile = slot_of(step), tile1 = slot_of(step + 1);
          v4u_t kv[kQSteps], v0[kDt], v1[kDt];
#pragma unroll
          for (int i = 0; i < kQSteps; ++i) kv[i] = key_operand(tile1, i);
#pragma unroll
          for (int i = 0; i < kDt; ++i) v0[i] = value_operand(tile, i);
          bf16x8_t pfr[2];
#pragma unroll
          for (int i = 0; i < kQSteps; ++i) score(next, i, kv[i]);
          weights(in, pfr);
#pragma unroll
          for (int i = 0; i < kDt; ++i) v1[i] = value_operand(tile, kDt + i);
#pragma unroll
          for (int i = 0; i < kDt; ++i) value(pfr, i, v0[i]);
#pragma unroll
          for (int i = 0; i < kDt; ++i) value(pfr, kDt + i, v1[i]);
          mask_max(next, step + 1);
          rescale();
        };
        floatx16 sa, sb;
#pragma unroll
        for (int i = 0; i < kQSteps; ++i) score(sa, i, key_operand(slot_of(first), i));
        mask_max(sa, first);
        int step = first;
#pragma unroll 1
        for (; step + 2 < last; step += 2) {
          turn(step, sa, sb);
          turn(step + 1, sb, sa);
        }
        if (step + 1 < last) {
          turn(step, sa, sb);
          sa = sb;
          ++step;
        }
        bf16x8_t pfr[2];
        weights(sa, pfr);
        const uint32_t tile = slot_of(step);
#pragma unroll
        for (int i = 0; i < 2 * kDt; ++i) value(pfr, i, value_operand(tile, i));
      } else {
#pragma unroll 1
        for (int step = first; step < last; ++step) {
          // (every wave is past the step before: its slot is free)
          if (step + SLOTS - 1 < last) request(step + SLOTS - 1);
          const uint32_t tile = slot_of(step);
          // (a wave alone on its tile passes over one without context)
          if (NCW == 1 && pos_of(step) >= ctx) {
            publish(step + 1, SLOTS - 2);
            continue;
          }
          floatx16 cur;
          pipelined<kQSteps, kAhead>([&](int i) __attribute__((always_inline)) { return key_operand(tile, i); },
                                     [&](int i, v4u_t x) __attribute__((always_inline)) { score(cur, i, x); });
          mask_max(cur, step);
          rescale();
          if constexpr (kScaled) {
            scaled_values(cur, step, tile);
          } else {
            bf16x8_t pfr[2];
            weights(cur, pfr);
            pipelined<2 * kDt, kAhead>([&](int i) __attribute__((always_inline)) { return value_operand(tile, i); },
                                       [&](int i, v4u_t x) __attribute__((always_inline)) { value(pfr, i, x); });
          }
          publish(step + 1, SLOTS - 2);
        }
      }
      if constexpr (kScaled) {
        // from units of 2^r_run to those of the totals; the totals' move up where the sums would not fit into fp32 (they are
        // below 2^33 here, and values, as what the totals divide them to, may be near 2^128)
        const float up = fmaxf(0.0f, r_run - m_run - 90.0f), f = fast_exp2(r_run - m_run - up), fl = fast_exp2(-up);
        m_run += up;
        l0 *= fl;
        l1 *= fl;
#pragma unroll
        for (int i = 0; i < kDt; ++i) o[i] *= f;
      }
    };
    if constexpr (P::kHalf) {
      if (scaled) steps(std::true_type{});
      else steps(std::false_type{});
    } else {
      steps(std::false_type{});
    }

    // ---- The end of the segment.
    const int lane_e = lane_again(), half_e = lane_e >> 5, col_e = lane_e & 31;
    float l = pair_sum(l0 + l1);
    // (every wave writes its note, before a barrier that the readers wait for and, at the next segment's start, behind one)
    const bool any_odd = __builtin_amdgcn_ballot_w64(odd != 0) != 0;
    if (lane_e == 0) s_odd[wave] = any_odd;
    if constexpr (NKW == 1) __syncthreads();   // (else the key groups' sums meet behind one)
    if constexpr (NKW > 1) {
      // the key groups' sums meet in the ring
      float4* xo = reinterpret_cast<float4*>(s_ring);
      __shared__ float s_ml[NKW > 1 ? (NKW - 1) * NCW * 32 * 2 : 1];
      __syncthreads();
      if (kg > 0) {
        const int w = (kg - 1) * NCW + cw;
#pragma unroll
        for (int i = 0; i < kDt; ++i) {
#pragma unroll
          for (int jq = 0; jq < 4; ++jq)
            xo[(w * kDt * 4 + 4 * i + jq) * kWave + lane_e] = make_float4(o[i][4 * jq], o[i][4 * jq + 1], o[i][4 * jq + 2], o[i][4 * jq + 3]);
        }
        if (half_e == 0) {
          s_ml[2 * (w * 32 + col_e)] = m_run;
          s_ml[2 * (w * 32 + col_e) + 1] = l;
        }
      }
      __syncthreads();
      if (kg == 0) {
#pragma unroll 1
        for (int k = 1; k < NKW; ++k) {
          const int w = (k - 1) * NCW + cw;
          const float m2 = s_ml[2 * (w * 32 + col_e)], l2 = s_ml[2 * (w * 32 + col_e) + 1];
          const float m = fmaxf(m_run, m2);
          const float f1 = fast_exp2(m_run - m), f2 = fast_exp2(m2 - m);
          m_run = m;
          l = l * f1 + l2 * f2;
#pragma unroll
          for (int i = 0; i < kDt; ++i) {
#pragma unroll
            for (int jq = 0; jq < 4; ++jq) {
              const float4 y = xo[(w * kDt * 4 + 4 * i + jq) * kWave + lane_e];
              o[i][4 * jq] = o[i][4 * jq] * f1 + y.x * f2;
              o[i][4 * jq + 1] = o[i][4 * jq + 1] * f1 + y.y * f2;
              o[i][4 * jq + 2] = o[i][4 * jq + 2] * f1 + y.z * f2;
              o[i][4 * jq + 3] = o[i][4 * jq + 3] * f1 + y.w * f2;
            }
          }
        }
      }
    }
    const size_t ws = 2 * (size_t)me + (first == 0 ? 1 : 0);   // the partial's slot
    if (kg == 0) {
      if (whole) {
        const float inv = l > 0.0f ? 1.0f / l : l == 0.0f ? 0.0f : l;   // (NaN stays)
        if (valid) write_columns<kDt>(static_cast<uint16_t*>(a.out) + orow * S::kDims, 0, o, inv, half_e);
      } else {
        // the accumulators as they lie: every store of the wave is 1 KiB contiguous
        float4* po = reinterpret_cast<float4*>(a.ws_o + ws * S::kSlotFloats) + cw * kDt * 4 * kWave + lane_e;
#pragma unroll
        for (int i = 0; i < kDt; ++i) {
#pragma unroll
          for (int jq = 0; jq < 4; ++jq)
            po[(4 * i + jq) * kWave] = make_float4(o[i][4 * jq], o[i][4 * jq + 1], o[i][4 * jq + 2], o[i][4 * jq + 3]);
        }
        if (half_e == 0) {
          float* ml = a.ws_ml + (ws * S::CT + 32 * cw + col_e) * 2;
          ml[0] = m_run;
          ml[1] = l;
        }
        if (tid == 0 && first == 0) *cut = Cut{s, g, t, seg.last_share(shares) * TEAM + member};
      }
    }
    // ---- Values that were left out and are seen: added to the rows that see them, where
    // those now lie. (Every key of the segment's masked tiles is looked at again, in memory.)
    if (kg == 0 && (*reinterpret_cast<const uint32_t*>(s_odd) & (0xffffffffu >> (32 - 8 * S::kWaves))) != 0) {
      const int tiles = cnt * NKW;
#pragma unroll 1
      for (int ti = 0; ti < tiles; ++ti) {
        const int pos0 = first * S::KS + kKeys * ti, e0 = pos0 / kBlockSize;
        const auto there = [&](int e) { return e < table.nblk && table.tbl[e] >= 0 && table.tbl[e] < a.num_blocks; };
        TileBlocks tb{there(e0), there(e0 + 1), 1, 1};
        if constexpr (P::kPaged) directions(a, s, e0, dir_all, tb);
        if (pos0 + kKeys <= full_below && tb.ok0 && tb.ok1) continue;
        const uint32_t win = row_window(a, q, ctx, j, valid, pos0, word0);
        // value row of tile row r, or null where no context is
        const auto value_row = [&](int r) -> const uint8_t* {
          const int pos = pos0 + (r & 16) + slot_of_offset(r & 15, r < 16 ? tb.dir0 : tb.dir1);
          if (!(r < 16 ? tb.ok0 : tb.ok1) || pos >= ctx) return nullptr;
          if constexpr (P::kPaged)
            return static_cast<const uint8_t*>(a.v_pool) + (((size_t)table.tbl[pos / kBlockSize] * Hkv + g) * kBlockSize + (r & 15)) * P::kVal;
          return static_cast<const uint8_t*>(a.v_pool) + ((size_t)g * a.dense_rows + at.row0 + pos0 + r) * P::kVal;
        };
        uint32_t any = 0;
        for (int i = lane_e; i < kKeys * (P::kVal / 16); i += kWave) {
          const uint8_t* row = value_row(i / (P::kVal / 16));
          if (row == nullptr) continue;
          const v4u_t w = *reinterpret_cast<const v4u_t*>(row + 16 * (i % (P::kVal / 16)));
          any |= not_finite<P::kHalf>(w[0]) | not_finite<P::kHalf>(w[1]) | not_finite<P::kHalf>(w[2]) | not_finite<P::kHalf>(w[3]);
        }
        if (__builtin_amdgcn_ballot_w64(any != 0) == 0) continue;
#pragma unroll 1
        for (int r = 0; r < kKeys; ++r) {
          const uint8_t* row = value_row(r);
          if (row == nullptr) continue;
          const int off = (r & 16) + slot_of_offset(r & 15, r < 16 ? tb.dir0 : tb.dir1);
          if (!((win >> off) & 1u)) continue;
#pragma unroll 1
          for (int i = 0; i < 4 * kDt; ++i) {
            const int d = 8 * i + 4 * half_e;   // four dims
            const uint2 w = *reinterpret_cast<const uint2*>(row + 2 * d);
            if ((not_finite<P::kHalf>(w.x) | not_finite<P::kHalf>(w.y)) == 0) continue;
            const float2_t v01 = two_values<P::kHalf>(w.x), v23 = two_values<P::kHalf>(w.y);
            const float v[4] = {v01[0], v01[1], v23[0], v23[1]};
            if (whole) {
              uint2* at_out = reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.out) + orow * S::kDims + d);
              const uint2 y = *at_out;
              float z[4] = {bf16_lo(y.x), bf16_hi(y.x), bf16_lo(y.y), bf16_hi(y.y)};
#pragma unroll
              for (int e = 0; e < 4; ++e) z[e] = fabsf(v[e]) < INFINITY ? z[e] : z[e] + v[e];
              *at_out = make_uint2(pack2_bf16(z[0], z[1]), pack2_bf16(z[2], z[3]));
            } else {
              float* at_ws = a.ws_o + ws * S::kSlotFloats + (cw * kDt * 4 + i) * (4 * kWave) + 4 * lane_e;
#pragma unroll
              for (int e = 0; e < 4; ++e)
                if (!(fabsf(v[e]) < INFINITY)) at_ws[e] += v[e];
            }
          }
        }
      }
    }

    }

    // ---- The next unit.
    at.step = 0;
    if (x < x_end) next_unit<P>(a, at, seg.tiles);
  }
}

// Folds the partials of the units cut between shares, in the order of their keys: bound by the chain of the note, maxima and sums (5
// us at least), for wide units by the partials' bytes (19 us for 64 MB). Workgroup (w, y) takes the chunks kWaves kEach y .. of the unit
// that share w noted. A chunk is 1 KiB of a partial: a wave's columns, four dims to a lane.
constexpr int kMergeWaves = 4, kMergeEach = 2;   // waves of a workgroup, chunks of a wave
template <class S, bool DENSE, int TEAM>
__global__ __launch_bounds__(kMergeWaves * kWave) void rows_merge_kernel(RowsArgs a) {
  constexpr int kGroups = S::CT / S::kLaneCols;            // column waves of a partial
  constexpr int kParts = S::kChunks / kMergeEach;          // waves to one of them
  static_assert(S::kChunks % kMergeEach == 0 && kGroups * kParts % kMergeWaves == 0, "");
  const int w0 = blockIdx.x, lane = threadIdx.x & (kWave - 1);
  const Cut cut = reinterpret_cast<const Cut*>(a.ws_cut)[w0];
  if (cut.last < 0) return;
  const int item = blockIdx.y * kMergeWaves + wave_id_uniform();
  const int cw = item / kParts, i0 = (item % kParts) * kMergeEach;
  const int col = S::kLaneCols * cw + lane % S::kLaneCols;
  const int pieces = (cut.last - w0) / TEAM + 1;
  const auto slot = [&](int p) -> size_t { return 2 * (size_t)(w0 + p * TEAM) + (p == 0 ? 1 : 0); };
  const auto ml = [&](int p) -> float2 { return reinterpret_cast<const float2*>(a.ws_ml)[slot(p) * S::CT + col]; };

  // (all that the first four pieces need is asked for at once: most units have no more)
  const Seq q = seq_of(a, cut.s);
  float2 y[4];
  float4 z[4][kMergeEach];
  const auto load_ml = [&](int p) __attribute__((always_inline)) {   // (past the end: the last again)
#pragma unroll
    for (int u = 0; u < 4; ++u) y[u] = ml(min(p + u, pieces - 1));
  };
  const auto load_sums = [&](int p) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const float4* po = reinterpret_cast<const float4*>(a.ws_o + slot(min(p + u, pieces - 1)) * S::kSlotFloats) + (cw * S::kChunks + i0) * kWave + lane;
#pragma unroll
      for (int i = 0; i < kMergeEach; ++i) z[u][i] = po[i * kWave];
    }
  };
  load_ml(0);
  load_sums(0);
  float m = fmaxf(fmaxf(y[0].x, y[1].x), fmaxf(y[2].x, y[3].x));
  for (int p = 4; p < pieces; p += 4) {
    float2 w[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) w[u] = ml(min(p + u, pieces - 1));
#pragma unroll
    for (int u = 0; u < 4; ++u) m = fmaxf(m, w[u].x);
  }
  m = fmaxf(m, kNoMax);   // (a maximum that is not a number)
  float l = 0.0f;
  float4 o[kMergeEach];
#pragma unroll
  for (int i = 0; i < kMergeEach; ++i) o[i] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  for (int p = 0;;) {
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (p + u >= pieces) break;
      const float f = fast_exp2(y[u].x - m);
      l = fmaf(y[u].y, f, l);
#pragma unroll
      for (int i = 0; i < kMergeEach; ++i) {
        o[i].x = fmaf(z[u][i].x, f, o[i].x);
        o[i].y = fmaf(z[u][i].y, f, o[i].y);
        o[i].z = fmaf(z[u][i].z, f, o[i].z);
        o[i].w = fmaf(z[u][i].w, f, o[i].w);
      }
    }
    p += 4;
    if (p >= pieces) break;
    load_ml(p);
    load_sums(p);
  }
  const int G = DENSE ? 1 : a.num_q_heads / a.num_kv_heads;
  const int c = cut.t * S::CT + col, j = c / G;
  if (j >= q.n) return;
  const float inv = l > 0.0f ? 1.0f / l : l == 0.0f ? 0.0f : l;   // (NaN stays)
  const size_t orow = (size_t)(q.q0 + j) * a.num_q_heads + a.head0 + cut.g * G + (c - j * G);
#pragma unroll
  for (int i = 0; i < kMergeEach; ++i) {
    uint2 w;
    w.x = pack2_bf16(o[i].x * inv, o[i].y * inv);
    w.y = pack2_bf16(o[i].z * inv, o[i].w * inv);
    *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.out) + orow * S::kDims + S::dim_of(i0 + i, lane)) = w;
  }
}

}  // namespace ra
}  // namespace bros
