// Attention of a few new rows of each sequence over its paged cache: drafted tokens over a
// K/V pool, queries in the latent space over a pool of latent rows, and causal chunks over
// keys and values expanded from latents. Shared by tree.hip and latent.hip.
//
// Columns. The G query heads that read one key make a column each of every new row, so a
// sequence has n G columns per KV head (a latent row is the key of all heads: n Hq
// columns). A unit is a (sequence, KV head, tile of 32 NCW columns); its keys come in steps of
// 32 NKW. A workgroup of NCW NKW H waves takes a step: wave (cw, kg, h) the columns 32 cw ..
// + 31 against the keys 32 kg .. + 31, and part h of H of the dims: of the score products, whose
// partial sums the H waves exchange in LDS, and of the values. (Long rows only: 576 dims of a query
// and 512 of sums in fp32 for 32 columns are 400 registers of a wave.)
//
// Products, transposed: S^T[key][column] = K Q^T and O^T[dim][column] += V^T P^T, both with
// 32x32x16 matrix instructions, so that a lane owns one column (lane % 32), the softmax needs
// one exchange between the two half-waves, and P goes from the score accumulators straight
// into the second product's operand (keys are permuted alike in P and V^T). K^T operands are
// 16-byte reads of LDS rows, V^T operands transposing reads; the chunks of a row are permuted
// (swz) so that neither meets a bank conflict. Rows reach LDS without registers.
//
// Work. The steps of all units are laid end to end and cut into equal shares, one per
// workgroup, whatever the sequences' lengths; a unit cut between workgroups leaves partial
// sums (fp32, with their maximum and total) that a merge folds.
//
// Masks. A row sees the keys before the drafts, and of those the ones its bits name (or the
// causal ones). Only steps that reach the drafts, the context's end or an invalid table
// entry look at masks: a row's 32 bits of the tile's positions. In such tiles a value that is
// not finite enters the product as zero (whatever a slot holds that some row does not see), and
// where it is seen, it is added to the finished rows that see it (rare).
#pragma once

#include "bros_device.h"
#include "bros_kernels.h"
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

constexpr int kKeys = 32;                // keys of a wave's tile
constexpr float kRescaleSlack = 8.0f;    // log2 units: weights stay <= 2^8
constexpr float kNoMax = -1.0e30f;       // finite "no score yet" reference
constexpr int kTable = 128;              // staged table entries of a wave: two windows of 64

typedef const v4u_t __attribute__((address_space(3)))* lds_v4u_ptr;
typedef short v4s_t __attribute__((ext_vector_type(4)));
typedef v4s_t __attribute__((address_space(3)))* lds_v4s_ptr;
__device__ __forceinline__ uint32_t lds_address(const void* p) { return (uint32_t)(uintptr_t)p; }   // (the aperture is 4 GiB aligned)
__device__ __forceinline__ v4u_t lds_read(uint32_t at) { return *(lds_v4u_ptr)(uintptr_t)at; }
__device__ __forceinline__ uint2 lds_read_turned(uint32_t at) {
  return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s_ptr)(uintptr_t)at));
}
// A word that a load into LDS may have written. (As LDS memory: a generic read would also wait for every load in flight.)
__device__ __forceinline__ int32_t lds_word(const int32_t* p) {
  return *(const volatile int32_t __attribute__((address_space(3)))*)(uintptr_t)lds_address(p);
}

// What is read. kMain: bytes of a key row's first part, kRot: of its second (0: none);
// kVal: bytes of a value row, or 0 where the first part is the value.
struct KvPool {          // 128 dims each, [blocks][Hkv][16][128]
  static constexpr int kMain = 256, kRot = 0, kVal = 256;
  static constexpr bool kPaged = true, kCausalUnits = false;
};
struct LatentPool {      // 512 shared dims and 64 rotated ones, [blocks][16][576]
  static constexpr int kMain = 1024, kRot = 128, kVal = 0;
  static constexpr bool kPaged = true, kCausalUnits = false;
};
struct Expanded {        // dense rows: keys of 128 dims and 64 rotated ones shared by the heads, values of 128
  static constexpr int kMain = 256, kRot = 128, kVal = 256;
  static constexpr bool kPaged = false, kCausalUnits = true;
};

// A sequence as the kernels see it. n = 0: nothing to do. ctx: its visible context
// (0 where lengths are inconsistent: its rows see nothing); c0: position of its first new row.
struct Seq {
  int q0, n, c0, ctx;
};
__device__ __forceinline__ Seq seq_of(const RowsArgs& a, int s) {
  Seq r;
  r.q0 = a.cu_q != nullptr ? a.cu_q[s] : s;
  const int end = a.cu_q != nullptr ? a.cu_q[s + 1] : s + 1;
  r.n = (r.q0 < 0 || end > a.num_q_tokens || end < r.q0) ? 0 : end - r.q0;
  const int ctx = a.ctx_lens[s];
  r.c0 = ctx - r.n;
  const int64_t room = (int64_t)a.max_blocks_per_seq * kBlockSize;
  r.ctx = r.c0 < 0 ? 0 : (int)min((int64_t)min(ctx, a.max_ctx), room);
  return r;
}

// Steps of a sequence's units. CT columns to a unit, KS keys to a step. Every unit has one
// at least: its rows are written even where they see nothing.
template <class P, int CT, int KS>
struct Steps {
  int tiles, each;   // units per KV head; steps of one (causal units: of the last)
  int before;        // causal units: steps of the keys before the new rows
  __device__ __forceinline__ Steps(const RowsArgs& a, const Seq& q, int group) {
    tiles = (int)(((int64_t)q.n * group + CT - 1) / CT);
    each = max(1, (q.ctx + KS - 1) / KS);
    before = (max(q.c0, 0) + KS - 1) / KS;
  }
  // Steps of unit t. Causal units (one column a row): those of its last row's keys.
  __device__ __forceinline__ int of(int t) const {
    if constexpr (P::kCausalUnits) return t + 1 < tiles ? min(before + (CT / KS) * (t + 1), each) : each;
    return each;
  }
  // Steps of units 0 .. t - 1 (t <= tiles).
  __device__ __forceinline__ int64_t first(int t) const {
    if constexpr (P::kCausalUnits) {
      int64_t sum = 0;
      // (the context may be cut short by max_ctx: units beyond it have `each` steps)
      const int free = min(t, min(tiles - 1, max(0, (each - before) / (CT / KS))));   // units whose `of` is not cut
      sum = (int64_t)free * before + (int64_t)(CT / KS) * free * (free + 1) / 2;
      return sum + (int64_t)(t - free) * each;
    }
    return (int64_t)t * each;
  }
  __device__ __forceinline__ int64_t per_head() const { return first(tiles); }
};

// The two blocks of a tile: whether their entries are valid, and their directions.
struct TileBlocks {
  bool ok0, ok1;
  int dir0, dir1;
};
// Bits 15 and 31: the halves that are infinite or NaN, as bf16.
__device__ __forceinline__ uint32_t not_finite(uint32_t w) { return ((w & 0x7f807f80u) + 0x00800080u) & 0x80008000u; }

// Bits of the positions pos0 .. + 31 that row j of a sequence sees, of a context of ctx.
__device__ __forceinline__ uint32_t row_window(const RowsArgs& a, const Seq& q, int ctx, int j, bool valid, int pos0) {
  const auto below = [](int k) -> uint32_t { return k >= 32 ? 0xffffffffu : k <= 0 ? 0u : (1u << k) - 1u; };
  uint32_t win;
  if (a.mask != nullptr) {
    const int i0 = pos0 - q.c0;   // draft of position pos0 (negative: before the drafts)
    win = below(-i0);
    const uint64_t* bits = a.mask + (size_t)(q.q0 + min(j, q.n - 1)) * a.mask_words;
    // the 64 bits from draft max(i0, 0) on
    const int f = max(i0, 0), wd = f >> 6, sh = f & 63;
    uint64_t b = wd < a.mask_words ? bits[wd] >> sh : 0;
    if (sh != 0 && wd + 1 < a.mask_words) b |= bits[wd + 1] << (64 - sh);
    if (q.n - f < 64) b &= q.n - f <= 0 ? 0 : (1ull << (q.n - f)) - 1;
    if (i0 > -32) win |= i0 < 0 ? (uint32_t)b << -i0 : (uint32_t)b;
  } else {
    win = below(q.c0 + j + 1 - pos0);
  }
  return valid ? win & below(ctx - pos0) : 0u;
}

// Where a workgroup's share begins.
struct Place {
  int s, g, t, step;
  int64_t total;        // steps of all units
  int64_t row0;         // dense keys: row of sequence s's position 0
};

__device__ __forceinline__ int64_t wave_scan64(int64_t v, int lane) {
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) {
    const int64_t u = __shfl_up(v, o);
    if (lane >= o) v += u;
  }
  return v;
}

// Rows that a sequence's keys take in the dense buffers: whole tiles.
__device__ __forceinline__ int dense_rows(int ctx) { return (ctx + kKeys - 1) / kKeys * kKeys; }

// The steps of all units, and the unit and step of number `at(total)` (at: a function of the
// total, the same for every thread; -1: no place wanted). All THREADS threads call it; `scratch` is 2 x (waves + 1) numbers of
// LDS and s_place a Place.
template <class P, int CT, int KS, int THREADS, class At>
__device__ __forceinline__ Place find_place(const RowsArgs& a, int group, At at, int64_t* scratch, Place* s_place) {
  constexpr int kW = THREADS / kWave;
  const int tid = threadIdx.x, lane = tid & (kWave - 1), w = tid / kWave;
  // a thread's run of sequences
  const int per = (a.num_seqs + THREADS - 1) / THREADS;
  const int s0 = min(tid * per, a.num_seqs), s1 = min(s0 + per, a.num_seqs);
  int64_t mine = 0, rows = 0;
  for (int s = s0; s < s1; ++s) {
    const Seq q = seq_of(a, s);
    const Steps<P, CT, KS> st(a, q, group);
    mine += st.per_head() * a.num_kv_heads;
    if constexpr (!P::kPaged) rows += dense_rows(q.ctx);
  }
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
  if (x >= first && x < first + mine) {
    int64_t left = x - first;
    for (int s = s0; s < s1; ++s) {
      const Seq q = seq_of(a, s);
      const Steps<P, CT, KS> st(a, q, group);
      const int64_t ph = st.per_head();
      if (left < ph * a.num_kv_heads) {
        Place p;
        p.s = s;
        p.g = (int)(left / ph);
        left -= p.g * ph;
        int lo = 0, hi = st.tiles - 1;   // the last unit that begins at or before it
        while (lo < hi) {
          const int mid = (lo + hi + 1) >> 1;
          if (st.first(mid) <= left) lo = mid; else hi = mid - 1;
        }
        p.t = lo;
        p.step = (int)(left - st.first(lo));
        p.total = total;
        p.row0 = rfirst;
        *s_place = p;
        break;
      }
      left -= ph * a.num_kv_heads;
      if constexpr (!P::kPaged) rfirst += dense_rows(q.ctx);
    }
  }
  __syncthreads();
  Place p = *s_place;
  p.s = __builtin_amdgcn_readfirstlane(p.s);
  p.g = __builtin_amdgcn_readfirstlane(p.g);
  p.t = __builtin_amdgcn_readfirstlane(p.t);
  p.step = __builtin_amdgcn_readfirstlane(p.step);
  p.total = total;
  return p;
}

// Workgroups that get a share of `total` steps, and where share w begins.
__device__ __forceinline__ int sharers(const RowsArgs& a, int64_t total) {
  return (int)max((int64_t)1, min((int64_t)a.workers, (total + a.min_steps - 1) / a.min_steps));
}
__device__ __forceinline__ int64_t share_begin(int64_t total, int w, int n) { return total * w / n; }
// The share that step x lies in.
__device__ __forceinline__ int share_of(int64_t total, int64_t x, int n) { return (int)(((x + 1) * n - 1) / total); }

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

template <class P, int NCW, int NKW, int H, int SLOTS>
struct Shape {
  static constexpr int kWaves = NCW * NKW * H, kThreads = kWaves * kWave;
  static constexpr int kSharers = NCW * H;                          // waves that share a tile
  static constexpr int CT = 32 * NCW, KS = kKeys * NKW;
  static constexpr int kDt = (P::kVal ? P::kVal : P::kMain) / 64;   // 32-dim pieces of a value
  static constexpr int kDims = 32 * kDt;
  static constexpr int kQDims = (P::kMain + P::kRot) / 2;
  static constexpr int kRotAt = kKeys * P::kMain;                   // LDS of a tile: first parts, second parts, values
  static constexpr int kValAt = kRotAt + kKeys * P::kRot;
  static constexpr int kTile = kValAt + kKeys * P::kVal;
  static constexpr int kRing = NKW * SLOTS * kTile;
  static constexpr int kRows = kKeys / kSharers;                    // rows of a tile that a wave loads
  // loads of a wave per step, 1 KiB each (second parts: eight rows, or fewer lanes)
  static constexpr int kLoads = (P::kVal ? 2 * kRows / 4 : kRows * P::kMain / 1024) + (P::kRot ? (kRows + 7) / 8 : 0);
  static constexpr int kExchange = H > 1 ? kWaves * 4096 : 16;      // score sums of a step
  static constexpr int kSlotFloats = CT * kDims;                    // a partial's sums
  static_assert(kRows % 4 == 0, "a load takes four rows of 256 bytes");
  static_assert(H == 1 || NKW == 1, "");
  static_assert(H > 1 || P::kVal != 0, "a shared row is cleaned behind the exchange's barrier");
  static_assert(kDt % H == 0 && (P::kMain / 32) % H == 0 && (P::kRot / 32) % H == 0, "");
  static_assert(H == 1 || (kDt / H) % 4 == 0, "a part starts at a multiple of 16 chunks");
  static_assert((NKW - 1) * NCW * 32 * kDims * 4 <= kRing, "the key groups' sums meet in the ring");
};

template <class P, int NCW, int NKW, int H, int SLOTS, int OCC>
__global__ __launch_bounds__(64 * NCW * NKW * H, OCC) void rows_kernel(RowsArgs a) {
  using S = Shape<P, NCW, NKW, H, SLOTS>;
  // of this wave: 32-dim pieces of its values, 16-dim steps of its score products
  constexpr int kDt = S::kDt / H, kMainSteps = P::kMain / 32 / H, kQSteps = kMainSteps + P::kRot / 32 / H;
  __shared__ __attribute__((aligned(16))) uint8_t s_x[S::kExchange];
  __shared__ __attribute__((aligned(1024))) uint8_t s_ring[S::kRing];
  __shared__ int32_t s_tab[S::kWaves][kTable];
  __shared__ int64_t s_scan[2 * S::kWaves];
  __shared__ Place s_place;
  __shared__ int s_odd;

  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = wave_id_uniform();
  const int cw = wave % NCW, kg = H > 1 ? 0 : wave / NCW, hp = H > 1 ? wave / NCW : 0;
  const int sharer = H > 1 ? wave : cw;   // among the waves of its tile
  const int half = lane >> 5, col = lane & 31;
  const int Hkv = a.num_kv_heads, G = P::kPaged ? a.num_q_heads / Hkv : 1;   // (expanded: heads of their own)
  // neighbouring shares to one die
  const int nb = gridDim.x;
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

  constexpr int kR = S::kRows;
  uint8_t* ring = s_ring + kg * SLOTS * S::kTile;
  int32_t* tab = s_tab[wave];
  const float sl2 = a.scale_log2;
  const bf16x2_t one2 = {(__bf16)1.0f, (__bf16)1.0f};

  // operand reads (see the top)
  const int k_sw = swz(col);
  const int k_lane = col * P::kMain + (((half ^ k_sw) & 1) << 4) + hp * (P::kMain / H);
  const int r_lane = (col >> 1) * 256 + ((col & 1) << 7), r_sw = ((col >> 1) & 7) ^ (hp * (P::kRot / 16 / H));
  constexpr int kVRow = P::kVal ? P::kVal : P::kMain, kVAt = P::kVal ? S::kValAt : 0;
  int v_off[2], v_sw[2];
#pragma unroll
  for (int part = 0; part < 2; ++part) {
    const int key = 8 * part + 4 * half + ((lane >> 2) & 3);
    v_sw[part] = swz(key);
    v_off[part] = key * kVRow + ((((2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ v_sw[part]) & 3) << 4) + (lane & 1) * 8 + hp * (kDt * 64);
  }

  while (x < x_end) {
    // ---- The segment: steps [first, first + cnt) of unit (s, g, t).
    const int s = at.s, g = at.g, t = at.t;
    const Seq q = seq_of(a, s);
    const Steps<P, S::CT, S::KS> st(a, q, G);
    const int usteps = __builtin_amdgcn_readfirstlane(st.of(t));
    const int first = at.step;
    const int cnt = (int)min((int64_t)(usteps - first), x_end - x);
    const bool whole = cnt == usteps;
    // (dense keys that do not fit their buffer: the sequence's rows see nothing)
    const bool fits = P::kPaged || at.row0 + dense_rows(q.ctx) <= a.dense_rows;
    const int ctx = fits ? q.ctx : 0, n = q.n;
    const int nblk = (ctx + kBlockSize - 1) / kBlockSize;
    const int c = t * S::CT + 32 * cw + col;        // the lane's column
    const int j = c / G;                            // its row
    const bool valid = j < n;
    const size_t orow = (size_t)(q.q0 + min(j, n - 1)) * a.num_q_heads + a.head0 + g * G + (c - j * G);
    // keys below this position are seen by every row of the unit
    const int full_below = a.mask != nullptr ? min(ctx, q.c0) : min(ctx, q.c0 + t * S::CT / G + 1);

    bf16x8_t qf[kQSteps];
    {
      const uint16_t* qp = static_cast<const uint16_t*>(a.q) + orow * S::kQDims + 8 * half;
#pragma unroll
      for (int i = 0; i < kQSteps; ++i) {
        v4u_t v = {0, 0, 0, 0};
        const int d = i < kMainSteps ? 16 * (hp * kMainSteps + i) : P::kMain / 2 + 16 * (hp * (kQSteps - kMainSteps) + i - kMainSteps);
        if (valid) v = *reinterpret_cast<const v4u_t*>(qp + d);
        qf[i] = as_bf16x8(v);
      }
    }

    // Table entries: a wave keeps two windows of 64 in LDS; the next is requested when the loads
    // enter the one before it.
    const int32_t* tbl = a.block_tables + (size_t)s * a.max_blocks_per_seq;
    auto load_window = [&](int e0) __attribute__((always_inline)) {   // e0: a multiple of 64
      const int e = max(0, min(e0 + lane, nblk - 1));
      load_word_to_lds(tbl, 4u * (uint32_t)e, tab + (e0 & (kTable - 1)));
    };
    auto entry = [&](int e) __attribute__((always_inline)) -> int {   // -1: none
      const int v = __builtin_amdgcn_readfirstlane(lds_word(tab + (e & (kTable - 1))));
      return (e < nblk && v >= 0 && v < a.num_blocks) ? v : -1;
    };
    // Requests the wave's part of the rows of step `step`; whether a block of them is missing.
    auto issue = [&](int step) __attribute__((always_inline)) -> bool {
      const int e = 2 * (step * NKW + kg);
      uint8_t* dst = ring + (step % SLOTS) * S::kTile;
      if ((e & 63) < 2 * NKW && step > first) load_window((e & ~63) + 64);
      const int b0 = entry(e), b1 = entry(e + 1);
      bool gone = b0 < 0 || b1 < 0;
      if constexpr (P::kPaged) {
        if constexpr (NCW > 1 && NKW > 1) {   // (the workgroup's waves meet at the step's barriers: all look at all its entries)
#pragma unroll
          for (int i = 2; i < 2 * NKW; ++i) gone |= entry((e - 2 * kg) + (2 * kg + i) % (2 * NKW)) < 0;
        }
        if constexpr (P::kVal != 0) {
#pragma unroll
          for (int i = 0; i < kR / 4; ++i) {
            const int row = kR * sharer + 4 * i;   // its first of four
            const size_t at_row = ((size_t)max((row >> 4) ? b1 : b0, 0) * Hkv + g) * (kBlockSize * P::kMain) + (row & 15) * P::kMain;
            const int r = row + (lane >> 4);
            const uint32_t off = (uint32_t)((lane >> 4) * P::kMain + (((lane & 15) ^ swz(r)) << 4));
            load_to_lds(static_cast<const uint8_t*>(a.k_pool) + at_row, off, dst + row * P::kMain);
            load_to_lds(static_cast<const uint8_t*>(a.v_pool) + at_row, off, dst + S::kValAt + row * P::kVal);
          }
        } else {
          constexpr int kRow = P::kMain + P::kRot;
#pragma unroll
          for (int i = 0; i < kR; ++i) {
            const int row = kR * sharer + i;
            const uint8_t* src = static_cast<const uint8_t*>(a.k_pool) +
                                 ((size_t)max((row >> 4) ? b1 : b0, 0) * kBlockSize + (row & 15)) * kRow;
            load_to_lds(src, (uint32_t)((lane ^ swz(row)) << 4), dst + row * P::kMain);
          }
#pragma unroll
          for (int i = 0; i < (kR + 7) / 8; ++i) {   // second parts, eight rows at once
            const int row = kR * sharer + 8 * i;
            const uint8_t* src = static_cast<const uint8_t*>(a.k_pool) +
                                 ((size_t)max((row >> 4) ? b1 : b0, 0) * kBlockSize + (row & 15)) * kRow + P::kMain;
            const int r = row + (lane >> 3);
            if (kR >= 8 || lane < 8 * kR)
              load_to_lds(src, (uint32_t)((lane >> 3) * kRow + (((lane & 7) ^ ((r >> 1) & 7)) << 4)),
                          dst + S::kRotAt + row * P::kRot);
          }
        }
      } else {
        const size_t row0 = fits ? (size_t)(at.row0 + (int64_t)step * S::KS + kKeys * kg) : 0;
        const size_t head = ((size_t)g * a.dense_rows + row0) * P::kMain;
#pragma unroll
        for (int i = 0; i < kR / 4; ++i) {
          const int row = kR * sharer + 4 * i, r = row + (lane >> 4);
          const uint32_t off = (uint32_t)((lane >> 4) * P::kMain + (((lane & 15) ^ swz(r)) << 4));
          load_to_lds(static_cast<const uint8_t*>(a.k_pool) + head + row * P::kMain, off, dst + row * P::kMain);
          load_to_lds(static_cast<const uint8_t*>(a.v_pool) + head + row * P::kMain, off, dst + S::kValAt + row * P::kVal);
        }
#pragma unroll
        for (int i = 0; i < kR / 8; ++i) {
          const int row = kR * sharer + 8 * i, r = row + (lane >> 3);
          load_to_lds(static_cast<const uint8_t*>(a.rot_rows) + (row0 + row) * P::kRot,
                      (uint32_t)((lane >> 3) * P::kRot + (((lane & 7) ^ ((r >> 1) & 7)) << 4)), dst + S::kRotAt + row * P::kRot);
        }
      }
      return gone;
    };

    floatx16 o[kDt];
#pragma unroll
    for (int i = 0; i < kDt; ++i) o[i] = floatx16{};
    float m_run = kNoMax, l0 = 0.0f, l1 = 0.0f;
    uint32_t odd = 0;   // a value that is not finite was left out of a product

    // The two blocks of the tile at pos0: whether they are there, and their directions.
    auto blocks_of = [&](int pos0) -> TileBlocks {
      const int e = pos0 / kBlockSize, em = max(nblk - 1, 0);
      const int v0 = tbl[min(e, em)], v1 = tbl[min(e + 1, em)];
      const bool ok0 = e < nblk && v0 >= 0 && v0 < a.num_blocks, ok1 = e + 1 < nblk && v1 >= 0 && v1 < a.num_blocks;
      if constexpr (!P::kPaged) return TileBlocks{ok0, ok1, 1, 1};   // (dense rows lie in the order of their positions)
      return TileBlocks{ok0, ok1, entry_direction(a.dir, a.cls, a.dir_per_entry, a.max_blocks_per_seq, s, min(e, em)),
                        entry_direction(a.dir, a.cls, a.dir_per_entry, a.max_blocks_per_seq, s, min(e + 1, em))};
    };

    // ---- Start: the first windows of the table, then the first SLOTS - 1 steps' rows.
    __syncthreads();   // (the ring's last use: the segment before this one)
    if (tid == 0) s_odd = 0;
    __syncthreads();
    {
      const int e = 2 * (first * NKW + kg) & ~63;
      load_window(e);
      load_window(e + 64);
    }
    __builtin_amdgcn_s_waitcnt(0x0F70);   // vmcnt(0): a wait the compiler sees, q's included
    asm volatile("" ::: "memory");
    uint32_t missing = 0;   // bit step % 32: a block of that step is missing
    const int last = first + cnt;
    auto request = [&](int step) __attribute__((always_inline)) {
      const bool gone = issue(step);
      missing = (missing & ~(1u << (step & 31))) | ((gone ? 1u : 0u) << (step & 31));
    };
#pragma unroll
    for (int i = 0; i < SLOTS - 1; ++i)
      if (first + i < last) request(first + i);

    for (int step = first; step < last; ++step) {
      // ---- This step's rows are in LDS (all waves'), and every wave is past the step before.
      const int ahead = min(SLOTS - 2, last - 1 - step);   // later steps still in flight
      if (ahead >= 2) wait_vmem<(2 * S::kLoads < 63 ? 2 * S::kLoads : 63)>();
      else if (ahead == 1) wait_vmem<S::kLoads>();
      else wait_vmem<0>();
      if constexpr (S::kSharers > 1) lds_barrier();
      else asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // (a wave's own rows: the step before is read out)
      if (step + SLOTS - 1 < last) request(step + SLOTS - 1);
      uint8_t* tile = ring + (step % SLOTS) * S::kTile;
      const int pos0 = step * S::KS + kKeys * kg;            // first position of this wave's tile
      const bool hole = (missing >> (step & 31)) & 1;
      const bool masked = hole || pos0 + kKeys > full_below;
      uint32_t win = 0xffffffffu;
      TileBlocks tb{true, true, 1, 1};
      if (masked) {
        win = row_window(a, q, ctx, j, valid, pos0);
        tb = blocks_of(pos0);
      }
      // The wave's rows of values: zeros where no context is, and for values that are not finite.
      // Then the waves that share the tile meet (the condition is the same for all of the workgroup).
      const auto clean = [&]() __attribute__((always_inline)) {
        if (masked) {
          constexpr int kChunks = kVRow / 16;
          for (int i = lane; i < kR * kChunks; i += kWave) {
            const int r = kR * sharer + i / kChunks;
            const int pos = pos0 + (r & 16) + slot_of_offset(r & 15, r < 16 ? tb.dir0 : tb.dir1);
            v4u_t* at_v = reinterpret_cast<v4u_t*>(tile + kVAt + r * kVRow) + i % kChunks;
            if (!((r < 16 ? tb.ok0 : tb.ok1) && pos < ctx)) {
              *at_v = v4u_t{0, 0, 0, 0};
              continue;
            }
            v4u_t w = *at_v;
            uint32_t any = 0;
  #pragma unroll
            for (int e = 0; e < 4; ++e) {
              const uint32_t bad = not_finite(w[e]);
              any |= bad;
              w[e] &= ~((bad >> 15) * 0xffffu);
            }
            if (any != 0) *at_v = w;
            odd |= any;
          }
        }
        if (S::kSharers > 1 && (hole || (step + 1) * S::KS > full_below)) lds_barrier();
      };
      if constexpr (P::kVal != 0) clean();

      // ---- Scores.
      floatx16 cur;
#pragma unroll
      for (int i = 0; i < kQSteps; ++i) {
        const uint8_t* src = i < kMainSteps ? tile + k_lane + (((2 * i) ^ (k_sw & 14)) << 4)
                                            : tile + S::kRotAt + r_lane + (((2 * (i - kMainSteps) + half) ^ r_sw) << 4);
        const v4u_t kv = *reinterpret_cast<const v4u_t*>(src);
        cur = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(kv), qf[i], i == 0 ? floatx16{} : cur, 0, 0, 0);
      }
      if constexpr (H > 1) {   // the other parts' sums
        float4* mine = reinterpret_cast<float4*>(s_x) + wave * 4 * kWave + lane;
#pragma unroll
        for (int i = 0; i < 4; ++i) mine[i * kWave] = make_float4(cur[4 * i], cur[4 * i + 1], cur[4 * i + 2], cur[4 * i + 3]);
        lds_barrier();
        // ((0 + 1) + (2 + 3), whichever part adds: the waves of a column must hold the same scores)
        const auto part = [&](int k, int i) { return (reinterpret_cast<const float4*>(s_x) + ((hp ^ k) * NCW + cw) * 4 * kWave + lane)[i * kWave]; };
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float4 y = part(1, i), z = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
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
      if constexpr (P::kVal == 0) clean();   // (the scores have been taken from the rows as they are)
      if (masked) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int k = 8 * (i >> 2) + 4 * half + (i & 3);
          const int off = (k & 16) + slot_of_offset(k & 15, (i >> 3) ? tb.dir1 : tb.dir0);
          cur[i] = ((i >> 3) ? tb.ok1 : tb.ok0) && ((win >> off) & 1u) ? cur[i] : -INFINITY;
        }
      }
      // ---- Running maximum (moved lazily) and weights, rounded to bf16 for the second
      // product; the totals add the rounded weights.
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

      // ---- Values.
      const uint8_t* vt = tile + kVAt;
      const auto values = [&](int c2, int dt) __attribute__((always_inline)) -> v4u_t {
        const uint2 x0 = lds_read_tr(vt + 16 * c2 * kVRow + v_off[0] + (((4 * dt) ^ (v_sw[0] & 12)) << 4));
        const uint2 x1 = lds_read_tr(vt + 16 * c2 * kVRow + v_off[1] + (((4 * dt) ^ (v_sw[1] & 12)) << 4));
        return v4u_t{x0.x, x0.y, x1.x, x1.y};
      };
#pragma unroll
      for (int c2 = 0; c2 < 2; ++c2) {
#pragma unroll
        for (int dt = 0; dt < kDt; ++dt)
          o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(values(c2, dt)), pfr[c2], o[dt], 0, 0, 0);
      }
    }

    // ---- The end of the segment.
    float l = pair_sum(l0 + l1);
    if (odd != 0) s_odd = 1;
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
            xo[(w * kDt * 4 + 4 * i + jq) * kWave + lane] = make_float4(o[i][4 * jq], o[i][4 * jq + 1], o[i][4 * jq + 2], o[i][4 * jq + 3]);
        }
        if (half == 0) {
          s_ml[2 * (w * 32 + col)] = m_run;
          s_ml[2 * (w * 32 + col) + 1] = l;
        }
      }
      __syncthreads();
      if (kg == 0) {
#pragma unroll 1
        for (int k = 1; k < NKW; ++k) {
          const int w = (k - 1) * NCW + cw;
          const float m2 = s_ml[2 * (w * 32 + col)], l2 = s_ml[2 * (w * 32 + col) + 1];
          const float m = fmaxf(m_run, m2);
          const float f1 = fast_exp2(m_run - m), f2 = fast_exp2(m2 - m);
          m_run = m;
          l = l * f1 + l2 * f2;
#pragma unroll
          for (int i = 0; i < kDt; ++i) {
#pragma unroll
            for (int jq = 0; jq < 4; ++jq) {
              const float4 y = xo[(w * kDt * 4 + 4 * i + jq) * kWave + lane];
              o[i][4 * jq] = o[i][4 * jq] * f1 + y.x * f2;
              o[i][4 * jq + 1] = o[i][4 * jq + 1] * f1 + y.y * f2;
              o[i][4 * jq + 2] = o[i][4 * jq + 2] * f1 + y.z * f2;
              o[i][4 * jq + 3] = o[i][4 * jq + 3] * f1 + y.w * f2;
            }
          }
        }
      }
    }
    if (kg == 0) {
      if (whole) {
        const float inv = l > 0.0f ? 1.0f / l : l < 0.0f ? 0.0f : l == 0.0f ? 0.0f : l;   // (NaN stays)
        if (valid) write_columns<kDt>(static_cast<uint16_t*>(a.out) + orow * S::kDims, hp * kDt, o, inv, half);
      } else {
        // the accumulators as they lie: every store of the wave is 1 KiB contiguous
        const size_t slot = 2 * (size_t)me + (first == 0 ? 1 : 0);
        float4* po = reinterpret_cast<float4*>(a.ws_o + slot * S::kSlotFloats) + (cw * S::kDt + hp * kDt) * 4 * kWave + lane;
#pragma unroll
        for (int i = 0; i < kDt; ++i) {
#pragma unroll
          for (int jq = 0; jq < 4; ++jq)
            po[(4 * i + jq) * kWave] = make_float4(o[i][4 * jq], o[i][4 * jq + 1], o[i][4 * jq + 2], o[i][4 * jq + 3]);
        }
        if (half == 0 && hp == 0) {
          float* ml = a.ws_ml + (slot * S::CT + 32 * cw + col) * 2;
          ml[0] = m_run;
          ml[1] = l;
        }
      }
    }

    // ---- Values that were left out and are seen: added to the rows that see them, where
    // those now lie. (Every key of the segment's masked tiles is looked at again, in memory.)
    if (kg == 0 && s_odd != 0) {
      const int tiles = cnt * NKW;
#pragma unroll 1
      for (int ti = 0; ti < tiles; ++ti) {
        const int pos0 = first * S::KS + kKeys * ti;
        TileBlocks tb{true, true, 1, 1};
        tb = blocks_of(pos0);
        bool hole = !tb.ok0 || !tb.ok1;
        if constexpr (NCW > 1 && NKW > 1) {
          for (int k = 0; k < NKW; ++k) {
            const TileBlocks other = blocks_of((pos0 / S::KS) * S::KS + kKeys * k);
            hole |= !other.ok0 || !other.ok1;
          }
        }
        if (pos0 + kKeys <= full_below && !hole) continue;
        const uint32_t win = row_window(a, q, ctx, j, valid, pos0);
        // value row of tile row r, or null where no context is
        const auto value_row = [&](int r) -> const uint8_t* {
          if constexpr (P::kPaged) {
            const int pos = pos0 + (r & 16) + slot_of_offset(r & 15, r < 16 ? tb.dir0 : tb.dir1);
            if (!(r < 16 ? tb.ok0 : tb.ok1) || pos >= ctx) return nullptr;
            const size_t slot = ((size_t)tbl[pos / kBlockSize] * Hkv + g) * kBlockSize + (r & 15);
            if constexpr (P::kVal != 0) return static_cast<const uint8_t*>(a.v_pool) + slot * P::kVal;
            return static_cast<const uint8_t*>(a.k_pool) + slot * (P::kMain + P::kRot);
          }
          if (!(r < 16 ? tb.ok0 : tb.ok1) || pos0 + r >= ctx) return nullptr;
          return static_cast<const uint8_t*>(a.v_pool) + ((size_t)g * a.dense_rows + at.row0 + pos0 + r) * P::kMain;
        };
        uint32_t any = 0;
        for (int i = lane; i < kKeys * (kVRow / 16); i += kWave) {
          const uint8_t* row = value_row(i / (kVRow / 16));
          if (row == nullptr) continue;
          const v4u_t w = *reinterpret_cast<const v4u_t*>(row + 16 * (i % (kVRow / 16)));
          any |= not_finite(w[0]) | not_finite(w[1]) | not_finite(w[2]) | not_finite(w[3]);
        }
        if (__builtin_amdgcn_ballot_w64(any != 0) == 0) continue;
#pragma unroll 1
        for (int r = 0; r < kKeys; ++r) {
          const uint8_t* row = value_row(r);
          if (row == nullptr) continue;
          const int off = P::kPaged ? (r & 16) + slot_of_offset(r & 15, r < 16 ? tb.dir0 : tb.dir1) : r;
          if (!((win >> off) & 1u)) continue;
#pragma unroll 1
          for (int i = 0; i < 4 * kDt; ++i) {
            const int d = 32 * hp * kDt + 8 * i + 4 * half;   // four dims
            const uint2 w = *reinterpret_cast<const uint2*>(row + 2 * d);
            if ((not_finite(w.x) | not_finite(w.y)) == 0) continue;
            const float v[4] = {bf16_lo(w.x), bf16_hi(w.x), bf16_lo(w.y), bf16_hi(w.y)};
            if (whole) {
              uint2* at_out = reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.out) + orow * S::kDims + d);
              uint2 y = *at_out;
              float x[4] = {bf16_lo(y.x), bf16_hi(y.x), bf16_lo(y.y), bf16_hi(y.y)};
#pragma unroll
              for (int e = 0; e < 4; ++e) x[e] = fabsf(v[e]) < INFINITY ? x[e] : x[e] + v[e];
              *at_out = make_uint2(pack2_bf16(x[0], x[1]), pack2_bf16(x[2], x[3]));
            } else {
              float* at_ws = a.ws_o + (2 * (size_t)me + (first == 0 ? 1 : 0)) * S::kSlotFloats +
                             ((cw * S::kDt + hp * kDt) * 4 + i) * (4 * kWave) + 4 * lane;
#pragma unroll
              for (int e = 0; e < 4; ++e)
                if (!(fabsf(v[e]) < INFINITY)) at_ws[e] += v[e];
            }
          }
        }
      }
    }

    // ---- The next unit.
    x += cnt;
    at.step = 0;
    if (x < x_end) {
      if (++at.t >= st.tiles) {
        at.t = 0;
        if (++at.g >= Hkv) {
          at.g = 0;
          do {
            if constexpr (!P::kPaged) at.row0 += dense_rows(seq_of(a, at.s).ctx);
            ++at.s;
          } while (seq_of(a, at.s).n <= 0);   // (steps are left, so a sequence with rows follows)
        }
      }
    }
  }
}

// Folds the partials of the units cut between shares: workgroup (w, cw) those of the unit in
// which share w's end is the first cut. Four waves, each a quarter of the value's dims.
template <class P, int NCW, int NKW, int H, int SLOTS>
__global__ __launch_bounds__(256) void rows_merge_kernel(RowsArgs a) {
  using S = Shape<P, NCW, NKW, H, SLOTS>;
  constexpr int kPer = S::kDt / 4;   // 32-dim pieces of a wave
  __shared__ int64_t s_scan[2 * 4];
  __shared__ Place s_place;
  const int G = P::kPaged ? a.num_q_heads / a.num_kv_heads : 1;
  const int w0 = blockIdx.x, cw = blockIdx.y;
  const int lane = threadIdx.x & (kWave - 1), wave = wave_id_uniform(), half = lane >> 5, col = lane & 31;
  const Place at = find_place<P, S::CT, S::KS, 256>(
      a, G, [&](int64_t total) -> int64_t {
        const int n = sharers(a, total);
        return w0 + 1 < n ? share_begin(total, w0 + 1, n) : -1;
      }, s_scan, &s_place);
  if (at.s < 0 || at.step == 0) return;
  const int n = sharers(a, at.total);
  const int64_t x = share_begin(at.total, w0 + 1, n), begin = x - at.step;
  if (share_begin(at.total, w0, n) > begin) return;   // an earlier share's end cuts this unit too
  const Seq q = seq_of(a, at.s);
  const Steps<P, S::CT, S::KS> st(a, q, G);
  const int w1 = share_of(at.total, begin + st.of(at.t) - 1, n);

  const int c = at.t * S::CT + 32 * cw + col, j = c / G;
  floatx16 o[kPer];
#pragma unroll
  for (int i = 0; i < kPer; ++i) o[i] = floatx16{};
  float m = kNoMax, l = 0.0f;
  for (int w = w0; w <= w1; ++w) {
    const size_t slot = 2 * (size_t)w + (w == w0 ? 1 : 0);
    const float4* po = reinterpret_cast<const float4*>(a.ws_o + slot * S::kSlotFloats) + (cw * S::kDt + wave * kPer) * 4 * kWave + lane;
    const float* ml = a.ws_ml + (slot * S::CT + 32 * cw + col) * 2;
    const float m2 = ml[0], l2 = ml[1];
    const float mn = fmaxf(m, m2), f1 = fast_exp2(m - mn), f2 = fast_exp2(m2 - mn);
    m = mn;
    l = l * f1 + l2 * f2;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
#pragma unroll
      for (int jq = 0; jq < 4; ++jq) {
        const float4 y = po[(4 * i + jq) * kWave];
        o[i][4 * jq] = o[i][4 * jq] * f1 + y.x * f2;
        o[i][4 * jq + 1] = o[i][4 * jq + 1] * f1 + y.y * f2;
        o[i][4 * jq + 2] = o[i][4 * jq + 2] * f1 + y.z * f2;
        o[i][4 * jq + 3] = o[i][4 * jq + 3] * f1 + y.w * f2;
      }
    }
  }
  if (j >= q.n) return;
  const float inv = l > 0.0f ? 1.0f / l : l == 0.0f ? 0.0f : l;
  const size_t orow = (size_t)(q.q0 + j) * a.num_q_heads + a.head0 + at.g * G + (c - j * G);
  write_columns<kPer>(static_cast<uint16_t*>(a.out) + orow * S::kDims, wave * kPer, o, inv, half);
}

}  // namespace ra
}  // namespace bros
