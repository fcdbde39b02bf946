// A cache of one latent vector per token on gfx950: bros_latent_append, bros_attn_latent
// (absorbed form) and bros_attn_latent_prefill (expanded form).
//
// A slot's row is 512 values of the latent vector c, which every head reads as key and value,
// and 64 of a rotated key. Absorbed: a query brought into the latent space meets c itself,
// 2 (576 + 512) operations a (key, column) for 1152 bytes a key: 16 columns are bound by
// memory, 128 by memory and matrix cores alike. Expanded: each head's 128 key and 128
// value dims are made from c once (2 * 512 * 256 operations a key and head) and then cost
// 2 (192 + 128) a (key, row, head): less from about 170 rows a context on.
#include "plan.h"
#include "rows_launch.h"

namespace bros {
namespace {

constexpr int kThreads = 256;
constexpr int kRot = 64, kLatent = 512, kRow = kLatent + kRot;

// ---------------------------------------------------------------------------
// append
// ---------------------------------------------------------------------------

// Rows of one kind to a workgroup: kTokens latent rows, a wave each, or kHeads query rows of 64 (several times as many where
// there are enough), four lanes each. One pass, bound by bytes: 6000 tokens of 128 heads, 253 MB, 63 us (4.0 TB/s of the 4.93
// that a copy reaches); a decode step of 64 tokens and 32 heads is all start and end, 4.3 us.
constexpr int kTokens = kThreads / kWave;
constexpr int kHeads = kThreads / 4;

__device__ __forceinline__ int axis_of(const LatentAppendArgs& a, int pair) {
  return (pair >= a.axis_end[0]) + (pair >= a.axis_end[1]) + (pair >= a.axis_end[2]);
}

// Sixteen dims of a rotated row, its pairs 8 l .. 8 l + 7 (l = 0 .. 3): the two chunks they lie in.
__device__ __forceinline__ int chunk_a(bool adjacent, int l) { return adjacent ? 2 * l : l; }
__device__ __forceinline__ int chunk_b(bool adjacent, int l) { return adjacent ? 2 * l + 1 : l + 4; }

__device__ __forceinline__ void widen8(const uint4& w, float (&x)[8]) {
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = bf16_lo(u[i]);
    x[2 * i + 1] = bf16_hi(u[i]);
  }
}
__device__ __forceinline__ uint4 narrow8(const float (&x)[8]) {   // the one rounding of a row's values
  return make_uint4(pf::pack2_bf16(x[0], x[1]), pf::pack2_bf16(x[2], x[3]), pf::pack2_bf16(x[4], x[5]), pf::pack2_bf16(x[6], x[7]));
}

// Cosines and sines of pairs 8 l .. + 7 of token t at logical position pos. (Positions outside the table: row 0; the
// caller drops them.)
__device__ __forceinline__ void angles(const LatentAppendArgs& a, int t, int pos, int l, float (&c)[8], float (&s)[8]) {
  const auto row_of = [&](int32_t at) -> const float* { return a.rope_table + (size_t)(at < 0 || at >= a.table_rows ? 0 : at) * kRot + 8 * l; };
  if (a.rope_pos == nullptr || a.axes == 1) {   // one row of the table
    const float4* row = reinterpret_cast<const float4*>(row_of(a.rope_pos == nullptr ? pos : a.rope_pos[t]));
    const float4 x[4] = {row[0], row[1], row[kRot / 8], row[kRot / 8 + 1]};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      c[4 * i] = x[i].x, c[4 * i + 1] = x[i].y, c[4 * i + 2] = x[i].z, c[4 * i + 3] = x[i].w;
      s[4 * i] = x[2 + i].x, s[4 * i + 1] = x[2 + i].y, s[4 * i + 2] = x[2 + i].z, s[4 * i + 3] = x[2 + i].w;
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float* row = row_of(a.rope_pos[(size_t)axis_of(a, 8 * l + i) * a.num_new_tokens + t]);
    c[i] = row[i];
    s[i] = row[kRot / 2 + i];
  }
}
// Turns those pairs.
template <bool ADJ>
__device__ __forceinline__ void turn(const float (&c)[8], const float (&s)[8], float (&xa)[8], float (&xb)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float& u = ADJ ? (i < 4 ? xa[2 * (i & 3)] : xb[2 * (i & 3)]) : xa[i];
    float& v = ADJ ? (i < 4 ? xa[2 * (i & 3) + 1] : xb[2 * (i & 3) + 1]) : xb[i];
    const float u0 = u, v0 = v;
    u = fmaf(u0, c[i], -(v0 * s[i]));
    v = fmaf(v0, c[i], u0 * s[i]);
  }
}
// Whether token t's position lies outside the table.
__device__ __forceinline__ bool outside(const LatentAppendArgs& a, int t, int pos) {
  if (a.rope_table == nullptr) return false;
  if (a.rope_pos == nullptr) return pos < 0 || pos >= a.table_rows;
  bool off = false;
  for (int x = 0; x < a.axes; ++x) {
    const int r = a.rope_pos[(size_t)x * a.num_new_tokens + t];
    off |= r < 0 || r >= a.table_rows;
  }
  return off;
}

// ADJ: pairs (2 i, 2 i + 1) instead of (i, i + 32). EACH: query rows of a thread; those of one token share its angles.
template <bool ADJ, int EACH>
__global__ __launch_bounds__(kThreads) void latent_append_kernel(LatentAppendArgs a, int kv_groups) {
  constexpr int kItems = kHeads * EACH;
  __shared__ int s_seq[kItems], s_pos[kItems];
  const int tid = threadIdx.x;
  const bool kv = (int)blockIdx.x < kv_groups;
  // the workgroup's tokens t0 .. t0 + n_tok - 1
  int t0, n_tok, h0 = 0;
  if (kv) {
    t0 = blockIdx.x * kTokens;
    n_tok = min(kTokens, a.num_new_tokens - t0);
  } else {
    const int64_t item0 = (int64_t)(blockIdx.x - kv_groups) * kItems;
    t0 = (int)(item0 / a.num_q_heads);
    h0 = (int)(item0 - (int64_t)t0 * a.num_q_heads);
    n_tok = min((h0 + kItems - 1) / a.num_q_heads + 1, a.num_new_tokens - t0);
  }
  // this thread's rows, requested before their positions are known
  const int lane = tid & (kWave - 1), l = kv ? lane & 3 : tid & 3;
  const int t = t0 + tid / kWave;                // of a latent row
  int tq[EACH], hq[EACH];                        // of query rows (tq: behind t0)
  bool live[EACH];
  uint4 w0{}, w1[EACH] = {}, w2[EACH] = {};
  if (kv) {
    live[0] = t < a.num_new_tokens;
    tq[0] = t - t0;
    const uint4* row = reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.kv) + (size_t)min(t, a.num_new_tokens - 1) * a.kv_stride);
    w0 = row[lane];
    w1[0] = row[kLatent / 8 + chunk_a(ADJ, l)];
    w2[0] = row[kLatent / 8 + chunk_b(ADJ, l)];
  } else {
#pragma unroll
    for (int r = 0; r < EACH; ++r) {
      const int item = h0 + kHeads * r + tid / 4;
      tq[r] = item / a.num_q_heads;
      hq[r] = item - tq[r] * a.num_q_heads;
      live[r] = tq[r] < n_tok;
      const uint4* row = reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.q) + (size_t)(t0 + min(tq[r], n_tok - 1)) * a.q_stride +
                                                        (size_t)hq[r] * a.q_head_stride);
      w1[r] = row[chunk_a(ADJ, l)];
      w2[r] = row[chunk_b(ADJ, l)];
    }
  }
#pragma unroll
  for (int r = 0; r < EACH; ++r) s_seq[kHeads * r + (tid & (kHeads - 1))] = -1;
  __syncthreads();
  for (int j = tid; j < a.num_seqs; j += kThreads) {
    const int lo = a.cu_new[j], hi = a.cu_new[j + 1], p0 = a.pos0[j];
    const int k0 = max(lo, t0), k1 = min(hi, t0 + n_tok);
    for (int k = k0; k < k1; ++k) {
      s_seq[k - t0] = j;
      s_pos[k - t0] = p0 + (k - lo);
    }
  }
  __syncthreads();
  float xa[8], xb[8], c[8], s[8];
  if (!kv) {
    int last = -1;
    bool off = false;
#pragma unroll
    for (int r = 0; r < EACH; ++r) {
      if (!live[r] || s_seq[tq[r]] < 0) continue;   // (in no sequence: left as it was)
      const int tr = t0 + tq[r];
      if (tq[r] != last) {
        off = outside(a, tr, s_pos[tq[r]]);
        if (a.rope_table != nullptr) angles(a, tr, s_pos[tq[r]], l, c, s);
        last = tq[r];
      }
      if (a.rope_table != nullptr) {
        widen8(w1[r], xa);
        widen8(w2[r], xb);
        turn<ADJ>(c, s, xa, xb);
        w1[r] = off ? make_uint4(0, 0, 0, 0) : narrow8(xa);
        w2[r] = off ? make_uint4(0, 0, 0, 0) : narrow8(xb);
      }
      uint4* row = reinterpret_cast<uint4*>(static_cast<uint16_t*>(a.q_out) + (size_t)tr * a.out_stride + (size_t)hq[r] * a.out_head_stride);
      row[chunk_a(ADJ, l)] = w1[r];
      row[chunk_b(ADJ, l)] = w2[r];
    }
    return;
  }
  const int seq = live[0] ? s_seq[t - t0] : -1;
  if (seq < 0) return;   // (uniform in a wave)
  const int pos = s_pos[t - t0];
  const bool off = outside(a, t, pos);
  // the latent's norm: every lane of the wave takes part
  if (a.norm != nullptr) {
    float x[8], g[8];
    widen8(w0, x);
    float ss = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) ss = fmaf(x[i], x[i], ss);
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) ss += __shfl_xor(ss, o);
    const float r = rsqrtf(ss * (1.0f / kLatent) + a.eps);
    widen8(reinterpret_cast<const uint4*>(a.norm)[lane], g);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = x[i] * r * g[i];
    w0 = narrow8(x);
  }
  if (off || pos < 0 || (pos >> 4) >= a.max_blocks_per_seq) return;
  const int b = a.block_tables[(size_t)seq * a.max_blocks_per_seq + (pos >> 4)];
  if (b < 0 || b >= a.num_blocks) return;
  const int slot = slot_of_offset(pos & 15, entry_direction(a.dir, a.cls, a.dir_per_entry, a.max_blocks_per_seq, seq, pos >> 4));
  uint4* row = reinterpret_cast<uint4*>(static_cast<uint16_t*>(a.pool) + ((size_t)b * kBlockSize + slot) * kRow);
  row[lane] = w0;
  if (lane < 4) {
    if (a.rope_table != nullptr) {
      angles(a, t, pos, lane, c, s);
      widen8(w1[0], xa);
      widen8(w2[0], xb);
      turn<ADJ>(c, s, xa, xb);
      w1[0] = narrow8(xa);
      w2[0] = narrow8(xb);
    }
    row[kLatent / 8 + chunk_a(ADJ, lane)] = w1[0];
    row[kLatent / 8 + chunk_b(ADJ, lane)] = w2[0];
  }
}

// ---------------------------------------------------------------------------
// expansion
// ---------------------------------------------------------------------------

// Dense rows: those of every sequence side by side, each sequence's to whole tiles of 32. A workgroup makes keys and
// values of some heads for 128 rows, 128 dims at a time: four waves of 64 x 64, 32 latent dims a stage, four stages
// in LDS, two workgroups a compute unit. Latent rows come straight from their slots. Both operands' rows go to
// LDS as they lie, 64 bytes a row and stage, chunks permuted so that an operand read meets no bank conflict.
// (Keys that are no context are made of whatever a slot holds: the attention masks them.)
//
// Keys are rounded to bf16, as the queries that they meet. Values are rounded to fp16, like the softmax weights that
// they meet: three bits more (with both in bf16 the result is 1.65 times as far from 64 bits as one that is
// rounded once, so 1.2). fp16's range is made up for by an exponent e of each row and head: a row is stored 2^-e of
// itself, its largest magnitude 2^13 .. 2^14. As nearly always, where each row of a tile of 32 is zeros or has a largest magnitude in
// kPlainLeast .. kPlainMost, the tile is stored as it is: what is lost there are steps of 2^-24 of weights on rows
// that are at most 2^11 times the smallest ones.
//
// Measured: 64 heads of 8400 rows (1.41e11 operations, 0.28 GB written) 234 us, 600 TFLOP/s. What it moves binds: both
// operands' 2.2 GB from L2 to LDS and the stores (without these 80 us less, without the products 47). 256 rows and 256 dims
// to a workgroup of eight waves move half of that, and took 211, but 23.5 for a prompt of 301 rows and 32 heads, now 12.8.
constexpr int kExpandThreads = 256, kExpandWaves = kExpandThreads / kWave;
constexpr int kStageDims = 32, kStages = 4, kTileRows = 128;
constexpr int kHalfTile = kTileRows * kStageDims * 2;
constexpr float kPlainLeast = 0x1p-6f, kPlainMost = 0x1p5f;

__device__ __forceinline__ uint32_t pack2_f16(float lo, float hi) {   // round to nearest even
  const pf::float2_t f = {lo, hi};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, ra::half2_t));
}
// 16 bytes from each lane's own address to LDS at dst + 16 * lane.
__device__ __forceinline__ void load_rows_to_lds(const uint8_t* lane_src, const uint8_t* dst) {
  const uint32_t m0 = (uint32_t)(uintptr_t)dst;
  asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(lane_src), "{m0}"(__builtin_amdgcn_readfirstlane(m0)));
}

__global__ __launch_bounds__(kExpandThreads, 2) void latent_expand_kernel(ExpandArgs a, int items_each) {
  constexpr int kTiles = kTileRows / ra::kKeys;   // of 32 rows
  __shared__ __attribute__((aligned(1024))) uint8_t s_tile[kStages][2 * kHalfTile];
  __shared__ int64_t s_scan[kExpandWaves];
  __shared__ int s_seq[kTiles], s_pos[kTiles];    // of each tile: its sequence (-1: none) and first position
  __shared__ float s_max[2][kTileRows];
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = wave_id_uniform();
  const int half = lane >> 5, col = lane & 31;
  const int shares = (2 * a.heads + items_each - 1) / items_each;   // workgroups of a tile of rows, one after another
  const int64_t row0 = (int64_t)(blockIdx.x / shares) * kTileRows;
  const int item0 = (int)(blockIdx.x % shares) * items_each, items = min(items_each, 2 * a.heads - item0);   // keys (even) or values of head item / 2

  // ---- The tiles' sequences.
  RowsArgs ra_{};
  ra_.cu_q = a.cu_q;
  ra_.ctx_lens = a.ctx_lens;
  ra_.num_q_tokens = a.num_q_tokens;
  ra_.max_ctx = a.max_ctx;
  ra_.max_blocks_per_seq = a.max_blocks_per_seq;
  const int per = (a.num_seqs + kExpandThreads - 1) / kExpandThreads;
  const int s0 = min(tid * per, a.num_seqs), s1 = min(s0 + per, a.num_seqs);
  int64_t mine = 0;
  for (int s = s0; s < s1; ++s) mine += ra::dense_rows(ra::seq_of(ra_, s).ctx);
  const int64_t inc = ra::wave_scan64(mine, lane);
  if (lane == kWave - 1) s_scan[wave] = inc;
  if (tid < kTiles) s_seq[tid] = -1;
  __syncthreads();
  int64_t first = inc - mine;
  for (int i = 0; i < wave; ++i) first += s_scan[i];
  if (first < row0 + kTileRows && first + mine > row0) {
    for (int s = s0; s < s1; ++s) {
      const int64_t rows = ra::dense_rows(ra::seq_of(ra_, s).ctx);
      for (int i = 0; i < kTiles; ++i) {
        const int64_t r = row0 + 32 * i;
        if (r >= first && r < first + rows) {
          s_seq[i] = s;
          s_pos[i] = (int)(r - first);
        }
      }
      first += rows;
    }
  }
  __syncthreads();
  if (s_seq[0] < 0) return;   // behind the last sequence (uniform)
  // Row r of the workgroup's, in the pool (one that is not there: the first row of the pool).
  const auto pool_row = [&](int r) -> const uint8_t* {
    const uint8_t* pool = static_cast<const uint8_t*>(a.pool);
    const int s = s_seq[r >> 5], pos = s_pos[r >> 5] + (r & 31);
    if (s < 0 || (pos >> 4) >= a.max_blocks_per_seq) return pool;
    const int b = a.block_tables[(size_t)s * a.max_blocks_per_seq + (pos >> 4)];
    if (b < 0 || b >= a.num_blocks) return pool;
    const int slot = slot_of_offset(pos & 15, entry_direction(a.dir, a.cls, a.dir_per_entry, a.max_blocks_per_seq, s, pos >> 4));
    return pool + ((size_t)b * kBlockSize + slot) * (kRow * 2);
  };

  const auto is_context = [&](int r) -> bool {
    const int s = s_seq[r >> 5], pos = s_pos[r >> 5] + (r & 31);
    if (s < 0 || pos >= ra::seq_of(ra_, s).ctx) return false;   // (ctx: within the table's width)
    const int b = a.block_tables[(size_t)s * a.max_blocks_per_seq + (pos >> 4)];
    return b >= 0 && b < a.num_blocks;
  };

  // A wave loads rows 32 wave .. + 31 of both operands, sixteen rows of 64 bytes to a load: row r's chunk c lies at
  // 64 r + 16 (c ^ (r / 4 % 4)), so that 16 rows' chunks of one operand read lie in 16 groups of banks.
  const uint8_t* csrc[2];
  uint32_t woff[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int r = 32 * wave + 16 * i + (lane >> 2);
    const uint32_t chunk = (uint32_t)(((lane & 3) ^ ((r >> 2) & 3)) << 4);
    csrc[i] = pool_row(r) + chunk;
    woff[i] = (uint32_t)r * (kLatent * 2) + chunk;
  }
  constexpr int kPerItem = kLatent / kStageDims;
  constexpr int kLoads = 4;                  // of a wave and stage
  const int stages = items * kPerItem;
  auto issue = [&](int k) __attribute__((always_inline)) {   // stage k: latent dims 32 (k % 16) .. of item k / 16
    const uint8_t* wsrc = static_cast<const uint8_t*>(a.w) + ((size_t)(item0 + k / kPerItem) * 128 * kLatent + (k % kPerItem) * kStageDims) * 2;
    uint8_t* dst = s_tile[k % kStages];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int r16 = 32 * wave + 16 * i;
      ra::load_to_lds(wsrc, woff[i], dst + r16 * 64);
      load_rows_to_lds(csrc[i] + (k % kPerItem) * (kStageDims * 2), dst + kHalfTile + r16 * 64);
    }
  };
  const int wd = wave & 1, wr = wave >> 1;   // the wave's 64 dims and 64 rows
  uint32_t context = 0;                      // bit k: row 64 wr + 32 k + col is one
#pragma unroll
  for (int k = 0; k < 2; ++k) context |= (is_context(64 * wr + 32 * k + col) ? 1u : 0u) << k;
  const int lane_at = col * 64, sw = (col >> 2) & 3;
  pf::floatx16 o[2][2];                      // [dims][rows]
  // (the addresses come from loads that the compiler sees: they are there before the first request)
#pragma unroll
  for (int k = 0; k < kStages - 1; ++k) issue(k);   // (an item has more)
#pragma unroll 1
  for (int item = 0; item < items; ++item) {
    const bool values = (item0 + item) & 1;
    const int head = (item0 + item) >> 1;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
#pragma unroll
      for (int k = 0; k < 2; ++k) o[i][k] = pf::floatx16{};
    }
#pragma unroll 1
    for (int kk = 0; kk < kPerItem; ++kk) {
      const int stage = item * kPerItem + kk;
      // (the stages behind it may be in flight, and what the item before stored)
      const int later = min(kStages - 2, stages - 1 - stage);
      if (later == 2) pf::wait_vmem<2 * kLoads>();
      else if (later == 1) pf::wait_vmem<kLoads>();
      else pf::wait_vmem<0>();
      pf::lds_barrier();
      if (stage + kStages - 1 < stages) issue(stage + kStages - 1);
      const uint8_t* tw = s_tile[stage % kStages] + wd * 64 * 64;
      const uint8_t* tc = s_tile[stage % kStages] + kHalfTile + wr * 64 * 64;
#pragma unroll
      for (int c = 0; c < kStageDims / 16; ++c) {
        const int at = lane_at + (((2 * c + half) ^ sw) << 4);
        pf::v4u_t x[2], y[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          x[i] = *reinterpret_cast<const pf::v4u_t*>(tw + 32 * 64 * i + at);
          y[i] = *reinterpret_cast<const pf::v4u_t*>(tc + 32 * 64 * i + at);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
#pragma unroll
          for (int k = 0; k < 2; ++k)
            o[i][k] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(pf::as_bf16x8(x[i]), pf::as_bf16x8(y[k]), o[i][k], 0, 0, 0);
        }
      }
    }
    // The values' exponents: of a row's largest finite magnitude. Rows that are no context are zeros, and rows of zeros have no
    // size that counts anywhere.
    float mul[2] = {1.0f, 1.0f};
    if (values) {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const bool there = (context >> k) & 1u;
        float m = 0.0f;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            o[i][k][e] = there ? o[i][k][e] : 0.0f;
            const float x = fabsf(o[i][k][e]);
            m = fmaxf(m, x < INFINITY ? x : 0.0f);
          }
        }
        m = pf::pair_max(m);
        if (half == 0) s_max[wd][64 * wr + 32 * k + col] = m;
      }
    }
    pf::lds_barrier();   // (and every wave has read the last stage: its place takes the results)
    if (values) {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int r = 64 * wr + 32 * k + col;
        const float m = fmaxf(s_max[0][r], s_max[1][r]);
        const bool scaled = __builtin_amdgcn_ballot_w64(m > 0.0f && !(m >= kPlainLeast && m < kPlainMost)) != 0;
        const int e = !scaled ? 0 : m > 0.0f ? max(-120, min(120, ilogbf(m) - 13)) : ra::kNoExponent;
        mul[k] = e == ra::kNoExponent ? 1.0f : ldexpf(1.0f, -e);
        const int64_t tile = row0 / 32 + 2 * wr + k;
        if (wd == 0 && 32 * tile < a.dense_rows) {
          if (lane == 0) a.scaled[(size_t)head * (a.dense_rows / 32) + tile] = scaled;
          if (scaled && half == 0) a.exps[(size_t)head * a.dense_rows + 32 * tile + col] = (int8_t)e;
        }
      }
    }
    uint16_t* dst = static_cast<uint16_t*>(values ? a.v_rows : a.k_rows) + (size_t)head * a.dense_rows * 128 + 64 * wd;
    // (through LDS to whole lines: as the products leave them, 16 bytes a row, the stores take as long as the products)
    uint8_t* out = s_tile[(item * kPerItem + kPerItem - 1) % kStages] + wave * 4096;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      // row `col`, 128 bytes: chunk c at 16 (c ^ (col % 8))
#pragma unroll
      for (int i = 0; i < 2; ++i) {
#pragma unroll
        for (int jq = 0; jq < 4; ++jq) {
          const float x[4] = {o[i][k][4 * jq], o[i][k][4 * jq + 1], o[i][k][4 * jq + 2], o[i][k][4 * jq + 3]};
          uint2 v;
          if (values) v = make_uint2(pack2_f16(x[0] * mul[k], x[1] * mul[k]), pack2_f16(x[2] * mul[k], x[3] * mul[k]));
          else v = make_uint2(pf::pack2_bf16(x[0], x[1]), pf::pack2_bf16(x[2], x[3]));
          *reinterpret_cast<uint2*>(out + col * 128 + (((4 * i + jq) ^ (col & 7)) << 4) + 8 * half) = v;
        }
      }
      // (the wave's own: reads follow its writes in order)
      const int64_t r0 = row0 + 64 * wr + 32 * k;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int r = 8 * i + (lane >> 3);
        const uint4 v = *reinterpret_cast<const uint4*>(out + r * 128 + (((lane & 7) ^ (r & 7)) << 4));
        if (r0 < a.dense_rows) *reinterpret_cast<uint4*>(dst + (r0 + r) * 128 + 8 * (lane & 7)) = v;
      }
    }
  }
  // The rotated keys' dense rows, once a call.
  if (item0 == 0 && a.with_rot) {
    const int r = tid >> 1;   // (two threads a row)
    if (row0 + r < a.dense_rows) {
      const uint4* src = reinterpret_cast<const uint4*>(pool_row(r) + kLatent * 2) + 4 * (tid & 1);
      uint4* to = reinterpret_cast<uint4*>(static_cast<uint8_t*>(a.rot_rows) + (row0 + r) * (kRot * 2)) + 4 * (tid & 1);
#pragma unroll
      for (int i = 0; i < 4; ++i) to[i] = src[i];
    }
  }
}

}  // namespace

template <int EACH>
static hipError_t append_rows(const LatentAppendArgs& a, hipStream_t stream) {
  const int64_t kv = ((int64_t)a.num_new_tokens + kTokens - 1) / kTokens;
  const int64_t q = ((int64_t)a.num_new_tokens * a.num_q_heads + kHeads * EACH - 1) / (kHeads * EACH);
  if ((kv + q) * kThreads > 0xffffffffLL) return hipErrorInvalidValue;
  if (kv + q == 0) return hipSuccess;
  if (a.adjacent) hipLaunchKernelGGL((latent_append_kernel<true, EACH>), dim3((unsigned)(kv + q)), dim3(kThreads), 0, stream, a, (int)kv);
  else hipLaunchKernelGGL((latent_append_kernel<false, EACH>), dim3((unsigned)(kv + q)), dim3(kThreads), 0, stream, a, (int)kv);
  return hipGetLastError();
}

hipError_t launch_latent_append(const LatentAppendArgs& a, hipStream_t stream) {
  // Query rows of a thread: more from two workgroups a compute unit on (fewer workgroups each look their tokens up), four
  // where heads enough share a token's angles. Us with 1, 2 and 4: 32 tokens of 128 heads 3.8, 4.2, 5.2; 256 5.4, 4.9, 5.8;
  // 1024 15.3, 10.6, 10.0; 4000 of 16 heads 12.3, 12.0, 13.0; 8000 21.1, 19.1, 20.0; 6000 of 128 86, 65, 63 (with 8: 66).
  const int64_t rows = (int64_t)a.num_new_tokens * a.num_q_heads, wide = 2 * kHeads * (int64_t)stream_compute_units(stream);
  if (rows >= 2 * wide && a.num_q_heads >= 64) return append_rows<4>(a, stream);
  return rows >= wide ? append_rows<2>(a, stream) : append_rows<1>(a, stream);
}

hipError_t launch_latent_expand(const ExpandArgs& a, hipStream_t stream) {
  const int64_t tiles = (a.dense_rows + kTileRows - 1) / kTileRows;
  // Items (a head's keys, or its values) of a workgroup, one, two or four: the number whose rounds over the compute units, two
  // workgroups each, end first; a workgroup's start (its rows' places) takes as long as two thirds of an item. Us of a whole call
  // with 1, 2, 4 and 8: four chunks of 1000 rows behind 1100, 64 heads, 623, 598, 600, 622; two of 512 behind 8000 883, 846, 806, 819;
  // one prompt of 301 rows, 128 heads, 72, 67, 73, 98; 32 heads 30, 36, 49, 73. (Odd numbers part a head: 3 622, 5 603.)
  const int64_t slots = 2 * (int64_t)stream_compute_units(stream), all = 2 * (int64_t)a.heads;
  int64_t each = 1;
  double best = 0.0;
  for (int n = 1; n <= 4; n *= 2) {
    const double us = (double)(((all + n - 1) / n * tiles + slots - 1) / slots) * (n + 0.67);
    if (n == 1 || us < best) {
      each = n;
      best = us;
    }
  }
  // (a grid holds 2^32 - 1 threads)
  while (each < all && (all + each - 1) / each * tiles > (1LL << 23)) each *= 2;
  hipLaunchKernelGGL(latent_expand_kernel, dim3((unsigned)((all + each - 1) / each * tiles)), dim3(kExpandThreads), 0, stream, a, (int)each);
  return hipGetLastError();
}

constexpr int kNarrowKeys = 1024;   // contexts of narrow units of the expanded form, at most

hipError_t launch_latent(RowsArgs a, void* workspace, hipStream_t stream) {
  const int64_t columns = planned_rows(a.max_q_len, a.num_q_tokens, a.num_seqs) * a.num_q_heads;
  const int64_t keys = 16 * (int64_t)longest_blocks(a.max_ctx, a.max_blocks_per_seq);
  switch (pick_rows_way(kLatentWays, columns, a.num_seqs, keys, stream_compute_units(stream))) {
    case 0: return ra::launch_latent_rows<1, 4>(a, 4, 6, 6, workspace, stream);
    case 1: return ra::launch_latent_rows<2, 2>(a, 4, 6, 6, workspace, stream);
    case 2: return ra::launch_latent_rows<4, 1>(a, 4, 6, 6, workspace, stream);
    default: return ra::launch_latent_rows<8, 1>(a, 6, 6, 6, workspace, stream);
  }
}

// Units of 128 rows over steps of 32 keys, cut into shares; where contexts are short and units few, whole units of 64
// rows over steps of 64 keys, a workgroup each: half the steps one after another, and no merge. Us of a whole call, wide
// and narrow: one prompt of 301 rows and 32 heads 44 and 30, of 1000 and 16 heads 50 and 42, of 500 and 64 heads 62 and 54;
// four of 200 and 16 heads 37 and 28. With more units the wide ones read less: 700 rows behind 100 and 128 heads
// 130 and 156; with longer contexts shares are even: 301 rows behind 700 and 16 heads 43 and 45, 150 behind 3000 89
// and 84 (cut), with 32 heads.
hipError_t launch_expanded(RowsArgs a, void* workspace, hipStream_t stream) {
  const int64_t rows = planned_rows(a.max_q_len, a.num_q_tokens, a.num_seqs);
  const int64_t units = (int64_t)a.num_seqs * a.num_kv_heads * ((rows + 63) / 64);
  if (16 * (int64_t)longest_blocks(a.max_ctx, a.max_blocks_per_seq) <= kNarrowKeys && units <= 2 * (int64_t)stream_compute_units(stream))
    return ra::launch_rows<ra::Expanded, 2, 2, 3, 1>(a, 4, kNarrowKeys / 64, 4, workspace, stream);
  switch (rows_team((rows + 127) / 128, a.num_q_tokens, rows, a.num_seqs)) {
    case 4: return ra::launch_rows<ra::Expanded, 4, 1, 3, 2, 4>(a, 4, 8, 4, workspace, stream);
    case 2: return ra::launch_rows<ra::Expanded, 4, 1, 3, 2, 2>(a, 4, 8, 4, workspace, stream);
    default: return ra::launch_rows<ra::Expanded, 4, 1, 3, 2>(a, 4, 8, 4, workspace, stream);
  }
}

}  // namespace bros
