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

// Rows of one kind to a workgroup: kTokens latent rows, a wave each, or kHeads query rows of 64, four lanes each.
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

// Turns pairs 8 l .. + 7 of token t at logical position pos. (Positions outside the table: row 0; the caller drops them.)
template <bool ADJ>
__device__ __forceinline__ void turn(const LatentAppendArgs& a, int t, int pos, int l, float (&xa)[8], float (&xb)[8]) {
  float c[8], s[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int pair = 8 * l + i;
    int row = pos;
    if (a.rope_pos != nullptr) row = a.rope_pos[(size_t)axis_of(a, pair) * a.num_new_tokens + t];
    row = row < 0 || row >= a.table_rows ? 0 : row;
    c[i] = a.rope_table[(size_t)row * kRot + pair];
    s[i] = a.rope_table[(size_t)row * kRot + kRot / 2 + pair];
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float& u = ADJ ? (i < 4 ? xa[2 * (i & 3)] : xb[2 * (i & 3)]) : xa[i];
    float& v = ADJ ? (i < 4 ? xa[2 * (i & 3) + 1] : xb[2 * (i & 3) + 1]) : xb[i];
    const float u0 = u, v0 = v;
    u = fmaf(u0, c[i], -(v0 * s[i]));
    v = fmaf(v0, c[i], u0 * s[i]);
  }
}

// ADJ: pairs (2 i, 2 i + 1) instead of (i, i + 32).
template <bool ADJ>
__global__ __launch_bounds__(kThreads) void latent_append_kernel(LatentAppendArgs a, int kv_groups) {
  __shared__ int s_seq[kHeads], s_pos[kHeads];
  const int tid = threadIdx.x;
  const bool kv = (int)blockIdx.x < kv_groups;
  // the workgroup's tokens t0 .. t0 + n_tok - 1
  int64_t item0 = 0;
  int t0, n_tok;
  if (kv) {
    t0 = blockIdx.x * kTokens;
    n_tok = min(kTokens, a.num_new_tokens - t0);
  } else {
    item0 = (int64_t)(blockIdx.x - kv_groups) * kHeads;
    t0 = (int)(item0 / a.num_q_heads);
    n_tok = min((int)((item0 + kHeads - 1) / a.num_q_heads) - t0 + 1, a.num_new_tokens - t0);
  }
  // this thread's row, requested before its position is known
  const int lane = tid & (kWave - 1), l4 = tid & 3;
  const int64_t item = item0 + tid / 4;
  const int t = kv ? t0 + tid / kWave : (int)min(item / a.num_q_heads, (int64_t)a.num_new_tokens - 1);
  const int h = kv ? 0 : (int)(item % a.num_q_heads);
  const bool live = kv ? t < a.num_new_tokens : item < (int64_t)a.num_new_tokens * a.num_q_heads;
  uint4 w0{}, w1{}, w2{};
  if (live) {
    if (kv) {
      const uint4* row = reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.kv) + (size_t)t * a.kv_stride);
      w0 = row[lane];
      if (lane < 4) {
        w1 = row[kLatent / 8 + chunk_a(ADJ, lane)];
        w2 = row[kLatent / 8 + chunk_b(ADJ, lane)];
      }
    } else {
      const uint4* row = reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.q) + (size_t)t * a.q_stride + (size_t)h * a.q_head_stride);
      w1 = row[chunk_a(ADJ, l4)];
      w2 = row[chunk_b(ADJ, l4)];
    }
  }
  if (tid < kHeads) s_seq[tid] = -1;
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
  if (!live) return;
  const int seq = s_seq[t - t0];
  if (seq < 0) return;   // in no sequence: left as it was
  const int pos = s_pos[t - t0];
  bool off = false;      // a position outside the table
  if (a.rope_table != nullptr) {
    if (a.rope_pos == nullptr) off = pos < 0 || pos >= a.table_rows;
    else {
      for (int x = 0; x < a.axes; ++x) {
        const int r = a.rope_pos[(size_t)x * a.num_new_tokens + t];
        off |= r < 0 || r >= a.table_rows;
      }
    }
  }
  float xa[8], xb[8];
  if (!kv) {
    widen8(w1, xa);
    widen8(w2, xb);
    if (a.rope_table != nullptr) turn<ADJ>(a, t, pos, l4, xa, xb);
    uint4* row = reinterpret_cast<uint4*>(static_cast<uint16_t*>(a.q_out) + (size_t)t * a.out_stride + (size_t)h * a.out_head_stride);
    const uint4 zero = make_uint4(0, 0, 0, 0);
    row[chunk_a(ADJ, l4)] = off ? zero : a.rope_table != nullptr ? narrow8(xa) : w1;
    row[chunk_b(ADJ, l4)] = off ? zero : a.rope_table != nullptr ? narrow8(xb) : w2;
    return;
  }
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
      widen8(w1, xa);
      widen8(w2, xb);
      turn<ADJ>(a, t, pos, lane, xa, xb);
      w1 = narrow8(xa);
      w2 = narrow8(xb);
    }
    row[kLatent / 8 + chunk_a(ADJ, lane)] = w1;
    row[kLatent / 8 + chunk_b(ADJ, lane)] = w2;
  }
}

// ---------------------------------------------------------------------------
// expansion
// ---------------------------------------------------------------------------

// Latent rows of every sequence side by side, each sequence's to whole tiles of 32, zeros where there
// is no context. A workgroup takes one tile.
__global__ __launch_bounds__(kThreads) void latent_gather_kernel(ExpandArgs a) {
  __shared__ int64_t s_scan[kThreads / kWave];
  __shared__ int s_seq, s_first;
  const int tid = threadIdx.x, lane = tid & (kWave - 1), w = tid / kWave;
  RowsArgs ra_{};
  ra_.cu_q = a.cu_q;
  ra_.ctx_lens = a.ctx_lens;
  ra_.num_q_tokens = a.num_q_tokens;
  ra_.max_ctx = a.max_ctx;
  ra_.max_blocks_per_seq = a.max_blocks_per_seq;
  const int per = (a.num_seqs + kThreads - 1) / kThreads;
  const int s0 = min(tid * per, a.num_seqs), s1 = min(s0 + per, a.num_seqs);
  int64_t mine = 0;
  for (int s = s0; s < s1; ++s) mine += ra::dense_rows(ra::seq_of(ra_, s).ctx);
  const int64_t inc = ra::wave_scan64(mine, lane);
  if (lane == kWave - 1) s_scan[w] = inc;
  if (tid == 0) s_seq = -1;
  __syncthreads();
  int64_t first = inc - mine;
  for (int i = 0; i < w; ++i) first += s_scan[i];
  const int64_t row0 = (int64_t)blockIdx.x * ra::kKeys;
  if (row0 >= first && row0 < first + mine) {
    for (int s = s0; s < s1; ++s) {
      const int rows = ra::dense_rows(ra::seq_of(ra_, s).ctx);
      if (row0 < first + rows) {
        s_seq = s;
        s_first = (int)(row0 - first);   // position of the tile's first row
        break;
      }
      first += rows;
    }
  }
  __syncthreads();
  const int s = s_seq;
  if (s < 0) return;   // behind the last sequence
  const int ctx = ra::seq_of(ra_, s).ctx;
  constexpr int kChunks = kRow / 8;
  for (int i = tid; i < ra::kKeys * kChunks; i += kThreads) {
    const int r = i / kChunks, ch = i % kChunks, pos = s_first + r;
    uint4 v = make_uint4(0, 0, 0, 0);
    if (pos < ctx) {
      const int b = a.block_tables[(size_t)s * a.max_blocks_per_seq + (pos >> 4)];
      if (b >= 0 && b < a.num_blocks) {
        const int slot = slot_of_offset(pos & 15, entry_direction(a.dir, a.cls, a.dir_per_entry, a.max_blocks_per_seq, s, pos >> 4));
        v = reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.pool) + ((size_t)b * kBlockSize + slot) * kRow)[ch];
      }
    }
    const size_t row = (size_t)row0 + r;
    if (ch < kLatent / 8) reinterpret_cast<uint4*>(static_cast<uint16_t*>(a.latents) + row * kLatent)[ch] = v;
    else reinterpret_cast<uint4*>(static_cast<uint16_t*>(a.rot_rows) + row * kRot)[ch - kLatent / 8] = v;
  }
}

// Rows [128 y, + 128) of the keys (even x) or values (odd x) of head x / 2: latents times
// weights, 128 x 128 values to a workgroup, four waves of 64 x 64, 64 latent dims a step.
// Both operands' rows go to LDS as they lie, 128 bytes a row and step, chunks permuted so that
// an operand read meets no bank conflict.
constexpr int kStepDims = 64, kTileRows = 128;
constexpr int kHalfTile = kTileRows * kStepDims * 2;
__global__ __launch_bounds__(kThreads, 2) void latent_expand_kernel(ExpandArgs a, int64_t rows) {
  __shared__ __attribute__((aligned(1024))) uint8_t s_tile[2][2 * kHalfTile];
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = wave_id_uniform();
  const int half = lane >> 5, col = lane & 31;
  const size_t row0 = (size_t)blockIdx.y * kTileRows;
  const int head = blockIdx.x >> 1, which = blockIdx.x & 1;
  const uint8_t* wsrc = static_cast<const uint8_t*>(a.w) + ((size_t)head * 256 + 128 * which) * kLatent * 2;
  const uint8_t* csrc = static_cast<const uint8_t*>(a.latents);

  // a wave loads rows 32 wave .. + 31 of both tiles, eight rows of 128 bytes to a load
  auto issue = [&](int step, int buf) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r8 = 32 * wave + 8 * i, r = r8 + (lane >> 3);
      const uint32_t chunk = (uint32_t)(((lane & 7) ^ ((r >> 1) & 7)) << 4);
      pf::load_to_lds(wsrc + step * 128, (uint32_t)r * (kLatent * 2) + chunk, s_tile[buf] + r8 * 128);
      // (rows behind the buffer's end: its last row again)
      const size_t cr = min(row0 + r, (size_t)a.dense_rows - 1);
      pf::load_to_lds(csrc + row0 * (kLatent * 2) + step * 128, (uint32_t)(cr - row0) * (kLatent * 2) + chunk, s_tile[buf] + kHalfTile + r8 * 128);
    }
  };
  const int wd = wave & 1, wr = wave >> 1;   // the wave's 64 dims and 64 rows
  pf::floatx16 o[2][2];                      // [dims][rows]
#pragma unroll
  for (int i = 0; i < 2; ++i) {
#pragma unroll
    for (int k = 0; k < 2; ++k) o[i][k] = pf::floatx16{};
  }
  const int r_lane = (col >> 1) * 256 + ((col & 1) << 7), r_sw = (col >> 1) & 7;
  constexpr int kSteps = kLatent / kStepDims;
  issue(0, 0);
#pragma unroll 1
  for (int step = 0; step < kSteps; ++step) {
    pf::wait_vmem<0>();
    pf::lds_barrier();
    if (step + 1 < kSteps) issue(step + 1, (step + 1) & 1);
    const uint8_t* tw = s_tile[step & 1] + wd * 64 * 128;
    const uint8_t* tc = s_tile[step & 1] + kHalfTile + wr * 64 * 128;
#pragma unroll
    for (int c = 0; c < kStepDims / 16; ++c) {
      const int at = r_lane + (((2 * c + half) ^ r_sw) << 4);
      pf::v4u_t x[2], y[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        x[i] = *reinterpret_cast<const pf::v4u_t*>(tw + 32 * 128 * i + at);
        y[i] = *reinterpret_cast<const pf::v4u_t*>(tc + 32 * 128 * i + at);
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
#pragma unroll
        for (int k = 0; k < 2; ++k)
          o[i][k] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(pf::as_bf16x8(x[i]), pf::as_bf16x8(y[k]), o[i][k], 0, 0, 0);
      }
    }
  }
  // (the expanded keys and values are rounded to bf16 once: the second operand type of the
  // matrix cores' products, as the rows of a K/V pool are)
  uint16_t* dst = static_cast<uint16_t*>(which == 0 ? a.k_rows : a.v_rows) + (size_t)head * a.dense_rows * 128;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const size_t r = row0 + 64 * wr + 32 * k + col;
    if (r >= (size_t)rows) continue;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
#pragma unroll
      for (int jq = 0; jq < 4; ++jq) {
        uint2 v;
        v.x = pf::pack2_bf16(o[i][k][4 * jq], o[i][k][4 * jq + 1]);
        v.y = pf::pack2_bf16(o[i][k][4 * jq + 2], o[i][k][4 * jq + 3]);
        *reinterpret_cast<uint2*>(dst + r * 128 + 64 * wd + 32 * i + 8 * jq + 4 * half) = v;
      }
    }
  }
}

}  // namespace

hipError_t launch_latent_append(const LatentAppendArgs& a, hipStream_t stream) {
  const int64_t kv = ((int64_t)a.num_new_tokens + kTokens - 1) / kTokens;
  const int64_t q = ((int64_t)a.num_new_tokens * a.num_q_heads + kHeads - 1) / kHeads;
  if ((kv + q) * kThreads > 0xffffffffLL) return hipErrorInvalidValue;
  if (kv + q == 0) return hipSuccess;
  if (a.adjacent) hipLaunchKernelGGL(latent_append_kernel<true>, dim3((unsigned)(kv + q)), dim3(kThreads), 0, stream, a, (int)kv);
  else hipLaunchKernelGGL(latent_append_kernel<false>, dim3((unsigned)(kv + q)), dim3(kThreads), 0, stream, a, (int)kv);
  return hipGetLastError();
}

hipError_t launch_latent_gather(const ExpandArgs& a, hipStream_t stream) {
  hipLaunchKernelGGL(latent_gather_kernel, dim3((unsigned)(a.dense_rows / ra::kKeys)), dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_latent_expand(const ExpandArgs& a, hipStream_t stream) {
  const unsigned tiles = (unsigned)((a.dense_rows + kTileRows - 1) / kTileRows);
  hipLaunchKernelGGL(latent_expand_kernel, dim3(2 * a.heads, tiles), dim3(kThreads), 0, stream, a, a.dense_rows);
  return hipGetLastError();
}

hipError_t launch_latent(RowsArgs a, void* workspace, hipStream_t stream) {
  const int64_t columns = (int64_t)a.max_q_len * a.num_q_heads;
  const int64_t keys = 16 * (int64_t)longest_blocks(a.max_ctx, a.max_blocks_per_seq);
  switch (pick_rows_way(kLatentWays, columns, a.num_seqs, keys, stream_compute_units(stream))) {
    case 0: return ra::launch_latent_rows<1, 4>(a, 4, 6, workspace, stream);
    case 1: return ra::launch_latent_rows<2, 2>(a, 4, 6, workspace, stream);
    case 2: return ra::launch_latent_rows<4, 1>(a, 4, 6, workspace, stream);
    default: return ra::launch_latent_rows<8, 1>(a, 6, 6, workspace, stream);
  }
}

hipError_t launch_expanded(RowsArgs a, void* workspace, hipStream_t stream) {
  return ra::launch_rows<ra::Expanded, 4, 1, 3, 2>(a, 4, 8, workspace, stream);
}

}  // namespace bros
