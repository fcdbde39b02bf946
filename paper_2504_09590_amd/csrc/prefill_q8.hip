// bros_attn_prefill_chunk_q8: the matrix-core prefill (prefill_device.h) over an
// 8-bit pool. Units, pieces and their merge are the 16-bit prefill's.
//
// The matrix cores bound it from a few dozen rows on: 512 rows on 16000 cached tokens,
// 32 / 8 heads, 142 us, 960 TFLOP/s of the formula's products (the 16-bit prefill over the same values
// 135 us; a large library product 1208 TFLOP/s). Few rows on short contexts run in smaller groups (below).
#include "decode_q8_device.h"
#include "plan.h"
#include "prefill_device.h"

#include <algorithm>

namespace bros {
namespace pf {

template <int G, bool kOff32, bool kRing>
__global__ __launch_bounds__(kThreads, 2) void prefill_q8_kernel(PrefillArgs a, const uint8_t* scales) {
  __shared__ __attribute__((aligned(1024))) uint8_t s_kring[kSlots * kQ8TileBytes];
  __shared__ __attribute__((aligned(1024))) uint8_t s_raw[kSlots * kQ8TileBytes];   // V as it is in the pool
  __shared__ __attribute__((aligned(1024))) uint8_t s_vring[2 * kTileBytes];
  __shared__ __attribute__((aligned(256))) uint32_t s_scale[kSlots * kThreads];      // per slot and wave
  __shared__ __attribute__((aligned(16))) uint16_t s_nan[kGuardKeys * 8];   // per key and 16 dims: values that are not finite
  __shared__ int s_tbl[kMaxTableLds + kTablePad];
  __shared__ int8_t s_dir[kMaxTableLds + kTablePad];
  __shared__ int s_first_bad, s_any_nan;
  prefill_unit<G, kOff32, kRing, true>(a, paired_id(a, blockIdx.x, gridDim.x), s_kring, s_vring, &s_first_bad, s_tbl, s_dir,
                                       scales, s_nan, &s_any_nan, s_raw, s_scale);
}

template <int G>
hipError_t launch_q8_group(PrefillArgs a, const uint8_t* scales, int num_units, hipStream_t stream) {
  long long grid = 0;
  const bool ring = plan_prefill_launch(a, num_units, stream, &grid);
  // (block, KV head) rows of 2 KiB: 32-bit offsets reach them all below 2^21 rows
  const bool off32 = (int64_t)a.num_blocks * a.num_kv_heads <= (int64_t)1 << 21;
  const dim3 g((unsigned)grid), b(kThreads);
  if (ring) {
    if (off32) hipLaunchKernelGGL((prefill_q8_kernel<G, true, true>), g, b, 0, stream, a, scales);
    else hipLaunchKernelGGL((prefill_q8_kernel<G, false, true>), g, b, 0, stream, a, scales);
  } else {
    if (off32) hipLaunchKernelGGL((prefill_q8_kernel<G, true, false>), g, b, 0, stream, a, scales);
    else hipLaunchKernelGGL((prefill_q8_kernel<G, false, false>), g, b, 0, stream, a, scales);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.num_cus == 0) return e;
  return launch_prefill_merge(a, G, num_units, stream);
}

}  // namespace pf

namespace dq {

// Few rows (plan.h: plan_q8_prefill_rows): the decode's steps (decode_q8_device.h), their 16 columns
// filled with 16 / G positions of G heads. A workgroup takes 16 columns, or a piece of the blocks they
// see; wave w folds every fourth pair of blocks into a running result of its own, and the four
// meet in LDS. Pieces leave partials (max, sum, unnormalised output) that a second kernel folds.
//
// In the other kernel a prompt of 301 rows is 80 chains of up to ten steps, one after another, behind a
// start of 9 us (Q's terms, the first tiles, their conversion); here it is 600 workgroups of at most three
// steps a wave. Latency bounds it: 5.7 us for 16 rows, 11.3 for the 301 (15.1 there; calls of one graph), 13.1 for 16
// rows on 4000 cached tokens in pieces (25.3 there). K and V are read once per 16 columns, from L2. (Two bf16 parts for the weights, as in the decode, take 2 to 8 % longer;
// the marks of values that are not finite made inside the step spill or take 0.4 us more.)

// The bytes of w whose values are not finite, as ones.
__device__ __forceinline__ uint32_t odd_ones(uint32_t w, uint32_t scale) { return q8::not_finite(w, scale) >> 7; }

// Removes what the lane's column does not see of a pair (slots from `limit` on) and, by selection, V
// rows that no column does (from `last` on). A row that only some columns see must not reach the
// others through 0 times infinity or NaN: its values that are not finite become zeros, and `found` is set.
__device__ __forceinline__ void mask_causal(const PrefillArgs& a, int seq, int limit, int last, int b0, const bool (&ok)[2], int grp,
                                            float (&s)[8], VRows& v, bool& found) {
  uint32_t odd = 0u;
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    const int b = b0 + x;
    const int dir = ok[x] ? entry_direction(a.dir, a.cls, a.dir_per_entry, a.max_blocks_per_seq, seq, b) : 1;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int at = b * kBlockSize + slot_of_offset(slot_of(grp, r), dir);
      if (!ok[x] || at >= limit) s[4 * x + r] = -INFINITY;
      if (!ok[x] || at >= last) {
        v.row[x][r] = v2u_t{0u, 0u};
        v.scales[x] &= ~(0xffu << (8 * r));   // (0 times 2^-127)
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) odd |= (v.row[x][r][i] & 0x7f7f7f7fu) + 0x01010101u;
    }
    odd |= ((v.scales[x] & 0x7f7f7f7fu) + 0x09090909u) & v.scales[x];   // scale bytes from 247 on
  }
  if (__builtin_amdgcn_ballot_w64((odd & 0x80808080u) != 0u) == 0) return;
#pragma unroll
  for (int x = 0; x < 2; ++x) {
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const uint32_t scale = (v.scales[x] >> (8 * r)) & 0xffu;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint32_t m = odd_ones(v.row[x][r][i], scale);
        found |= m != 0u;
        v.row[x][r][i] &= ~(m * 255u);
      }
      if (scale == 255u) v.scales[x] &= ~(0xffu << (8 * r));
    }
  }
}

// After the last pair, where a wave found such values (rare): the pairs that mask_causal cleaned once
// more (fold_pairs: those that not every column sees whole, or with a block outside the pool), and
// NaN where a column sees one, by a product of their places and what the columns see.
__device__ __forceinline__ void spoil_pairs(const PrefillArgs& a, const Q8Pool& pool, int seq, int g, int limit, int last, int first,
                                            int b1, int plain, Running& run) {
  const int lane = threadIdx.x & (kWave - 1);
  const int grp = lane >> 4;
  const int col = lane & 15;
  for (int b0 = first; b0 < b1; b0 += 2 * kWaves) {
    bool ok[2];
    size_t tile[2];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const int e = load_uniform(a.block_tables, (size_t)seq * a.max_blocks_per_seq + min(b0 + x, b1 - 1));
      ok[x] = b0 + x < b1 && e >= 0 && e < a.num_blocks;
      tile[x] = (size_t)(ok[x] ? e : 0) * a.num_kv_heads + g;
    }
    if (ok[0] && ok[1] && (b0 + 2) * kBlockSize <= plain) continue;
    VRegs raw;
    issue_v(pool, tile[0], tile[1], grp, col, raw);
    VRows v = exchange(raw, pair_scales(raw.scales));
    uint32_t seen[4] = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const int b = b0 + x;
      const int dir = ok[x] ? entry_direction(a.dir, a.cls, a.dir_per_entry, a.max_blocks_per_seq, seq, b) : 1;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int at = b * kBlockSize + slot_of_offset(slot_of(grp, r), dir);
        const uint32_t scale = (v.scales[x] >> (8 * r)) & 0xffu;
#pragma unroll
        for (int i = 0; i < 2; ++i) v.row[x][r][i] = ok[x] && at < last ? odd_ones(v.row[x][r][i], scale) : 0u;
        if (ok[x] && at < limit) seen[2 * x + r / 2] |= r % 2 ? 0x3f800000u : 0x3f80u;
      }
    }
    run.spoil(v, seen);
  }
}

// Rows [j0, j0 + 16 / G) of sequence s, KV head g.
struct Group {
  int s, g, j0, q_begin, n, c0, ctx;
};
template <int G>
__device__ __forceinline__ bool find_group(const PrefillArgs& a, Group& u) {
  constexpr int P = 16 / G;
  const int lane = threadIdx.x & (kWave - 1);
  u.g = blockIdx.x % a.num_kv_heads;
  const int x = gridDim.x / a.num_kv_heads - 1 - blockIdx.x / a.num_kv_heads;   // (the longest rows of a chunk first)
  // Sequence s has the groups cu_q[s] / P + s and on: the last one that starts at or below x.
  u.s = -1;
  for (int s0 = 0; s0 < a.num_seqs; s0 += kWave) {
    const int i = s0 + lane;
    const bool below = i < a.num_seqs && a.cu_q[min(i, a.num_seqs - 1)] / P + i <= x;
    const int c = __builtin_popcountll(__builtin_amdgcn_ballot_w64(below));
    if (c > 0) u.s = s0 + c - 1;
    if (c < kWave) break;
  }
  if (u.s < 0) return false;
  u.q_begin = load_uniform(a.cu_q, u.s);
  u.n = load_uniform(a.cu_q, u.s + 1) - u.q_begin;
  const int ctx_s = load_uniform(a.ctx_lens, u.s);
  u.j0 = (x - (u.q_begin / P + u.s)) * P;
  u.c0 = ctx_s - u.n;
  u.ctx = min(ctx_s, min(a.max_ctx, a.max_blocks_per_seq * kBlockSize));
  return u.q_begin >= 0 && u.n > 0 && u.q_begin + u.n <= a.num_q_tokens && u.j0 >= 0 && u.j0 < u.n && ctx_s >= u.n;
}
// Output row of the group's column c.
template <int G>
__device__ __forceinline__ size_t out_row(const PrefillArgs& a, const Group& u, int c) {
  return (size_t)(u.q_begin + u.j0 + c / G) * a.num_q_heads + u.g * G + c % G;
}

// Blocks [sp S, (sp + 1) S) of what group blockIdx.x sees, S = split_blocks (even) and sp = blockIdx.y:
// all of it where it has no more than S blocks, else a partial in slot (group * pieces + sp) * 16 + column.
template <int G>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(3))) void prefill_q8_rows_kernel(PrefillArgs a, Q8Pool pool, int split_blocks) {
  constexpr int P = 16 / G;   // positions of a group
  __shared__ float s_o[kWaves][16][kHeadDim + 4];
  __shared__ float s_m[kWaves][16], s_l[kWaves][16];
  const int tid = threadIdx.x;
  const int lane = tid & (kWave - 1);
  const int w = wave_id_uniform();
  const int grp = lane >> 4;
  const int col = lane & 15;
  Group u;
  if (!find_group<G>(a, u)) return;
  const int j = min(u.j0 + col / G, u.n - 1);                      // the lane's row (behind the chunk: its last)
  const int limit = min(u.ctx, u.c0 + j + 1);                      // positions its column sees,
  const int last = min(u.ctx, u.c0 + min(u.j0 + P, u.n));          // any column,
  const int plain = min(u.ctx, u.c0 + u.j0 + 1);                   // and every one
  const int nblk = (last + kBlockSize - 1) / kBlockSize;
  const int b0 = blockIdx.y * split_blocks, b1 = min(nblk, b0 + split_blocks);
  if (b0 > 0 && b0 >= nblk) return;
  const size_t head = (size_t)(u.q_begin + j) * a.num_q_heads + u.g * G + col % G;
  Running run;
  run.clear();
  bool found = false;
  fold_pairs<2 * kWaves, false>(a, pool, u.s, u.g, head, b0 + 2 * w, b1, plain, true, run,
                                [&](int b, const bool (&ok)[2], float (&sc)[8], VRows& v) { mask_causal(a, u.s, limit, last, b, ok, grp, sc, v, found); });
  if (__builtin_amdgcn_ballot_w64(found) != 0) spoil_pairs(a, pool, u.s, u.g, limit, last, b0 + 2 * w, b1, plain, run);

  const float l = run.total();
  run.store(s_o[w][col], grp);
  if (grp == 0) {
    s_m[w][col] = run.m_ref;
    s_l[w][col] = l;
  }
  __syncthreads();
  for (int i = tid; i < 16 * (kHeadDim / 2); i += kThreads) {
    const int c = i / (kHeadDim / 2), d = 2 * (i % (kHeadDim / 2));
    if (u.j0 + c / G >= u.n) break;   // (a later c is a later row)
    float M = kNoMax;
#pragma unroll
    for (int y = 0; y < kWaves; ++y) M = fmaxf(M, s_m[y][c]);
    float L = 0.0f, A0 = 0.0f, A1 = 0.0f;
#pragma unroll
    for (int y = 0; y < kWaves; ++y) {
      const float wt = fast_exp2(s_m[y][c] - M);
      const float2 o = *reinterpret_cast<const float2*>(&s_o[y][c][d]);
      L = fmaf(s_l[y][c], wt, L);
      A0 = fmaf(o.x, wt, A0);
      A1 = fmaf(o.y, wt, A1);
    }
    if (nblk > split_blocks) {
      const size_t slot = ((size_t)blockIdx.x * gridDim.y + blockIdx.y) * 16 + c;
      *reinterpret_cast<float2*>(a.ws_o + slot * kHeadDim + d) = make_float2(A0, A1);
      if (d == 0) {
        a.ws_ml[2 * slot] = M;
        a.ws_ml[2 * slot + 1] = L;
      }
      continue;
    }
    const float inv = L > 0.0f ? 1.0f / L : 0.0f;
    *reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(a.out) + out_row<G>(a, u, c) * kHeadDim + d) = q8::pack2_bf16(A0 * inv, A1 * inv);
  }
}

// Folds the pieces of a group, o = sum_i 2^(m_i - M) acc_i / sum_i 2^(m_i - M) l_i: four columns a
// workgroup (blockIdx.y), a thread two dims of one.
template <int G>
__global__ __launch_bounds__(kThreads) void prefill_q8_rows_merge_kernel(PrefillArgs a, int split_blocks, int pieces) {
  constexpr int kRound = 8;   // partials requested at once
  Group u;
  if (!find_group<G>(a, u)) return;
  const int nblk = (min(u.ctx, u.c0 + min(u.j0 + 16 / G, u.n)) + kBlockSize - 1) / kBlockSize;
  if (nblk <= split_blocks) return;   // (written whole)
  const int n = (nblk + split_blocks - 1) / split_blocks;
  const int c = 4 * blockIdx.y + threadIdx.x / (kHeadDim / 2), d = 2 * (threadIdx.x % (kHeadDim / 2));
  if (u.j0 + c / G >= u.n) return;
  const size_t slot0 = (size_t)blockIdx.x * pieces * 16 + c;
  float M = kNoMax, L = 0.0f, A0 = 0.0f, A1 = 0.0f;
  for (int i = 0; i < n; i += kRound) {   // indices clamped in range
    float2 x[kRound], v[kRound];
#pragma unroll
    for (int y = 0; y < kRound; ++y) {
      const size_t slot = slot0 + 16 * (size_t)min(i + y, n - 1);
      x[y] = *reinterpret_cast<const float2*>(a.ws_ml + 2 * slot);
      v[y] = *reinterpret_cast<const float2*>(a.ws_o + slot * kHeadDim + d);
    }
    float Mn = M;
#pragma unroll
    for (int y = 0; y < kRound; ++y) Mn = fmaxf(Mn, x[y].x);
    const float alpha = fast_exp2(M - Mn);
    L *= alpha;
    A0 *= alpha;
    A1 *= alpha;
    M = Mn;
#pragma unroll
    for (int y = 0; y < kRound; ++y) {
      const bool use = i + y < n;   // (the rest of a round repeats a partial)
      const float wt = use ? fast_exp2(x[y].x - M) : 0.0f;
      L = fmaf(use ? x[y].y : 0.0f, wt, L);
      A0 = fmaf(use ? v[y].x : 0.0f, wt, A0);
      A1 = fmaf(use ? v[y].y : 0.0f, wt, A1);
    }
  }
  const float inv = L > 0.0f ? 1.0f / L : 0.0f;
  *reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(a.out) + out_row<G>(a, u, c) * kHeadDim + d) = q8::pack2_bf16(A0 * inv, A1 * inv);
}

// Launches the groups where they are the better arrangement; false: not taken.
template <int G>
bool launch_rows(const PrefillArgs& a, const uint8_t* scales, hipStream_t stream, hipError_t* e) {
  const int64_t groups = ((int64_t)(a.num_q_tokens / (16 / G)) + a.num_seqs) * a.num_kv_heads;
  const int64_t blocks = std::min<int64_t>((a.max_ctx + kBlockSize - 1LL) / kBlockSize, a.max_blocks_per_seq);
  int32_t split = 0, pieces = 0;
  if (!plan_q8_prefill_rows(groups, blocks, stream_compute_units(stream), (int64_t)a.ws_slots * pf::kRows, &split, &pieces)) return false;
  const Q8Pool pool{static_cast<const uint8_t*>(a.k_pool), static_cast<const uint8_t*>(a.v_pool), scales};
  hipLaunchKernelGGL(prefill_q8_rows_kernel<G>, dim3((unsigned)groups, (unsigned)pieces), dim3(kThreads), 0, stream, a, pool, split);
  *e = hipGetLastError();
  if (*e != hipSuccess || pieces == 1) return true;
  hipLaunchKernelGGL(prefill_q8_rows_merge_kernel<G>, dim3((unsigned)groups, 4), dim3(kThreads), 0, stream, a, split, pieces);
  *e = hipGetLastError();
  return true;
}

}  // namespace dq

namespace {

template <int G>
hipError_t launch_chunks(const PrefillArgs& a, const uint8_t* scales, int num_units, hipStream_t stream) {
  hipError_t e = hipSuccess;
  return dq::launch_rows<G>(a, scales, stream, &e) ? e : pf::launch_q8_group<G>(a, scales, num_units, stream);
}

}  // namespace

hipError_t launch_prefill_q8(PrefillArgs a, const uint8_t* scales, int group, int num_tiles_total, hipStream_t stream) {
  if (num_tiles_total <= 0) return hipSuccess;
  switch (group) {
    case 1: return launch_chunks<1>(a, scales, num_tiles_total, stream);
    case 2: return launch_chunks<2>(a, scales, num_tiles_total, stream);
    case 4: return launch_chunks<4>(a, scales, num_tiles_total, stream);
    case 8: return launch_chunks<8>(a, scales, num_tiles_total, stream);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace bros
