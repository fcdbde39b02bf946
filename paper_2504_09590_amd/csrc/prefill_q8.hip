// bros_attn_prefill_chunk_q8: the matrix-core prefill (prefill_device.h) over an
// 8-bit pool. Units, pieces and their merge are the 16-bit prefill's.
//
// The matrix cores bound it from a few dozen rows on: 512 rows on 16000 cached tokens,
// 32 / 8 heads, 144 us, 946 TFLOP/s of the formula's products (the 16-bit prefill 143 us; a
// large library product 1208 TFLOP/s). Few rows on short contexts run in smaller groups (below).
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
  __shared__ __attribute__((aligned(16))) uint16_t s_nan[kGuardKeys * 8];   // per key and 16 dims: values that are not numbers
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

// Few rows (plan.h: q8_prefill_by_rows): the decode's steps (decode_q8_device.h), their 16 columns
// filled with 16 / G positions of G heads. A workgroup takes 16 columns; wave w folds every fourth
// pair of blocks into a running result of its own, and the four meet in LDS.
//
// In the other kernel a prompt of 301 rows is 80 chains of up to ten steps, one after another, behind a
// start of 9 us (Q's terms, the first tiles, their conversion); here it is 600 workgroups of at most three
// steps a wave. Latency bounds it: 5.2 us for 16 rows, 10.6 for the 301 (14.6 there). K and V are read
// once per 16 columns, from L2. (Two bf16 parts for the weights, as in the decode, take 2 to 8 % longer;
// the marks of values that are not numbers made inside the step spill or take 0.4 us more.)

// The bytes of w that are the NaN code as ones, all of them where the row's scale is none.
__device__ __forceinline__ uint32_t not_numbers(uint32_t w, uint32_t scale) {
  return scale == 255u ? 0x01010101u : (((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) >> 7;
}

// Removes what the lane's column does not see of a pair (slots from `limit` on) and, by selection, V
// rows that no column does (from `last` on). A row that only some columns see must not reach the
// others through 0 * NaN: its values that are not numbers become zeros, and `found` is set.
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
    odd |= ((v.scales[x] & 0x7f7f7f7fu) + 0x01010101u) & v.scales[x];
  }
  if (__builtin_amdgcn_ballot_w64((odd & 0x80808080u) != 0u) == 0) return;
#pragma unroll
  for (int x = 0; x < 2; ++x) {
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const uint32_t scale = (v.scales[x] >> (8 * r)) & 0xffu;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint32_t m = not_numbers(v.row[x][r][i], scale);
        found |= m != 0u;
        v.row[x][r][i] &= ~(m * 255u);
      }
      if (scale == 255u) v.scales[x] &= ~(0xffu << (8 * r));
    }
  }
}

// After the last pair, where a wave found such values (rare): its pairs that not every column
// sees once more, and NaN where a column sees one, by a product of their places and what the
// columns see.
__device__ __forceinline__ void spoil_pairs(const PrefillArgs& a, const Q8Pool& pool, int seq, int g, int limit, int last, int first,
                                            int stride, int plain, Running& run) {
  const int lane = threadIdx.x & (kWave - 1);
  const int grp = lane >> 4;
  const int col = lane & 15;
  const int nblk = (last + kBlockSize - 1) / kBlockSize;
  for (int b0 = first; b0 < nblk; b0 += stride) {
    if ((b0 + 2) * kBlockSize <= plain) continue;
    bool ok[2];
    size_t tile[2];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const int e = load_uniform(a.block_tables, (size_t)seq * a.max_blocks_per_seq + min(b0 + x, nblk - 1));
      ok[x] = b0 + x < nblk && e >= 0 && e < a.num_blocks;
      tile[x] = (size_t)(ok[x] ? e : 0) * a.num_kv_heads + g;
    }
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
        for (int i = 0; i < 2; ++i) v.row[x][r][i] = ok[x] && at < last ? not_numbers(v.row[x][r][i], scale) : 0u;
        if (ok[x] && at < limit) seen[2 * x + r / 2] |= r % 2 ? 0x3f800000u : 0x3f80u;
      }
    }
    run.spoil(v, seen);
  }
}

template <int G>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(3))) void prefill_q8_rows_kernel(PrefillArgs a, Q8Pool pool) {
  constexpr int P = 16 / G;   // positions of a workgroup
  __shared__ float s_o[kWaves][16][kHeadDim + 4];
  __shared__ float s_m[kWaves][16], s_l[kWaves][16];
  const int tid = threadIdx.x;
  const int lane = tid & (kWave - 1);
  const int w = wave_id_uniform();
  const int grp = lane >> 4;
  const int col = lane & 15;
  const int nkv = a.num_kv_heads;
  const int g = blockIdx.x % nkv;
  const int x = gridDim.x / nkv - 1 - blockIdx.x / nkv;   // (the longest rows of a chunk first)
  // Sequence s has the groups of rows cu_q[s] / P + s and on: the last one that starts at or below x.
  int s = -1;
  for (int s0 = 0; s0 < a.num_seqs; s0 += kWave) {
    const int i = s0 + lane;
    const bool below = i < a.num_seqs && a.cu_q[min(i, a.num_seqs - 1)] / P + i <= x;
    const int c = __builtin_popcountll(__builtin_amdgcn_ballot_w64(below));
    if (c > 0) s = s0 + c - 1;
    if (c < kWave) break;
  }
  if (s < 0) return;
  const int q_begin = load_uniform(a.cu_q, s);
  const int n = load_uniform(a.cu_q, s + 1) - q_begin;
  const int ctx_s = load_uniform(a.ctx_lens, s);
  const int j0 = (x - (q_begin / P + s)) * P;
  if (q_begin < 0 || n <= 0 || q_begin + n > a.num_q_tokens || j0 < 0 || j0 >= n || ctx_s < n) return;
  const int ctx = min(ctx_s, min(a.max_ctx, a.max_blocks_per_seq * kBlockSize));
  const int c0 = ctx_s - n;
  const int j = min(j0 + col / G, n - 1);                          // the lane's row (behind the chunk: its last)
  const int limit = min(ctx, c0 + j + 1);                          // positions its column sees
  const int last = min(ctx, c0 + min(j0 + P, n));                  // and any
  const size_t head = (size_t)(q_begin + j) * a.num_q_heads + g * G + col % G;
  Running run;
  run.clear();
  const int plain = min(ctx, c0 + j0 + 1);                         // positions that every column sees
  bool found = false;
  fold_pairs<2 * kWaves, false>(a, pool, s, g, head, 2 * w, (last + kBlockSize - 1) / kBlockSize, plain, true, run,
                         [&](int b, const bool (&ok)[2], float (&sc)[8], VRows& v) { mask_causal(a, s, limit, last, b, ok, grp, sc, v, found); });
  if (__builtin_amdgcn_ballot_w64(found) != 0) spoil_pairs(a, pool, s, g, limit, last, 2 * w, 2 * kWaves, plain, run);

  const float l = run.total();
  run.store(s_o[w][col], grp);
  if (grp == 0) {
    s_m[w][col] = run.m_ref;
    s_l[w][col] = l;
  }
  __syncthreads();
  for (int i = tid; i < 16 * (kHeadDim / 2); i += kThreads) {
    const int c = i / (kHeadDim / 2), d = 2 * (i % (kHeadDim / 2));
    if (j0 + c / G >= n) break;   // (a later c is a later row)
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
    const float inv = L > 0.0f ? 1.0f / L : 0.0f;
    const size_t row = (size_t)(q_begin + j0 + c / G) * a.num_q_heads + g * G + c % G;
    *reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(a.out) + row * kHeadDim + d) = q8::pack2_bf16(A0 * inv, A1 * inv);
  }
}

// Launches the groups where they are the better arrangement; false: not taken.
template <int G>
bool launch_rows(const PrefillArgs& a, const uint8_t* scales, hipStream_t stream, hipError_t* e) {
  const int64_t groups = ((int64_t)(a.num_q_tokens / (16 / G)) + a.num_seqs) * a.num_kv_heads;
  const int64_t blocks = std::min<int64_t>((a.max_ctx + kBlockSize - 1LL) / kBlockSize, a.max_blocks_per_seq);
  if (!q8_prefill_by_rows(groups, blocks, stream_compute_units(stream))) return false;
  const Q8Pool pool{static_cast<const uint8_t*>(a.k_pool), static_cast<const uint8_t*>(a.v_pool), scales};
  hipLaunchKernelGGL(prefill_q8_rows_kernel<G>, dim3((unsigned)groups), dim3(kThreads), 0, stream, a, pool);
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
