// bros_attn_decode_q8 on gfx950: one bf16 query row per sequence over the 8-bit
// cache. decode_q8_device.h says what a step computes and how its operands lie.
//
// For short contexts and few rows a workgroup takes a whole (row, KV head) segment, or
// split_blocks blocks of it; wave w takes every fourth pair of blocks, and the waves'
// results are folded in LDS. Pieces of one segment leave partials (max, sum,
// unnormalised output) that a second kernel folds, the one of the 16-bit decode's
// pieces. Large batches run the even split below (plan.h says which calls).
//
// Memory bounds the large ones (820 us for the 4.94 GB of 288 rows of 256 to 16384 tokens, 64 / 8
// heads; 108 us for the 0.59 GB of 64 rows of 128 to 8192, 32 / 8 heads, 4.4 of them the merge), the
// launch and the chain context, table entry, rows the small ones (six rows of up to
// 2000 tokens 7.4 us and 2.3 the merge of their pieces).
#include "decode_q8_device.h"
#include "plan.h"

#include <algorithm>

namespace bros {
namespace dq {

// Pairs whose loads a wave of the even split keeps in flight (register sets).
constexpr int kDepth = 2;

// One wave of a worker of the even split (decode_q8_even_kernel): head `hh` of the
// H heads of the pairs [t0, t0 + n) in (row, group of H KV heads, pair) order
// (n >= 1). a.num_kv_heads counts the groups; `wid` names the worker's partials.
template <int G, int H>
__device__ __forceinline__ void even_worker(const DecodeArgs& a, const Q8Pool& pool, const int* s_pre, int chunk, int nch,
                                            int wid, int hh, int t0, int n, const dm::Shares& shares) {
  const int lane = threadIdx.x & (kWave - 1);
  const int grp = lane >> 4;
  const int col = lane & 15;
  const bool head_lane = col < G;
  const int groups = a.num_kv_heads;
  const int nkv = groups * H;
  const int Hq = a.num_q_heads;

  // Where a pair lies: its cursor, and its blocks' pool tiles (tile g of block 0 in
  // place of one that is not there: masked whole).
  struct Pair {
    dm::Cursor c;
    size_t tile[2];
    bool ok[2];
  };
  auto entries = [&](Pair& p) {
    const int nb = (p.c.ctx + kBlockSize - 1) / kBlockSize;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const int b = 2 * p.c.b + x;
      const int e = load_uniform(a.block_tables, (size_t)p.c.s * a.max_blocks_per_seq + min(b, nb - 1));
      p.ok[x] = b < nb && e >= 0 && e < a.num_blocks;
      p.tile[x] = (size_t)(p.ok[x] ? e : 0) * nkv + (p.c.g * H + hh);
    }
  };
  // Past the share: rows that every worker's last loads read, so that they come from the caches
  // (64 rows of 128 to 8192 tokens, 32 / 8 heads: 108.3 us a call; 109.0 where each read its last pair again).
  auto nothing = [&](Pair& p) { p.tile[0] = p.tile[1] = (size_t)hh; };
  auto first_head = [&](const Pair& p) -> size_t { return (size_t)p.c.row * Hq + (p.c.g * H + hh) * G; };   // of q and out
  v4u_t qf[4];
  KRegs k_[kDepth];
  VRegs v_[kDepth];
  Running run;
  run.clear();

  Pair cur[kDepth + 2];   // cur[d]: pair i + d (entries are read one pair before their loads issue)
  dm::locate<kPairSlots>(a, s_pre, chunk, nch, t0, cur[0].c);
  entries(cur[0]);
  issue_k(pool, cur[0].tile[0], cur[0].tile[1], grp, col, k_[0]);
  load_q<G>(a.q, first_head(cur[0]), grp, col, qf);
  issue_v(pool, cur[0].tile[0], cur[0].tile[1], grp, col, v_[0]);
  bool whole = cur[0].c.b == 0;   // this wave saw the segment's first pair
#pragma unroll
  for (int d = 1; d <= kDepth; ++d) {
    cur[d] = cur[d - 1];
    if (d < n) {
      dm::advance<kPairSlots>(a, cur[d].c);
      entries(cur[d]);
    } else {
      nothing(cur[d]);
    }
    if (d < kDepth) {
      issue_k(pool, cur[d].tile[0], cur[d].tile[1], grp, col, k_[d]);
      issue_v(pool, cur[d].tile[0], cur[d].tile[1], grp, col, v_[d]);
    }
  }
  cur[kDepth + 1] = cur[kDepth];

  // Pair i, its rows in (k, v).
  auto body = [&](int i, KRegs& k, VRegs& v) __attribute__((always_inline)) {
    Pair& p = cur[0];
    cur[kDepth + 1] = cur[kDepth];
    if (i + kDepth + 1 < n) {
      dm::advance<kPairSlots>(a, cur[kDepth + 1].c);
      entries(cur[kDepth + 1]);
    } else {
      nothing(cur[kDepth + 1]);
    }
    float s[8];
    const PairScales ps = pair_scales(v.scales);
    pair_scores(k, qf, ps, a.scale_log2, s);
    const bool last = p.c.b == p.c.nblk - 1;
    const bool seg_end = last || i + 1 == n;
    if (i + 1 == n) {
      // the cut list: the segment this worker started and leaves unfinished, and the
      // worker that holds its last pair
      const bool starts_cut = whole && !last;
      if (lane == 0 && hh == 0) {
        a.ws_cut[2 * wid] = starts_cut ? p.c.row * groups + p.c.g : -1;
        a.ws_cut[2 * wid + 1] = starts_cut ? shares.holder(t0 + i + (p.c.nblk - 1 - p.c.b)) : -1;
      }
    }
    // (past the share: no branch, see `nothing`)
    issue_k(pool, cur[kDepth].tile[0], cur[kDepth].tile[1], grp, col, k);
    if (i + 1 < n && seg_end) load_q<G>(a.q, first_head(cur[1]), grp, col, qf);
    VRows rows = exchange(v, ps);
    if (!p.ok[0] || !p.ok[1] || last) mask_pair(a, p.c.row, p.c.ctx, 2 * p.c.b, p.ok, grp, s, rows);
    run.fold<true>(s, rows, head_lane);
    // (V's registers are free before the fold, but requested there they come no sooner
    // and everything takes longer: 848 us against 832 in the case above)
    asm volatile("" ::: "memory");
    issue_v(pool, cur[kDepth].tile[0], cur[kDepth].tile[1], grp, col, v);

    if (seg_end) {
      const float l_head = run.total();
      const bool direct = whole && last;   // the whole segment was this wave's
      if (head_lane) {
        if (direct) {
          const float inv = l_head > 0.0f ? 1.0f / l_head : 0.0f;
          run.store_bf16(static_cast<uint16_t*>(a.out) + (first_head(p) + col) * kHeadDim, grp, inv);
        } else {
          const size_t slot = (((size_t)p.c.row * groups + p.c.g + wid) * H + hh) * G + col;   // partial (run + worker)
          run.store(a.ws_acc + slot * kHeadDim, grp);
          if (grp == 0) {
            a.ws_ml[2 * slot] = run.m_ref;
            a.ws_ml[2 * slot + 1] = l_head;
          }
        }
      }
      run.clear();
      whole = true;
    }
#pragma unroll
    for (int d = 0; d <= kDepth; ++d) cur[d] = cur[d + 1];
  };
#pragma clang loop unroll(disable)
  for (int i = 0; i < n; i += kDepth) {
#pragma unroll
    for (int d = 0; d < kDepth; ++d) {
      if (i + d >= n) break;
      body(i + d, k_[d], v_[d]);
    }
  }
}

__device__ __forceinline__ int row_context(const DecodeArgs& a, int row) {
  return max(0, min(load_uniform(a.ctx_lens, row), min(a.max_ctx, a.max_blocks_per_seq * kBlockSize)));
}

// Folds pairs first, first + STRIDE, ... of blocks below b1 of a (row, KV head) segment into `run`.
template <int G, int STRIDE>
__device__ __forceinline__ void fold_segment(const DecodeArgs& a, const Q8Pool& pool, int row, int g, int ctx, int first, int b1,
                                             Running& run) {
  const int lane = threadIdx.x & (kWave - 1);
  const int grp = lane >> 4;
  const int col = lane & 15;
  const size_t head = (size_t)row * a.num_q_heads + g * G + min(col, G - 1);
  fold_pairs<STRIDE, true>(a, pool, row, g, head, first, b1, ctx, col < G, run,
                     [&](int b, const bool (&ok)[2], float (&s)[8], VRows& v) { mask_pair(a, row, ctx, b, ok, grp, s, v); });
}

// Many short contexts (plan.h: q8_decode_by_waves): a wave takes whole segments, x, x + W, ... of
// W waves, four neighbours to a workgroup. Nothing to fold, no barrier, a quarter of the
// workgroups: 512 rows of 10 to 100 tokens, 64 / 8 heads, 32.6 us with a workgroup per segment, 23.1
// here; 128 of 6 to 60, 32 / 8 heads, 10.2 and 7.1. (A workgroup of four waves for every four
// segments, none taking a second: 26.7 and 6.9. The next segment's loads requested before a
// segment ends: 22.1 and 7.0, and slower from 200 tokens on.)
constexpr int kWavesPerSimd = 3;
template <int G>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(kWavesPerSimd))) void decode_q8_wave_kernel(DecodeArgs a, Q8Pool pool) {
  const int lane = threadIdx.x & (kWave - 1);
  const int col = lane & 15;
  const int total = a.num_rows * a.num_kv_heads;
#pragma clang loop unroll(disable)
  for (int seg = blockIdx.x * kWaves + wave_id_uniform(); seg < total; seg += gridDim.x * kWaves) {
    const int row = seg / a.num_kv_heads, g = seg - row * a.num_kv_heads;
    const int ctx = row_context(a, row);
    Running run;
    run.clear();
    fold_segment<G, 2>(a, pool, row, g, ctx, 0, (ctx + kBlockSize - 1) / kBlockSize, run);
    const float l = run.total();
    if (col < G)
      run.store_bf16(static_cast<uint16_t*>(a.out) + ((size_t)row * a.num_q_heads + g * G + col) * kHeadDim, lane >> 4,
                     l > 0.0f ? 1.0f / l : 0.0f);   // (a row without context is zeros)
  }
}

// Blocks [sp S, (sp + 1) S) of segment seg0 + blockIdx.x, S = split_blocks (even) and
// sp = blockIdx.y: the whole segment when it has no more than S blocks, else a
// partial in slot (segment * n_split_max + sp) * G + head.
template <int G>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(kWavesPerSimd))) void decode_q8_kernel(DecodeArgs a, Q8Pool pool, int seg0) {
  __shared__ float s_o[kWaves][G][kHeadDim + 4];
  __shared__ float s_m[kWaves][G], s_l[kWaves][G];
  const int tid = threadIdx.x;
  const int lane = tid & (kWave - 1);
  const int w = wave_id_uniform();
  const int grp = lane >> 4;
  const int col = lane & 15;
  const bool head_lane = col < G;
  const int nkv = a.num_kv_heads;
  const int Hq = a.num_q_heads;
  const int seg = seg0 + (int)blockIdx.x;
  const int row = seg / nkv, g = seg - row * nkv;
  const int ctx = row_context(a, row);
  const int nblk = (ctx + kBlockSize - 1) / kBlockSize;
  const int sp = blockIdx.y;
  const int b0 = sp * a.split_blocks, b1 = min(nblk, b0 + a.split_blocks);
  if (sp > 0 && b0 >= nblk) return;
  Running run;
  run.clear();
  fold_segment<G, 2 * kWaves>(a, pool, row, g, ctx, b0 + 2 * w, b1, run);   // this wave's pairs: every fourth

  // The waves' results.
  const float l_head = run.total();
  if (head_lane) {
    run.store(s_o[w][col], grp);
    if (grp == 0) {
      s_m[w][col] = run.m_ref;
      s_l[w][col] = l_head;
    }
  }
  __syncthreads();
  for (int i = tid; i < G * (kHeadDim / 2); i += kThreads) {
    const int h = i / (kHeadDim / 2), d = 2 * (i % (kHeadDim / 2));
    float M = kNoMax;
#pragma unroll
    for (int x = 0; x < kWaves; ++x) M = fmaxf(M, s_m[x][h]);
    float L = 0.0f, A0 = 0.0f, A1 = 0.0f;
#pragma unroll
    for (int x = 0; x < kWaves; ++x) {
      const float wt = fast_exp2(s_m[x][h] - M);
      const float2 o = *reinterpret_cast<const float2*>(&s_o[x][h][d]);
      L = fmaf(s_l[x][h], wt, L);
      A0 = fmaf(o.x, wt, A0);
      A1 = fmaf(o.y, wt, A1);
    }
    if (nblk > a.split_blocks) {
      const size_t slot = ((size_t)seg * a.n_split_max + sp) * G + h;
      *reinterpret_cast<float2*>(a.ws_acc + slot * kHeadDim + d) = make_float2(A0, A1);
      if (d == 0) {
        a.ws_ml[2 * slot] = M;
        a.ws_ml[2 * slot + 1] = L;
      }
      continue;
    }
    const float inv = L > 0.0f ? 1.0f / L : 0.0f;   // (a row without context is zeros)
    uint32_t* out = reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(a.out) + ((size_t)row * Hq + g * G + h) * kHeadDim + d);
    *out = q8::pack2_bf16(A0 * inv, A1 * inv);
  }
}

// The even split. A run is the pairs of H neighbouring KV heads of a row, and a worker
// H waves, one per head: the worker takes an equal contiguous share of all pairs in
// (row, group of heads, pair) order, its waves walk it side by side. A block's rows of
// H heads lie side by side in the pool, so the waves' reads of a block meet in 2 H KiB
// of it, and in the H heads' 32 H bytes of scales, where one head's tile alone is 2 KiB.
// Runs cut between workers leave partials in slot ((run + worker) * H + head) * G +
// head-in-group, unique as both are in order; the merge folds them.
template <int G, int H>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2))) void decode_q8_even_kernel(DecodeArgs a, Q8Pool pool) {
  __shared__ int s_pre[kMaxRowsLds + 1];
  __shared__ int s_scan[kWaves];
  constexpr int W = kWaves / H;   // workers of a workgroup
  const int chunk = (a.num_rows + kMaxRowsLds - 1) / kMaxRowsLds;
  const int nch = (a.num_rows + chunk - 1) / chunk;
  const int total = dm::build_tile_prefix<kPairSlots>(a, s_pre, s_scan, chunk, nch);
  const dm::Shares shares(a, total);
  const int workers = shares.workers;
  const int wave = wave_id_uniform();
  const int hh = wave % H;
  // (fewer workers than the grid holds are spread over the workgroups)
  const int wid = workers < a.num_workers ? wave / H * gridDim.x + blockIdx.x : blockIdx.x * W + wave / H;
  if (wid >= workers) {
    if (hh == 0 && (threadIdx.x & (kWave - 1)) == 0) a.ws_cut[2 * wid] = -1;   // idle: nothing to merge
    return;
  }
  int t0 = shares.start(wid), t1 = shares.start(wid + 1);
  asm volatile("" : "+v"(t0), "+v"(t1));
  even_worker<G, H>(a, pool, s_pre, chunk, nch, wid, hh, t0, t1 - t0, shares);
}

// The merge: workgroups (w, y) fold the run that worker w started and left unfinished (its
// entry of the cut list names the run and the worker of its last pair), o = sum_i
// 2^(m_i - M) acc_i / sum_i 2^(m_i - M) l_i over the partials of the workers between, four heads
// each, a thread two dims of one. Workgroups behind the workers' write the zeros of
// rows without context, one wave a row. (One workgroup for all heads of a run, in
// passes, took 7.2 us after 64 rows of 128 to 8192 tokens.)
constexpr int kRound = 8;   // partials requested at once

template <int HG>   // query heads of a run
__global__ __launch_bounds__(kThreads) void decode_q8_merge_kernel(DecodeArgs a) {
  const int w = blockIdx.x;
  if (w >= a.num_workers) {
    if (blockIdx.y > 0) return;
    const int row = (w - a.num_workers) * kWaves + wave_id_uniform();
    if (row >= a.num_rows) return;
    int s, ctx;
    resolve_row(a, row, s, ctx);
    if (ctx > 0) return;
    uint32_t* z = reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(a.out) + (size_t)row * a.num_q_heads * kHeadDim);
    for (int i = threadIdx.x & (kWave - 1); i < a.num_q_heads * kHeadDim / 2; i += kWave) z[i] = 0u;
    return;
  }
  const int run = load_uniform(a.ws_cut, 2 * (size_t)w);
  if (run < 0) return;
  const int w1 = load_uniform(a.ws_cut, 2 * (size_t)w + 1);
  const int n = w1 - w + 1;
  const size_t slot0 = ((size_t)run + w) * HG;
  const int i = blockIdx.y * kThreads + threadIdx.x;
  if (i < HG * (kHeadDim / 2)) {
    const int h = i / (kHeadDim / 2), d = 2 * (i % (kHeadDim / 2));
    const float2* ml = reinterpret_cast<const float2*>(a.ws_ml) + slot0 + h;
    const float* acc = a.ws_acc + (slot0 + h) * kHeadDim + d;
    float M = kNoMax, L = 0.0f, A0 = 0.0f, A1 = 0.0f;
    for (int c = 0; c < n; c += kRound) {   // indices clamped in range
      float2 x[kRound], v[kRound];
#pragma unroll
      for (int u = 0; u < kRound; ++u) {
        const int j = min(c + u, n - 1);
        x[u] = ml[(size_t)j * HG];
        v[u] = *reinterpret_cast<const float2*>(acc + (size_t)j * HG * kHeadDim);
      }
      float Mn = M;
#pragma unroll
      for (int u = 0; u < kRound; ++u) Mn = fmaxf(Mn, x[u].x);
      const float alpha = fast_exp2(M - Mn);
      L *= alpha;
      A0 *= alpha;
      A1 *= alpha;
      M = Mn;
#pragma unroll
      for (int u = 0; u < kRound; ++u) {
        // (a round's padding adds zero by selection: the partial it repeats may hold a NaN)
        const bool use = c + u < n;
        const float wt = use ? fast_exp2(x[u].x - M) : 0.0f;
        L = fmaf(use ? x[u].y : 0.0f, wt, L);
        A0 = fmaf(use ? v[u].x : 0.0f, wt, A0);
        A1 = fmaf(use ? v[u].y : 0.0f, wt, A1);
      }
    }
    const float inv = L > 0.0f ? 1.0f / L : 0.0f;
    // (a run's heads are neighbours, and runs are in the order of rows and heads)
    *reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(a.out) + ((size_t)run * HG + h) * kHeadDim + d) =
        q8::pack2_bf16(A0 * inv, A1 * inv);
  }
}

template <int G, int H>
hipError_t launch_even(DecodeArgs a, Q8Pool pool, hipStream_t stream, int slot, int cus) {
  // (the workspace's partials: a slot per query row and kDecodeGroupSlots groups of heads)
  const int wgs = std::min(workgroups_per_cu(reinterpret_cast<const void*>(&decode_q8_even_kernel<G, H>), kThreads, slot) * cus,
                           kDecodeGroupSlots / kWaves);
  a.num_kv_heads /= H;
  a.num_workers = wgs * (kWaves / H);
  hipLaunchKernelGGL((decode_q8_even_kernel<G, H>), dim3(wgs), dim3(kThreads), 0, stream, a, pool);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(decode_q8_merge_kernel<G * H>, dim3(a.num_workers + (a.num_rows + kWaves - 1) / kWaves, (G * H + 3) / 4), dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

constexpr long long kMaxSegmentsPerLaunch = 1 << 23;   // (a launch's threads must stay below 2^32)

template <int G>
hipError_t launch_group(DecodeArgs a, Q8Pool pool, hipStream_t stream, int slot) {
  const int64_t segments = (int64_t)a.num_rows * a.num_kv_heads;
  const int32_t blocks = longest_blocks(a.max_ctx, a.max_blocks_per_seq);
  // (partials: the workspace has a slot per query row and kDecodeGroupSlots groups more)
  const int64_t slots = (int64_t)a.num_rows * a.num_q_heads + (int64_t)kDecodeGroupSlots * std::min(a.num_q_heads, 8);
  const int cus = stream_compute_units(stream);
  if (q8_decode_by_waves(segments, blocks, cus)) {
    const int64_t wgs = std::min<int64_t>((segments + kWaves - 1) / kWaves, kWavesPerSimd * (int64_t)cus);   // (four SIMDs, four waves)
    hipLaunchKernelGGL(decode_q8_wave_kernel<G>, dim3((unsigned)wgs), dim3(kThreads), 0, stream, a, pool);
    return hipGetLastError();
  }
  if (!plan_q8_decode(segments, G, blocks, cus, slots, &a.split_blocks, &a.n_split_max)) {
    if (a.num_kv_heads % 4 == 0) return launch_even<G, 4>(a, pool, stream, slot + 2, cus);
    if (a.num_kv_heads % 2 == 0) return launch_even<G, 2>(a, pool, stream, slot + 1, cus);
    return launch_even<G, 1>(a, pool, stream, slot, cus);
  }
  for (int64_t s0 = 0; s0 < segments; s0 += kMaxSegmentsPerLaunch) {
    const dim3 grid((unsigned)std::min<int64_t>(segments - s0, kMaxSegmentsPerLaunch), (unsigned)a.n_split_max);
    hipLaunchKernelGGL(decode_q8_kernel<G>, grid, dim3(kThreads), 0, stream, a, pool, (int)s0);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return a.n_split_max > 1 ? launch_decode_pieces_merge(a, G, stream) : hipSuccess;
}

}  // namespace dq

hipError_t launch_decode_q8(DecodeArgs a, Q8Pool pool, int group, hipStream_t stream) {
  switch (group) {
    case 1: return dq::launch_group<1>(a, pool, stream, 8);
    case 2: return dq::launch_group<2>(a, pool, stream, 11);
    case 4: return dq::launch_group<4>(a, pool, stream, 14);
    case 8: return dq::launch_group<8>(a, pool, stream, 17);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace bros
