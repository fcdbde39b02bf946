// bros_attn_decode_q8 on gfx950: one bf16 query row per sequence over the 8-bit
// cache. decode_q8_device.h says what a step computes and how its operands lie.
//
// A workgroup takes a whole (row, KV head) segment, or split_blocks blocks of it;
// wave w takes every fourth pair of blocks, and the waves' results are folded in LDS. Pieces
// of one segment leave partials (max, sum, unnormalised output) that a second
// kernel folds, the one of the 16-bit decode's pieces.
#include "decode_q8_device.h"

#include <algorithm>

namespace bros {
namespace dq {

// Blocks [sp S, (sp + 1) S) of segment seg0 + blockIdx.x, S = split_blocks (even) and
// sp = blockIdx.y: the whole segment when it has no more than S blocks, else a
// partial in slot (segment * n_split_max + sp) * G + head.
template <int G>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(3))) void decode_q8_kernel(DecodeArgs a, Q8Pool pool, int seg0) {
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
  const int ctx = max(0, min(load_uniform(a.ctx_lens, row), min(a.max_ctx, a.max_blocks_per_seq * kBlockSize)));
  const int nblk = (ctx + kBlockSize - 1) / kBlockSize;
  const int sp = blockIdx.y;
  const int b0 = sp * a.split_blocks, b1 = min(nblk, b0 + a.split_blocks);
  if (sp > 0 && b0 >= nblk) return;
  const int first = b0 + 2 * w;                                                       // this wave's pairs: first, first + 8, ...
  const int n = b1 > first ? (b1 - first + 2 * kWaves - 1) / (2 * kWaves) : 0;

  v4u_t qf[4];
  KRegs k[2];
  VRegs v[2];
  Running run;
  run.clear();

  // Pool tile of the x-th block of this wave's i-th pair: tile 0 of the head in place
  // of an entry outside the pool or past the piece (masked whole), so that the loads
  // need no branch. (The table is not read past the piece.)
  auto entry = [&](int i, int x, bool& ok) -> size_t {
    const int b = first + 2 * kWaves * i + x;
    const int e = load_uniform(a.block_tables, (size_t)row * a.max_blocks_per_seq + min(b, b1 - 1));
    ok = b < b1 && e >= 0 && e < a.num_blocks;
    return (size_t)(ok ? e : 0) * nkv + g;
  };

  if (n > 0) {
    bool ok[2];
    size_t tile[2];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      tile[x] = entry(0, x, ok[x]);
      issue_k(pool, tile[x], grp, col, k[x]);
    }
    load_q<G>(a.q, (size_t)row * Hq + g * G, grp, col, qf);
#pragma unroll
    for (int x = 0; x < 2; ++x) issue_v(pool, tile[x], grp, col, v[x]);
#pragma clang loop unroll(disable)
    for (int i = 0; i < n; ++i) {
      const int b = first + 2 * kWaves * i;
      bool next_ok[2];
#pragma unroll
      for (int x = 0; x < 2; ++x) tile[x] = entry(i + 1, x, next_ok[x]);
      float s[8];
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const floatx4_t sc = block_scores(k[x], qf);
#pragma unroll
        for (int r = 0; r < 4; ++r) s[4 * x + r] = sc[r] * a.scale_log2;
      }
#pragma unroll
      for (int x = 0; x < 2; ++x) issue_k(pool, tile[x], grp, col, k[x]);   // the K registers are free
      if (!ok[0] || !ok[1] || (b + 2) * kBlockSize > ctx) mask_pair(a, row, ctx, b, ok, grp, s, v);
      run.fold(s, v, head_lane);
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        issue_v(pool, tile[x], grp, col, v[x]);   // the V registers are free
        ok[x] = next_ok[x];
      }
    }
  }

  // The waves' results.
  const float l_head = run.total();
  if (head_lane) {
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      float* o = &s_o[w][col][32 * grp + 8 * r];
      *reinterpret_cast<floatx4_t*>(o) = floatx4_t{run.acc[0][r], run.acc[1][r], run.acc[2][r], run.acc[3][r]};
      *reinterpret_cast<floatx4_t*>(o + 4) = floatx4_t{run.acc[4][r], run.acc[5][r], run.acc[6][r], run.acc[7][r]};
    }
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

constexpr long long kMaxSegmentsPerLaunch = 1 << 23;   // (a launch's threads must stay below 2^32)

template <int G>
hipError_t launch_group(DecodeArgs a, Q8Pool pool, hipStream_t stream) {
  const int64_t segments = (int64_t)a.num_rows * a.num_kv_heads;
  const int64_t blocks = std::max<int64_t>(1, std::min<int64_t>(((int64_t)a.max_ctx + 15) / 16, a.max_blocks_per_seq));
  const int64_t slots = (int64_t)a.num_rows * a.num_q_heads + (int64_t)kDecodeGroupSlots * std::min(a.num_q_heads, 8);
  const int64_t cus = stream_compute_units(stream);
  int64_t want = std::min<int64_t>((4 * cus + segments - 1) / segments, slots / (segments * G));
  want = std::max<int64_t>(1, std::min<int64_t>(want, (blocks + 7) / 8));
  const int64_t per = ((blocks + want - 1) / want + 7) / 8 * 8;
  a.split_blocks = (int32_t)per;
  a.n_split_max = (int32_t)((blocks + per - 1) / per);
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
    case 1: return dq::launch_group<1>(a, pool, stream);
    case 2: return dq::launch_group<2>(a, pool, stream);
    case 4: return dq::launch_group<4>(a, pool, stream);
    case 8: return dq::launch_group<8>(a, pool, stream);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace bros
