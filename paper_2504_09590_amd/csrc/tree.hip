// bros_attn_tree and bros_tree_commit on gfx950.
//
// The attention is rows_device.h's over a K/V pool. With M columns (rows times heads of a KV
// head) a key of 512 bytes takes 512 M operations: few columns are bound by memory, from about
// 150 on by the matrix cores. A unit holds 32 columns (two waves along the keys), 64 (two by two) or 128 (four waves, each with
// columns of its own), as plan.h expects them to end first; units of 128 that share their keys run side by side.
//
// Measured, kernel and merge: 16 trees of 17 to 32 drafts on up to 8192 tokens, 32 / 8 heads, 67 + 11 us, 271 MB at 4.0 TB/s
// (loads alone take 50: starts of shares and masked steps are the rest); six of 64 drafts on 8000 to 32000, 64 / 8 heads,
// 266 + 13 us (306 + 15 in the middle of the first twelve calls), 820 TFLOP/s, 0.44 GB read, matrix cores busy 38 % of the cycles, waves waiting 25, no bank conflicts: what
// the matrix cores wait for is not shown; one chain of four on 300 tokens, 8 / 2 heads, 12.8 us, a chain of latencies: offsets,
// table, rows, three steps a wave, the masked one, the groups' sums.
#include "plan.h"
#include "rows_launch.h"

namespace bros {

namespace {

constexpr int kCommitThreads = 256;
constexpr int kCommitRows = kCommitThreads / 16;   // rows a workgroup moves at once, 16 lanes each
constexpr int kCommitRounds = 16;                  // so many times at most

// Sequence blockIdx.x, 256 bytes (16 chunks) blockIdx.y of its slots' rows in pool blockIdx.z (K's, V's). Every row is in
// registers before the first is written, so a path may go any way. Bound by its chain of loads (offsets, path,
// table entries, rows): 64 sequences of a bf16 pool with 8 heads 4.6 us, 256 of a latent pool 6.4 us, for 2.3 and 2.8 MB.
__global__ __launch_bounds__(kCommitThreads) void commit_kernel(CommitArgs a) {
  const int s = blockIdx.x;
  const int64_t drafts = (int64_t)a.cu_q[s + 1] - a.cu_q[s];
  const int ctx = a.ctx_lens[s];
  if (drafts <= 0 || drafts > ctx) return;   // (inconsistent offsets and lengths may be any numbers)
  const int n = (int)drafts, c0 = ctx - n;
  const int len = min(a.path_lens[s], min(n, a.max_path));
  // 256-byte pieces of a (slot, head) row
  const int pieces = (a.row_bytes + 255) / 256;
  const int piece = blockIdx.y % pieces, head = blockIdx.y / pieces;
  uint8_t* pool = static_cast<uint8_t*>(blockIdx.z == 0 ? a.k_pool : a.v_pool);
  const int at = 256 * piece + 16 * (threadIdx.x & 15);
  const int r0 = threadIdx.x >> 4;
  if (len <= 0) return;

  const auto place = [&](int pos) -> uint8_t* {
    const int e = pos >> 4;
    if (e >= a.max_blocks_per_seq) return nullptr;
    const int b = a.block_tables[(size_t)s * a.max_blocks_per_seq + e];
    if (b < 0 || b >= a.num_blocks) return nullptr;
    const int slot = slot_of_offset(pos & 15, entry_direction(a.dir, a.cls, a.dir_per_entry, a.max_blocks_per_seq, s, e));
    return pool + (((size_t)b * a.num_heads + head) * kBlockSize + slot) * a.row_bytes + at;
  };
  // (constant indices: the rows stay in registers)
  uint4 v[kCommitRounds];
  uint8_t* to[kCommitRounds];
#pragma unroll
  for (int i = 0; i < kCommitRounds; ++i) {
    const int r = kCommitRows * i + r0;
    v[i] = make_uint4(0, 0, 0, 0);
    to[i] = nullptr;
    if (kCommitRows * i < len && r < len && at < a.row_bytes) {
      const int from = a.path[(size_t)s * a.max_path + r];
      if (from >= 0 && from < n && from != r) {
        const uint8_t* src = place(c0 + from);
        uint8_t* dst = place(c0 + r);
        if (src != nullptr && dst != nullptr) {
          v[i] = *reinterpret_cast<const uint4*>(src);
          to[i] = dst;
        }
      }
    }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kCommitRounds; ++i)
    if (to[i] != nullptr) *reinterpret_cast<uint4*>(to[i]) = v[i];
}

}  // namespace

size_t rows_workspace_bytes(bool latent) {
  return latent ? ra::kLatentWorkspace : ra::kRowsWorkspace;
}

hipError_t launch_tree(RowsArgs a, void* workspace, hipStream_t stream) {
  const int64_t rows = planned_rows(a.max_q_len, a.num_q_tokens, a.num_seqs), columns = rows * (a.num_q_heads / a.num_kv_heads);
  const int64_t keys = 16 * (int64_t)longest_blocks(a.max_ctx, a.max_blocks_per_seq);
  const int64_t segments = (int64_t)a.num_seqs * a.num_kv_heads;
  switch (pick_rows_way(kTreeWays, columns, segments, keys, stream_compute_units(stream))) {
    case 0:
      // Short contexts and no more units than compute units: a unit has one to itself, with a third step's rows in LDS.
      // Us, so and two to a compute unit: one sequence of four rows on 300, 8 / 2 heads 12.6 and 13.8; 32 / 8 heads:
      // four of 4 on 500 16.8 and 18.5, 32 of 6 19.6 and 27; but 64 of 4 on 300, 512 units, 26 and 20.4.
      if (keys <= 8 * 64 && segments * ((columns + 31) / 32) <= stream_compute_units(stream))
        return ra::launch_rows<ra::KvPool, 1, 2, 3, 1>(a, 4, 8, 4, workspace, stream);
      return ra::launch_rows<ra::KvPool, 1, 2, 2, 2>(a, 4, 8, 4, workspace, stream);
    case 1: return ra::launch_rows<ra::KvPool, 2, 2, 2, 2>(a, 4, 8, 4, workspace, stream);
    default:
      switch (rows_team((columns + 127) / 128, a.num_q_tokens, rows, a.num_seqs)) {
        case 4: return ra::launch_rows<ra::KvPool, 4, 1, 4, 2, 4>(a, 4, 12, 8, workspace, stream);
        case 2: return ra::launch_rows<ra::KvPool, 4, 1, 4, 2, 2>(a, 4, 12, 8, workspace, stream);
        default: return ra::launch_rows<ra::KvPool, 4, 1, 4, 2>(a, 4, 12, 8, workspace, stream);
      }
  }
}

hipError_t launch_tree_commit(const CommitArgs& a, hipStream_t stream) {
  // (16384 heads of two pieces at most: within a grid's 65535)
  const unsigned pieces = (unsigned)((a.row_bytes + 255) / 256) * a.num_heads;
  hipLaunchKernelGGL(commit_kernel, dim3(a.num_seqs, pieces, a.v_pool != nullptr ? 2 : 1), dim3(kCommitThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace bros
