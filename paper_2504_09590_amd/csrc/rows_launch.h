// Launching the kernels of rows_device.h and latent_device.h: shares for a stream's compute units,
// the partials' workspace, the merge.
#pragma once

#include "latent_device.h"

#include <algorithm>

namespace bros {
namespace ra {

constexpr int kMaxCus = 256;   // compute units whose shares' partials the workspace holds

// Bytes of the notes and partials of `groups` workgroups whose units have CT columns and `dims` dims.
constexpr size_t partial_bytes(size_t groups, size_t ct, size_t dims) {
  return groups * sizeof(Cut) + 2 * groups * ct * (dims + 2) * sizeof(float);
}
// The workspaces: what the widest units take. (Every launch is checked against them where it is compiled.)
constexpr size_t kRowsWorkspace = partial_bytes(2 * kMaxCus, 128, 128), kLatentWorkspace = partial_bytes(kMaxCus, 128, 512);

// Launches `kernel` on per_cu workgroups a compute unit, and the merge. min_steps: the least steps of a share.
// whole: steps of the longest unit up to which units are not cut. start: steps that a unit's start counts as
// in a share (us with 0, 3 and 6: decode of 16 heads, 64 contexts up to 8192, 77, 69, 64; of 64 heads 101, 93, 85; of 128 heads, 96 up to
// 16384, 351, 341, 332; drafts of 32 heads 42, 38, 36; with 0, 4 and 8: 16 trees of 17 to 32 on up to 8192, 32 / 8 heads, 77, 69, 68).
template <class S, bool DENSE, int TEAM = 1, class Kernel>
hipError_t launch_shares(Kernel kernel, RowsArgs a, int per_cu, int min_steps, int whole, int start, void* workspace, hipStream_t stream) {
  a.workers = std::max(1, std::min(stream_compute_units(stream), kMaxCus) * per_cu / TEAM);
  const int groups = a.workers * TEAM;
  a.min_steps = min_steps;
  a.whole_units = ((int64_t)std::min<int64_t>(a.max_ctx, (int64_t)a.max_blocks_per_seq * kBlockSize) + S::KS - 1) / S::KS <= whole;
  a.start_steps = start;
  if (a.whole_units) a.min_steps = 1;
  a.ws_cut = workspace;
  a.ws_o = reinterpret_cast<float*>(static_cast<Cut*>(workspace) + groups);
  a.ws_ml = a.ws_o + 2 * (size_t)groups * S::kSlotFloats;
  hipLaunchKernelGGL(kernel, dim3(groups), dim3(S::kThreads), 0, stream, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.whole_units) return e;
  constexpr int kItems = S::CT / S::kLaneCols * S::kChunks / kMergeEach;
  hipLaunchKernelGGL((rows_merge_kernel<S, DENSE, TEAM>), dim3(std::max(1, groups - 1), kItems / kMergeWaves), dim3(kMergeWaves * kWave), 0,
                     stream, a);
  return hipGetLastError();
}

template <class P, int NCW, int NKW, int SLOTS, int PER_CU, int TEAM = 1>
hipError_t launch_rows(const RowsArgs& a, int min_steps, int whole, int start, void* workspace, hipStream_t stream) {
  using S = Shape<P, NCW, NKW, SLOTS>;
  static_assert(partial_bytes(kMaxCus * PER_CU, S::CT, S::kDims) <= kRowsWorkspace && PER_CU * kMaxCus % TEAM == 0, "");
  constexpr int kEachEu = std::max(1, S::kWaves * PER_CU / 4);
  return launch_shares<S, !P::kPaged, TEAM>(&rows_kernel<P, NCW, NKW, SLOTS, kEachEu, TEAM>, a, PER_CU, min_steps, whole, start, workspace, stream);
}

template <int NCW, int HV>
hipError_t launch_latent_rows(const RowsArgs& a, int min_steps, int whole, int start, void* workspace, hipStream_t stream) {
  using S = LatentShape<NCW, HV>;
  static_assert(partial_bytes(kMaxCus, S::CT, S::kDims) <= kLatentWorkspace, "");
  return launch_shares<S, false>(&latent_kernel<NCW, HV, S::kWaves / 4>, a, 1, min_steps, whole, start, workspace, stream);
}

}  // namespace ra
}  // namespace bros
