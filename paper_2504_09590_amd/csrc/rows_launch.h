// Launching the kernels of rows_device.h: shares for a stream's compute units, the partials'
// workspace, the merge.
#pragma once

#include "latent_device.h"

#include <algorithm>

namespace bros {
namespace ra {

constexpr int kMaxCus = 256;   // compute units whose shares' partials the workspace holds

// Bytes of the partials of `workers` shares of units of CT columns and `dims` dims.
constexpr size_t partial_bytes(size_t workers, size_t ct, size_t dims) { return 2 * workers * ct * (dims + 2) * sizeof(float); }

// PER_CU: workgroups a compute unit holds. MIN: the least steps of a share.
template <class P, int NCW, int NKW, int H, int SLOTS, int PER_CU, int MIN>
hipError_t launch_rows(RowsArgs a, void* workspace, hipStream_t stream) {
  using S = Shape<P, NCW, NKW, H, SLOTS>;
  constexpr int kEachEu = std::max(1, S::kWaves * PER_CU / 4);
  a.workers = std::min(stream_compute_units(stream), kMaxCus) * PER_CU;
  a.min_steps = MIN;
  a.ws_o = static_cast<float*>(workspace);
  a.ws_ml = a.ws_o + 2 * (size_t)a.workers * S::kSlotFloats;
  hipLaunchKernelGGL((rows_kernel<P, NCW, NKW, H, SLOTS, kEachEu>), dim3(a.workers), dim3(S::kThreads), 0, stream, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((rows_merge_kernel<P, NCW, NKW, H, SLOTS>), dim3(std::max(1, a.workers - 1), NCW), dim3(256), 0, stream, a);
  return hipGetLastError();
}

template <int NCW, int H, int MIN>
hipError_t launch_latent_rows(RowsArgs a, void* workspace, hipStream_t stream) {
  using S = LatentShape<NCW, H>;
  a.workers = std::min(stream_compute_units(stream), kMaxCus);
  a.min_steps = MIN;
  a.ws_o = static_cast<float*>(workspace);
  a.ws_ml = a.ws_o + 2 * (size_t)a.workers * S::kSlotFloats;
  hipLaunchKernelGGL((latent_kernel<NCW, H, S::kWaves / 4>), dim3(a.workers), dim3(S::kThreads), 0, stream, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((rows_merge_kernel<LatentPool, NCW, 1, H, 3>), dim3(std::max(1, a.workers - 1), NCW), dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace ra
}  // namespace bros
