// bros_attn_prefill_chunk_q8: the matrix-core prefill (prefill_device.h) over an
// 8-bit pool. Units, pieces and their merge are the 16-bit prefill's.
//
// The matrix cores bound it from a few dozen rows on: 512 rows on 16000 cached tokens,
// 32 / 8 heads, 144 us, 946 TFLOP/s of the formula's products (the 16-bit prefill 143 us; a
// large library product 1208 TFLOP/s). A prompt of 301 rows takes 14.2 us, most of it the
// steps of one unit after another and their start.
#include "prefill_device.h"

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

hipError_t launch_prefill_q8(PrefillArgs a, const uint8_t* scales, int group, int num_tiles_total, hipStream_t stream) {
  if (num_tiles_total <= 0) return hipSuccess;
  switch (group) {
    case 1: return pf::launch_q8_group<1>(a, scales, num_tiles_total, stream);
    case 2: return pf::launch_q8_group<2>(a, scales, num_tiles_total, stream);
    case 4: return pf::launch_q8_group<4>(a, scales, num_tiles_total, stream);
    case 8: return pf::launch_q8_group<8>(a, scales, num_tiles_total, stream);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace bros
