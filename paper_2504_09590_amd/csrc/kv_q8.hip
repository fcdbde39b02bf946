// Rows of the 8-bit cache by slot id, on gfx950.
//   gather:  codes and scales of slots into dense [n][Hkv][128] and [n][Hkv][2]
//   scatter: the reverse (lazy checkpointing, Sec. 5.2, as swap.hip)
//   read:    the values the slots stand for, bf16 or fp32, dense [n][Hkv][128]
// An id outside the pool: zeros from gather and read, skipped by scatter.
//
// Byte movement in 16-byte chunks (eight a row), bound by memory, and for a few
// slots by the launch and one chain of two loads (id, then chunk). A workgroup moves
// whole ids of K (blockIdx.y = 0) or V, as many as one pass of its threads holds,
// so that a chunk's place takes 32-bit arithmetic. The thread that moves a row's
// first chunk moves its scale byte.
//
// Device time at 8 KV heads: 4096 slots out or in 5.1 us (17 MB each way, 3.3 TB/s: two
// thirds of it start and end, 24 slots take 2.7 us); 12000 slots read as bf16 14.0 us.
#include "bros_kernels.h"
#include "q8_device.h"

#include <algorithm>

namespace bros {
namespace {

constexpr int kThreads = 256;
constexpr int kIter = 4;                     // 16-byte chunks per thread
constexpr int kRowChunks = kHeadDim / 16;    // chunks of a row

using q8::v4u_t;

enum Move { kGather, kScatter, kRead };

// OUT_BF16: type of the values read.
template <int MOVE, int ITERS, bool OUT_BF16>
__global__ __launch_bounds__(kThreads) void move_q8_kernel(KvMoveQ8Args a, int ids_per_group, float rcp) {
  const int tid = threadIdx.x;
  const int per_id = a.num_kv_heads * kRowChunks;
  const int i0 = blockIdx.x * ids_per_group;
  const int n = min(ids_per_group, a.num_slots - i0) * per_id;
  const int64_t pool_slots = (int64_t)a.num_blocks * kBlockSize;
  const int v = blockIdx.y;
  uint8_t* pool = static_cast<uint8_t*>(v ? a.v_pool : a.k_pool);
  uint8_t* dense = static_cast<uint8_t*>(v ? a.v_dense : a.k_dense);

  for (int base = 0; base < n; base += kThreads * ITERS) {
    v4u_t data[ITERS];
    uint8_t sc[ITERS];
    int64_t row[ITERS];   // pool row (block, head, slot), -1 when the id lies outside
    int64_t srow[ITERS];  // its scale's place
#pragma unroll
    for (int it = 0; it < ITERS; ++it) {
      const int c = min(base + it * kThreads + tid, n - 1);
      const int i = div_small(c, per_id, rcp);
      const int rem = c - i * per_id;
      const int h = rem / kRowChunks, cc = rem % kRowChunks;
      const int sid = a.slot_ids[i0 + i];
      const int64_t tile = (int64_t)(sid / kBlockSize) * a.num_kv_heads + h;
      const bool in = sid >= 0 && sid < pool_slots;
      row[it] = in ? (tile * kBlockSize + sid % kBlockSize) : -1;
      srow[it] = in ? ((2 * tile + v) * kBlockSize + sid % kBlockSize) : -1;
      sc[it] = 0;
      data[it] = v4u_t{0u, 0u, 0u, 0u};
      if (MOVE == kScatter) {
        data[it] = reinterpret_cast<const v4u_t*>(dense)[(size_t)i0 * per_id + c];
        if (cc == 0) sc[it] = a.scales_dense[2 * (((size_t)(i0 + i)) * a.num_kv_heads + h) + v];
      }
    }
    if (MOVE != kScatter) {
#pragma unroll
      for (int it = 0; it < ITERS; ++it) {
        const int c = min(base + it * kThreads + tid, n - 1);
        if (row[it] >= 0) {
          data[it] = reinterpret_cast<const v4u_t*>(pool)[row[it] * kRowChunks + c % kRowChunks];
          if (MOVE == kRead || c % kRowChunks == 0) sc[it] = a.kv_scales[srow[it]];
        }
      }
    }
#pragma unroll
    for (int it = 0; it < ITERS; ++it) {
      const int c = base + it * kThreads + tid;
      if (c >= n) continue;
      const size_t at = (size_t)i0 * per_id + c;   // chunk of the dense side
      if (MOVE == kGather) {
        reinterpret_cast<v4u_t*>(dense)[at] = data[it];
        if (c % kRowChunks == 0) a.scales_dense[2 * (at / kRowChunks) + v] = sc[it];
      } else if (MOVE == kScatter) {
        if (row[it] < 0) continue;
        reinterpret_cast<v4u_t*>(pool)[row[it] * kRowChunks + c % kRowChunks] = data[it];
        if (c % kRowChunks == 0) a.kv_scales[srow[it]] = sc[it];
      } else {
        const float s = q8::scale_of(sc[it]);
        if (OUT_BF16) {
          v4u_t* o = reinterpret_cast<v4u_t*>(dense) + 2 * at;
#pragma unroll
          for (int k = 0; k < 2; ++k)
            o[k] = v4u_t{q8::values2_bf16<false>(data[it][2 * k], s), q8::values2_bf16<true>(data[it][2 * k], s),
                         q8::values2_bf16<false>(data[it][2 * k + 1], s), q8::values2_bf16<true>(data[it][2 * k + 1], s)};
        } else {
          v4u_t* o = reinterpret_cast<v4u_t*>(dense) + 4 * at;
#pragma unroll
          for (int k = 0; k < 4; ++k) {   // (bf16 holds the values exactly: widened)
            const uint32_t lo = q8::values2_bf16<false>(data[it][k], s), hi = q8::values2_bf16<true>(data[it][k], s);
            o[k] = v4u_t{lo << 16, lo & 0xffff0000u, hi << 16, hi & 0xffff0000u};
          }
        }
      }
    }
  }
}

template <int MOVE, bool OUT_BF16>
hipError_t launch_move(const KvMoveQ8Args& a, hipStream_t stream) {
  const int per_id = a.num_kv_heads * kRowChunks;
  const int ids = std::max(1, kThreads * kIter / per_id);
  const int64_t groups = ((int64_t)a.num_slots + ids - 1) / ids;
  if (groups == 0) return hipSuccess;
  if (groups > 0x7fffffffLL / kThreads) return hipErrorInvalidValue;
  const dim3 grid((unsigned)groups, 2);
  const float rcp = 1.0f / (float)per_id;
  if ((int64_t)a.num_slots * per_id <= kThreads)
    hipLaunchKernelGGL((move_q8_kernel<MOVE, 1, OUT_BF16>), grid, dim3(kThreads), 0, stream, a, ids, rcp);
  else
    hipLaunchKernelGGL((move_q8_kernel<MOVE, kIter, OUT_BF16>), grid, dim3(kThreads), 0, stream, a, ids, rcp);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_kv_move_q8(const KvMoveQ8Args& a, bool gather, hipStream_t stream) {
  return gather ? launch_move<kGather, true>(a, stream) : launch_move<kScatter, true>(a, stream);
}
hipError_t launch_kv_read_q8(const KvMoveQ8Args& a, bool bf16, hipStream_t stream) {
  return bf16 ? launch_move<kRead, true>(a, stream) : launch_move<kRead, false>(a, stream);
}

}  // namespace bros
