// bros_qkv_append / bros_qkv_append_q8 on gfx950: a step's projected rows on their
// way to the attention, in one pass. For head row x (128 values) of a new token,
//   n = x * rsqrt(mean(x^2) + eps) * w             (q and k, where weights are given)
//   (a, b) -> (a cos - b sin, b cos + a sin)       for the pairs of the first R dims,
// cos and sin from the row of the caller's table that the pair's position names.
// q rows go to q_out, k and v rows to the slot of their token (kv_write.hip says which),
// as they are or as 8-bit codes and a scale (q8_device.h).
//
// Every byte is read once and written once, so memory bounds it, and for a decode
// step's few rows the chain of dependent loads: offsets, then table entry. Eight
// lanes take a head row, 16 dims each, so that a lane holds both halves of its
// eight pairs and only the sum of squares and the row's largest value cross lanes
// (three exchanges in a row of 16 lanes). A workgroup takes 32 consecutive head
// rows, one per eight lanes, whatever tokens they belong to. Loads that depend on
// nothing (the rows themselves, the sequences' offsets, given positions) are
// requested first; the cosines are requested as soon as the position is known,
// beside the table entry.
//
// Device time, and bytes that must move by it: four prompts of 2000 rows (64 / 8 heads,
// bf16, three position axes) 63.0 us, 4.9 TB/s, what a large copy reaches here; 2176 rows
// (32 / 8 heads) 12.4 us, 4.4 TB/s; four rows 3.2 us. (The eight pairs of a lane's cosines
// loaded one by one, each from its own axis, where most lanes' pairs have one: 106 us for the
// four prompts.)
#include "bros_kernels.h"
#include "q8_device.h"

namespace bros {
namespace {

constexpr int kThreads = 256;
constexpr int kLanes = 8;                    // lanes of a head row
constexpr int kRows = kThreads / kLanes;     // head rows of a workgroup
constexpr int kDims = kHeadDim / kLanes;     // dims of a lane
constexpr int kPairs = kDims / 2;

using q8::v2u_t;
using q8::v4u_t;

// Sum / maximum over the eight lanes of a head row.
__device__ __forceinline__ float row_sum(float x) {
  x += __shfl_xor(x, 1);
  x += __shfl_xor(x, 2);
  x += __shfl_xor(x, 4);
  return x;
}
__device__ __forceinline__ float row_max(float x) {
  x = fmaxf(x, __shfl_xor(x, 1));
  x = fmaxf(x, __shfl_xor(x, 2));
  x = fmaxf(x, __shfl_xor(x, 4));
  return x;
}

// The eight values of a chunk (chunk c: dims 8 c .. 8 c + 7) as fp32.
template <bool BF16>
__device__ __forceinline__ void widen(const v4u_t (&raw)[BF16 ? 1 : 2], float (&x)[kPairs]) {
  if constexpr (BF16) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = bf16_lo(raw[0][i]);
      x[2 * i + 1] = bf16_hi(raw[0][i]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(raw[i >> 2][i & 3]);
  }
}
template <bool BF16>
__device__ __forceinline__ void narrow(const float (&x)[kPairs], v4u_t (&raw)[BF16 ? 1 : 2]) {
  if constexpr (BF16) {
    // (the one rounding of a row's values; the arithmetic before it is fp32)
#pragma unroll
    for (int i = 0; i < 4; ++i) raw[0][i] = q8::pack2_bf16(x[2 * i], x[2 * i + 1]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) raw[i >> 2][i & 3] = __float_as_uint(x[i]);
  }
}
template <bool BF16>
__device__ __forceinline__ void load_chunk(const void* row, int chunk, v4u_t (&raw)[BF16 ? 1 : 2]) {
  const v4u_t* p = static_cast<const v4u_t*>(row) + chunk * (BF16 ? 1 : 2);
#pragma unroll
  for (int i = 0; i < (BF16 ? 1 : 2); ++i) raw[i] = p[i];
}
template <bool BF16>
__device__ __forceinline__ void store_chunk(void* row, int chunk, const v4u_t (&raw)[BF16 ? 1 : 2]) {
  v4u_t* p = static_cast<v4u_t*>(row) + chunk * (BF16 ? 1 : 2);
#pragma unroll
  for (int i = 0; i < (BF16 ? 1 : 2); ++i) p[i] = raw[i];
}

// The axis of a pair.
__device__ __forceinline__ int axis_of(const AppendArgs& a, int pair) {
  return (pair >= a.axis_end[0]) + (pair >= a.axis_end[1]) + (pair >= a.axis_end[2]);
}

// BF16: type of the rows (and of the pool unless Q8). ADJ: pairs (2 i, 2 i + 1)
// instead of (i, i + R / 2).
template <bool BF16, bool Q8, bool ADJ>
__global__ __launch_bounds__(kThreads) void append_kernel(AppendArgs a) {
  __shared__ int s_seq[kRows];   // sequence of each of the workgroup's tokens, or -1
  __shared__ int s_pos[kRows];   // its logical position
  __shared__ int s_dst[kRows];   // block * 16 + slot, or -1 when it is not stored
  constexpr int kElem = BF16 ? 2 : 4;
  constexpr int N = BF16 ? 1 : 2;   // 16-byte pieces of a chunk

  const int tid = threadIdx.x;
  const int heads = a.num_q_heads + 2 * a.num_kv_heads;   // head rows of a token: q, k, v
  const int item0 = blockIdx.x * kRows;
  const int t0 = item0 / heads;                           // (uniform)
  const int head0 = item0 - t0 * heads;
  const int n_tok = min((head0 + kRows - 1) / heads + 1, a.num_new_tokens - t0);   // <= kRows

  // This lane's part of the workgroup's head row tid / 8: token t0 + tok, head h of q, k or v.
  const int lane8 = tid % kLanes;
  int tok = 0, h = head0 + tid / kLanes;
  while (h >= heads) {   // (at most kRows / 2 rounds: without q rows a token may have one k and one v row)
    h -= heads;
    ++tok;
  }
  const bool live = tok < n_tok;
  const bool is_q = h < a.num_q_heads;
  const bool is_k = !is_q && h < a.num_q_heads + a.num_kv_heads;
  const int hk = is_q ? h : is_k ? h - a.num_q_heads : h - a.num_q_heads - a.num_kv_heads;
  // Chunks of 8 dims: the pairs' two halves, or two neighbours for adjacent pairs
  // and behind the rotated dims.
  const int turning = ADJ ? kLanes : a.rotary_dim / (2 * kPairs);   // lanes that hold split pairs
  const int ca = lane8 < turning ? (ADJ ? 2 * lane8 : lane8) : 2 * turning + 2 * (lane8 - turning);
  const int cb = lane8 < turning ? (ADJ ? 2 * lane8 + 1 : lane8 + turning) : ca + 1;

  // Loads that depend on nothing else.
  int m_lo = 0, m_hi = 0, m_p0 = 0;
  if (tid < a.num_seqs) {
    m_lo = a.cu_new[tid];
    m_hi = a.cu_new[tid + 1];
    m_p0 = a.pos0[tid];
  }
  v4u_t ra[N], rb[N];
  if (live) {
    const size_t t = (size_t)(t0 + tok);
    const char* base = static_cast<const char*>(is_q ? a.q : is_k ? a.k : a.v);
    const size_t stride = (size_t)(is_q ? a.q_stride : is_k ? a.k_stride : a.v_stride);
    const char* row = base + (t * stride + (size_t)hk * kHeadDim) * kElem;
    load_chunk<BF16>(row, ca, ra);
    load_chunk<BF16>(row, cb, rb);
  }
  const bool turned = (is_q || is_k) && lane8 * 2 * kPairs < a.rotary_dim;   // this lane's eight pairs are rotated
  // Given positions: that of the axis of the lane's first pair (most lanes' pairs have one axis).
  const int axis0 = axis_of(a, kPairs * lane8), axis7 = axis_of(a, kPairs * lane8 + kPairs - 1);
  int given = 0;
  if (live && turned && a.rope_pos != nullptr) given = a.rope_pos[(size_t)axis0 * a.num_new_tokens + t0 + tok];

  // The sequence and position of each token, as kv_write.hip finds them.
  if (tid < kRows) s_seq[tid] = -1;
  __syncthreads();
  for (int j = tid; j < a.num_seqs; j += kThreads) {
    const bool first = j == tid;
    const int lo = first ? m_lo : a.cu_new[j], hi = first ? m_hi : a.cu_new[j + 1];
    const int p0 = first ? m_p0 : a.pos0[j];
    const int k0 = max(lo, t0), k1 = min(hi, t0 + n_tok);
    for (int k = k0; k < k1; ++k) {
      s_seq[k - t0] = j;
      s_pos[k - t0] = p0 + (k - lo);
    }
  }
  __syncthreads();
  const int seq = live ? s_seq[tok] : -1;
  const int pos = seq >= 0 ? s_pos[tok] : -1;

  // Cosines and sines of this lane's pairs 8 lane8 .. 8 lane8 + 7. A position
  // outside the table: the token is not stored and its q rows are zeros.
  float c[kPairs], s[kPairs];
  if (seq >= 0 && turned && a.rope_table != nullptr) {
    const int row = a.rope_pos == nullptr ? pos : given;
    const bool outside = row < 0 || row >= a.table_rows;   // (dropped below)
    const float4* r4 = reinterpret_cast<const float4*>(a.rope_table + (size_t)(outside ? 0 : row) * a.rotary_dim) + 2 * lane8;
    const float4* s4 = r4 + a.rotary_dim / 8;
    const float4 c0 = r4[0], c1 = r4[1], s0 = s4[0], s1 = s4[1];
    c[0] = c0.x; c[1] = c0.y; c[2] = c0.z; c[3] = c0.w; c[4] = c1.x; c[5] = c1.y; c[6] = c1.z; c[7] = c1.w;
    s[0] = s0.x; s[1] = s0.y; s[2] = s0.z; s[3] = s0.w; s[4] = s1.x; s[5] = s1.y; s[6] = s1.z; s[7] = s1.w;
    if (a.rope_pos != nullptr && axis0 != axis7) {   // an axis ends among the lane's pairs: those behind it
#pragma unroll
      for (int i = 1; i < kPairs; ++i) {
        const int pair = kPairs * lane8 + i, x = axis_of(a, pair);
        if (x == axis0) continue;
        const int other = a.rope_pos[(size_t)x * a.num_new_tokens + t0 + tok];
        const bool bad = other < 0 || other >= a.table_rows;
        const float* r = a.rope_table + (size_t)(bad ? 0 : other) * a.rotary_dim + pair;
        c[i] = r[0];
        s[i] = r[a.rotary_dim / 2];
      }
    }
  }
  // A token's position is inside the table on every lane or the token is dropped:
  // with several axes a lane sees its own pairs' alone, so the tokens' flags meet in LDS.
  if (tid < n_tok) {
    int dst = -1;
    const int j = s_seq[tid], p = s_pos[tid];
    bool off = false;
    if (j >= 0 && a.rope_table != nullptr) {
      if (a.rope_pos == nullptr) {
        off = p < 0 || p >= a.table_rows;
      } else {
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const int r = a.rope_pos[(size_t)min(x, a.axes - 1) * a.num_new_tokens + t0 + tid];
          off |= r < 0 || r >= a.table_rows;
        }
      }
    }
    if (j >= 0 && !off && p >= 0 && (p >> 4) < a.max_blocks_per_seq) {
      const int blk = a.block_tables[(size_t)j * a.max_blocks_per_seq + (p >> 4)];
      const int dirv = entry_direction(a.dir, a.cls, a.dir_per_entry, a.max_blocks_per_seq, j, p >> 4);
      if (blk >= 0 && blk < a.num_blocks) dst = blk * kBlockSize + slot_of_offset(p & 15, dirv);
    }
    s_dst[tid] = off ? -2 : dst;
  }

  // The row's values.
  float xa[kPairs], xb[kPairs];
  if (live) {
    widen<BF16>(ra, xa);
    widen<BF16>(rb, xb);
  } else {
#pragma unroll
    for (int i = 0; i < kPairs; ++i) xa[i] = xb[i] = 0.0f;
  }
  if (a.q_norm != nullptr || a.k_norm != nullptr) {   // (uniform: every lane takes part in the exchange)
    float ss = 0.0f;
#pragma unroll
    for (int i = 0; i < kPairs; ++i) ss = fmaf(xa[i], xa[i], fmaf(xb[i], xb[i], ss));
    ss = row_sum(ss);
    const void* w = is_q ? a.q_norm : is_k ? a.k_norm : nullptr;
    if (w != nullptr) {
      const float r = rsqrtf(ss * (1.0f / kHeadDim) + a.eps);
      v4u_t wr[N];
      float wa[kPairs];
      load_chunk<BF16>(w, ca, wr);
      widen<BF16>(wr, wa);
#pragma unroll
      for (int i = 0; i < kPairs; ++i) xa[i] = xa[i] * r * wa[i];
      load_chunk<BF16>(w, cb, wr);
      widen<BF16>(wr, wa);
#pragma unroll
      for (int i = 0; i < kPairs; ++i) xb[i] = xb[i] * r * wa[i];
    }
  }
  if (turned && seq >= 0 && a.rope_table != nullptr) {   // (outside: the result is dropped)
#pragma unroll
    for (int i = 0; i < kPairs; ++i) {
      // pair i: (xa[i], xb[i]); adjacent: values 2 i and 2 i + 1 of the lane's sixteen
      float& u = ADJ ? (i < kPairs / 2 ? xa[2 * i] : xb[2 * i - kPairs]) : xa[i];
      float& v = ADJ ? (i < kPairs / 2 ? xa[2 * i + 1] : xb[2 * i + 1 - kPairs]) : xb[i];
      const float u0 = u, v0 = v;
      u = fmaf(u0, c[i], -(v0 * s[i]));
      v = fmaf(v0, c[i], u0 * s[i]);
    }
  }
  // 8 bits: the scale of a k or v row (the exchange on every lane).
  int e = 0;
  if constexpr (Q8) {
    float m = 0.0f;
#pragma unroll
    for (int i = 0; i < kPairs; ++i) m = fmaxf(m, fmaxf(q8::finite_magnitude(xa[i]), q8::finite_magnitude(xb[i])));
    e = q8::row_exponent(row_max(m));
  }
  __syncthreads();
  if (seq < 0) return;   // in no sequence: left as it was
  const int dst = s_dst[tok];

  if (is_q) {
    v4u_t za[N], zb[N];
    narrow<BF16>(xa, za);
    narrow<BF16>(xb, zb);
    if (dst == -2) {
#pragma unroll
      for (int i = 0; i < N; ++i) za[i] = zb[i] = v4u_t{0u, 0u, 0u, 0u};
    }
    char* row = static_cast<char*>(a.q_out) + ((size_t)(t0 + tok) * a.num_q_heads + hk) * kHeadDim * kElem;
    store_chunk<BF16>(row, ca, za);
    store_chunk<BF16>(row, cb, zb);
    return;
  }
  if (dst < 0) return;
  const size_t tile = (size_t)(dst >> 4) * a.num_kv_heads + hk;
  if constexpr (Q8) {
    uint8_t* row = static_cast<uint8_t*>(is_k ? a.k_pool : a.v_pool) + (tile * kBlockSize + (dst & 15)) * kHeadDim;
    const float mul = q8::exp2_int(-e);
    const v2u_t qa = {q8::codes4(xa[0], xa[1], xa[2], xa[3], mul), q8::codes4(xa[4], xa[5], xa[6], xa[7], mul)};
    const v2u_t qb = {q8::codes4(xb[0], xb[1], xb[2], xb[3], mul), q8::codes4(xb[4], xb[5], xb[6], xb[7], mul)};
    reinterpret_cast<v2u_t*>(row)[ca] = qa;
    reinterpret_cast<v2u_t*>(row)[cb] = qb;
    if (lane8 == 0) a.kv_scales[(2 * tile + (is_k ? 0 : 1)) * kBlockSize + (dst & 15)] = (uint8_t)(e + 127);
  } else {
    char* row = static_cast<char*>(is_k ? a.k_pool : a.v_pool) + (tile * kBlockSize + (dst & 15)) * kHeadDim * kElem;
    if (is_k) {   // (a v row's bytes go as they came)
      narrow<BF16>(xa, ra);
      narrow<BF16>(xb, rb);
    }
    store_chunk<BF16>(row, ca, ra);
    store_chunk<BF16>(row, cb, rb);
  }
}

template <bool BF16, bool Q8>
void launch_pairs(const AppendArgs& a, unsigned grid, hipStream_t stream) {
  if (a.adjacent) hipLaunchKernelGGL((append_kernel<BF16, Q8, true>), dim3(grid), dim3(kThreads), 0, stream, a);
  else hipLaunchKernelGGL((append_kernel<BF16, Q8, false>), dim3(grid), dim3(kThreads), 0, stream, a);
}

}  // namespace

hipError_t launch_append(const AppendArgs& a, bool bf16, hipStream_t stream) {
  const int64_t rows = (int64_t)a.num_new_tokens * (a.num_q_heads + 2 * a.num_kv_heads);
  const unsigned grid = (unsigned)((rows + kRows - 1) / kRows);
  if (grid == 0) return hipSuccess;
  const bool eight = a.kv_scales != nullptr;
  if (bf16 && eight) launch_pairs<true, true>(a, grid, stream);
  else if (bf16) launch_pairs<true, false>(a, grid, stream);
  else if (eight) launch_pairs<false, true>(a, grid, stream);
  else launch_pairs<false, false>(a, grid, stream);
  return hipGetLastError();
}

}  // namespace bros
