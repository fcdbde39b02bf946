// How the attention of a few new rows of each sequence (rows_device.h, latent_device.h) lays its work out: units,
// their steps, the shares that workgroups take, and the walk of a workgroup through its share. Plain integers without HIP, so
// that it can be compiled and tested on the host too.
#pragma once

#include <stddef.h>
#include <stdint.h>

#if defined(__HIP__)
#define BROS_UNITS __device__ __forceinline__
#else
#include <algorithm>
#define BROS_UNITS inline
#endif

namespace bros {

// Attention of a few new rows of each sequence (rows_device.h): drafts over a K/V pool, latent
// queries over a pool of latent rows, causal chunks over expanded keys and values.
struct RowsArgs {
  void* out;
  const void* q;
  const int32_t* cu_q;        // null: one row per sequence
  const uint64_t* mask;       // [num_q_tokens][mask_words], or null: causal
  int32_t mask_words;
  const void* k_pool;         // latent: the only pool; expanded: keys [heads][dense_rows][128]
  const void* v_pool;
  const void* rot_rows;       // expanded: [dense_rows][64]
  const int32_t* scaled;      // expanded: [heads][dense_rows / 32], of a tile: its values stand behind exponents
  const int8_t* exps;         // expanded: [heads][dense_rows], the exponents of such tiles' rows
  int64_t dense_rows;
  const int32_t* block_tables;
  const int8_t* dir;
  const uint8_t* cls;
  const int32_t* ctx_lens;
  int32_t dir_per_entry;      // dir is [S][max_blocks_per_seq] (else [S])
  int32_t num_q_tokens;
  int32_t max_q_len;          // host bound of a sequence's rows
  int32_t num_seqs;
  int32_t num_blocks;
  int32_t max_blocks_per_seq;
  int32_t max_ctx;
  int32_t num_q_heads;
  int32_t num_kv_heads;       // expanded: heads of this pass
  int32_t head0;              // expanded: the first of them (else 0)
  float scale_log2;
  int32_t workers;            // shares the work is cut into, at most: those of workgroups or of teams (set by the launch)
  int32_t min_steps;          // the least steps of a share (set by the launch)
  int32_t whole_units;        // shares are of whole units (set by the launch)
  int32_t start_steps;        // what a unit's start counts among its steps (set by the launch)
  // (workgroups: workers times those of a team)
  void* ws_cut;               // [workgroups] notes of cut units
  float* ws_o;                // [2 workgroups] x (columns of a unit x value dims) partial sums
  float* ws_ml;               // [2 workgroups][columns of a unit][2] maximum (log2 units) and total
};

namespace ra {

#if !defined(__HIP__)
using std::max;
using std::min;
#endif

constexpr int kKeys = 32;                // keys of a wave's tile
constexpr int kBlockKeys = 16;           // keys of a block

// A number that is the same for every lane of a wave, as a scalar.
BROS_UNITS int uniform(int x) {
#if defined(__HIP__)
  return __builtin_amdgcn_readfirstlane(x);
#else
  return x;
#endif
}

// What is read. kMain: bytes of a key row's first part, kRot: of its second (0: none);
// kVal: bytes of a value row, or 0 where the first part is the value.
struct KvPool {          // 128 dims each, [blocks][Hkv][16][128]
  static constexpr int kMain = 256, kRot = 0, kVal = 256;
  static constexpr bool kPaged = true, kCausalUnits = false, kHalf = false;
};
struct LatentPool {      // 512 shared dims and 64 rotated ones, [blocks][16][576]
  static constexpr int kMain = 1024, kRot = 128, kVal = 0;
  static constexpr bool kPaged = true, kCausalUnits = false;
};
struct Expanded {        // dense rows: keys of 128 dims and 64 rotated ones shared by the heads, values of 128 in fp16
  static constexpr int kMain = 256, kRot = 128, kVal = 256;
  static constexpr bool kPaged = false, kCausalUnits = true, kHalf = true;
};

// A sequence as the kernels see it. n = 0: nothing to do. ctx: its visible context
// (0 where lengths are inconsistent: its rows see nothing); c0: position of its first new row.
struct Seq {
  int q0, n, c0, ctx;
};
BROS_UNITS Seq seq_of(const RowsArgs& a, int s) {
  Seq r;
  r.q0 = a.cu_q != nullptr ? a.cu_q[s] : s;
  const int end = a.cu_q != nullptr ? a.cu_q[s + 1] : s + 1;
  r.n = (r.q0 < 0 || end > a.num_q_tokens || end < r.q0) ? 0 : end - r.q0;
  const int ctx = max(a.ctx_lens[s], -1);   // (what is below zero is inconsistent, however far)
  r.c0 = ctx - r.n;
  const int64_t room = (int64_t)a.max_blocks_per_seq * kBlockKeys;
  r.ctx = r.c0 < 0 ? 0 : (int)min((int64_t)min(ctx, a.max_ctx), room);
  return r;
}

// Steps of a sequence's units. CT columns to a unit, KS keys to a step. Every unit has one
// at least: its rows are written even where they see nothing. A sequence without rows has no units.
template <class P, int CT, int KS>
struct Steps {
  int tiles, each;   // units per KV head; steps of one (causal units: of the last)
  int before;        // causal units: steps of the keys before the new rows
  bool whole;        // shares are of whole units
  int start;         // what a unit's start counts: its steps are those from `start` on in what is shared out
  BROS_UNITS Steps(const RowsArgs& a, const Seq& q, int group) {
    tiles = (int)(((int64_t)q.n * group + CT - 1) / CT);
    each = max(1, steps_of(q.ctx));
    before = steps_of(max(q.c0, 0));
    whole = a.whole_units != 0;
    start = a.start_steps;
  }
  // (in 32 bits without sign: lengths go up to 2^31 - 1)
  static BROS_UNITS int steps_of(int keys) { return (int)(((uint32_t)keys + KS - 1) / KS); }
  // Steps of unit t. Causal units (one column a row): those of its last row's keys.
  BROS_UNITS int of(int t) const {
    if constexpr (P::kCausalUnits) return t + 1 < tiles ? min(before + (CT / KS) * (t + 1), each) : each;
    return each;
  }
  // What units 0 .. t - 1 (t <= tiles) count, in what is shared out.
  BROS_UNITS int64_t first(int t) const {
    if (whole) return t;
    if constexpr (P::kCausalUnits) {
      // (the context may be cut short by max_ctx: units beyond it have `each` steps)
      const int free = max(0, min(t, min(tiles - 1, (each - before) / (CT / KS))));   // units whose `of` is not cut
      return (int64_t)free * before + (int64_t)(CT / KS) * free * (free + 1) / 2 + (int64_t)(t - free) * each + (int64_t)t * start;
    }
    return (int64_t)t * (each + start);
  }
  BROS_UNITS int64_t per_head() const { return first(tiles); }   // (0 without rows)
};

// Rows that a sequence's keys take in the dense buffers: whole tiles.
BROS_UNITS int64_t dense_rows(int ctx) { return ((int64_t)ctx + kKeys - 1) / kKeys * kKeys; }

// Where a workgroup's share begins.
struct Place {
  int s, g, t, step;
  int64_t total;        // steps of all units
  int64_t row0;         // dense keys: row of sequence s's position 0
};

// How `total` steps are shared out: n shares, the first `more` of them one step longer than `per`.
struct Shares {
  int n;
  int64_t per, more;
  BROS_UNITS Shares(const RowsArgs& a, int64_t total) {
    // (32-bit division is a tenth of the other, and nearly every call's steps fit)
    if (total < (1 << 30)) {
      const uint32_t x = (uint32_t)total;
      n = max(1u, min((uint32_t)a.workers, (x + a.min_steps - 1) / a.min_steps));
      per = x / (uint32_t)n;
    } else {
      n = a.workers;
      per = total / n;
    }
    more = total - per * n;
  }
  BROS_UNITS int64_t begin(int w) const { return per * w + min((int64_t)w, more); }
  // The share that step x lies in.
  BROS_UNITS int of(int64_t x) const {
    const int64_t longer = more * (per + 1);
    if (x < longer) return (int)(x / (per + 1));
    return (int)(more + (x - longer) / per);
  }
};

// The run of sequences that thread `tid` of `threads` counts.
struct Run {
  int s0, s1;
  BROS_UNITS Run(int num_seqs, int threads, int tid) {
    const int per = (num_seqs + threads - 1) / threads;
    s0 = min(tid * per, num_seqs);
    s1 = min(s0 + per, num_seqs);
  }
};
// What a run's units count in what is shared out, and its dense rows.
template <class P, int CT, int KS>
BROS_UNITS void count_run(const RowsArgs& a, int group, Run run, int64_t& steps, int64_t& rows) {
  steps = rows = 0;
  for (int s = run.s0; s < run.s1; ++s) {
    const Seq q = seq_of(a, s);
    const Steps<P, CT, KS> st(a, q, group);
    steps += st.per_head() * a.num_kv_heads;
    if constexpr (!P::kPaged) rows += dense_rows(q.ctx);
  }
}
// The unit and step of number `left` (of `total`) of a run, before which lie `rows` dense rows.
template <class P, int CT, int KS>
BROS_UNITS void place_in_run(const RowsArgs& a, int group, Run run, int64_t left, int64_t rows, int64_t total, Place* out) {
  Place p{-1, 0, 0, 0, total, rows};
  for (int s = run.s0; s < run.s1; ++s) {
    const Seq q = seq_of(a, s);
    const Steps<P, CT, KS> st(a, q, group);
    const int64_t ph = st.per_head();
    if (left < ph * a.num_kv_heads) {
      p.s = s;
      p.g = (int)(left / ph);
      left -= p.g * ph;
      int lo = 0, hi = st.tiles - 1;   // the last unit that begins at or before it
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (st.first(mid) <= left) lo = mid; else hi = mid - 1;
      }
      p.t = lo;
      p.step = (int)(left - st.first(lo));
      *out = p;
      return;
    }
    left -= ph * a.num_kv_heads;
    if constexpr (!P::kPaged) p.row0 += dense_rows(q.ctx);
  }
}

// What a workgroup (member of a team of TEAM) does of the unit at `at`, its share being [x, x_end): steps [first, last) of
// the `steps` that its own unit t has; `tiles` units of the team's width there are. (count <= 0: nothing. A share may end within
// a unit's start; a team's last units may not be there, and causal ones end one before the other.)
template <class P, int CT, int KS, int TEAM>
struct Segment {
  Seq q;
  int t, tiles, steps, first, last, count;
  bool whole;
  int64_t next;   // x behind it
  BROS_UNITS Segment(const RowsArgs& a, const Place& at, int group, int member, int64_t x, int64_t x_end) {
    q = seq_of(a, at.s);
    t = at.t * TEAM + member;
    const Steps<P, CT * TEAM, KS> st(a, q, group);
    const int tsteps = uniform(st.of(at.t));
    tiles = st.tiles;
    steps = tsteps;
    if constexpr (TEAM > 1) {
      const Steps<P, CT, KS> own(a, q, group);
      steps = t < own.tiles ? uniform(own.of(t)) : 0;
    }
    const int taken = st.whole ? 0 : (int)min((int64_t)(st.start + tsteps - at.step), x_end - x);
    first = st.whole ? 0 : max(0, at.step - st.start);
    last = st.whole ? steps : min(at.step + taken - st.start, steps);
    count = last - first;
    next = x + (st.whole ? 1 : taken);
    whole = count == steps;
  }
  // The share of the unit's last step. (Of a cut unit, at its first segment.)
  BROS_UNITS int last_share(const Shares& shares) const { return shares.of(next - last + steps - 1); }
};

// The unit behind one of `tiles` of its sequence and head. (Steps are left, so a sequence with rows follows.)
template <class P>
BROS_UNITS void next_unit(const RowsArgs& a, Place& at, int tiles) {
  if (++at.t < tiles) return;
  at.t = 0;
  if (++at.g < a.num_kv_heads) return;
  at.g = 0;
  do {
    if constexpr (!P::kPaged) at.row0 += dense_rows(seq_of(a, at.s).ctx);
    ++at.s;
  } while (seq_of(a, at.s).n <= 0);
}

}  // namespace ra
}  // namespace bros
